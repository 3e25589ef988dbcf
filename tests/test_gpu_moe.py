"""Mixture of experts on a few tokens against the definition in 64 bits.

Tolerances.  X is a multiple of 1/4 up to 4 and the router one of 2^-8 up to 1/4, so that logits are multiples of 2^-10 below 2^11, exact in
fp32 in any order: which experts a row takes is exactly determined (ties go to the lowest).  A softmax or sigmoid score is relatively
off by at most 16 * 2^-24 (exp of 2 units at arguments below 2^4 whose rounding is worth 2^-20 relative; a sum; a division), so 2^-19
covers it, and 2^-18 one that is renormalised.
Products of a chunk of 64 are added inside the tensor core, with at most 2^-22 of the magnitudes a step of 16, chunks and CTAs' parts in
fp32: (16 + chunks + 148) 2^-23 of the sum of the magnitudes bounds both.  silu has a slope of at most 1.1, the hidden rows are held
to 2^-17 (bf16 results) or 2^-25, and what they are off by goes through the down product.  Half a step of Y's type on top."""
import math

import pytest
import torch

from paper_2609_32814_b200 import binding

pytestmark = pytest.mark.gpu


class Layer:
    def __init__(self, m, d, f, e, k, score="softmax", renormalise=True, bias=False, router="bf16", scale=1.0, seed=0, pad=0):
        gen = torch.Generator().manual_seed(10007 * m + 101 * d + 7 * e + seed)
        rnd = lambda *s: torch.randn(*s, generator=gen)  # noqa: E731
        self.m, self.d, self.f, self.e, self.k, self.score, self.renormalise, self.scale = m, d, f, e, k, score, renormalise, scale
        wide = torch.full((m, d + pad), 9.0).bfloat16().cuda()
        self.X = wide[:, :d]
        self.X.copy_((rnd(m, d) * 4).round().clamp(-16, 16) / 4)
        self.Wr = ((rnd(d, e) * 2 / math.sqrt(d) * 256).round().clamp(-64, 64) / 256).to(torch.bfloat16 if router == "bf16" else torch.float32).cuda()
        self.bias = (rnd(e) * 0.2).cuda() if bias else None
        while bias and self.margin() <= 2.0 ** -18:      # (no order that hangs on a rounding)
            self.bias = (rnd(e) * 0.2).cuda()
        self.Wgu = (rnd(e, d, 2 * f) / math.sqrt(d)).bfloat16().cuda()
        self.Wd = (rnd(e, f, d) / math.sqrt(f)).bfloat16().cuda()
        self.h = binding.MoE(d, f, e, k, score=score, renormalise=renormalise, route_scale=scale, router_dtype=router)

    def run(self, **kw):
        return self.h.forward(self.X, self.Wr, self.Wgu, self.Wd, select_bias=self.bias, routing=True, **kw)

    def scores(self):
        logits = self.X.double().cpu() @ self.Wr.double().cpu()
        p = torch.softmax(logits, 1) if self.score == "softmax" else torch.sigmoid(logits)
        return p, logits if self.bias is None else p + self.bias.double().cpu()

    def margin(self):
        top = torch.sort(self.scores()[1], dim=1, descending=True)[0]
        return float((top[:, :-1] - top[:, 1:])[:, :self.k].min())

    def choice(self):
        """(experts, weights, the weights' bound) in 64 bits."""
        p, by = self.scores()
        idx = torch.argsort(by, dim=1, descending=True, stable=True)[:, :self.k]
        assert self.bias is None or self.margin() > 2.0 ** -18
        wt, rel = p.gather(1, idx), 2.0 ** -19
        if self.renormalise:
            wt, rel = wt / wt.sum(1, keepdim=True), 2.0 ** -18
        return idx, wt * self.scale, (wt * self.scale).abs() * rel

    def expect(self, idx, wt, wt_off, planes):
        x = self.X.double().cpu()
        y, bound = torch.zeros(self.m, self.d, dtype=torch.float64), torch.zeros(self.m, self.d, dtype=torch.float64)
        u1, u2 = (16 + self.d / 64 + 148) * 2.0 ** -23, (16 + self.k * self.f / 64 + 148) * 2.0 ** -23
        for e in idx[idx >= 0].unique().tolist():
            rows, at = (idx == e).nonzero(as_tuple=True)
            gu, dn = self.Wgu[e].double().cpu(), self.Wd[e].double().cpu()
            pre, size = x[rows] @ gu, x[rows].abs() @ gu.abs()
            g, u = pre[:, :self.f], pre[:, self.f:]
            s = g * torch.sigmoid(g)
            w = wt[rows, at][:, None]
            h = s * u * w
            off = (1.1 * u1 * size[:, :self.f] * u.abs() + s.abs() * u1 * size[:, self.f:]) * w.abs() * 2
            off = off + h.abs() * (8 * 2.0 ** -24 + 2.0 ** (-17 if planes == 2 else -25)) + (s * u).abs() * wt_off[rows, at][:, None]
            y[rows] += h @ dn
            bound[rows] += off @ dn.abs() + u2 * (h.abs() @ dn.abs())
        return y, bound

    def check(self, y, experts, weights):
        idx, wt, off = self.choice()
        assert torch.equal(experts.cpu().long(), idx)
        assert bool(((weights.double().cpu() - wt).abs() <= off).all())
        want, bound = self.expect(idx, wt, off, 2 if y.dtype is torch.bfloat16 else 3)
        bound = bound + torch.finfo(y.dtype).eps / 2 * want.abs() + 1e-30
        err = (y.double().cpu() - want).abs()
        assert bool((err <= bound).all()), f"worst {float((err / bound).max()):.2f} of the bound"
        assert self.h.last_status() == 0


@pytest.mark.parametrize("m,d,f,e,k", [(1, 64, 64, 4, 2), (1, 8, 8, 1, 1), (1, 8, 8, 3, 2), (3, 72, 40, 5, 5), (8, 256, 192, 16, 4), (9, 520, 136, 33, 3),
                                       (2, 1024, 8, 2, 1), (33, 1024, 256, 100, 7), (64, 256, 128, 8, 2), (64, 512, 64, 512, 32), (17, 2048, 768, 24, 8),
                                       (1, 2048, 768, 128, 8), (5, 136, 1032, 40, 1), (16, 200, 72, 300, 2)])
@pytest.mark.parametrize("out", [torch.bfloat16, torch.float32])
def test_layer(m, d, f, e, k, out):
    layer = Layer(m, d, f, e, k)
    layer.check(*layer.run(out_dtype=out))


@pytest.mark.parametrize("score,renormalise,bias,router,scale", [("sigmoid", True, True, "bf16", 2.5), ("sigmoid", False, False, "f32", 1.0),
                                                                 ("softmax", False, True, "f32", 1.0), ("softmax", True, True, "bf16", 0.5),
                                                                 ("softmax", False, False, "bf16", 1.0)])
@pytest.mark.parametrize("m,e", [(1, 48), (12, 48), (40, 21)])
def test_scores(score, renormalise, bias, router, scale, m, e):
    layer = Layer(m, 384, 96, e, 6, score, renormalise, bias, router, scale)
    layer.check(*layer.run(out_dtype=torch.float32))


def test_strided_rows_and_what_lies_between_them():
    layer = Layer(11, 264, 64, 9, 3, pad=16)
    wide = torch.full((11, 280), 3.0, dtype=torch.bfloat16, device="cuda")
    y, experts, weights = layer.run(out=wide[:, :264])
    layer.check(y, experts, weights)
    assert bool((wide[:, 264:] == 3.0).all())


@pytest.mark.parametrize("m", [1, 7, 40, 64])
def test_every_row_takes_the_same_experts(m):
    layer = Layer(m, 256, 320, 32, 3, score="sigmoid", bias=True)
    layer.bias[[4, 9, 31]] += torch.tensor([30.0, 20.0, 10.0], device="cuda")
    y, experts, weights = layer.run(out_dtype=torch.float32)
    assert bool((experts.cpu() == torch.tensor([4, 9, 31])).all())
    layer.check(y, experts, weights)


def test_equal_scores_go_to_the_lowest_expert():
    layer = Layer(6, 64, 64, 70, 5)
    layer.X.copy_(torch.randint(-3, 4, (6, 64)))
    layer.Wr.copy_(torch.randint(-2, 3, (64, 1)).expand(64, 70))          # every logit of a row is the same, exactly
    layer.Wr[:, 40] += layer.X[2].sign() * 1.0                              # row 2 prefers expert 40
    y, experts, weights = layer.run()
    idx = torch.argsort(layer.X.double().cpu() @ layer.Wr.double().cpu(), dim=1, descending=True, stable=True)[:, :5]
    assert torch.equal(experts.cpu().long(), idx) and experts[2, 0] == 40
    layer.X.zero_()
    y, experts, weights = layer.run()
    assert torch.equal(experts.cpu(), torch.arange(5, dtype=torch.int32).expand(6, 5)) and bool((y == 0).all())
    assert bool(((weights - 0.2).abs() < 1e-6).all())


def test_masked_experts_and_rows_that_find_none():
    layer = Layer(5, 128, 64, 8, 3, score="sigmoid", renormalise=False, bias=True)
    layer.bias[:] = -math.inf
    layer.bias[[2, 6]] = 0.0
    layer.bias[3] = math.nan
    y, experts, weights = layer.run(out_dtype=torch.float32)
    x, w = layer.X.double().cpu(), layer.Wr.double().cpu()
    p = torch.sigmoid(x @ w)
    first = torch.where(p[:, 2] >= p[:, 6], 2, 6)
    idx = torch.stack([first, 8 - first, torch.full((5,), -1)], 1)
    assert torch.equal(experts.cpu().long(), idx) and bool((weights[:, 2] == 0).all())
    wt = torch.where(idx >= 0, p.gather(1, idx.clamp(min=0)), 0.0)
    want, bound = layer.expect(idx, wt, wt * 2.0 ** -16, 3)
    assert bool(((y.double().cpu() - want).abs() <= bound + 2.0 ** -24 * want.abs()).all())
    layer.bias[:] = -math.inf
    for renormalise in (False, True):
        h = binding.MoE(128, 64, 8, 3, score="sigmoid", renormalise=renormalise)
        y, experts, weights = h.forward(layer.X, layer.Wr, layer.Wgu, layer.Wd, select_bias=layer.bias, routing=True,
                                        out=torch.full((5, 128), 5.0, dtype=torch.bfloat16, device="cuda"))
        assert bool((experts == -1).all()) and bool((weights == 0).all()) and bool((y == 0).all())


def test_rows_and_weights_that_are_not_finite_stay_apart():
    layer = Layer(10, 192, 64, 12, 2, bias=True, score="sigmoid")
    want, experts, weights = layer.run()
    layer.X[3, 5], layer.X[8, 0] = math.nan, math.inf
    layer.Wr[0] = 1.0
    layer.X[:, 0].masked_fill_(torch.isfinite(layer.X[:, 0]), 0.0)
    clean = layer.X.clone()
    clean[3, 5], clean[8, 0] = 0.0, 0.0
    y, ex, wt = layer.run()
    layer.X.copy_(clean)
    y0, ex0, wt0 = layer.run()
    rest = [r for r in range(10) if r not in (3, 8)]
    assert torch.equal(y[rest], y0[rest]) and torch.equal(ex[rest], ex0[rest])
    for r in (3, 8):
        assert bool(y[r].isnan().all()) and bool((ex[r] == -1).all()) and bool(wt[r].isnan().all())
    # an expert's bad weight reaches the rows that take it and no others
    e = int(ex0[0, 0])
    layer.Wd[e, 7, 9] = math.inf
    y, ex, wt = layer.run()
    took = (ex0.cpu() == e).any(1)
    assert bool((~torch.isfinite(y[took.cuda(), 9])).all()) and torch.equal(y[~took.cuda()], y0[~took.cuda()])


def test_calls_of_all_sizes_through_one_handle_and_workspace():
    layer = Layer(64, 320, 200, 20, 4)
    x = layer.X.clone()
    ws = torch.full((layer.h.workspace_bytes(64),), 255, dtype=torch.uint8, device="cuda")
    for m in (64, 1, 63, 8, 9, 17, 2, 64):
        layer.X, layer.m = x[:m], m
        got = layer.run(workspace=ws)
        layer.check(*got)
        again = layer.run(workspace=ws)
        assert all(torch.equal(p, q) for p, q in zip(got, again))           # the same every time, bit for bit
        ws.fill_(255)


def test_captured_calls_share_a_workspace_and_see_new_inputs():
    layer = Layer(13, 512, 192, 30, 4)
    ws = torch.empty(layer.h.workspace_bytes(13), dtype=torch.uint8, device="cuda")
    x2 = torch.zeros(3, 512, dtype=torch.bfloat16, device="cuda")
    y1, y2 = torch.zeros(13, 512, dtype=torch.bfloat16, device="cuda"), torch.zeros(3, 512, dtype=torch.bfloat16, device="cuda")
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    graphs = [torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()]
    with torch.cuda.graph(graphs[0], stream=stream):
        for _ in range(3):
            layer.h.forward(layer.X, layer.Wr, layer.Wgu, layer.Wd, out=y1, workspace=ws)
    with torch.cuda.graph(graphs[1], stream=stream):
        layer.h.forward(x2, layer.Wr, layer.Wgu, layer.Wd, out=y2, workspace=ws)
    for seed in (1, 2):
        gen = torch.Generator().manual_seed(seed)
        layer.X.copy_(torch.randn(13, 512, generator=gen))
        x2.copy_(torch.randn(3, 512, generator=gen))
        for g in graphs + graphs[::-1]:
            g.replay()
        torch.cuda.synchronize()
        got = layer.run()
        layer.check(*got)
        assert torch.equal(y1, got[0])
        assert torch.equal(y2, layer.h.forward(x2, layer.Wr, layer.Wgu, layer.Wd))


def test_a_captured_call_outlives_larger_calls_of_its_handle():
    """The handle's own workspace is the same memory for every number of rows."""
    layer = Layer(64, 256, 64, 10, 3)
    args = (layer.Wr, layer.Wgu, layer.Wd)
    x = layer.X[:1].clone()
    want = layer.h.forward(x, *args)
    y = torch.zeros_like(want)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        layer.h.forward(x, *args, out=y)
    at = layer.h._ws.data_ptr()
    layer.check(*layer.run())                       # 64 rows
    assert layer.h._ws.data_ptr() == at
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(y, want)


def test_banks_past_32_bits():
    """Experts whose weights lie more than 2^32 bytes, and elements, into the banks."""
    e, d, f = 48, 4096, 11264
    h = binding.MoE(d, f, e, 2, score="sigmoid")
    gu, dn = torch.zeros(e, d, 2 * f, dtype=torch.bfloat16, device="cuda"), torch.zeros(e, f, d, dtype=torch.bfloat16, device="cuda")
    wr = torch.zeros(d, e, dtype=torch.bfloat16, device="cuda")
    wr[0, e - 1], wr[1, e - 2] = 8.0, 4.0
    x = torch.zeros(1, d, dtype=torch.bfloat16, device="cuda")
    x[0, 0] = x[0, 1] = 1.0
    gu[e - 1, 0, f - 1], gu[e - 1, 1, 2 * f - 1], dn[e - 1, f - 1, d - 1] = 2.0, 3.0, 0.5
    gu[e - 2, 0, 0], gu[e - 2, 1, f], dn[e - 2, 0, 0] = 1.0, 2.0, 4.0
    y, experts, weights = h.forward(x, wr, gu, dn, out_dtype=torch.float32, routing=True)
    assert experts.tolist() == [[e - 1, e - 2]]
    silu = lambda v: v / (1 + math.exp(-v))  # noqa: E731
    a, b = 1 / (1 + math.exp(-8.0)), 1 / (1 + math.exp(-4.0))
    assert abs(float(y[0, d - 1]) - a / (a + b) * silu(2.0) * 3 * 0.5) < 1e-5 and abs(float(y[0, 0]) - b / (a + b) * silu(1.0) * 2 * 4) < 1e-5
    assert int((y != 0).sum()) == 2


def test_empty_batch_and_refusals():
    layer = Layer(4, 64, 64, 8, 2)
    args = (layer.Wr, layer.Wgu, layer.Wd)
    before = binding.launch_count()
    assert layer.h.forward(layer.X[:0], *args).shape == (0, 64)
    with pytest.raises(binding.AlgError) as err:
        layer.h.forward(torch.zeros(65, 64, dtype=torch.bfloat16, device="cuda"), *args)
    assert err.value.code == 2
    for bad in ((layer.X.float(), *args), (layer.X[:, :56], *args), (layer.X.cpu(), *args), (layer.X, layer.Wr.float(), *args[1:]),
                (layer.X, layer.Wr, layer.Wgu[:, :, :64], layer.Wd), (layer.X, layer.Wr, layer.Wgu, layer.Wd.transpose(1, 2))):
        with pytest.raises(ValueError):
            layer.h.forward(*bad)
    with pytest.raises(binding.AlgError) as err:
        layer.h.forward(layer.X, *args, out=layer.X)                       # Y over X
    assert err.value.code == 1
    with pytest.raises(binding.AlgError) as err:
        layer.h.forward(layer.X, *args, workspace=torch.empty(256, dtype=torch.uint8, device="cuda"))
    assert err.value.code == 3
    odd = torch.zeros(4, 68, dtype=torch.bfloat16, device="cuda")
    with pytest.raises(binding.AlgError):
        layer.h.forward(odd[:, :64], *args)                                # rows off 16 bytes
    assert binding.launch_count() == before
    for d, f, e, k, code in ((60, 64, 8, 2, 2), (64, 60, 8, 2, 2), (64, 64, 513, 2, 2), (64, 64, 40, 33, 2), (64, 64, 8, 9, 1), (64, 64, 8, 0, 1)):
        with pytest.raises(binding.AlgError) as err:
            binding.MoE(d, f, e, k)
        assert err.value.code == code


@pytest.mark.parametrize("m,d,f,e,k,router,out", [(1, 2048, 768, 128, 8, "bf16", torch.bfloat16), (40, 1024, 256, 33, 4, "f32", torch.float32),
                                                  (64, 520, 200, 300, 6, "bf16", torch.bfloat16)])
def test_a_wait_that_runs_out_ends_the_call(m, d, f, e, k, router, out):
    """Rows that never come whole (their barriers are told to expect more bytes than are sent; every copy that is sent lands): the calls return, the status
    word says so and reading it clears it and the handle's counters: the next call is right, bit for bit."""
    layer = Layer(m, d, f, e, k, router=router)
    first = layer.run(out_dtype=out)
    layer.check(*first)
    layer.h.set_option("test_stall_bytes", 1024)
    for limit in (1000, 20000, 4_000_000):
        layer.h.set_option("wait_limit_cycles", limit)
        layer.run(out_dtype=out)
        layer.run(out_dtype=out)
        assert layer.h.last_status() == 6 and layer.h.last_status() == 0
    layer.h.set_option("test_stall_bytes", 0)
    layer.h.set_option("wait_limit_cycles", 4_000_000_000)
    again = layer.run(out_dtype=out)
    assert layer.h.last_status() == 0 and all(torch.equal(p, q) for p, q in zip(first, again))
    for name, value in (("test_stall_bytes", 8), ("test_stall_bytes", 65552), ("wait_limit_cycles", 999), ("stage_k", 64)):
        with pytest.raises(binding.AlgError):
            layer.h.set_option(name, value)


def test_a_workspace_that_the_gpu_cannot_reach_is_refused():
    layer = Layer(4, 64, 64, 8, 2)
    size = layer.h.workspace_bytes(4)
    before = binding.launch_count()
    for bad in (torch.empty(size, dtype=torch.uint8), torch.empty(2 * size, dtype=torch.uint8, device="cuda")[::2]):
        with pytest.raises(ValueError):
            layer.run(workspace=bad)
    assert binding.launch_count() == before


@pytest.mark.parametrize("m,d,f,e,k", [(1, 2048, 768, 128, 8), (9, 520, 136, 33, 3), (64, 256, 128, 8, 2), (5, 136, 1032, 40, 1)])
def test_a_bf16_result_is_the_fp32_result_rounded_once(m, d, f, e, k):
    """Nothing on the way is held in fewer bits for a result of fewer."""
    layer = Layer(m, d, f, e, k)
    y, experts, weights = layer.run(out_dtype=torch.float32)
    short = layer.run(out_dtype=torch.bfloat16)
    assert torch.equal(short[0], y.bfloat16()) and torch.equal(short[1], experts) and torch.equal(short[2], weights)
