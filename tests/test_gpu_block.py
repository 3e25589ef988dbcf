"""The calls around the projections together with them: a training step of a feed-forward block, and decode steps of a block whose
feed-forward layer is a mixture of experts, against 64-bit compositions.

Tolerances (relative 2-norms).  The chain rounds to bf16 five times on the way up (2^-9 each in the root mean square, 2e-3) and as often
down.  A checkpoint's int8 codes are off by half a step, a step being at most max / 63.5 of its block of 32, max about 2.2 standard
deviations: at most 1 % of the standard deviation in the root mean square, which moves the activation's slope (whose own slope is below 0.8) by
1 % of its size; with the roundings, 3 % bounds what comes through a checkpoint, 1 % what does not."""
import pytest
import torch

from paper_2609_32814_b200 import binding

pytestmark = pytest.mark.gpu


def off(got, want):
    got, want = got.double().cpu(), want.double().cpu()
    return float((got - want).norm() / want.norm())


def star(x, types, w, dw, fw):
    """X *_q W by its definition."""
    y = torch.zeros(x.shape[0], sum(fw), dtype=x.dtype)
    so, ro = [0], [0]
    for a, b in zip(dw, fw):
        so.append(so[-1] + a), ro.append(ro[-1] + b)
    rows = []
    for b in range(x.shape[0]):
        t, parts = int(types[b]), []
        for j in range(len(dw)):
            parts.append(sum(x[b, so[k]:so[k + 1]] @ w[so[k]:so[k + 1], ro[j]:ro[j + 1]] for k in sorted({t, j})))
        rows.append(torch.cat(parts))
    return torch.stack(rows) + y


@pytest.mark.parametrize("fmt,stream", [("int8", torch.float32), ("int8", torch.bfloat16)])
def test_training_step_of_a_block(fmt, stream):
    """N = norm(R); Z = N * W_up; A = gelu(Z); F = A * W_down; R' = R + alpha scale gate norm(F): both passes."""
    m, dw, fw = 150, [128, 128], [256, 256]
    d, f = sum(dw), sum(fw)
    gen = torch.Generator().manual_seed(3)
    rnd = lambda *s: torch.randn(*s, generator=gen)  # noqa: E731
    types = torch.randint(0, 2, (m,), generator=gen).to(torch.int32)
    R, dR2 = rnd(m, d).to(stream), rnd(m, d).to(stream)
    W_up, W_down = (rnd(d, f) * d ** -0.5).bfloat16(), (rnd(f, d) * f ** -0.5).bfloat16()
    gate = rnd(m).bfloat16()
    pre, post, scale = 1 + 0.1 * rnd(d), 1 + 0.1 * rnd(d), 0.5 + 0.1 * rnd(d)
    # on the GPU
    c = lambda t: t.cuda()  # noqa: E731
    sd = "f32" if stream is torch.float32 else "bf16"
    before = binding.BlockNorm(d, dtype="bf16", stream_dtype=sd)
    border = binding.BlockNorm(d, join=True, pre=False, post=True, gate="row", gate_act="sigmoid", dtype="bf16", stream_dtype=sd)
    up, down = binding.Proj(dw, fw), binding.Proj(fw, dw)
    up_g, down_g = binding.ProjGrad(dw, fw), binding.ProjGrad(fw, dw)
    kept = binding.ActCheckpoint(f, act="gelu", fmt=fmt)
    kept_n = binding.ActCheckpoint(d, fmt=fmt)
    t, Wu, Wd = c(types), c(W_up), c(W_down)
    _, N = before.forward(c(R), pre_weight=c(pre))
    Z = up.forward(N, t, Wu)
    A, rec = kept.forward(Z)
    rec_n = kept_n.store(N)
    F = down.forward(A, t, Wd)
    kw = dict(F=F, gate=c(gate), post_weight=c(post), scale=c(scale), alpha=0.5)
    R2, _ = border.forward(c(R), **kw)
    del N, Z, A                                       # what the backward pass has are records
    g = border.backward(R2, dY=c(dR2), **kw)
    dA = down_g.grad_input(g["F"], t, Wd)
    dZ, A = kept.backward(rec, dA)
    dW_down = down_g.grad_weight(A, g["F"], t)
    dN = up_g.grad_input(dZ, t, Wu)
    dW_up = up_g.grad_weight(kept_n.load(rec_n), dZ, t)
    gr = before.backward(c(R), dY=g["R"], dN=dN, pre_weight=c(pre))
    # the same in 64 bits
    v = {k: x.double().requires_grad_(True) for k, x in dict(R=R, W_up=W_up, W_down=W_down, gate=gate, pre=pre, post=post, scale=scale).items()}
    rms = lambda x: x / torch.sqrt((x * x).mean(1, keepdim=True) + 1e-6)  # noqa: E731
    n = rms(v["R"]) * v["pre"]
    z = star(n, types, v["W_up"], dw, fw)
    ff = star(z * torch.special.ndtr(z), types, v["W_down"], fw, dw)
    want = v["R"] + 0.5 * v["scale"] * torch.sigmoid(v["gate"])[:, None] * rms(ff) * v["post"]
    assert off(R2, want.detach()) < 1e-2
    grads = dict(zip(v, torch.autograd.grad(want, list(v.values()), dR2.double())))
    for k, got in (("gate", g["gate"]), ("post", g["post_weight"]), ("scale", g["scale"])):
        assert off(got, grads[k]) < 1e-2, k
    for k, got in (("R", gr["R"]), ("W_up", dW_up), ("W_down", dW_down), ("pre", gr["pre_weight"])):
        assert off(got, grads[k]) < 3e-2, k


@pytest.mark.parametrize("m", [1, 6])
def test_decode_steps_through_a_block_of_experts(m):
    """Two layers of norm, experts and border in one captured graph, replayed on new tokens."""
    d, f, e, k = 512, 192, 16, 4
    gen = torch.Generator().manual_seed(8)
    rnd = lambda *s: torch.randn(*s, generator=gen)  # noqa: E731
    layers = [dict(pre=1 + 0.1 * rnd(d), post=1 + 0.1 * rnd(d), Wr=(rnd(d, e) * 3 * d ** -0.5).bfloat16(), Wgu=(rnd(e, d, 2 * f) * d ** -0.5).bfloat16(),
                   Wd=(rnd(e, f, d) * f ** -0.5).bfloat16()) for _ in range(2)]
    dev = [{n: t.cuda() for n, t in L.items()} for L in layers]
    first = binding.BlockNorm(d, dtype="bf16", stream_dtype="f32")
    border = binding.BlockNorm(d, join=True, post=True, dtype="bf16", stream_dtype="f32")
    moe = binding.MoE(d, f, e, k)
    R = torch.zeros(m, d, device="cuda")
    bufs = [torch.zeros(m, d, device="cuda") for _ in range(2)]
    norms = [torch.zeros(m, d, device="cuda", dtype=torch.bfloat16) for _ in range(3)]
    outs = [torch.zeros(m, d, device="cuda", dtype=torch.bfloat16) for _ in range(2)]
    ws = torch.empty(moe.workspace_bytes(m), dtype=torch.uint8, device="cuda")
    experts = [torch.zeros(m, k, dtype=torch.int32, device="cuda") for _ in range(2)]

    def step():
        first.forward(R, pre_weight=dev[0]["pre"], normed=norms[0])
        x = R
        for i, L in enumerate(dev):
            moe.forward(norms[i], L["Wr"], L["Wgu"], L["Wd"], out=outs[i], workspace=ws, experts=experts[i])
            border.forward(x, F=outs[i], post_weight=L["post"], pre_weight=dev[(i + 1) % 2]["pre"], out=bufs[i], normed=norms[i + 1])
            x = bufs[i]

    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        step()
    rms = lambda x: x / torch.sqrt((x * x).mean(1, keepdim=True) + 1e-6)  # noqa: E731
    for _ in range(3):
        new = rnd(m, d)
        R.copy_(new)
        graph.replay()
        torch.cuda.synchronize()
        x = new.double()
        for i, L in enumerate(layers):
            n = norms[i].double().cpu()               # (the router chooses by what it was given)
            assert off(norms[i], rms(x) * layers[i]["pre"].double()) < 1e-2
            p = torch.softmax(n @ L["Wr"].double(), 1)
            idx = torch.argsort(p, dim=1, descending=True, stable=True)[:, :k]
            assert torch.equal(experts[i].cpu().long(), idx)
            w = p.gather(1, idx)
            w = w / w.sum(1, keepdim=True)
            y = torch.zeros(m, d, dtype=torch.float64)
            for r in range(m):
                for j in range(k):
                    gu = n[r] @ L["Wgu"][idx[r, j]].double()
                    h = torch.nn.functional.silu(gu[:f]) * gu[f:]
                    y[r] += w[r, j] * (h @ L["Wd"][idx[r, j]].double())
            assert off(outs[i], y) < 1e-2
            x = x + rms(y) * L["post"].double()
            assert off(bufs[i], x) < 1e-2
            x = bufs[i].double().cpu()
    assert moe.last_status() == first.last_status() == border.last_status() == 0
