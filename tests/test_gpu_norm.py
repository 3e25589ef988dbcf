"""The border of a block -- norms before and after it, gate, residual scale -- and its gradients, against the definitions in 64 bits
(gradients by autograd of the definition).

Tolerances.  All arithmetic is fp32 with sums of at most 16 columns a thread, then trees: 16 + 10 additions, a reciprocal root of 2 units,
sigmoids of 4 units and fewer than 20 roundings otherwise, so every result is off by at most 64 * 2^-24 of the sum of the magnitudes that went
into it (written beside each), plus half a step of its type.  Column sums add at most 14 rows a thread, 15 groups, 19 CTAs and 8 slices: the
same 64 once more."""
import math

import pytest
import torch

from paper_2609_32814_b200 import binding

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "f32": torch.float32}
EPS = 1e-5
U = 64 * 2.0 ** -24


def norm(x, kind, w=None, b=None):
    mu = x.mean(1, keepdim=True) if kind == "layer" else 0.0
    v = (x - mu) / torch.sqrt(((x - mu) ** 2).mean(1, keepdim=True) + EPS)
    v = v if w is None else v * w
    return v if b is None else v + b


def norm_size(x, kind, w=None, b=None):
    """Magnitudes behind norm(x)."""
    r = 1 / torch.sqrt(((x - (x.mean(1, keepdim=True) if kind == "layer" else 0.0)) ** 2).mean(1, keepdim=True) + EPS)
    v = (x.abs() + (x.abs().mean(1, keepdim=True) if kind == "layer" else 0.0)) * r
    v = v if w is None else v * w.abs()
    return v if b is None else v + b.abs()


def through(x, kind, h):
    """Magnitudes behind the gradient of the normed x for the gradient h."""
    mu = x.mean(1, keepdim=True) if kind == "layer" else 0.0
    r = 1 / torch.sqrt(((x - mu) ** 2).mean(1, keepdim=True) + EPS)
    v = (x.abs() + (x.abs().mean(1, keepdim=True) if kind == "layer" else 0.0)) * r
    h = h.abs()
    return 2 * r * (h + h.mean(1, keepdim=True) + v * (h * v).mean(1, keepdim=True))


def near(got, want, size, what, u=U):
    assert got.shape == want.shape, what
    bound = u * size + torch.finfo(got.dtype).eps / 2 * want.abs() + 1e-30
    off = (got.double().cpu() - want).abs()
    bad = ~(off <= bound)
    assert not bool(bad.any()), f"{what}: {int(bad.sum())} of {bad.numel()}, worst {float((off / bound).max()):.2f} of the bound"


class Border:
    """Inputs of one call, and what the definitions give for them."""

    def __init__(self, m, d, kind, post, pre, gate, sig, vectors, dtype, stream, seed=0, pitch=0, at=0, join=True, mean=0.0):
        gen = torch.Generator().manual_seed(1000 * m + d + seed)
        self.m, self.d, self.kind, self.post, self.pre, self.join = m, d, kind, post, pre, join
        rnd = lambda *s: torch.randn(*s, generator=gen, dtype=torch.float64)  # noqa: E731
        self.bufs = []

        def rows(dt, x):
            ld = pitch or d
            buf = torch.full((m * ld + at + 16,), 5.0, dtype=DT[dt], device="cuda")
            t = buf[at:at + m * ld].view(m, ld)[:, :d]
            t.copy_(x)
            return t

        x = rnd(m, d) + mean
        x[:, ::29] *= 12.0
        self.R, self.dY, self.dN = rows(stream, x), rows(stream, rnd(m, d)), rows(dtype, rnd(m, d))
        self.F = rows(dtype, rnd(m, d) + mean)
        self.out = {k: rows(t, torch.zeros(m, d)) for k, t in (("Y", stream), ("N", dtype), ("R", stream), ("F", dtype))}
        self.gate = None if gate is None else rnd(m).to(DT[dtype]).cuda() if gate == "row" else rows(dtype, rnd(m, d))
        vec = lambda on, c: (c + 0.3 * rnd(d)).float().cuda() if on and vectors else None  # noqa: E731
        self.vec = {"post_weight": vec(post, 1), "post_bias": vec(post, 0), "scale": vec(join, 0.5), "pre_weight": vec(pre, 1),
                    "pre_bias": vec(pre, 0)}
        self.alpha, self.sig = 0.75, sig
        self.h = binding.BlockNorm(d, kind=kind, join=join, pre=pre, post=post, gate=gate, gate_act="sigmoid" if sig else None, eps=EPS,
                                   dtype=dtype, stream_dtype=stream)
        w = lambda t: None if t is None else t.double().cpu()  # noqa: E731
        self.w = {k: w(t) for k, t in {**self.vec, "R": self.R, "F": self.F, "gate": self.gate, "dY": self.dY, "dN": self.dN}.items()}

    def call(self):
        kw = dict(self.vec, alpha=self.alpha)
        if self.join:
            kw.update(F=self.F, gate=self.gate)
        return kw

    def factor(self, v):
        """alpha * scale * gate."""
        f = torch.full((self.m, self.d), self.alpha, dtype=torch.float64)
        if v["scale"] is not None:
            f = f * v["scale"]
        if v["gate"] is not None:
            g = torch.sigmoid(v["gate"]) if self.sig else v["gate"]
            f = f * (g[:, None] if g.dim() == 1 else g)
        return f

    def branch(self, v):
        return norm(v["F"], self.kind, v["post_weight"], v["post_bias"]) if self.post else v["F"]

    def check_forward(self, y, n):
        w = self.w
        if not self.join:
            want, size = w["R"], torch.zeros_like(w["R"])
        else:
            want = w["R"] + self.factor(w) * self.branch(w)
            v = norm_size(w["F"], self.kind, w["post_weight"], w["post_bias"]) if self.post else w["F"].abs()
            size = w["R"].abs() + self.factor(w).abs() * v
            near(y, want, size, "Y")
        if self.pre:
            # (Y's own error comes through the norm as a gradient does)
            near(n, norm(want, self.kind, w["pre_weight"], w["pre_bias"]),
                 norm_size(want, self.kind, w["pre_weight"], w["pre_bias"]) +
                 through(want, self.kind, size) * (1 if w["pre_weight"] is None else w["pre_weight"].abs()), "N")

    def check_backward(self, y, got, dy=True):
        w = self.w
        y = y.double().cpu()
        leaf = lambda t: None if t is None else t.clone().requires_grad_(True)  # noqa: E731
        T = w["dY"].clone() if dy else torch.zeros_like(y)
        size = T.abs()
        if self.pre:
            yl, pw, pb = leaf(y), leaf(w["pre_weight"]), leaf(w["pre_bias"])
            xs = [t for t in (yl, pw, pb) if t is not None]
            gr = list(torch.autograd.grad(norm(yl, self.kind, pw, pb), xs, w["dN"]))
            T = T + gr.pop(0)
            h = w["dN"] if pw is None else w["dN"] * w["pre_weight"]
            size = size + through(y, self.kind, h)
            if pw is not None:
                near(got["pre_weight"], gr.pop(0), (w["dN"].abs() * norm_size(y, self.kind)).sum(0), "pre_weight", 2 * U)
            if pb is not None:
                near(got["pre_bias"], gr.pop(0), w["dN"].abs().sum(0), "pre_bias", 2 * U)
        near(got["R"], T, size, "dR")
        if not self.join:
            return
        v = {k: leaf(t) for k, t in w.items()}
        names = [k for k in ("F", "gate", "post_weight", "post_bias", "scale") if v[k] is not None]
        gr = dict(zip(names, torch.autograd.grad(self.factor(v) * self.branch(v), [v[k] for k in names], T)))
        vs = norm_size(w["F"], self.kind) if self.post else w["F"].abs()           # V
        nb = norm_size(w["F"], self.kind, w["post_weight"], w["post_bias"]) if self.post else vs
        fac = self.factor(w).abs()
        bare = self.factor(dict(w, scale=None)).abs()
        e = size * fac * (1 if w["post_weight"] is None else w["post_weight"].abs())
        near(got["F"], gr["F"], through(w["F"], self.kind, e) if self.post else e, "dF")
        if "gate" in gr:
            one = dict(w, gate=None)
            k = size * self.factor(one).abs() * nb      # (a sigmoid's slope is at most its gate)
            k = k.sum(1) if w["gate"].dim() == 1 else k
            near(got["gate"], gr["gate"], k, "dgate")
        if "post_weight" in gr:
            near(got["post_weight"], gr["post_weight"], (size * fac * vs).sum(0), "post_weight", 2 * U)
            near(got["post_bias"], gr["post_bias"], (size * fac).sum(0), "post_bias", 2 * U)
        if "scale" in gr:
            near(got["scale"], gr["scale"], (size * bare * nb).sum(0), "scale", 2 * U)


FORMS = [  # kind, post, pre, gate, sigmoid, vectors
    ("rms", True, True, None, False, True), ("rms", True, True, "element", True, True), ("layer", True, True, "row", True, True),
    ("layer", True, True, "element", False, True), ("rms", False, True, "row", False, True), ("layer", False, True, None, False, False),
    ("rms", True, False, "element", False, True), ("layer", True, False, "row", False, False), ("rms", False, False, "element", True, True),
    ("rms", False, False, None, False, False)]


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("dtype,stream,m,d,pitch,at", [("bf16", "bf16", 1, 8, 0, 0), ("bf16", "f32", 37, 264, 272, 8), ("f32", "bf16", 5, 1000, 0, 0),
                                                       ("bf16", "bf16", 9, 333, 335, 1), ("f32", "f32", 3, 1, 0, 0),
                                                       ("bf16", "f32", 37, 256, 260, 4), ("bf16", "bf16", 300, 513, 0, 0), ("bf16", "f32", 40, 770, 771, 3)])
def test_border_and_its_gradients(form, dtype, stream, m, d, pitch, at):
    kind, post, pre, gate, sig, vectors = form
    b = Border(m, d, kind, post, pre, gate, sig, vectors, dtype, stream, pitch=pitch, at=at)
    y, n = b.h.forward(b.R, **b.call(), out=b.out["Y"], normed=b.out["N"] if pre else None)
    b.check_forward(y, n)
    got = b.h.backward(y, dY=b.dY, dN=b.dN if pre else None, **b.call(), out={"R": b.out["R"], "F": b.out["F"]})
    b.check_backward(y, got)
    first = {k: v.clone() for k, v in got.items()}
    again = b.h.backward(y, dY=b.dY, dN=b.dN if pre else None, **b.call(), out={"R": b.out["R"], "F": b.out["F"]})
    for k in got:
        assert torch.equal(first[k], again[k]), k                     # bitwise repeatable
    if pre:
        b.check_backward(y, b.h.backward(y, dN=b.dN, **b.call()), dy=False)
    for t in (b.R, b.F, b.out["Y"], b.out["R"]):                      # nothing between the rows was touched
        base = t._base if t._base is not None else t
        while base._base is not None:
            base = base._base
        edge = torch.ones_like(base, dtype=torch.bool)
        edge[at:at + m * (pitch or d)].view(m, -1)[:, :d] = False
        assert bool((base[edge] == 5.0).all())
    assert b.h.last_status() == 0


@pytest.mark.parametrize("kind,dtype,stream,m,d", [("rms", "bf16", "bf16", 1999, 768), ("layer", "bf16", "f32", 700, 2048), ("rms", "f32", "f32", 300, 4096),
                                                   ("layer", "f32", "f32", 310, 8192), ("rms", "bf16", "bf16", 450, 7168), ("layer", "bf16", "bf16", 160, 4104),
                                                   ("rms", "bf16", "f32", 155, 5003), ("layer", "bf16", "bf16", 2001, 96), ("rms", "bf16", "bf16", 1201, 1002), ("layer", "bf16", "f32", 903, 2047),
                                                   ("rms", "bf16", "bf16", 333, 4097), ("layer", "bf16", "bf16", 320, 8192), ("layer", "bf16", "f32", 301, 5003),
                                                   ("layer", "bf16", "f32", 299, 8192), ("layer", "bf16", "bf16", 170, 4091), ("layer", "f32", "f32", 150, 4095),
                                                   ("rms", "bf16", "bf16", 163, 8191), ("layer", "bf16", "f32", 161, 8186), ("layer", "bf16", "bf16", 320, 8184)])
def test_many_rows(kind, dtype, stream, m, d):
    """More rows than a grid takes at once, every width of a thread's share, stages that wrap."""
    b = Border(m, d, kind, True, True, "element", True, True, dtype, stream)
    y, n = b.h.forward(b.R, **b.call())
    b.check_forward(y, n)
    b.check_backward(y, b.h.backward(y, dY=b.dY, dN=b.dN, **b.call()))


@pytest.mark.parametrize("dtype,stream", [("bf16", "f32"), ("f32", "bf16"), ("bf16", "bf16"), ("f32", "f32")])
@pytest.mark.parametrize("kind,vectors", [("rms", False), ("layer", True)])
@pytest.mark.parametrize("m,d,pitch", [(1, 596, 0), (1, 2956, 0), (7, 596, 600), (3, 4, 8), (5, 8188, 8192)])
def test_rows_on_sixteen_bytes_that_end_inside_them(dtype, stream, kind, vectors, m, d, pitch):
    """Four columns are 16 bytes of fp32 and half of that in bf16: the rows begin on 16 bytes and end between them."""
    b = Border(m, d, kind, True, True, "element", True, vectors, dtype, stream, pitch=pitch)
    y, n = b.h.forward(b.R, **b.call())
    b.check_forward(y, n)
    b.check_backward(y, b.h.backward(y, dY=b.dY, dN=b.dN, **b.call()))
    assert b.h.last_status() == 0


@pytest.mark.parametrize("kind,back", [("rms", 0), ("layer", 0), ("rms", 1), ("layer", 1)])
def test_operands_that_lie_off_sixteen_bytes_each_in_its_own_way(kind, back):
    """Rows of R, F and the outputs begin at different places of a 16-byte word: single accesses, and the same results."""
    b = Border(23, 520, kind, True, True, "element", False, True, "bf16", "bf16")
    y, n = b.h.forward(b.R, **b.call())
    want = b.h.backward(y, dY=b.dY, dN=b.dN, **b.call())

    def moved(t, ld, at):
        buf = torch.full((23 * ld + at + 8,), 3.0, dtype=t.dtype, device="cuda")
        out = buf[at:at + 23 * ld].view(23, ld)[:, :520]
        out.copy_(t)
        return out, buf

    r, f, g = moved(b.R, 521, 1)[0], moved(b.F, 523, 0)[0], moved(b.gate, 520, 5)[0]
    out, buf = moved(b.R, 527, 3)
    kw = dict(b.call(), F=f, gate=g)
    if not back:
        y2, n2 = b.h.forward(r, **kw, out=out)
        # (sums run in another order: fp32 rounding, then one step of bf16 at most)
        assert bool(((y2.float() - y.float()).abs() <= 2.0 ** -8 * y.float().abs() + 1e-6).all())
        assert bool(((n2.float() - n.float()).abs() <= 2.0 ** -7 * n.float().abs() + 1e-5).all())
        assert bool((buf[3:3 + 23 * 527].view(23, 527)[:, 520:] == 3.0).all() & (buf[:3] == 3.0).all() & (buf[-5:] == 3.0).all())
        return
    got = b.h.backward(moved(y, 525, 2)[0], dY=moved(b.dY, 522, 7)[0], dN=moved(b.dN, 520, 0)[0], **kw, out={"R": out})
    for k in want:
        size = float(want[k].float().abs().max())
        assert bool(((got[k].float() - want[k].float()).abs() <= 2.0 ** -7 * want[k].float().abs() + 1e-5 * size).all()), k


@pytest.mark.parametrize("kind", ["rms", "layer"])
@pytest.mark.parametrize("m,d,mean", [(1, 2048, 0.0), (70, 640, 0.0), (33, 1001, 30.0)])
def test_plain_norm_without_a_block(kind, m, d, mean):
    """No F: Y is R.  A mean far from zero is taken off before the squares are added."""
    b = Border(m, d, kind, False, True, None, False, True, "bf16", "f32", join=False, mean=mean)
    kw = {k: b.vec[k] for k in ("pre_weight", "pre_bias")}
    y, n = b.h.forward(b.R, **kw)
    assert y is b.R
    b.check_forward(y, n)
    b.check_backward(y, b.h.backward(y, dY=b.dY, dN=b.dN, **kw))


def test_gradients_against_differences():
    """Central differences of the forward pass, in the direction of each operand."""
    b = Border(6, 48, "layer", True, True, "row", True, True, "f32", "f32")
    cy, cn = torch.randn(6, 48, device="cuda"), torch.randn(6, 48, device="cuda")

    def value(**change):
        kw = dict(b.call(), **{k: v for k, v in change.items() if k != "R"})
        y, n = b.h.forward(change.get("R", b.R), **kw)
        return float((y.double() * cy).sum() + (n.double() * cn).sum())

    y, _ = b.h.forward(b.R, **b.call())
    got = b.h.backward(y, dY=cy, dN=cn, **b.call())
    h = 2.0 ** -7
    for k in ("R", "F", "gate", "post_weight", "post_bias", "scale", "pre_weight", "pre_bias"):
        x = b.R if k == "R" else b.call()[k]
        step = torch.randn(x.shape, device="cuda")
        slope = (value(**{k: x + h * step}) - value(**{k: x - h * step})) / (2 * h)
        want = float((got[k].double() * step).sum())
        # the sum of 576 products of fp32 results of size < 10 is off by < 576 * 10 * 2^-22 / h; third differences add h^2 times a few
        # hundred times the slope's size at most
        size = float((got[k].double().abs() * step.abs()).sum())
        assert abs(slope - want) <= 576 * 10 * 2.0 ** -22 / h + 40 * h * h * size, k


def test_rows_in_place():
    b = Border(50, 512, "rms", True, True, "element", False, True, "bf16", "bf16")
    y, n = b.h.forward(b.R, **b.call())
    want = b.h.backward(y, dY=b.dY, dN=b.dN, **b.call())
    r, f = b.R.clone(), b.F.clone()
    y2, n2 = b.h.forward(r, **dict(b.call(), F=f), out=r, normed=f)
    assert y2 is r and torch.equal(y2, y) and torch.equal(n2, n)
    dy, dn, g = b.dY.clone(), b.dN.clone(), b.gate.clone()
    got = b.h.backward(y, dY=dy, dN=dn, **dict(b.call(), gate=g), out={"R": dy, "F": dn, "gate": g})
    for k in want:
        assert torch.equal(got[k], want[k]), k


def test_infinities_and_nans_stay_in_their_rows():
    b = Border(20, 256, "layer", True, True, "row", False, True, "f32", "f32")
    y0, n0 = b.h.forward(b.R, **b.call())
    b.R[3, 7], b.F[11, 0], b.gate[17] = math.inf, math.nan, math.inf
    y, n = b.h.forward(b.R, **b.call())
    rest = [r for r in range(20) if r not in (3, 11, 17)]
    assert torch.equal(y[rest], y0[rest]) and torch.equal(n[rest], n0[rest])
    assert bool(n[3].isnan().any()) and bool(y[11].isnan().all()) and not bool(torch.isfinite(y[17]).any())


def test_zero_rows_and_constant_rows():
    b = Border(4, 64, "layer", True, True, None, False, False, "f32", "f32")
    b.R.zero_()
    b.F.fill_(3.0)
    y, n = b.h.forward(b.R, **dict(b.call()))
    assert bool((y == 0).all()) and bool((n == 0).all())
    got = b.h.backward(y, dY=b.dY, dN=b.dN, **b.call())
    assert all(bool(torch.isfinite(t).all()) for t in got.values())


def test_empty_batch():
    b = Border(1, 64, "rms", True, True, None, False, True, "bf16", "bf16")
    e = torch.empty(0, 64, dtype=torch.bfloat16, device="cuda")
    before = binding.launch_count()
    y, n = b.h.forward(e, **dict(b.call(), F=e))
    assert y.shape == n.shape == (0, 64) and binding.launch_count() == before
    got = b.h.backward(e, dY=e, dN=e, **dict(b.call(), F=e))
    for k in ("post_weight", "scale", "pre_weight", "pre_bias"):
        assert bool((got[k] == 0).all())


def test_replayed_graph_and_another_stream():
    b = Border(300, 768, "rms", True, True, "row", True, True, "bf16", "bf16")
    y, n = b.h.forward(b.R, **b.call())
    want = b.h.backward(y, dY=b.dY, dN=b.dN, **b.call())
    ws = torch.empty(b.h.workspace_bytes(), dtype=torch.uint8, device="cuda")
    out = {k: torch.zeros_like(v) for k, v in want.items()}
    y2, n2 = torch.zeros_like(y), torch.zeros_like(n)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        b.h.forward(b.R, **b.call(), out=y2, normed=n2)
        b.h.backward(y2, dY=b.dY, dN=b.dN, **b.call(), out=out, workspace=ws)
    ws.fill_(255)
    for _ in range(2):
        for v in out.values():
            v.fill_(9.0)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y2, y) and torch.equal(n2, n)
        for k in want:
            assert torch.equal(out[k], want[k]), k


def test_refusals():
    h = binding.BlockNorm(64, join=True, post=True, gate="element")
    x = lambda: torch.zeros(4, 64, dtype=torch.bfloat16, device="cuda")  # noqa: E731
    w = torch.ones(64, device="cuda")
    before = binding.launch_count()
    for bad in (dict(F=x()), dict(gate=x()), dict(F=x(), gate=torch.zeros(4, device="cuda").bfloat16()), dict(F=x()[:, :63], gate=x()),
                dict(F=x().float(), gate=x()), dict(F=x().cpu(), gate=x()), dict(F=x(), gate=x(), post_weight=w[:63]),
                dict(F=x(), gate=x(), post_weight=w.bfloat16())):
        with pytest.raises((ValueError, IndexError, binding.AlgError)):
            h.forward(x(), **bad)
    wide = torch.zeros(4, 96, dtype=torch.bfloat16, device="cuda")
    with pytest.raises(binding.AlgError) as e:
        h.forward(wide[:, :64], F=x(), gate=x(), out=wide[:, 32:])    # overlaps, but is not the same
    assert e.value.code == 1
    r = x()
    with pytest.raises(binding.AlgError):
        h.forward(r, F=x(), gate=x(), out=r, normed=r)                # two outputs in one place
    with pytest.raises(binding.AlgError) as e:
        h.backward(x(), dY=x(), dN=x(), F=x(), gate=x(), post_weight=w, workspace=torch.empty(256, dtype=torch.uint8, device="cuda"))
    assert e.value.code == 3
    with pytest.raises(binding.AlgError):
        h.backward(x(), dY=x(), F=x(), gate=x())                      # a PRE handle needs dN
    two = torch.ones(100, device="cuda")
    for out in ({"scale": w}, {"scale": two[:64], "post_weight": two[36:]}):   # gradients over what is read, and over one another
        with pytest.raises(binding.AlgError):
            h.backward(x(), dY=x(), dN=x(), F=x(), gate=x(), scale=w, post_weight=torch.ones(64, device="cuda"), out=out)
    plain = binding.BlockNorm(64)
    with pytest.raises(binding.AlgError):
        plain.forward(x(), F=x())
    with pytest.raises(ValueError):
        plain.backward(x(), dN=x(), want=["nothing"])
    assert binding.launch_count() == before
    for kw in (dict(D=0), dict(D=64, pre=False), dict(D=64, post=True), dict(D=64, join=True, gate_act="sigmoid"), dict(D=64, eps=-1.0)):
        with pytest.raises(binding.AlgError) as e:
            binding.BlockNorm(**kw)
        assert e.value.code == 1
    with pytest.raises(binding.AlgError) as e:
        binding.BlockNorm(8193)
    assert e.value.code == 2


@pytest.mark.parametrize("kind,gate,dtype,stream,d", [("rms", "element", "bf16", "bf16", 512), ("layer", "element", "bf16", "f32", 264), ("rms", "row", "bf16", "bf16", 512),
                                                      ("layer", "row", "f32", "f32", 96), ("rms", "element", "f32", "f32", 333), ("layer", "element", "bf16", "bf16", 4104)])
def test_slope_of_a_saturated_sigmoid(kind, gate, dtype, stream, d):
    """The gate's gradient where the sigmoid is nearly 0 or 1, to a bound that shrinks with the slope.

    slope = s s e with e = exp(-x), s = 1 / (1 + e): in units of 2^-24 of it e is off by 4 + 2 |x| (exp2 of two units in the last place, the
    rounding of x log2 e and of the constant), which reaches the slope at most once (its logarithmic derivative in e is (1 - e) / (1 + e)), the
    reciprocal and its sum by 3 each time, two products by 2: 12 + 2 |x| <= 52 for |x| <= 20, beside the 64 of the module's account."""
    m = 16
    b = Border(m, d, kind, True, True, gate, True, True, dtype, stream)
    x = torch.tensor([8.0, -8.0, 12.0, -12.0, 16.0, -16.0, 20.0, -20.0], dtype=torch.float64)
    b.gate.copy_(x.repeat(2) if gate == "row" else x.repeat(-(-d // 8))[:d].expand(m, d))
    b.w["gate"] = b.gate.double().cpu()
    y, n = b.h.forward(b.R, **b.call())
    b.check_forward(y, n)
    got = b.h.backward(y, dY=b.dY, dN=b.dN, **b.call())
    b.check_backward(y, got)
    w, y64 = b.w, y.double().cpu()
    yl = y64.clone().requires_grad_(True)
    T = w["dY"] + torch.autograd.grad(norm(yl, kind, w["pre_weight"], w["pre_bias"]), yl, w["dN"])[0]
    size = w["dY"].abs() + through(y64, kind, w["dN"] * w["pre_weight"])
    s = 1 / (1 + torch.exp(-w["gate"].abs()))
    slope = torch.exp(-w["gate"].abs()) * s * s
    f = b.factor(dict(w, gate=None))
    want, bound = T * f * b.branch(w), size * f.abs() * norm_size(w["F"], kind, w["post_weight"], w["post_bias"])
    if gate == "row":
        want, bound = want.sum(1), bound.sum(1)
    near(got["gate"], want * slope, bound * slope, "dgate", 2 * U)


@pytest.mark.parametrize("gate", ["row", "element"])
def test_gates_that_shut_a_row_off(gate):
    """A sigmoid of -infinity, of the types' lowest values and of +infinity: the gate is 0 or 1 and has no slope."""
    for dtype in ("bf16", "f32"):
        b = Border(6, 72, "rms", True, True, gate, True, True, dtype, "f32")
        low = torch.finfo(DT[dtype]).min
        x = torch.tensor([-math.inf, low, -1000.0, math.inf, -low, 1000.0], dtype=torch.float64)
        b.gate.copy_(x if gate == "row" else x[:, None].expand(6, 72))
        y, n = b.h.forward(b.R, **b.call())
        assert torch.equal(y[:3], b.R[:3])
        got = b.h.backward(y, dY=b.dY, dN=b.dN, **b.call())
        assert all(bool(torch.isfinite(v).all()) for v in got.values())
        assert bool((got["gate"] == 0).all()) and bool((got["F"][:3] == 0).all()) and bool((got["F"][3:] != 0).any(1).all())


@pytest.mark.parametrize("kind,dtype,stream,m,d,pitch", [("rms", "bf16", "bf16", 5000, 64, 0), ("layer", "bf16", "f32", 900, 1024, 0), ("layer", "f32", "f32", 310, 8192, 0),
                                                         ("rms", "bf16", "bf16", 700, 1001, 1003)])
def test_a_wait_that_runs_out_ends_the_call(kind, dtype, stream, m, d, pitch):
    """Copies that never come (the rows' barriers are told to expect more bytes than are sent; every copy that is sent lands): the calls return, the status
    word says so and is cleared by reading it, nothing beside the outputs is touched, and the next calls are right, bit for bit."""
    b = Border(m, d, kind, True, True, "element", True, True, dtype, stream, pitch=pitch)
    kw = dict(b.call())
    y, n = b.h.forward(b.R, **kw, out=b.out["Y"], normed=b.out["N"])
    y = y.clone()
    first = {"Y": y, "N": n.clone(), **{k: v.clone() for k, v in b.h.backward(y, dY=b.dY, dN=b.dN, **kw).items()}}
    b.h.set_option("test_stall_bytes", 1024)
    for limit in (1000, 20000, 4_000_000):
        b.h.set_option("wait_limit_cycles", limit)
        b.h.forward(b.R, **kw, out=b.out["Y"], normed=b.out["N"])
        assert b.h.last_status() == 6 and b.h.last_status() == 0
        b.h.backward(y, dY=b.dY, dN=b.dN, **kw)
        assert b.h.last_status() == 6 and b.h.last_status() == 0
    b.h.set_option("test_stall_bytes", 0)
    b.h.set_option("wait_limit_cycles", 4_000_000_000)
    y2, n2 = b.h.forward(b.R, **kw, out=b.out["Y"], normed=b.out["N"])
    again = {"Y": y2, "N": n2, **b.h.backward(y, dY=b.dY, dN=b.dN, **kw)}
    assert b.h.last_status() == 0
    for k in first:
        assert torch.equal(first[k], again[k]), k
    if pitch:
        for t in (b.R, b.F, b.out["Y"], b.out["N"]):
            assert bool((t._base[:m * pitch].view(m, pitch)[:, d:] == 5.0).all())
    with pytest.raises(binding.AlgError):
        b.h.set_option("test_stall_bytes", 8)
    with pytest.raises(binding.AlgError):
        b.h.set_option("test_stall_bytes", 65552)
    with pytest.raises(binding.AlgError):
        b.h.set_option("wait_limit_cycles", 999)
    with pytest.raises(binding.AlgError):
        b.h.set_option("stage_k", 64)


@pytest.mark.parametrize("kind", ["rms", "layer"])
def test_sums_of_no_rows_are_zero_whatever_the_vectors_hold(kind):
    b = Border(1, 64, kind, True, True, None, False, True, "bf16", "bf16")
    e = torch.empty(0, 64, dtype=torch.bfloat16, device="cuda")
    for bad in (math.inf, math.nan):
        for k, v in b.vec.items():
            v[::3] = bad
        out = {k: torch.full((64,), 7.0, device="cuda") for k in b.vec}
        got = b.h.backward(e, dY=e, dN=e, F=e, alpha=2.0, **b.vec, out=dict(out, R=e.clone()))
        for k in b.vec:
            assert bool((got[k] == 0).all()), k


def test_a_workspace_that_the_gpu_cannot_reach_is_refused():
    b = Border(4, 64, "rms", True, True, None, False, True, "bf16", "bf16")
    y, n = b.h.forward(b.R, **b.call())
    size = b.h.workspace_bytes()
    before = binding.launch_count()
    for bad in (torch.empty(size, dtype=torch.uint8), torch.empty(2 * size, dtype=torch.uint8, device="cuda")[::2]):
        with pytest.raises(ValueError):
            b.h.backward(y, dY=b.dY, dN=b.dN, **b.call(), workspace=bad)
    assert binding.launch_count() == before
