"""Activations kept in 8 bits: store and load, and the activation's forward and backward pass around a checkpoint, against the
definitions in 64 bits.

Tolerances.  Codes are exact functions of the values, so what reads back is compared for equality.  Activations and slopes are
fp32 expressions: exp and reciprocal approximations of 2 units each (with an argument whose rounding is worth |z| 2^-24 relative, which
counts only where exp(-|z|) has not made the value vanish: |z| exp(-|z|) <= 0.37), erf of 2 units, and at most eight roundings of terms no larger
than 1.2 |z| + 1.2, all times |u dA|: 16 * 2^-23 * (1.2 |z| + 1.2) |u dA| bounds them, plus half a step of the result's type."""
import math

import pytest
import torch

from paper_2609_32814_b200 import binding

pytestmark = pytest.mark.gpu

TOP = {"e4m3": 448.0, "int8": 127.0}
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def kept(x, fmt):
    """What a checkpoint of x stands for, in 64 bits."""
    m, n = x.shape
    full = torch.zeros(m, -(-n // 32) * 32, dtype=torch.float64)
    full[:, :n] = x.double().cpu()
    out = torch.empty_like(full)
    for b in range(full.shape[1] // 32):
        blk = full[:, 32 * b:32 * b + 32]
        for r in range(m):
            row = blk[r]
            if not torch.isfinite(row).all():
                out[r, 32 * b:32 * b + 32] = math.nan
                continue
            top = float(row.abs().max())
            e = -120
            if top > TOP[fmt] * 2.0 ** -120:
                e = math.frexp(top / TOP[fmt])[1] - 1
                while top > TOP[fmt] * 2.0 ** e:
                    e += 1
            q = row * 2.0 ** -e
            if fmt == "int8":
                q = torch.round(q)
            else:
                step = 2.0 ** (torch.floor(torch.log2(q.abs().clamp(min=2.0 ** -6))) - 3)
                q = torch.round(q / step) * step
            out[r, 32 * b:32 * b + 32] = q * 2.0 ** e
    return out[:, :n]


def act_and_slope(z, act):
    z = z.clone().requires_grad_(True)
    a = {"gelu": lambda: z * torch.special.ndtr(z), "silu": lambda: z * torch.sigmoid(z), None: lambda: z * 1.0,
         "gelu_tanh": lambda: z / 2 * (1 + torch.tanh(math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3)))}[act]()
    return a.detach(), torch.autograd.grad(a.sum(), z)[0]


def close(got, want, z, factor, what):
    eps = torch.finfo(got.dtype).eps / 2
    bound = 16 * 2.0 ** -23 * (1.2 * z.abs() + 1.2) * factor.abs() + eps * want.abs() + 1e-30
    bad = (got.double().cpu() - want).abs() > bound
    assert not bool(bad.any()), f"{what}: {int(bad.sum())} of {bad.numel()}, first at {bad.nonzero()[0].tolist()}"


def matrix(gen, m, n, dtype, ld=None, at=0):
    """m x n values, rows ld apart, beginning `at` elements into their memory."""
    ld = ld or n
    buf = torch.full((m * ld + at + 8,), 7.0, dtype=DT[dtype], device="cuda")
    t = buf[at:at + m * ld].view(m, ld)[:, :n]
    x = torch.randn((m, n), generator=gen, dtype=torch.float64)
    x[:, ::37] *= 20.0
    t.copy_(x)
    return t, buf


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("m,n,ld,at", [(1, 1, 0, 0), (1, 32, 0, 0), (3, 31, 0, 0), (5, 33, 40, 1), (2, 4104, 0, 0), (67, 256, 264, 8),
                                       (130, 1000, 1001, 0), (1, 20001, 0, 0)])
def test_store_and_load_are_exact(fmt, dtype, m, n, ld, at):
    gen = torch.Generator().manual_seed(m * 1000 + n)
    x, _ = matrix(gen, m, n, dtype, ld or n, at)
    c = binding.ActCheckpoint(n, fmt=fmt)
    rec = c.store(x)
    want = kept(x, fmt)
    assert torch.equal(c.load(rec, out_dtype=torch.float32).double().cpu(), want)
    assert torch.equal(c.load(rec).double().cpu(), want)           # (8 significant bits: exact in bf16)
    out, buf = matrix(gen, m, n, dtype, ld or n, at)
    before = buf.clone()
    c.load(rec, out=out)
    assert torch.equal(out.double().cpu(), want)
    out.copy_(before[at:at + m * (ld or n)].view(m, -1)[:, :n])
    assert torch.equal(buf, before)                                # nothing between and behind the rows was touched
    half = m // 2
    assert torch.equal(c.load(rec[half:], out_dtype=torch.float32).double().cpu(), want[half:])


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
def test_borders_of_the_scale_and_of_the_format(fmt):
    """Largest magnitudes on, just below and just above a power of two's reach; ties; subnormals; zero, tiny and huge blocks."""
    top = TOP[fmt]
    rows = []
    for k in (-130, -125, -100, -3, 0, 5, 100):
        for f in (top, top * (1 + 2.0 ** -23), top * (1 - 2.0 ** -24), 2.0 ** 8, 2.0 ** 8 * (1 - 2.0 ** -24), 1.0):
            row = torch.linspace(-1, 1, 32, dtype=torch.float64) * f * 2.0 ** k
            row[5] = f * 2.0 ** k
            rows.append(row)
    ties = torch.tensor([top] + [j + 0.5 for j in range(15)] + [-(j + 0.5) for j in range(16)], dtype=torch.float64)
    rows += [ties, ties / 16, ties * 2.0 ** -9, torch.zeros(32, dtype=torch.float64), torch.full((32,), 2.0 ** -149, dtype=torch.float64),
             torch.full((32,), torch.finfo(torch.float32).max, dtype=torch.float64)]
    x = torch.stack(rows).float().cuda()
    c = binding.ActCheckpoint(32, fmt=fmt)
    want = kept(x, fmt)
    assert torch.equal(c.load(c.store(x), out_dtype=torch.float32).double().cpu(), want.float().double())


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
def test_a_block_with_an_infinity_or_a_nan_reads_back_as_nan_and_no_other(fmt):
    x = torch.randn(4, 100, device="cuda")
    x[0, 3], x[1, 40], x[2, 99] = math.inf, -math.inf, math.nan
    c = binding.ActCheckpoint(100, fmt=fmt)
    got = c.load(c.store(x), out_dtype=torch.float32).cpu()
    nan = torch.zeros(4, 100, dtype=torch.bool)
    nan[0, :32], nan[1, 32:64], nan[2, 96:] = True, True, True
    assert torch.equal(got.isnan(), nan)
    assert torch.equal(got[~nan].double(), kept(x, fmt)[~nan])


@pytest.mark.parametrize("act,gated", [("gelu", False), ("gelu_tanh", False), ("silu", False), (None, False), ("silu", True), ("gelu", True),
                                       (None, True)])
@pytest.mark.parametrize("fmt,dtype,m,f,ld,at", [("e4m3", "bf16", 1, 8, 0, 0), ("int8", "bf16", 131, 200, 0, 0), ("int8", "f32", 3, 33, 0, 0),
                                                 ("e4m3", "f32", 70, 96, 104, 4), ("e4m3", "bf16", 9, 1031, 1033, 3)])
def test_activation_and_its_gradient_from_the_checkpoint(act, gated, fmt, dtype, m, f, ld, at):
    gen = torch.Generator().manual_seed(f)
    wide = 2 * f if gated else f
    z, _ = matrix(gen, m, wide, dtype, ld and (wide + ld - f), at)
    da, _ = matrix(gen, m, f, dtype, ld or f, at)
    c = binding.ActCheckpoint(f, act=act, gated=gated, fmt=fmt)
    a, rec = c.forward(z)
    z64, d64 = z.double().cpu(), da.double().cpu()
    g, u = (z64[:, :f], z64[:, f:]) if gated else (z64, torch.ones_like(z64))
    close(a, act_and_slope(g, act)[0] * u, g, u, "A")
    dz, again = c.backward(rec, da)
    kg, ku = (kept(z[:, :f], fmt), kept(z[:, f:], fmt)) if gated else (kept(z, fmt), torch.ones_like(z64))
    ak, slope = act_and_slope(kg, act)
    close(again, ak * ku, kg, ku, "the activation once more")
    close(dz[:, :f], slope * ku * d64, kg, ku * d64, "dZ")
    if gated:
        close(dz[:, f:], ak * d64, kg, d64, "dU")
    # without the second output, without a checkpoint, and in place
    assert torch.equal(c.backward(rec, da, again=False)[0], dz) and c.backward(rec, da, again=False)[1] is None
    plain, none = c.forward(z, keep=False)
    assert none is None and torch.equal(plain, a)
    if not gated:
        over = da.clone()
        c.backward(rec, over, out=over, again=False)
        assert torch.equal(over, dz)
        over = z.clone()
        _, rec2 = c.forward(over, out=over)
        assert torch.equal(over, a) and torch.equal(c.load(rec2), c.load(rec))


@pytest.mark.parametrize("act", ["gelu", "gelu_tanh", "silu"])
def test_slope_against_differences(act):
    """dZ is what the forward pass changes by: central differences at points that the format holds exactly."""
    z = (torch.arange(-48, 48, dtype=torch.float32) / 8).view(3, 32).cuda()     # int8 codes under a scale of 1/8
    c = binding.ActCheckpoint(32, act=act, fmt="int8")
    dz, _ = c.backward(c.store(z), torch.ones_like(z))
    h = 2.0 ** -6
    hi, lo = c.forward(z + h, keep=False)[0], c.forward(z - h, keep=False)[0]
    # third derivatives of these are below 2.5, so a difference is off by h^2 / 6 * 2.5; its terms by 6 * 2^-22
    assert float(((hi - lo).double() / (2 * h) - dz.double()).abs().max()) <= h * h / 6 * 2.5 + 2 * 6 * 2.0 ** -22 / (2 * h)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("act", ["gelu", "gelu_tanh", "silu"])
def test_values_that_are_not_finite_reach_the_activation(act, dtype):
    z = torch.zeros(2, 64, device="cuda", dtype=DT[dtype])
    z[0, 3], z[1, 40], z[1, 41] = math.nan, math.inf, 3.0
    a, _ = binding.ActCheckpoint(64, act=act).forward(z, keep=False)
    assert bool(a[0, 3].isnan()) and float(a[1, 40]) == math.inf and bool(torch.isfinite(a[1, 41]))
    assert int(a.isnan().sum()) == 1 and int(a.isinf().sum()) == 1


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("act", ["gelu", "gelu_tanh", "silu"])
def test_magnitudes_whose_square_is_infinite(act, dtype):
    """2^70: the activation is z or 0, the slope 1 or 0 (a power of two is its own code)."""
    z = torch.tensor([[2.0 ** 70, -2.0 ** 70] * 20], dtype=torch.bfloat16 if dtype == "bf16" else torch.float32, device="cuda")
    c = binding.ActCheckpoint(40, act=act, fmt="e4m3")
    a, rec = c.forward(z)
    dz, again = c.backward(rec, torch.ones_like(z))
    on = z > 0
    # all exact, but for GELU in bf16 below -6: its lower tail stays there at -6 Phi(-6) = -6 * 9.866e-10 = -5.92e-9, which 2^-27 = 7.45e-9 holds
    assert torch.equal(a[on], z[on]) and torch.equal(again, a) and torch.equal(dz, on.to(z.dtype))
    assert float(a[~on].abs().max()) <= (2.0 ** -27 if act == "gelu" and dtype == "bf16" else 0.0)


def test_far_tails_are_finite():
    z = torch.tensor([[-3e4, -200.0, -88.5, -20.0, 0.0, -0.0, 20.0, 88.5, 200.0, 3e4] + [0.0] * 22], device="cuda")
    for act in ("gelu", "gelu_tanh", "silu"):
        c = binding.ActCheckpoint(32, act=act, fmt="e4m3")
        a, rec = c.forward(z)
        dz, _ = c.backward(rec, torch.ones_like(z))
        assert bool(torch.isfinite(a).all()) and bool(torch.isfinite(dz).all()), act
        assert torch.equal(a[0, 7:10], z[0, 7:10]) and float(a[0, :3].abs().max()) == 0.0


def test_more_rows_than_a_grid_and_a_replayed_graph():
    c = binding.ActCheckpoint(8, act="silu", gated=True, fmt="int8")
    z = torch.randn(300_001, 16, device="cuda").bfloat16()
    a, rec = c.forward(z)
    da = torch.randn(300_001, 8, device="cuda").bfloat16()
    dz, again = c.backward(rec, da)
    g, u = kept(z[-2:, :8], "int8"), kept(z[-2:, 8:], "int8")
    ak, slope = act_and_slope(g, "silu")
    close(dz[-2:, :8], slope * u * da[-2:].double().cpu(), g, u * da[-2:].double().cpu(), "last rows")
    close(again[-2:], ak * u, g, u, "last rows")
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    rec2, a2, dz2 = c.new(300_001), torch.zeros_like(a), torch.zeros_like(z)
    with torch.cuda.graph(graph, stream=stream):
        c.forward(z, out=a2, ckpt=rec2)
        c.backward(rec2, da, out=dz2, again=False)
    z.copy_(z.flip(0))
    da.copy_(da.flip(0))
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(a2, a.flip(0)) and torch.equal(dz2, dz.flip(0))


def test_empty_batch_launches_nothing():
    c = binding.ActCheckpoint(64, act="gelu")
    before = binding.launch_count()
    a, rec = c.forward(torch.empty(0, 64, device="cuda"))
    dz, again = c.backward(rec, torch.empty(0, 64, device="cuda"))
    assert a.shape == dz.shape == again.shape == (0, 64) and rec.shape[0] == 0 and binding.launch_count() == before


def test_refusals_leave_the_outputs_alone():
    c, g = binding.ActCheckpoint(64, act="gelu"), binding.ActCheckpoint(64, act="silu", gated=True)
    x = torch.zeros(4, 64, device="cuda")
    rec = c.new(4)
    before = binding.launch_count()
    with pytest.raises(ValueError):
        c.forward(torch.zeros(4, 63, device="cuda"))
    with pytest.raises(ValueError):
        c.forward(torch.zeros(4, 64))                                  # not on the device
    with pytest.raises(ValueError):
        c.forward(torch.zeros(64, 4, device="cuda").t())
    with pytest.raises(KeyError):
        c.forward(torch.zeros(4, 64, device="cuda", dtype=torch.float16))
    with pytest.raises(ValueError):
        c.backward(rec, torch.zeros(5, 64, device="cuda"))
    with pytest.raises(ValueError):
        c.load(rec[:, :32])
    with pytest.raises(ValueError):
        g.forward(x)
    for call in (lambda: g.store(x), lambda: g.load(g.new(4))):        # one part only
        with pytest.raises((binding.AlgError, ValueError)):
            call()
    wide = torch.zeros(4, 129, device="cuda")
    with pytest.raises(binding.AlgError) as e:
        c.forward(wide[:, :64], out=wide[:, 32:96])                    # overlaps, but is not the same
    assert e.value.code == 1
    with pytest.raises(binding.AlgError):
        g.backward(g.new(4), wide[:, :64], out=wide[:, :128])
    assert binding.launch_count() == before
    c.forward(wide[:, :64], out=wide[:, 64:128])                       # column slices of one buffer do not overlap
    assert binding.launch_count() == before + 1


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_lower_tail_of_gelu_keeps_its_bits(dtype):
    """z Phi(z) and its slope down to -13, where Phi is 6e-39, to a bound that shrinks with them.

    fp32, in units of 2^-24 of the value: Phi(-u) = t P(t) exp(-u^2/2), t = 1 / (1 + 0.275 u): fit and evaluation 8, t off by 3 (a rounding and an
    approximate reciprocal of one unit in the last place) times 2.9 at most (the logarithmic slope of t P(t)), exp2 of two units in the last place 4, its argument
    0.72 u^2 off by three roundings: 3 u^2 / 2; products and sums 6.  Together less than 32 + 2 z^2, of Phi(z) + |z| phi(z) for the slope.  bf16: a fit to
    8.1e-4 of the value, 13 600 units (its exponent's own roundings among them), which is a fifth of half a step."""
    z = (torch.arange(-104, 104, dtype=torch.float64) / 8).view(-1, 16).repeat(1, 2)[:, :32].contiguous()     # int8 codes under a scale of 1/8
    z[:, 0] = z[:, 0].abs()
    z[:, 31] = 13.0                                                                                            # (every block has that scale)
    c = binding.ActCheckpoint(32, act="gelu", fmt="int8")
    a, rec = c.forward(z.to(DT[dtype]).cuda())
    assert torch.equal(c.load(rec, out_dtype=torch.float32).double().cpu(), z)
    dz, again = c.backward(rec, torch.ones_like(a))
    # (special.ndtr is a difference below -1, and 0 from -8.4 on)
    Phi, zphi = torch.erfc(-z * math.sqrt(0.5)) / 2, z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    rel = (32 + (13600 if dtype == "bf16" else 0) + 2 * z * z) * 2.0 ** -24
    half, least = torch.finfo(DT[dtype]).eps / 2, 16 * 2.0 ** -126
    for got, want, size in ((a, z * Phi, (z * Phi).abs()), (again, z * Phi, (z * Phi).abs()), (dz, Phi + zphi, Phi + zphi.abs())):
        off = (got.double().cpu() - want).abs() / (rel * size + half * want.abs() + least)
        assert float(off.max()) <= 1.0, (float(off.max()), float(z.flatten()[off.argmax()]))
