"""What stands around the projections of a feed-forward block, as a program that trains or serves one has it computed.

    join       one call at a block's border: the block's output F, normed, scaled and gated, is added to the residual stream R,
               and the sum is normed for the next block:  Y = R + alpha * scale * gate * norm(F),  N = norm(Y)
    join_grad  the gradients of that call with respect to everything it read
    act        the activation between the up and the down projection in a training step: the forward pass writes the activation
               and an 8-bit checkpoint of its input, the backward pass has the gradient of the input, and the activation once
               more for the weight gradient, from the checkpoint alone
    ckpt       any other activation kept for the backward pass in 8 bits: stored and read back
    moe        one mixture-of-experts layer on a few tokens: router, top-k, gated expert FFNs, weighted sum

Sizes are those of the feed-forward layers this library is timed on (512 to 7168 wide), with odd ones among them; activations are
N(0, 1) with a few larger features, as residual streams have them, weights N(0, 0.02^2).  ``run`` computes the plain forms in
elementary torch operations where ``own`` is false, and calls ``paper_2609_32814_b200.binding`` where it is true.
"""
import math

import torch

own = False

EPS = 1e-6
BLOCK = 32          # columns that share a scale in a checkpoint
TOP = {"e4m3": 448.0, "int8": 127.0}


# ---- cases ------------------------------------------------------------------------------------------------------------

def _join(use, m, d, *, kind="rms", gate="none", sigmoid=False, post=True, pre=True, scale=True, dtype="bf16", stream="bf16"):
    return {"use": use, "m": m, "d": d, "kind": kind, "gate": gate, "sigmoid": sigmoid, "post": post, "pre": pre, "scale": scale,
            "dtype": dtype, "stream": stream}


def _act(m, f, *, act="gelu", gated=False, fmt="e4m3", dtype="bf16"):
    return {"use": "act", "m": m, "f": f, "act": act, "gated": gated, "fmt": fmt, "dtype": dtype}


def _ckpt(m, d, *, fmt="e4m3", dtype="bf16"):
    return {"use": "ckpt", "m": m, "d": d, "fmt": fmt, "dtype": dtype}


def _moe(m, d, f, experts, k, *, score="softmax", renormalise=True, bias=False, out="bf16"):
    return {"use": "moe", "m": m, "d": d, "f": f, "experts": experts, "k": k, "score": score, "renormalise": renormalise, "bias": bias,
            "out": out}


def listed():
    named = {
        # one token of one user at a block's border: the latency of a call
        "join_m1": _join("join", 1, 2048),
        # a prompt of odd length: LayerNorm, a gate for each token, the residual stream in 32 bits
        "join_ragged": _join("join", 1777, 768, kind="layer", gate="row", stream="f32"),
        # prefill or the forward half of training: sandwich norms with a learned gate for each feature
        "join_large": _join("join", 32768, 4096, gate="element", sigmoid=True),
        # the backward half for packed sequences (a batch that is no multiple of anything)
        "join_grad": _join("join_grad", 8003, 1024, gate="row"),
        # the same, wide, with everything a block border can have
        "join_grad_wide": _join("join_grad", 16384, 4096, kind="layer", gate="element", sigmoid=True, stream="f32"),
        # a GELU layer on packed sequences, kept as 8-bit integers
        "act_gelu": _act(8003, 4096, fmt="int8"),
        # SwiGLU of a wide layer, kept as e4m3
        "act_swiglu": _act(16384, 6144, act="silu", gated=True),
        # the input of a narrow layer kept for its weight gradient; 1000 columns end inside a block
        "ckpt_small": _ckpt(517, 1000, fmt="int8"),
        # the residual stream of a wide layer in 32 bits
        "ckpt_large": _ckpt(16384, 7168, dtype="f32"),
        # one token through 128 narrow experts, eight of them chosen
        "moe_m1": _moe(1, 2048, 768, 128, 8),
        # a batch of users through the same layer: nearly every expert has a token or a few
        "moe_m40": _moe(40, 2048, 768, 128, 8),
        # wide experts, sigmoid scores with a selection bias, an odd number of tokens, 32-bit results
        "moe_wide": _moe(5, 4096, 1536, 64, 6, score="sigmoid", bias=True, out="f32"),
    }
    return [dict(case, name=name) for name, case in named.items()]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, lo, hi):
    d = _log(rng, lo, hi)
    return d if rng.random() < 0.25 else max(8, d // 64 * 64 if d >= 512 else d // 8 * 8)


def draw(rng):
    use = rng.choice(("join", "join", "join_grad", "join_grad", "act", "act", "ckpt", "moe", "moe"))
    if use in ("join", "join_grad"):
        d = _width(rng, 128, 8192)
        m = _log(rng, 1, min(32768, (1 << 26) // d))
        post, pre = rng.choice(((True, True), (True, True), (False, True), (True, False)))
        return _join(use, m, d, kind=rng.choice(("rms", "rms", "layer")), gate=rng.choice(("none", "row", "element")),
                     sigmoid=rng.random() < 0.5, post=post, pre=pre, scale=rng.random() < 0.7, dtype=rng.choice(("bf16", "bf16", "f32")),
                     stream=rng.choice(("bf16", "f32")))
    if use == "act":
        f = _width(rng, 128, 16384)
        act, gated = rng.choice((("gelu", False), ("gelu_tanh", False), ("silu", True), ("silu", True), ("gelu", True)))
        return _act(_log(rng, 1, min(32768, (1 << 26) // f)), f, act=act, gated=gated, fmt=rng.choice(("e4m3", "int8")),
                    dtype=rng.choice(("bf16", "bf16", "f32")))
    if use == "ckpt":
        d = _width(rng, 64, 8192)
        return _ckpt(_log(rng, 1, min(32768, (1 << 26) // d)), d, fmt=rng.choice(("e4m3", "int8")), dtype=rng.choice(("bf16", "f32")))
    d, f = 8 * _log(rng, 64, 512), 8 * _log(rng, 32, 256)
    experts = min(_log(rng, 4, 128), (1 << 30) // (3 * d * f))
    return _moe(_log(rng, 1, 64), d, f, experts, rng.randint(1, min(8, experts)), score=rng.choice(("softmax", "sigmoid")),
                renormalise=rng.random() < 0.7, bias=rng.random() < 0.5, out=rng.choice(("bf16", "f32")))


# ---- inputs -----------------------------------------------------------------------------------------------------------

_DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def _normal(gen, shape, dtype, std=1.0, mean=0.0):
    return (torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32) * std + mean).to(dtype)


def _features(gen, m, d, dtype):
    """N(0, 1) with one feature in about a hundred ten times as large."""
    size = torch.where(torch.rand((d,), generator=gen, device="cuda") < 0.01, 10.0, 1.0)
    return (torch.randn((m, d), generator=gen, device="cuda", dtype=torch.float32) * size).to(dtype)


def prepare(case, seed):
    c = dict(case)
    gen = torch.Generator(device="cuda").manual_seed(seed)
    s = {"case": c}
    if c["use"] in ("join", "join_grad"):
        m, d = c["m"], c["d"]
        dt, st = _DT[c["dtype"]], _DT[c["stream"]]
        s["R"], s["F"] = _features(gen, m, d, st), _normal(gen, (m, d), dt)
        s["gate"] = None if c["gate"] == "none" else _normal(gen, (m,) if c["gate"] == "row" else (m, d), dt)
        layer = c["kind"] == "layer"
        vector = lambda on, mean: _normal(gen, (d,), torch.float32, 0.1, mean) if on else None  # noqa: E731
        s["post_weight"], s["post_bias"] = vector(c["post"], 1.0), vector(c["post"] and layer, 0.0)
        s["pre_weight"], s["pre_bias"] = vector(c["pre"], 1.0), vector(c["pre"] and layer, 0.0)
        s["scale"], s["alpha"] = vector(c["scale"], 0.5), 0.5
        if c["use"] == "join_grad":
            # what the forward pass left, and the gradients that arrive
            s["Y"] = _plain_join(s)[0].to(st)
            s["dY"] = _normal(gen, (m, d), st)
            s["dN"] = _normal(gen, (m, d), dt) if c["pre"] else None
        if own:
            from paper_2609_32814_b200 import binding
            s["norm"] = binding.BlockNorm(d, kind=c["kind"], join=True, post=c["post"], pre=c["pre"],
                                          gate=None if c["gate"] == "none" else c["gate"],
                                          gate_act="sigmoid" if c["sigmoid"] and c["gate"] != "none" else None, eps=EPS, dtype=c["dtype"], stream_dtype=c["stream"])
        return s
    if c["use"] in ("act", "ckpt"):
        m, n = c["m"], c["d"] if c["use"] == "ckpt" else c["f"] * (2 if c["gated"] else 1)
        s["X"] = _features(gen, m, n, _DT[c["dtype"]])
        if c["use"] == "act":
            s["dA"] = _normal(gen, (m, c["f"]), _DT[c["dtype"]])
        if own:
            from paper_2609_32814_b200 import binding
            if c["use"] == "act":
                s["checkpoint"] = binding.ActCheckpoint(c["f"], act=c["act"], gated=c["gated"], fmt=c["fmt"])
            else:
                s["checkpoint"] = binding.ActCheckpoint(c["d"], fmt=c["fmt"])
        return s
    m, d, f, e = c["m"], c["d"], c["f"], c["experts"]
    s["X"] = _normal(gen, (m, d), torch.bfloat16)
    s["W_router"] = _normal(gen, (d, e), torch.bfloat16, 1.0 / math.sqrt(d))
    s["select_bias"] = _normal(gen, (e,), torch.float32, 0.1) if c["bias"] else None
    s["W_gate_up"] = torch.randn((e, d, 2 * f), generator=gen, device="cuda", dtype=torch.bfloat16).mul_(0.02)
    s["W_down"] = torch.randn((e, f, d), generator=gen, device="cuda", dtype=torch.bfloat16).mul_(0.02)
    if own:
        from paper_2609_32814_b200 import binding
        s["moe"] = binding.MoE(d, f, e, c["k"], score=c["score"], renormalise=c["renormalise"])
    return s


# ---- the plain forms --------------------------------------------------------------------------------------------------

def _normed(x, layer):
    """(x - mean) / sqrt(var + eps), or x / sqrt(mean square + eps); and the factor."""
    if layer:
        x = x - x.mean(1, keepdim=True)
    r = torch.rsqrt((x * x).mean(1, keepdim=True) + EPS)
    return x * r, r


def _gate(s):
    """(gate, its derivative) as columns or matrices, 1 without one."""
    if s["gate"] is None:
        return 1.0, 0.0
    g = s["gate"].float()
    g = g[:, None] if g.dim() == 1 else g
    if not s["case"]["sigmoid"]:
        return g, 1.0
    g = 1 / (1 + torch.exp(-g))
    return g, g * (1 - g)


def _branch(s):
    """What the gate multiplies, without scale: norm(F) * weight + bias, or F; and the norm's pieces."""
    v, r = _normed(s["F"].float(), s["case"]["kind"] == "layer") if s["case"]["post"] else (s["F"].float(), None)
    n = v
    if s["post_weight"] is not None:
        n = n * s["post_weight"]
    if s["post_bias"] is not None:
        n = n + s["post_bias"]
    return n, v, r


def _plain_join(s):
    c = s["case"]
    n = _branch(s)[0]
    if s["scale"] is not None:
        n = n * s["scale"]
    y = s["R"].float() + s["alpha"] * _gate(s)[0] * n
    if not c["pre"]:
        return y, None
    out = _normed(y, c["kind"] == "layer")[0] * s["pre_weight"]
    return y, out if s["pre_bias"] is None else out + s["pre_bias"]


def _norm_grad(v, r, h, layer):
    """Gradient through v = (x - mean) r for the gradient h of v."""
    g = h - v * (h * v).mean(1, keepdim=True)
    return r * (g - h.mean(1, keepdim=True) if layer else g)


def _plain_join_grad(s):
    c, st, dt = s["case"], s["R"].dtype, s["F"].dtype
    layer = c["kind"] == "layer"
    t = s["dY"].float()
    out = {}
    if c["pre"]:
        dn = s["dN"].float()
        v, r = _normed(s["Y"].float(), layer)
        t = t + _norm_grad(v, r, dn * s["pre_weight"], layer)
        out["pre_weight"] = (dn * v).sum(0)
        if s["pre_bias"] is not None:
            out["pre_bias"] = dn.sum(0)
    out["R"] = t.to(st)
    n, v, r = _branch(s)
    g, dg = _gate(s)
    scale = 1.0 if s["scale"] is None else s["scale"]
    a = s["alpha"] * t
    e = a * scale * g
    if s["gate"] is not None:
        k = a * scale * n * dg
        out["gate"] = (k.sum(1) if c["gate"] == "row" else k).to(dt)
    if s["scale"] is not None:
        out["scale"] = (a * g * n).sum(0)
    if c["post"]:
        out["post_weight"] = (e * v).sum(0)
        if s["post_bias"] is not None:
            out["post_bias"] = e.sum(0)
        e = _norm_grad(v, r, e * s["post_weight"], layer)
    out["F"] = e.to(dt)
    return out


def _kept(x, fmt):
    """The values that 8-bit codes with a power-of-two scale for every 32 columns stand for, in 32 bits."""
    m, n = x.shape
    b = torch.nn.functional.pad(x.float(), (0, -n % BLOCK)).view(m, -1, BLOCK)
    mant, ex = torch.frexp(b.abs().amax(2, keepdim=True))
    top, tex = math.frexp(TOP[fmt])
    ex = (ex - tex + (mant > top)).clamp(min=-120)
    code = torch.ldexp(b, -ex)
    code = code.to(torch.float8_e4m3fn).float() if fmt == "e4m3" else torch.round(code)
    return torch.ldexp(code, ex).view(m, -1)[:, :n]


def _act_and_slope(z, act):
    if act == "silu":
        p = 1 / (1 + torch.exp(-z))
        return z * p, p * (1 + z * (1 - p))
    if act == "gelu":
        p = 0.5 * (1 + torch.erf(z * math.sqrt(0.5)))
        return z * p, p + z * torch.exp(-0.5 * z * z) * (1 / math.sqrt(2 * math.pi))
    k = math.sqrt(2 / math.pi)
    t = torch.tanh(k * (z + 0.044715 * z * z * z))
    return 0.5 * z * (1 + t), 0.5 * (1 + t) + 0.5 * z * (1 - t * t) * k * (1 + 3 * 0.044715 * z * z)


def _plain_act(s):
    c, dt = s["case"], s["X"].dtype
    f = c["f"]
    z, da = s["X"].float(), s["dA"].float()
    if not c["gated"]:
        zk = _kept(s["X"], c["fmt"])
        again, slope = _act_and_slope(zk, c["act"])
        return {"A": _act_and_slope(z, c["act"])[0].to(dt), "dZ": (da * slope).to(dt), "again": again.to(dt)}
    g, u = _kept(s["X"][:, :f], c["fmt"]), _kept(s["X"][:, f:], c["fmt"])
    again, slope = _act_and_slope(g, c["act"])
    return {"A": (_act_and_slope(z[:, :f], c["act"])[0] * z[:, f:]).to(dt),
            "dZ": torch.cat((da * u * slope, da * again), 1).to(dt), "again": (again * u).to(dt)}


def _plain_moe(s):
    c = s["case"]
    # (scores in 64 bits: which experts are chosen hangs on their order)
    logits = s["X"].double() @ s["W_router"].double()
    if c["score"] == "softmax":
        p = torch.exp(logits - logits.amax(1, keepdim=True))
        p = p / p.sum(1, keepdim=True)
    else:
        p = 1 / (1 + torch.exp(-logits))
    by = p if s["select_bias"] is None else p + s["select_bias"].double()
    idx = torch.sort(by, dim=1, descending=True, stable=True)[1][:, :c["k"]]
    w = torch.gather(p, 1, idx)
    if c["renormalise"]:
        w = w / w.sum(1, keepdim=True)
    w = w.float()
    rows = []
    for m in range(c["m"]):
        x = s["X"][m].float()
        gu = (x[None, :, None] * s["W_gate_up"][idx[m]].float()).sum(1) if c["m"] == 1 else torch.einsum("d,kdf->kf", x, s["W_gate_up"][idx[m]].float())
        g, u = gu[:, :c["f"]], gu[:, c["f"]:]
        h = g / (1 + torch.exp(-g)) * u * w[m][:, None]
        rows.append(torch.einsum("kf,kfd->d", h, s["W_down"][idx[m]].float()))
    return {"Y": torch.stack(rows).to(_DT[c["out"]]), "experts": idx.to(torch.int32), "weights": w}


# ---- one pass ---------------------------------------------------------------------------------------------------------

_JOIN = ("F", "gate", "post_weight", "post_bias", "scale", "alpha", "pre_weight", "pre_bias")


def run(s):
    c = s["case"]
    use = c["use"]
    if not own:
        if use == "join":
            y, n = _plain_join(s)
            return {"Y": y.to(s["R"].dtype), "N": None if n is None else n.to(s["F"].dtype)}
        if use == "join_grad":
            return _plain_join_grad(s)
        if use == "act":
            return _plain_act(s)
        if use == "ckpt":
            return _kept(s["X"], c["fmt"]).to(s["X"].dtype)
        return _plain_moe(s)
    if use == "join":
        y, n = s["norm"].forward(s["R"], **{k: s[k] for k in _JOIN})
        return {"Y": y, "N": n}
    if use == "join_grad":
        return s["norm"].backward(s["Y"], dY=s["dY"], dN=s["dN"], **{k: s[k] for k in _JOIN})
    if use == "act":
        a, kept = s["checkpoint"].forward(s["X"])
        dz, again = s["checkpoint"].backward(kept, s["dA"])
        return {"A": a, "dZ": dz, "again": again}
    if use == "ckpt":
        kept = s["checkpoint"].store(s["X"])
        return s["checkpoint"].load(kept, out_dtype=s["X"].dtype)
    y, experts, weights = s["moe"].forward(s["X"], s["W_router"], s["W_gate_up"], s["W_down"], select_bias=s["select_bias"],
                                           out_dtype=_DT[c["out"]], routing=True)
    return {"Y": y, "experts": experts, "weights": weights}


def work(case):
    c = case
    use, m = c["use"], c["m"]
    size = lambda t: 4 if t == "f32" else 2  # noqa: E731
    if use in ("join", "join_grad"):
        d, b, st = c["d"], size(c["dtype"]), size(c["stream"])
        gate = {"none": 0, "row": m, "element": m * d}[c["gate"]]
        vectors = 4 * d * ((c["post"] + c["pre"]) * (2 if c["kind"] == "layer" else 1) + c["scale"])
        if use == "join":   # R, F, gate in; Y, N out
            return {"bytes": m * d * (2 * st + b * (2 if c["pre"] else 1)) + b * gate + vectors, "flops": 16 * m * d}
        # Y, dY, dN, F, gate in; dR, dF, dgate out
        return {"bytes": m * d * (st * (3 if c["pre"] else 2) + b * (3 if c["pre"] else 2)) + 2 * b * gate + 2 * vectors, "flops": 40 * m * d}
    if use == "act":
        f, b, parts = c["f"], size(c["dtype"]), 2 if c["gated"] else 1
        kept = m * parts * (f + -(-f // BLOCK))
        # Z in, A and the checkpoint out; the checkpoint and dA in, dZ and A out
        return {"bytes": m * f * b * (2 * parts + 3) + 2 * kept, "flops": 60 * m * f}
    if use == "ckpt":
        d, b = c["d"], size(c["dtype"])
        return {"bytes": 2 * m * d * b + 2 * m * (d + -(-d // BLOCK)), "flops": 6 * m * d}
    d, f, e, k = c["d"], c["f"], c["experts"], c["k"]
    used = e * (1 - (1 - k / e) ** m)   # experts that some token chooses, were the choices uniform
    return {"bytes": 2 * (d * e + used * 3 * d * f + m * d) + size(c["out"]) * m * d + 8 * m * k, "flops": 2 * m * (d * e + 3 * k * d * f)}


# ---- the same from the definitions, in 64 bits --------------------------------------------------------------------------

def _exact_norm(x, kind, weight, bias):
    """One norm as its definition has it."""
    mu = torch.mean(x, dim=1, keepdim=True) if kind == "layer" else torch.zeros((x.shape[0], 1), dtype=x.dtype, device=x.device)
    z = (x - mu) / torch.sqrt(torch.mean((x - mu) ** 2, dim=1, keepdim=True) + EPS)
    return z if weight is None else z * weight + (0.0 if bias is None else bias)


def _exact_border(s, v):
    """(Y, N) of a block's border from values in 64 bits."""
    c = s["case"]
    branch = _exact_norm(v["F"], c["kind"], v["post_weight"], v["post_bias"]) if c["post"] else v["F"]
    for name in ("scale", "gate"):
        if v[name] is not None:
            f = torch.sigmoid(v[name]) if name == "gate" and c["sigmoid"] else v[name]
            branch = branch * (f.unsqueeze(1) if name == "gate" and f.dim() == 1 else f)
    y = v["R"] + s["alpha"] * branch
    return y, _exact_norm(y, c["kind"], v["pre_weight"], v["pre_bias"]) if c["pre"] else None


def _exact_code(x, fmt):
    """Codes of one format with the smallest power-of-two scale that holds each block, and the values they stand for."""
    m, n = x.shape
    blocks = -(-n // BLOCK)
    full = torch.zeros((m, blocks * BLOCK), dtype=torch.float64, device=x.device)
    full[:, :n] = x
    full = full.reshape(m, blocks, BLOCK)
    largest = full.abs().max(dim=2, keepdim=True).values
    scale = torch.exp2(torch.ceil(torch.log2(largest / TOP[fmt])).clamp(min=-120.0).nan_to_num(neginf=-120.0))
    scale = torch.where(largest > TOP[fmt] * scale, 2 * scale, torch.where((largest <= TOP[fmt] * scale / 2) & (scale > 2.0 ** -120), scale / 2, scale))
    q = full / scale
    if fmt == "int8":
        q = torch.round(q)
    else:   # three bits behind the leading one, the smallest exponent is -6
        step = torch.exp2(torch.floor(torch.log2(q.abs().clamp(min=2.0 ** -6))) - 3)
        q = torch.round(q / step) * step
    return (q * scale).reshape(m, -1)[:, :n]


def _exact_act(z, act):
    """Activation and its derivative, by autograd of the definition."""
    z = z.detach().requires_grad_(True)
    if act == "gelu":
        a = z * torch.special.ndtr(z)
    elif act == "gelu_tanh":
        a = z / 2 * (1 + torch.tanh((2 / math.pi) ** 0.5 * (z + 0.044715 * z ** 3)))
    else:
        a = z * torch.sigmoid(z)
    slope, = torch.autograd.grad(a.sum(), z)
    return a.detach(), slope


def exact(case, seed):
    global own
    was, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = was
    c = s["case"]
    use = c["use"]
    wide = lambda t: t.double() if isinstance(t, torch.Tensor) else t  # noqa: E731
    if use == "join":
        y, n = _exact_border(s, {k: wide(v) for k, v in s.items()})
        return {"Y": y, "N": n}
    if use == "join_grad":
        # the forward pass's Y is an input here: the norm behind it takes its gradient there, the branch takes what arrives at Y
        out, rows, parts = {}, c["m"], []
        each = max(1, min(rows, (1 << 24) // c["d"]))
        names = ["F", "gate", "post_weight", "post_bias", "scale", "pre_weight", "pre_bias"]
        for at in range(0, rows, each):
            cut = lambda t: t[at:at + each] if t.dim() and t.shape[0] == rows and t is not None else t  # noqa: E731, B023
            v = {k: None if s[k] is None else (wide(s[k][at:at + each]) if k in ("F", "gate") else wide(s[k])).requires_grad_(True) for k in names}
            y = wide(cut(s["Y"])).requires_grad_(True)
            t = wide(cut(s["dY"]))
            grads = {}
            if c["pre"]:
                pre = [("y", y)] + [(k, v[k]) for k in ("pre_weight", "pre_bias") if v[k] is not None]
                got = torch.autograd.grad(_exact_norm(y, c["kind"], v["pre_weight"], v["pre_bias"]), [x for _, x in pre], wide(cut(s["dN"])))
                grads = dict(zip([k for k, _ in pre], got))
                t = t + grads.pop("y")
            grads["R"] = t
            rest = [(k, v[k]) for k in names[:5] if v[k] is not None]
            zero = dict(v, R=torch.zeros_like(t))
            plain = dict(s, case=dict(c, pre=False))
            grads.update(zip([k for k, _ in rest], torch.autograd.grad(_exact_border(plain, zero)[0], [x for _, x in rest], t)))
            parts.append(grads)
        for k in parts[0]:
            got = [p[k] for p in parts]
            out[k] = torch.cat(got) if k in ("R", "F", "gate") else torch.stack(got).sum(0)
        return out
    if use == "ckpt":
        return _exact_code(wide(s["X"]), c["fmt"])
    if use == "act":
        f, x, da = c["f"], wide(s["X"]), wide(s["dA"])
        if not c["gated"]:
            again, slope = _exact_act(_exact_code(x, c["fmt"]), c["act"])
            return {"A": _exact_act(x, c["act"])[0], "dZ": da * slope, "again": again}
        g, u = _exact_code(x[:, :f], c["fmt"]), _exact_code(x[:, f:], c["fmt"])
        again, slope = _exact_act(g, c["act"])
        return {"A": _exact_act(x[:, :f], c["act"])[0] * x[:, f:], "dZ": torch.hstack((slope * u * da, again * da)), "again": again * u}
    # moe: expert by expert
    x, w = wide(s["X"]), wide(s["W_router"])
    score = torch.softmax(x @ w, dim=1) if c["score"] == "softmax" else torch.sigmoid(x @ w)
    order = (score if s["select_bias"] is None else score + wide(s["select_bias"])).argsort(dim=1, descending=True, stable=True)[:, :c["k"]]
    share = torch.zeros_like(score).scatter_(1, order, score.gather(1, order))
    if c["renormalise"]:
        share = share / share.sum(dim=1, keepdim=True)
    y = torch.zeros_like(x)
    for e in torch.unique(order).tolist():
        here = share[:, e].nonzero().flatten()
        pre = x[here] @ wide(s["W_gate_up"][e])
        y[here] += share[here, e].unsqueeze(1) * ((torch.nn.functional.silu(pre[:, :c["f"]]) * pre[:, c["f"]:]) @ wide(s["W_down"][e]))
    return {"Y": y, "experts": None, "weights": share.gather(1, order)}
