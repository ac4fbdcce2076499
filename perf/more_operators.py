"""The parts of a Sparse-BitNet training step around its layers and its head, for timing and comparing: the way in, the norms with their
gradients, and what makes new latent weights of the gradients.

A case is a dict of plain values.  Its "kind" says what one pass does:

kind        one pass
embed       the rows of a table that T tokens name, scaled
embed_grad  the gradient of the table; with "accumulate" added to one that is there (a table that is the head's matrix too)
norm        RMS or layer norm of T rows; with "residual" of their sum with other rows, which is given back
norm_grad   the gradients of rows, gain and (layer norm) bias; with "residual" the rows' own gradient is added
adamw       one AdamW step over many tensors, moments in 32 bits or in 8; with "clip" the norm of all gradients first, and gradients scaled by it

The sizes are those of the repository's benchmark (hidden 2560, FFN 6912, 16384 tokens, the matrices of a block) and generic vocabularies.
"""
import math

import torch

own = False

DEV = "cuda"
BF16, F32 = torch.bfloat16, torch.float32
BLOCK = [2560 * 2560] * 4 + [6912 * 2560] * 3   # the matrices of one block of the benchmark
BETA1, BETA2, EPS = 0.9, 0.95, 1e-8
NORM_EPS = 1e-6


def listed():
    return [
        # a decode batch looks its tokens up: latency only
        {"name": "embed_32_tokens", "kind": "embed", "tokens": 32, "d": 2560, "vocab": 131072, "dtype": "bf16", "left_out": 0.0},
        # the benchmark's training step, 8 sequences of 2048
        {"name": "embed_16384_tokens", "kind": "embed", "tokens": 16384, "d": 2560, "vocab": 131072, "dtype": "bf16", "left_out": 0.02},
        # fine-tuning with padded sequences, a table shared with the head; sizes that fit no vector
        {"name": "embed_grad_ragged", "kind": "embed_grad", "tokens": 1531, "d": 1001, "vocab": 50001, "dtype": "fp32", "left_out": 0.3, "accumulate": True},
        # the training step: 16384 of 131072 rows at most have a gradient, all are written
        {"name": "embed_grad_16384_tokens", "kind": "embed_grad", "tokens": 16384, "d": 2560, "vocab": 131072, "dtype": "bf16", "left_out": 0.02, "accumulate": False},
        # decode: one token between two layers
        {"name": "norm_1_token", "kind": "norm", "form": "rms", "tokens": 1, "d": 2560, "dtype": "bf16", "residual": True},
        # the training step, between two layers
        {"name": "norm_16384_tokens", "kind": "norm", "form": "layer", "tokens": 16384, "d": 2560, "dtype": "bf16", "residual": True},
        # a short odd sequence in 32 bits
        {"name": "norm_grad_ragged", "kind": "norm_grad", "form": "layer", "tokens": 1531, "d": 1001, "dtype": "fp32", "residual": False},
        # the training step's way back between two layers
        {"name": "norm_grad_16384_tokens", "kind": "norm_grad", "form": "rms", "tokens": 16384, "d": 2560, "dtype": "bf16", "residual": True},
        # the gains of 30 blocks' norms: many small tensors, latency only
        {"name": "adamw_gains", "kind": "adamw", "sizes": "61*2560", "dtype": "fp32", "grad": "fp32", "bits": 32, "clip": False, "stochastic": False},
        # odd tensors with moments in 8 bits
        {"name": "adamw8_ragged", "kind": "adamw", "sizes": "1*1,3*31,5*1000,2*1002001,1*2053", "dtype": "fp32", "grad": "bf16", "bits": 8, "clip": True, "stochastic": False},
        # the matrices of one block, moments in 32 bits
        {"name": "adamw_block", "kind": "adamw", "sizes": "block", "dtype": "bf16", "grad": "bf16", "bits": 32, "clip": True, "stochastic": True},
        # four blocks, moments in 8 bits: a model whose optimizer is to leave room for activations
        {"name": "adamw8_blocks", "kind": "adamw", "sizes": "4*block", "dtype": "bf16", "grad": "bf16", "bits": 8, "clip": True, "stochastic": True},
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["embed", "embed_grad", "embed_grad", "norm", "norm_grad", "norm_grad", "adamw", "adamw", "adamw"])
    dtype = rng.choice(["bf16", "bf16", "fp32"])
    if kind == "adamw":
        sizes, total = [], 0
        for _ in range(_log(rng, 1, 12)):
            many, size = _log(rng, 1, 40), _log(rng, 1, 20_000_000)
            if total + many * size <= 150_000_000:
                sizes.append(f"{many}*{size}")
                total += many * size
        return {"kind": kind, "sizes": ",".join(sizes or ["1*4097"]), "dtype": dtype, "grad": rng.choice(["bf16", "fp32"]), "bits": rng.choice([8, 32]),
                "clip": rng.random() < 0.5, "stochastic": rng.random() < 0.5}
    tokens, d = _log(rng, 1, 65536), _log(rng, 32, 8192)
    while tokens * d > 1 << 27:
        tokens, d = _log(rng, 1, 65536), _log(rng, 32, 8192)
    if rng.random() < 0.6:
        d = -(-d // 8) * 8   # most rows are whole vectors, some are odd
    case = {"kind": kind, "tokens": tokens, "d": d, "dtype": dtype}
    if kind in ("norm", "norm_grad"):
        return {**case, "form": rng.choice(["rms", "layer"]), "residual": rng.random() < 0.5}
    vocab = _log(rng, 300, 262144)
    while vocab * d > 1 << 29:
        vocab = _log(rng, 300, 262144)
    case = {**case, "vocab": vocab, "left_out": rng.choice([0.0, 0.02, 0.4])}
    return case if kind == "embed" else {**case, "accumulate": rng.random() < 0.4}


# ---- inputs ------------------------------------------------------------------------------------------------------------------------
def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def _randn(g, *shape, scale=1.0, dtype=BF16):
    return torch.randn(*shape, generator=g, device=DEV, dtype=F32).mul_(scale).to(dtype)


def _sizes(case):
    sizes = []
    for part in case["sizes"].split(","):
        many, _, size = part.rpartition("*")
        sizes += (BLOCK if size == "block" else [int(size)]) * int(many or 1)
    return sizes


def prepare(case, seed):
    g = _gen(seed)
    kind = case["kind"]
    s = {"kind": kind}
    if kind == "adamw":
        # every tensor of a group in one buffer, each from a place that is a multiple of 32
        sizes = _sizes(case)
        wide = [-(-n // 32) * 32 for n in sizes]
        first = [sum(wide[:i]) for i in range(len(wide))]
        total = sum(wide)
        real = torch.zeros(total, dtype=torch.bool, device=DEV)
        for n, at in zip(sizes, first):
            real[at:at + n] = True
        f32 = {"dtype": F32, "device": DEV}
        s.update(sizes=sizes, wide=wide, first=first, bits=case["bits"], clip=1.0 if case["clip"] else None, seed=seed * 2654435761 + 12345 if case["stochastic"] else None)
        s["p"] = (_randn(g, total, scale=0.02, dtype=F32) * real).to(BF16 if case["dtype"] == "bf16" else F32)
        s["g"] = (_randn(g, total, scale=1e-3, dtype=F32) * real).to(BF16 if case["grad"] == "bf16" else F32)
        m = _randn(g, total, scale=3e-4, dtype=F32) * real
        v = (_randn(g, total, scale=1e-3, dtype=F32) ** 2 * torch.rand(total, generator=g, device=DEV)) * real
        if case["bits"] == 32:
            s.update(m=m, v=v)
        else:
            s["m"], s["m_scales"] = _encode(m, 15, None)
            s["v"], s["v_scales"] = _encode(v, 31, None)
        s.update(lr=torch.full((1,), 3e-4, **f32), step=torch.full((1,), 10, dtype=torch.int64, device=DEV),
                 decay=[0.1 if n > 10000 else 0.0 for n in sizes])   # matrices decay, gains do not
        return s
    T, d, dtype = case["tokens"], case["d"], BF16 if case["dtype"] == "bf16" else F32
    if kind in ("embed", "embed_grad"):
        V = case["vocab"]
        ids = (torch.rand(T, generator=g, device=DEV) ** 3 * V).long().clamp_(max=V - 1)   # towards the frequent tokens
        ids[torch.rand(T, generator=g, device=DEV) < 0.04] = V // 7                          # and one that is everywhere
        ids[torch.rand(T, generator=g, device=DEV) < case["left_out"]] = -100
        s.update(ids=ids, scale=math.sqrt(d))
        if kind == "embed":
            s["E"] = _randn(g, V, d, scale=0.02, dtype=dtype)
        else:
            s.update(dY=_randn(g, T, d, scale=1e-3, dtype=dtype), vocab=V, dE=_randn(g, V, d, scale=1e-2, dtype=dtype) if case["accumulate"] else None)
        return s
    channels = torch.exp(_randn(g, d, scale=0.7, dtype=F32))   # some channels are larger, and they lie off zero
    X = (_randn(g, T, d, dtype=F32) + 0.3 * _randn(g, d, dtype=F32)) * channels
    s.update(layer=case["form"] == "layer", X=X.to(dtype), gain=1 + _randn(g, d, scale=0.2, dtype=F32), bias=None, other=None)
    if kind == "norm" and s["layer"]:
        s["bias"] = _randn(g, d, scale=0.1, dtype=F32)
    if kind == "norm_grad":
        s["dY"] = _randn(g, T, d, scale=1e-2, dtype=dtype)
    if case["residual"]:
        s["other"] = _randn(g, T, d, scale=1.0 if kind == "norm" else 1e-2, dtype=dtype)
    return s


# ---- plain forms -------------------------------------------------------------------------------------------------------------------
def _plain_embed(s):
    E, ids = s["E"], s["ids"]
    inside = (ids >= 0) & (ids < E.shape[0])
    rows = E[torch.where(inside, ids, 0)].float() * s["scale"]
    return torch.where(inside[:, None], rows, 0.0).to(E.dtype)


def _plain_embed_grad(s):
    dY, ids, V = s["dY"], s["ids"], s["vocab"]
    inside = (ids >= 0) & (ids < V)
    rows = torch.where(inside[:, None], dY.float(), 0.0)
    total = torch.zeros(V, dY.shape[1], device=DEV)
    total.index_add_(0, torch.where(inside, ids, 0), rows)
    total.mul_(s["scale"])
    if s["dE"] is None:
        return total.to(dY.dtype)
    return s["dE"].copy_(total.add_(s["dE"]))


def _statistics(x, layer):
    """Rows less their mean (RMS: as they are), and what they are multiplied with."""
    if layer:
        x = x - x.mean(1, keepdim=True)
    return x, torch.rsqrt(x.square().mean(1, keepdim=True) + NORM_EPS)


def _plain_norm(s):
    X, out = s["X"], {}
    if s["other"] is not None:
        X = out["sum"] = (X.float() + s["other"].float()).to(X.dtype)
    x, r = _statistics(X.float(), s["layer"])
    y = x * r * s["gain"]
    out["Y"] = (y if s["bias"] is None else y + s["bias"]).to(X.dtype)
    return out


def _plain_norm_grad(s):
    X, dy = s["X"], s["dY"].float()
    x, r = _statistics(X.float(), s["layer"])
    x = x * r
    a = dy * s["gain"]
    dx = a - x * (a * x).mean(1, keepdim=True)
    if s["layer"]:
        dx = dx - a.mean(1, keepdim=True)
    dx = dx * r
    if s["other"] is not None:
        dx = dx + s["other"].float()
    out = {"dX": dx.to(X.dtype), "dgain": (dy * x).sum(0)}
    if s["layer"]:
        out["dbias"] = dy.sum(0)
    return out


def _mix(x, key):
    """32 random bits of a 32-bit counter and two 32-bit keys."""
    x = x ^ key[0]
    x = (x ^ (x >> 16)) * 0x9E3779B1 & 0xFFFFFFFF
    x = (x ^ (x >> 15)) + key[1] & 0xFFFFFFFF
    x = x * 0x85A308D3 & 0xFFFFFFFF
    return x ^ (x >> 16)


def _tensor_of_blocks(s):
    """Which tensor every 32 values of the buffer belong to."""
    ends = torch.tensor(s["first"] + [sum(s["wide"])], device=DEV)[1:] // 32
    return torch.bucketize(torch.arange(sum(s["wide"]) // 32, device=DEV), ends, right=True)


def _noise(s):
    """16 random bits for the rounding of every weight, first and second moment of the buffer, from seed, step, tensor and place."""
    count = len(s["wide"])
    k0 = _mix(torch.full((count,), s["seed"] & 0xFFFFFFFF, device=DEV), ((s["seed"] >> 32) & 0xFFFFFFFF, 0))
    k0 = _mix(k0, (s["step"] & 0xFFFFFFFF, s["step"] >> 32 & 0xFFFFFFFF))
    k0 = _mix(k0, (torch.arange(count, device=DEV), 0))
    k1 = _mix(k0, (0x243F6A88, 0))
    which = _tensor_of_blocks(s)
    key = (k0[which, None], k1[which, None])
    block = torch.arange(len(which), device=DEV) - torch.tensor(s["first"], device=DEV)[which] // 32
    place = block[:, None] * 16 + torch.arange(16, device=DEV)
    bits = (_mix(3 * place, key), _mix(3 * place + 1, key), _mix(3 * place + 2, key))
    return tuple(torch.stack((b & 0xFFFF, b >> 16), 2).view(-1).int() for b in bits)


def _encode(x, below, noise):
    """Codes and block exponents of moments in 8 bits: 3 bits of mantissa, the exponent as far `below` the block's largest as there are codes."""
    bits = x.view(torch.int32)
    a = bits & 0x7FFFFFFF
    exponent = ((a.view(-1, 32).amax(1) + 0xFFFFF) >> 23).clamp_(min=below)
    half = 0x7FFFF + ((a >> 20) & 1) if noise is None else 16 * noise + 8
    code = (((a + half) >> 20).view(-1, 32) - (exponent - below)[:, None] * 8).view(-1)
    if below == 31:   # second moments: no sign, and what is not zero stays above it
        return torch.where(a > 0, code.clamp_(min=1), 0).to(torch.uint8), exponent.to(torch.uint8)
    return (code.clamp_(min=0) | (bits < 0).int() << 7).to(torch.uint8), exponent.to(torch.uint8)


def _values(codes, scales, below):
    code = codes.int()
    low = code if below == 31 else code & 127
    a = (low.view(-1, 32) + (scales.int() - below)[:, None] * 8).view(-1) << 20
    v = torch.where(low > 0, a, 0).view(F32)
    return v if below == 31 else torch.where(code > 127, -v, v)


def _plain_adamw(s):
    out = {}
    g, p = s["g"].float(), s["p"].float()
    if s["clip"] is not None:
        norm = g.double().square().sum().sqrt()
        factor = torch.where(norm.isfinite(), (s["clip"] / norm).clamp(max=1.0), math.nan).float()
        out["norm"] = torch.stack((norm.float(), factor))
        g = g * factor
    m, v = (s["m"], s["v"]) if s["bits"] == 32 else (_values(s["m"], s["m_scales"], 15), _values(s["v"], s["v_scales"], 31))
    m = m * BETA1 + g * (1 - BETA1)
    v = v * BETA2 + g * (1 - BETA2) * g
    t, lr = s["step"].double(), s["lr"].double()
    keep = (1 - lr * torch.tensor(s["decay"], dtype=torch.float64, device=DEV)).float()[_tensor_of_blocks(s), None]
    p = (p.view(-1, 32) * keep).view(-1) - m * (lr / (1 - BETA1 ** t)).float() / (torch.sqrt(v) * (1 / torch.sqrt(1 - BETA2 ** t)).float() + EPS)
    noise = _noise(s) if s["seed"] is not None else (None, None, None)
    if s["p"].dtype == BF16 and s["seed"] is not None:
        p = (p.view(torch.int32) + noise[0] & -65536).view(F32)
    s["p"].copy_(p)
    out["p"] = s["p"]
    if s["bits"] == 32:
        s["m"].copy_(m)
        s["v"].copy_(v)
        return {**out, "m": s["m"], "v": s["v"]}
    for name, x, below, bits in (("m", m, 15, noise[1]), ("v", v, 31, noise[2])):
        codes, scales = _encode(x, below, bits)
        s[name].copy_(codes)
        s[name + "_scales"].copy_(scales)
        out[name] = _values(codes, scales, below).to(BF16)   # exact in this type
    return out


def run(state):
    s = state
    if own:
        return _own(s)
    return {"embed": _plain_embed, "embed_grad": _plain_embed_grad, "norm": _plain_norm, "norm_grad": _plain_norm_grad, "adamw": _plain_adamw}[s["kind"]](s)


# ---- the framework's calls ---------------------------------------------------------------------------------------------------------
_kept = {}


def _workspace(sbn, nbytes):
    """One scratch buffer for the program, grown where a call needs more."""
    if "ws" not in _kept or _kept["ws"].numel() < nbytes:
        _kept["ws"] = None
        _kept["ws"] = sbn.new_workspace(nbytes, DEV)
    return _kept["ws"]


def _own(s):
    import paper_2603_05168_amd as sbn
    if s["kind"] == "adamw":
        return _own_adamw(sbn, s)
    if s["kind"] == "embed":
        E, ids = s["E"], s["ids"]
        Y = torch.empty(ids.shape[0], E.shape[1], dtype=E.dtype, device=DEV)
        sbn.sbn_embedding(E, ids, Y, scale=s["scale"])
        return Y
    if s["kind"] == "embed_grad":
        dY, V = s["dY"], s["vocab"]
        T, d = dY.shape
        dE = torch.empty(V, d, dtype=dY.dtype, device=DEV) if s["dE"] is None else s["dE"]
        sbn.sbn_embedding_backward(dY, s["ids"], dE, _workspace(sbn, sbn.sbn_embedding_workspace_bytes(T, d, V)), scale=s["scale"], accumulate=s["dE"] is not None)
        return dE
    X = s["X"]
    T, d = X.shape
    if s["kind"] == "norm":
        out = {"Y": torch.empty_like(X)}
        if s["other"] is not None:
            out["sum"] = torch.empty_like(X)
        sbn.sbn_norm(X, out["Y"], gain=s["gain"], bias=s["bias"], eps=NORM_EPS, layer=s["layer"], residual=s["other"], sum_out=out.get("sum"))
        return out
    out = {"dX": torch.empty_like(X), "dgain": torch.empty_like(s["gain"])}
    if s["layer"]:
        out["dbias"] = torch.empty_like(s["gain"])
    sbn.sbn_norm_backward(X, s["dY"], _workspace(sbn, sbn.sbn_norm_workspace_bytes(T, d)), gain=s["gain"], eps=NORM_EPS, layer=s["layer"], d_residual=s["other"], **out)
    return out


def _own_adamw(sbn, s):
    if "group" not in s:   # a program's lists of tensors, made once
        parts = lambda x, step=1: [x[at // step:at // step + -(-n // step)] for n, at in zip(s["sizes"], s["first"])]
        whole = lambda x: [x[at:at + n] for n, at in zip(s["wide"], s["first"])]
        grads = parts(s["g"])
        if s["bits"] == 32:
            states = {"m": parts(s["m"]), "v": parts(s["v"])}
        else:
            states = {"m": whole(s["m"]), "v": whole(s["v"]), "m_scales": parts(s["m_scales"], 32), "v_scales": parts(s["v_scales"], 32)}
        s["group"] = sbn.AdamWGroup(parts(s["p"]), grads, **states, weight_decay=s["decay"], betas=(BETA1, BETA2), eps=EPS)
        s["norms"] = sbn.GradNormGroup(grads, _workspace(sbn, sbn.sbn_grad_norm_workspace_bytes(s["sizes"]))) if s["clip"] is not None else None
    out = {}
    if s["clip"] is not None:
        out["norm"] = torch.empty(2, dtype=F32, device=DEV)
        s["norms"].run(s["clip"], out["norm"])
    s["group"].run(s["lr"], s["step"], clip=out["norm"][1:] if out else None, seed=s["seed"])
    out["p"] = s["p"]
    if s["bits"] == 32:
        return {**out, "m": s["m"], "v": s["v"]}
    for name in ("m", "v"):
        out[name] = torch.empty(s[name].shape, dtype=BF16, device=DEV)
        sbn.sbn_adamw_state_values(s[name], s[name + "_scales"], out[name], second=name == "v")
    return out


# ---- what a pass cannot do without, and its values in 64 bits ------------------------------------------------------------------------
def work(case):
    size = 2 if case["dtype"] == "bf16" else 4
    if case["kind"] == "adamw":
        n = sum(_sizes(case))
        grad = 2 if case["grad"] == "bf16" else 4
        if case["bits"] == 32:
            return {"bytes": n * (2 * size + grad + 16), "flops": 12 * n}
        return {"bytes": n * (2 * size + grad + 4 + 4 / 32 + 4), "flops": 30 * n}   # 8-bit moments in and out, and the values that they stand for
    T, d = case["tokens"], case["d"]
    if case["kind"] == "embed":
        return {"bytes": T * (2 * d * size + 8), "flops": T * d}
    if case["kind"] == "embed_grad":
        V = case["vocab"]
        often = T * 0.96 * (1 - case["left_out"]) * torch.linspace(0, 1, V + 1, dtype=torch.float64).pow(1 / 3).diff()
        named = float((1 - torch.exp(-often)).sum())   # rows that are expected to have a gradient: where it is added, the others stay as they are
        return {"bytes": T * (d * size + 8) + (2 * named if case["accumulate"] else V) * d * size, "flops": T * d}
    rows = 2 if case["kind"] == "norm" else 3
    if case["residual"]:
        rows += 2 if case["kind"] == "norm" else 1
    return {"bytes": rows * T * d * size + 12 * d, "flops": (8 if case["kind"] == "norm" else 16) * T * d}


def _exact_moment(x, below, noise):
    """What moments in 8 bits stand for: magnitudes on a grid of eight steps to the binade, those far below their block's largest zero (second
    moments: the smallest there is)."""
    a = x.abs()
    exponent = torch.frexp(a)[1] - 1
    unit = torch.exp2(exponent.double() - 3)
    near = torch.round(a / unit) if noise is None else torch.floor(a / unit + (noise.double() * 16 + 8) / 2 ** 20)
    near = torch.where(a > 0, near * unit, 0.0)
    top = a.view(-1, 32).amax(1)
    e = torch.frexp(top)[1] - 1
    e = torch.where(top > 1.875 * torch.exp2(e.double()), e + 1, e)   # where rounding may reach the next binade
    low = torch.exp2(torch.where(top > 0, e, 0).clamp(min=below - 127).double() - below).repeat_interleave(32)
    floor = 1.125 * low if below == 31 else torch.zeros_like(low)
    near = torch.where(near > low, near, torch.where(a > 0, floor, 0.0))
    return torch.where(x < 0, -near, near)


def _exact_adamw(s):
    g, p = s["g"].double(), s["p"].double()
    out = {}
    if s["clip"] is not None:
        norm = torch.linalg.vector_norm(g)
        factor = min(1.0, s["clip"] / float(norm))
        out["norm"] = torch.tensor([float(norm), factor], dtype=torch.float64, device=DEV)
        g *= factor
    if s["bits"] == 32:
        m, v = s["m"].double(), s["v"].double()
    else:
        m, v = _values(s["m"], s["m_scales"], 15).double(), _values(s["v"], s["v_scales"], 31).double()
    m = m + (1 - BETA1) * (g - m)
    v = v + (1 - BETA2) * (g * g - v)
    t, lr = int(s["step"]), float(s["lr"])
    p -= lr * (m / (1 - BETA1 ** t)) / ((v / (1 - BETA2 ** t)).sqrt() + EPS)
    for n, at, decay in zip(s["wide"], s["first"], s["decay"]):
        p[at:at + n] -= lr * decay * s["p"][at:at + n].double()
    noise = _noise(s) if s["seed"] is not None else (None, None, None)
    if s["seed"] is not None and s["p"].dtype == BF16:
        unit = torch.exp2(torch.frexp(p)[1].double() - 8)
        p = torch.sign(p) * torch.floor(p.abs() / unit + noise[0].double() / 65536) * unit
    out["p"] = p
    if s["bits"] == 8:
        m, v = _exact_moment(m, 15, noise[1]), _exact_moment(v, 31, noise[2])
    return {**out, "m": m, "v": v}


def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind == "adamw":
        return _exact_adamw(s)
    if kind == "embed":
        table = torch.cat((s["E"], torch.zeros_like(s["E"][:1])))   # one row more, for tokens that are left out
        return table[s["ids"].clamp(min=-1)].double() * s["scale"]
    if kind == "embed_grad":
        T, V = case["tokens"], case["vocab"]
        order = torch.argsort(s["ids"], stable=True)
        ids, rows = s["ids"][order], s["dY"][order].double()
        rows, ids = rows[ids >= 0], ids[ids >= 0]
        names, counts = torch.unique_consecutive(ids, return_counts=True)
        ends = counts.cumsum(0)
        sums = torch.cat((torch.zeros_like(rows[:1]), rows.cumsum(0))) if len(rows) else rows
        out = torch.zeros(V, case["d"], dtype=torch.float64, device=DEV)
        if len(rows):
            out[names] = (sums[ends] - sums[ends - counts]) * s["scale"]
        return out if s["dE"] is None else out + s["dE"].double()
    X, gain, d = s["X"].double(), s["gain"].double(), case["d"]
    if kind == "norm":
        out = {}
        if s["other"] is not None:
            out["sum"] = X + s["other"].double()
            X = out["sum"].to(s["X"].dtype).double()
        var, mu = torch.var_mean(X, 1, correction=0, keepdim=True)
        if not s["layer"]:
            var, mu = var + mu * mu, 0.0
        Y = (X - mu) / torch.sqrt(var + NORM_EPS) * gain
        out["Y"] = Y if s["bias"] is None else Y + s["bias"].double()
        return out
    dY = s["dY"].double()
    mu = X.mean(1, keepdim=True) if s["layer"] else torch.zeros(1, 1, dtype=torch.float64, device=DEV)
    std = torch.sqrt(((X - mu) ** 2).mean(1, keepdim=True) + NORM_EPS)
    h = (X - mu) / std
    a = dY * gain
    dX = (a - (a.mean(1, keepdim=True) if s["layer"] else 0.0) - h * ((a * h).sum(1, keepdim=True) / d)) / std
    out = {"dX": dX if s["other"] is None else dX + s["other"].double(), "dgain": torch.einsum("td,td->d", dY, h)}
    if s["layer"]:
        out["dbias"] = dY.sum(0)
    return out
