"""The norm of gradients and AdamW on the GPU.

Moments: every operation is one fp32 operation, so fp32 moments and the codes of 8-bit ones are equal to the same arithmetic on the CPU; against 64 bits an
fp32 moment is off by at most 4 steps of 2^-24 of its terms (two rounded constants, two products, a sum).
Weights: p keep - rate m / (sqrt(v) of_v + eps): keep, rate and of_v are rounded from 64 bits, and each operation rounds or is off by a step: 3 2^-24 |p|
and 16 2^-24 of the update (a root and a quotient of a step or two each), and what the moments are off by (8 2^-24 at most); bf16 then rounds by half a step."""
import numpy as np
import pytest
import torch

from gpu_util import DEV, sbn

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
BF16, F32 = torch.bfloat16, torch.float32
B1, B2, EPS = 0.9, 0.95, 1e-8


# ---- the definition on the CPU ------------------------------------------------------------------------------------------------------
def mix(x, k0, k1):
    x = x ^ k0
    x = ((x ^ (x >> 16)) * 0x9E3779B1) & 0xffffffff
    x = ((x ^ (x >> 15)) + k1) & 0xffffffff
    x = (x * 0x85A308D3) & 0xffffffff
    return x ^ (x >> 16)


def noise(n, seed, step, place):
    """16 bits for every p, m and v of a tensor."""
    u64 = lambda v: np.array([v], dtype=np.uint64)   # noqa: E731
    with np.errstate(over="ignore"):
        k0 = mix(u64(seed & 0xffffffff), u64(seed >> 32), u64(0))
        k0 = mix(k0, u64(step & 0xffffffff), u64(step >> 32))
        k0 = mix(k0, u64(place), u64(0))
        k1 = mix(k0, u64(0x243F6A88), u64(0))
        pair = np.arange((n + 1) // 2, dtype=np.uint64)
        bits = [mix(3 * pair + np.uint64(j), k0, k1) for j in range(3)]
    return [np.stack((b & 0xffff, b >> 16), 1).reshape(-1)[:n].astype(np.int64) for b in bits]


def encode(x, below, bits):
    """Codes and exponents of fp32 moments; bits None: to nearest."""
    n = len(x)
    pattern = np.zeros(-(-n // 32) * 32, dtype=np.int64)
    pattern[:n] = x.view(np.uint32)
    a = pattern & 0x7fffffff
    exponent = np.maximum((a.reshape(-1, 32).max(1) + 0xfffff) >> 23, below)
    half = np.zeros_like(a)
    half[:n] = 0x7ffff + ((a[:n] >> 20) & 1) if bits is None else 16 * bits + 8
    code = ((a + half) >> 20) - np.repeat(exponent - below, 32) * 8
    code = np.where(a > 0, np.maximum(code, 1), 0) if below == 31 else np.maximum(code, 0) | (pattern >> 31 << 7)
    code[n:] = 0
    return code.astype(np.uint8), exponent.astype(np.uint8)


def values(codes, scales, n, below):
    c = codes.astype(np.int64)
    low = c if below == 31 else c & 127
    a = np.where(low > 0, (low + np.repeat(scales.astype(np.int64) - below, 32) * 8) << 20, 0).astype(np.uint32).view(np.float32)
    return np.where((c > 127) & (below == 15), -a, a).astype(np.float32)[:n]


class Tensors:
    """Weights, gradients and moments of given sizes on the host, and on the GPU where a step is made."""

    def __init__(self, sizes, pt=F32, gt=F32, bits=32, seed=0, scale=1e-3):
        g = torch.Generator().manual_seed(seed)
        self.sizes, self.bits = sizes, bits
        self.p = [(torch.randn(n, generator=g) * 0.02).to(pt) for n in sizes]
        self.g = [(torch.randn(n, generator=g) * scale).to(gt) for n in sizes]
        self.m = [torch.randn(n, generator=g) * 0.3 * scale for n in sizes]
        self.v = [(torch.randn(n, generator=g) * scale) ** 2 * torch.rand(n, generator=g) for n in sizes]
        if bits == 8:
            self.coded = [[encode(t.numpy(), below, None) for t in ts] for ts, below in ((self.m, 15), (self.v, 31))]
            self.m, self.v = ([torch.from_numpy(values(*c, n, below)) for c, n in zip(cs, sizes)] for cs, below in zip(self.coded, (15, 31)))

    def to_gpu(self):
        dev = lambda ts: [t.to(DEV) for t in ts]   # noqa: E731
        out = {"params": dev(self.p), "grads": dev(self.g)}
        if self.bits == 32:
            return {**out, "m": dev(self.m), "v": dev(self.v)}
        for name, coded in zip("mv", self.coded):
            out[name], out[name + "_scales"] = ([torch.from_numpy(c[k]).to(DEV) for c in coded] for k in (0, 1))
        return out


def run(t, lr=3e-4, step=7, clip=None, seed=None, **over):
    s = sbn()
    d = t.to_gpu() if isinstance(t, Tensors) else t
    group = s.AdamWGroup(**d, betas=(B1, B2), **over)
    group.run(torch.tensor([lr], device=DEV), torch.tensor([step], device=DEV), clip=None if clip is None else torch.tensor([clip], device=DEV), seed=seed)
    torch.cuda.synchronize()
    return d


def check_step(t, lr=3e-4, step=7, clip=None, seed=None, decay=0.1, eps=EPS):
    d = run(t, lr, step, clip, seed, weight_decay=decay, eps=eps)
    decays = decay if isinstance(decay, list) else [decay] * len(t.sizes)
    f32 = lambda x: float(np.float32(x))   # noqa: E731
    lr = f32(lr)
    for i, n in enumerate(t.sizes):
        g = t.g[i].float()
        if clip is not None:
            g = g * f32(clip)
        m = t.m[i] * f32(B1) + g * f32(1 - B1)
        v = t.v[i] * f32(B2) + g * f32(1 - B2) * g
        bits = noise(n, seed, step, i) if seed is not None else (None, None, None)
        if t.bits == 32:
            assert torch.equal(d["m"][i].cpu(), m) and torch.equal(d["v"][i].cpu(), v)
        else:
            for name, x, below, b in (("m", m, 15, bits[1]), ("v", v, 31, bits[2])):
                codes, scales = encode(x.numpy(), below, b)
                assert np.array_equal(d[name + "_scales"][i].cpu().numpy(), scales), (name, i)
                assert np.array_equal(d[name][i].cpu().numpy(), codes), (name, i)
                for dtype in (F32, BF16):
                    out = torch.full((n,), float("nan"), dtype=dtype, device=DEV)
                    sbn().sbn_adamw_state_values(d[name][i], d[name + "_scales"][i], out, second=name == "v")
                    assert np.array_equal(out.float().cpu().numpy(), values(codes, scales, n, below))
        # the step in 64 bits from the same moments before
        g, p = t.g[i].double() * (1.0 if clip is None else f32(clip)), t.p[i].double()
        m, v = B1 * t.m[i].double() + (1 - B1) * g, B2 * t.v[i].double() + (1 - B2) * g * g
        terms = B1 * t.m[i].double().abs() + (1 - B1) * g.abs()
        under = torch.sqrt(v / (1 - B2 ** step)) + eps
        update = lr / (1 - B1 ** step) * m / under
        want = p * (1 - lr * f32(decays[i])) - update
        tol = U * (3 * p.abs() + 24 * lr / (1 - B1 ** step) * terms / under)
        got = d["params"][i].double().cpu()
        if t.p[i].dtype == BF16 and seed is not None:
            cut = lambda x: ((x.float().view(torch.int32).long() + torch.from_numpy(bits[0])) & -65536).to(torch.int32).view(F32).double()   # noqa: E731
            # what is nearer to zero is cut at or below, what is farther at or above
            low, high = cut(torch.sign(want) * (want.abs() - tol).clamp(min=0)), cut(torch.sign(want) * (want.abs() + tol))
            assert ((got - low) * torch.sign(want) >= 0).all() and ((high - got) * torch.sign(want) >= 0).all()
        else:
            if t.p[i].dtype == BF16:
                tol = tol + 2.0 ** -8 * (want.abs() + tol)
            assert ((got - want).abs() <= tol).all(), ((got - want).abs() - tol).max()
    return d


ODD = [1, 31, 32, 33, 1000, 8191, 8192, 8193, 20011]


@pytest.mark.parametrize("pt,gt", [(F32, F32), (F32, BF16), (BF16, BF16), (BF16, F32)])
@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("seed", [None, 12345678901234567])
def test_step(pt, gt, bits, seed):
    check_step(Tensors(ODD, pt, gt, bits, seed=1), seed=seed)
    check_step(Tensors(ODD, pt, gt, bits, seed=2), seed=seed, clip=0.37, decay=[0.01 * i for i in range(len(ODD))], step=1)


@pytest.mark.parametrize("bits", [32, 8])
def test_many_tensors(bits):
    """More tensors than one launch has in its table."""
    sizes = [1 + (37 * i) % 90 for i in range(61 + 60 + 5)]
    check_step(Tensors(sizes, BF16, BF16, bits, seed=3), seed=5)


@pytest.mark.parametrize("bits", [32, 8])
def test_first_step_from_nothing(bits):
    t = Tensors([100, 64], F32, F32, bits, seed=4)
    t.m, t.v = [torch.zeros(n) for n in t.sizes], [torch.zeros(n) for n in t.sizes]
    if bits == 8:
        t.coded = [[(np.zeros(-(-n // 32) * 32, np.uint8), np.zeros(-(-n // 32), np.uint8)) for n in t.sizes]] * 2
    t.g[0][10:20] = 0.0   # no gradient and no moments: only the decay
    d = check_step(t, step=1)
    assert torch.equal(d["params"][0][10:20].cpu(), t.p[0][10:20] * float(np.float32(1 - float(np.float32(3e-4)) * float(np.float32(0.1)))))


def test_moments_over_many_binades():
    """Blocks from the smallest fp32 numbers to the largest that a moment takes, and blocks whose values lie 40 binades apart."""
    t = Tensors([32 * 64], F32, F32, 8, seed=6)
    e = torch.arange(64).repeat_interleave(32).float()
    spread = torch.arange(32).repeat(64).float()
    t.g[0] = torch.exp2(e * 2.9 - 120.0) * (1 + torch.arange(2048) / 2048)
    t.g[0][1024:] = torch.exp2(-spread[1024:] * 1.3 + 20) * (1 + torch.arange(1024) / 1024)
    check_step(t)
    check_step(t, seed=3)


def test_rounding_borders():
    """Moments next to a border between two codes, ties among them, and blocks whose largest value rounds into the next binade."""
    t = Tensors([32 * 16], F32, F32, 8, seed=7)
    zero = (np.zeros(512, np.uint8), np.zeros(16, np.uint8))
    t.coded, t.m, t.v = [[zero], [zero]], [torch.zeros(512)], [torch.zeros(512)]
    top = torch.tensor([1.0, 1.0625, 1.1875, 1.8125, 1.875, 1.9375, 1.99, 1.9999999])
    unit = float(np.float32(1 - B1))
    g = (1 + (torch.arange(512) % 16) / 16) / 2
    for k in range(16):
        g[32 * k] = top[k % 8] * (1 if k < 8 else 2.0 ** 10)
    t.g[0] = g / unit
    check_step(t)
    check_step(t, seed=11)


def test_stochastic_rounding_is_even_on_average():
    """Many values between two neighbours: the mean of what they become is the value, to 5 deviations of a mean of that many."""
    n = 1 << 17
    t = Tensors([n], BF16, F32, 8, seed=8)
    t.p[0] = torch.full((n,), 1.0, dtype=BF16)
    t.g[0] = torch.full((n,), 1.0)
    zero = (np.zeros(n, np.uint8), np.zeros(n // 32, np.uint8))
    t.coded, t.m, t.v = [[zero], [zero]], [torch.zeros(n)], [torch.zeros(n)]
    d = check_step(t, lr=1e-3, step=1, seed=99, decay=0.0)
    p = d["params"][0].double().cpu()
    # 1 - 1e-3 lies between 1 - 2^-8 and 1: a quarter of the way
    assert set(p.tolist()) == {1.0, 1 - 2.0 ** -8}
    share = 1e-3 * 2 ** 8
    assert abs((p != 1).double().mean() - share) < 5 * (share * (1 - share) / n) ** 0.5
    m = torch.empty(n, device=DEV)
    sbn().sbn_adamw_state_values(d["m"][0], d["m_scales"][0], m)
    unit = 2.0 ** -7   # 0.1 lies between 12 and 13 steps of 2^-7
    share = float(np.float32(1 - B1)) / unit - 12
    assert set((m / unit).tolist()) == {12.0, 13.0}
    assert abs((m / unit - 12).double().mean().item() - share) < 5 * (share * (1 - share) / n) ** 0.5


def test_bits_differ_by_seed_step_and_place():
    n = 4096
    all_bits = [noise(n, seed, step, place) for seed, step, place in ((1, 1, 0), (2, 1, 0), (1, 2, 0), (1, 1, 1), (1 + (1 << 32), 1, 0))]
    series = [b.astype(float) for bits in all_bits for b in bits]
    for b in series:
        assert abs(b.mean() / 65536 - 0.5) < 5 / (12 * n) ** 0.5
    c = np.corrcoef(np.stack(series + [np.roll(series[0], 1), np.roll(series[0], 2)]))
    assert np.abs(c - np.eye(len(c))).max() < 5 / n ** 0.5


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("bits", [32, 8])
def test_no_step_where_the_factor_is_not_finite(bits, bad):
    t = Tensors([33, 1000], BF16, BF16, bits, seed=9)
    before, after = t.to_gpu(), run(t, clip=bad, seed=1)
    for name in before:
        assert all(torch.equal(a, b) for a, b in zip(before[name], after[name])), name


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("seed", [None, 5])
@pytest.mark.parametrize("pt", [F32, BF16])
def test_gradients_of_every_nan_leave_none_but_nan(pt, seed, bits):
    """A NaN of all ones (memory filled with 0xff) is one too: what is added to its pattern must not make a number of it."""
    t = Tensors([100], pt=pt, bits=bits)
    t.g[0].view(torch.int32)[:64] = torch.tensor([-1, 0x7fffffff]).int().repeat(32)
    d = run(t, seed=seed)
    assert torch.isnan(d["params"][0][:64]).all() and torch.isfinite(d["params"][0][64:]).all()


def test_tensors_of_a_buffer():
    """Weights and moments that lie in one buffer at odd places; what lies between them is not touched."""
    s = sbn()
    sizes, at = [33, 1001, 8], [1, 40, 1050]
    t = Tensors(sizes, BF16, BF16, 32, seed=10)
    want = check_step(t)
    d = t.to_gpu()
    bufs = {}
    for name in ("params", "grads", "m", "v"):
        bufs[name] = torch.full((1100,), 77.0, dtype=d[name][0].dtype, device=DEV)
        for k, n in enumerate(sizes):
            bufs[name][at[k]:at[k] + n] = d[name][k]
        d[name] = [bufs[name][a:a + n] for a, n in zip(at, sizes)]
    run(d, weight_decay=0.1)
    for name in ("params", "m", "v"):
        assert all(torch.equal(a, b) for a, b in zip(d[name], want[name]))
        gaps = torch.ones(1100, dtype=torch.bool)
        for a, n in zip(at, sizes):
            gaps[a:a + n] = False
        assert (bufs[name][gaps.to(DEV)] == 77).all()
    with pytest.raises(s.SbnError):
        s.AdamWGroup(d["params"] + d["params"][:1], d["grads"] + d["grads"][:1], d["m"] + d["m"][:1], d["v"] + d["v"][:1]).run(
            torch.ones(1, device=DEV), torch.ones(1, dtype=torch.int64, device=DEV))


def test_a_large_tensor():
    """2^31 values, the most that a tensor may have: the last ones are what a small tensor's would be."""
    n = 1 << 31
    d = {"params": [torch.full((n,), 0.5, dtype=BF16, device=DEV)], "grads": [torch.full((n,), 0.25, dtype=BF16, device=DEV)]}
    for name in "mv":
        d[name], d[name + "_scales"] = [torch.zeros(n, dtype=torch.uint8, device=DEV)], [torch.zeros(n // 32, dtype=torch.uint8, device=DEV)]
    run(d, lr=1e-2, weight_decay=0.0)
    small = {"params": [torch.full((64,), 0.5, dtype=BF16, device=DEV)], "grads": [torch.full((64,), 0.25, dtype=BF16, device=DEV)]}
    for name in "mv":
        small[name], small[name + "_scales"] = [torch.zeros(64, dtype=torch.uint8, device=DEV)], [torch.zeros(2, dtype=torch.uint8, device=DEV)]
    run(small, lr=1e-2, weight_decay=0.0)
    for name in ("params", "m", "v"):
        x = small[name][0][0].item()
        part = d[name][0].view(16, -1)
        assert all((part[k] == x).all() for k in range(16)), name
    s = sbn()
    out = torch.empty(1, device=DEV)
    norms = torch.empty(2, device=DEV)
    s.sbn_grad_norm(d["grads"], 1.0, norms, s.new_workspace(s.sbn_grad_norm_workspace_bytes([n])))
    assert norms[0].item() == 0.25 * 2 ** 15.5 or abs(norms[0].item() / (0.25 * 2 ** 15.5) - 1) < 2 * U
    del out


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("sizes", [[1], [7, 1000], [32768, 32769, 5], [200001, 3], [1 + i % 50 for i in range(340)]])
def test_grad_norm(sizes, dtype):
    s = sbn()
    g = torch.Generator().manual_seed(sum(sizes))
    grads = [(torch.randn(n, generator=g) * 10.0 ** (i % 5 - 2)).to(dtype) for i, n in enumerate(sizes)]
    ref = torch.cat([x.double() for x in grads]).norm().item()
    ws = s.new_workspace(s.sbn_grad_norm_workspace_bytes(sizes)).fill_(0xff)
    out = torch.full((2,), -1.0, device=DEV)
    group = s.GradNormGroup([x.to(DEV) for x in grads], ws)
    for max_norm in (ref / 3, ref * 3):
        group.run(max_norm, out)
        norm, factor = out.tolist()
        assert abs(norm - ref) <= 1.01 * U * ref
        want = min(1.0, float(np.float32(max_norm)) / ref)
        assert abs(factor - want) <= 1.01 * U * want


def test_grad_norm_at_the_ends_of_the_range():
    s = sbn()
    ws, out = s.new_workspace(s.sbn_grad_norm_workspace_bytes([1000])), torch.empty(2, device=DEV)
    x = torch.full((1000,), 1e30, device=DEV)   # squares past fp32, the norm within
    s.sbn_grad_norm([x], 1.0, out, ws)
    assert abs(out[0].item() / (1e30 * 1000 ** 0.5) - 1) < 1e-6 and out[1] > 0
    s.sbn_grad_norm([torch.full((1000,), 1e-30, device=DEV)], 1.0, out, ws)
    assert abs(out[0].item() / (1e-30 * 1000 ** 0.5) - 1) < 1e-6 and out[1] == 1
    s.sbn_grad_norm([torch.zeros(1000, device=DEV)], 1.0, out, ws)
    assert out.tolist() == [0.0, 1.0]
    for bad in (float("nan"), float("inf")):
        x[7] = bad
        s.sbn_grad_norm([x], 1.0, out, ws)
        assert not torch.isfinite(out[0]) and torch.isnan(out[1])
