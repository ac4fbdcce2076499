"""Where rows and gradients lie: norms of rows that begin at different places of a vector, the gradient norm on both sides of the sizes at which its blocks
change.  Tolerances as in the tests of the operators."""
import numpy as np
import pytest
import torch

from gpu_util import DEV, sbn
from test_gpu_step_norm import U, backward_reference, check_forward, near, rows

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32


# ---- norms --------------------------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("layer", [False, True])
@pytest.mark.parametrize("T,d", [(2500, 1001), (8200, 301), (2100, 2001), (4099, 2563)])
def test_equal_rows_that_begin_alike_have_equal_gradients(T, d, layer, dtype):
    """A row's sums go by where it begins in memory: rows that are eight apart begin at the same place of a vector, whatever their length."""
    s = sbn()
    X, g = rows(1, d, dtype, d, offset=0.3)
    dY, gain = (torch.randn(1, d, generator=g) * 0.02).to(dtype), 1 + 0.3 * torch.randn(d, generator=g)
    x, dy = (t.to(DEV).expand(T, d).contiguous() for t in (X, dY))
    Y, dX = torch.empty_like(x), torch.empty_like(x)
    ws = s.new_workspace(s.sbn_norm_workspace_bytes(T, d))
    s.sbn_norm(x, Y, gain=gain.to(DEV), layer=layer)
    s.sbn_norm_backward(x, dy, ws, dX=dX, dgain=torch.empty(d, device=DEV), gain=gain.to(DEV), layer=layer)
    for t in (Y, dX):
        for first in range(8):
            alike = t[first::8]
            assert (alike == alike[0]).all(), (first, (alike != alike[0]).any(1).sum().item())


AT = {"X": 0, "dY": 1, "R": 3, "S": 5, "Y": 2, "dX": 7}


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("layer", [False, True])
@pytest.mark.parametrize("T,d", [(13, 264), (13, 1003), (9, 2560), (9, 2565), (5, 8192), (3, 16383), (1030, 65)])
@pytest.mark.parametrize("places", [AT, dict.fromkeys(AT, 1)], ids=["apart", "alike"])
def test_rows_at_places_of_their_own(T, d, layer, dtype, places):
    """Each tensor begins elsewhere in a vector, or all of them off its beginning: no row takes values of its neighbours, and nothing around the rows is written."""
    s = sbn()
    X, g = rows(T, d, dtype, d + T, offset=0.3)
    R, dY, gain = torch.randn(T, d, generator=g).to(dtype), (torch.randn(T, d, generator=g) * 0.02).to(dtype), 1 + 0.3 * torch.randn(d, generator=g)
    n = T * d
    bufs = {name: torch.full((n + 48,), 77.0, dtype=dtype, device=DEV) for name in places}
    t = {name: bufs[name][16 + at:16 + at + n].view(T, d) for name, at in places.items()}
    for name, value in (("X", X), ("R", R), ("dY", dY)):
        t[name].copy_(value)
    gain_d = gain.to(DEV)
    s.sbn_norm(t["X"], t["Y"], gain=gain_d, layer=layer)
    check_forward(X, layer, gain, Y=t["Y"])
    s.sbn_norm(t["X"], t["Y"], gain=gain_d, layer=layer, residual=t["R"], sum_out=t["S"])
    S = (X.float() + R.float()).to(dtype)
    assert torch.equal(t["S"].cpu(), S)
    check_forward(S, layer, gain, Y=t["Y"])
    half = torch.finfo(dtype).eps / 2
    need = s.sbn_norm_workspace_bytes(T, d)
    ws = s.new_workspace(need + 1024).fill_(0xa5)
    for residual in (None, "R"):
        dgain, dbias = torch.empty(d, device=DEV), torch.empty(d, device=DEV)
        s.sbn_norm_backward(t["X"], t["dY"], ws[:need], dX=t["dX"], dgain=dgain, dbias=dbias, gain=gain_d, layer=layer, d_residual=t.get(residual))
        dX, tol, *sums, tol_gain, tol_bias = backward_reference(X, dY, layer, gain, 1e-6, R if residual else None)
        near(t["dX"], dX, half * dX.abs() + tol, "dX")
        near(dgain, sums[0], tol_gain, "dgain")
        near(dbias, sums[1], tol_bias, "dbias")
    assert (ws[need:] == 0xa5).all()
    for name, at in places.items():
        assert (bufs[name][:16 + at] == 77.0).all() and (bufs[name][16 + at + n:] == 77.0).all(), name


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("T,d", [(1, 300), (3, 2559), (40, 512), (600, 513), (5000, 300), (3000, 512), (1100, 2559), (700, 4096), (300, 16384), (300, 16383)])
def test_shares_stay_in_the_workspace(T, d, dtype):
    """Rows and lengths at which the shares of the blocks take most of the workspace, or few rows less of it."""
    s = sbn()
    need = s.sbn_norm_workspace_bytes(T, d)
    ws = s.new_workspace(need + 4096).fill_(0xa5)
    X = torch.randn(T, d, generator=torch.Generator(device=DEV).manual_seed(d), device=DEV).to(dtype)
    out = {"dgain": torch.empty(d, device=DEV), "dbias": torch.empty(d, device=DEV)}
    s.sbn_norm_backward(X, X, ws[:need], layer=True, **out)
    assert (ws[need:] == 0xa5).all()
    x = X.double()
    h = (x - x.mean(1, keepdim=True)) / torch.sqrt(x.var(1, correction=0, keepdim=True) + 1e-6)
    assert ((out["dgain"] - (x * h).sum(0)).abs() <= U * 200 * (x.abs() * (h.abs() + 1)).sum(0)).all()
    assert ((out["dbias"] - x.sum(0)).abs() <= U * 200 * x.abs().sum(0)).all()


# ---- gradient norm ------------------------------------------------------------------------------------------------------------------
MB32 = 32 << 20


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("total", [MB32 - 4, MB32, MB32 + 4, (256 << 20) + 4], ids=["below_32MB", "32MB", "above_32MB", "above_256MB"])
def test_grad_norm_of_ragged_tensors(total, dtype):
    """Several tensors whose ends lie in the middle of a block, where blocks become longer and where gradients go past the caches."""
    s = sbn()
    values = total // dtype.itemsize
    sizes = [1, 32769, 65537, 1 << 20, 3]
    sizes.append(values - sum(sizes) - 16385)
    sizes.append(16385)
    g = torch.Generator(device=DEV).manual_seed(total)
    grads = [(torch.randn(n, generator=g, device=DEV) * 10.0 ** (i % 5 - 2)).to(dtype) for i, n in enumerate(sizes)]
    assert sum(t.numel() for t in grads) == values
    ref = sum(t.double().square().sum() for t in grads).sqrt().item()
    need = s.sbn_grad_norm_workspace_bytes(sizes)
    ws = s.new_workspace(need + 512).fill_(0xff)
    out = torch.full((2,), -1.0, device=DEV)
    s.sbn_grad_norm(grads, ref / 3, out, ws[:need])
    norm, factor = out.tolist()
    assert abs(norm - ref) <= 1.01 * U * ref   # squares and sums in double, one rounding
    assert abs(factor - float(np.float32(ref / 3)) / ref) <= 1.01 * U / 3
    assert (ws[need:] == 0xff).all()
