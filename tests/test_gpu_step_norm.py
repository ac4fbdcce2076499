"""RMS and layer norm with their gradients on the GPU against 64 bits.

Tolerances, with u = 2^-24 (half a step of fp32) and half = eps / 2 of the rows' type for the rounding of a result.  No sum of a row has more than 64
additions in a chain (at most 46 values in a thread, or 32 and 22 more across the row's threads), each off by at most u of the sum of magnitudes:
  mean: 64 u mean|x - mu| once the first sum has been taken off;  r: 32 u of its value from the sum of squares, and 8 u more
  h = (x - mu) r is off by at most u (64 + 64 |h|),  Y by |gain| times that and u (4 |Y| + 2 |bias|) for its own operations
  dX / r = a - mean a - h mean(a h): with A = mean|a| and B = mean|a h|, 64 u A + 64 u (B + A) |h| from the sums, u (64 + 64 |h|) (B + A) from h, 64 u of
  all terms from r and the products
  dgain, dbias: chains of T / rows at once + 64 additions, at most 200 for the sizes here, and what h is off by"""
import pytest
import torch

from gpu_util import DEV, sbn

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
BF16, F32 = torch.bfloat16, torch.float32


def rows(T, d, dtype, seed, offset=0.0):
    g = torch.Generator().manual_seed(seed)
    X = (torch.randn(T, d, generator=g) + offset) * torch.exp(torch.randn(d, generator=g))
    return X.to(dtype), g


def statistics(X, layer, eps):
    x = X.double()
    mu = x.mean(1, keepdim=True) if layer else torch.zeros(len(x), 1, dtype=torch.float64)
    r = 1 / torch.sqrt(((x - mu) ** 2).mean(1, keepdim=True) + eps)
    return (x - mu) * r, r


def near(got, ref, tol, what):
    got = got.double().cpu()
    assert torch.isfinite(got).all(), what
    worst = ((got - ref).abs() - tol).max()
    assert worst <= 0, f"{what}: {worst} beyond the tolerance, {(got - ref).abs().max()} off"


def check_forward(X, layer, gain=None, bias=None, residual=None, eps=1e-6, Y=None):
    """Y: where the result is already, else the call is made."""
    s = sbn()
    half = torch.finfo(X.dtype).eps / 2
    dev = lambda t: None if t is None else t.to(DEV)   # noqa: E731
    made = Y is None
    Y = torch.full(X.shape, float("nan"), dtype=X.dtype, device=DEV) if made else Y
    S = torch.full_like(Y, float("nan")) if residual is not None else None
    if made:
        s.sbn_norm(X.to(DEV), Y, gain=dev(gain), bias=dev(bias), eps=eps, layer=layer, residual=dev(residual), sum_out=S)
    if residual is not None:
        X = (X.float() + residual.float()).to(X.dtype)
        assert torch.equal(S.cpu(), X)
    h, _ = statistics(X, layer, eps)
    g = gain.double() if gain is not None else torch.ones(X.shape[1], dtype=torch.float64)
    b = bias.double() if bias is not None else torch.zeros(X.shape[1], dtype=torch.float64)
    ref = h * g + b
    near(Y, ref, half * ref.abs() + U * (g.abs() * (64 + 64 * h.abs()) + 4 * ref.abs() + 2 * b.abs()), "Y")
    return Y


SIZES = [(1, 1), (1, 8), (3, 7), (2, 63), (5, 64), (4, 127), (9, 520), (33, 1000), (17, 1001), (6, 2560), (5, 2563), (3, 4100), (3, 8192), (2, 8195), (2, 16384), (1, 16383)]


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("layer", [False, True])
@pytest.mark.parametrize("T,d", SIZES)
def test_forward(T, d, layer, dtype):
    X, g = rows(T, d, dtype, d, offset=0.5)
    gain, bias = 1 + 0.3 * torch.randn(d, generator=g), 0.1 * torch.randn(d, generator=g)
    check_forward(X, layer, gain, bias)
    check_forward(X, layer, gain, residual=torch.randn(T, d, generator=g).to(dtype))
    check_forward(X, layer)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_rows_far_off_zero(dtype):
    """Rows whose mean is a thousand times their deviation: fp32 sums of their squares would lose it."""
    X, _ = rows(7, 1000, F32, 3)
    check_forward((X / X.std() + 1000.0).to(dtype), True)


def test_zero_and_constant_rows():
    for X in (torch.zeros(3, 200), torch.full((3, 200), 7.25), torch.full((3, 200), 1e-30)):
        for layer in (False, True):
            check_forward(X, layer, eps=1e-6)
    Y = torch.empty(3, 200, device=DEV)
    sbn().sbn_norm(torch.zeros(3, 200, device=DEV), Y, eps=0.0, layer=False)   # 0 / 0
    assert torch.isnan(Y).all()


def test_one_bad_row_leaves_the_others():
    X, _ = rows(9, 1001, BF16, 5)
    want = check_forward(X, True)
    for bad in (float("nan"), float("inf")):
        B = X.clone()
        B[4, 700] = bad
        for layer in (False, True):
            Y, dX = torch.empty(9, 1001, dtype=BF16, device=DEV), torch.empty(9, 1001, dtype=BF16, device=DEV)
            sbn().sbn_norm(B.to(DEV), Y, layer=layer)
            ws = sbn().new_workspace(sbn().sbn_norm_workspace_bytes(9, 1001))
            sbn().sbn_norm_backward(B.to(DEV), X.to(DEV), ws, dX=dX, layer=layer)
            keep = torch.arange(9) != 4
            assert torch.isfinite(Y.cpu()[keep]).all() and torch.isfinite(dX.cpu()[keep]).all()
            assert torch.isnan(dX.cpu()[4]).all() and torch.isnan(Y.cpu()[4, 700])
            if layer:
                assert torch.isnan(Y.cpu()[4]).all() and torch.equal(Y.cpu()[keep], want.cpu()[keep])


@pytest.mark.parametrize("layer", [False, True])
@pytest.mark.parametrize("d", [60, 2560, 8192])
def test_a_nan_in_a_row_is_a_nan_in_every_gradient(d, layer):
    """r of such a row is NaN, and so is its share of every dgain."""
    s = sbn()
    X, g = rows(9, d, F32, d)
    dY = torch.randn(9, d, generator=g)
    X[4, 7] = float("nan")
    dX, dgain, dbias = torch.empty(9, d, device=DEV), torch.empty(d, device=DEV), torch.empty(d, device=DEV)
    s.sbn_norm_backward(X.to(DEV), dY.to(DEV), s.new_workspace(s.sbn_norm_workspace_bytes(9, d)), dX=dX, dgain=dgain, dbias=dbias, layer=layer)
    assert torch.isnan(dgain).all() and torch.isfinite(dbias).all()
    assert torch.isnan(dX[4]).all() and torch.isfinite(dX[:4]).all() and torch.isfinite(dX[5:]).all()
    Y = torch.empty(9, d, device=DEV)
    s.sbn_norm(torch.full((9, d), 1e30).index_fill_(1, torch.arange(0, d, 2), -1e30).to(DEV), Y, layer=True)   # squares past the range: no number, or r = 0
    assert (torch.isnan(Y) | (Y == 0)).all()


def test_rms_is_the_fused_norm_of_the_quantizer():
    """Y of the RMS form is what sbn_rmsnorm_act_quant normalises to, bit for bit."""
    s = sbn()
    for T, d in ((1, 2560), (40, 1000), (70, 4104), (3, 16384)):
        X, g = rows(T, d, BF16, T)
        gain = (1 + 0.3 * torch.randn(d, generator=g)).to(DEV)
        Xd, xn, Y = X.to(DEV), torch.empty(T, d, dtype=BF16, device=DEV), torch.empty(T, d, dtype=BF16, device=DEV)
        s.sbn_rmsnorm_act_quant(Xd, torch.empty(T, d, dtype=torch.int8, device=DEV), torch.empty(T, device=DEV), gain=gain, eps=1e-5, xn_out=xn)
        s.sbn_norm(Xd, Y, gain=gain, eps=1e-5)
        assert torch.equal(xn, Y)


def backward_reference(X, dY, layer, gain, eps, residual):
    h, r = statistics(X, layer, eps)
    dy = dY.double()
    a = dy * gain.double() if gain is not None else dy
    dX = r * (a - (a.mean(1, keepdim=True) if layer else 0.0) - h * (a * h).mean(1, keepdim=True))
    A, B = a.abs().mean(1, keepdim=True), (a * h).abs().mean(1, keepdim=True)
    tol = U * r * (64 * a.abs() + 128 * A + (192 * h.abs() + 64) * (A + B))
    if residual is not None:
        dX = dX + residual.double()
        tol = tol + 2 * U * residual.double().abs()
    near_gain = U * 200 * (dy.abs() * (h.abs() + 1)).sum(0)
    return dX, tol, (dy * h).sum(0), dy.sum(0), near_gain, U * 200 * dy.abs().sum(0)


def check_backward(X, dY, layer, gain=None, residual=None, eps=1e-6, want=("dX", "dgain", "dbias")):
    s = sbn()
    T, d = X.shape
    dev = lambda t: None if t is None else t.to(DEV)   # noqa: E731
    out = {"dX": torch.full((T, d), float("nan"), dtype=X.dtype, device=DEV), "dgain": torch.full((d,), float("nan"), device=DEV), "dbias": torch.full((d,), float("nan"), device=DEV)}
    out = {k: v for k, v in out.items() if k in want}
    ws = s.new_workspace(s.sbn_norm_workspace_bytes(T, d)).fill_(0xff)
    s.sbn_norm_backward(X.to(DEV), dY.to(DEV), ws, gain=dev(gain), eps=eps, layer=layer, d_residual=dev(residual), **out)
    dX, tol, dgain, dbias, tol_gain, tol_bias = backward_reference(X, dY, layer, gain, eps, residual)
    if "dX" in out:
        near(out["dX"], dX, torch.finfo(X.dtype).eps / 2 * dX.abs() + tol, "dX")
    if "dgain" in out:
        near(out["dgain"], dgain, tol_gain, "dgain")
    if "dbias" in out:
        near(out["dbias"], dbias, tol_bias, "dbias")
    return out


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("layer", [False, True])
@pytest.mark.parametrize("T,d", SIZES + [(4099, 264), (2500, 1001), (2100, 33)])
def test_backward(T, d, layer, dtype):
    X, g = rows(T, d, dtype, 2 * d, offset=0.3)
    dY, gain = (torch.randn(T, d, generator=g) * 0.02).to(dtype), 1 + 0.3 * torch.randn(d, generator=g)
    first = check_backward(X, dY, layer, gain)
    again = check_backward(X, dY, layer, gain)
    assert all(torch.equal(first[k], again[k]) for k in first)
    check_backward(X, dY, layer, gain, residual=(torch.randn(T, d, generator=g) * 0.02).to(dtype))
    check_backward(X, dY, layer)
    for want in (["dX"], ["dgain"], ["dbias"]):
        only = check_backward(X, dY, layer, gain, want=want)
        assert torch.equal(only[want[0]], first[want[0]])


@pytest.mark.parametrize("layer", [False, True])
def test_backward_against_differences(layer):
    """The reference itself: central differences of the formula in 64 bits."""
    g = torch.Generator().manual_seed(8)
    X, gain, dY = (torch.randn(*n, generator=g, dtype=torch.float64) for n in ((3, 9), (9,), (3, 9)))
    value = lambda x, w: ((statistics(x, layer, 1e-6)[0] * w) * dY).sum()   # noqa: E731
    dX, _, dgain, *_ = backward_reference(X, dY, layer, gain, 1e-6, None)
    e = 1e-6
    for i in range(27):
        step = torch.zeros(27, dtype=torch.float64)
        step[i] = e
        step = step.view(3, 9)
        assert abs((value(X + step, gain) - value(X - step, gain)) / (2 * e) - dX.view(-1)[i]) < 1e-7
    for i in range(9):
        step = torch.zeros(9, dtype=torch.float64)
        step[i] = e
        assert abs((value(X, gain + step) - value(X, gain - step)) / (2 * e) - dgain[i]) < 1e-7


def test_results_in_place_of_operands():
    """dX in place of dY or d_residual, Y in place of X, the sum in place of the residual."""
    s = sbn()
    X, g = rows(37, 1001, BF16, 9)
    R, dY, gain = torch.randn(37, 1001, generator=g).to(BF16), torch.randn(37, 1001, generator=g).to(BF16), torch.randn(1001, generator=g)
    want = check_backward(X, dY, True, gain, R)["dX"]
    ws = s.new_workspace(s.sbn_norm_workspace_bytes(37, 1001))
    for same in ("dY", "R"):
        t = {"dY": dY.to(DEV), "R": R.to(DEV)}
        s.sbn_norm_backward(X.to(DEV), t["dY"], ws, dX=t[same], gain=gain.to(DEV), layer=True, d_residual=t["R"])
        assert torch.equal(t[same], want)
    Y = check_forward(X, True, gain, residual=R)
    x, r = X.to(DEV), R.to(DEV)
    s.sbn_norm(x, x, gain=gain.to(DEV), layer=True, residual=r, sum_out=r)
    assert torch.equal(x, Y) and torch.equal(r.cpu(), (X.float() + R.float()).to(BF16))


def test_rows_at_odd_addresses_and_what_lies_around_them():
    """Rows that begin at any value of a buffer; nothing before or behind them is written."""
    s = sbn()
    for dtype in (BF16, F32):
        X, g = rows(5, 1003, dtype, 11)
        dY = torch.randn(5, 1003, generator=g).to(dtype)
        n = X.numel()
        for at in (1, 3, 8):
            place = lambda t: torch.full((n + 32,), 77.0, dtype=t.dtype, device=DEV)   # noqa: E731
            bufs = [place(X) for _ in range(4)]
            x, dy, Y, dX = (b[at:at + n].view(5, 1003) for b in bufs)
            x.copy_(X)
            dy.copy_(dY)
            s.sbn_norm(x, Y, layer=True)
            s.sbn_norm_backward(x, dy, s.new_workspace(s.sbn_norm_workspace_bytes(5, 1003)), dX=dX, layer=True)
            # against 64 bits and not bit for bit: a row that begins elsewhere in a vector is added up in another order, which the tolerances allow for any
            check_forward(X, True, Y=Y)
            want, tol, *_ = backward_reference(X, dY, True, None, 1e-6, None)
            near(dX, want, torch.finfo(dtype).eps / 2 * want.abs() + tol, "dX")
            for b in bufs:
                assert (b[:at] == 77.0).all() and (b[at + n:] == 77.0).all()


def test_many_rows():
    """More rows than a launch of one row to a thread block has in flight, and an offset past 2^31 values."""
    s = sbn()
    T, d = 1 << 18, 8200
    X = torch.empty(T, d, dtype=BF16, device=DEV).normal_(generator=torch.Generator(device=DEV).manual_seed(1))
    Y = torch.empty_like(X)
    s.sbn_norm(X, Y, layer=True)
    at = [0, 1, T // 2 + 1, T - 1]
    h, _ = statistics(X[at].cpu(), True, 1e-6)
    near(Y[at], h, 2.0 ** -8 * h.abs() + U * (64 + 68 * h.abs()), "Y")
    dgain, dbias = torch.empty(d, device=DEV), torch.empty(d, device=DEV)
    ws = s.new_workspace(s.sbn_norm_workspace_bytes(T, d))
    s.sbn_norm_backward(X, Y, ws, dX=Y, dgain=dgain, dbias=dbias, layer=True)   # in place: dX of rows whose gradient is their norm is nearly nothing
    assert Y.abs().max() < 0.05 and torch.isfinite(dgain).all()
    assert ((dgain / T - 1).abs() < 0.02).all()   # the sum of h^2 over the rows is near their number
