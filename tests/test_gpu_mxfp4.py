"""Microscaled 4-bit floating point on the GPU: codes, scales and values bit for bit, products against 64 bits.

A product of two quantized values is exact; a sum of K of them loses at most 2^-23 of the sum of their magnitudes at each addition, and the bias
one step more."""
import pytest
import torch

from gpu_util import DEV, sbn

pytestmark = pytest.mark.gpu

GRID = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6], dtype=torch.float64)


def quantize(X):
    """Codes and scales by the definition: the nearest code, the even one of two that are as near."""
    X = X.cpu().double()
    rows, cols = X.shape
    wide = -(-cols // 128) * 128
    x = torch.zeros(rows, wide, dtype=torch.float64)
    sign = torch.zeros(rows, wide, dtype=torch.bool)
    x[:, :cols] = X.abs()
    sign[:, :cols] = torch.signbit(X)
    x = x.view(rows, -1, 32)
    most = x.amax(2)
    exponent = torch.frexp(most)[1] - 1           # floor(log2)
    field = torch.where(most >= 2.0 ** -126, exponent + 127, 0)
    s = (field - 2).clamp(min=0)
    v = x * torch.exp2(127.0 - s.double())[:, :, None]
    far = (v[..., None] - GRID).abs()
    near = far.amin(-1, keepdim=True)
    even = torch.arange(8) % 2 == 0
    code = torch.where(far == near, torch.where(even, 0, 1), 2).argmin(-1)
    code = code.view(rows, wide) | (sign.long() << 3)
    return (code[:, 0::2] | (code[:, 1::2] << 4)).to(torch.uint8), s.to(torch.uint8)


def values(codes, scales, cols):
    rows = codes.shape[0]
    code = torch.stack((codes & 15, codes >> 4), 2).view(rows, -1).long()
    v = GRID[code & 7] * torch.where(code > 7, -1.0, 1.0)
    return (v.view(rows, -1, 32) * torch.exp2(scales.double() - 127)[:, :, None]).view(rows, -1)[:, :cols]


def hip_quantize(X):
    s = sbn()
    rows, cols = X.shape
    nc, ns = s.sbn_mxfp4_bytes(rows, cols)
    codes, scales = torch.full((rows, nc // rows), 0xee, dtype=torch.uint8, device=DEV), torch.full((rows, ns // rows), 0xee, dtype=torch.uint8, device=DEV)
    s.sbn_mxfp4_quantize(X, codes, scales)
    return codes, scales


def check_quantize(X):
    codes, scales = hip_quantize(X.to(DEV))
    want_codes, want_scales = quantize(X)
    assert torch.equal(scales.cpu(), want_scales)
    assert torch.equal(codes.cpu(), want_codes)
    Y = torch.full(X.shape, float("nan"), dtype=X.dtype, device=DEV)
    sbn().sbn_mxfp4_dequantize(codes, scales, Y)
    want = values(want_codes, want_scales, X.shape[1])
    assert torch.equal(Y.cpu().double(), want)
    return codes, scales


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rows,cols", [(1, 8), (1, 128), (3, 40), (77, 1000), (33, 256), (257, 136), (5, 4104)])
def test_quantize(rows, cols, dtype):
    g = torch.Generator().manual_seed(rows)
    X = torch.randn(rows, cols, generator=g) * torch.exp2(torch.randint(-8, 9, (rows, 1), generator=g))
    check_quantize(X.to(dtype))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_rounding_borders(dtype):
    """Every border between two codes, the values next to it on either side, and both signs, at several scales."""
    borders = torch.tensor([0.25, 0.5, 0.75, 1.0, 1.25, 1.5, 1.75, 2, 2.5, 3, 3.5, 4, 5, 6, 7, 7.9])
    step = torch.finfo(dtype).eps
    row = torch.cat([borders, borders * (1 + step), borders * (1 - step), -borders, -borders * (1 + step), -borders * (1 - step)]).to(dtype).float()
    blocks = torch.zeros(len(row), 32)
    blocks[:, 0], blocks[:, 1:], blocks[:, 5] = 4.0, row[:, None], 7.5
    blocks = blocks.view(3, -1)
    for scale in (1.0, 2.0 ** -20, 2.0 ** 60, 2.0 ** -120, 2.0 ** 124):
        check_quantize((blocks * scale).to(dtype))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_extremes(dtype):
    top = torch.finfo(dtype).max
    tiny = torch.finfo(dtype).tiny
    X = torch.zeros(8, 64)
    X[1, 3], X[1, 40] = top, -top
    X[2, :32] = tiny
    X[3] = -0.0
    X[4, 7], X[4, 8], X[4, 50] = tiny / 2, -tiny / 2, tiny * 3     # below the normal numbers
    X[5, 0], X[5, 1], X[5, 33] = top, 1e-30, 1e-30
    X[6, :] = torch.linspace(-1, 1, 64) * tiny * 8
    check_quantize(X.to(dtype))


LINEAR = [(1, 8, 1, False), (1, 128, 5, True), (1, 2560, 1000, False), (1, 1000, 333, True), (2, 136, 17, False), (3, 520, 200, True), (7, 384, 129, False),
          (16, 256, 64, True), (17, 1000, 300, False), (31, 2560, 130, True), (33, 128, 64, False), (64, 264, 1001, True), (65, 640, 257, False),
          (130, 1000, 391, True), (300, 1288, 515, False), (515, 512, 1026, True)]


@pytest.fixture
def tiles():
    yield sbn().sbn_test_set_head_tiles
    sbn().sbn_test_set_head_tiles()


@pytest.mark.parametrize("size", [0, 1, 2])
@pytest.mark.parametrize("tokens,d_in,d_out,bias", [(1, 8, 1, True), (33, 264, 129, False), (130, 1000, 391, True), (300, 1288, 515, False), (600, 136, 260, True)])
def test_linear_in_every_tile_size(tokens, d_in, d_out, bias, size, tiles):
    tiles(mxfp4=size)
    test_linear(tokens, d_in, d_out, bias)


@pytest.mark.parametrize("tokens,d_in,d_out,bias", LINEAR)
def test_linear(tokens, d_in, d_out, bias):
    s = sbn()
    g = torch.Generator().manual_seed(tokens + d_out)
    X = torch.randn(tokens, d_in, generator=g) * torch.exp2(torch.randint(-3, 4, (tokens, d_in), generator=g))
    X = X.bfloat16()
    W = torch.randn(d_out, d_in, generator=g) * torch.exp2(torch.randint(-3, 4, (d_out, 1), generator=g)) / d_in ** 0.5
    b = torch.randn(d_out, generator=g) if bias else None
    codes, scales = hip_quantize(W.to(DEV))
    Y = torch.full((tokens, d_out), float("nan"), device=DEV)
    ws = torch.full((s.sbn_mxfp4_workspace_bytes(tokens, d_in),), 0xff, dtype=torch.uint8, device=DEV)
    s.sbn_mxfp4_linear(X.to(DEV), codes, scales, Y, ws, bias=None if b is None else b.to(DEV))
    torch.cuda.synchronize()
    x, w = values(*quantize(X), d_in), values(*quantize(W), d_in)
    want = x @ w.t()
    off = d_in * 2.0 ** -23 * (x.abs() @ w.abs().t())
    if bias:
        want = want + b.double()
        off = off + 2.0 ** -23 * want.abs()
    bad = ~((Y.cpu().double() - want).abs() <= off)
    assert not bad.any(), f"{int(bad.sum())} of {bad.numel()} off, worst {(Y.cpu().double() - want).abs().nan_to_num(1e30).amax().item()}"


def test_linear_of_zeros_and_far_scales():
    """Blocks of zeros beside blocks of very small and very large scales: no scale makes something of a zero."""
    s = sbn()
    X = torch.zeros(20, 256)
    X[:, 32:64] = 1.0
    X[3] = 0.0
    X[4, 32:] = 2.0 ** -60
    X[5, :32], X[5, 32:] = 2.0 ** 50, 0.0   # (no sum below needs more than 24 bits)
    W = torch.zeros(40, 256)
    W[:, 32:64] = 0.5
    W[7] = 2.0 ** -50
    W[8, :32] = 2.0 ** 40
    codes, scales = hip_quantize(W.to(DEV))
    for tokens in (1, 20):
        Y = torch.full((tokens, 40), float("nan"), device=DEV)
        s.sbn_mxfp4_linear(X[:tokens].bfloat16().to(DEV), codes, scales, Y, s.new_workspace(s.sbn_mxfp4_workspace_bytes(tokens, 256)))
        torch.cuda.synchronize()
        assert torch.equal(Y.cpu().double(), X[:tokens].double() @ W.double().t())


def test_linear_in_a_graph_and_on_another_stream():
    s = sbn()
    g = torch.Generator().manual_seed(3)
    codes, scales = hip_quantize(torch.randn(700, 512, generator=g).to(DEV))
    for tokens in (1, 12, 200):
        X = torch.randn(tokens, 512, generator=g).bfloat16().to(DEV)
        ws = s.new_workspace(s.sbn_mxfp4_workspace_bytes(tokens, 512))
        eager, Y, other = (torch.zeros(tokens, 700, device=DEV) for _ in range(3))
        s.sbn_mxfp4_linear(X, codes, scales, eager, ws)
        torch.cuda.synchronize()
        stream = torch.cuda.Stream()
        with torch.cuda.stream(stream):
            s.sbn_mxfp4_linear(X, codes, scales, other, ws)
        torch.cuda.synchronize()
        assert torch.equal(other, eager)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            s.sbn_mxfp4_linear(X, codes, scales, Y, ws)
        for _ in range(3):
            Y.fill_(float("nan"))
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(Y, eager)
            s.sbn_mxfp4_linear(X, codes, scales, other, ws)
            torch.cuda.synchronize()
            assert torch.equal(other, eager)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("value", [float("nan"), float("inf"), -float("inf")])
def test_a_block_that_is_not_finite_touches_no_other(value, dtype):
    s = sbn()
    g = torch.Generator().manual_seed(9)
    X = torch.randn(9, 264, generator=g).to(dtype)
    broken = X.clone()
    broken[4, 70], broken[4, 71], broken[8, 263] = value, -value, value     # blocks 2 and 8 of rows of 12
    codes, scales = hip_quantize(X.to(DEV))
    c, sc = hip_quantize(broken.to(DEV))
    assert (sc < 255).all()
    same = torch.ones(9, 12, dtype=torch.bool, device=DEV)
    same[4, 2] = same[8, 8] = False
    assert torch.equal(sc[same], scales[same]) and torch.equal(c.view(9, 12, 16)[same], codes.view(9, 12, 16)[same])
    W = hip_quantize(torch.randn(300, 264, generator=g).to(DEV))
    for rows in (9, 9 * 40):   # both kernels of the product
        Y = [torch.full((rows, 300), float("nan"), device=DEV) for _ in range(2)]
        for x, y in zip((X, broken), Y):
            x = x.bfloat16().repeat(rows // 9, 1).to(DEV)
            s.sbn_mxfp4_linear(x, *W, y, s.new_workspace(s.sbn_mxfp4_workspace_bytes(rows, 264)))
        others = torch.arange(rows, device=DEV) % 9
        others = (others != 4) & (others != 8)
        assert torch.equal(Y[0][others], Y[1][others])
