"""The output head and 4-bit floating point at the ends of the ranges that their calls take."""
import pytest
import torch

from gpu_util import DEV, sbn

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("tokens", [2 ** 27 - 1, 2 ** 27])
def test_4bit_product_of_the_most_tokens(tokens):
    # the tokens' rows are padded to 256 columns, 2^32 vectors of eight values at 2^27 of them; small integers: sums are exact in any order
    s = sbn()
    torch.cuda.empty_cache()
    d_in, d_out = 8, 3
    g = torch.Generator().manual_seed(1)
    some = torch.randint(-2, 3, (64, d_in), generator=g).bfloat16()
    W = torch.randint(-2, 3, (d_out, d_in), generator=g).bfloat16()
    some[:, 0], W[:, 0] = 4, 4       # the largest of a block: its scale is 1
    X = some.to(DEV).repeat(2 ** 27 // 64, 1)[:tokens]
    codes, scales = (torch.empty(n, dtype=torch.uint8, device=DEV) for n in s.sbn_mxfp4_bytes(d_out, d_in))
    s.sbn_mxfp4_quantize(W.to(DEV), codes, scales)
    Y = torch.full((tokens, d_out), float("nan"), device=DEV)
    ws = torch.full((s.sbn_mxfp4_workspace_bytes(tokens, d_in),), 0xff, dtype=torch.uint8, device=DEV)   # NaN whatever is read of it
    s.sbn_mxfp4_linear(X, codes, scales, Y, ws)
    want = (some.float() @ W.float().t()).to(DEV)
    whole = tokens // 64 * 64
    assert torch.equal(Y[:whole].view(-1, 64, d_out), want.expand(whole // 64, 64, d_out))
    assert torch.equal(Y[whole:], want[:tokens - whole])
    del X, Y, ws
    torch.cuda.empty_cache()


def test_gradient_of_17_billion_values_in_pieces():
    # 2^34 values of dH, the most that a call takes, added up over two pieces of the vocabulary: every 64th token is the same
    s = sbn()
    torch.cuda.empty_cache()
    tokens, d, vocab, period = 2 ** 24, 1024, 257, 64
    g = torch.Generator().manual_seed(2)
    some, W = torch.randn(period, d, generator=g).bfloat16(), (torch.randn(vocab, d, generator=g) * 2 / d ** 0.5).bfloat16()
    targets, d_ce = torch.randint(0, vocab, (period,), generator=g), torch.randn(period, generator=g)
    targets[5] = 256                 # of the second piece
    H, y, grad = some.to(DEV).repeat(tokens // period, 1), targets.to(DEV).repeat(tokens // period), d_ce.to(DEV).repeat(tokens // period)
    lse = torch.logsumexp(some.double() @ W.double().t(), 1)
    dH = torch.full((tokens, d), float("nan"), dtype=torch.bfloat16, device=DEV)
    ws = s.new_workspace(s.sbn_head_workspace_bytes(tokens, d, vocab))
    s.sbn_head_cross_entropy_backward(H, W.to(DEV), y, lse.float().to(DEV).repeat(tokens // period), grad, ws, dH=dH)
    torch.cuda.synchronize()
    del H, ws
    # G off by the rounding of lse (half a step of 2^-23), by dz <= d 2^-23 sum |h w| and by 2^-8 for its own, dH by that, its additions and 2^-8
    h, w = some.double(), W.double()
    z = h @ w.t()
    dz = d * 2.0 ** -23 * (h.abs() @ w.abs().t()).amax() + 32 * 2.0 ** -23 * (z.abs().amax() + 20)
    p = torch.exp(z - lse[:, None])
    off = p * 2 * dz
    p[torch.arange(period), targets] -= 1
    G, off = p * d_ce.double()[:, None], off * d_ce.double().abs()[:, None]
    off += 2.0 ** -8 * (G.abs() + off)
    want = G @ w
    off = (off @ w.abs() + vocab * 2.0 ** -23 * (G.abs() @ w.abs()) + 2.0 ** -8 * want.abs() + 1e-37) * (1 + 2.0 ** -8)
    assert ((dH[:period].double().cpu() - want).abs() <= off).all()
    blocks = dH.view(tokens // period, period, d)
    for first in range(0, tokens // period, 2 ** 14):
        assert (blocks[first:first + 2 ** 14] == blocks[:1]).all(), first
    del dH, blocks
    torch.cuda.empty_cache()
