"""The output head where offsets pass 32 bits: buffers of more than 2^32 bytes, results of more than 2^32 values.

Most words of the large vocabulary have rows of zeros, whose logits are 0, so the formulas need the others' rows alone.  The bounds are those of
the small cases: a logit is off by dz <= d 2^-23 sum |h w|, a loss by two of those and 32 steps of its terms, G by 2^-8 relative for its rounding, a
gradient by that, its additions and 2^-8 relative for its own."""
import pytest
import torch

from gpu_util import DEV, sbn

pytestmark = pytest.mark.gpu

HALF, STEP = 2.0 ** -8, 2.0 ** -23


@pytest.mark.parametrize("tokens", [3, 40, 70])
def test_weights_of_more_than_4_gigabytes(tokens):
    s = sbn()
    vocab, d, some = 300000, 8192, 300
    g = torch.Generator().manual_seed(tokens)
    H = torch.randn(tokens, d, generator=g).bfloat16()
    rows = torch.cat((torch.arange(some), torch.arange(vocab - some, vocab)))
    Wn = (torch.randn(2 * some, d, generator=g) * 4 / d ** 0.5).bfloat16()
    at = torch.randint(some, 2 * some, (tokens,), generator=g)      # targets among the last words
    d_ce = torch.randn(tokens, generator=g) * 0.1
    W = torch.zeros(vocab, d, dtype=torch.bfloat16, device=DEV)
    W[rows.to(DEV)] = Wn.to(DEV)
    assert W.numel() > 2 ** 31 and W.numel() * 2 > 2 ** 32
    ce, lse = torch.full((2, tokens), float("nan"), device=DEV)
    dH, dW = torch.full((tokens, d), float("nan"), dtype=torch.bfloat16, device=DEV), torch.full_like(W, float("nan"))
    ws = s.new_workspace(s.sbn_head_workspace_bytes(tokens, d, vocab))
    x, y, grad = H.to(DEV), rows[at].to(DEV), d_ce.to(DEV)
    s.sbn_head_cross_entropy(x, W, y, ce, lse, ws)
    s.sbn_head_cross_entropy_backward(x, W, y, lse, grad, ws, dH=dH, dW=dW)
    torch.cuda.synchronize()

    H, Wn, t = H.double(), Wn.double(), torch.arange(tokens)
    z = H @ Wn.t()
    dz = d * STEP * (H.abs() @ Wn.abs().t()).amax()
    want = torch.log(z.exp().sum(1) + vocab - 2 * some)
    arith = 32 * STEP * (z.abs().amax() + 20)
    assert ((lse.cpu().double() - want).abs() <= 2 * dz + arith).all()
    assert ((ce.cpu().double() - (want - z[t, at])).abs() <= 2 * dz + arith).all()
    w, p = d_ce.double()[:, None], torch.exp(z - want[:, None])
    dG = w.abs() * p * 2 * (dz + arith)
    p[t, at] -= 1
    G, rest = w * p, w * torch.exp(-want)[:, None]
    dG += HALF * (G.abs() + dG) + 1e-37
    d_rest = rest.abs() * (2 * (dz + arith) + HALF * 1.01)

    def near(got, value, off):
        assert ((got.cpu().double() - value).abs() <= (off + HALF * value.abs() + 1e-37) * (1 + HALF)).all()
    near(dH, G @ Wn, dG @ Wn.abs() + vocab * STEP * (G.abs() @ Wn.abs()))
    near(dW[rows.to(DEV)], G.t() @ H, dG.t() @ H.abs() + tokens * STEP * (G.abs().t() @ H.abs()))
    for first in (some, 2 ** 32 // (2 * d) - 2, vocab - some - 8):
        near(dW[first:first + 8], rest.t() @ H, d_rest.t() @ H.abs() + tokens * STEP * (rest.abs().t() @ H.abs()))
    assert not dW.isnan().any()


def test_codes_of_more_than_4_billion_values():
    s = sbn()
    rows, cols = 270000, 16384
    assert rows * cols > 2 ** 32
    g = torch.Generator().manual_seed(5)
    X = torch.randn(rows, 1, generator=g).bfloat16().to(DEV) * torch.randn(1, cols, generator=g).bfloat16().to(DEV)

    def there_and_back(x):
        nc, ns = s.sbn_mxfp4_bytes(*x.shape)
        codes, scales = torch.full((nc,), 0xee, dtype=torch.uint8, device=DEV), torch.full((ns,), 0xee, dtype=torch.uint8, device=DEV)
        s.sbn_mxfp4_quantize(x, codes, scales)
        y = torch.full_like(x, float("nan"))
        s.sbn_mxfp4_dequantize(codes, scales, y)
        return codes.view(len(x), -1), scales.view(len(x), -1), y
    whole = there_and_back(X)
    for first in (0, 2 ** 31 // cols - 2, 2 ** 32 // cols - 2, rows - 5):
        for a, b in zip(whole, there_and_back(X[first:first + 5].contiguous())):
            assert torch.equal(a[first:first + 5], b)


def test_product_of_more_than_4_billion_values():
    # small integers: products and sums are exact in any order
    s = sbn()
    tokens, d_in, d_out = 32768, 64, 140000
    assert tokens * d_out > 2 ** 32
    g = torch.Generator().manual_seed(6)
    X = torch.randint(-2, 3, (tokens, d_in), generator=g).bfloat16()
    W = torch.randint(-2, 3, (d_out, d_in), generator=g).bfloat16()
    X[:, ::32], W[:, ::32] = 4, 4        # the largest of a block: its scale is 1
    nc, ns = s.sbn_mxfp4_bytes(d_out, d_in)
    codes, scales = torch.empty(nc, dtype=torch.uint8, device=DEV), torch.empty(ns, dtype=torch.uint8, device=DEV)
    s.sbn_mxfp4_quantize(W.to(DEV), codes, scales)
    Y = torch.full((tokens, d_out), float("nan"), device=DEV)
    s.sbn_mxfp4_linear(X.to(DEV), codes, scales, Y, s.new_workspace(s.sbn_mxfp4_workspace_bytes(tokens, d_in)))
    for first in (0, 2 ** 31 // d_out - 1, 2 ** 32 // d_out - 1, tokens - 3):
        want = X[first:first + 3].float() @ W.float().t()
        assert torch.equal(Y[first:first + 3].cpu(), want)
    assert not Y.isnan().any()
