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
