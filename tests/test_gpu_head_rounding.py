"""What the rounding of G to bf16 costs the gradients of the output head.

Up to 16 tokens (64 of a distillation) G is taken with what its rounding left over: it is off by 2^-16 relative, so that a gradient has its own
rounding alone.  With more tokens G has a rounding of its own: errors that are independent of each other, uniform over half a step, which
is at most 2^-8 of the value, so of a deviation of at most 2^-8 / sqrt(3) of it."""
import pytest
import torch

from test_gpu_head import BF16_HALF, FP32_STEP, make, reference, run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("alike", [True, False])
@pytest.mark.parametrize("tokens,d,vocab", [(9, 72, 65), (10, 96, 909), (10, 112, 2050), (13, 64, 775), (15, 1000, 129), (16, 128, 20000), (16, 256, 1000)])
def test_gradients_of_up_to_16_tokens_are_rounded_once(tokens, d, vocab, alike):
    case = make(tokens, d, vocab, 900 + tokens)
    case["targets"].clamp_(min=0)
    if alike:
        case["d_ce"].fill_(1 / tokens)
    H, W, w = case["H"].double(), case["W"].double(), case["d_ce"].double()[:, None]
    z = H @ W.t()
    dz = d * FP32_STEP * (H.abs() @ W.abs().t()).amax()
    G = torch.softmax(z, 1)
    dG = G * w.abs() * 2 * (dz + 32 * FP32_STEP * (z.abs().amax() + 20))
    G[torch.arange(tokens), case["targets"]] -= 1
    G *= w
    dG += BF16_HALF ** 2 * (G.abs() + dG) + 1e-37
    got = run(case)
    for name, want, off, terms, size in (("dH", G @ W, dG @ W.abs(), vocab, G.abs() @ W.abs()), ("dW", G.t() @ H, dG.t() @ H.abs(), tokens, G.abs().t() @ H.abs())):
        off = off + 2 * terms * FP32_STEP * size + 1e-37
        off = (off + BF16_HALF * want.abs()) * (1 + BF16_HALF)
        assert not (~((got[name].double().cpu() - want).abs() <= off)).any(), name


@pytest.mark.parametrize("tau", [None, 2.0])
@pytest.mark.parametrize("tokens,d,vocab", [(65, 256, 2000), (512, 200, 3000), (2048, 128, 1000)])
def test_gradients_of_many_tokens_have_two_roundings(tokens, d, vocab, tau):
    # d_ce and d_kd of any values
    case = make(tokens, d, vocab, 1100 + tokens, top=7)
    ref, got = reference(case, tau), run(case, tau)
    rounding = reference_G(case, tau)
    for name, other, G in (("dH", case["W"], rounding), ("dW", case["H"], rounding.t())):
        want = ref[name]
        least = (want.bfloat16().double() - want).norm()
        of_G = BF16_HALF / 3 ** 0.5 * (G.square() @ other.double().square()).sum().sqrt()
        off = (got[name].double().cpu() - want).norm()
        assert off <= 1.1 * (least.square() + of_G.square()).sqrt() + 2.0 ** -12 * want.norm(), name


@pytest.mark.parametrize("tokens", [17, 33, 64])
def test_cross_entropy_of_17_to_64_tokens_has_two_roundings(tokens):
    test_gradients_of_many_tokens_have_two_roundings(tokens, 256, 2000, None)


def reference_G(case, tau):
    """G in 64 bits."""
    H, W = case["H"].double(), case["W"].double()
    tokens, vocab = len(H), len(W)
    z, rows = H @ W.t(), torch.arange(len(H))
    kept = (case["targets"] >= 0) & (case["targets"] < vocab)
    G = torch.softmax(z, 1)
    G[rows[kept], case["targets"][kept]] -= 1
    G *= torch.where(kept, case["d_ce"].double(), 0.0)[:, None]
    if tau is not None:
        P = torch.softmax(z / tau, 1)
        P.scatter_add_(1, case["top_idx"], -torch.softmax(case["top_logits"].double() / tau, 1))
        G += P * (case["d_kd"].double() * tau)[:, None]
    return G
