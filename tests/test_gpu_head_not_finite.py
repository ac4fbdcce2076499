"""Losses of the output head where logits are not finite: a NaN or +inf among a token's or its teacher's logits makes its loss NaN, one of -inf has no
share."""
import pytest
import torch

from gpu_util import sbn
from test_gpu_head import check, make, reference, run

pytestmark = pytest.mark.gpu


@pytest.fixture(params=[0, 1, 2])
def tiles(request):
    sbn().sbn_test_set_head_tiles(request.param, request.param)
    yield
    sbn().sbn_test_set_head_tiles()


def losses(case, tau, **over):
    return {k: v.cpu() for k, v in run({**case, **over}, tau).items() if k in ("ce", "kd", "lse1", "lse2")}


# one word in a last part of its own; whole parts, wherever tiles of 64, 128 and 256 begin; a word among others; all words
@pytest.mark.parametrize("words", [slice(256, 257), slice(0, 128), slice(128, 256), slice(32, 64), slice(70, 71), slice(0, 257)])
@pytest.mark.parametrize("value", [float("nan"), float("inf")])
def test_words_that_are_not_finite(words, value, tiles):
    case = make(9, 64, 257, 1, top=5)
    case["H"][:, 0], case["W"][:, 0] = 1.0, 0.0       # (an infinity reaches the logit as such)
    case["targets"][:] = torch.arange(9) + 3
    case["top_idx"][:] = torch.arange(5) + 20
    before = losses(case, 2.0)
    check(before, reference(case, 2.0))
    W = case["W"].clone()
    W[words, 0] = value
    for tau in (None, 2.0):
        got = losses(case, tau, W=W)
        assert len(got) == (2 if tau is None else 4)
        for name, x in got.items():
            assert x.isnan().all(), (name, x)


def test_a_token_that_is_not_finite(tiles):
    case = make(9, 64, 300, 2, top=5)
    case["targets"][:] = torch.arange(9)
    H = case["H"].clone()
    H[4, 7] = float("nan")
    for tau in (None, 2.0):
        want, got = losses(case, tau), losses(case, tau, H=H)
        others = torch.arange(9) != 4
        for name in want:
            assert got[name][4].isnan() and torch.equal(got[name][others], want[name][others]), name


def test_words_of_minus_infinity_have_no_share(tiles):
    case = make(9, 64, 300, 3, top=5)
    case["H"][:, 0], case["W"][:, 0] = 1.0, 0.0
    case["targets"][:], case["top_idx"][:] = torch.arange(9), torch.arange(5)
    W = case["W"].clone()
    W[200:, 0] = -float("inf")
    short = {**case, "W": case["W"][:200].contiguous()}
    check(losses(case, 2.0, W=W), reference(short, 2.0))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("value", [float("nan"), float("inf")])
@pytest.mark.parametrize("top,entries", [(1, slice(0, 1)), (5, slice(2, 3)), (5, slice(0, 5)), (130, slice(129, 130))])
def test_teacher_logits_that_are_not_finite(top, entries, value, dtype):
    case = make(9, 64, 300, 4, top=top, dtype=dtype)
    broken = {**case, "top_logits": case["top_logits"].clone()}
    broken["top_logits"][4, entries] = value
    want, got = run(case, 2.0), run(broken, 2.0)
    others = torch.arange(9) != 4
    assert got["kd"][4].isnan() and torch.equal(got["kd"][others], want["kd"][others])
    assert got["dH"][4].isnan().all() and torch.equal(got["dH"][others], want["dH"][others])
    assert got["dW"][case["top_idx"][4]].isnan().all()
    for name in ("ce", "lse1", "lse2"):
        assert torch.equal(got[name], want[name]), name
    # of an entry that is missing it is not looked at
    broken["top_idx"] = case["top_idx"].clone()
    broken["top_idx"][4, entries] = 300
    check(run(broken, 2.0), reference(broken | {"top_logits": case["top_logits"]}, 2.0))


@pytest.mark.parametrize("tokens", [2, 5, 8])
def test_gradients_beyond_the_range_of_bf16_are_infinite(tokens):
    # d_ce 3.4e38 lies between the largest bf16 and infinity, nearer the latter, and the first token's 1.0 leaves the common factor at 1: G is
    # infinite at the last token's target, and what its rounding left over must not make a NaN of that
    case = make(tokens, 64, 1000, 5)
    last = tokens - 1
    case["targets"][:] = torch.arange(tokens) + 10
    case["targets"][last] = 3
    case["d_ce"][:] = 1.0
    case["d_ce"][last] = 3.4e38
    case["H"][last] = torch.where(case["H"][last] == 0, 1.0, case["H"][last])
    case["W"][3] = -case["W"][3].abs().clamp(min=0.01) * case["H"][last].sign() * 4    # an unlikely target: its softmax is nearly 0
    assert torch.softmax(case["H"].double() @ case["W"].double().t(), 1)[last, 3] < 1e-4
    assert torch.tensor(3.4e38).bfloat16().isinf()
    got = run(case)
    infinite = torch.tensor(float("inf"))
    assert torch.equal(got["dW"][3].float().cpu(), -infinite * case["H"][last].float())
    assert torch.equal(got["dH"][last].float().cpu(), -infinite * case["W"][3].float())
    assert got["dH"][:last].isfinite().all() and got["dW"][10:10 + last].isfinite().all()
