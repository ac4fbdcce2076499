"""The output head on the GPU: cross entropy and distillation with their gradients against the formulas in 64 bits.

Bounds, element by element.  A product of two bf16 values is exact in fp32 and each of the additions of a sum loses at most 2^-23 of the sum of
the magnitudes (a whole step, whatever the matrix unit's way of rounding), so a logit is off by dz <= d 2^-23 sum |h w|.  A loss adds two such
errors and those of its own fp32 arithmetic (32 steps of its terms).  G is off by the relative error of an exponential, by dz and by 2^-8
relative for its rounding to bf16; the gradients' sums by that, by their additions, and by 2^-8 relative for theirs."""
import pytest
import torch

from gpu_util import DEV, sbn

pytestmark = pytest.mark.gpu

BF16_HALF, FP32_STEP = 2.0 ** -8, 2.0 ** -23


def make(tokens, d, vocab, seed, scale=2.0, top=0, dtype=torch.float32):
    g = torch.Generator().manual_seed(seed)
    H = torch.randn(tokens, d, generator=g).bfloat16()
    W = (torch.randn(vocab, d, generator=g) * scale / d ** 0.5).bfloat16()
    targets = torch.randint(0, vocab, (tokens,), generator=g)
    targets[torch.rand(tokens, generator=g) < 0.2] = -100
    case = {"H": H, "W": W, "targets": targets, "d_ce": torch.randn(tokens, generator=g) * 0.1}
    if top:
        idx = torch.stack([torch.randperm(max(vocab, top), generator=g)[:top] for _ in range(tokens)])   # beyond the vocabulary: missing
        logits = (torch.randn(tokens, top, generator=g) * 3).to(dtype)
        case |= {"top_idx": idx, "top_logits": logits, "d_kd": torch.randn(tokens, generator=g) * 0.1}
    return case


def reference(case, tau=None, hard=True):
    """Losses, gradients and the bounds of both, in 64 bits (on the device where it is large)."""
    H, W = case["H"].double(), case["W"].double()
    (tokens, d), vocab = H.shape, W.shape[0]
    rows = torch.arange(tokens, device=H.device)
    z = H @ W.t()
    dz = d * FP32_STEP * (H.abs() @ W.abs().t()).amax()
    arith = 32 * FP32_STEP * (z.abs().amax() + 20)
    G, dG = torch.zeros_like(z), torch.zeros_like(z)
    out = {}
    if hard:
        y = case["targets"]
        kept = (y >= 0) & (y < vocab)
        at = y.clamp(0, vocab - 1)
        logp = torch.log_softmax(z, 1)
        out["ce"] = torch.where(kept, -logp[rows, at], 0.0)
        out["lse1"] = torch.logsumexp(z, 1)
        w = torch.where(kept, case["d_ce"].double(), 0.0)[:, None]
        p = logp.exp()
        dG += w.abs() * p * 2 * (dz + arith)
        p[rows, at] -= 1.0
        G += w * p
    if tau is not None:
        idx, a = case["top_idx"], case["top_logits"].double() / tau
        valid = (idx >= 0) & (idx < vocab) & (a > -torch.inf)
        a = torch.where(valid, a, -torch.inf)
        some = valid.any(1)
        e = torch.where(valid, torch.exp(a - torch.where(some, a.amax(1), 0.0)[:, None]), 0.0)
        q = torch.zeros(tokens, vocab + 1, dtype=torch.float64, device=H.device)
        q.scatter_add_(1, torch.where(valid, idx, vocab), e / e.sum(1, keepdim=True).clamp(min=1e-300))
        q = q[:, :vocab]
        logp = torch.log_softmax(z / tau, 1)
        out["kd"] = torch.where(some, tau ** 2 * (torch.xlogy(q, q) - q * logp).sum(1), 0.0)
        out["lse2"] = torch.logsumexp(z / tau, 1)
        w = torch.where(some, case["d_kd"].double() * tau, 0.0)[:, None]
        amax = torch.where(valid, a.abs(), 0.0).amax()
        dG += w.abs() * (logp.exp() * 2 * (dz / tau + arith * max(1.0, 1 / tau)) + q * 32 * FP32_STEP * (1 + amax))
        G += w * (logp.exp() - q)
        out["lse2_off"] = 2 * dz / tau + 32 * FP32_STEP * (2 * amax + 2 * z.abs().amax() / tau + 40)
        out["kd_off"] = tau ** 2 * out["lse2_off"]
    out["ce_off"] = 2 * dz + arith
    dG += BF16_HALF * (G.abs() + dG) + 1e-37   # the last: what lies under the smallest normal number
    out["dH"], out["dW"] = G @ W, G.t() @ H
    out["dH_off"] = dG @ W.abs() + vocab * FP32_STEP * (G.abs() @ W.abs()) + BF16_HALF * out["dH"].abs() + 1e-37
    out["dW_off"] = dG.t() @ H.abs() + tokens * FP32_STEP * (G.abs().t() @ H.abs()) + BF16_HALF * out["dW"].abs() + 1e-37
    out["dH_off"] *= 1 + BF16_HALF
    out["dW_off"] *= 1 + BF16_HALF
    return out


def run(case, tau=None, hard=True, dH=True, dW=True):
    s = sbn()
    c = {k: v.to(DEV) for k, v in case.items()}
    (tokens, d), vocab = c["H"].shape, c["W"].shape[0]
    nan = lambda *shape, dtype=torch.float32: torch.full(shape, float("nan"), dtype=dtype, device=DEV)   # noqa: E731
    top = c["top_idx"].shape[1] if tau is not None else 0
    ws = torch.full((s.sbn_head_workspace_bytes(tokens, d, vocab, top),), 0xff, dtype=torch.uint8, device=DEV)   # NaN whatever is read of it
    grads = {"dH": nan(tokens, d, dtype=torch.bfloat16) if dH else None, "dW": nan(vocab, d, dtype=torch.bfloat16) if dW else None}
    out = {}
    if tau is None:
        out["ce"], out["lse1"] = nan(tokens), nan(tokens)
        s.sbn_head_cross_entropy(c["H"], c["W"], c["targets"], out["ce"], out["lse1"], ws)
        ws.fill_(0xff)
        s.sbn_head_cross_entropy_backward(c["H"], c["W"], c["targets"], out["lse1"], c["d_ce"], ws, **grads)
    else:
        out["kd"], lse = nan(tokens), nan(2, tokens)
        more = {"targets": c["targets"]} if hard else {}
        if hard:
            out["ce"] = nan(tokens)
        s.sbn_head_distill(c["H"], c["W"], c["top_idx"], c["top_logits"], tau, out["kd"], lse, ws, ce=out.get("ce"), **more)
        out["lse2"] = lse[1]
        if hard:
            out["lse1"] = lse[0]
        ws.fill_(0xff)
        s.sbn_head_distill_backward(c["H"], c["W"], c["top_idx"], c["top_logits"], tau, lse, c["d_kd"], ws, d_ce=c["d_ce"] if hard else None, **more,
                                    **grads)
    torch.cuda.synchronize()
    return out | {k: v for k, v in grads.items() if v is not None}


def check(got, ref):
    for name, x in got.items():
        want = ref[name].to(x.device)
        off = ref[{"lse1": "ce_off"}.get(name, name + "_off")]
        off = off.to(x.device) if isinstance(off, torch.Tensor) else off
        bad = ~((x.double() - want).abs() <= off)
        assert not bad.any(), f"{name}: {int(bad.sum())} of {bad.numel()} off, worst {(x.double() - want).abs().nan_to_num(1e30).amax().item()}"


SIZES = [(1, 8, 1), (1, 64, 1000), (2, 72, 7), (5, 136, 63), (16, 256, 1000), (33, 64, 129), (37, 1000, 777), (64, 128, 256), (65, 520, 1025), (127, 8, 5001),
         (129, 200, 300), (300, 320, 515), (513, 64, 2049)]


@pytest.mark.parametrize("tokens,d,vocab", SIZES)
def test_cross_entropy(tokens, d, vocab):
    case = make(tokens, d, vocab, 100 + tokens)
    check(run(case), reference(case))


@pytest.mark.parametrize("hard", [True, False])
@pytest.mark.parametrize("tokens,d,vocab,top,tau,dtype", [
    (1, 8, 1, 1, 1.0, torch.float32), (1, 64, 1000, 3, 2.0, torch.bfloat16), (5, 136, 63, 63, 0.5, torch.float32), (16, 256, 1000, 17, 4.0, torch.bfloat16),
    (37, 1000, 777, 7, 1.0, torch.float32), (65, 520, 1025, 64, 2.0, torch.bfloat16), (129, 200, 300, 65, 8.0, torch.float32),
    (300, 320, 5000, 128, 3.0, torch.bfloat16), (6, 64, 4097, 1024, 1.5, torch.float32)])
def test_distillation(tokens, d, vocab, top, tau, dtype, hard):
    case = make(tokens, d, vocab, 200 + tokens, top=top, dtype=dtype)
    case["top_idx"][torch.rand(tokens, generator=torch.Generator().manual_seed(1)) < 0.2] = -1
    check(run(case, tau, hard), reference(case, tau, hard))


@pytest.fixture
def tiles():
    yield sbn().sbn_test_set_head_tiles
    sbn().sbn_test_set_head_tiles()


@pytest.mark.parametrize("size", [0, 1, 2])
@pytest.mark.parametrize("tokens,d,vocab", [(1, 8, 1), (5, 136, 63), (37, 1000, 777), (130, 520, 1025), (300, 64, 515), (700, 200, 130)])
def test_every_tile_size(tokens, d, vocab, size, tiles):
    tiles(size, size)
    case = make(tokens, d, vocab, 1000 + tokens, top=min(vocab, 13))
    check(run(case, 2.0), reference(case, 2.0))
    check(run(case), reference(case))


@pytest.mark.parametrize("tokens,d,vocab", [(1, 8, 1), (3, 64, 5000), (16, 256, 1000), (17, 520, 129), (33, 1000, 777), (64, 136, 4100)])
def test_gradients_of_few_tokens(tokens, d, vocab, tiles):
    tiles(gradients=3)
    case = make(tokens, d, vocab, 1100 + tokens, top=min(vocab, 13))
    check(run(case, 2.0), reference(case, 2.0))
    check(run(case, 2.0, dW=False), reference(case, 2.0))
    check(run(case, dH=False), reference(case))


def test_many_tiles_for_a_block(tiles):
    """More tiles than blocks run at once, of every size: a block's next tile begins under the results of its last one."""
    for size, vocab in ((0, 20000), (1, 40001), (2, 70001)):
        tiles(size, size)
        case = {k: v.to(DEV) for k, v in make(200 if size < 2 else 600, 72, vocab, 1200 + size, top=9).items()}
        check(run(case, 2.0), reference(case, 2.0))


@pytest.mark.parametrize("what", ["all left out", "beyond the vocabulary", "lowest", "far logits", "one kept", "no gradient"])
def test_cross_entropy_masks(what):
    case = make(70, 192, 900, 300)
    if what == "all left out":
        case["targets"][:] = -1
    elif what == "beyond the vocabulary":
        case["targets"][::2] = 900
        case["targets"][1::4] = 2 ** 40
    elif what == "lowest":
        case["targets"][::3] = -2 ** 63
        case["d_ce"][::3] = float("nan")   # of tokens without a share
    elif what == "far logits":
        case["W"] = (case["W"].float() * 40).bfloat16()
    elif what == "one kept":
        case["targets"][:] = -100
        case["targets"][69] = 899
    else:
        case["d_ce"][:] = 0.0
    got, ref = run(case), reference({**case, "d_ce": case["d_ce"].nan_to_num(0.0)})
    check(got, ref)
    if what in ("all left out", "no gradient"):
        assert not got["dH"].any() and not got["dW"].any()
    dropped = ~((case["targets"] >= 0) & (case["targets"] < 900)).to(DEV)
    assert not got["ce"][dropped].any() and not got["dH"][dropped].any()


@pytest.mark.parametrize("what", ["no entry", "-inf", "twice", "beyond the vocabulary", "one token's", "cold", "lowest"])
def test_teacher_masks(what):
    case = make(70, 192, 900, 400, top=20)
    idx, logits, tau = case["top_idx"], case["top_logits"], 1.5
    if what == "no entry":
        idx[:] = -1
    elif what == "-inf":
        logits[::2, 3:] = -torch.inf
        logits[1::4] = -torch.inf
    elif what == "twice":
        idx[:, 7] = idx[:, 2]
        idx[:, 19] = idx[:, 2]
        idx[::3] = 5
    elif what == "beyond the vocabulary":
        idx[::2] = 900
        idx[1::2, 4] = 2 ** 32 + 3   # not word 3
        idx[1::2, 5] = -2 ** 63
    elif what == "one token's":
        idx[:] = torch.arange(20)
    elif what == "cold":
        tau = 0.02
    else:
        logits[:, 5:] = torch.finfo(torch.float32).min   # far below the others: no share
        logits[::2] = torch.finfo(torch.float32).min     # all alike: equal shares
    got, ref = run(case, tau), None
    for_reference = dict(case)
    if what == "lowest":   # the same shares from logits whose differences 64 bits bound sensibly
        for_reference["top_logits"] = torch.where(logits < -1e30, torch.where((logits < -1e30).all(1, keepdim=True), 0.0, -torch.inf), logits)
        for_reference["top_idx"] = idx
    ref = reference(for_reference, tau)
    check(got, ref)
    if what == "no entry":
        assert not got["kd"].any()


@pytest.mark.parametrize("skip", ["dH", "dW"])
def test_one_gradient_alone(skip):
    case = make(90, 128, 700, 500, top=9)
    both = run(case, 2.0)
    one = run(case, 2.0, **{skip: False})
    for k, v in one.items():
        assert torch.equal(v, both[k]), k


def test_vocabulary_in_pieces():
    """More tokens x words than G is held of at a time (2^28): pieces of the vocabulary, dH added up over them."""
    case = {k: v.to(DEV) for k, v in make(70001, 16, 5003, 600, top=5).items()}
    assert 70001 * 5003 > 2 ** 28
    got = run(case, 2.0)
    for first in (0, 35000, 69000):   # tokens of the reference at a time
        rows = slice(first, first + 1001)
        part = {k: v if k == "W" else v[rows] for k, v in case.items()}
        ref = reference(part, 2.0)
        check({k: v[rows] for k, v in got.items() if k != "dW"}, ref)
    total, off = 0.0, 0.0
    for first in range(0, 70001, 8192):
        ref = reference({k: v if k == "W" else v[first:first + 8192] for k, v in case.items()}, 2.0)
        total, off = total + ref["dW"], off + ref["dW_off"]
    check({"dW": got["dW"]}, {"dW": total, "dW_off": off * 9})   # additions of nine times as many terms


def test_gradients_against_differences():
    """The derivative along a direction from differences of the loss in 64 bits."""
    case, tau = make(60, 64, 500, 700, top=11), 2.0
    got, ref = run(case, tau), reference(case, tau)
    g = torch.Generator().manual_seed(5)
    for name, grad in (("H", "dH"), ("W", "dW")):
        D = torch.randn(case[name].shape, generator=g, dtype=torch.float64)
        eps = 1e-4

        def loss(step):
            moved = {**case, name: case[name].double() + step * D}
            r = reference(moved, tau)
            return (r["ce"] * case["d_ce"].double()).sum() + (r["kd"] * case["d_kd"].double()).sum()

        want = (loss(eps) - loss(-eps)) / (2 * eps)
        have = (got[grad].double().cpu() * D).sum()
        assert abs(want - have) <= (ref[grad + "_off"] * D.abs()).sum() + 1e-6 * abs(want)


def test_repeats_bit_for_bit_and_on_another_stream():
    case = make(200, 136, 3000, 800, top=10)
    first = run(case, 2.0)
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        second = run(case, 2.0)
    for k in first:
        assert torch.equal(first[k], second[k]), k


def test_graph_replay():
    s = sbn()
    case = {k: v.to(DEV) for k, v in make(48, 128, 1500, 900, top=6).items()}
    eager = run(case, 2.0)
    tokens, d, vocab = 48, 128, 1500
    ws = s.new_workspace(s.sbn_head_workspace_bytes(tokens, d, vocab, 6))
    kd, ce, lse = torch.zeros(tokens, device=DEV), torch.zeros(tokens, device=DEV), torch.zeros(2, tokens, device=DEV)
    dH, dW = torch.zeros_like(case["H"]), torch.zeros_like(case["W"])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        s.sbn_head_distill(case["H"], case["W"], case["top_idx"], case["top_logits"], 2.0, kd, lse, ws, targets=case["targets"], ce=ce)
        s.sbn_head_distill_backward(case["H"], case["W"], case["top_idx"], case["top_logits"], 2.0, lse, case["d_kd"], ws, targets=case["targets"],
                                    d_ce=case["d_ce"], dH=dH, dW=dW)
    for _ in range(3):
        for t in (kd, ce, lse, dH, dW):
            t.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        for k, v in (("kd", kd), ("ce", ce), ("lse1", lse[0]), ("lse2", lse[1]), ("dH", dH), ("dW", dW)):
            assert torch.equal(v, eager[k]), k
        again = run(case, 2.0)
        assert torch.equal(again["dW"], eager["dW"])


def test_marshalling_in_python_gives_the_same(monkeypatch):
    import paper_2603_05168_amd.binding as b
    case = make(40, 128, 900, 950, top=5)
    fast = run(case, 2.0) | {"alone": run(case)["dW"]}
    for name in [n for n in dir(b) if n.startswith("_fast_")]:
        monkeypatch.setattr(b, name, lambda *args: None)
    slow = run(case, 2.0) | {"alone": run(case)["dW"]}
    for k in fast:
        assert torch.equal(fast[k], slow[k]), k


def test_refusals_reach_the_caller():
    s = sbn()
    case = {k: v.to(DEV) for k, v in make(40, 128, 900, 950, top=5).items()}
    f = torch.zeros(40, device=DEV)
    small = s.new_workspace(256)
    for call in (lambda: s.sbn_head_cross_entropy(case["H"], case["W"], case["targets"], f, f, small),
                 lambda: s.sbn_head_distill(case["H"], case["W"], case["top_idx"], case["top_logits"], 2.0, f, torch.zeros(2, 40, device=DEV), small)):
        with pytest.raises(s.SbnError) as e:
            call()
        assert e.value.status == s.SBN_ESIZE
    with pytest.raises(s.SbnError) as e:
        s.sbn_head_distill(case["H"], case["W"], case["top_idx"], case["top_logits"], 0.0, f, torch.zeros(2, 40, device=DEV), small)
    assert e.value.status == s.SBN_EINVAL
    with pytest.raises(ValueError):
        s.sbn_head_cross_entropy(case["H"], case["W"].t().contiguous().t(), case["targets"], f, f, small)


@pytest.mark.parametrize("tokens,d,vocab", [(1, 648, 5674), (2, 648, 5674), (2, 8, 1), (3, 72, 65), (7, 136, 1000), (8, 1000, 129), (8, 128, 20000)])
def test_weight_gradient_of_up_to_eight_tokens_is_rounded_once(tokens, d, vocab):
    # G is taken with what its rounding left over: it is off by 2^-16 relative instead of 2^-8
    case = make(tokens, d, vocab, 900 + tokens)
    case["targets"].clamp_(min=0)
    case["d_ce"].fill_(1 / tokens)
    H, W = case["H"].double(), case["W"].double()
    z = H @ W.t()
    dz = d * FP32_STEP * (H.abs() @ W.abs().t()).amax()
    G = torch.softmax(z, 1)
    dG = G / tokens * 2 * (dz + 32 * FP32_STEP * (z.abs().amax() + 20))
    G[torch.arange(tokens), case["targets"]] -= 1
    G /= tokens
    dG += BF16_HALF ** 2 * (G.abs() + dG) + 1e-37
    want = G.t() @ H
    off = dG.t() @ H.abs() + 2 * tokens * FP32_STEP * (G.abs().t() @ H.abs()) + 1e-37
    off = (off + BF16_HALF * want.abs()) * (1 + BF16_HALF)
    for grads in ({"dH": False}, {}):
        got = run(case, **grads)["dW"].double().cpu()
        assert not (~((got - want).abs() <= off)).any()


def test_weight_gradient_beyond_the_range_of_bf16_stays_infinite():
    # a value that rounds to infinity leaves no rest that would make the sum a NaN
    case = make(1, 64, 1000, 950)
    case["targets"][0] = 3
    case["d_ce"][0] = 3.4e38
    case["W"][3] = -case["W"][3].abs() * case["H"][0].sign() * 4    # an unlikely target: G is nearly -d_ce there
    got = run(case)["dW"].float().cpu()
    assert not got[3].isnan().any() and (got[3].isinf() | (got[3].abs() > 0) | (case["H"][0] == 0)).all()


@pytest.mark.parametrize("hard", [True, False])
@pytest.mark.parametrize("tokens,d,vocab,top", [(2, 64, 1000, 3), (9, 136, 63, 7), (17, 256, 3000, 2), (37, 1000, 5001, 7), (48, 72, 515, 1), (64, 648, 4001, 33)])
def test_gradients_of_a_short_distillation_are_rounded_once(tokens, d, vocab, top, hard):
    # up to 64 tokens G is taken with what its rounding left over, for either product: the errors are those of rounding the results, which are
    # at most 2^-8 relative and 2^-8 / sqrt(3) in the mean of many where all are as large, with room for the rest of the bound
    case, tau = make(tokens, d, vocab, 1000 + tokens, top=top), 2.0
    ref, got = reference(case, tau, hard), run(case, tau, hard)
    for name in ("dH", "dW"):
        want = ref[name]
        once = want.bfloat16().double()
        off, least = (got[name].cpu().double() - want).norm(), (once - want).norm()
        assert off <= 1.1 * least + 2.0 ** -12 * want.norm()
