"""Refusals and workspace sizes of the output head, on the CPU: every argument error is found before anything is launched, so no pointer below is
ever read."""
import ctypes

import pytest
import torch

import paper_2603_05168_amd as sbn
from paper_2603_05168_amd.binding import _lib

P = 1 << 20   # an address that is aligned to everything


def head(backward=False, teacher=False, **over):
    a = dict(H=P, W=P, targets=P, top_idx=P, top_logits=P, dtype=sbn.SBN_F32, top_k=8, tau=2.0, tokens=10, d_in=64, vocab=100, kd=P, ce=P, lse=P, d_kd=P, d_ce=P,
             dH=P, dW=P, ws=P, nbytes=0) | over
    size = (a["tokens"], a["d_in"], a["vocab"])
    tail = (a["ws"], a["nbytes"], None)
    if not teacher:
        if not backward:
            return _lib.sbn_head_cross_entropy(a["H"], a["W"], a["targets"], *size, a["ce"], a["lse"], *tail)
        return _lib.sbn_head_cross_entropy_backward(a["H"], a["W"], a["targets"], a["lse"], a["d_ce"], *size, a["dH"], a["dW"], *tail)
    t = (a["top_idx"], a["top_logits"], a["dtype"], a["top_k"], a["tau"], a["targets"])
    if not backward:
        return _lib.sbn_head_distill(a["H"], a["W"], *t, *size, a["kd"], a["ce"], a["lse"], *tail)
    return _lib.sbn_head_distill_backward(a["H"], a["W"], *t, a["lse"], a["d_kd"], a["d_ce"], *size, a["dH"], a["dW"], *tail)


CALLS = [(b, t) for b in (False, True) for t in (False, True)]


@pytest.mark.parametrize("backward,teacher", CALLS)
def test_head_refusals(backward, teacher):
    call = lambda **over: head(backward, teacher, **over)   # noqa: E731
    assert call() == sbn.SBN_ESIZE   # all is well but for the workspace of no bytes
    for name in ["H", "W", "lse", "ws"] + (["top_idx", "top_logits"] if teacher else ["targets"]):
        assert call(**{name: None}) == sbn.SBN_EINVAL, name
    for name in ("tokens", "d_in", "vocab"):
        assert call(**{name: 0}) == sbn.SBN_EINVAL and call(**{name: -8}) == sbn.SBN_EINVAL, name
    assert call(d_in=60) == sbn.SBN_EUNSUPPORTED and call(d_in=(1 << 16) + 8) == sbn.SBN_EUNSUPPORTED
    assert call(tokens=(1 << 24) + 1) == sbn.SBN_EUNSUPPORTED and call(vocab=(1 << 24) + 1) == sbn.SBN_EUNSUPPORTED
    assert call(tokens=1 << 62) == sbn.SBN_EUNSUPPORTED
    assert call(tokens=1 << 20, vocab=(1 << 18) + 1, d_in=8) == sbn.SBN_EUNSUPPORTED and call(tokens=1 << 20, vocab=1 << 18, d_in=8) == sbn.SBN_ESIZE
    assert call(tokens=1 << 19, d_in=(1 << 15) + 8) == sbn.SBN_EUNSUPPORTED and call(vocab=1 << 19, d_in=(1 << 15) + 8) == sbn.SBN_EUNSUPPORTED
    for name in ("H", "W"):
        assert call(**{name: P + 8}) == sbn.SBN_EALIGN, name
    assert call(ws=P + 128) == sbn.SBN_EALIGN and call(targets=P + 4) == sbn.SBN_EALIGN
    if backward:
        assert call(dH=None, dW=None) == sbn.SBN_EINVAL
        assert call(dH=None) == sbn.SBN_ESIZE and call(dW=None) == sbn.SBN_ESIZE
        assert call(dH=P + 8) == sbn.SBN_EALIGN and call(dW=P + 2) == sbn.SBN_EALIGN
    if teacher:
        for tau in (0.0, -1.0, float("inf"), float("nan")):
            assert call(tau=tau) == sbn.SBN_EINVAL, tau
        assert call(top_k=0) == sbn.SBN_EINVAL and call(top_k=1025) == sbn.SBN_EUNSUPPORTED and call(dtype=2) == sbn.SBN_EINVAL
        assert call(vocab=(1 << 21) + 1) == sbn.SBN_EUNSUPPORTED
        assert call(top_idx=P + 4) == sbn.SBN_EALIGN and call(top_logits=P + 2) == sbn.SBN_EALIGN
        assert call(top_logits=P + 2, dtype=sbn.SBN_BF16) == sbn.SBN_ESIZE
        hard = "d_ce" if backward else "ce"
        assert call(targets=None) == sbn.SBN_EINVAL and call(**{hard: None}) == sbn.SBN_EINVAL   # both or neither
        assert call(**{"targets": None, hard: None}) == sbn.SBN_ESIZE
    need = sbn.sbn_head_workspace_bytes(10, 64, 100, 8 if teacher else 0, backward=backward)
    assert call(nbytes=need - 1) == sbn.SBN_ESIZE


def test_head_workspace_grows_and_refuses():
    small = sbn.sbn_head_workspace_bytes(16, 64, 1000, backward=False)
    assert 0 < small <= sbn.sbn_head_workspace_bytes(16, 64, 1000, backward=True)
    assert small < sbn.sbn_head_workspace_bytes(16, 64, 1000, top_k=8, backward=False)
    # no logits are kept: far less than their bytes, and in pieces for the gradients
    tokens, vocab = 16384, 131072
    assert sbn.sbn_head_workspace_bytes(tokens, 2560, vocab, backward=False) < tokens * vocab // 8
    assert sbn.sbn_head_workspace_bytes(tokens, 2560, vocab, backward=True) < tokens * vocab * 2 // 4
    for bad in ((0, 64, 10, 0), (1, 0, 10, 0), (1, 64, 0, 0), (1, 64, 10, -1), (1, 63, 10, 0), (1 << 25, 64, 10, 0)):
        with pytest.raises(sbn.SbnError):
            sbn.sbn_head_workspace_bytes(*bad)


def test_head_tensors_are_checked():
    H, W = torch.zeros(4, 64, dtype=torch.bfloat16), torch.zeros(10, 64, dtype=torch.bfloat16)
    y, f, ws = torch.zeros(4, dtype=torch.int64), torch.zeros(4), torch.zeros(256, dtype=torch.uint8)
    for bad in ((H.float(), W, y, f, f), (H, W.half(), y, f, f), (H, W, y.int(), f, f), (H, W, y, f.double(), f)):
        with pytest.raises(TypeError):
            sbn.sbn_head_cross_entropy(*bad, ws)
    for bad in ((H, W[:, :32], y, f, f), (H, W, y[:3], f, f), (H, W, y, torch.zeros(8)[::2], f), (torch.zeros(4, 128, dtype=torch.bfloat16)[:, :64], W, y, f, f)):
        with pytest.raises(ValueError):
            sbn.sbn_head_cross_entropy(*bad, ws)
    idx, a = torch.zeros(4, 3, dtype=torch.int64), torch.zeros(4, 3)
    with pytest.raises(ValueError):
        sbn.sbn_head_distill(H, W, idx, a[:, :2], 1.0, f, torch.zeros(2, 4), ws)
    with pytest.raises(TypeError):
        sbn.sbn_head_distill(H, W, idx.int(), a, 1.0, f, torch.zeros(2, 4), ws)


def test_mxfp4_refusals():
    q = lambda **o: (lambda a: _lib.sbn_mxfp4_quantize(a["X"], a["dt"], a["rows"], a["cols"], a["codes"], a["scales"], None))(   # noqa: E731
        dict(X=P, dt=0, rows=4, cols=64, codes=P, scales=P) | o)
    d = lambda **o: (lambda a: _lib.sbn_mxfp4_dequantize(a["codes"], a["scales"], a["rows"], a["cols"], a["X"], a["dt"], None))(   # noqa: E731
        dict(X=P, dt=0, rows=4, cols=64, codes=P, scales=P) | o)
    for call in (q, d):
        for name in ("X", "codes", "scales"):
            assert call(**{name: None}) == sbn.SBN_EINVAL
        assert call(dt=2) == sbn.SBN_EINVAL and call(rows=0) == sbn.SBN_EINVAL and call(cols=-8) == sbn.SBN_EINVAL
        assert call(cols=60) == sbn.SBN_EUNSUPPORTED and call(cols=(1 << 20) + 8) == sbn.SBN_EUNSUPPORTED
        assert call(rows=(1 << 27) + 1) == sbn.SBN_EUNSUPPORTED and call(rows=(1 << 22) + 1, cols=1 << 12) == sbn.SBN_EUNSUPPORTED
        assert call(rows=1 << 62) == sbn.SBN_EUNSUPPORTED
        assert call(X=P + 8) == sbn.SBN_EALIGN and call(codes=P + 8) == sbn.SBN_EALIGN and call(scales=P + 2) == sbn.SBN_EALIGN
    lin = lambda **o: (lambda a: _lib.sbn_mxfp4_linear(a["X"], a["t"], a["k"], a["n"], a["codes"], a["scales"], a["b"], a["Y"], a["ws"], a["nb"], None))(   # noqa: E731
        dict(X=P, t=4, k=64, n=10, codes=P, scales=P, b=None, Y=P, ws=P, nb=0) | o)
    assert lin() == sbn.SBN_ESIZE
    for name in ("X", "codes", "scales", "Y", "ws"):
        assert lin(**{name: None}) == sbn.SBN_EINVAL
    assert lin(t=0) == sbn.SBN_EINVAL and lin(n=0) == sbn.SBN_EINVAL and lin(k=0) == sbn.SBN_EINVAL and lin(k=12) == sbn.SBN_EUNSUPPORTED
    assert lin(n=(1 << 27) + 1) == sbn.SBN_EUNSUPPORTED and lin(t=1 << 19, n=1 << 19) == sbn.SBN_EUNSUPPORTED
    assert lin(X=P + 8) == sbn.SBN_EALIGN and lin(ws=P + 16) == sbn.SBN_EALIGN and lin(b=P + 2) == sbn.SBN_EALIGN and lin(Y=P + 4) == sbn.SBN_EALIGN
    assert lin(nb=sbn.sbn_mxfp4_workspace_bytes(4, 64) - 1) == sbn.SBN_ESIZE


def test_mxfp4_sizes():
    assert sbn.sbn_mxfp4_bytes(3, 128) == (3 * 64, 3 * 4)
    assert sbn.sbn_mxfp4_bytes(3, 136) == (3 * 128, 3 * 8)
    codes = ctypes.c_size_t(0)
    assert _lib.sbn_mxfp4_bytes(3, 128, ctypes.byref(codes), None) == sbn.SBN_EINVAL
    X = torch.zeros(3, 136)
    with pytest.raises(ValueError):
        sbn.sbn_mxfp4_quantize(X, torch.zeros(3 * 68, dtype=torch.uint8), torch.zeros(24, dtype=torch.uint8))
    with pytest.raises(TypeError):
        sbn.sbn_mxfp4_quantize(X.half(), torch.zeros(3 * 128, dtype=torch.uint8), torch.zeros(24, dtype=torch.uint8))
    with pytest.raises(ValueError):
        sbn.sbn_mxfp4_quantize(torch.zeros(136, 3).t(), torch.zeros(3 * 128, dtype=torch.uint8), torch.zeros(24, dtype=torch.uint8))


def test_host_tensors_are_refused_and_declined_by_the_marshalling():
    import paper_2603_05168_amd.binding as b
    H, W = torch.zeros(4, 64, dtype=torch.bfloat16), torch.zeros(10, 64, dtype=torch.bfloat16)
    y, f, ws = torch.zeros(4, dtype=torch.int64), torch.zeros(4), torch.zeros(1 << 16, dtype=torch.uint8)
    idx, a, lse = torch.zeros(4, 3, dtype=torch.int64), torch.zeros(4, 3), torch.zeros(2, 4)
    X, codes, scales, Y = torch.zeros(4, 64, dtype=torch.bfloat16), torch.zeros(10 * 64, dtype=torch.uint8), torch.zeros(40, dtype=torch.uint8), torch.zeros(4, 10)
    for name, fast, args in [
            ("sbn_head_cross_entropy", b._fast_head_ce, (H, W, y, f, f, ws)),
            ("sbn_head_cross_entropy_backward", b._fast_head_ce_backward, (H, W, y, f, f, ws, H, W)),
            ("sbn_head_distill", b._fast_head_distill, (H, W, idx, a, 1.0, f, lse, ws, y, f)),
            ("sbn_head_distill_backward", b._fast_head_distill_backward, (H, W, idx, a, 1.0, lse, f, ws, y, f, H, W)),
            ("sbn_mxfp4_quantize", b._fast_mxfp4_quantize, (W, codes, scales)),
            ("sbn_mxfp4_dequantize", b._fast_mxfp4_dequantize, (codes, scales, W)),
            ("sbn_mxfp4_linear", b._fast_mxfp4_linear, (X, codes, scales, Y, ws, None))]:
        assert fast(*args) is None and fast(*args[:-1]) is None and fast(*args[:-1], 7) is None, name
        with pytest.raises(ValueError, match="GPU"):
            getattr(b, name)(*args)
    assert b._fast_head_bytes(0, 64, 10, 0, 1) is None and b._fast_mxfp4_bytes(1.0, 8) is None and b._fast_mxfp4_workspace_bytes(1 << 70, 8) is None


def test_4bit_products_launch_fewer_than_4_billion_threads():
    """Whatever sizes the call takes; the estimate alone prefers small tiles in some of these."""
    wide = 1 << 27
    for tokens, d_in, d_out in [(513, 64, wide), (512, 64, wide), (511, 64, wide), (577, 128, wide), (1025, 64, wide), (2047, 8, wide), (wide, 8, 2047), (wide, 64, 513),
                                (4161, 1024, 1 << 24), (1 << 19, 64, (1 << 19) - 1), (65, 1 << 20, 1 << 14), (300001, 64, 300001)]:
        size, threads = sbn.sbn_test_chosen_mxfp4_tile(tokens, d_in, d_out)
        edge = (64, 128, 256)[size]
        least = -(-tokens // edge) * -(-d_out // edge) * (512 if size == 2 else 256)
        assert least <= threads < 2 ** 32, (tokens, d_in, d_out, size)
    assert sbn.sbn_test_chosen_mxfp4_tile(128, 2560, 6912)[0] == 0 and sbn.sbn_test_chosen_mxfp4_tile(4096, 2560, 6912)[0] == 2
    for bad in ((0, 64, 64), (64, 63, 64), (1 << 19, 64, 1 << 19)):
        with pytest.raises(sbn.SbnError):
            sbn.sbn_test_chosen_mxfp4_tile(*bad)


@pytest.mark.parametrize("tokens,vocab,top_k,held", [
    (16384, 131072, 0, (2 ** 14, 2 ** 14 + 64)), (2 ** 19, 5000, 0, (2 ** 19, 512 + 64)), (2 ** 20, 5000, 0, (2 ** 20, 256 + 64)), (2 ** 24, 256, 0, (2 ** 24, 256 + 64)),
    (64, 2 ** 24, 0, (64, 2 ** 24)), (16, 2 ** 24, 0, (2 * 16, 2 ** 24)), (64, 2 ** 21, 8, (2 * 64, 2 ** 21))])
def test_head_workspace_holds_one_piece_of_the_gradient_of_the_logits(tokens, vocab, top_k, held):
    # pieces of 2^28 logits or 256 words, rows an odd number of lines apart; of few tokens the vocabulary, with the rests' rows
    nbytes, G = sbn.sbn_head_workspace_bytes(tokens, 8, vocab, top_k), 2 * held[0] * held[1]
    assert G <= nbytes <= G + 4 * 8 * tokens + 2 ** 22   # dH in fp32 over the pieces, splits of few tokens and the teacher's lists
