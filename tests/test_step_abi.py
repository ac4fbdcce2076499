"""Refusals and sizes of norms, embedding and optimizer, on the CPU: every argument error is found before anything is launched, so no pointer below is
ever read."""
import ctypes

import pytest
import torch

import paper_2603_05168_amd as sbn
from paper_2603_05168_amd import binding
from paper_2603_05168_amd.binding import _lib

P = 1 << 20   # an address that is aligned to everything
BF16, F32 = torch.bfloat16, torch.float32


def call(name, defaults, **over):
    a = defaults | over
    assert not set(over) - set(defaults)
    return getattr(_lib, name)(*a.values(), None)


def test_norm_refusals():
    base = dict(X=P, residual=None, dtype=sbn.SBN_BF16, tokens=4, d=63, gain=P, bias=P, eps=1e-6, layer=1, Y=P, sum_out=None)
    for over, want in ((dict(X=None), sbn.SBN_EINVAL), (dict(Y=None), sbn.SBN_EINVAL), (dict(residual=P), sbn.SBN_EINVAL), (dict(sum_out=P), sbn.SBN_EINVAL),
                       (dict(residual=P, sum_out=P), sbn.SBN_EINVAL),   # Y and sum_out in one place
                       (dict(dtype=2), sbn.SBN_EINVAL), (dict(tokens=0), sbn.SBN_EINVAL), (dict(d=0), sbn.SBN_EINVAL), (dict(eps=-1.0), sbn.SBN_EINVAL),
                       (dict(eps=float("nan")), sbn.SBN_EINVAL), (dict(eps=float("inf")), sbn.SBN_EINVAL), (dict(d=16385), sbn.SBN_EUNSUPPORTED),
                       (dict(tokens=(1 << 24) + 1), sbn.SBN_EUNSUPPORTED), (dict(tokens=1 << 62), sbn.SBN_EUNSUPPORTED), (dict(X=P + 1), sbn.SBN_EALIGN),
                       (dict(Y=P + 2, dtype=sbn.SBN_F32), sbn.SBN_EALIGN), (dict(gain=P + 2), sbn.SBN_EALIGN), (dict(bias=P + 1), sbn.SBN_EALIGN),
                       (dict(residual=P + 1, sum_out=P + 8), sbn.SBN_EALIGN)):
        assert call("sbn_norm", base, **over) == want, over
    need = sbn.sbn_norm_workspace_bytes(4, 63)
    base = dict(X=P, dY=P, d_residual=None, dtype=sbn.SBN_BF16, tokens=4, d=63, gain=None, eps=1e-6, layer=0, dX=P, dgain=P, dbias=None, ws=P, nbytes=need - 1)
    assert call("sbn_norm_backward", base) == sbn.SBN_ESIZE
    for over, want in ((dict(X=None), sbn.SBN_EINVAL), (dict(dY=None), sbn.SBN_EINVAL), (dict(ws=None), sbn.SBN_EINVAL), (dict(dX=None, dgain=None), sbn.SBN_EINVAL),
                       (dict(dX=None, d_residual=P), sbn.SBN_EINVAL), (dict(dX=None), sbn.SBN_ESIZE), (dict(dgain=None), sbn.SBN_ESIZE), (dict(ws=P + 128), sbn.SBN_EALIGN),
                       (dict(dX=P + 1), sbn.SBN_EALIGN), (dict(dgain=P + 2), sbn.SBN_EALIGN), (dict(d=16385), sbn.SBN_EUNSUPPORTED)):
        assert call("sbn_norm_backward", base, **over) == want, over
    for bad in ((0, 8), (1, 0), (1, 16385)):
        with pytest.raises(sbn.SbnError):
            sbn.sbn_norm_workspace_bytes(*bad)


def test_embedding_refusals():
    base = dict(E=P, table=sbn.SBN_BF16, vocab=100, d=63, ids=P, tokens=4, scale=1.0, Y=P, rows=sbn.SBN_F32)
    for over, want in ((dict(E=None), sbn.SBN_EINVAL), (dict(ids=None), sbn.SBN_EINVAL), (dict(Y=None), sbn.SBN_EINVAL), (dict(table=2), sbn.SBN_EINVAL),
                       (dict(rows=-1), sbn.SBN_EINVAL), (dict(vocab=0), sbn.SBN_EINVAL), (dict(tokens=-1), sbn.SBN_EINVAL), (dict(d=0), sbn.SBN_EINVAL),
                       (dict(scale=float("inf")), sbn.SBN_EINVAL), (dict(vocab=(1 << 24) + 1), sbn.SBN_EUNSUPPORTED), (dict(tokens=1 << 62), sbn.SBN_EUNSUPPORTED),
                       (dict(d=(1 << 16) + 1), sbn.SBN_EUNSUPPORTED), (dict(vocab=1 << 20, d=(1 << 14) + 1), sbn.SBN_EUNSUPPORTED), (dict(E=P + 1), sbn.SBN_EALIGN),
                       (dict(Y=P + 2), sbn.SBN_EALIGN), (dict(ids=P + 4), sbn.SBN_EALIGN)):
        assert call("sbn_embedding", base, **over) == want, over
    need = sbn.sbn_embedding_workspace_bytes(4, 63, 100)
    base = dict(dY=P, rows=sbn.SBN_BF16, ids=P, tokens=4, vocab=100, d=63, scale=1.0, accumulate=0, dE=P, table=sbn.SBN_F32, ws=P, nbytes=need - 1)
    assert call("sbn_embedding_backward", base) == sbn.SBN_ESIZE
    for over, want in ((dict(dY=None), sbn.SBN_EINVAL), (dict(dE=None), sbn.SBN_EINVAL), (dict(ids=None), sbn.SBN_EINVAL), (dict(ws=None), sbn.SBN_EINVAL),
                       (dict(scale=float("nan")), sbn.SBN_EINVAL), (dict(dE=P + 2), sbn.SBN_EALIGN), (dict(dY=P + 1), sbn.SBN_EALIGN), (dict(ws=P + 64), sbn.SBN_EALIGN),
                       (dict(tokens=1 << 20, d=(1 << 14) + 1), sbn.SBN_EUNSUPPORTED)):
        assert call("sbn_embedding_backward", base, **over) == want, over
    # room for every token's place and for the sums of runs that go on, no more than half the rows' values in fp32
    assert sbn.sbn_embedding_workspace_bytes(16384, 2560, 131072) < 16384 * 2560 * 2 + 131072 * 8
    with pytest.raises(sbn.SbnError):
        sbn.sbn_embedding_workspace_bytes(0, 8, 8)


def pointers(*p):
    return (ctypes.c_void_p * len(p))(*p)


def sizes(*n):
    return (ctypes.c_int64 * len(n))(*n)


def step(over=None, n=(1000, 40), at=(P, P + 4096), bits8=False, decay=(0.0, 0.1)):
    """A call of two tensors that is refused only for what is changed; a step that is not refused would be launched, so beta1 is 1 where nothing else is."""
    lists = {k: pointers(*(a + (i << 30) for a in at)) for i, k in enumerate(("params", "grads", "m", "v", "ms", "vs"))}
    if not bits8:
        lists["ms"] = lists["vs"] = None
    a = dict(count=len(n), params=lists["params"], pt=sbn.SBN_F32, grads=lists["grads"], gt=sbn.SBN_BF16, m=lists["m"], v=lists["v"], ms=lists["ms"], vs=lists["vs"],
             sizes=sizes(*n), decay=(ctypes.c_float * len(n))(*decay), lr=P, step=P, b1=1.0, b2=0.95, eps=1e-8, clip=None, seed=None) | (over or {})
    return _lib.sbn_adamw_step(*a.values(), None)


def test_adamw_refusals():
    assert step() == sbn.SBN_EINVAL   # beta1 of 1
    good = dict(b1=0.9)
    inval = [dict(params=None), dict(grads=None), dict(m=None), dict(v=None), dict(sizes=None), dict(lr=None), dict(step=None), dict(pt=2), dict(gt=-1), dict(b1=-0.1),
             dict(b1=float("nan")), dict(b2=1.0), dict(eps=-1.0), dict(eps=float("nan")), dict(eps=1e300), dict(count=0), dict(count=-1), dict(ms=pointers(P, P + 64)),
             dict(params=pointers(P, None)), dict(grads=pointers(None, P)), dict(decay=(ctypes.c_float * 2)(0.0, float("inf"))), dict(sizes=sizes(1000, 0))]
    for over in inval:
        assert step(good | over) == sbn.SBN_EINVAL, over
    assert step(good | dict(count=4097)) == sbn.SBN_EUNSUPPORTED
    assert step(good | dict(sizes=sizes(1000, (1 << 31) + 1))) == sbn.SBN_EUNSUPPORTED
    for over in (dict(params=pointers(P, P + 4098)), dict(grads=pointers(P + 1, P + 4096)), dict(m=pointers(P + 2, P + 8192)), dict(lr=P + 2), dict(step=P + 4), dict(clip=P + 2)):
        assert step(good | over) == sbn.SBN_EALIGN, over
    assert step(good | dict(m=pointers(P + 4, P + 8192)), bits8=True) == sbn.SBN_EALIGN
    # a tensor that is listed twice, or that reaches into the next, in either order
    for over in (dict(params=pointers(P, P)), dict(params=pointers(P, P + 3996)), dict(params=pointers(P + 100, P)), dict(m=pointers(P, P)), dict(v=pointers(P + 8, P))):
        assert step(good | over) == sbn.SBN_EINVAL, over
    assert step(good | dict(ms=pointers(P, P + 31)), bits8=True) == sbn.SBN_EINVAL
    assert step(good | dict(m=pointers(P, P + 1016)), bits8=True) == sbn.SBN_EINVAL


def test_grad_norm_and_state_refusals():
    need = sbn.sbn_grad_norm_workspace_bytes([1000, 40])
    base = dict(count=2, grads=pointers(P, P + 4096), dtype=sbn.SBN_F32, sizes=sizes(1000, 40), max_norm=1.0, out=P, ws=P, nbytes=need - 1)
    assert call("sbn_grad_norm", base) == sbn.SBN_ESIZE
    for over, want in ((dict(grads=None), sbn.SBN_EINVAL), (dict(out=None), sbn.SBN_EINVAL), (dict(ws=None), sbn.SBN_EINVAL), (dict(count=0), sbn.SBN_EINVAL),
                       (dict(max_norm=0.0), sbn.SBN_EINVAL), (dict(max_norm=float("nan")), sbn.SBN_EINVAL), (dict(sizes=sizes(1000, -1)), sbn.SBN_EINVAL),
                       (dict(grads=pointers(P, None)), sbn.SBN_EINVAL), (dict(grads=pointers(P, P + 2)), sbn.SBN_EALIGN), (dict(ws=P + 8), sbn.SBN_EALIGN),
                       (dict(count=4097), sbn.SBN_EUNSUPPORTED)):
        assert call("sbn_grad_norm", base, **over) == want, over
    assert sbn.sbn_adamw_state_bytes(1) == (32, 1) and sbn.sbn_adamw_state_bytes(65) == (96, 3)
    for bad in (0, -1, (1 << 31) + 1):
        with pytest.raises(sbn.SbnError):
            sbn.sbn_adamw_state_bytes(bad)
    base = dict(codes=P, scales=P, n=40, second=0, out=P, dtype=sbn.SBN_BF16)
    for over, want in ((dict(codes=None), sbn.SBN_EINVAL), (dict(scales=None), sbn.SBN_EINVAL), (dict(out=None), sbn.SBN_EINVAL), (dict(n=0), sbn.SBN_EINVAL),
                       (dict(dtype=3), sbn.SBN_EINVAL), (dict(codes=P + 4), sbn.SBN_EALIGN), (dict(out=P + 1), sbn.SBN_EALIGN)):
        assert call("sbn_adamw_state_values", base, **over) == want, over


def test_tensors_are_checked():
    X, Y, g, ws = torch.zeros(4, 64, dtype=BF16), torch.zeros(4, 64, dtype=BF16), torch.zeros(64), torch.zeros(256, dtype=torch.uint8)
    for bad in (dict(X=X.half()), dict(Y=Y.float()), dict(gain=g.bfloat16()), dict(bias=g.double())):
        with pytest.raises(TypeError):
            sbn.sbn_norm(**(dict(X=X, Y=Y) | bad))
    for bad in (dict(Y=Y[:3]), dict(X=torch.zeros(64, 4, dtype=BF16).t()), dict(gain=g[:32]), dict(residual=X[:, :32]), dict(X=X[0], Y=Y[0]), dict()):
        with pytest.raises(ValueError):   # the last: tensors of the host
            sbn.sbn_norm(**(dict(X=X, Y=Y) | bad))
    with pytest.raises(TypeError):
        sbn.sbn_norm_backward(X, Y, ws, dX=X.float())
    with pytest.raises(ValueError):
        sbn.sbn_norm_backward(X, Y, ws, dgain=g[::2])
    ids, E = torch.zeros(4, dtype=torch.int64), torch.zeros(10, 64)
    with pytest.raises(TypeError):
        sbn.sbn_embedding(E, ids.int(), X)
    for bad in ((E, ids[:3], X), (E[:, :32], ids, X), (E, ids, X)):
        with pytest.raises(ValueError):
            sbn.sbn_embedding(*bad)
    with pytest.raises(ValueError):
        sbn.sbn_embedding_backward(X[:, :32], ids, E, ws)
    with pytest.raises(ValueError):
        sbn.GradNormGroup([], ws)
    with pytest.raises(TypeError):
        sbn.GradNormGroup([g.double()], ws)
    with pytest.raises(ValueError):
        sbn.AdamWGroup([g], [g, g], [g], [g])


class Elsewhere:
    """A tensor of another card, as far as the checks look."""
    is_cuda = True
    device = torch.device("cuda", 3)


def test_tensors_of_another_card_are_refused(monkeypatch):
    monkeypatch.setattr(binding, "_current_device", lambda: 0)
    with pytest.raises(ValueError, match="current device"):
        binding._here(None, Elsewhere())
    monkeypatch.setattr(binding, "_current_device", lambda: 3)
    binding._here(None, Elsewhere())
