"""Embedding and its gradient on the GPU.

A looked-up row is one product and one rounding: equal to fp32 arithmetic.  The gradient of a row that n tokens name is a sum of n fp32 values, in runs:
no more than n additions, each off by at most 2^-24 of the sum of magnitudes; then a product, an addition where dE is added to, and a rounding."""
import pytest
import torch

from gpu_util import DEV, sbn

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
BF16, F32 = torch.bfloat16, torch.float32
TYPES = [(BF16, BF16), (F32, BF16), (BF16, F32), (F32, F32)]


def some_ids(T, V, g, often=0.3, out=0.2):
    ids = torch.randint(0, V, (T,), generator=g)
    ids[torch.rand(T, generator=g) < often] = V // 2
    ids[torch.rand(T, generator=g) < out] = -100
    ids[torch.rand(T, generator=g) < out / 4] = V            # the first that is outside, and far ones
    ids[torch.rand(T, generator=g) < out / 4] = (1 << 40) + 1
    ids[torch.rand(T, generator=g) < out / 8] = -(1 << 63)
    return ids


@pytest.mark.parametrize("table,out", TYPES)
@pytest.mark.parametrize("T,V,d", [(1, 1, 1), (3, 5, 7), (5, 100, 64), (70, 1000, 1000), (33, 77, 1001), (9, 4, 5000)])
def test_lookup(T, V, d, table, out):
    g = torch.Generator().manual_seed(T)
    E, ids = torch.randn(V, d, generator=g).to(table), some_ids(T, V, g)
    Y = torch.full((T, d), float("nan"), dtype=out, device=DEV)
    sbn().sbn_embedding(E.to(DEV), ids.to(DEV), Y, scale=1.7)
    inside = (ids >= 0) & (ids < V)
    want = torch.where(inside[:, None], E[torch.where(inside, ids, 0)].float() * 1.7, 0.0).to(out)
    assert torch.equal(Y.cpu(), want)


def test_a_left_out_token_is_zeros_whatever_the_table_holds():
    E = torch.full((4, 40), float("nan"), device=DEV)
    E[1] = 2.0
    Y = torch.full((3, 40), 5.0, device=DEV)
    sbn().sbn_embedding(E, torch.tensor([-1, 1, 4], device=DEV), Y)
    assert (Y[0] == 0).all() and (Y[1] == 2).all() and (Y[2] == 0).all()


def check_gradient(dY, ids, V, table, scale=1.3, old=None, more=0):
    """more: tokens besides that have no share; many tokens go another way than few."""
    s = sbn()
    dY, ids = torch.cat([dY, dY.new_full((more, dY.shape[1]), float("nan"))]), torch.cat([ids, torch.full((more,), -1)])
    T, d = dY.shape
    dE = torch.full((V, d), float("nan"), dtype=table, device=DEV) if old is None else old.to(DEV)
    ws = s.new_workspace(s.sbn_embedding_workspace_bytes(T, d, V)).fill_(0xff)
    idd, dyd = ids.to(DEV), dY.to(DEV)
    s.sbn_embedding_backward(dyd, idd, dE, ws, scale=scale, accumulate=old is not None)
    inside = (ids >= 0) & (ids < V)
    at, some = ids[inside], dY[inside].double()
    scale = float(torch.tensor(scale, dtype=F32))
    total = torch.zeros(V, d, dtype=torch.float64).index_add_(0, at, some) * scale
    size = torch.zeros(V, d, dtype=torch.float64).index_add_(0, at, some.abs()) * scale
    count = torch.zeros(V, dtype=torch.float64).index_add_(0, at, torch.ones(len(at), dtype=torch.float64))[:, None]
    tol = U * (count + 2) * size
    if old is not None:
        total = total + old.double()
        tol = tol + 2 * U * total.abs()
        assert torch.equal(dE.cpu()[count[:, 0] == 0], old[count[:, 0] == 0])
    tol = tol + torch.finfo(table).eps / 2 * (total.abs() + tol)
    off = (dE.double().cpu() - total).abs()
    assert torch.isfinite(off).all() and (off <= tol).all(), (off - tol).max()
    assert old is not None or (dE.cpu()[count[:, 0] == 0] == 0).all()
    other = torch.full((V, d), float("nan"), dtype=table, device=DEV) if old is None else old.to(DEV)
    s.sbn_embedding_backward(dyd, idd, other, ws.fill_(0x33), scale=scale, accumulate=old is not None)
    assert torch.equal(other, dE)
    return dE


@pytest.mark.parametrize("table,out", TYPES)
@pytest.mark.parametrize("T,V,d", [(1, 1, 1), (2, 3, 5), (16, 4, 64), (17, 300, 40), (100, 50, 1001), (500, 2000, 264), (9000, 700, 72), (20000, 30, 33), (300, 70000, 8),
                                   (1536, 300, 1001), (1537, 300, 1001), (2100, 3000, 264), (1500, 9, 2563), (1000, 40, 12), (64, 2, 8), (400, 390, 9000)])
def test_gradient(T, V, d, table, out):
    g = torch.Generator().manual_seed(T + V)
    dY, ids = torch.randn(T, d, generator=g).to(out), some_ids(T, V, g)
    for more in (0, 1600) if T <= 1536 else (0,):
        check_gradient(dY, ids, V, table, more=more)
        check_gradient(dY, ids, V, table, old=torch.randn(V, d, generator=g).to(table), more=more)


@pytest.mark.parametrize("T", [1, 15, 16, 17, 31, 32, 33, 48, 1000, 1535, 1536, 1537, 8191, 8193, 16384, 16385, 40000])
def test_one_id_for_all_and_none(T):
    g = torch.Generator().manual_seed(T)
    dY = torch.randn(T, 24, generator=g)
    for more in (0, 1600):
        check_gradient(dY, torch.full((T,), 5), 9, F32, more=more)
        check_gradient(dY, torch.full((T,), -1), 9, F32, more=more)
    check_gradient(dY, torch.full((T,), 9), 9, F32, old=torch.randn(9, 24, generator=g))


def test_runs_that_end_where_pieces_do():
    """Ids whose tokens fill pieces of the order exactly, reach over one border, or over several."""
    g = torch.Generator().manual_seed(2)
    for lengths in ([16, 16, 16], [8, 8, 17, 15, 16], [1, 47, 1, 32, 31, 1], [15, 2, 15, 16, 33], [64, 1, 1, 14, 160], [15, 17, 16, 1, 31, 2], [15, 18, 15], [1, 31, 1, 32, 1, 30, 17],
                    [16, 32, 33, 32, 31], [15, 33, 5, 300, 3]):
        # ids that lie in one block's share of the vocabulary are neighbours in the order
        ids = torch.cat([torch.full((n,), 256 * k) for k, n in enumerate(lengths)])
        ids = ids[torch.randperm(len(ids), generator=g)]
        dY = torch.randn(len(ids), 40, generator=g)
        for more in (0, 1600):
            check_gradient(dY, ids, 256 * len(lengths), F32, more=more)


def test_left_out_tokens_may_hold_anything():
    ids = torch.tensor([1, -1, 1, 2])
    dY = torch.ones(4, 16)
    dY[1] = float("nan")
    dE = torch.empty(4, 16, device=DEV)
    sbn().sbn_embedding_backward(dY.to(DEV), ids.to(DEV), dE, sbn().new_workspace(sbn().sbn_embedding_workspace_bytes(4, 16, 4)))
    assert (dE.cpu() == torch.tensor([0.0, 2.0, 1.0, 0.0])[:, None]).all()


def test_large_vocabularies():
    """Vocabularies whose ids share out to more blocks than there are processors, to 2^24."""
    g = torch.Generator().manual_seed(4)
    for V in ((1 << 22) + 3, 1 << 24):
        ids = torch.cat([torch.randint(0, V, (3000,), generator=g), torch.tensor([0, V - 1, V, V - 2, 1]).repeat(20)])
        check_gradient(torch.randn(len(ids), 3, generator=g), ids, V, F32)


def test_offsets_past_32_bits():
    """A table and rows of more than 2^32 values."""
    s = sbn()
    V, d = 1 << 19, 8200
    E = torch.zeros(V, d, dtype=BF16, device=DEV)
    E[V - 1] = 3.0
    ids = torch.tensor([V - 1, 5, V - 1], device=DEV)
    Y = torch.empty(3, d, dtype=BF16, device=DEV)
    s.sbn_embedding(E, ids, Y)
    assert (Y[0] == 3).all() and (Y[1] == 0).all()
    Y[1] = 2.0
    E.fill_(float("nan"))
    s.sbn_embedding_backward(Y, ids, E, s.new_workspace(s.sbn_embedding_workspace_bytes(3, d, V)))
    assert (E[V - 1] == 6).all() and (E[5] == 2).all() and E.view(-1).view(torch.int16).count_nonzero() == 2 * d
    del E
    T = (1 << 19) + 1
    dY = torch.zeros(T, d, dtype=BF16, device=DEV)
    dY[T - 1] = 1.5
    dE = torch.empty(7, d, device=DEV)
    s.sbn_embedding_backward(dY, torch.arange(T, device=DEV) % 7, dE, s.new_workspace(s.sbn_embedding_workspace_bytes(T, d, 7)))
    assert dE.count_nonzero() == d and (dE[(T - 1) % 7] == 1.5).all()


def test_rows_at_odd_addresses_and_what_lies_around_them():
    s = sbn()
    g = torch.Generator().manual_seed(6)
    for dtype in (BF16, F32):
        V, d, T = 11, 45, 30
        dY, ids = torch.randn(T, d, generator=g).to(dtype), some_ids(T, V, g)
        want = check_gradient(dY, ids, V, dtype)
        buf = torch.full((V * d + 16,), 77.0, dtype=dtype, device=DEV)
        dE = buf[3:3 + V * d].view(V, d)
        s.sbn_embedding_backward(dY.to(DEV), ids.to(DEV), dE, s.new_workspace(s.sbn_embedding_workspace_bytes(T, d, V)), scale=1.3)
        assert torch.equal(dE, want) and (buf[:3] == 77).all() and (buf[3 + V * d:] == 77).all()
