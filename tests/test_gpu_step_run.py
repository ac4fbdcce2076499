"""The parts of a training step around the layers and the head together, as a program uses them: a step from tokens to new packed weights against the same
in 64 bits, steps captured into a graph and replayed, several streams, and the two ways that a call is marshalled."""
import numpy as np
import pytest
import torch

import oracle
from gpu_util import DEV, sbn
from paper_2603_05168_amd import binding as b

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32


class Model:
    """Embedding, a norm, one sparse ternary layer added to the residual stream, a norm, and the table again as the output head."""

    def __init__(self, T=64, V=500, d=256, seed=0):
        s = sbn()
        g = torch.Generator().manual_seed(seed)
        self.T, self.V, self.d = T, V, d
        self.ids = torch.randint(0, V, (T,), generator=g).to(DEV)
        self.ids[5:9] = 7
        self.targets = torch.randint(0, V, (T,), generator=g).to(DEV)
        self.ids[-2:], self.targets[-2:] = -100, -100   # padding
        self.E = (torch.randn(V, d, generator=g) * 0.2).to(BF16).to(DEV)
        self.W = (torch.randn(d, d, generator=g) * 0.05).to(BF16).to(DEV)
        self.g1, self.g2 = ((1 + 0.1 * torch.randn(d, generator=g)).to(DEV) for _ in range(2))
        f32 = {"dtype": F32, "device": DEV}
        rows = lambda: torch.empty(T, d, dtype=BF16, device=DEV)   # noqa: E731
        self.x, self.n1, self.h, self.n2, self.yb = rows(), rows(), rows(), rows(), rows()
        self.y, self.ce, self.lse = torch.empty(T, d, **f32), torch.empty(T, **f32), torch.empty(T, **f32)
        self.dn2, self.dh, self.dn1, self.dx = rows(), rows(), rows(), rows()
        self.dE, self.dW = torch.empty(V, d, dtype=BF16, device=DEV), torch.empty(d, d, dtype=BF16, device=DEV)
        self.dg1, self.dg2 = torch.empty(d, **f32), torch.empty(d, **f32)
        self.packed, self.gamma = torch.empty(s.sbn_packed_bytes(d, d, 2, 4), dtype=torch.uint8, device=DEV), torch.empty(1, **f32)
        self.xq, self.sx = torch.empty(T, d, dtype=torch.int8, device=DEV), torch.empty(T, **f32)
        need = max(s.sbn_workspace_bytes(s.SBN_OP_QUANTIZE_MASK_PACK, 1, d, d, 2, 4), s.sbn_workspace_bytes(s.SBN_OP_LINEAR, T, d, d, 2, 4),
                   s.sbn_workspace_bytes(s.SBN_OP_BACKWARD, T, d, d, 2, 4), s.sbn_head_workspace_bytes(T, d, V), s.sbn_norm_workspace_bytes(T, d),
                   s.sbn_embedding_workspace_bytes(T, d, V))
        self.ws = s.new_workspace(need)
        kept = (self.targets >= 0).float()
        self.d_ce = kept / kept.sum()
        self.lr, self.step, self.norm = torch.full((1,), 1e-2, **f32), torch.ones(1, dtype=torch.int64, device=DEV), torch.empty(2, **f32)
        gains, d_gains = [self.g1, self.g2], [self.dg1, self.dg2]
        state = lambda ps: [torch.zeros(p.shape, **f32) for p in ps]   # noqa: E731
        self.gain_states = state(gains), state(gains)
        self.optim_gains = s.AdamWGroup(gains, d_gains, *self.gain_states)
        weights, d_weights = [self.E, self.W], [self.dE, self.dW]
        sizes = [s.sbn_adamw_state_bytes(p.numel()) for p in weights]
        self.codes = [[torch.zeros(n[k], dtype=torch.uint8, device=DEV) for n in sizes] for k in (0, 0, 1, 1)]
        self.optim = s.AdamWGroup(weights, d_weights, *self.codes, weight_decay=[0.0, 0.1])
        self.norms = s.GradNormGroup(d_weights, s.new_workspace(s.sbn_grad_norm_workspace_bytes([p.numel() for p in weights])))

    def forward(self):
        s, d = sbn(), self.d
        s.sbn_embedding(self.E, self.ids, self.x, scale=d ** 0.5)
        s.sbn_quantize_mask_pack(self.W, 2, 4, self.packed, self.gamma, self.ws)
        s.sbn_norm(self.x, self.n1, gain=self.g1)
        s.sbn_sparse_ternary_linear(self.n1, self.packed, self.gamma, self.y, 2, 4, self.ws, xq_out=self.xq, sx_out=self.sx)
        self.yb.copy_(self.y)
        s.sbn_norm(self.yb, self.n2, gain=self.g2, residual=self.x, sum_out=self.h)
        s.sbn_head_cross_entropy(self.n2, self.E, self.targets, self.ce, self.lse, self.ws)

    def backward(self):
        s, d = sbn(), self.d
        s.sbn_head_cross_entropy_backward(self.n2, self.E, self.targets, self.lse, self.d_ce, self.ws, dH=self.dn2, dW=self.dE)
        s.sbn_norm_backward(self.h, self.dn2, self.ws, dX=self.dh, dgain=self.dg2, gain=self.g2)
        s.sbn_sparse_ternary_linear_backward(self.dh, self.packed, self.gamma, self.xq, self.sx, 2, 4, self.ws, d, dX=self.dn1, dW=self.dW)
        s.sbn_norm_backward(self.x, self.dn1, self.ws, dX=self.dx, dgain=self.dg1, gain=self.g1, d_residual=self.dh)
        s.sbn_embedding_backward(self.dx, self.ids, self.dE, self.ws, scale=d ** 0.5, accumulate=True)

    def update(self, seed=None):
        self.norms.run(0.5, self.norm)
        self.optim.run(self.lr, self.step, clip=self.norm[1:], seed=seed)
        self.optim_gains.run(self.lr, self.step)

    def all_steps(self):
        self.forward()
        self.backward()
        self.update(seed=11)

    def learned(self):
        return [t.clone() for t in (self.E, self.W, self.g1, self.g2, *self.codes[0], *self.codes[1], *self.codes[2], *self.codes[3])]

    def put(self, values):
        for t, v in zip((self.E, self.W, self.g1, self.g2, *self.codes[0], *self.codes[1], *self.codes[2], *self.codes[3]), values):
            t.copy_(v)


def test_a_step_against_64_bits():
    """The gradients of a step, with the readings of the paper where rounding is passed through (dual straight-through estimator): the layer's weights are
    W_eff gamma, its rows the quantized ones.  Each stage rounds to bf16, and a gradient is a sum over many: a few of 2^-8 of its norm."""
    m = Model()
    m.forward()
    m.backward()
    torch.cuda.synchronize()
    T, d = m.T, m.d
    E, W = m.E.double().cpu(), m.W
    inside = m.ids.cpu() >= 0
    x = torch.where(inside[:, None], E[m.ids.cpu().clamp(min=0)], 0.0) * d ** 0.5
    near = lambda got, want, most, what: print(what, r := ((got.double().cpu() - want).norm() / want.norm()).item()) or (r < most or pytest.fail(f"{what}: {r}"))   # noqa: E731
    near(m.x, x, 2.0 ** -8, "x")
    x = m.x.double().cpu()
    r1 = 1 / torch.sqrt((x * x).mean(1, keepdim=True) + 1e-6)
    near(m.n1, x * r1 * m.g1.double().cpu(), 2.0 ** -8, "n1")
    W_eff, _, gamma = oracle.quantize_mask(W.float().cpu().numpy(), 2, 4)
    W_eff = torch.from_numpy(W_eff).double() * float(gamma)
    xq = m.xq.double().cpu() / m.sx.double().cpu()[:, None]
    h = x + (xq @ W_eff.t())
    near(m.h, h, 2.0 ** -7, "h")
    h = m.h.double().cpu()
    r2 = 1 / torch.sqrt((h * h).mean(1, keepdim=True) + 1e-6)
    n2 = h * r2 * m.g2.double().cpu()
    z = n2 @ E.t()
    kept = m.targets.cpu() >= 0
    y = m.targets.cpu().clamp(min=0)
    near(m.ce, torch.where(kept, torch.logsumexp(z, 1) - z[torch.arange(T), y], 0.0), 2.0 ** -7, "ce")
    G = (torch.softmax(z, 1) - torch.nn.functional.one_hot(y, m.V)) * m.d_ce.double().cpu()[:, None]
    dn2 = G @ E
    a2 = dn2 * m.g2.double().cpu()
    u2 = h * r2
    dh = r2 * (a2 - u2 * (a2 * u2).mean(1, keepdim=True))
    near(m.dh, dh, 2.0 ** -6, "dh")
    near(m.dg2, (dn2 * u2).sum(0), 2.0 ** -6, "dg2")
    near(m.dW, dh.t() @ xq, 2.0 ** -6, "dW")
    dn1 = dh @ W_eff
    a1, u1 = dn1 * m.g1.double().cpu(), x * r1
    dx = dh + r1 * (a1 - u1 * (a1 * u1).mean(1, keepdim=True))
    near(m.dx, dx, 2.0 ** -6, "dx")
    near(m.dg1, (dn1 * u1).sum(0), 2.0 ** -6, "dg1")
    dE = G.t() @ n2
    dE.index_add_(0, m.ids.cpu()[inside], dx[inside] * d ** 0.5)
    near(m.dE, dE, 2.0 ** -6, "dE")
    m.update()
    norm = np.sqrt(sum((t.double() ** 2).sum().item() for t in (m.dE, m.dW)))
    assert abs(m.norm[0].item() - norm) <= 1.01 * 2.0 ** -24 * norm


def test_steps_replayed_from_a_graph():
    """A whole step in one graph: replays go on from the weights and moments that they find, read the step and the learning rate that are there, and give
    what eager steps give, bit for bit."""
    m = Model(seed=1)
    start = m.learned()
    gains0 = [t.clone() for t in m.gain_states[0] + m.gain_states[1]]

    def back():
        m.put(start)
        for t, v in zip(m.gain_states[0] + m.gain_states[1], gains0):
            t.copy_(v)

    ids = [torch.randint(0, m.V, (m.T,), generator=torch.Generator().manual_seed(50 + k)).to(DEV) for k in range(4)]
    want = []
    for k in range(4):
        m.ids.copy_(ids[k])
        m.step.fill_(k + 1)
        m.lr.fill_(1e-2 / (k + 1))
        m.all_steps()
        want.append(m.learned() + [m.ce.clone(), m.norm.clone()])
    back()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        m.all_steps()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        m.all_steps()
    back()
    for k in range(4):
        m.ids.copy_(ids[k])
        m.step.fill_(k + 1)
        m.lr.fill_(1e-2 / (k + 1))
        m.ws.fill_(0xff)   # nothing of the replay before is needed
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for i, (got, ref) in enumerate(zip(m.learned() + [m.ce, m.norm], want[k])):
            assert torch.equal(got, ref), (k, i)
        (torch.randn(1000, device=DEV) @ torch.randn(1000, device=DEV)).item()   # work of its own between the replays


def test_two_graphs_share_a_workspace():
    """Two captured gradients on one workspace, replayed in turn on one stream."""
    s = sbn()
    g = torch.Generator(device=DEV).manual_seed(3)
    T, d, V = 900, 72, 300
    ws = s.new_workspace(max(s.sbn_embedding_workspace_bytes(T, d, V), s.sbn_norm_workspace_bytes(T, d)))
    calls, held = [], []
    for k in range(2):
        ids, dY = torch.randint(0, V, (T,), generator=g, device=DEV), torch.randn(T, d, generator=g, device=DEV)
        dE, dX, dg = torch.empty(V, d, device=DEV), torch.empty(T, d, device=DEV), torch.empty(d, device=DEV)

        def call(ids=ids, dY=dY, dE=dE, dX=dX, dg=dg):
            s.sbn_norm_backward(dY, dY, ws, dX=dX, dgain=dg, layer=True)
            s.sbn_embedding_backward(dX, ids, dE, ws)
        call()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            call()
        calls.append((graph, dE, dE.clone(), dg, dg.clone()))
        held.append(call)   # and with it the buffers whose addresses the graph has
    for _ in range(3):
        for graph, dE, *_, dg, _ in calls:
            dE.fill_(float("nan"))
            dg.fill_(float("nan"))
        for graph, *_ in calls:
            graph.replay()
        torch.cuda.synchronize()
        for _, dE, want, dg, want_g in calls:
            assert torch.equal(dE, want) and torch.equal(dg, want_g)


def test_calls_on_streams_of_their_own():
    s = sbn()
    g = torch.Generator(device=DEV).manual_seed(5)
    T, d, V = 3000, 1000, 700
    ids, dY = torch.randint(0, V, (T,), generator=g, device=DEV), torch.randn(T, d, generator=g, device=DEV)
    want = torch.empty(V, d, device=DEV)
    s.sbn_embedding_backward(dY, ids, want, s.new_workspace(s.sbn_embedding_workspace_bytes(T, d, V)))
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(3)]
    outs = [torch.empty(V, d, device=DEV) for _ in streams]
    spaces = [s.new_workspace(s.sbn_embedding_workspace_bytes(T, d, V)) for _ in streams]
    torch.cuda.synchronize()
    for _ in range(5):
        for stream, out, ws in zip(streams, outs, spaces):
            with torch.cuda.stream(stream):
                s.sbn_embedding_backward(dY, ids, out, ws)
    torch.cuda.synchronize()
    assert all(torch.equal(o, want) for o in outs)


FAST = ["_fast_norm", "_fast_norm_backward", "_fast_embedding", "_fast_embedding_backward", "_fast_grad_norm", "_fast_adamw", "_fast_state_values", "_fast_norm_bytes",
        "_fast_embedding_bytes", "_fast_gather"]


def test_marshalled_in_cpp_and_in_python_alike(monkeypatch):
    """Every call by both ways: the same results, the same errors; whatever the C++ does not take goes to the Python code."""
    out = {}
    for way in ("fast", "python"):
        if way == "python":
            for name in FAST:
                monkeypatch.setattr(b, name, lambda *args: None)
        m = Model(seed=2)
        m.all_steps()
        X, Y = m.x, torch.empty_like(m.x)
        values = torch.empty(m.E.shape, dtype=BF16, device=DEV)
        b.sbn_adamw_state_values(m.codes[1][0], m.codes[3][0], values, second=True)
        b.sbn_norm(X, Y, layer=True, eps=1, bias=m.g1)          # a whole number for eps: Python's
        errors = []
        for call in (lambda: b.sbn_norm(X, Y, residual=X), lambda: b.sbn_norm(X, Y, eps=-1.0), lambda: b.sbn_norm(X, Y.cpu()), lambda: b.sbn_norm(X, Y[:3]),
                     lambda: b.sbn_norm(X, Y, gain=m.g1.bfloat16()), lambda: b.sbn_norm_backward(X, Y, m.ws[:256], dX=Y), lambda: b.sbn_norm_backward(X, Y, m.ws),
                     lambda: b.sbn_norm_backward(X, Y, m.ws[64:], dX=Y), lambda: b.sbn_embedding(m.E, m.ids[:3], Y), lambda: b.sbn_embedding(m.E, m.ids.int(), Y),
                     lambda: b.sbn_embedding(m.E, m.ids, Y, scale=float("nan")), lambda: b.sbn_embedding_backward(X, m.ids, m.dE, m.ws[:256]),
                     lambda: b.sbn_embedding_backward(X.cpu(), m.ids, m.dE, m.ws), lambda: m.norms.run(-1.0, m.norm), lambda: m.norms.run(1.0, m.norm[:1]),
                     lambda: m.optim.run(m.lr, m.step.int()), lambda: m.optim.run(m.lr.cpu(), m.step), lambda: b.sbn_adamw_state_values(m.codes[1][0], m.codes[3][0], values[:3]),
                     lambda: b.AdamWGroup([m.g1, m.g2], [m.dg1], [m.g1] * 2, [m.g1] * 2), lambda: b.AdamWGroup([m.g1, m.E], [m.dg1] * 2, [m.g1] * 2, [m.g1] * 2),
                     lambda: b.AdamWGroup([m.g1], [m.dg1[:-1]], [m.g1], [m.g1]), lambda: b.AdamWGroup([m.g1], [m.dg1], [m.g1], [m.g1.cpu()]),
                     lambda: b.AdamWGroup([m.g1], [m.dg1], m.codes[0], m.codes[1], m.codes[2], m.codes[3]), lambda: b.GradNormGroup([m.E.t()], m.ws),
                     lambda: b.AdamWGroup([m.g1, m.g2], [m.dg1, m.dg2], [m.g1, m.g1], [m.g1, m.g2]).run(m.lr, m.step),
                     lambda: b.sbn_norm_workspace_bytes(0, 1), lambda: b.sbn_embedding_workspace_bytes(1, 1, 1 << 30)):
            with pytest.raises(Exception) as e:
                call()
            errors.append((type(e.value).__name__, str(e.value)))
        torch.cuda.synchronize()
        out[way] = m.learned() + [m.ce, m.norm, m.dg1, m.dE, values, Y] + errors
    assert len(out["fast"]) == len(out["python"])
    for x, y in zip(out["fast"], out["python"]):
        assert torch.equal(x, y) if torch.is_tensor(x) else x == y


def test_groups_of_another_device_are_refused(monkeypatch):
    m = Model(seed=4)
    monkeypatch.setattr(b, "_current_device", lambda: 1)
    with pytest.raises(ValueError, match="current device"):
        m.optim.run(m.lr, m.step)
