"""AdamW on both sides of the eps at which its root and quotient change.  Tolerances as in the tests of the step."""
import numpy as np
import pytest
import torch

from test_gpu_step_adamw import B1, B2, U, Tensors, check_step, run

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32


@pytest.mark.parametrize("pt", [F32, BF16])
@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("eps", [0.0, 9e-13, 1e-12, 1e-8, 1e-3])
def test_step_on_both_sides_of_the_eps(eps, bits, pt):
    check_step(Tensors([1, 33, 1000, 8193], pt, F32, bits, seed=21), eps=eps)
    check_step(Tensors([1000], pt, F32, bits, seed=22, scale=1e-9), eps=eps, clip=0.7, seed=4)


@pytest.mark.parametrize("eps", [0.0, 1e-20, 1e-12])
def test_second_moments_below_the_normal_numbers(eps):
    """v' below 2^-126: with an eps under 1e-12 its root is taken as it is, else it counts as 0, which is 2^-63 / sqrt(1 - beta2^t) to an eps at most."""
    n, step, lr = 1000, 3, 0.01
    t = Tensors([n], F32, F32, 32, seed=23, scale=3e-21)
    t.v[0] = (3e-21 * (1 + torch.rand(n, generator=torch.Generator().manual_seed(24)))) ** 2
    t.p[0] = torch.zeros(n)
    d = run(t, lr, step, eps=eps)
    g, m, v = t.g[0].double(), t.m[0].double(), t.v[0].double()
    terms = B1 * m.abs() + (1 - B1) * g.abs()
    m, v = B1 * m + (1 - B1) * g, B2 * v + (1 - B2) * g * g
    assert v.max() < 2.0 ** -126 and v.min() > 2.0 ** -140
    rate, eps = float(np.float32(lr)) / (1 - B1 ** step), float(np.float32(eps))
    # each of v's three operations is off by half of 2^-149 here, the constants by 2^-24 of it
    off = 2.0 ** -148 + 4 * U * v
    least = 0 * v if eps >= 1e-12 else torch.sqrt((v - off) / (1 - B2 ** step))
    most = torch.sqrt((v + off) / (1 - B2 ** step))
    got = d["params"][0].double().cpu()
    low, high = (-m).sign() * rate * m.abs() / (most + eps), (-m).sign() * rate * m.abs() / (least + eps)
    tol = 24 * U * rate * terms / (least + eps)
    assert (got >= torch.minimum(low, high) - tol).all() and (got <= torch.maximum(low, high) + tol).all()
