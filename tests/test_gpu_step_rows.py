"""Where rows lie and what that may change."""
import pytest
import torch

from gpu_util import DEV, sbn
from test_gpu_step_norm import rows

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32


# ---- norms --------------------------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("layer", [False, True])
@pytest.mark.parametrize("T,d", [(2500, 1001), (8200, 301), (2100, 2001), (4099, 2563)])
def test_equal_rows_that_begin_alike_have_equal_gradients(T, d, layer, dtype):
    """A row's sums go by where it begins in memory: rows that are eight apart begin at the same place of a vector, whatever their length."""
    s = sbn()
    X, g = rows(1, d, dtype, d, offset=0.3)
    dY, gain = (torch.randn(1, d, generator=g) * 0.02).to(dtype), 1 + 0.3 * torch.randn(d, generator=g)
    x, dy = (t.to(DEV).expand(T, d).contiguous() for t in (X, dY))
    Y, dX = torch.empty_like(x), torch.empty_like(x)
    ws = s.new_workspace(s.sbn_norm_workspace_bytes(T, d))
    s.sbn_norm(x, Y, gain=gain.to(DEV), layer=layer)
    s.sbn_norm_backward(x, dy, ws, dX=dX, dgain=torch.empty(d, device=DEV), gain=gain.to(DEV), layer=layer)
    for t in (Y, dX):
        for first in range(8):
            alike = t[first::8]
            assert (alike == alike[0]).all(), (first, (alike != alike[0]).any(1).sum().item())
