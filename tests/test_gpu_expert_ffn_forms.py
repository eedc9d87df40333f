"""GPU parity of one expert's block in forms that few sizes reach, with the bounds of test_gpu_expert_ffn."""
import pytest
import torch

import paper_2402_14800_amd as pkg
from paper_2402_14800_amd import binding
from tests.test_gpu_expert_ffn import DEV, check, reference, step

pytestmark = pytest.mark.gpu


def test_more_rows_than_one_grid_holds():
    """16 rows a workgroup of the transposes and of the branch pass: two launches each, the second one's rows are the last ones."""
    T, H, F, n = (1 << 28) + 52, 4, 4, 300
    g = torch.Generator(device=DEV).manual_seed(50)
    x = torch.randn((T, H), generator=g, device=DEV)
    W1, W3, W2 = (torch.randn(s, generator=g, device=DEV) / 2 for s in ((F, H), (F, H), (H, F)))
    dy = torch.zeros((T, H), device=DEV)
    ends = torch.cat([torch.arange(n), torch.arange(T - n, T)]).to(DEV)
    dy[ends] = torch.randn((2 * n, H), generator=g, device=DEV)
    (y, dx, *dW), _ = step(x, W1, W3, W2, dy)                # (its workspace holds NaN: what no launch wrote would show)
    ref, mag = reference(x[ends], W1, W3, W2, dy[ends])
    check((y[ends], dx[ends], *dW), ref, mag, torch.float32)
    dx[ends] = 0
    assert not bool(dx.any()) and bool(torch.isfinite(y).all())
