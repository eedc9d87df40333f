"""GPU parity of one expert's block in forms that few sizes reach, with the bounds of test_gpu_expert_ffn."""
import pytest
import torch

import paper_2402_14800_amd as pkg
from tests.test_gpu_expert_ffn import DEV, check, make_block, reference, step

pytestmark = pytest.mark.gpu

# Steps whose last products are launches of their own, and the ranges that K of dh, of dx, of dW2 and of dW1 and dW3 is cut into.  That the
# plan is still this one is checked on the host (test_host_ffn_plan), where another choice of cuts would show.
APART = {
    (2305, 2048, 5632, torch.bfloat16): (1, 2, 1, 1),        # dW1 and dW3 as a batch of two, dW2 in one piece, dx summed
    (4001, 2048, 3584, torch.bfloat16): (1, 2, 2, 1),        # the batch beside a dW2 in ranges
    (6001, 1024, 5120, torch.bfloat16): (1, 2, 3, 3),        # an odd number of ranges
    (16385, 1024, 3584, torch.bfloat16): (1, 1, 4, 2),       # half as many for da^T over db^T; dx in one piece
    (300, 8192, 14336, torch.bfloat16): (2, 4, 1, 1),        # dh summed by the branch pass
    (5999, 1024, 1024, torch.float32): (1, 1, 2, 1),
    (1501, 1024, 640, torch.float32): (2, 1, 3, 3),
}


@pytest.mark.parametrize("T,H,F,dtype", APART)
def test_products_apart(T, H, F, dtype):
    ops = make_block(T, H, F, dtype, seed=T)
    x, W1, W3, W2, dy = ops
    got, gate_up = step(*ops)
    ref, mag = reference(*ops)
    check(got, ref, mag, dtype)
    only_x = pkg.expert_ffn_backward(dy, x, W1, W3, W2, gate_up, weight_gradients=False)
    only_w = pkg.expert_ffn_backward(dy, x, W1, W3, W2, gate_up, input_gradient=False)
    assert torch.equal(only_x[0], got[1]) and only_x[1:] == (None, None, None)
    assert only_w[0] is None and all(torch.equal(a, b) for a, b in zip(only_w[1:], got[2:]))


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
