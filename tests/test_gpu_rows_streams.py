"""moe_dispatch_rows, moe_combine_rows and their gradients where a call's rows are more than the caches hold (268.5 MB) and go past them: every
form of the kernels on rows that differ from column to column, against the definitions as in test_gpu_rows.py, whose bounds these share."""
import pytest
import torch

from tests.test_gpu_rows import BF16, DEV, F32, check_dispatch, check_sums, make_routing

pytestmark = pytest.mark.gpu
CACHES = 268.5e6

# 1, 2, 4 and 8 slots at once, 16 in two turns; rows by a workgroup (256 chunks and more) and by wavefronts or parts of them; odd rows
SHAPES = [(9001, 1, 8, 4096, F32), (12001, 2, 8, 4096, BF16), (16001, 4, 16, 1028, F32), (9001, 8, 32, 2048, BF16), (20001, 16, 3, 256, F32),
          (200001, 2, 8, 256, BF16), (50001, 2, 8, 1024, BF16), (70001, 7, 9, 320, BF16), (130001, 1, 4, 1088, BF16)]


@pytest.mark.parametrize("T,k,E,H,dtype", SHAPES)
def test_rows_past_the_caches(T, k, E, H, dtype):
    assert (T * k + T) * H * (2 if dtype == BF16 else 4) > CACHES
    experts, used = make_routing(T, k, E, seed=H)
    x = torch.randn((T, H), generator=torch.Generator(device=DEV).manual_seed(k), device=DEV).to(dtype)
    slot_of = check_dispatch(x, experts, used, E)
    for weighted in (True, False):
        check_sums(T, k, H, dtype, slot_of, T * k, seed=H, weighted=weighted)


def test_unused_slots_past_the_caches():
    """Every kernel with slots that are not used, and rows that no slot names."""
    T, k, E, H = 60001, 3, 8, 1024
    experts, used = make_routing(T, k, E, seed=1, use=True)
    x = torch.randn((T, H), generator=torch.Generator(device=DEV).manual_seed(2), device=DEV).to(BF16)
    check_sums(T, k, H, BF16, check_dispatch(x, experts, used, E), T * k, seed=3)
