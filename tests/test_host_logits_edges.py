"""What moe_distill_topk refuses at the ends of its arguments, on the host.  Nothing is launched here."""
import ctypes

import pytest

from paper_2402_14800_amd import binding

OK, EINVAL = 0, 1


@pytest.mark.parametrize("name", ["moe_distill_topk", "moe_distill_topk_backward"])
def test_temperatures_without_a_32_bit_square_or_inverse_are_refused(name):
    at, T = ctypes.c_void_p(1 << 20), 0                      # (no rows: what is not refused launches nothing)

    def call(tau):
        if name == "moe_distill_topk":
            return binding._lib.moe_distill_topk(at, 100, at, at, T, 100, 5, 1, ctypes.c_float(tau), None, at, at, at, 100, None)
        return binding._lib.moe_distill_topk_backward(at, 100, at, at, at, at, T, 100, 5, 1, ctypes.c_float(tau), at, 100, None)

    for tau in (2.0 ** -60, 1e-6, 0.5, 1.0, 1e6, 2.0 ** 60):
        assert call(tau) == OK
    for tau in (0.0, -0.0, -1.0, 2.0 ** -149, 1e-40, 2.0 ** -61, 2.0 ** 61, 1e20, 1e30, float("inf"), float("nan")):
        assert call(tau) == EINVAL
