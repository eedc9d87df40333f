"""What the preference loss's entry points for a gradient of all rows refuse.  Nothing is launched here."""
import ctypes

import pytest

from paper_2402_14800_amd import binding
from tests.test_host_answers_rows import BAD, EINVAL, EUNSUPPORTED, OK, ONE, P

LIB = binding._lib


def whole(z=ONE, ld=100, tok=ONE, off=ONE, ref=ONE, T=4, V=100, pairs=2, dt=1, beta=0.1, ls=0.0, avg=0, w=None, loss=ONE, rew=ONE, lp=ONE, stats=ONE,
          grad=ONE, ldg=100):
    f = ctypes.c_float
    return LIB.moe_preference_loss_all_rows(z, ld, tok, off, ref, T, V, pairs, dt, f(beta), f(ls), avg, w, loss, rew, lp, stats, grad, ldg, None)


def whole_back(z=ONE, ld=100, tok=ONE, off=ONE, stats=ONE, gl=ONE, T=4, V=100, pairs=2, dt=1, grad=ONE, ldg=100):
    return LIB.moe_preference_loss_backward_all_rows(z, ld, tok, off, stats, gl, T, V, pairs, dt, grad, ldg, None)


@pytest.mark.parametrize("call", [whole, whole_back])
def test_refusals(call):
    assert call(dt=7) == EINVAL and call(T=-1) == EINVAL and call(T=(1 << 30) + 1) == EINVAL
    assert call(V=0) == EINVAL and call(V=(1 << 28) + 1, ld=1 << 30, ldg=1 << 30) == EINVAL and call(ld=99) == EINVAL and call(ldg=99) == EINVAL
    assert call(z=P((1 << 20) + 1)) == EUNSUPPORTED and call(grad=P((1 << 20) + 1)) == EUNSUPPORTED and call(grad=P((1 << 20) + 2), dt=0) == EUNSUPPORTED
    for name in ("z", "tok", "off", "stats", "grad"):
        assert call(**{name: None}) == EINVAL
        assert call(pairs=0, **{name: None}) == EINVAL       # (without pairs every row is one of no answer)
    assert call(tok=P((1 << 20) + 4)) == EUNSUPPORTED and call(off=P((1 << 20) + 4)) == EUNSUPPORTED and call(stats=P((1 << 20) + 2)) == EUNSUPPORTED
    assert call(pairs=-1) == EINVAL and call(pairs=(1 << 22) + 1) == EINVAL
    assert call(T=0, pairs=0, z=None, tok=None, stats=None, grad=None) == OK
    if call is whole:
        for name in ("ref", "loss", "rew", "lp"):
            assert call(**{name: None}) == EINVAL
        for x in BAD:
            assert call(beta=x) == EINVAL and call(ls=x) == EINVAL
        assert call(avg=2) == EINVAL
    else:
        assert call(gl=None) == EINVAL
