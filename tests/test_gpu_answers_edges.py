"""moe_policy_loss and moe_preference_loss at their arguments' ends, beside test_gpu_answers.py, whose bounds these share."""
import pytest
import torch

import paper_2402_14800_amd as pkg
from tests.test_gpu_answers import BF16, DEV, F32, make_policy, reference
from tests.test_gpu_logits import make_logits

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kl", [0.0, 0.1])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_an_advantage_that_is_no_number_shows(dtype, kl):
    """NaN in the advantage is NaN in loss, derivative and gradient on either side of the clip's bounds, as the formula's products are."""
    T, V = 6, 70
    z = make_logits(T, V, dtype, seed=50)
    tokens = torch.full((T,), 3, device=DEV)
    old, A, ref, _ = make_policy(z, tokens, 1.0, seed=51)
    lp = reference(z, tokens)[0]
    shift = torch.tensor([0.0, 0.9, -0.9, 3.0, -3.0, 0.0]).double()          # ratios 1, below and above the bounds
    old = (lp - shift).float().to(DEV)
    A[:5] = float("nan")
    loss, got, stats, grad = pkg.moe_policy_loss(z, tokens, old, A, ref, kl=kl, gradient=True)
    back = pkg.moe_policy_loss_backward(z, tokens, stats, torch.ones(T, device=DEV))
    for x in (loss, stats[:, 2], grad, back):
        assert bool(torch.isnan(x[:5]).all()) and bool(torch.isfinite(x[5]).all())
    assert bool(torch.isfinite(got).all())
