"""moe_policy_loss and moe_preference_loss at their arguments' ends, beside test_gpu_answers.py, whose bounds these share."""
import pytest
import torch

import paper_2402_14800_amd as pkg
from tests.test_gpu_answers import BF16, DEV, F32, make_pairs, make_policy, reference
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


def junk(T, V, dtype):
    """Leaves NaN in the memory that a gradient of this size is given next."""
    torch.full((T, V), float("nan"), dtype=dtype, device=DEV)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("T,V,P,pad,tail,head", [(40, 257, 3, 3, 4, 3), (2300, 301, 6, 0, 100, 1), (300, 5003, 2, 0, 0, 7), (5, 50001, 2, 5, 2, 0), (700, 9001, 2, 0, 699, 0)])
def test_rows_of_no_answer_get_zeros_in_a_gradient_of_its_own(T, V, P, pad, tail, head, dtype):
    """Without `out` the gradient's rows in front of the answers and behind them are 0: what goes on with the whole of it (a head's
    gradient, dlogits.T @ rows) finds numbers.  In a given `out` they stay."""
    z = make_logits(T, V, dtype, seed=V, pad=pad)
    tokens = torch.randint(-1, V, (T,), generator=torch.Generator().manual_seed(T)).to(DEV)
    offsets = make_pairs(T, P, seed=P, tail=tail, head=head)
    ref, w = torch.full((T,), -6.0, device=DEV), torch.rand(P, generator=torch.Generator().manual_seed(1)).to(DEV)
    want = pkg.moe_preference_loss(z, tokens, offsets, ref, weights=w, gradient=True, out=torch.zeros_like(z))
    junk(T, V, dtype)
    got = pkg.moe_preference_loss(z, tokens, offsets, ref, weights=w, gradient=True)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    junk(T, V, dtype)
    assert torch.equal(pkg.moe_preference_loss_backward(z, tokens, offsets, want[3], w), want[4])
    kept = pkg.moe_preference_loss_backward(z, tokens, offsets, want[3], w, out=torch.full_like(z, 5.0))
    assert bool((kept[:head] == 5.0).all()) and bool((kept[T - tail:] == 5.0).all()) and torch.equal(kept[head:T - tail], want[4][head:T - tail])


@pytest.mark.parametrize("T,V", [(1, 7), (60, 5003), (2300, 301)])
def test_no_pairs_give_a_gradient_of_zeros(T, V):
    z, tokens, ref = make_logits(T, V, BF16, seed=60), torch.zeros(T, dtype=torch.int64, device=DEV), torch.zeros(T, device=DEV)
    offsets = torch.zeros(1, dtype=torch.int64, device=DEV)
    for at in (0, T // 2):
        offsets[0] = at
        junk(T, V, BF16)
        loss, rew, lp, stats, grad = pkg.moe_preference_loss(z, tokens, offsets, ref, gradient=True)
        assert loss.shape == (0,) and not bool(lp.any()) and torch.equal(grad, torch.zeros_like(z))
        junk(T, V, BF16)
        assert torch.equal(pkg.moe_preference_loss_backward(z, tokens, offsets, stats, ref[:0]), torch.zeros_like(z))
    out = torch.full_like(z, 5.0)
    assert pkg.moe_preference_loss(z, tokens, offsets, ref, gradient=True, out=out)[4] is out and bool((out == 5.0).all())


def test_rows_of_no_answer_in_a_graph():
    """The gradient's memory is the graph's own, which other nodes write to as well; the answers move from replay to replay."""
    T, V, P = 300, 1003, 4
    z, tokens, ref = make_logits(T, V, F32, seed=61), torch.arange(T, device=DEV), torch.full((T,), -6.0, device=DEV)
    offsets = make_pairs(T, P, seed=62, tail=5, head=2)

    out = torch.zeros_like(z)

    def run():
        grad = pkg.moe_preference_loss(z, tokens, offsets, ref, gradient=True)[4]
        torch.add(grad, 0.0, out=out)
        grad.fill_(float("nan"))

    run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    for seed in range(3):
        offsets.copy_(make_pairs(T, P, seed=70 + seed, tail=3 + 40 * seed, head=9 * seed))
        want = pkg.moe_preference_loss(z, tokens, offsets, ref, gradient=True, out=torch.zeros_like(z))[4]
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)
