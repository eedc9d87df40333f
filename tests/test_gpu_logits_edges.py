"""moe_distill_topk where its arguments go to their ends, against the definition in 64 bits; bounds as in test_gpu_logits."""
import pytest
import torch

import paper_2402_14800_amd as pkg
from tests.test_gpu_logits import ABS, DEV, check_gradient, make_logits, make_teacher, ref_distill

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V", [70, 4099, 33000, 140000])
def test_rows_left_out_of_the_loss_have_no_gradient(V, dtype):
    """The loss of a row of weight 0 is the constant 0: whatever comes back for it, its gradient is 0, also where its logits would
    overflow an exponential or hold NaN."""
    T, tau = 9, 1.5
    z = make_logits(T, V, dtype, seed=40)
    z[2] += 300.0
    z[5] = float("nan")
    z[8] = -z[8].abs() - 200.0
    ids, teacher = make_teacher(torch.nan_to_num(z), 8, seed=41)
    weights = torch.ones(T, device=DEV)
    out = [0, 2, 5, 8]
    weights[out] = 0.0
    upstream = torch.linspace(0.5, 2.0, T, device=DEV)
    kept = [t for t in range(T) if t not in out]
    want = ref_distill(z[kept], ids[kept], teacher[kept], tau, upstream[kept])[1]
    for gradient in (False, True):
        loss, stats, *_ = pkg.moe_distill_topk(z, ids, teacher, tau, weights=weights, gradient=gradient)
        assert not bool(loss[out].any())
        back = pkg.moe_distill_topk_backward(z, ids, teacher, stats, upstream, tau)
        assert bool((back[out] == 0).all())
        check_gradient(back[kept], want, upstream[kept] * tau, dtype)
        z2 = z.clone()                                       # in the logits' own memory
        pkg.moe_distill_topk_backward(z2, ids, teacher, stats, upstream, tau, out=z2)
        assert torch.equal(z2, back)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("tau", [0.5, 0.7, 1.0, 1.5])
def test_alternative_masked_by_the_lowest_value(tau, dtype):
    """The student masks one of four equal alternatives with its type's lowest value: the loss is tau / 4 of that, a number of 32 bits."""
    z = make_logits(3, 500, dtype, seed=42)
    ids, _ = make_teacher(z, 4, seed=43)
    teacher = torch.zeros((3, 4), device=DEV)
    z[1, ids[1, 2].long()] = torch.finfo(dtype).min
    want, rgrad = ref_distill(z, ids, teacher, tau)
    loss, stats, grad = pkg.moe_distill_topk(z, ids, teacher, tau, gradient=True)
    assert bool(((loss.double().cpu() - want).abs() <= ABS * want.abs() + 4 * ABS * max(1.0, tau) ** 2).all()), (loss, want)
    check_gradient(grad, rgrad, torch.full((3,), tau), dtype)
    check_gradient(pkg.moe_distill_topk_backward(z, ids, teacher, stats, torch.ones(3, device=DEV), tau), rgrad, torch.full((3,), tau), dtype)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("tau", [2.0 ** -60, 2.0 ** -20, 2.0 ** 20, 2.0 ** 60])
def test_temperatures_to_their_ends(tau, dtype):
    """Cold, p and q pick one entry each and the loss is tau times a difference of logits; hot, both are level and it is tau^2 log(V / K)."""
    T, V, K = 5, 1003, 8
    z = make_logits(T, V, dtype, seed=44)
    ids, teacher = make_teacher(z, K, seed=45)
    want, rgrad = ref_distill(z, ids, teacher, tau)
    loss, stats, grad = pkg.moe_distill_topk(z, ids, teacher, tau, gradient=True)
    assert bool(((loss.double().cpu() - want).abs() <= ABS * want.abs()).all()), (loss, want)
    check_gradient(grad, rgrad, torch.full((T,), tau), dtype)
    check_gradient(pkg.moe_distill_topk_backward(z, ids, teacher, stats, torch.ones(T, device=DEV), tau), rgrad, torch.full((T,), tau), dtype)


def test_rows_that_are_not_rows_of_logits_are_refused():
    """On the GPU, where nothing but their strides is wrong."""
    V = 64
    z = make_logits(V, V, torch.float32, seed=46)
    ids, teacher = make_teacher(z, 3, seed=47)
    tokens = ids[:, 0].long().contiguous()
    stats, ones = torch.zeros((V, 2), device=DEV), torch.ones(V, device=DEV)
    overlapping = torch.zeros(2 * V, device=DEV).as_strided((V, V), (1, 1))
    repeated = z[:1].expand(V, V)
    for bad in (z.t(), torch.zeros((V, 2 * V), device=DEV)[:, ::2], overlapping, repeated):
        assert bad.shape == (V, V) and bad.is_cuda
        for call in (lambda: pkg.moe_token_logprobs(bad, tokens), lambda: pkg.moe_distill_topk(bad, ids, teacher),
                     lambda: pkg.moe_distill_topk_backward(bad, ids, teacher, stats, ones),
                     lambda: pkg.moe_distill_topk(z, ids, teacher, gradient=True, out=bad),
                     lambda: pkg.moe_distill_topk_backward(z, ids, teacher, stats, ones, out=bad)):
            with pytest.raises(ValueError, match="rows of logits must be contiguous"):
                call()
    for bad in (ids.t().contiguous().t(), ids.long(), ids.cpu(), ids[:-1], ids[:, :2]):
        with pytest.raises(ValueError):
            pkg.moe_distill_topk(z, bad, teacher)
    for bad in (tokens.cpu(), tokens.int(), tokens[:-1], torch.cat([tokens, tokens])[::2]):
        with pytest.raises(ValueError, match="tokens must be"):
            pkg.moe_token_logprobs(z, bad)
    for bad in (ones[:1].expand(V), ones.double(), ones[:-1]):
        with pytest.raises(ValueError, match="grad_loss must be"):
            pkg.moe_distill_topk_backward(z, ids, teacher, stats, bad)
        with pytest.raises(ValueError, match="weights must be"):
            pkg.moe_distill_topk(z, ids, teacher, weights=bad)
