"""GPU parity of moe_token_logprobs and moe_distill_topk with their definitions in 64 bits.

Bounds.  A log probability is (z - m) - log s: z - m is off by 2^-24 of itself; a term of s by 2^-24 of its exponent (at most 128
log2 units where it counts) and of itself, hence s by less than 1.3e-5 of itself at the very most (by 1e-6 for terms that weigh),
log s by as much.  ABS covers it with room for the sums' own roundings; the entropy sums (z - m) p: the same, times z - m.
A gradient is a difference of p and q, each off by ABS of ITSELF, however small their difference; in bf16 it is rounded once, by
2^-8 of itself at most."""
import numpy as np
import pytest
import torch

import paper_2402_14800_amd as pkg

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
INF = float("inf")
ABS = 2e-5


def make_logits(T, V, dtype, seed=0, pad=0, offset=0, scale=2.5):
    """[T, V] logits in rows of V + pad elements that begin `offset` elements into an aligned allocation."""
    g = torch.Generator().manual_seed(seed)
    z = scale * torch.randn((T, V), generator=g)
    z[torch.arange(T), torch.randint(0, V, (T,), generator=g)] += 6.0
    flat = torch.zeros(T * (V + pad) + offset, dtype=dtype, device=DEV)
    rows = flat[offset:].view(T, V + pad)[:, :V]
    rows.copy_(z.to(dtype))
    return rows


def ref_logprobs(z, tokens, K):
    z = z.double().cpu()
    logp = torch.log_softmax(z, 1)
    p = logp.exp()
    order = torch.sort(z, dim=1, descending=True, stable=True).indices[:, :K]
    lp = logp.gather(1, tokens.cpu().clamp(min=0)[:, None])[:, 0]
    lp[tokens.cpu() < 0] = 0.0
    return lp, -torch.xlogy(p, p).sum(1), logp.gather(1, order), order


def check_logprobs(z, tokens, K):
    lp, ent, tlp, ids = pkg.moe_token_logprobs(z, tokens, K)
    torch.cuda.synchronize()
    rlp, rent, rtlp, rids = ref_logprobs(z, tokens, K)
    spread = float((rtlp.max() - torch.nan_to_num(rlp, neginf=0.0)).abs().max()) if K else 60.0
    tol = ABS + 2.0 ** -22 * spread
    assert torch.equal(ids.cpu().long(), rids)
    close = lambda a, b, t: torch.allclose(a.double().cpu(), b, rtol=2.0 ** -22, atol=t)  # noqa: E731
    assert close(lp, rlp, tol) and close(tlp, rtlp, tol) and close(ent, rent, 8 * ABS)


SHAPES = [(1, 1, 1), (3, 2, 2), (2, 7, 3), (5, 8, 8), (4, 9, 9), (2, 64, 33), (3, 255, 128), (7, 257, 100), (3, 1003, 64), (2, 4097, 16),
          (2600, 300, 5), (2100, 777, 32), (2049, 130, 128), (600, 4104, 3), (3, 8192, 64), (2, 32000, 100), (515, 32768, 20),
          (1, 50001, 1), (2, 131075, 128), (520, 40007, 7), (1, 300007, 64)]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("T,V,K", SHAPES)
def test_logprobs_over_shapes(T, V, K, dtype):
    z = make_logits(T, V, dtype, seed=V + K)
    tokens = torch.randint(0, V, (T,), generator=torch.Generator().manual_seed(1)).to(DEV)
    check_logprobs(z, tokens, K)
    if T > 2:
        tokens[1] = -100
        lp = pkg.moe_token_logprobs(z, tokens)[0]
        assert float(lp[1]) == 0.0


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V,pad,offset", [(1000, 1, 0), (1003, 0, 1), (4096, 3, 5), (33001, 7, 3), (9, 4, 1), (40001, 0, 1)])
def test_logprobs_of_unaligned_rows(V, pad, offset, dtype):
    z = make_logits(6, V, dtype, seed=V, pad=pad, offset=offset)
    check_logprobs(z, torch.arange(6, device=DEV) % V, min(V, 10))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V", [40, 1000, 33000, 140000])
def test_logprobs_of_masked_and_level_rows(V, dtype):
    """Rows with few logits above -inf, with the type's lowest value as a mask, of equal logits (every one is among the candidates),
    of two values, negative throughout, of zeros with either sign."""
    low = torch.finfo(dtype).min
    z = make_logits(9, V, dtype, seed=3)
    z[0] = -INF
    z[0, V // 2], z[0, 3], z[0, V - 1] = 1.0, 1.0, -2.0
    z[1, 5:] = low
    z[2] = 0.25
    z[3] = torch.where(torch.arange(V, device=DEV) % 3 == 0, 1.0, -1.0)
    z[4] = -z[4].abs() - 100.0
    z[5] = torch.where(torch.arange(V, device=DEV) % 2 == 0, -0.0, 0.0)
    z[6] = low
    z[7, 1:] = -INF
    z[8] = torch.finfo(dtype).max
    check_logprobs(z, torch.tensor([3, 1, V - 1, 0, 7, 2, V - 2, 0, 11], device=DEV), 32)
    lp = pkg.moe_token_logprobs(z, torch.full((9,), 9, device=DEV))[0]
    assert float(lp[0]) == -INF and float(lp[7]) == -INF


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V", [50, 33000])
def test_logprobs_without_a_distribution(V, dtype):
    """Empty rows, NaN, +inf and tokens that do not exist: defined results, indices that can be used, and the rows beside them whole."""
    z = make_logits(5, V, dtype, seed=4)
    z[0] = -INF
    z[1, V // 3] = float("nan")
    z[2, V - 1] = INF
    lp, ent, tlp, ids = pkg.moe_token_logprobs(z, torch.tensor([2, 2, 2, V, V - 1], device=DEV), 8)
    assert float(lp[0]) == -INF and float(ent[0]) == 0.0 and ids[0].tolist() == list(range(8)) and bool((tlp[0] == -INF).all())
    assert all(bool(torch.isnan(v[r]).all()) for v in (ent, tlp) for r in (1, 2)) and bool(torch.isnan(lp[1:4]).all())
    assert int(ids.min()) >= 0 and int(ids.max()) < V
    check_logprobs(z[4:], torch.tensor([V - 1], device=DEV), 8)


def test_logprobs_keep_to_their_row_and_repeat():
    """A row alone and in batches that take other workgroup sizes: the same choice and the bound; twice the same call: the same bits."""
    z = make_logits(2600, 900, torch.bfloat16, seed=8)
    tokens = torch.arange(2600, device=DEV) % 900
    a, b = pkg.moe_token_logprobs(z, tokens, 20), pkg.moe_token_logprobs(z, tokens, 20)
    assert all(torch.equal(x, y) for x, y in zip(a, b))
    one = pkg.moe_token_logprobs(z[77:78], tokens[77:78], 20)
    assert torch.equal(one[3], a[3][77:78]) and torch.allclose(one[0], a[0][77:78], atol=ABS)


def test_logprobs_beyond_32_bit_offsets():
    V, T = 131072, 16400                                     # 2^31 elements and more
    z = torch.zeros((T, V), dtype=torch.bfloat16, device=DEV)
    z[T - 1] = make_logits(1, V, torch.bfloat16, seed=5)[0]
    z[:, 70001] += 9.0
    tokens = torch.full((T,), 70001, device=DEV)
    lp, _, _, ids = pkg.moe_token_logprobs(z, tokens, 1)
    assert bool((ids[:-1] == 70001).all())
    want = 9.0 - np.log(np.exp(9.0) + V - 1)
    assert float((lp[:-1] - want).abs().max()) <= ABS
    rlp = ref_logprobs(z[T - 1:], tokens[:1], 1)[0]
    assert abs(float(lp[-1]) - float(rlp)) <= ABS


def test_more_rows_than_a_launch_has():
    T, V = (1 << 22) + 1001, 3
    z = make_logits(T, V, torch.bfloat16, seed=6)
    tokens = torch.arange(T, device=DEV) % V
    lp, ent, tlp, ids = pkg.moe_token_logprobs(z, tokens, 2)
    want = torch.log_softmax(z.double(), 1)
    assert float((lp - want.gather(1, tokens[:, None])[:, 0]).abs().max()) <= ABS
    assert float((tlp[:, 0] - want.max(1).values).abs().max()) <= ABS
    teacher = torch.zeros((T, 1), device=DEV)
    alternative = tokens[:, None].to(torch.int32).contiguous()
    loss, stats, grad = pkg.moe_distill_topk(z, alternative, teacher, gradient=True)
    assert float((loss + want.gather(1, tokens[:, None])[:, 0]).abs().max()) <= 4 * ABS
    back = pkg.moe_distill_topk_backward(z, alternative, teacher, stats, torch.ones(T, device=DEV))
    ref = want.exp()
    ref[torch.arange(T, device=DEV), tokens] -= 1
    for g in (grad, back):
        assert float((g.double() - ref).abs().max()) <= 2.0 ** -8


# ---------------------------------------------------------------- distillation
def make_teacher(z, K, seed):
    g = torch.Generator().manual_seed(seed)
    t = z.float().cpu() + torch.randn(z.shape, generator=g)
    v, i = torch.topk(t, K, dim=1)
    return i.to(torch.int32).to(DEV), v.contiguous().to(DEV)


def ref_distill(z, ids, teacher, tau, weights=None):
    """Loss of every row, the gradient of the weighted sum and the sum of its two terms' magnitudes, in 64 bits, row by row from the
    definition."""
    z, ids, teacher = z.double().cpu(), ids.cpu().long(), teacher.double().cpu()
    T, V = z.shape
    loss, grad = torch.zeros(T, dtype=torch.float64), torch.zeros((T, V), dtype=torch.float64)
    terms = torch.zeros((T, V), dtype=torch.float64)
    for t in range(T):
        w = 1.0 if weights is None else float(weights[t])
        there = (ids[t] >= 0) & (ids[t] < V) & (teacher[t] > -INF)
        if w == 0.0 or not bool(there.any()) or bool((z[t] == -INF).all()):
            continue
        i, q = ids[t][there], torch.softmax(teacher[t][there] / tau, 0)
        logp = torch.log_softmax(z[t] / tau, 0)
        loss[t] = tau ** 2 * (torch.xlogy(q, q) - torch.where(q > 0, q * logp[i], 0.0)).sum()
        g = logp.exp()
        terms[t] = abs(w) * tau * g.clone().index_add_(0, i, q)
        grad[t] = w * tau * g.index_add_(0, i, -q)
    return loss, (grad, terms)


def check_gradient(got, ref, scale, dtype):
    """`scale`: weight and temperature of each row; 1e-3 of it for the smallest p, whose exponents are large."""
    ref, terms = ref
    rel = 2.0 ** -8 if dtype == torch.bfloat16 else 0.0
    d = (got.double().cpu() - ref).abs()
    bound = rel * ref.abs() + ABS * (terms + 1e-3 * scale[:, None].cpu().double())
    assert bool((d <= bound + 1e-38).all()), float((d - bound).max())


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("T,V,K,tau,pad,offset", [
    (1, 1, 1, 1.0, 0, 0), (3, 7, 3, 2.0, 0, 0), (5, 64, 64, 1.0, 0, 1), (4, 257, 128, 1.5, 3, 0), (33, 1003, 8, 1.0, 0, 0),
    (2100, 301, 10, 0.7, 0, 0), (2050, 4096, 4, 1.0, 5, 3), (9, 8193, 65, 4.0, 1, 0), (3, 32000, 64, 2.0, 0, 0), (2, 50001, 100, 1.5, 64, 7),
    (3, 131075, 5, 1.0, 0, 0), (516, 33001, 2, 1.0, 0, 0)])
def test_distillation_over_shapes(T, V, K, tau, pad, offset, dtype):
    z = make_logits(T, V, dtype, seed=V, pad=pad, offset=offset)
    ids, teacher = make_teacher(z, K, seed=T)
    g = torch.Generator().manual_seed(7)
    weights = (torch.rand((T,), generator=g) - 0.2).to(DEV)             # (of either sign)
    if T > 2:
        weights[1] = 0.0
    loss, stats, grad = pkg.moe_distill_topk(z, ids, teacher, tau, weights=weights, gradient=True)
    torch.cuda.synchronize()
    rloss, rgrad = ref_distill(z, ids, teacher, tau, weights)
    tol = ABS * max(1.0, tau) ** 2 * 4
    assert float((loss.double().cpu() - rloss).abs().max()) <= tol + 1e-6 * float(rloss.abs().max())
    check_gradient(grad, rgrad, weights.abs() * tau, dtype)
    # the loss alone, and the gradient from its stats
    loss1, stats1 = pkg.moe_distill_topk(z, ids, teacher, tau)
    keep = weights != 0
    assert torch.equal(stats1[keep], stats[keep])
    back = pkg.moe_distill_topk_backward(z, ids, teacher, stats1, weights, tau)
    torch.cuda.synchronize()
    check_gradient(back, rgrad, weights.abs() * tau, dtype)
    assert float((loss1.double().cpu() - ref_distill(z, ids, teacher, tau)[0]).abs().max()) <= tol + 1e-6 * float(rloss.abs().max())
    # into the logits' own memory
    for own in ("forward", "backward"):
        z2 = torch.zeros(T * (V + pad) + offset, dtype=dtype, device=DEV)[offset:].view(T, V + pad)[:, :V]
        z2.copy_(z)
        if own == "forward":
            pkg.moe_distill_topk(z2, ids, teacher, tau, weights=weights, gradient=True, out=z2)
            assert torch.equal(z2, grad)
        else:
            pkg.moe_distill_topk_backward(z2, ids, teacher, stats1, weights, tau, out=z2)
            assert torch.equal(z2, back)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V", [70, 33000, 140000])
def test_distillation_of_masked_and_empty_rows(V, dtype):
    z = make_logits(10, V, dtype, seed=11)
    ids, teacher = make_teacher(z, 16, seed=12)
    low = torch.finfo(dtype).min
    ids[0] = -1                                             # no alternatives
    teacher[1] = -INF                                       # none either
    z[2] = -INF                                             # no distribution
    ids[3, 4:] = -1
    ids[3, 5], ids[3, 6] = V, 2 ** 31 - 1                   # not there
    teacher[4, 3:] = -INF
    ids[5] = ids[5, 0].item()                               # one alternative, sixteen times
    ids[6, 8:] = ids[6, :8].clone()                         # each twice
    z[7, :] = low
    z[8, : V // 2] = -INF
    ids[8] = (V // 2 + torch.arange(16, device=DEV)).to(torch.int32)
    weights = torch.ones(10, device=DEV)
    z[9], weights[9] = float("nan"), 0.0                    # left out, whatever it holds
    out = pkg.moe_distill_topk(z, ids, teacher, 1.5, weights=weights, gradient=True)
    loss, stats, grad = out
    rloss, rgrad = ref_distill(z, ids, teacher, 1.5, weights)
    assert bool(torch.isfinite(loss).all()) and bool(torch.isfinite(grad).all())
    assert float((loss.double().cpu() - rloss).abs().max()) <= 9 * ABS + 1e-6 * float(rloss.abs().max())
    check_gradient(grad, rgrad, weights * 1.5, dtype)
    for r in (0, 1, 2, 9):
        assert float(loss[r]) == 0.0 and not bool(grad[r].any())
    back = pkg.moe_distill_topk_backward(z, ids, teacher, stats, weights, 1.5)
    check_gradient(back, rgrad, weights * 1.5, dtype)
    # an alternative that the student has at -inf: the loss is infinite, the gradient is not
    z[6, ids[6, 0].long()] = -INF
    loss, _, grad = pkg.moe_distill_topk(z, ids, teacher, 1.5, weights=weights, gradient=True)
    assert float(loss[6]) == INF and bool(torch.isfinite(grad).all())
    check_gradient(grad, ref_distill(z, ids, teacher, 1.5, weights)[1], weights * 1.5, dtype)


def test_distillation_beyond_32_bit_offsets():
    V, T = 131072, 16400                                     # 2^31 elements and more, the gradient in the logits' own memory
    z = torch.zeros((T, V), dtype=torch.bfloat16, device=DEV)
    z[T - 1] = make_logits(1, V, torch.bfloat16, seed=5)[0]
    ids = torch.tensor([[70001, 131071]], dtype=torch.int32, device=DEV).repeat(T, 1).contiguous()
    teacher = torch.tensor([[1.0, 0.0]], device=DEV).repeat(T, 1).contiguous()
    last = [0, T - 2, T - 1]                                 # (all rows but the last are alike)
    rloss, ref = ref_distill(z[last], ids[last], teacher[last], 2.0)
    loss, stats, grad = pkg.moe_distill_topk(z, ids, teacher, temperature=2.0, gradient=True, out=z)
    assert grad.data_ptr() == z.data_ptr()
    assert float((loss[last].double().cpu() - rloss).abs().max()) <= ABS * 2.0 ** 2 * 4 + 1e-6 * float(rloss.abs().max())
    assert bool((loss[:-1] == loss[0]).all()) and all(torch.equal(grad[t], grad[0]) for t in range(16381, T - 1))
    check_gradient(grad[last], ref, torch.full((3,), 2.0), torch.bfloat16)


@pytest.mark.parametrize("V,K,tau", [(37, 5, 1.0), (1003, 20, 2.0), (9000, 64, 0.8)])
def test_distillation_gradient_against_differences(V, K, tau):
    """<grad, d> = (L(z + e d) - L(z - e d)) / 2 e + O(e^2 L'''): with e = 2^-5 and |d| <= 1, third derivatives of a log-sum-exp at most
    2 / tau^3, the remainder is under e^2 tau^2 / (3 tau^3) a row; the losses' own error 8 ABS tau^2 / 2 e."""
    T, e = 4, 2.0 ** -5
    z = make_logits(T, V, torch.float32, seed=V, scale=1.0)
    ids, teacher = make_teacher(z, K, seed=2)
    d = (torch.rand((T, V), generator=torch.Generator().manual_seed(3)) * 2 - 1).to(DEV)
    _, _, grad = pkg.moe_distill_topk(z, ids, teacher, tau, gradient=True)
    up, down = (pkg.moe_distill_topk(z + s * e * d, ids, teacher, tau)[0].double() for s in (1, -1))
    want, got = (up - down) / (2 * e), (grad.double() * d.double()).sum(1)
    assert bool(((want - got).abs() <= e * e / tau + 8 * ABS * tau ** 2 / (2 * e)).all()), (want, got)


def test_rows_on_another_stream_and_none_at_all():
    z = make_logits(40, 1003, torch.bfloat16, seed=20)
    ids, teacher = make_teacher(z, 8, seed=21)
    a, b = pkg.moe_token_logprobs(z, ids[:, 0].long().contiguous(), 4), pkg.moe_distill_topk(z, ids, teacher, gradient=True)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        c, d = pkg.moe_token_logprobs(z, ids[:, 0].long().contiguous(), 4), pkg.moe_distill_topk(z, ids, teacher, gradient=True)
    s.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(a + b, c + d))
    e = pkg.moe_token_logprobs(z[:0], ids[:0, 0].long(), 4)
    assert e[2].shape == (0, 4)
    assert pkg.moe_distill_topk(z[:0], ids[:0], teacher[:0], gradient=True)[2].shape == (0, 1003)


def test_rows_in_a_graph():
    z = make_logits(300, 5003, torch.bfloat16, seed=22)
    ids, teacher = make_teacher(z, 20, seed=23)
    tokens = ids[:, 0].long().contiguous()
    run = lambda: pkg.moe_token_logprobs(z, tokens, 4) + pkg.moe_distill_topk(z, ids, teacher, gradient=True)  # noqa: E731
    run()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = run()
    for seed in range(3):
        z.copy_(make_logits(300, 5003, torch.bfloat16, seed=30 + seed))
        want = run()
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(out, want))
