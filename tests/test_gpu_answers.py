"""GPU parity of moe_policy_loss and moe_preference_loss with their definitions in 64 bits.

Bounds.  A log probability is off by ABS as in test_gpu_logits, and by 2^-22 of itself (its two subtractions and, with a temperature, a
division).  Call that e.  With r = exp(lp - old) the policy loss is off by what e makes of it, e (|r A| + kl |exp(d) - 1|), to first order;
e is under 1e-3 throughout, so twice that covers the rest; and by 2^-21 of its two terms for the exponentials and products themselves.  Its derivative c is off by e (|r A| +
kl exp(d)) and the same 2^-21.  A gradient c (onehot - p) / tau is off by that times |onehot - p| / tau, and by ABS (and
1e-3 ABS for the smallest p, whose exponents are large) of c (onehot + p) / tau; in bf16 by 2^-8 of itself more.  Of a pair, h is off by
beta times the sum of its rows' e (over their number with `average`), and the loss by as much, its derivative by a quarter of that."""
import math

import pytest
import torch

import paper_2402_14800_amd as pkg
from tests.test_gpu_logits import ABS, DEV, INF, make_logits

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16
EPS = 2.0 ** -21


def reference(z, tokens, tau=1.0):
    """log p of each row's token (of token 0 where none is given) and p, in 64 bits on the host."""
    logp = torch.log_softmax(z.double().cpu() / tau, 1)
    return logp.gather(1, tokens.cpu().clamp(min=0)[:, None])[:, 0], logp.exp()


def onehot_minus(p, tokens):
    g = -p
    g[torch.arange(len(p)), tokens.cpu().clamp(min=0)] += 1.0
    return g


def check_grad(got, c, dc, p, tokens, tau, dtype):
    """`c`, `dc`: the derivative by each row's lp and how far it may be off."""
    g = onehot_minus(p, tokens)
    want = c[:, None] * g / tau
    size = p.clone()
    size[torch.arange(len(p)), tokens.cpu().clamp(min=0)] += 1.0
    bound = (2.0 ** -8 if dtype == BF16 else 0.0) * want.abs() + dc[:, None] * g.abs() / tau + ABS * c.abs()[:, None] * (size + 1e-3) / tau
    d = (got.double().cpu() - want).abs()
    assert bool((d <= bound + 1e-38).all()), float((d - bound).max())


def make_policy(z, tokens, tau, seed, lo=0.2, hi=0.2, spread=0.3):
    """Old and reference log probabilities near the present ones, no ratio within 1e-2 of the clip's bounds."""
    g = torch.Generator().manual_seed(seed)
    lp, _ = reference(z, tokens, tau)
    T = len(lp)
    d = spread * torch.randn(T, generator=g).double()
    for border in (math.log1p(-lo) if lo < 1 else -100.0, math.log1p(hi)):
        d = torch.where((d - border).abs() < 1e-2, torch.full_like(d, border + 2e-2), d)
    lp = torch.nan_to_num(lp, neginf=-5.0)
    return ((lp - d).float().to(DEV), torch.randn(T, generator=g).to(DEV), (lp + 0.3 * torch.randn(T, generator=g)).float().to(DEV),
            (torch.rand(T, generator=g) + 0.1).to(DEV))


def ref_policy(z, tokens, old, A, ref, lo, hi, kl, tau):
    """loss, its derivative by lp, and how far each may be off; lp and p."""
    lp, p = reference(z, tokens, tau)
    old, A = old.double().cpu(), A.double().cpu()
    lo, hi = (float(torch.tensor(v, dtype=F32)) for v in (lo, hi))
    r = torch.exp(lp - old)
    inside = r.clamp(1 - lo, 1 + hi)
    loss, c = -torch.minimum(r * A, inside * A), torch.where(r * A <= inside * A, -r * A, 0.0)
    e = ABS + 2.0 ** -22 * lp.abs()
    size, moves, bends = (inside * A).abs() + (r * A).abs(), (r * A).abs(), (r * A).abs()
    if kl:
        d = ref.double().cpu() - lp
        loss, c = loss + kl * (torch.expm1(d) - d), c - kl * torch.expm1(d)
        size, moves, bends = size + kl * (torch.expm1(d) - d), moves + kl * torch.expm1(d).abs(), bends + kl * torch.exp(d)
    given = tokens.cpu() >= 0
    zero = lambda v: torch.where(given, v, 0.0)  # noqa: E731
    return zero(loss), zero(2 * e * moves + EPS * size), zero(c), zero(2 * e * bends + EPS * bends), torch.where(given, lp, 0.0), p


def check_policy(z, tokens, old, A, ref, weights=None, lo=0.2, hi=0.2, kl=0.1, tau=1.0):
    dtype, T = z.dtype, z.shape[0]
    rloss, tol, c, dc, rlp, p = ref_policy(z, tokens, old, A, ref, lo, hi, kl, tau)
    args = (z, tokens, old, A, ref if kl else None, lo, hi, kl, tau)
    loss, lp, stats, grad = pkg.moe_policy_loss(*args, weights=weights, gradient=True)
    torch.cuda.synchronize()
    w = torch.ones(T, dtype=torch.float64) if weights is None else weights.double().cpu()
    on = w != 0
    assert bool(((lp.double().cpu() - rlp).abs() <= ABS + 2.0 ** -22 * rlp.abs())[on].all())
    d = (loss.double().cpu() - rloss).abs()
    assert bool((d <= tol + 1e-38)[on].all()), float((d - tol)[on].max())
    assert not bool(loss.cpu()[~on].any()) and not bool(lp.cpu()[~on].any())
    check_grad(grad, c * w, dc * w.abs(), p, tokens, tau, dtype)
    loss1, lp1, stats1 = pkg.moe_policy_loss(*args)
    back = pkg.moe_policy_loss_backward(z, tokens, stats1, weights if weights is not None else torch.ones(T, device=DEV), tau)
    torch.cuda.synchronize()
    assert bool(((loss1.double().cpu() - rloss).abs() <= tol + 1e-38).all())
    check_grad(back, c * w, dc * w.abs(), p, tokens, tau, dtype)
    return grad, back, stats1


def again(z, pad, offset):
    T, V = z.shape
    z2 = torch.zeros(T * (V + pad) + offset, dtype=z.dtype, device=DEV)[offset:].view(T, V + pad)[:, :V]
    return z2.copy_(z)


SHAPES = [(1, 1, 1.0, 0, 0), (3, 7, 2.0, 0, 0), (5, 64, 1.0, 0, 1), (4, 257, 0.5, 3, 0), (33, 1003, 1.0, 0, 0), (2100, 301, 0.7, 0, 0),
          (2050, 4096, 1.0, 5, 3), (9, 8193, 1.3, 1, 0), (3, 32000, 2.0, 0, 0), (2, 50001, 1.0, 64, 7), (3, 131075, 1.0, 0, 0), (516, 33001, 1.0, 0, 0)]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("T,V,tau,pad,offset", SHAPES)
def test_policy_over_shapes(T, V, tau, pad, offset, dtype):
    z = make_logits(T, V, dtype, seed=V, pad=pad, offset=offset)
    tokens = torch.randint(0, V, (T,), generator=torch.Generator().manual_seed(T)).to(DEV)
    if T > 2:
        tokens[2] = -1
    old, A, ref, w = make_policy(z, tokens, tau, seed=T)
    if T > 1:
        w[1] = 0.0
    for kl in (0.0, 0.1):
        grad, back, stats = check_policy(z, tokens, old, A, ref, w, kl=kl, tau=tau)
    # into the logits' own memory, and into rows that start unlike the logits'
    z2 = again(z, pad, offset)
    pkg.moe_policy_loss(z2, tokens, old, A, ref, kl=0.1, temperature=tau, weights=w, gradient=True, out=z2)
    assert torch.equal(z2, grad)
    z2 = again(z, pad, offset)
    pkg.moe_policy_loss_backward(z2, tokens, stats, w, tau, out=z2)
    assert torch.equal(z2, back)
    wide = torch.full((T, V + 5), 3.0, dtype=dtype, device=DEV)
    pkg.moe_policy_loss(z, tokens, old, A, ref, kl=0.1, temperature=tau, weights=w, gradient=True, out=wide[:, 2:V + 2])
    assert torch.equal(wide[:, 2:V + 2], grad) and bool((wide[:, :2] == 3.0).all()) and bool((wide[:, V + 2:] == 3.0).all())


@pytest.mark.parametrize("lo,hi", [(0.0, 0.0), (1.0, 0.5), (0.2, 0.28), (0.1, 1000.0)])
def test_clip_bounds(lo, hi):
    z = make_logits(400, 130, F32, seed=1)
    tokens = torch.randint(0, 130, (400,), generator=torch.Generator().manual_seed(1)).to(DEV)
    old, A, ref, w = make_policy(z, tokens, 1.0, seed=2, lo=lo, hi=hi, spread=0.6)
    A[::7] = 0.0
    check_policy(z, tokens, old, A, ref, w, lo=lo, hi=hi, kl=0.0)
    check_policy(z, tokens, old, A, ref, w - 0.5, lo=lo, hi=hi, kl=0.3)                  # (weights of either sign)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("V", [70, 33000, 140000])
def test_policy_of_masked_and_empty_rows(V, dtype):
    low = torch.finfo(dtype).min
    z = make_logits(9, V, dtype, seed=11)
    tokens = (torch.arange(9, device=DEV) * 7 + 3) % V
    z[0, V // 2:] = -INF
    z[1, 40:] = low
    z[2] = low
    z[3] = 0.25
    z[4] = -z[4].abs() - 300.0
    tokens[0], tokens[1] = 3, 5
    old, A, ref, w = make_policy(z, tokens, 1.0, seed=13)
    z[5], tokens[5] = float("nan"), -7                       # left out, whatever it and its numbers hold
    old[5] = A[5] = ref[5] = float("nan")
    z[6], w[6] = float("nan"), 0.0
    keep = [0, 1, 2, 3, 4, 7, 8]
    loss, lp, stats, grad = pkg.moe_policy_loss(z, tokens, old, A, ref, kl=0.1, weights=w, gradient=True)
    for r in (5, 6):
        assert float(loss[r]) == 0.0 and float(lp[r]) == 0.0 and not bool(grad[r].any()) and stats[r].tolist() == [-INF, 0.0, 0.0]
    assert bool(torch.isfinite(loss).all()) and bool(torch.isfinite(grad).all())
    check_policy(z[keep], tokens[keep], old[keep], A[keep], ref[keep], w[keep])
    assert torch.equal(pkg.moe_policy_loss_backward(z, tokens, stats, torch.full((9,), float("inf"), device=DEV))[5:7].float(), torch.zeros((2, V), device=DEV))


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("V", [70, 33000])
def test_policy_beyond_its_range(V, dtype):
    """Tokens of probability 0, rows of nothing but -inf, ratios beyond 32 bits: the loss of the formula, and gradient 0 where it is
    infinite.  NaN in a row, or a token that does not exist: NaN.  The rows beside them stay whole."""
    z = make_logits(8, V, dtype, seed=14)
    tokens = torch.full((8,), 3, device=DEV)
    old, A, ref, _ = make_policy(z, tokens, 1.0, seed=15)
    A[:] = torch.tensor([1.0, -1.0, 1.0, -1.0, 0.0, 1.0, 1.0, 1.0], device=DEV)
    z[0, 3] = z[1, 3] = -INF                                 # r = 0
    z[2] = -INF
    old[3] = old[4] = -200.0                                 # r = exp(190 or so)
    z[5, V - 1] = float("nan")
    tokens[6] = V
    for kl in (0.0, 0.1):
        loss, lp, stats, grad = pkg.moe_policy_loss(z, tokens, old, A, ref, kl=kl, gradient=True)
        if kl == 0:
            assert float(loss[0]) == 0.0 and abs(float(loss[1]) - 0.8) <= 1e-6 and float(loss[2]) == 0.0 and float(loss[4]) == 0.0
        else:
            assert float(loss[0]) == INF and float(loss[1]) == INF and float(loss[2]) == INF and math.isfinite(float(loss[4]))
        assert float(loss[3]) == INF and float(lp[0]) == -INF and float(lp[2]) == -INF
        assert not bool(grad[:4].any()) and bool(torch.isfinite(grad[4]).all()) and bool(torch.isnan(loss[5:7]).all())
        assert bool(torch.isnan(grad[5:7]).all())
        back = pkg.moe_policy_loss_backward(z, tokens, stats, torch.ones(8, device=DEV))
        assert not bool(back[:4].any()) and bool(torch.isnan(back[6]).all())
        check_policy(z[7:], tokens[7:], old[7:], A[7:], ref[7:], kl=kl)


@pytest.mark.parametrize("kl", [0.0, 0.1])
def test_an_advantage_of_zero_hides_no_nan(kl):
    """A token that does not exist, and NaN in a row, show in its loss and gradient whatever the advantage."""
    z = make_logits(3, 70, F32, seed=18)
    z[1, 69] = float("nan")
    tokens = torch.tensor([70, 3, 3], device=DEV)
    old, A, ref, _ = make_policy(z[2:].expand(3, 70), torch.full((3,), 3), 1.0, seed=19)
    loss, lp, stats, grad = pkg.moe_policy_loss(z, tokens, old, torch.zeros_like(A), ref, kl=kl, gradient=True)
    back = pkg.moe_policy_loss_backward(z, tokens, stats, torch.ones(3, device=DEV))
    for got in (loss, lp, grad, back):
        assert bool(torch.isnan(got[:2]).all()) and bool(torch.isfinite(got[2]).all())
    assert kl or (float(loss[2]) == 0.0 and not bool(grad[2].any()))


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("tau", [2.0 ** -60, 2.0 ** -20, 2.0 ** 20, 2.0 ** 60])
def test_policy_at_the_temperatures_ends(tau, dtype):
    T, V = 6, 1003
    z = make_logits(T, V, dtype, seed=44)
    tokens = z.float().argmax(1)
    old, A, _, w = make_policy(z, tokens, tau, seed=45)
    check_policy(z, tokens, old, A, None, w, kl=0.0, tau=tau)


def test_policy_gradient_against_differences():
    """<grad, d> = (L(z + e d) - L(z - e d)) / 2 e + O(e^2): with e = 2^-6, |d| <= 1 and ratios that stay within 2, lp has derivatives along d of at
    most 2, 1 and 2 (of a log-sum-exp), so the third one of r A + kl terms is under (2 + 0.3) (2^3 + 3 * 2 * 1 + 2) = 37, the remainder under 37 / 6 e^2;
    the losses' own error is under 5 ABS, over 2 e.  No ratio crosses a bound: those within 4 e of one are moved away first."""
    T, V, e = 64, 203, 2.0 ** -6
    z = make_logits(T, V, F32, seed=3, scale=1.0)
    tokens = torch.randint(0, V, (T,), generator=torch.Generator().manual_seed(3)).to(DEV)
    lp = reference(z, tokens)[0]
    # (the ratios: inside the bounds, beyond either)
    d = torch.tensor([0.0, 0.05, -0.08, 0.5, -0.5]).double()[torch.arange(T) % 5]
    old, ref = (lp - d).float().to(DEV), (lp + 0.2).float().to(DEV)
    A = (torch.rand(T, generator=torch.Generator().manual_seed(4)) * 2 - 1).to(DEV)
    step = (torch.rand((T, V), generator=torch.Generator().manual_seed(5)) * 2 - 1).to(DEV)
    at = lambda q: pkg.moe_policy_loss(z + q * step, tokens, old, A, ref, kl=0.1)[0].double()  # noqa: E731
    grad = pkg.moe_policy_loss(z, tokens, old, A, ref, kl=0.1, gradient=True)[3]
    want, got = (at(e) - at(-e)) / (2 * e), (grad.double() * step.double()).sum(1)
    assert bool(((want - got).abs() <= 37 / 6 * e * e + 5 * ABS / e).all()), (want - got).abs().max()


# ---------------------------------------------------------------- pairs
def ref_pairs(z, tokens, offsets, ref, beta, ls, average, weights=None):
    beta, ls = (float(torch.tensor(v, dtype=F32)) for v in (beta, ls))
    lp, p = reference(z, tokens)
    cut, P, T = offsets.tolist(), offsets.shape[0] // 2, z.shape[0]
    given = tokens.cpu() >= 0
    inside = torch.zeros(T, dtype=torch.bool)
    inside[cut[0]:cut[-1]] = True
    lp = torch.where(given & inside, lp, 0.0)
    e = ABS + 2.0 ** -22 * lp.abs()
    rewards, off, by = torch.zeros(2 * P).double(), torch.zeros(2 * P).double(), torch.zeros(2 * P).double()
    ratio = lp - ref.double().cpu()
    for a in range(2 * P):
        t = torch.arange(cut[a], cut[a + 1])
        t = t[given[t]]
        by[a] = beta / (max(1, len(t)) if average else 1)
        rewards[a], off[a] = by[a] * ratio[t].sum(), by[a] * e[t].sum()
    h = rewards[:P] - rewards[P:]
    dh = off[:P] + off[P:] + 2.0 ** -40
    soft = torch.nn.functional.softplus
    loss = (1 - ls) * soft(-h) + (ls * soft(h) if ls else 0.0)
    by_h = ls - torch.sigmoid(-h)
    w = torch.ones(P, dtype=torch.float64) if weights is None else weights.double().cpu()
    c, dc = torch.zeros(T, dtype=torch.float64), torch.zeros(T, dtype=torch.float64)
    for a in range(2 * P):
        t, i = slice(cut[a], cut[a + 1]), a % P
        c[t] = (1 if a < P else -1) * by[a] * by_h[i] * w[i]
        dc[t] = by[a] * w[i].abs() * (dh[i] / 4 + EPS * by_h[i].abs())
    return loss, dh + EPS * loss, rewards, off + EPS * rewards.abs(), torch.where(given, c, 0.0), torch.where(given, dc, 0.0), lp, e, p, inside


def check_pairs(z, tokens, offsets, ref, beta=0.1, ls=0.0, average=False, weights=None):
    dtype, (T, V), P = z.dtype, z.shape, offsets.shape[0] // 2
    rloss, tol, rrew, rtol, c, dc, rlp, e, p, inside = ref_pairs(z, tokens, offsets, ref, beta, ls, average, weights)
    args = (z, tokens, offsets, ref, beta, ls, average)
    out = torch.full((T, V), 5.0, dtype=dtype, device=DEV)
    loss, rew, lp, stats, grad = pkg.moe_preference_loss(*args, weights=weights, gradient=True, out=out)
    torch.cuda.synchronize()
    assert grad is out and bool((out[~inside.to(DEV)] == 5.0).all())
    assert bool(((lp.double().cpu() - rlp).abs() <= e).all())
    assert bool(((rew.double().cpu().view(-1) - rrew).abs() <= rtol + 1e-38).all())
    assert bool(((loss.double().cpu() - rloss).abs() <= tol).all())
    if bool(inside.any()):
        check_grad(grad[inside.to(DEV)], c[inside], dc[inside], p[inside], tokens.cpu()[inside], 1.0, dtype)
    loss1, rew1, lp1, stats1 = pkg.moe_preference_loss(*args)
    assert all(torch.equal(a, b) for a, b in zip((loss, rew, lp, stats), (loss1, rew1, lp1, stats1)))
    up = weights if weights is not None else torch.ones(P, device=DEV)
    back = pkg.moe_preference_loss_backward(z, tokens, offsets, stats1, up, out=torch.full((T, V), 5.0, dtype=dtype, device=DEV))
    assert torch.equal(back, grad)
    return grad, stats


def make_pairs(T, P, seed, tail=0, head=0):
    g = torch.Generator().manual_seed(seed)
    cuts = torch.sort(torch.randint(head, T - tail + 1, (2 * P - 1,), generator=g)).values
    return torch.cat([torch.tensor([head]), cuts, torch.tensor([T - tail])]).to(DEV)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("T,V,P,pad,offset,tail,head", [
    (2, 1, 1, 0, 0, 0, 0), (1, 7, 1, 0, 0, 0, 0), (9, 64, 2, 0, 1, 1, 0), (40, 257, 31, 3, 0, 4, 3), (64, 1003, 32, 0, 0, 5, 0), (300, 130, 40, 0, 0, 0, 7),
    (2300, 301, 6, 0, 0, 100, 0), (2050, 4096, 3, 5, 3, 2, 2), (700, 40, 2100, 0, 0, 3, 0), (12, 32000, 2, 0, 0, 1, 0), (5, 50001, 2, 64, 7, 0, 0),
    (6, 131075, 1, 0, 0, 1, 1), (3, 300007, 1, 0, 0, 0, 0)])
def test_pairs_over_shapes(T, V, P, pad, offset, tail, head, dtype):
    z = make_logits(T, V, dtype, seed=V, pad=pad, offset=offset)
    g = torch.Generator().manual_seed(T + P)
    tokens = torch.randint(0, V, (T,), generator=g)
    tokens[torch.rand(T, generator=g) < 0.2] = -100          # the prompts'
    tokens = tokens.to(DEV)
    offsets = make_pairs(T, P, seed=P, tail=tail, head=head)
    ref = (reference(z, tokens)[0] + 0.4 * torch.randn(T, generator=g)).float().to(DEV)
    w = (torch.rand(P, generator=g) - 0.2).to(DEV)
    w[P // 2] = 0.0
    check_pairs(z, tokens, offsets, ref)
    check_pairs(z, tokens, offsets, ref, beta=0.7, ls=0.1, average=True)
    grad, stats = check_pairs(z, tokens, offsets, ref, beta=0.3, weights=w)
    # into the logits' own memory
    z2 = again(z, pad, offset)
    pkg.moe_preference_loss(z2, tokens, offsets, ref, 0.3, weights=w, gradient=True, out=z2)
    rows = slice(head, T - tail)
    assert torch.equal(z2[rows], grad[rows]) and torch.equal(z2[:head], z[:head]) and torch.equal(z2[T - tail:], z[T - tail:])
    z2 = again(z, pad, offset)
    pkg.moe_preference_loss_backward(z2, tokens, offsets, stats, w, out=z2)
    assert torch.equal(z2[rows], grad[rows]) and torch.equal(z2[T - tail:], z[T - tail:])


def test_pairs_far_apart_and_of_nothing():
    """Margins that a sigmoid in 32 bits has no number for, empty answers, answers without a token; log 2 for pairs of equals."""
    T, V, P = 40, 50, 4
    z = make_logits(T, V, F32, seed=5)
    tokens = torch.arange(T, device=DEV) % V
    offsets = torch.tensor([0, 10, 10, 10, 20, 30, 30, 30, 40], device=DEV)
    tokens[20:30] = -1                                       # pair 0: ten tokens against ten without; 1: nothing against nothing
    ref = reference(z, tokens)[0].float().to(DEV)
    ref[:10] -= 300.0
    ref[30:] += 50.0
    ref[20:30] = float("nan")                                # (not read)
    z[20:30] = float("inf")
    loss, rew, lp, stats, grad = pkg.moe_preference_loss(z, tokens, offsets, ref, 1.0, gradient=True)
    assert bool(torch.isfinite(loss).all()) and bool(torch.isfinite(grad).all()) and not bool(grad[20:30].any())
    assert abs(float(loss[1]) - math.log(2)) <= 1e-6 and abs(float(loss[2]) - math.log(2)) <= 1e-6
    assert float(loss[0]) <= 1e-30 and abs(float(rew[0, 0]) - 3000) <= 1e-2
    swapped = torch.tensor([30, 40], device=DEV)             # the other way round the loss is the margin
    check = pkg.moe_preference_loss(z[30:], tokens[30:], torch.tensor([0, 0, 10], device=DEV), ref[30:], 1.0)
    assert len(swapped) == 2 and abs(float(check[0]) - math.log1p(math.exp(-500.0))) <= 1e-3
    check = pkg.moe_preference_loss(z[30:], tokens[30:], torch.tensor([0, 10, 10], device=DEV), ref[30:], 1.0, gradient=True)
    assert abs(float(check[0]) - 500.0) <= 1e-2
    want = -onehot_minus(reference(z[30:], tokens[30:])[1], tokens[30:])                   # (the sigmoid is 1)
    assert float((check[4].double().cpu() - want).abs().max()) <= 2 * ABS


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_pairs_with_masked_tokens(dtype):
    """A token of probability 0, a row of nothing but -inf, a lowest value as a mask: the formula's loss, and gradients that are numbers.  A
    token that does not exist: NaN for its pair, the other pair whole."""
    T, V = 24, 300
    z = make_logits(T, V, dtype, seed=6)
    tokens = torch.arange(T, device=DEV)
    ref = reference(z, tokens)[0].float().to(DEV)
    offsets = torch.tensor([0, 6, 12, 18, 24], device=DEV)
    z[1, 1] = -INF
    z[13] = z[13]
    loss, rew, lp, stats, grad = pkg.moe_preference_loss(z, tokens, offsets, ref, 0.5, gradient=True)
    assert float(lp[1]) == -INF and float(rew[0, 0]) == -INF and float(loss[0]) == INF and bool(torch.isfinite(grad).all())
    z[1] = -INF                                              # (no distribution: no gradient)
    loss, rew, lp, stats, grad = pkg.moe_preference_loss(z, tokens, offsets, ref, 0.5, gradient=True)
    assert float(loss[0]) == INF and bool(torch.isfinite(grad).all()) and not bool(grad[1].any())
    z[1] = torch.finfo(dtype).min
    z[1, 1:] = 0.0
    tokens[1] = 0
    loss, rew, lp, stats, grad = pkg.moe_preference_loss(z, tokens, offsets, ref, 0.5, gradient=True)
    low = -0.5 * torch.finfo(dtype).min
    assert abs(float(loss[0]) - low) <= 1e-5 * low and bool(torch.isfinite(grad).all())
    tokens[14] = V
    loss, rew, lp, stats, grad = pkg.moe_preference_loss(z, tokens, offsets, ref, 0.5, gradient=True)
    assert bool(torch.isnan(loss[0])) and bool(torch.isnan(lp[14])) and math.isfinite(float(loss[1]))
    check_pairs(z[6:12].contiguous(), tokens[6:12].contiguous() % V, torch.tensor([0, 3, 6], device=DEV), ref[6:12].contiguous(), beta=0.5)


def test_offsets_in_no_order_stay_within_the_arrays():
    """Unspecified results, but no row behind the logits is read or written."""
    T, V, P = 50, 70, 5
    z = make_logits(T, V, F32, seed=7)
    tokens, ref = torch.arange(T, device=DEV), torch.zeros(T, device=DEV)
    room = torch.full((T + 20, V), 9.0, device=DEV)
    for offsets in ([50, 3, 40, 2, 2, 49, 50, 0, 9, 1, 50], [0, 5, 9, 70, 900, 2 ** 62, 50, 50, 50, 50, 2 ** 62], [-5, -2 ** 62, 3, 4, 5, 6, 7, 8, 9, 10, 50]):
        pkg.moe_preference_loss(z, tokens, torch.tensor(offsets, device=DEV), ref, gradient=True, out=room[10:T + 10])
        torch.cuda.synchronize()
        assert bool((room[:10] == 9.0).all()) and bool((room[T + 10:] == 9.0).all())


def test_pair_gradient_against_differences():
    """As for the policy loss: h moves by beta times the sum over 2 x 10 rows, whose lp have derivatives of at most 2, 1 and 2 along d, |d| <= 1, so with
    beta = 0.02 h has under 0.8, 0.4 and 0.8; the loss's third derivative is under 0.1 * 0.8^3 + 3 * 0.25 * 0.8 * 0.4 + 0.8 = 1.1."""
    T, V, e = 40, 203, 2.0 ** -5
    z = make_logits(T, V, F32, seed=8, scale=1.0)
    tokens = torch.arange(T, device=DEV)
    offsets = torch.tensor([0, 10, 20, 30, 40], device=DEV)
    ref = (reference(z, tokens)[0] + 0.3 * torch.randn(T, generator=torch.Generator().manual_seed(8))).float().to(DEV)
    step = (torch.rand((T, V), generator=torch.Generator().manual_seed(9)) * 2 - 1).to(DEV)
    for ls in (0.0, 0.2):
        grad = pkg.moe_preference_loss(z, tokens, offsets, ref, 0.02, ls, gradient=True)[4]
        at = lambda q: pkg.moe_preference_loss(z + q * step, tokens, offsets, ref, 0.02, ls)[0].double()  # noqa: E731
        got = (grad.double() * step.double()).sum(1).view(4, 10).sum(1)
        want = (at(e) - at(-e)) / (2 * e)
        bound = 1.1 / 6 * e * e + 2 * (0.02 * 20 * 2 * ABS) / (2 * e)
        assert bool(((got[:2] + got[2:] - want).abs() <= bound).all())


# ---------------------------------------------------------------- both
def test_answers_beyond_32_bit_offsets():
    V, T = 131072, 16400                                     # 2^31 elements and more, the gradient in the logits' own memory
    z = torch.zeros((T, V), dtype=BF16, device=DEV)
    z[T - 1] = make_logits(1, V, BF16, seed=5)[0]
    z[:, 70001] += 9.0
    last = [0, T - 2, T - 1]                                 # (all rows but the last are alike)
    tokens = torch.full((T,), 70001, device=DEV)
    lp3, p3 = reference(z[last], tokens[last])
    old, A = torch.full((T,), float(lp3[0]), device=DEV), torch.ones(T, device=DEV)
    old[-1] = float(lp3[2])
    before = z[last].clone()
    loss, lp, stats = pkg.moe_policy_loss(z, tokens, old, A)
    grad = pkg.moe_policy_loss_backward(z, tokens, stats, A, out=z)
    assert float((lp[last].double().cpu() - lp3).abs().max()) <= ABS
    r = torch.exp(lp3 - old[last].double().cpu())
    check_grad(grad[last], -r, 2 * ABS * r, p3, tokens[last], 1.0, BF16)
    assert all(torch.equal(grad[t], grad[0]) for t in range(16381, T - 1))
    z[last] = before
    z[1:T - 2] = before[0]
    offsets = torch.tensor([0, T - 1, T], device=DEV)
    loss, rew, lp, stats, grad = pkg.moe_preference_loss(z, tokens, offsets, old, 1e-4, gradient=True, out=z)
    by_h = -torch.sigmoid(-(rew[0, 0] - rew[1, 0])).double().cpu()
    c = torch.stack([by_h, by_h, -by_h]) * 1e-4
    check_grad(grad[last], c, c.abs() * 1e-3, p3, tokens[last], 1.0, BF16)
    assert all(torch.equal(grad[t], grad[0]) for t in range(16381, T - 1))


def test_more_rows_than_a_launch_has():
    T, V = (1 << 22) + 1001, 3
    z = make_logits(T, V, BF16, seed=6)
    tokens = torch.arange(T, device=DEV) % V
    logp = torch.log_softmax(z.double(), 1)
    lp = logp.gather(1, tokens[:, None])[:, 0]
    g = -logp.exp()
    g[torch.arange(T, device=DEV), tokens] += 1.0
    old, A = lp.float(), torch.ones(T, device=DEV)
    loss, got, stats, grad = pkg.moe_policy_loss(z, tokens, old, A, gradient=True)
    back = pkg.moe_policy_loss_backward(z, tokens, stats, A)
    assert float((got.double() - lp).abs().max()) <= ABS and float((loss + 1.0).abs().max()) <= 4 * ABS
    for x in (grad, back):
        assert float((x.double() + g).abs().max()) <= 2.0 ** -8
    # one answer over the launches' border against a short one
    offsets = torch.tensor([100, T - 50, T - 9], device=DEV)
    ref = (lp + 0.25 * torch.rand(T, device=DEV) / T).float()
    loss, rew, got, stats, grad = pkg.moe_preference_loss(z, tokens, offsets, ref, 1.0, average=True, gradient=True, out=torch.full_like(z, 2.0))
    ratio = lp - ref.double()
    want = ratio[100:T - 50].mean() - ratio[T - 50:T - 9].mean()
    assert abs(float(loss[0]) - math.log1p(math.exp(-float(want)))) <= 2 * ABS
    assert bool((grad[:100] == 2.0).all()) and bool((grad[T - 9:] == 2.0).all())
    c = torch.full((T, 1), -0.5 / (T - 150), dtype=torch.float64, device=DEV)
    c[T - 50:] = 0.5 / 41
    d = (grad.double() - c * g)[100:T - 9].abs()
    assert bool((d <= (2.0 ** -8 * (c * g).abs() + 4 * ABS * c.abs())[100:T - 9]).all())


def test_answers_on_other_streams_and_none_at_all():
    T, V, P = 60, 5003, 4
    z = make_logits(T, V, BF16, seed=20)
    tokens = torch.arange(T, device=DEV)
    old, A, ref, w = make_policy(z, tokens, 1.0, seed=21)
    offsets = make_pairs(T, P, seed=22)
    run = lambda: (*pkg.moe_policy_loss(z, tokens, old, A, ref, kl=0.1, weights=w, gradient=True),  # noqa: E731
                   *pkg.moe_preference_loss(z, tokens, offsets, ref, gradient=True))
    a = run()
    torch.cuda.synchronize()
    outs = []
    for s in [torch.cuda.Stream(), torch.cuda.Stream()]:     # two calls in flight at once
        with torch.cuda.stream(s):
            outs.append(run())
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for out in outs for x, y in zip(a, out))
    none = pkg.moe_policy_loss(z[:0], tokens[:0], old[:0], A[:0], gradient=True)
    assert none[0].shape == (0,) and none[3].shape == (0, V)
    loss, rew, *_ = pkg.moe_preference_loss(z[:0], tokens[:0], torch.zeros(7, dtype=torch.int64, device=DEV), ref[:0], gradient=True)
    assert float((loss - math.log(2)).abs().max()) <= 1e-6 and not bool(rew.any())
    loss, rew, lp, stats = pkg.moe_preference_loss(z, tokens, torch.zeros(1, dtype=torch.int64, device=DEV), ref)
    assert loss.shape == (0,) and rew.shape == (2, 0) and not bool(lp.any()) and not bool(stats[:, 1:].any())


def test_refusals_on_the_gpu():
    z, t, f = torch.zeros((4, 8), device=DEV), torch.zeros(4, dtype=torch.int64, device=DEV), torch.zeros(4, device=DEV)
    for bad in (lambda: pkg.moe_policy_loss(z, t.int(), f, f), lambda: pkg.moe_policy_loss(z, t, f.cpu(), f), lambda: pkg.moe_policy_loss(z, t, f, f[:3]),
                lambda: pkg.moe_policy_loss(z.t(), t, f, f), lambda: pkg.moe_policy_loss(z, t, f, f, gradient=True, out=z.to(BF16)),
                lambda: pkg.moe_policy_loss(z, t, f, f[:1].expand(4)), lambda: pkg.moe_policy_loss_backward(z, t, z[:, :2], f),
                lambda: pkg.moe_preference_loss(z, t, t, f), lambda: pkg.moe_preference_loss(z, t, t[:3].int(), f),
                lambda: pkg.moe_preference_loss(z, t, t[:3], f, weights=f), lambda: pkg.moe_preference_loss_backward(z, t, t[:3].cpu(), z[:, :3], f[:1])):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: pkg.moe_policy_loss(z, t, f, f, kl=0.1), lambda: pkg.moe_policy_loss(z, t, f, f, clip_low=2.0),
                lambda: pkg.moe_policy_loss(z, t, f, f, temperature=0.0), lambda: pkg.moe_preference_loss(z, t, t[:3], f, beta=0.0)):
        with pytest.raises(pkg.MoepError):
            bad()


def test_answers_in_a_graph():
    T, V, P = 300, 5003, 5
    z = make_logits(T, V, BF16, seed=22)
    tokens = torch.arange(T, device=DEV)
    old, A, ref, w = make_policy(z, tokens, 1.0, seed=23)
    offsets = make_pairs(T, P, seed=24)
    outs = [torch.zeros_like(z) for _ in range(2)]

    def run(out):
        a = pkg.moe_policy_loss(z, tokens, old, A, ref, kl=0.1, weights=w, gradient=True)
        b = pkg.moe_preference_loss(z, tokens, offsets, ref, gradient=True, out=out)
        return a + b + (pkg.moe_policy_loss_backward(z, tokens, a[2], w),)

    run(outs[0])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = run(outs[1])
    for seed in range(3):
        z.copy_(make_logits(T, V, BF16, seed=30 + seed))
        offsets.copy_(make_pairs(T, P, seed=40 + seed, tail=seed))
        for out in outs:
            out.zero_()
        want = run(outs[0])
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(got, want))
