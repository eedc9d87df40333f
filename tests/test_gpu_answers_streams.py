"""moe_policy_loss and moe_preference_loss on logits that the caches do not hold: what a call reads past them beyond 134 MB (160 MB of the preference
loss) and writes past them beyond 268.5 MB, by every number of threads to a row and by rows that no workgroup holds.  All rows against the
definitions in 64 bits, with the bounds of test_gpu_answers.py."""
import pytest
import torch

import paper_2402_14800_amd as pkg
from tests.test_gpu_answers import BF16, DEV, EPS, F32, make_pairs
from tests.test_gpu_logits import ABS

pytestmark = pytest.mark.gpu


def make_rows(T, V, dtype, pad, seed):
    """[T, V] logits in rows of V + pad elements, other ones in every row and column; tokens, some of them without; lp in 64 bits."""
    g = torch.Generator(device=DEV).manual_seed(seed)
    z = torch.zeros(T * (V + pad), dtype=dtype, device=DEV).view(T, V + pad)[:, :V]
    tokens = torch.randint(0, V, (T,), generator=g, device=DEV)
    lp = torch.empty(T, dtype=torch.float64, device=DEV)
    for r in blocks(T, V):
        z[r] = (2.5 * torch.randn((len(tokens[r]), V), generator=g, device=DEV)).to(dtype)
        lp[r] = torch.log_softmax(z[r].double(), 1).gather(1, tokens[r, None])[:, 0]
    tokens[torch.rand(T, generator=g, device=DEV) < 0.1] = -1
    return z, tokens, lp, g


def blocks(T, V):
    step = max(1, (1 << 26) // V)
    return [slice(r, min(T, r + step)) for r in range(0, T, step)]


def check_rows(z, tokens, got, c, dc):
    """All of a gradient, c (onehot - p) by rows: `c` and `dc` the derivative by each row's lp and how far it may be off."""
    half = 2.0 ** -8 if z.dtype == BF16 else 0.0
    for r in blocks(*z.shape):
        p = torch.softmax(z[r].double(), 1)
        y = tokens[r].clamp(min=0)[:, None]
        g = (-p).scatter_add_(1, y, torch.ones_like(y, dtype=torch.float64))
        size = p.scatter_add_(1, y, torch.ones_like(y, dtype=torch.float64))
        cr, dr = c[r, None], dc[r, None]
        bound = half * (cr * g).abs() + dr * g.abs() + ABS * cr.abs() * (size + 1e-3) + 1e-38
        assert bool(((got[r].double() - cr * g).abs() <= bound).all()), r


# logits of 141 MB (read past the caches alone), then beyond 268.5 MB: rows held by 64, 128, 256, 512 and 1024 threads, and not held
@pytest.mark.parametrize("T,V,dtype,pad", [(2201, 32003, BF16, 5), (20001, 7001, BF16, 1), (14001, 10007, BF16, 0), (6001, 24003, BF16, 3), (4401, 32003, BF16, 1),
                                           (1101, 128003, BF16, 5), (1101, 131075, BF16, 0), (20001, 4001, F32, 3), (2201, 32003, F32, 1), (1001, 70003, F32, 0)])
def test_policy_loss_past_the_caches(T, V, dtype, pad):
    assert T * V * (2 if dtype == BF16 else 4) > (268.5e6 if T != 2201 or dtype == F32 else 134e6)
    z, tokens, lp, g = make_rows(T, V, dtype, pad, seed=V)
    d = 0.3 * torch.randn(T, generator=g, device=DEV).double()
    for border in (-0.2231435513, 0.1823215568):             # log 0.8 and log 1.2: no ratio next to the clip's bounds
        d = torch.where((d - border).abs() < 1e-2, torch.full_like(d, border + 2e-2), d)
    old, ref = (lp - d).float(), (lp + 0.3 * torch.randn(T, generator=g, device=DEV)).float()
    A, w = torch.randn(T, generator=g, device=DEV), torch.rand(T, generator=g, device=DEV) + 0.1
    w[5] = 0.0
    kl = 0.1
    given = (tokens >= 0) & (w != 0)
    r, e = torch.exp(lp - old.double()), ref.double() - lp
    inside = r.clamp(1 - 0.2, 1 + 0.2)
    want = -torch.minimum(r * A, inside * A) + kl * (torch.expm1(e) - e)
    c = torch.where(r * A <= inside * A, -r * A, 0.0) - kl * torch.expm1(e)
    off = ABS + 2.0 ** -22 * lp.abs()
    tol = 2 * off * ((r * A).abs() + kl * torch.expm1(e).abs()) + EPS * ((inside * A).abs() + (r * A).abs() + kl * (torch.expm1(e) - e))
    bend = (r * A).abs() + kl * torch.exp(e)
    loss, got, stats, grad = pkg.moe_policy_loss(z, tokens, old, A, ref, kl=kl, weights=w, gradient=True)
    zero = lambda v: torch.where(given, v, 0.0)  # noqa: E731
    assert bool(((got.double() - zero(lp)).abs() <= off).all())
    assert bool(((loss.double() - zero(want)).abs() <= zero(tol)).all())
    check_rows(z, tokens, grad, zero(c * w), zero(w * (2 * off + EPS) * bend))
    before = z.clone()
    assert torch.equal(pkg.moe_policy_loss(z, tokens, old, A, ref, kl=kl, weights=w, gradient=True, out=z)[3], grad)
    z.copy_(before)
    alone = pkg.moe_policy_loss(z, tokens, old, A, ref, kl=kl)
    back = pkg.moe_policy_loss_backward(z, tokens, alone[2], w, out=z)
    check_rows(before, tokens, back, zero(c * w), zero(w * (2 * off + EPS) * bend))


@pytest.mark.parametrize("T,V,dtype,pad,P", [(3301, 32003, BF16, 3, 8), (9001, 16384, BF16, 0, 100), (30001, 4001, BF16, 1, 3), (1301, 131075, BF16, 0, 5), (1501, 50001, F32, 1, 40),
                                             (231, 400003, BF16, 1, 3)])
def test_preference_loss_past_the_caches(T, V, dtype, pad, P):
    assert T * V * (2 if dtype == BF16 else 4) > 160e6
    z, tokens, lp, g = make_rows(T, V, dtype, pad, seed=T)
    offsets = make_pairs(T, P, seed=P, tail=7, head=3)
    ref = (lp + 0.4 * torch.randn(T, generator=g, device=DEV)).float()
    cut, beta = offsets.tolist(), float(torch.tensor(0.1))
    there = torch.zeros(T, dtype=torch.bool, device=DEV)
    there[cut[0]:cut[-1]] = True
    given = there & (tokens >= 0)
    off = ABS + 2.0 ** -22 * lp.abs()
    sums, offs, counts = [], [], []
    for a, b in zip(cut, cut[1:]):
        counts.append(max(1, int(given[a:b].sum())))
        sums.append(float((lp - ref.double())[a:b][given[a:b]].sum()) * beta / counts[-1])
        offs.append(float(off[a:b][given[a:b]].sum()) * beta / counts[-1])
    c, dc = torch.zeros(T, dtype=torch.float64, device=DEV), torch.zeros(T, dtype=torch.float64, device=DEV)
    rewards, far = torch.tensor(sums, dtype=torch.float64), torch.tensor(offs, dtype=torch.float64)
    h, dh = rewards[:P] - rewards[P:], far[:P] + far[P:] + 2.0 ** -40
    by_h = -torch.sigmoid(-h)
    for a in range(2 * P):
        rows = slice(cut[a], cut[a + 1])
        c[rows] = (1 if a < P else -1) * beta / counts[a] * float(by_h[a % P])
        dc[rows] = beta / counts[a] * float(dh[a % P] / 4 + EPS * by_h[a % P].abs())
    c, dc = torch.where(given, c, 0.0), torch.where(given, dc, 0.0)
    out = torch.full((T, V + pad), 5.0, dtype=dtype, device=DEV)[:, :V]
    loss, rew, got, stats, grad = pkg.moe_preference_loss(z, tokens, offsets, ref, 0.1, average=True, gradient=True, out=out)
    assert bool(((got.double() - torch.where(given, lp, 0.0)).abs() <= off).all())
    assert bool(((rew.double().cpu().view(-1) - rewards).abs() <= far + EPS * rewards.abs()).all())
    want = torch.nn.functional.softplus(-h)
    assert bool(((loss.double().cpu() - want).abs() <= dh + EPS * want).all())
    assert bool((grad[~there] == 5.0).all())
    check_rows(z[there], tokens[there], grad[there], c[there], dc[there])
    before = z.clone()
    pkg.moe_preference_loss(z, tokens, offsets, ref, 0.1, average=True, gradient=True, out=z)
    assert torch.equal(z[there], grad[there]) and torch.equal(z[~there], before[~there])
