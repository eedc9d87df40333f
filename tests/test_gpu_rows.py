"""GPU parity of moe_dispatch_rows, moe_combine_rows and their gradients with their definitions in 64 bits.

Bounds.  A sum of k products in 32 bits is off by at most (k + 1) 2^-24 of the sum of their magnitudes, a result in bf16 by 2^-8 of itself
more, dy (one product) by 2^-24 and 2^-8.  A weight's gradient is added up by lanes: L products one after the other and at most 8 sums
over lanes and wavefronts, so (L + 9) 2^-24 of the sum of the magnitudes, L at most 16 / size times the chunks of a row over the lanes."""
import pytest
import torch

import paper_2402_14800_amd as pkg

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F32, BF16 = torch.float32, torch.bfloat16


def make_routing(T, k, E, seed, use=False):
    g = torch.Generator().manual_seed(seed)
    score = torch.randn((T, E), generator=g) + 0.7 * torch.randn((1, E), generator=g)
    experts = torch.topk(score, min(k, E), dim=1).indices
    if k > E:
        experts = torch.randint(0, E, (T, k), generator=g)
    used = torch.randint(0, k + 1, (T,), generator=g).to(torch.int32) if use else None
    return experts.to(torch.int32), used


def ref_slots(experts, used, E):
    """Slot by slot, from the definition."""
    T, k = experts.shape
    there = (experts >= 0) & (experts < E)
    if used is not None:
        there &= torch.arange(k) < used[:, None]
    flat = torch.where(there, experts, E).reshape(-1).long()
    order = torch.sort(flat, stable=True).indices[: int(there.sum())]
    slot = torch.full((T * k,), -1, dtype=torch.int32)
    slot[order] = torch.arange(len(order), dtype=torch.int32)
    offsets = torch.cat([torch.zeros(1, dtype=torch.int64), torch.bincount(flat, minlength=E + 1)[:E].cumsum(0)]).to(torch.int32)
    return slot.view(T, k), offsets, order


def check_dispatch(x, experts, used, E):
    T, k = experts.shape
    rows = torch.full((T * k, x.shape[1]), 7.0, dtype=x.dtype, device=DEV)
    got, slot_of, offsets = pkg.moe_dispatch_rows(x, experts.to(DEV), E, used=None if used is None else used.to(DEV), rows=rows)
    torch.cuda.synchronize()
    slot, off, order = ref_slots(experts, used, E)
    assert got is rows and torch.equal(slot_of.cpu(), slot) and torch.equal(offsets.cpu(), off)
    n = len(order)
    assert torch.equal(rows[:n], x[(order // k).to(DEV)])
    assert bool((rows[n:] == 7.0).all())                     # behind the last: as they were
    return slot_of


def close(got, want, magnitude, terms, dtype):
    half = 2.0 ** -8 if dtype == BF16 else 0.0
    return bool(((got.double() - want).abs() <= half * want.abs() + (terms + 1) * 2.0 ** -24 * magnitude + 1e-38).all())


def check_sums(T, k, H, dtype, slot_of, R, seed, weighted=True):
    g = torch.Generator(device=DEV).manual_seed(seed)
    y = torch.randn((R, H), generator=g, device=DEV).to(dtype)
    w = torch.randn((T, k), generator=g, device=DEV) if weighted else None
    dout = torch.randn((T, H), generator=g, device=DEV).to(dtype)
    there = (slot_of >= 0) & (slot_of < R)
    w64 = (w.double() if weighted else torch.ones((T, k), dtype=torch.float64, device=DEV)) * there
    out, mag = torch.zeros((T, H), dtype=torch.float64, device=DEV), torch.zeros((T, H), dtype=torch.float64, device=DEV)
    dw, dw_mag = torch.zeros((T, k), dtype=torch.float64, device=DEV), torch.zeros((T, k), dtype=torch.float64, device=DEV)
    dy, named = torch.zeros((R, H), dtype=torch.float64, device=DEV), torch.zeros(R, dtype=torch.bool, device=DEV)
    for j in range(k):
        t = there[:, j].nonzero()[:, 0]
        at = slot_of[t, j].long()
        term = w64[t, j, None] * y[at].double()
        out[t] += term
        mag[t] += term.abs()
        products = dout[t].double() * y[at].double()
        dw[t, j], dw_mag[t, j] = products.sum(1), products.abs().sum(1)
        dy[at], named[at] = w64[t, j, None] * dout[t].double(), True
    got = pkg.moe_combine_rows(y, slot_of, w) if weighted else pkg.moe_dispatch_rows_backward(y, slot_of)
    assert got.dtype == dtype and close(got, out, mag, k, dtype)
    before = torch.full((R, H), -3.0, dtype=dtype, device=DEV)
    got_dy, got_dw = pkg.moe_combine_rows_backward(dout, y, slot_of, w, dy=before)
    assert got_dy is before and bool((before[~named] == -3.0).all())
    assert close(got_dy[named], dy[named], dy[named].abs(), 0, dtype)
    n = 16 // y.element_size()
    chunks = H // n
    lanes = 64
    while lanes > 1 and lanes // 2 >= chunks:
        lanes //= 2
    per_lane = n * -(-chunks // lanes)
    assert bool(((got_dw.double() - dw).abs() <= (per_lane + 9) * 2.0 ** -24 * dw_mag + 1e-38).all())
    assert not bool(got_dw[~there].any())
    only, none = pkg.moe_combine_rows_backward(dout, y, slot_of, w, weight_gradient=False)
    assert none is None and torch.equal(only[named], got_dy[named])
    # into y's own memory, whose rows that no slot names stay
    y2 = y.clone()
    pkg.moe_combine_rows_backward(dout, y2, slot_of, w, dy=y2)
    assert torch.equal(y2[named], got_dy[named]) and torch.equal(y2[~named], y[~named])
    return got


# one token to many pieces, one to sixteen slots, rows of one chunk to many, on both sides of 256, 1024, 4096 and 8192 slots
SHAPES = [(1, 1, 1, 64), (1, 2, 8, 4096), (512, 2, 8, 64), (513, 2, 8, 128), (1024, 4, 8, 64), (2, 16, 32, 128), (7, 3, 5, 192), (63, 2, 8, 320), (65, 5, 16, 64), (300, 16, 3, 64), (777, 8, 32, 1024),
          (1025, 1, 2, 512), (2047, 4, 16, 256), (2049, 4, 16, 2048), (2050, 2, 8, 576), (2049, 2, 8, 128), (8192, 1, 8, 64), (4097, 2, 8, 64), (5003, 6, 32, 128), (33000, 2, 8, 64)]


@pytest.mark.parametrize("use", [False, True])
@pytest.mark.parametrize("T,k,E,H", SHAPES)
def test_rows_there_and_back(T, k, E, H, use):
    for dtype in (BF16, F32):
        experts, used = make_routing(T, k, E, seed=T + k, use=use)
        x = torch.randn((T, H), generator=torch.Generator(device=DEV).manual_seed(T), device=DEV).to(dtype)
        slot_of = check_dispatch(x, experts, used, E)
        for weighted in (True, False):
            check_sums(T, k, H, dtype, slot_of, T * k, seed=H, weighted=weighted)


@pytest.mark.parametrize("T,k,E,H", [(1, 1, 1, 4), (5, 2, 4, 12), (130, 3, 32, 20), (777, 4, 32, 1012), (3000, 4, 7, 36), (2500, 2, 9, 1028)])
def test_odd_rows_in_fp32(T, k, E, H):
    experts, used = make_routing(T, k, E, seed=H, use=True)
    x = torch.randn((T, H), device=DEV, generator=torch.Generator(device=DEV).manual_seed(2))
    check_sums(T, k, H, F32, check_dispatch(x, experts, used, E), T * k, seed=H)


@pytest.mark.parametrize("T,k", [(40, 2), (6000, 3)])
def test_routing_at_its_ends(T, k):
    """All tokens to one expert, to none, ids outside the experts, an expert named twice, counts of slots beyond both ends."""
    E, H = 6, 64
    x = torch.randn((T, H), generator=torch.Generator(device=DEV).manual_seed(3), device=DEV).to(BF16)
    ends = torch.tensor([-1, E, 2 ** 31 - 1, -2 ** 31, 0, E - 1, 2, 2], dtype=torch.int32)
    mixed = ends[torch.randint(0, 8, (T, k), generator=torch.Generator().manual_seed(4))]
    for experts in (torch.full((T, k), 3), torch.full((T, k), 0), torch.full((T, k), E - 1), torch.full((T, k), -1), torch.full((T, k), E), mixed):
        slot_of = check_dispatch(x, experts.to(torch.int32), None, E)
        check_sums(T, k, H, BF16, slot_of, T * k, seed=5)
    used = torch.tensor([-5, 0, 1, k, k + 1, 2 ** 31 - 1], dtype=torch.int32)[torch.arange(T) % 6]
    check_dispatch(x, mixed, used, E)
    rows, slot_of, offsets = pkg.moe_dispatch_rows(x, torch.full((T, k), -1, dtype=torch.int32, device=DEV), E)
    assert not bool(offsets.any()) and bool((slot_of == -1).all()) and not bool(pkg.moe_combine_rows(rows, slot_of).any())


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_slots_outside_the_rows_are_not_read(dtype):
    """Fewer rows than slots, or more: what lies outside them is no slot; nothing beyond the rows is touched."""
    T, k, H, R = 50, 3, 128, 60
    g = torch.Generator().manual_seed(6)
    slot_of = torch.full((T, k), -1, dtype=torch.int32)
    pick = torch.randperm(T * k, generator=g)
    slot_of.view(-1)[pick[:R // 2]] = torch.randperm(R, generator=g)[:R // 2].to(torch.int32)
    slot_of.view(-1)[pick[R // 2:]] = torch.tensor([-1, R, R + 5, 2 ** 31 - 1, -2 ** 31], dtype=torch.int32)[torch.arange(T * k - R // 2) % 5]
    for weighted in (True, False):
        check_sums(T, k, H, dtype, slot_of.to(DEV), R, seed=7, weighted=weighted)
    empty = torch.empty((0, H), dtype=dtype, device=DEV)
    assert not bool(pkg.moe_combine_rows(empty, slot_of.to(DEV)).any())
    dy, dw = pkg.moe_combine_rows_backward(torch.ones((T, H), dtype=dtype, device=DEV), empty, slot_of.to(DEV))
    assert dy.shape == (0, H) and not bool(dw.any())


def test_unused_slots_hold_anything():
    """What belongs to a slot that is not used, NaN and infinities among it, does not reach a result."""
    T, k, E, H = 90, 4, 8, 64
    experts, used = make_routing(T, k, E, seed=9, use=True)
    x = torch.randn((T, H), generator=torch.Generator(device=DEV).manual_seed(9), device=DEV).to(BF16)
    x[used.to(DEV) == 0] = float("nan")
    slot_of = check_dispatch(torch.nan_to_num(x), experts, used, E)
    rows, _, offsets = pkg.moe_dispatch_rows(x, experts.to(DEV), E, used=used.to(DEV))
    n = int(offsets[-1])
    assert bool(torch.isfinite(rows[:n]).all())
    y = rows.clone()
    y[n:] = float("inf")
    w = torch.where(slot_of >= 0, 0.5, float("nan"))
    out = pkg.moe_combine_rows(y, slot_of, w)
    dy, dw = pkg.moe_combine_rows_backward(torch.ones_like(out), y, slot_of, w)
    assert bool(torch.isfinite(out).all()) and bool(torch.isfinite(dy[:n]).all()) and bool(torch.isfinite(dw).all())


def test_gradients_against_differences():
    """All of it is linear in each argument: <gradient, d> = L(a + d) - L(a), up to the roundings of the sums (fp32), which are at most
    2^-24 of magnitudes as above, added up over H and T."""
    T, k, E, H = 37, 3, 8, 68
    g = torch.Generator(device=DEV).manual_seed(10)
    randn = lambda *s: torch.randn(s, generator=g, device=DEV)  # noqa: E731
    experts, used = make_routing(T, k, E, seed=11, use=True)
    x, d, w, dw, up = randn(T, H), randn(T, H), randn(T, k), randn(T, k), randn(T, H)

    def loss(x, w):
        rows, slot_of, _ = pkg.moe_dispatch_rows(x, experts.to(DEV), E, used=used.to(DEV), rows=torch.zeros((T * k, H), device=DEV))
        return pkg.moe_combine_rows(rows, slot_of, w), rows, slot_of

    out, rows, slot_of = loss(x, w)
    drows, dweights = pkg.moe_combine_rows_backward(up, rows, slot_of, w, dy=torch.zeros_like(rows))
    dx = pkg.moe_dispatch_rows_backward(drows, slot_of)
    for change, gradient, moved in ((d, dx, loss(x + d, w)[0]), (dw, dweights, loss(x, w + dw)[0])):
        there = up.double() * (moved.double() - out.double())
        scale = float((up.double().abs() * (moved.double().abs() + out.double().abs() + k)).sum())
        assert abs(float(there.sum()) - float((change.double() * gradient.double()).sum())) <= (k + 4) * 2.0 ** -23 * scale + H * 2.0 ** -24 * scale


def test_rows_beyond_32_bit_offsets():
    """More than 2^31 elements and 2^32 bytes among the rows."""
    T, k, E, H = 140000, 4, 4, 4096
    experts = (torch.arange(T, device=DEV)[:, None] + torch.arange(k, device=DEV)) % E
    x = (torch.arange(T, device=DEV) % 251).to(BF16)[:, None].expand(T, H).contiguous()
    rows, slot_of, offsets = pkg.moe_dispatch_rows(x, experts.to(torch.int32).contiguous(), E)
    assert offsets.tolist() == [0, T, 2 * T, 3 * T, 4 * T]
    assert torch.equal(slot_of, (experts * T + torch.arange(T, device=DEV)[:, None]).to(torch.int32))
    for e in range(E):
        assert torch.equal(rows[e * T:(e + 1) * T], x)
    out = pkg.moe_combine_rows(rows, slot_of, torch.full((T, k), 0.25, device=DEV))
    assert torch.equal(out, x)
    dy, dw = pkg.moe_combine_rows_backward(x, rows, slot_of, torch.full((T, k), 0.5, device=DEV), dy=rows)
    assert all(torch.equal(dy[e * T:(e + 1) * T], x / 2) for e in range(E))
    want = (x[:, 0].double() ** 2 * H)[:, None]
    assert bool(((dw.double() - want).abs() <= (512 + 9) * 2.0 ** -24 * want).all())


def test_no_tokens():
    for dtype in (F32, BF16):
        rows, slot_of, offsets = pkg.moe_dispatch_rows(torch.empty((0, 64), dtype=dtype, device=DEV), torch.empty((0, 2), dtype=torch.int32, device=DEV), 8)
        assert rows.shape == (0, 64) and slot_of.shape == (0, 2) and offsets.tolist() == [0] * 9
        assert pkg.moe_combine_rows(rows, slot_of).shape == (0, 64) and pkg.moe_dispatch_rows_backward(rows, slot_of).shape == (0, 64)
        dy, dw = pkg.moe_combine_rows_backward(rows, rows, slot_of)
        assert dy.shape == (0, 64) and dw.shape == (0, 2)


def test_refusals_on_the_gpu():
    x, ids = torch.zeros((4, 64), device=DEV), torch.zeros((4, 2), dtype=torch.int32, device=DEV)
    with pytest.raises(ValueError):
        pkg.moe_dispatch_rows(x[:, ::2], ids, 8)
    with pytest.raises(ValueError):
        pkg.moe_dispatch_rows(x, ids.cpu(), 8)
    with pytest.raises(TypeError):
        pkg.moe_dispatch_rows(x.half(), ids, 8)
    with pytest.raises(pkg.MoepError):
        pkg.moe_dispatch_rows(x, ids, 33)
    with pytest.raises(pkg.MoepError):
        pkg.moe_dispatch_rows(x[:, :6].contiguous(), ids, 8)
    with pytest.raises(ValueError):
        pkg.moe_combine_rows(x, ids, torch.zeros((2, 4), device=DEV))
    with pytest.raises(pkg.MoepError):
        pkg.moe_dispatch_rows(torch.zeros((9000, 64), device=DEV), torch.zeros((9000, 1), dtype=torch.int32, device=DEV), 8,
                              workspace=torch.zeros(8, dtype=torch.uint8, device=DEV))


def test_other_streams_and_repeats():
    T, k, E, H = 6001, 4, 16, 256
    experts, _ = make_routing(T, k, E, seed=20)
    experts = experts.to(DEV)
    x = torch.randn((T, H), generator=torch.Generator(device=DEV).manual_seed(20), device=DEV).to(BF16)
    w = torch.rand((T, k), device=DEV)

    def run():
        rows, slot_of, offsets = pkg.moe_dispatch_rows(x, experts, E)
        return rows, slot_of, offsets, pkg.moe_combine_rows(rows, slot_of, w), *pkg.moe_combine_rows_backward(x, rows, slot_of, w)

    a = run()
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    outs = []
    for s in streams:                                        # two calls in flight at once
        with torch.cuda.stream(s):
            outs.append(run())
    torch.cuda.synchronize()
    assert all(torch.equal(p, q) for out in outs for p, q in zip(a, out))


@pytest.mark.parametrize("T", [200, 5000])
def test_rows_in_a_graph(T):
    k, E, H = 3, 8, 128
    x = torch.zeros((T, H), dtype=BF16, device=DEV)
    experts = torch.zeros((T, k), dtype=torch.int32, device=DEV)
    used = torch.full((T,), k, dtype=torch.int32, device=DEV)
    w = torch.rand((T, k), device=DEV)
    keep = [torch.zeros((T * k, H), dtype=BF16, device=DEV) for _ in range(4)]

    def run(rows, dy):
        rows, slot_of, offsets = pkg.moe_dispatch_rows(x, experts, E, used=used, rows=rows)
        out = pkg.moe_combine_rows(rows, slot_of, w)
        dy, dw = pkg.moe_combine_rows_backward(out, rows, slot_of, w, dy=dy)
        return slot_of, offsets, out, dw, pkg.moe_dispatch_rows_backward(dy, slot_of)

    run(*keep[:2])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = run(*keep[2:])
    for seed in range(3):
        ids, n = make_routing(T, k, E, seed=seed, use=True)
        experts.copy_(ids)
        used.copy_(n)
        x.copy_(torch.randn((T, H), generator=torch.Generator(device=DEV).manual_seed(seed), device=DEV))
        want = run(*keep[:2])
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(out, want))
