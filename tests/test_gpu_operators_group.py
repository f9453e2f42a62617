"""Products with one matrix per group of rows, and their gradients, against float64."""
import ctypes

import numpy as np
import pytest
import torch

from paper_1903_12287_amd import operators as ops
from paper_1903_12287_amd import pbg
from tests.operators_cases import (SENTINEL, TYPES, Guarded, context, group_products, offsets_of, product_tolerance,
                                   ragged_sizes, rows)

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    c = context()
    yield c
    pbg.pbg_free(c)


def check(name, got, exact, size, depth, inside=None):
    got = got.double().cpu()
    tol = product_tolerance(exact, size, depth, got_type(name))
    off = (got - exact).abs() - tol
    if inside is not None:
        off = off[inside]
    assert off.numel() == 0 or float(off.max()) <= 0.0, f"{name[0]}: {float(off.max()):.3g} beyond the tolerance"


def got_type(name):
    return name[1]


def run_case(ctx, dtype, sizes, k, m, first=0, tail=0, pads=(0, 0, 0, 0), fronts=(0, 0, 0, 0), seed=0, scale=1.0):
    rng = np.random.default_rng(seed)
    off = offsets_of(sizes, first)
    G, n = len(sizes), int(off[-1]) + tail
    x = rows(rng, n, k, dtype, pads[0], fronts[0], scale)
    dy = rows(rng, n, m, dtype, pads[1], fronts[1])
    a = rows(rng, G * m, k, dtype, 0, fronts[2], k ** -0.5).view(G, m, k)
    offsets = torch.from_numpy(off).cuda()
    y = Guarded(n, m, dtype, pads[2], fronts[0])
    dx = Guarded(n, k, dtype, pads[3], fronts[1])
    da = Guarded(G * m, k, dtype, 0, fronts[3])
    ops.pbg_group_linear(ctx, x, a, offsets, y.view)
    ops.pbg_group_linear_backward(ctx, x, a, offsets, dy, dx.view, da.view.view(G, m, k))
    exact, size = group_products(x, a, dy, off)
    inside = slice(int(off[0]), int(off[-1]))
    check(("y", dtype), y.view, exact["y"], size["y"], k, inside)
    check(("dx", dtype), dx.view, exact["dx"], size["dx"], m, inside)
    longest = int(max(sizes)) if len(sizes) else 0
    check(("da", dtype), da.view.view(G, m, k), exact["da"], size["da"], longest)
    for o in (y, dx, da):
        assert o.outside_untouched()
    for o in (y, dx):   # rows of no group
        assert bool((o.view[:int(off[0])] == SENTINEL).all()) and bool((o.view[int(off[-1]):] == SENTINEL).all())
    # each gradient alone, and a second time: the same bits
    dx2, da2 = Guarded(n, k, dtype, pads[3]), Guarded(G * m, k, dtype)
    ops.pbg_group_linear_backward(ctx, None, a, offsets, dy, dx2.view, None)
    ops.pbg_group_linear_backward(ctx, x, None, offsets, dy, None, da2.view.view(G, m, k))
    assert torch.equal(dx2.view, dx.view) and torch.equal(da2.view, da.view)


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("sizes,k,m", [
    ([1], 1, 1), ([1], 8, 8), ([3, 0, 2], 5, 7), ([1, 1, 1, 1], 64, 32), ([0, 0, 9, 0], 33, 65), ([17, 40], 100, 100),
    ([64, 128, 1], 128, 128), ([129, 127, 0, 256, 255], 96, 72), ([300], 401, 257), ([31, 33, 2, 70], 264, 136),
    ([1000], 48, 24), ([513, 600], 256, 512)])
def test_sizes(ctx, t, sizes, k, m):
    run_case(ctx, TYPES[t], sizes, k, m, seed=k)


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("groups,n,k,m", [(7, 900, 64, 80), (70, 500, 40, 48), (200, 3001, 24, 16), (4099, 2000, 8, 8),
                                          (5, 2600, 136, 200), (64, 64, 512, 256), (300, 40, 72, 128)])
def test_many_ragged_groups(ctx, t, groups, n, k, m):
    run_case(ctx, TYPES[t], ragged_sizes(np.random.default_rng(n), groups, n), k, m, seed=groups)


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("k,m,pads,fronts", [
    (64, 64, (8, 8, 8, 8), (0, 0, 0, 0)),      # rows apart, all at 16 bytes
    (64, 64, (1, 3, 5, 7), (0, 0, 0, 0)),      # rows at odd places
    (64, 64, (0, 0, 0, 0), (1, 1, 1, 1)),      # everything one element off
    (66, 62, (2, 2, 2, 2), (2, 0, 4, 2)),      # rows at multiples of four bytes
    (61, 67, (3, 5, 1, 3), (1, 3, 5, 1)),
    (200, 8, (0, 56, 0, 0), (4, 4, 4, 4))])
def test_strides_and_alignments(ctx, t, k, m, pads, fronts):
    run_case(ctx, TYPES[t], [37, 0, 150, 1, 90], k, m, first=5, tail=11, pads=pads, fronts=fronts, seed=m)


@pytest.mark.parametrize("t", TYPES)
def test_few_rows_in_many_groups(ctx, t):
    """Single tokens: most groups without a row, the others with one or a few."""
    sizes = np.zeros(48, dtype=np.int64)
    sizes[[3, 17, 18, 40, 47]] = (1, 2, 1, 16, 5)
    run_case(ctx, TYPES[t], sizes, 320, 192)
    run_case(ctx, TYPES[t], sizes, 72, 1000, seed=4)


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("sizes,k,m", [([2501, 0, 3100, 2700], 72, 2048), ([2501, 0, 3100, 2700], 2043, 61),
                                       ([300, 513, 0, 290], 2048, 2048), ([257, 255, 900, 3], 1999, 2053)])
def test_wide_products(ctx, t, sizes, k, m):
    """Enough rows and columns for the largest tiles, forward, dx and da."""
    run_case(ctx, TYPES[t], sizes, k, m, seed=1)


@pytest.mark.parametrize("t,small,large", [("f16", -20, 8), ("f16", -16, 8), ("bf16", -130, 20), ("f32", -140, 30)])
def test_values_below_the_normal_range(ctx, t, small, large):
    """One factor of a product below its type's normal range, the other large: the product keeps every bit."""
    dt, n, k, m = TYPES[t], 40, 64, 48
    rng = np.random.default_rng(0)
    x, a = rows(rng, n, k, dt, scale=2.0 ** small), rows(rng, m, k, dt, scale=2.0 ** large).view(1, m, k)
    dy = rows(rng, n, m, dt, scale=2.0 ** large)
    off = torch.tensor([0, n], dtype=torch.int64, device="cuda")
    y, da = torch.empty(n, m, dtype=dt, device="cuda"), torch.empty(1, m, k, dtype=dt, device="cuda")
    ops.pbg_group_linear(ctx, x, a, off, y)
    ops.pbg_group_linear_backward(ctx, x, None, off, dy, None, da)
    exact, size = group_products(x, a, dy, [0, n])
    check(("y", dt), y, exact["y"], size["y"], k)
    check(("da", dt), da, exact["da"], size["da"], n)


@pytest.mark.parametrize("t", TYPES)
def test_no_rows(ctx, t):
    dt = TYPES[t]
    a = torch.ones(3, 4, 5, dtype=dt, device="cuda")
    da = torch.full((3, 4, 5), SENTINEL, dtype=dt, device="cuda")
    off = torch.zeros(4, dtype=torch.int64, device="cuda")
    x, y = torch.empty(0, 5, dtype=dt, device="cuda"), torch.empty(0, 4, dtype=dt, device="cuda")
    ops.pbg_group_linear(ctx, x, a, off, y)
    ops.pbg_group_linear_backward(ctx, x, a, off, y, torch.empty_like(x), da)
    assert bool((da == 0).all())


def test_values_that_are_not_finite_stay_in_their_rows(ctx):
    """An infinity or NaN reaches its own row of y and dx and its group's da, and nothing else: not the rows of
    neighbouring tiles or groups, nor through the zeros that fill a tile."""
    for t, k, m in (("f32", 36, 20), ("bf16", 40, 24), ("f16", 37, 21)):
        dt = TYPES[t]
        rng = np.random.default_rng(3)
        sizes = [20, 13, 0, 70]
        off = offsets_of(sizes)
        x, dy = rows(rng, 103, k, dt), rows(rng, 103, m, dt)
        a = rows(rng, 4 * m, k, dt).view(4, m, k)
        x[25, 3], x[26, k - 1], dy[25, 1] = float("inf"), float("nan"), float("-inf")
        y, dx = Guarded(103, m, dt), Guarded(103, k, dt)
        da = Guarded(4 * m, k, dt)
        offsets = torch.from_numpy(off).cuda()
        ops.pbg_group_linear(ctx, x, a, offsets, y.view)
        ops.pbg_group_linear_backward(ctx, x, a, offsets, dy, dx.view, da.view.view(4, m, k))
        fine = torch.isfinite(y.view).all(1).cpu()
        assert not fine[25] and not fine[26] and int((~fine).sum()) == 2
        fine = torch.isfinite(dx.view).all(1).cpu()
        assert not fine[25] and int((~fine).sum()) == 1
        fine = torch.isfinite(da.view.view(4, m, k)).flatten(1).all(1).cpu()
        assert fine.tolist() == [True, False, True, True]


def test_rows_past_four_gib(ctx):
    """Offsets of rows beyond 2^32 bytes, in x, y and the gradients."""
    n, k, m = 70_001, 16, 24
    ld = 33_000                                   # 70,001 rows of 66,000 bytes: 4.6 GB
    rng = np.random.default_rng(0)
    dt = torch.bfloat16
    big = torch.zeros(n, ld, dtype=dt, device="cuda")
    x, y, dx = big[:, :k], big[:, 64:64 + m], big[:, 128:128 + k]
    x.copy_(torch.from_numpy(rng.standard_normal((n, k))).to(dt))
    dy = big[:, 192:192 + m]
    dy.copy_(torch.from_numpy(rng.standard_normal((n, m))).to(dt))
    sizes = [35_000, 1, 34_000, 1_000]
    off = offsets_of(sizes)
    a = rows(rng, 4 * m, k, dt, scale=0.25).view(4, m, k)
    da = torch.empty(4, m, k, dtype=dt, device="cuda")
    offsets = torch.from_numpy(off).cuda()
    ops.pbg_group_linear(ctx, x, a, offsets, y)
    ops.pbg_group_linear_backward(ctx, x, a, offsets, dy, dx, da)
    exact, size = group_products(x, a, dy, off)
    check(("y", dt), y, exact["y"], size["y"], k)
    check(("dx", dt), dx, exact["dx"], size["dx"], m)
    check(("da", dt), da, exact["da"], size["da"], 35_000)
    rest = torch.ones(ld, dtype=torch.bool, device="cuda")
    for lo, w in ((0, k), (64, m), (128, k), (192, m)):
        rest[lo:lo + w] = False
    assert all(float(big[i:i + 10_000][:, rest].abs().max()) == 0.0 for i in range(0, n, 10_000))


def test_gradients_against_differences(ctx):
    """<dy, y(x + e u) - y(x - e u)> / 2e is <dx, u>, and the same for a: y is linear in both, so the differences are
    exact but for the roundings of their sums."""
    rng = np.random.default_rng(7)
    sizes, k, m = [10, 0, 25, 60], 30, 18
    off = torch.from_numpy(offsets_of(sizes)).cuda()
    dt = torch.float32
    x, dy, a = rows(rng, 95, k, dt), rows(rng, 95, m, dt), rows(rng, 4 * m, k, dt).view(4, m, k)
    dx, da = torch.empty_like(x), torch.empty(4, m, k, device="cuda")
    ops.pbg_group_linear_backward(ctx, x, a, off, dy, dx, da)

    def value(x, a):
        y = torch.empty(95, m, device="cuda")
        ops.pbg_group_linear(ctx, x.contiguous(), a.contiguous(), off, y)
        return (y.double() * dy.double()).sum()

    for u, grad, at in ((torch.randn_like(x), dx, 0), (torch.randn_like(da), da, 1)):
        plus, minus = ([x + u, a] if at == 0 else [x, a + u]), ([x - u, a] if at == 0 else [x, a - u])
        diff = (value(*plus) - value(*minus)) / 2
        want = (grad.double() * u.double()).sum()
        # float32 roundings of x + u (one each), of y's 30-term sums and of dx's and da's sums, at most 100 half
        # steps each of terms whose absolute sum is below this
        size = float(dy.abs().sum()) * float((x.abs().max() + u.abs().max()) * (a.abs().max() + 1) * k)
        assert abs(float(diff - want)) <= 100 * 2.0 ** -24 * size


def test_layouts_of_the_framework(ctx):
    """A relation-grouped bucket: pbg_group_by_relation's order and its run bounds feed the grouped product, whose
    rows are the linear operator's: their products with the destinations are pbg_score_edges' scores."""
    n, R, d, E = 50, 6, 24, 400
    rng = np.random.default_rng(1)
    c = pbg.pbg_bucket_init(n, 1, R, d, "linear", "dot", "ranking")
    try:
        emb = torch.from_numpy(rng.standard_normal((n, d)).astype(np.float32)).cuda()
        A = torch.from_numpy(rng.standard_normal((R, d, d)).astype(np.float32)).cuda()
        pbg.pbg_bind_partition(c, 0, emb, torch.zeros(n, device="cuda"))
        pbg.pbg_bind_relations(c, A, torch.zeros_like(A))
        src, rel, dst = (torch.from_numpy(rng.integers(0, z, E).astype(np.int32)).cuda() for z in (n, R, n))
        s2, r2, d2 = torch.empty_like(src), torch.empty_like(rel), torch.empty_like(dst)
        pbg.pbg_group_by_relation(c, src, rel, dst, s2, r2, d2)
        off = torch.searchsorted(r2, torch.arange(R + 1, dtype=torch.int32, device="cuda"))
        q = torch.empty(E, d, device="cuda")
        ops.pbg_group_linear(c, emb[s2.long()], A, off, q)
        scores = torch.empty(E, device="cuda")
        pbg.pbg_score_edges(c, 0, 0, s2, r2, d2, scores)
        x, y = emb[s2.long()].double(), emb[d2.long()].double()
        size = (torch.einsum("ei,eji->ej", x.abs().cpu(), A.double().abs().cpu()[r2.cpu().long()]) * y.abs().cpu()).sum(1)
        off_by = ((q.double() * y).sum(1) - scores.double()).abs().cpu()
        # two float32 evaluations of a sum of d * d products: 2 d roundings on either side
        assert bool((off_by <= 4 * d * 2.0 ** -24 * size).all())
    finally:
        pbg.pbg_free(c)


def test_refusals(ctx):
    dt = torch.float32
    x, y = torch.zeros(10, 4, device="cuda"), torch.full((10, 6), SENTINEL, device="cuda")
    a = torch.ones(2, 6, 4, device="cuda")

    def off(*v):
        return torch.tensor(v, dtype=torch.int64, device="cuda")

    good = off(0, 4, 10)
    for bad in (off(0, 5, 4), off(-1, 4, 10), off(0, 4, 11), off(11, 11, 11), off(0, 2 ** 40, 10)):
        with pytest.raises(pbg.PbgError, match="offsets"):
            ops.pbg_group_linear(ctx, x, a, bad, y)
        assert bool((y == SENTINEL).all())
        dx, da = torch.full_like(x, SENTINEL), torch.full_like(a, SENTINEL)
        with pytest.raises(pbg.PbgError, match="offsets"):
            ops.pbg_group_linear_backward(ctx, x, a, bad, y, dx, da)
        assert bool((dx == SENTINEL).all()) and bool((da == SENTINEL).all())
        ops.pbg_group_linear(ctx, x, a, good, y)   # the next call is not held to it
        assert bool((y == 0).all())
        y.fill_(SENTINEL)
    both = torch.zeros(10, 12, device="cuda")
    with pytest.raises(pbg.PbgError, match="overlap"):
        ops.pbg_group_linear(ctx, both[:, :4], a, good, both[:, 3:9])
    ops.pbg_group_linear(ctx, both[:, :4], a, good, both[:, 4:10])   # columns of their own
    with pytest.raises(pbg.PbgError, match="overlap"):
        ops.pbg_group_linear_backward(ctx, x, a, good, y, None, a)
    with pytest.raises(pbg.PbgError, match="stride"):
        ops.pbg_group_linear(ctx, x[:1].expand(10, 4), a, good, y)
    with pytest.raises(ValueError):
        ops.pbg_group_linear(ctx, x, a, off(0, 10), y)
    with pytest.raises(ValueError):
        ops.pbg_group_linear(ctx, x.t(), a, good, y)
    with pytest.raises(TypeError):
        ops.pbg_group_linear(ctx, x.double(), a.double(), good, y)
    with pytest.raises(TypeError):
        ops.pbg_group_linear(ctx, x.to(torch.bfloat16), a, good, y)
    with pytest.raises(ValueError):
        ops.pbg_group_linear(ctx, x, a.transpose(1, 2), good, y)
    with pytest.raises(ValueError):
        ops.pbg_group_linear_backward(ctx, None, a, good, y, None, torch.empty_like(a))
    lib = ops.library()
    p = [v.data_ptr() for v in (x, a, good, y)]
    for args in ((3, p[0], 4, p[1], p[2], 2, 10, 4, 6, p[3], 6), (0, p[0], 3, p[1], p[2], 2, 10, 4, 6, p[3], 6),
                 (0, p[0], 4, p[1], p[2], 0, 10, 4, 6, p[3], 6), (0, p[0], 4, p[1], p[2], 2, -1, 4, 6, p[3], 6),
                 (0, p[0], 4, p[1], p[2], 2, 10, 0, 6, p[3], 6), (0, p[0], 4, p[1], p[2], 2, 10, 4, 70_000, p[3], 70_000),
                 (0, None, 4, p[1], p[2], 2, 10, 4, 6, p[3], 6), (0, p[0], 4, p[1], None, 2, 10, 4, 6, p[3], 6),
                 (0, p[0] + 2, 4, p[1], p[2], 2, 10, 4, 6, p[3], 6), (0, p[0], 1 << 21, p[1], p[2], 2, 10, 4, 6, p[3], 6)):
        assert lib.pbg_group_linear(ctx, *args) == 1, args
    assert bool((y == SENTINEL).all())


def test_neither_gradient_and_pending_errors(ctx):
    x, a = torch.ones(4, 4, device="cuda"), torch.ones(1, 4, 4, device="cuda")
    y = torch.full((4, 4), SENTINEL, device="cuda")
    off = torch.tensor([0, 4], dtype=torch.int64, device="cuda")
    ops.pbg_group_linear_backward(ctx, x, a, off, y, None, None)
    bad = torch.tensor([0, 5], dtype=torch.int64, device="cuda")
    ops.pbg_group_linear_backward(ctx, x, a, bad, y, None, None)   # nothing to write, nothing looked at
    lib = ctypes.CDLL(pbg.LIB_PATH)   # and the HIP runtime it is linked against
    assert lib.hipSetDevice(9999) != 0
    with pytest.raises(pbg.PbgError, match="pending"):
        ops.pbg_group_linear(ctx, x, a, off, y)
    assert bool((y == SENTINEL).all())
    ops.pbg_group_linear(ctx, x, a, off, y)
    assert bool((y == 4).all())


def test_a_capturing_stream_is_refused_and_its_capture_goes_on(ctx):
    c = context()
    s = torch.cuda.Stream()
    pbg.pbg_set_streams(c, s, None)
    x, a = torch.ones(4, 4, device="cuda"), torch.ones(1, 4, 4, device="cuda")
    off = torch.tensor([0, 4], dtype=torch.int64, device="cuda")
    y, z = torch.zeros(4, 4, device="cuda"), torch.zeros(4, device="cuda")
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        z.add_(1.0)
        with pytest.raises(pbg.PbgError, match="graph"):
            ops.pbg_group_linear(c, x, a, off, y)
    for i in range(3):
        g.replay()
        torch.cuda.synchronize()
        assert bool((z == i + 1).all())
        ops.pbg_group_linear(c, x, a, off, y)
        assert bool((y == 4).all())
    pbg.pbg_free(c)


def test_a_stream_of_the_callers(ctx):
    """Inputs made on the stream that the context works on, with the null stream busy elsewhere."""
    c = context()
    s = torch.cuda.Stream()
    pbg.pbg_set_streams(c, s, None)
    off = torch.tensor([0, 3000], dtype=torch.int64, device="cuda")
    a = torch.eye(64, device="cuda")[None].contiguous()
    y = torch.zeros(3000, 64, device="cuda")
    torch.cuda.synchronize()
    for i in range(5):
        with torch.cuda.stream(s):
            x = torch.full((3000, 64), float(i), device="cuda")
            for _ in range(20):
                x = x + 1.0
            ops.pbg_group_linear(c, x, a, off, y)
        assert bool((y == i + 20.0).all())
    pbg.pbg_free(c)
