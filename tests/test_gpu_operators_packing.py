"""Grouped products of operands whose rows do not lie at multiples of 16 bytes: what is copied, and what is not."""
import numpy as np
import pytest
import torch

from paper_1903_12287_amd import operators as ops
from paper_1903_12287_amd import pbg
from tests.operators_cases import SENTINEL, TYPES, context
from tests.test_gpu_operators_group import run_case

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    c = context()
    yield c
    pbg.pbg_free(c)


def test_matrices_of_empty_groups_take_no_memory():
    """24 rows in 1,000 groups of 501 x 333 float16 (334 MB of matrices): copies of at most 24 of them."""
    groups, n, k, m = 1_000, 24, 501, 333
    dt = torch.float16
    a = torch.full((groups, m, k), float("nan"), dtype=dt, device="cuda")
    at = np.sort(np.random.default_rng(0).choice(groups, n, replace=False))
    offsets = torch.from_numpy(np.searchsorted(at, np.arange(groups + 1)).astype(np.int64)).cuda()
    mine = torch.from_numpy(at).cuda()
    g = torch.Generator(device="cuda").manual_seed(0)
    a[mine] = torch.randint(-2, 3, (n, m, k), generator=g, device="cuda").to(dt)
    x = torch.randint(-2, 3, (n, k), generator=g, device="cuda").to(dt)
    dy = torch.randint(-1, 2, (n, m), generator=g, device="cuda").to(dt)
    y, dx = torch.empty_like(dy), torch.empty_like(x)
    # whole numbers below 2^11: exact in float16
    want_y, want_dx = torch.empty_like(y), torch.empty_like(dx)
    for i in range(n):
        want_y[i] = (a[at[i]].double() @ x[i].double()).to(dt)
        want_dx[i] = (a[at[i]].double().t().contiguous() @ dy[i].double()).to(dt)
    assert float(want_y.abs().max()) < 2_048 and float(want_dx.abs().max()) < 2_048
    c = context()
    try:
        torch.cuda.synchronize()
        before = torch.cuda.mem_get_info()[0]
        ops.pbg_group_linear(c, x, a, offsets, y)
        ops.pbg_group_linear_backward(c, None, a, offsets, dy, dx, None)
        torch.cuda.synchronize()
        taken = before - torch.cuda.mem_get_info()[0]
    finally:
        pbg.pbg_free(c)
    # 24 matrices of 333 rows of 1,008 bytes are 8 MB; allocations are rounded up to a few MB
    assert taken <= 64 << 20, taken
    assert torch.equal(y, want_y) and torch.equal(dx, want_dx)


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("k,m", [(37, 21), (13, 200), (301, 5)])
@pytest.mark.parametrize("sizes,first", [
    ([0, 1, 0, 0, 0, 2, 0, 0], 0),                       # fewer rows than groups
    ([0, 1, 0, 0, 0, 2, 0, 0], 3),                       # rows of no group in front: places start behind them
    ([0] * 30 + [1, 0, 1] + [0] * 20 + [4], 0),          # up to 63 groups, one empty one after the other
    ([0] * 100 + [1, 0, 1, 3] + [0] * 97 + [7, 0], 2),   # more groups than a wave has lanes
    ([1] * 70, 0), ([1] * 64 + [0], 0), ([2] * 40, 1),   # as many rows as groups, one fewer, more
    ([0, 90, 0, 0, 33], 5)])
def test_places_of_matrices(ctx, t, sizes, first, k, m):
    run_case(ctx, TYPES[t], sizes, k, m, first=first, tail=4, seed=len(sizes))


@pytest.mark.parametrize("t", TYPES)
def test_many_empty_groups(ctx, t):
    """Groups by the thousand with an odd width, a few of them with rows, the last one too."""
    sizes = np.zeros(5_000, dtype=np.int64)
    sizes[[0, 63, 64, 65, 1_000, 4_095, 4_096, 4_999]] = (3, 1, 1, 2, 40, 1, 5, 9)
    run_case(ctx, TYPES[t], sizes, 11, 7)


@pytest.mark.parametrize("groups,n", [(5, 3), (5, 40), (200, 30), (200, 900)])
def test_bad_offsets_ahead_of_the_copies(ctx, groups, n):
    """The copies run before the offsets have been checked; nothing but the workspace is written."""
    k, m = 9, 7
    x, dy = torch.ones(n, k, device="cuda"), torch.ones(n, m, device="cuda")
    a = torch.ones(groups, m, k, device="cuda")
    y, dx, da = torch.full_like(dy, SENTINEL), torch.full_like(x, SENTINEL), torch.full_like(a, SENTINEL)
    good = np.linspace(0, n, groups + 1).astype(np.int64)
    for at, value in ((0, -1), (0, 2 ** 63 - 1), (groups, 2 ** 63 - 1), (groups, -(2 ** 63)), (groups // 2, n + 7),
                      (groups - 1, -(2 ** 40)), (groups, 0), (1, n)):
        bad = good.copy()
        bad[at] = value
        if sorted(bad) == list(bad) and bad[0] >= 0 and bad[-1] <= n:
            continue
        bad = torch.from_numpy(bad).cuda()
        with pytest.raises(pbg.PbgError, match="offsets"):
            ops.pbg_group_linear(ctx, x, a, bad, y)
        with pytest.raises(pbg.PbgError, match="offsets"):
            ops.pbg_group_linear_backward(ctx, x, a, bad, dy, dx, da)
    for o in (y, dx, da):
        assert bool((o == SENTINEL).all())
    ops.pbg_group_linear(ctx, x, a, torch.from_numpy(good).cuda(), y)
    assert bool((y == k).all())
