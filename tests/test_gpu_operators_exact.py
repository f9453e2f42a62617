"""Grouped products of small whole numbers, whose sums are exact in float32 in any order: not a row may be lost or taken
twice, wherever rows and matrices lie."""
import numpy as np
import pytest
import torch

from paper_1903_12287_amd import operators as ops
from paper_1903_12287_amd import pbg
from tests.operators_cases import TYPES, context

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    c = context()
    yield c
    pbg.pbg_free(c)


def whole(seed, *shape, dtype, ld=0):
    """-2 .. 2; ld: a matrix whose rows lie so many values apart."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    v = torch.randint(-2, 3, shape, generator=g, device="cuda", dtype=torch.int8).to(dtype)
    if ld:
        wide = torch.empty(shape[0], ld, dtype=dtype, device="cuda")[:, :shape[1]]
        wide.copy_(v)
        return wide
    return v


def sums(dy, x):
    """dy^T x by blocks of rows in float64: a float32 product's own partial sums stay out of it."""
    out = torch.zeros(dy.shape[1], x.shape[1], dtype=torch.float64, device="cuda")
    for i in range(0, dy.shape[0], 1 << 15):
        out += dy[i:i + (1 << 15)].double().t().contiguous() @ x[i:i + (1 << 15)].double()
    return out


# |sums| and the sums of their parts: 2^20 products of variance 4 at most, 2^11 a standard deviation, far below 2^24
@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("sizes,k,m", [([300_001], 24, 40), ([200_000, 1, 0, 99_999, 513], 16, 24), ([400_003, 3], 7, 9),
                                       ([70_000, 130_000, 5], 128, 136), ([1_000_000, 0], 8, 8)])
def test_long_groups(ctx, t, sizes, k, m):
    dt, n = TYPES[t], sum(sizes)
    x, dy = whole(0, n, k, dtype=dt), whole(1, n, m, dtype=dt)
    bounds = np.concatenate([[0], np.cumsum(sizes)]).astype(np.int64)
    da = torch.full((len(sizes), m, k), 9.0, dtype=dt, device="cuda")
    ops.pbg_group_linear_backward(ctx, x, None, torch.from_numpy(bounds).cuda(), dy, None, da)
    for g in range(len(sizes)):
        r = slice(int(bounds[g]), int(bounds[g + 1]))
        exact = sums(dy[r], x[r])
        assert float(exact.abs().max()) < 2 ** 16
        assert torch.equal(da[g], exact.float().to(dt)), g


@pytest.mark.parametrize("t,ld", [("f32", 17_000), ("bf16", 33_000), ("f16", 33_003)])
def test_gradients_of_rows_past_four_gib(ctx, t, ld):
    """70,001 rows of 66,000 bytes and more in x, dy and dx (the last stride: not whole 16 bytes)."""
    dt, n, k, m = TYPES[t], 70_001, 16, 24
    x, dy, dx = whole(2, n, k, dtype=dt, ld=ld), whole(3, n, m, dtype=dt, ld=ld), whole(4, n, k, dtype=dt, ld=ld)
    a = whole(5, 4, m, k, dtype=dt)
    bounds = (0, 35_000, 35_001, 69_001, n)
    da = torch.full((4, m, k), 9.0, dtype=dt, device="cuda")
    ops.pbg_group_linear_backward(ctx, x, a, torch.tensor(bounds, device="cuda"), dy, dx, da)
    for g in range(4):
        r = slice(bounds[g], bounds[g + 1])
        assert torch.equal(da[g], sums(dy[r], x[r]).float().to(dt)), g
        assert torch.equal(dx[r], (dy[r].double() @ a[g].double()).float().to(dt)), g


@pytest.mark.parametrize("t,groups,k", [("f32", 300, 2_048), ("bf16", 560, 2_048), ("f16", 560, 2_045)])
def test_matrices_past_four_gib(ctx, t, groups, k):
    """a and da of more than 2^32 bytes (k = 2,045: the copies of a as well)."""
    dt, m = TYPES[t], 2_048
    rows = np.ones(groups, dtype=np.int64)
    rows[[0, 7, groups - 2]] = (3, 40, 0)
    bounds = np.concatenate([[0], np.cumsum(rows)]).astype(np.int64)
    n = int(bounds[-1])
    assert n >= groups and groups * m * k * torch.finfo(dt).bits // 8 > 2 ** 32
    x, dy, a = whole(6, n, k, dtype=dt), whole(7, n, m, dtype=dt), whole(8, groups, m, k, dtype=dt)
    y, dx, da = torch.empty_like(dy), torch.empty_like(x), torch.full_like(a, 9.0)
    off = torch.from_numpy(bounds).cuda()
    ops.pbg_group_linear(ctx, x, a, off, y)
    ops.pbg_group_linear_backward(ctx, x, a, off, dy, dx, da)
    for g in range(groups):
        r = slice(int(bounds[g]), int(bounds[g + 1]))
        ag = a[g].double()
        assert torch.equal(y[r], (x[r].double() @ ag.t().contiguous()).float().to(dt)), g
        assert torch.equal(dx[r], (dy[r].double() @ ag).float().to(dt)), g
        assert torch.equal(da[g], (dy[r].double().t().contiguous() @ x[r].double()).float().to(dt)), g
