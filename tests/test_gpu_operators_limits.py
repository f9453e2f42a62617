"""The operators where ranges are largest, where their checks change place, and in two contexts at once."""
import threading

import numpy as np
import pytest
import torch

from paper_1903_12287_amd import operators as ops
from paper_1903_12287_amd import pbg
from tests.operators_cases import context

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    c = context()
    yield c
    pbg.pbg_free(c)


def offsets(*v):
    return torch.tensor(v, dtype=torch.int64, device="cuda")


def small_integers(seed, *shape, dtype=torch.float32):
    """-2 .. 2: products and their sums are exact in every type they are summed in here."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randint(-2, 3, shape, generator=g, device="cuda", dtype=torch.int8).to(dtype)


# offsets of few groups are checked by the products of a small call, by a kernel of their own otherwise
@pytest.mark.parametrize("groups,n,k,m", [(3, 60, 8, 8), (63, 300, 16, 24), (64, 300, 16, 24), (200, 300, 16, 24),
                                          (3, 70000, 8, 256)])
@pytest.mark.parametrize("t", [torch.float32, torch.bfloat16])
def test_bad_offsets_wherever_they_are_checked(ctx, groups, n, k, m, t):
    x, dy, a = small_integers(0, n, k, dtype=t), small_integers(1, n, m, dtype=t), small_integers(2, groups, m, k, dtype=t)
    good = np.linspace(0, n, groups + 1).astype(np.int64)
    for at, value in ((0, -1), (groups, n + 1), (groups // 2, n + 7), (groups - 1, -(2 ** 40)), (groups, 0)):
        bad = good.copy()
        bad[at] = value
        bad = torch.from_numpy(bad).cuda()
        y, dx, da = torch.full_like(dy, 9), torch.full_like(x, 9), torch.full_like(a, 9)
        for call in (lambda: ops.pbg_group_linear(ctx, x, a, bad, y),
                     lambda: ops.pbg_group_linear_backward(ctx, x, a, bad, dy, dx, da),
                     lambda: ops.pbg_group_linear_backward(ctx, x, None, bad, dy, None, da),
                     lambda: ops.pbg_group_linear_backward(ctx, None, a, bad, dy, dx, None)):
            with pytest.raises(pbg.PbgError, match="offsets"):
                call()
        for o in (y, dx, da):
            assert bool((o == 9).all())
        ops.pbg_group_linear(ctx, x, a, torch.from_numpy(good).cuda(), y)   # and the next call is answered
        for g in (0, groups - 1):
            s = slice(int(good[g]), int(good[g + 1]))
            assert torch.equal(y[s].double(), (x[s].double() @ a[g].double().t()).to(t).double())


@pytest.mark.parametrize("n", [512, 513, 40])
def test_bad_labels_and_offsets_of_a_gradient(ctx, n):
    V = 24
    z = torch.randn(n, V, device="cuda")
    labels = torch.zeros(n, dtype=torch.int32, device="cuda")
    stats, dlogp = torch.zeros(n, 2, device="cuda"), torch.ones(2, device="cuda")
    for bad_off, bad_label, match in (((0, 5, n + 1), None, "offsets"), ((0, 9, 5), None, "offsets"),
                                      ((-1, 5, n), None, "offsets"), ((0, 5, n), n - 1, "label"),
                                      ((0, 5, n), 0, "label")):
        lab = labels.clone()
        if bad_label is not None:
            lab[bad_label] = V
        dz = torch.full_like(z, 9.0)
        with pytest.raises(pbg.PbgError, match=match):
            ops.pbg_preference_loss_backward(ctx, z, lab, offsets(*bad_off), stats, dlogp, dz)
        assert bool((dz == 9.0).all())
    lab = labels.clone()
    lab[n - 1] = V + 3   # behind the last sequence: not looked at
    ops.pbg_preference_loss_backward(ctx, z, lab, offsets(0, 5, n - 1), stats, dlogp, dz)
    assert bool((dz[n - 1] == 9.0).all()) and bool(torch.isfinite(dz[:n - 1]).all())


def test_more_tiles_than_a_launch_takes(ctx):
    """2^27 rows of four values: five million slots of 32."""
    n, k, m = (1 << 27) + 5, 4, 4
    x, dy, a = small_integers(3, n, k), small_integers(4, n, m), small_integers(5, 3, m, k)
    bounds = (1, 1000, (1 << 26) + 77, n - 2)
    off = offsets(*bounds)
    y, dx, da = torch.full_like(dy, 9), torch.full_like(x, 9), torch.empty_like(a)
    ops.pbg_group_linear(ctx, x, a, off, y)
    ops.pbg_group_linear_backward(ctx, x, a, off, dy, dx, da)
    for g in range(3):
        s = slice(bounds[g], bounds[g + 1])
        # |sums| of da are below 2^24: 2^26 terms with mean 0 and variance 4, 1.6e4 each standard deviation
        for r in range(m):
            assert torch.equal(y[s, r], sum(x[s, c] * a[g, r, c] for c in range(k)))
            for c in range(k):
                assert float(da[g, r, c]) == float((dy[s, r] * x[s, c]).sum(dtype=torch.float64))
        for c in range(k):
            assert torch.equal(dx[s, c], sum(dy[s, r] * a[g, r, c] for r in range(m)))
    for o in (y, dx):
        assert bool((o[:1] == 9).all()) and bool((o[n - 2:] == 9).all())


def test_more_rows_to_lay_out_than_a_launch_takes(ctx):
    n, k, m = (1 << 27) + 3, 3, 8
    x, a = small_integers(6, n, k, dtype=torch.float16), small_integers(7, 1, m, k, dtype=torch.float16)
    y = torch.empty(n, m, dtype=torch.float16, device="cuda")
    ops.pbg_group_linear(ctx, x, a, offsets(0, n), y)
    for r in range(m):
        assert torch.equal(y[:, r], sum(x[:, c] * a[0, r, c] for c in range(k)))


def test_no_rows_for_many_wide_matrices(ctx):
    da = torch.full((40, 300, 500), 3.0, device="cuda")
    dy, x = torch.empty(0, 300, device="cuda"), torch.empty(0, 500, device="cuda")
    ops.pbg_group_linear_backward(ctx, x, None, offsets(*([0] * 41)), dy, None, da)
    assert bool((da == 0).all())
    with pytest.raises(pbg.PbgError, match="offsets"):
        ops.pbg_group_linear_backward(ctx, x, None, offsets(*([0] * 40 + [1])), dy, None, da.fill_(3.0))
    assert bool((da == 3).all())


def test_values_on_another_device_are_refused(ctx, monkeypatch):
    x, a = torch.ones(4, 8, device="cuda"), torch.ones(1, 8, 8, device="cuda")
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 1)
    with pytest.raises(ValueError, match="device"):
        ops.pbg_group_linear(ctx, x, a, offsets(0, 4), torch.empty(4, 8, device="cuda"))
    with pytest.raises(ValueError, match="device"):
        ops.pbg_clip_gradients(ctx, [x, a], 1.0)
    assert bool((x == 1).all())


def test_more_values_than_memory_are_refused(ctx):
    import ctypes
    x = torch.ones(8, device="cuda")
    for counts in ((2 ** 62, 2 ** 62), (8, -1), (2 ** 38, 1)):
        p = (ctypes.c_void_p * 2)(x.data_ptr(), x.data_ptr())
        status = ops.library().pbg_clip_gradients(ctx, 2, (ctypes.c_int32 * 2)(0, 0), (ctypes.c_int64 * 2)(*counts), p,
                                                  None, 1.0, None)
        assert status == 1   # INVALID_ARG
    assert bool((x == 1).all())


def test_two_contexts_at_once():
    """Two threads, each with a context and a stream of its own; every answer has the bits of a call made alone."""
    def work(c, seed, out, rounds):
        try:
            g = torch.Generator(device="cuda").manual_seed(seed)
            n, k, m, V = 700, 96, 72, 300
            x, dy = torch.randn(n, k, generator=g, device="cuda"), torch.randn(n, m, generator=g, device="cuda")
            a = torch.randn(5, m, k, generator=g, device="cuda")
            z = torch.randn(n, V, generator=g, device="cuda")
            labels = torch.randint(0, V, (n,), generator=g, device="cuda", dtype=torch.int32)
            off, seq = offsets(0, 10, 10, 300, 600, n), offsets(0, 200, 350, 500, n)
            torch.cuda.synchronize()
            for _ in range(rounds):
                y, dx, da = torch.empty_like(dy), torch.empty_like(x), torch.empty_like(a)
                loss, logp, dlogp = (torch.empty(s, device="cuda") for s in (2, 4, 4))
                stats, dz = torch.empty(n, 2, device="cuda"), torch.empty_like(z)
                torch.cuda.synchronize()
                ops.pbg_group_linear(c, x, a, off, y)
                ops.pbg_group_linear_backward(c, x, a, off, dy, dx, da)
                ops.pbg_preference_loss(c, z, labels, seq, None, 0.1, 0.0, loss, logp, dlogp, stats)
                ops.pbg_preference_loss_backward(c, z, labels, seq, stats, dlogp, dz)
                norm = ops.pbg_clip_gradients(c, [dx, da], 1.0)
                out.append([t.cpu() for t in (y, dx, da, loss, logp, dlogp, stats, dz)] + [torch.tensor(norm)])
        except Exception as e:   # seen by the test below
            out.append(e)

    contexts, results = [], []
    for _ in range(2):
        c = context()
        pbg.pbg_set_streams(c, torch.cuda.Stream(), None)
        contexts.append(c)
    alone = []
    for i in range(2):
        out = []
        work(contexts[i], i, out, 1)
        alone.append(out[0])
        results.append([])
    threads = [threading.Thread(target=work, args=(contexts[i], i, results[i], 10)) for i in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    for i in range(2):
        assert len(results[i]) == 10
        for r in results[i]:
            assert not isinstance(r, Exception), r
            assert all(torch.equal(p, q) for p, q in zip(r, alone[i]))
    for c in contexts:
        pbg.pbg_free(c)


@pytest.mark.parametrize("sizes,k,m", [([600] * 7 + [4000, 0], 2048, 2048),    # wide tiles, one group longer than a slot
                                       ([513, 700, 499] * 19 + [2500], 500, 1000),   # matrices that end inside a tile
                                       ([900] * 4, 264, 520), ([64, 0, 1], 1030, 1040)])
@pytest.mark.parametrize("t", [torch.bfloat16, torch.float16])
def test_gradients_of_large_matrices(ctx, sizes, k, m, t):
    n, groups = sum(sizes), len(sizes)
    x, dy = small_integers(8, n, k, dtype=t), small_integers(9, n, m, dtype=t)
    # sums of whole numbers below 2^24: exact in float32 in any order
    off = torch.tensor(np.concatenate([[0], np.cumsum(sizes)]), dtype=torch.int64, device="cuda")
    da = torch.full((groups, m, k), 9.0, dtype=t, device="cuda")
    ops.pbg_group_linear_backward(ctx, x, None, off, dy, None, da)
    for g in range(groups):
        r = slice(int(off[g]), int(off[g + 1]))
        exact = dy[r].float().t().contiguous() @ x[r].float()
        assert torch.equal(da[g], exact.to(t))


@pytest.mark.parametrize("t", [torch.float32, torch.float16])
@pytest.mark.parametrize("n,k,m", [(300, 64, 72), (300, 50, 33), (40, 1, 1)])
def test_largest_row_stride(ctx, t, n, k, m):
    ld = 1 << 20
    x, dy, a = small_integers(10, n, k, dtype=t), small_integers(11, n, m, dtype=t), small_integers(12, 2, m, k, dtype=t)
    off = offsets(0, n // 3, n)

    def wide(v=None, width=None):
        w = torch.full((n, ld), 9.0, dtype=t, device="cuda")[:, 5:5 + (width or v.shape[1])]
        if v is not None:
            w.copy_(v)
        return w

    y, dx = wide(width=m), wide(width=k)
    da = torch.empty(2, m, k, dtype=t, device="cuda")
    ops.pbg_group_linear(ctx, wide(x), a, off, y)
    ops.pbg_group_linear_backward(ctx, wide(x), a, off, wide(dy), dx, da)
    y2, dx2, da2 = torch.empty_like(dy), torch.empty_like(x), torch.empty_like(da)
    ops.pbg_group_linear(ctx, x, a, off, y2)
    ops.pbg_group_linear_backward(ctx, x, a, off, dy, dx2, da2)
    assert torch.equal(y, y2) and torch.equal(dx, dx2) and torch.equal(da, da2)
    for g, r in ((0, slice(0, n // 3)), (1, slice(n // 3, n))):
        assert torch.equal(y2[r], (x[r].double() @ a[g].double().t()).to(t))
        assert torch.equal(dx2[r], (dy[r].double() @ a[g].double()).to(t))
        assert torch.equal(da2[g], (dy[r].double().t() @ x[r].double()).to(t))


@pytest.mark.parametrize("t", [torch.float32, torch.bfloat16])
def test_largest_number_of_groups(ctx, t):
    G, n, k, m = 1 << 20, 3000, 4, 8
    rows = np.sort(np.random.default_rng(0).integers(0, G, n))   # most groups are empty
    off = torch.from_numpy(np.searchsorted(rows, np.arange(G + 1)).astype(np.int64)).cuda()
    group = torch.from_numpy(rows).cuda()
    x, dy, a = small_integers(13, n, k, dtype=t), small_integers(14, n, m, dtype=t), small_integers(15, G, m, k, dtype=t)
    y, dx, da = torch.empty_like(dy), torch.empty_like(x), torch.full_like(a, 9)
    ops.pbg_group_linear(ctx, x, a, off, y)
    ops.pbg_group_linear_backward(ctx, x, a, off, dy, dx, da)
    mine = a[group].double()
    assert torch.equal(y.double(), (mine * x.double()[:, None, :]).sum(2))
    assert torch.equal(dx.double(), (mine * dy.double()[:, :, None]).sum(1))
    want = torch.zeros(G, m, k, dtype=torch.float64, device="cuda")
    want.index_add_(0, group, dy.double()[:, :, None] * x.double()[:, None, :])
    assert torch.equal(da.double(), want)
