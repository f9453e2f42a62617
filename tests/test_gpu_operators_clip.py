"""The joint norm of many gradients and their clipping, against float64; and the operators together."""
import math

import numpy as np
import pytest
import torch

from paper_1903_12287_amd import operators as ops
from paper_1903_12287_amd import pbg
from tests.operators_cases import SENTINEL, TYPES, context, half_step, offsets_of, smallest_step

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    c = context()
    yield c
    pbg.pbg_free(c)


def tensors(seed, sizes, types, fronts=(0,), scale=1.0):
    rng = np.random.default_rng(seed)
    out = []
    for i, n in enumerate(sizes):
        dt, f = TYPES[types[i % len(types)]], fronts[i % len(fronts)]
        buf = torch.full((f + n + 40,), SENTINEL, dtype=dt, device="cuda")
        buf[f:f + n] = torch.from_numpy(rng.standard_normal(n) * scale).to(dt).cuda()
        out.append((buf, buf[f:f + n]))
    return out


def norm_of(ts):
    return math.sqrt(sum(float(t.double().cpu().square().sum()) for t in ts))


def check(got, g, factor):
    """One rounding of a product in float64."""
    want = g.double().cpu() * factor
    tol = half_step(g.dtype) * want.abs() * (1 + 1e-6) + smallest_step(g.dtype)
    assert bool(((got.double().cpu() - want).abs() <= tol).all())


SIZES = [[1], [5], [64, 1, 3], [4096], [16_384, 16_385, 16_383], [100_003, 7], [1] * 100, [1_000_003], [9_000_001, 3],
         [30_000] * 97 + [5, 70_001], list(range(1, 210, 7))]


@pytest.mark.parametrize("types", [("f32",), ("bf16",), ("f16",), ("f32", "bf16", "f16")])
@pytest.mark.parametrize("sizes", SIZES, ids=lambda s: f"{len(s)}x{max(s)}")
def test_norm_and_scaling(ctx, sizes, types):
    for fronts in ((0,), (0, 1, 2, 3, 8)):
        pairs = tensors(len(sizes), sizes, types, fronts)
        gs = [v for _, v in pairs]
        before = [v.clone() for v in gs]
        norm = norm_of(gs)
        for bound in (0.31 * norm, 3.0 * norm):
            outs = [torch.full((v.numel() + 2,), SENTINEL, dtype=v.dtype, device="cuda") for v in gs]
            got = ops.pbg_clip_gradients(ctx, gs, bound, [o[1:-1] for o in outs])
            # sums of squares in float64, at most their number of roundings apart
            assert abs(got - norm) <= sum(sizes) * 2.0 ** -53 * norm
            factor = min(1.0, bound / got)
            for o, g, b in zip(outs, gs, before):
                assert float(o[0]) == SENTINEL and float(o[-1]) == SENTINEL
                check(o[1:-1], b, factor)
                assert torch.equal(g, b)
            if factor == 1.0:
                assert all(torch.equal(o[1:-1], b) for o, b in zip(outs, before))
            again = ops.pbg_clip_gradients(ctx, gs, bound, [o[1:-1] for o in outs])
            assert again == got
        ops.pbg_clip_gradients(ctx, gs, 0.31 * norm)   # in place
        for (buf, v), b, o, f in zip(pairs, before, outs, fronts * len(gs)):
            check(v, b, 0.31 * norm / got)
            assert bool((buf[v.numel() + f:] == SENTINEL).all()) and bool((buf[:f] == SENTINEL).all())


def test_norms_out_of_range(ctx):
    """Squares beyond float32's range, and far below it."""
    for v in (1e30, 1e-30, 1e-44):
        g = torch.full((1000,), v, device="cuda")
        x = float(g[0])
        assert abs(ops.pbg_clip_gradients(ctx, [g], math.inf) / (x * math.sqrt(1000)) - 1) < 1e-12
        assert bool((g == x).all())
        got = ops.pbg_clip_gradients(ctx, [g], x)
        assert abs(got / (x * math.sqrt(1000)) - 1) < 1e-12
        want = torch.full((1000,), x, dtype=torch.float64) * (x / got)
        assert bool(((g.double().cpu() - want).abs() <= want * 2.0 ** -24 * (1 + 1e-6) + 2.0 ** -150).all())


@pytest.mark.parametrize("bad", [math.inf, -math.inf, math.nan])
def test_a_norm_that_is_not_finite_scales_nothing(ctx, bad):
    g = [torch.ones(70_000, device="cuda"), torch.ones(100, dtype=torch.bfloat16, device="cuda")]
    g[0][50_001] = bad
    keep = [v.clone() for v in g]
    outs = [torch.zeros_like(v) for v in g]
    got = ops.pbg_clip_gradients(ctx, g, 0.5, outs)
    assert not math.isfinite(got)
    got = ops.pbg_clip_gradients(ctx, g, 0.5)
    assert not math.isfinite(got)
    for a, b, o in zip(g, keep, outs):
        assert torch.equal(a.nan_to_num(3.0), b.nan_to_num(3.0)) and torch.equal(o.nan_to_num(3.0), b.nan_to_num(3.0))


def test_nothing_to_clip(ctx):
    assert ops.pbg_clip_gradients(ctx, [], 1.0) == 0.0
    empty = torch.empty(0, device="cuda")
    assert ops.pbg_clip_gradients(ctx, [empty, empty], 1.0) == 0.0
    z = torch.zeros(10, device="cuda")
    assert ops.pbg_clip_gradients(ctx, [z, empty], 1.0, [z, empty]) == 0.0
    assert bool((z == 0).all())


def test_refusals(ctx):
    g = torch.ones(100, device="cuda")
    for bound in (0.0, -1.0, math.nan):
        with pytest.raises(pbg.PbgError, match="max_norm"):
            ops.pbg_clip_gradients(ctx, [g], bound)
    with pytest.raises(pbg.PbgError, match="overlap"):
        ops.pbg_clip_gradients(ctx, [g, g], 1.0)             # the same tensor twice, in place
    with pytest.raises(pbg.PbgError, match="overlap"):
        ops.pbg_clip_gradients(ctx, [g[:60], g[50:]], 1.0)
    o = torch.zeros(200, device="cuda")
    with pytest.raises(pbg.PbgError, match="overlap"):
        ops.pbg_clip_gradients(ctx, [g, g], 1.0, [o[:100], o[50:150]])
    with pytest.raises(pbg.PbgError, match="overlap"):
        ops.pbg_clip_gradients(ctx, [o[:100]], 1.0, [o[1:101]])
    assert bool((g == 1).all()) and bool((o == 0).all())
    ops.pbg_clip_gradients(ctx, [g, g], 1.0, [o[:100], o[100:]])   # read twice, written apart
    assert bool((o == o[0]).all()) and abs(float(o[0]) - 1 / math.sqrt(200)) < 1e-7
    ops.pbg_clip_gradients(ctx, [g[:50], g[50:]], 1.0)
    with pytest.raises(TypeError):
        ops.pbg_clip_gradients(ctx, [g.double()], 1.0)
    with pytest.raises(ValueError):
        ops.pbg_clip_gradients(ctx, [torch.ones(4, 4, device="cuda").t()[:, :2]], 1.0)
    with pytest.raises(ValueError):
        ops.pbg_clip_gradients(ctx, [g], 1.0, [o])
    with pytest.raises(ValueError):
        ops.pbg_clip_gradients(ctx, [g, g], 1.0, [o[:100]])


def test_more_than_four_gib(ctx):
    """One tensor of more than 2^31 values; squares of ones, so that the norm is exact."""
    n = (1 << 31) + 12_345
    g = torch.ones(n, dtype=torch.bfloat16, device="cuda")
    got = ops.pbg_clip_gradients(ctx, [g], 1.0)
    assert abs(got - math.sqrt(n)) <= 1e-9 * math.sqrt(n)
    want = torch.tensor(1.0 / got, dtype=torch.float64).to(torch.bfloat16).item()
    assert all(bool((g[i:i + (1 << 28)] == want).all()) for i in range(0, n, 1 << 28))


def test_a_training_step_of_the_operators(ctx):
    """The operators together, as a step uses them: queries by relation, scores of all candidates, the loss on pairs
    of paths, all gradients back, clipped by their joint norm; against float64 autograd of the same step."""
    rng = np.random.default_rng(4)
    n, d, G, V, Q = 120, 24, 5, 90, 8
    goff = offsets_of(rng.multinomial(n, [0.4, 0.0, 0.3, 0.2, 0.1]))
    soff = offsets_of(rng.multinomial(n, [1.0 / Q] * Q))
    f = {"dtype": torch.float32}
    x, A, C = (torch.from_numpy(rng.standard_normal(s)).to(**f) for s in ((n, d), (G, d, d), (V, d)))
    A, C = A * d ** -0.5, C * 0.5
    labels = torch.from_numpy(rng.integers(-1, V, n).astype(np.int32))
    ref = torch.from_numpy(rng.standard_normal(Q)).to(**f) * 3 - 40
    beta, eps = 0.25, 0.125
    # float64
    X, AA, CC = (v.double().requires_grad_() for v in (x, A, C))
    q = torch.cat([X[int(a):int(b)] @ AA[g].t() for g, (a, b) in enumerate(zip(goff[:-1], goff[1:]))])
    lp = torch.log_softmax(q @ CC.t(), 1)
    l = torch.where(labels >= 0, lp[torch.arange(n), labels.clamp(min=0).long()], torch.zeros(1).double())
    s = torch.stack([l[int(a):int(b)].sum() for a, b in zip(soff[:-1], soff[1:])]) - ref.double()
    h = beta * (s[0::2] - s[1::2])
    loss = (1 - eps) * torch.nn.functional.softplus(-h) + eps * torch.nn.functional.softplus(h)
    loss.sum().backward()
    grads = (X.grad, AA.grad, CC.grad)
    norm = math.sqrt(sum(float(v.square().sum()) for v in grads))
    # the operators
    dev = {"device": "cuda", "dtype": torch.float32}
    x, A, C, ref = x.cuda(), A.cuda(), C.cuda(), ref.cuda()
    labels, go, so = labels.cuda(), torch.from_numpy(goff).cuda(), torch.from_numpy(soff).cuda()
    one = torch.tensor([0, n], dtype=torch.int64, device="cuda")
    q32, z = torch.empty(n, d, **dev), torch.empty(n, V, **dev)
    ops.pbg_group_linear(ctx, x, A, go, q32)
    ops.pbg_group_linear(ctx, q32, C[None], one, z)
    l32, logp, dlogp, stats = (torch.empty(s, **dev) for s in (Q // 2, Q, Q, (n, 2)))
    ops.pbg_preference_loss(ctx, z, labels, so, ref, beta, eps, l32, logp, dlogp, stats)
    ops.pbg_preference_loss_backward(ctx, z, labels, so, stats, dlogp, z)
    dq, dC, dx, dA = torch.empty(n, d, **dev), torch.empty(1, V, d, **dev), torch.empty(n, d, **dev), torch.empty(G, d, d, **dev)
    ops.pbg_group_linear_backward(ctx, q32, C[None], one, z, dq, dC)
    ops.pbg_group_linear_backward(ctx, x, A, go, dq, dx, dA)
    got = ops.pbg_clip_gradients(ctx, [dx, dA, dC], 0.5 * norm)
    assert float((l32.double().cpu() - loss.detach()).abs().max()) <= 1e-5 * float(loss.detach().abs().max())
    assert abs(got / norm - 1) <= 1e-5
    for mine, want in zip((dx, dA, dC[0]), grads):
        want = 0.5 * want
        # float32 products of depth up to 120 over values of a few units: 1e-5 of the largest gradient is over a
        # hundred half steps of it
        assert float((mine.double().cpu() - want).abs().max()) <= 1e-5 * float(want.abs().max()) * 4
