"""The binding of the operators on a caller's own tensors: what it has to see before the library is called."""
import pytest
import torch

from paper_1903_12287_amd import operators as ops
from paper_1903_12287_amd import pbg
from tests.operators_cases import SENTINEL, context

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    c = context()
    yield c
    pbg.pbg_free(c)


def test_more_groups_than_32_bits_hold(ctx):
    """2^32 + 1 groups: the low 32 bits alone would be one group, with good offsets."""
    groups, n = (1 << 32) + 1, 5
    a = torch.empty(groups, 1, 1, dtype=torch.bfloat16, device="cuda")
    offsets = torch.empty(groups + 1, dtype=torch.int64, device="cuda")
    a[0], offsets[0], offsets[1] = 1.0, 0, n
    x, y = torch.ones(n, 1, dtype=torch.bfloat16, device="cuda"), torch.full((n, 1), SENTINEL, dtype=torch.bfloat16, device="cuda")
    with pytest.raises(ValueError, match="groups"):
        ops.pbg_group_linear(ctx, x, a, offsets, y)
    with pytest.raises(ValueError, match="groups"):
        ops.pbg_group_linear_backward(ctx, None, a, offsets, x, y, None)
    with pytest.raises(ValueError, match="groups"):
        ops.pbg_group_linear_backward(ctx, x, None, offsets, x, None, a)
    assert bool((y == SENTINEL).all()) and float(a[0]) == 1.0


def test_more_pairs_than_the_library_takes(ctx):
    pairs, n = (1 << 19) + 1, 3
    offsets = torch.full((2 * pairs + 1,), n, dtype=torch.int64, device="cuda")
    z, labels = torch.zeros(n, 4, device="cuda"), torch.zeros(n, dtype=torch.int32, device="cuda")
    logp, stats = torch.full((2 * pairs,), SENTINEL, device="cuda"), torch.full((n, 2), SENTINEL, device="cuda")
    with pytest.raises(pbg.PbgError, match="pairs"):
        ops.pbg_preference_loss(ctx, z, labels, offsets, None, 0.1, 0.0, None, logp, None, stats)
    with pytest.raises(pbg.PbgError, match="pairs"):
        ops.pbg_preference_loss_backward(ctx, z, labels, offsets, stats, logp, z)
    assert bool((logp == SENTINEL).all()) and bool((stats == SENTINEL).all()) and bool((z == 0).all())


def saved(shape):
    """A leaf, the tensor that its graph keeps for its backward, and a handle to the same memory outside the graph."""
    leaf = torch.zeros(shape, device="cuda", requires_grad=True)
    kept = torch.exp(leaf)   # keeps its result
    return leaf, kept, kept.detach()


@pytest.mark.parametrize("name", ["y", "dx", "da", "loss", "logp", "dlogp", "row_stats", "dlogits", "logits", "grads", "outs"])
def test_autograd_sees_what_is_written(ctx, name):
    n, k, m = 4, 3, 3
    off, seq = (torch.tensor(v, dtype=torch.int64, device="cuda") for v in ([0, n], [0, 2, n]))
    shapes = {"y": (n, m), "dx": (n, k), "da": (1, m, k), "loss": (1,), "logp": (2,), "dlogp": (2,), "row_stats": (n, 2),
              "dlogits": (n, k), "logits": (n, k), "grads": (n, k), "outs": (n, k)}
    leaf, kept, mine = saved(shapes[name])
    t = {s: torch.ones(shape, device="cuda") for s, shape in shapes.items()}
    t[name] = mine
    x, a, labels = torch.ones(n, k, device="cuda"), torch.ones(1, m, k, device="cuda"), torch.zeros(n, dtype=torch.int32, device="cuda")
    if name == "y":
        ops.pbg_group_linear(ctx, x, a, off, t["y"])
    elif name in ("dx", "da"):
        ops.pbg_group_linear_backward(ctx, x, a, off, torch.ones(n, m, device="cuda"), t["dx"], t["da"])
    elif name in ("loss", "logp", "dlogp", "row_stats"):
        ops.pbg_preference_loss(ctx, x, labels, seq, None, 0.1, 0.0, t["loss"], t["logp"], t["dlogp"], t["row_stats"])
    elif name == "dlogits":
        ops.pbg_preference_loss_backward(ctx, x, labels, seq, t["row_stats"], t["dlogp"], t["dlogits"])
    elif name == "logits":   # the gradient over the scores
        ops.pbg_preference_loss_backward(ctx, t["logits"], labels, seq, t["row_stats"], t["dlogp"], t["logits"])
    else:
        ops.pbg_clip_gradients(ctx, [t["grads"]], 0.5, [t["outs"]] if name == "outs" else None)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        kept.sum().backward()


def test_autograd_goes_on_where_nothing_is_written(ctx):
    leaf, kept, mine = saved((5, 3))
    for bound in (float("inf"), 100.0):   # the norm alone, or within its bound
        assert abs(ops.pbg_clip_gradients(ctx, [mine], bound) - 15 ** 0.5) < 1e-12
    off = torch.tensor([0, 9], dtype=torch.int64, device="cuda")
    with pytest.raises(pbg.PbgError, match="offsets"):
        ops.pbg_group_linear(ctx, torch.ones(5, 3, device="cuda"), torch.ones(1, 3, 3, device="cuda"), off, mine)
    kept.sum().backward()
    assert bool((leaf.grad == 1).all())


def test_tensors_of_inference_mode(ctx):
    """They have no version to count."""
    with torch.inference_mode():
        g = torch.ones(16, device="cuda")
        ops.pbg_clip_gradients(ctx, [g], 1.0)
    assert bool((g == 0.25).all())
    ops.pbg_clip_gradients(ctx, [g], 0.5)
    assert bool((g == 0.125).all())
