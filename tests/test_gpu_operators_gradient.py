"""The preference loss to the last bits of float32: its gradient, value by value, and its rows' log sums."""
import pytest
import torch

from paper_1903_12287_amd import operators as ops
from paper_1903_12287_amd import pbg
from tests.operators_cases import U32, context

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    c = context()
    yield c
    pbg.pbg_free(c)


@pytest.mark.parametrize("scale", [1.0, 3.0])
@pytest.mark.parametrize("n,V", [(4_096, 300), (40, 2_000), (4_096, 2_000), (4_096, 15_000), (64, 50_000)])
def test_probabilities_to_float32(ctx, n, V, scale):
    g = torch.Generator(device="cuda").manual_seed(V)
    z = torch.randn(n, V, generator=g, device="cuda") * scale
    labels = torch.randint(0, V, (n,), generator=g, device="cuda", dtype=torch.int32)
    off = torch.tensor([0, n // 2, n], dtype=torch.int64, device="cuda")
    loss, logp, dlogp = (torch.empty(s, device="cuda") for s in (1, 2, 2))
    stats, dz = torch.empty(n, 2, device="cuda"), torch.empty(n, V, device="cuda")
    ops.pbg_preference_loss(ctx, z, labels, off, None, 0.1, 0.0, loss, logp, dlogp, stats)
    ops.pbg_preference_loss_backward(ctx, z, labels, off, stats, torch.ones(2, device="cuda"), dz)
    m, ls = stats.double()[:, :1], stats.double()[:, 1:]
    d = z.double() - m
    p = torch.exp(d - ls)
    assert float(d.min()) > -60.0   # every probability is in the normal range
    # z - m is rounded once, by half a step of its own size, which is what exp(z - m) is off by, relative.  The hardware's
    # power of two is off by 2 half steps (one unit in the last place), the correction of its argument adds one rounding,
    # exp(-log sum) one and the product of the two one; one more for all terms of second order.
    step = torch.where(d == 0, torch.zeros_like(d), torch.exp2(torch.floor(torch.log2(d.abs()))))
    units = step + 6.0
    hot = torch.zeros_like(p).scatter_(1, labels.long()[:, None], 1.0)
    want = hot - p
    # the label's 1 - p is rounded once more
    assert bool(((dz.double() - want).abs() <= U32 * (units * p + hot * want.abs())).all())


@pytest.mark.parametrize("t", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("n,V", [(4_096, 15_000), (2_100, 50_000)])
def test_log_sums_as_good_as_a_plain_sum(ctx, t, n, V):
    """Within a tenth of what a float32 softmax's log sums, rounded to float32, are off by (root mean square over
    thousands of rows, whose own chance is a few hundredths).  Long rows: sums that are joined."""
    g = torch.Generator(device="cuda").manual_seed(V)
    z = (torch.randn(n, V, generator=g, device="cuda") * 3).to(t)
    labels = torch.randint(0, V, (n,), generator=g, device="cuda", dtype=torch.int32)
    off = torch.tensor([0, n // 2, n], dtype=torch.int64, device="cuda")
    loss, logp, dlogp, stats = (torch.empty(s, device="cuda") for s in (1, 2, 2, (n, 2)))
    ops.pbg_preference_loss(ctx, z, labels, off, None, 0.1, 0.0, loss, logp, dlogp, stats)
    exact = torch.cat([torch.exp(b.double() - b.double().amax(1, keepdim=True)).sum(1).log() for b in z.split(512)])
    plain = torch.exp(z.float() - z.float().amax(1, keepdim=True)).sum(1).double().log().float()
    mine, other = ((v.double() - exact).square().mean().sqrt() for v in (stats[:, 1], plain))
    assert float(mine) <= 1.1 * float(other), (float(mine), float(other))
