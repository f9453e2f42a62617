"""The preference loss where a row's work passes from a wave to a workgroup, and the rows from a few to many."""
import pytest

from paper_1903_12287_amd import pbg
from tests.operators_cases import TYPES, context
from tests.test_gpu_operators_preference import Case, compare

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    c = context()
    yield c
    pbg.pbg_free(c)


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("V", [2_048, 2_049, 4_096, 4_097, 6_144, 6_145, 12_288, 12_289])
def test_rows_by_waves_and_workgroups(ctx, t, V):
    compare(Case(TYPES[t], [900, 0, 650, 550], V, first=1, tail=2, pad=V % 3, hidden=0.05, seed=V), ctx)


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("rows", [2_047, 2_048, 2_049])
def test_few_and_many_rows(ctx, t, rows):
    compare(Case(TYPES[t], [rows - 700, 0, 699, 1], 130, seed=rows), ctx)


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("lengths,V", [([512, 0], 64), ([511, 1], 64), ([0, 513], 63), ([100, 156, 0, 256], 64),
                                       ([1] * 512, 64), ([1] * 514, 60), ([3, 4], 4_681), ([3, 4], 4_682), ([1, 0], 32_768)])
def test_small_calls(ctx, t, lengths, V):
    compare(Case(TYPES[t], lengths, V, first=0, hidden=0.05, seed=V), ctx)
