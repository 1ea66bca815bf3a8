"""Sizes at the ends of their range, which the calls for weights and eviction refuse or take: none of it needs a device."""
import pytest

from paper_2602_14236_b200 import binding as sc
from test_paged_serving_refusals import _keep, _select


@pytest.mark.parametrize("budget", [2 ** 30 + 1, 2 ** 31 - 1])
def test_a_budget_past_every_position_is_refused(budget):
    assert _select(budget=budget) == sc.E_PARAM
    assert _keep(kw=budget) == sc.E_SHAPE


def test_the_largest_ones_still_need_a_context():
    assert _select(budget=2 ** 30, sinks=2 ** 29, recent=2 ** 29) == sc.E_NULL
    assert _keep(kw=2 ** 30) == sc.E_NULL
