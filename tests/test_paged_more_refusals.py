"""More arguments that the paged calls refuse or take: none of it needs a device."""
import pytest

from test_paged_refusals import CALLS, _attend, _pages, _seqs
from paper_2602_14236_b200 import binding as sc


def test_a_scale_that_leaves_binary32_in_powers_of_two():
    assert _attend(_pages(), _seqs(), scale=3.0e38) == sc.E_PARAM
    assert _attend(_pages(), _seqs(), scale=2.0 ** 127) == sc.E_NULL           # a context is missing, nothing else


@pytest.mark.parametrize("call", CALLS)
def test_sixteen_bit_pages_have_no_scales_to_look_at(call):
    assert call(_pages(format=sc.FP16, d_scale=2), _seqs()) == sc.E_NULL
