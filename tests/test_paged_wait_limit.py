"""Arguments of salicache_paged_wait_limit: needs no device."""
from paper_2602_14236_b200 import binding as sc


def test_the_wait_limit_needs_a_context():
    assert sc.lib().salicache_paged_wait_limit(None, 5) == sc.E_NULL
