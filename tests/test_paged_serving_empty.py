"""Arrays without elements need no address, which an empty tensor has none of: none of it needs a device.  Each call has a mistake that
is looked for after its addresses."""
import pytest

from paper_2602_14236_b200 import binding as sc
from test_paged_serving_refusals import A, _keep, _pages, _select, _seqs, _tree, _weigh, _write


def test_no_rows_need_no_address():
    none = _seqs(n_rows=0)
    assert _write(seqs=none, pos=None, q=None, qo=None, k=None, v=A + 8) == sc.E_ALIGN
    assert _write(seqs=none, pos=None, qo=None, k=None, v=None, qs=504) == sc.E_SHAPE
    assert _tree(seqs=none, tree=None, q=None, out=None, lse=None, words=0) == sc.E_PARAM
    assert _weigh(seqs=none, q=None, lse=None, decay=1.5) == sc.E_PARAM
    assert sc.lib().salicache_paged_write(None, _pages(), none, None, None, 256, 252, None) == sc.E_SHAPE
    assert sc.lib().salicache_paged_attend(None, _pages(), none, None, 512, 2, 0.1, 0, 0, None, 512, None, A + 8, 1 << 40, None) == sc.E_ALIGN


def test_no_sequences_need_no_address():
    none = _seqs(n_seqs=0, n_rows=0, d_row_start=None, d_len=None, d_table=None)
    assert _weigh(seqs=none, q=None, lse=None, w_in=None, w_out=None, ws=0) == sc.E_SHAPE
    assert _select(n=0, w=None, ln=None, keep=None, kept=None, budget=0) == sc.E_PARAM
    assert _keep(seqs=none, keep=None, kept=None, kh=3) == sc.E_SHAPE


def test_no_entries_need_no_address():
    assert _keep(keep=None, kw=0, kh=3) == sc.E_SHAPE
    assert _keep(keep=None, kw=1, kh=3) == sc.E_NULL


def test_offsets_that_moving_does_not_use_may_be_missing():
    assert _keep(seqs=_seqs(d_row_start=None), kh=3) == sc.E_SHAPE
    assert _keep(to=_seqs(d_row_start=None, d_len=None, d_table=2 * A), kh=3) == sc.E_SHAPE
    assert _keep(seqs=_seqs(d_row_start=None), to=_seqs(d_row_start=None, d_len=None, d_table=2 * A), first=A + 2) == sc.E_ALIGN
    assert _keep(to=_seqs(d_table=None), kh=3) == sc.E_NULL


@pytest.mark.parametrize("call", [_write, _tree, _weigh])
def test_rows_that_belong_to_nobody_still_need_one(call):
    assert call(seqs=_seqs(n_seqs=0, n_rows=3), q=None, **({} if call is not _write else dict(k=None))) == sc.E_NULL
