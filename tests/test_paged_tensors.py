"""What the binding of the paged calls compares before it hands an address on: types, sizes, devices.  None of it needs a device:
the current one is taken to be -1, which is where torch says that host tensors are, and a context without a handle is what the
library refuses last (E_NULL)."""
from types import SimpleNamespace

import pytest
import torch

from paper_2602_14236_b200 import binding as sc

A = 1 << 20          # an aligned address that nothing dereferences
CTX = SimpleNamespace(handle=None)
HEADS, D, ROWS, G = 2, 64, 5, 3


@pytest.fixture(autouse=True)
def _host(monkeypatch):
    monkeypatch.setattr(sc, "_here", lambda: (-1, None))


def _pages(dtype=sc.F16):
    return sc.Pages(d_data=A, d_scale=A, n_pages=4, page=16, heads=HEADS, head_dim=D, format=sc.INT8, dtype=dtype)


def _seqs(**kw):
    return sc.SeqsC(**dict(dict(n_seqs=2, table_width=3, n_rows=ROWS, d_row_start=A, d_len=A, d_table=A), **kw))


def _rows(n=ROWS, width=HEADS * D, dtype=torch.float16):
    return torch.zeros((n, width), dtype=dtype)


def _move(k=None, v=None, ks=HEADS * D, vs=HEADS * D, pages=None, seqs=None, **kw):
    for call in (sc.salicache_paged_write, sc.salicache_paged_read):
        call(CTX, pages or _pages(), seqs or _seqs(), _rows() if k is None else k, _rows() if v is None else v, ks, vs, **kw)


def _attend(pages=None, seqs=None, q=None, out=None, lse=None, work=None, wb=64, qs=HEADS * G * D, os=HEADS * G * D, **kw):
    wide = lambda: _rows(width=HEADS * G * D)
    sc.salicache_paged_attend(CTX, pages or _pages(), seqs or _seqs(), wide() if q is None else q, qs, G, 0.1, 0, 0,
                              wide() if out is None else out, os, lse, torch.zeros(64, dtype=torch.uint8) if work is None else work, wb, **kw)


def _accepted(call, **kw):
    with pytest.raises(sc.SalicacheError) as e:
        call(**kw)
    assert e.value.status == sc.E_NULL


def test_what_fits_is_handed_on():
    _accepted(_move)
    _accepted(_attend, lse=torch.zeros(ROWS * HEADS * G), work=torch.zeros(16))
    _accepted(_move, k=_rows(dtype=torch.bfloat16), v=_rows(dtype=torch.bfloat16), pages=_pages(sc.BF16))
    wide = _rows(width=2 * HEADS * D + 8)            # K and V as parts of wider rows: the last row of V ends with the memory
    _accepted(_move, k=wide, v=wide[:, HEADS * D + 8:], ks=wide.shape[1], vs=wide.shape[1])
    wide = _rows(width=HEADS * (G + 2) * D)
    _accepted(_attend, q=wide, qs=wide.shape[1])
    _accepted(_move, k=_rows(0), v=_rows(0), seqs=_seqs(n_rows=0))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.int16])
def test_another_type_is_refused(dtype):
    for kw in (dict(k=_rows(dtype=dtype)), dict(v=_rows(dtype=dtype))):
        with pytest.raises(ValueError, match="type"):
            _move(**kw)
    for kw in (dict(q=_rows(width=HEADS * G * D, dtype=dtype)), dict(out=_rows(width=HEADS * G * D, dtype=dtype)),
               dict(lse=torch.zeros(ROWS * HEADS * G, dtype=torch.float64))):
        with pytest.raises(ValueError, match="type"):
            _attend(**kw)


def test_too_little_memory_is_refused():
    part = _rows(ROWS + 1)[2:]
    for kw in (dict(k=_rows(ROWS - 1)), dict(v=part), dict(ks=HEADS * D + 8), dict(k=_rows(1).expand(ROWS, -1))):
        with pytest.raises(ValueError, match="memory"):
            _move(**kw)
    wide = _rows(width=2 * HEADS * D)
    with pytest.raises(ValueError, match="memory"):
        _move(k=wide, v=wide[:, HEADS * D + 8:], ks=2 * HEADS * D, vs=2 * HEADS * D)
    for kw in (dict(q=_rows(width=HEADS * G * D - 8)), dict(out=_rows(ROWS - 1, HEADS * G * D)), dict(os=HEADS * G * D + 8),
               dict(lse=torch.zeros(ROWS * HEADS * G - 1)), dict(work=torch.zeros(15)), dict(wb=65)):
        with pytest.raises(ValueError, match="memory"):
            _attend(**kw)


def test_another_device_is_refused():
    for which, struct in (("pages", _pages()), ("seqs", _seqs())):
        struct.device = 1
        for call in (_move, _attend):
            with pytest.raises(ValueError, match="cuda:1"):
                call(**{which: struct})
    for call in (_move, _attend):
        with pytest.raises(ValueError, match="cuda:1"):
            call(stream=SimpleNamespace(device_index=1, cuda_stream=0))
        _accepted(call, stream=SimpleNamespace(device_index=-1, cuda_stream=0))
