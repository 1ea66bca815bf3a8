"""Arguments that the paged calls refuse, and what the binding refuses before them: none of it needs a device."""
import ctypes as C

import pytest

from paper_2602_14236_b200 import binding as sc

A = 1 << 20          # an aligned address that nothing dereferences


def _pages(**kw):
    d = dict(d_data=A, d_scale=A, n_pages=4, page=16, heads=2, head_dim=128, format=sc.INT8, dtype=sc.F16)
    d.update(kw)
    return sc.Pages(**d)


def _seqs(**kw):
    d = dict(n_seqs=2, table_width=3, n_rows=5, d_row_start=A, d_len=A, d_table=A)
    d.update(kw)
    return sc.SeqsC(**d)


def _write(pages, seqs, k=A, v=A, ks=256, vs=256):
    return sc.lib().salicache_paged_write(None, pages, seqs, k, v, ks, vs, None)


def _read(pages, seqs, k=A, v=A, ks=256, vs=256):
    return sc.lib().salicache_paged_read(None, pages, seqs, k, v, ks, vs, None)


def _attend(pages, seqs, q=A, qs=512, g=2, scale=0.1, window=0, sinks=0, out=A, os=512, lse=A, work=A, wb=1 << 40):
    return sc.lib().salicache_paged_attend(None, pages, seqs, q, qs, g, scale, window, sinks, out, os, lse, work, wb, None)


CALLS = [_write, _read, _attend]


@pytest.mark.parametrize("call", CALLS)
@pytest.mark.parametrize("pages,want", [
    (dict(d_data=None), sc.E_NULL), (dict(d_scale=None), sc.E_NULL), (dict(format=sc.REUSE), sc.E_PARAM), (dict(format=5), sc.E_PARAM),
    (dict(dtype=2), sc.E_PARAM), (dict(page=8), sc.E_PARAM), (dict(page=48), sc.E_PARAM), (dict(page=256), sc.E_PARAM),
    (dict(head_dim=96), sc.E_PARAM), (dict(head_dim=256), sc.E_PARAM), (dict(heads=0), sc.E_PARAM), (dict(heads=257), sc.E_PARAM),
    (dict(n_pages=0), sc.E_SHAPE), (dict(n_pages=2 ** 22, heads=16, page=128), sc.E_SHAPE), (dict(d_data=A + 8), sc.E_ALIGN), (dict(d_scale=A + 2), sc.E_ALIGN),
])
def test_pages_are_checked(call, pages, want):
    assert call(_pages(**pages), _seqs()) == want


@pytest.mark.parametrize("call", CALLS)
@pytest.mark.parametrize("seqs,want", [
    (dict(n_seqs=-1), sc.E_SHAPE), (dict(n_rows=-1), sc.E_SHAPE), (dict(table_width=0), sc.E_SHAPE), (dict(d_row_start=None), sc.E_NULL),
    (dict(d_len=None), sc.E_NULL), (dict(d_table=None), sc.E_NULL), (dict(d_len=A + 2), sc.E_ALIGN),
])
def test_sequences_are_checked(call, seqs, want):
    assert call(_pages(), _seqs(**seqs)) == want


@pytest.mark.parametrize("call", [_write, _read])
@pytest.mark.parametrize("rows,want", [
    (dict(k=None), sc.E_NULL), (dict(v=None), sc.E_NULL), (dict(ks=248), sc.E_SHAPE), (dict(vs=260), sc.E_SHAPE), (dict(k=A + 8), sc.E_ALIGN),
])
def test_rows_are_checked(call, rows, want):
    assert call(_pages(), _seqs(), **rows) == want


@pytest.mark.parametrize("args,want", [
    (dict(g=0), sc.E_PARAM), (dict(g=65), sc.E_PARAM), (dict(window=-1), sc.E_PARAM), (dict(sinks=-1), sc.E_PARAM), (dict(scale=0.0), sc.E_PARAM),
    (dict(scale=float("nan")), sc.E_PARAM), (dict(scale=float("inf")), sc.E_PARAM), (dict(q=None), sc.E_NULL), (dict(out=None), sc.E_NULL),
    (dict(work=None), sc.E_NULL), (dict(work=A + 8), sc.E_ALIGN), (dict(lse=A + 2), sc.E_ALIGN), (dict(qs=504), sc.E_SHAPE), (dict(os=516), sc.E_SHAPE),
])
def test_attention_arguments_are_checked(args, want):
    assert _attend(_pages(), _seqs(), **args) == want


def test_too_many_rows_for_one_attention_call():
    assert _attend(_pages(), _seqs(n_rows=1 << 29), g=2) == sc.E_SHAPE


@pytest.mark.parametrize("call", CALLS)
def test_sound_arguments_still_need_a_context(call):
    assert call(_pages(), _seqs()) == sc.E_NULL
    assert call(_pages(format=sc.FP16, d_scale=None), _seqs()) == sc.E_NULL


def test_work_bytes_checks():
    f = sc.lib().salicache_paged_work_bytes
    assert f(None, C.byref(_pages(page=8)), 1) == sc.E_PARAM
    assert f(None, C.byref(_pages()), 0) == sc.E_PARAM
    assert f(None, C.byref(_pages()), 4) == sc.E_NULL
    assert f(None, None, 4) == sc.E_NULL


def test_the_binding_refuses_host_tensors():
    import torch
    z = torch.zeros(4, dtype=torch.int32)
    with pytest.raises(ValueError):
        sc.Seqs(z, z[:3], z[:3].view(3, 1), 4)
    with pytest.raises(ValueError):
        sc.PageSet(4, 16, 2, 128, sc.FP16, torch.float16, device="cpu")
