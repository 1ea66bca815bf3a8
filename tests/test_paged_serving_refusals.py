"""Arguments that the calls for positions, trees, weights and eviction refuse, and what the binding refuses before them: none of
it needs a device."""
import ctypes as C
from types import SimpleNamespace

import pytest
import torch

from paper_2602_14236_b200 import binding as sc

A = 1 << 20          # an aligned address that nothing dereferences


def _pages(**kw):
    return sc.Pages(**dict(dict(d_data=A, d_scale=A, n_pages=4, page=16, heads=2, head_dim=128, format=sc.INT8, dtype=sc.F16), **kw))


def _seqs(**kw):
    return sc.SeqsC(**dict(dict(n_seqs=2, table_width=3, n_rows=5, d_row_start=A, d_len=A, d_table=A), **kw))


def _rotary(pairs=64, **kw):
    r = sc.Rotary([0.5] * pairs)
    for k, v in kw.items():
        if k in ("freq", "axis"):
            getattr(r, k)[v[0]] = v[1]
        else:
            setattr(r, k, v)
    return r


def _write(pages=None, seqs=None, rotary=None, pos=A, q=A, qs=512, g=2, qo=A, qos=512, k=A, v=A, ks=256, vs=256):
    return sc.lib().salicache_paged_write_rotary(None, pages or _pages(), seqs or _seqs(), rotary or _rotary(), pos, q, qs, g, qo, qos, k, v, ks,
                                                 vs, None)


def _tree(pages=None, seqs=None, tree=A, words=1, q=A, qs=512, g=2, scale=0.1, window=0, sinks=0, out=A, os=512, lse=A, work=A):
    return sc.lib().salicache_paged_attend_tree(None, pages or _pages(), seqs or _seqs(), tree, words, q, qs, g, scale, window, sinks, out, os,
                                                lse, work, 1 << 40, None)


def _weigh(pages=None, seqs=None, q=A, qs=512, g=2, scale=0.1, lse=A, decay=1.0, w_in=A, w_out=A, ws=48, work=A):
    return sc.lib().salicache_paged_weigh(None, pages or _pages(), seqs or _seqs(), q, qs, g, scale, lse, decay, w_in, w_out, ws, work, 1 << 40,
                                          None)


def _select(w=A, ws=48, heads=2, n=2, ln=A, budget=8, sinks=2, recent=2, keep=A, kept=A):
    return sc.lib().salicache_select_heavy(None, w, ws, heads, n, ln, budget, sinks, recent, keep, kept, None)


def _keep(pages=None, seqs=None, keep=A, kh=2, kw=8, first=None, kept=A, to=None, w_in=None, w_out=None, ws=0):
    return sc.lib().salicache_paged_keep(None, pages or _pages(), seqs or _seqs(), keep, kh, kw, first, kept, to, w_in, w_out, ws, None)


OVER_PAGES = [_write, _tree, _weigh, _keep]


@pytest.mark.parametrize("call", OVER_PAGES)
@pytest.mark.parametrize("pages,want", [
    (dict(d_data=None), sc.E_NULL), (dict(d_scale=None), sc.E_NULL), (dict(format=sc.REUSE), sc.E_PARAM), (dict(dtype=2), sc.E_PARAM),
    (dict(page=8), sc.E_PARAM), (dict(head_dim=96), sc.E_PARAM), (dict(heads=257), sc.E_PARAM), (dict(n_pages=0), sc.E_SHAPE),
    (dict(d_data=A + 8), sc.E_ALIGN), (dict(d_scale=A + 2), sc.E_ALIGN),
])
def test_pages_are_checked(call, pages, want):
    assert call(pages=_pages(**pages)) == want


@pytest.mark.parametrize("call", OVER_PAGES)
@pytest.mark.parametrize("seqs,want", [
    (dict(n_seqs=-1), sc.E_SHAPE), (dict(n_rows=-1), sc.E_SHAPE), (dict(table_width=0), sc.E_SHAPE), (dict(d_len=None), sc.E_NULL),
    (dict(d_table=None), sc.E_NULL), (dict(d_len=A + 2), sc.E_ALIGN),
])
def test_sequences_are_checked(call, seqs, want):
    assert call(seqs=_seqs(**seqs)) == want


@pytest.mark.parametrize("kw,want", [
    (dict(pos=None), sc.E_NULL), (dict(pos=A + 2), sc.E_ALIGN), (dict(q=A + 8), sc.E_ALIGN), (dict(qo=None), sc.E_NULL), (dict(qo=A + 8), sc.E_ALIGN),
    (dict(qs=504), sc.E_SHAPE), (dict(qos=516), sc.E_SHAPE), (dict(qos=520), sc.E_SHAPE), (dict(g=0), sc.E_PARAM), (dict(g=65), sc.E_PARAM),
    (dict(k=None), sc.E_NULL), (dict(v=None), sc.E_NULL), (dict(ks=248), sc.E_SHAPE), (dict(v=A + 8), sc.E_ALIGN),
    (dict(rotary=_rotary(0)), sc.E_PARAM), (dict(rotary=_rotary(12)), sc.E_PARAM), (dict(rotary=_rotary(pairs=64, n_axes=0)), sc.E_PARAM),
    (dict(rotary=_rotary(n_axes=5)), sc.E_PARAM), (dict(rotary=_rotary(pairing=2)), sc.E_PARAM), (dict(rotary=_rotary(axis=(63, 1))), sc.E_PARAM),
    (dict(rotary=_rotary(freq=(0, float("nan")))), sc.E_PARAM), (dict(rotary=_rotary(freq=(63, float("inf")))), sc.E_PARAM),
    (dict(rotary=_rotary(40), pages=_pages(head_dim=64)), sc.E_PARAM),
])
def test_positions_are_checked(kw, want):
    assert _write(**kw) == want


def test_a_missing_rotary_is_refused():
    assert sc.lib().salicache_paged_write_rotary(None, _pages(), _seqs(), None, A, A, 512, 2, A, 512, A, A, 256, 256, None) == sc.E_NULL


ATTENDS = [(dict(g=0), sc.E_PARAM), (dict(g=65), sc.E_PARAM), (dict(scale=0.0), sc.E_PARAM), (dict(scale=float("nan")), sc.E_PARAM),
           (dict(q=None), sc.E_NULL), (dict(work=None), sc.E_NULL), (dict(work=A + 8), sc.E_ALIGN), (dict(lse=A + 2), sc.E_ALIGN), (dict(qs=504), sc.E_SHAPE),
           (dict(seqs=_seqs(n_rows=1 << 29)), sc.E_SHAPE)]


@pytest.mark.parametrize("kw,want", ATTENDS + [
    (dict(tree=None), sc.E_NULL), (dict(tree=A + 4), sc.E_ALIGN), (dict(words=0), sc.E_PARAM), (dict(words=17), sc.E_PARAM), (dict(window=-1), sc.E_PARAM),
    (dict(sinks=-1), sc.E_PARAM), (dict(out=None), sc.E_NULL), (dict(os=516), sc.E_SHAPE)])
def test_trees_are_checked(kw, want):
    assert _tree(**kw) == want


@pytest.mark.parametrize("kw,want", ATTENDS + [
    (dict(lse=None), sc.E_NULL), (dict(w_out=None), sc.E_NULL), (dict(w_in=A + 2), sc.E_ALIGN), (dict(w_out=A + 1), sc.E_ALIGN), (dict(ws=0), sc.E_SHAPE),
    (dict(decay=-0.1), sc.E_PARAM), (dict(decay=1.5), sc.E_PARAM), (dict(decay=float("nan")), sc.E_PARAM)])
def test_weights_are_checked(kw, want):
    assert _weigh(**kw) == want


@pytest.mark.parametrize("kw,want", [
    (dict(w=None), sc.E_NULL), (dict(ln=None), sc.E_NULL), (dict(keep=None), sc.E_NULL), (dict(kept=None), sc.E_NULL), (dict(budget=0), sc.E_PARAM),
    (dict(sinks=-1), sc.E_PARAM), (dict(recent=-1), sc.E_PARAM), (dict(sinks=5, recent=4), sc.E_PARAM), (dict(heads=0), sc.E_SHAPE),
    (dict(heads=257), sc.E_SHAPE), (dict(n=-1), sc.E_SHAPE), (dict(n=1 << 15), sc.E_SHAPE), (dict(ws=0), sc.E_SHAPE), (dict(w=A + 2), sc.E_ALIGN),
    (dict(kept=A + 2), sc.E_ALIGN), (dict(sinks=2 ** 31 - 1, recent=2 ** 31 - 1), sc.E_PARAM)])
def test_the_selection_is_checked(kw, want):
    assert _select(**kw) == want


@pytest.mark.parametrize("kw,want", [
    (dict(keep=None), sc.E_NULL), (dict(kept=None), sc.E_NULL), (dict(w_in=A, ws=4), sc.E_NULL), (dict(w_out=A, ws=4), sc.E_NULL),
    (dict(w_in=A, w_out=A), sc.E_SHAPE), (dict(kh=3), sc.E_SHAPE), (dict(kw=-1), sc.E_SHAPE), (dict(to=_seqs(n_seqs=3)), sc.E_SHAPE),
    (dict(to=_seqs()), sc.E_PARAM), (dict(to=_seqs(table_width=0)), sc.E_SHAPE), (dict(keep=A + 2), sc.E_ALIGN), (dict(first=A + 2), sc.E_ALIGN),
    (dict(seqs=_seqs(n_seqs=1 << 15)), sc.E_SHAPE)])
def test_moving_is_checked(kw, want):
    assert _keep(**kw) == want


@pytest.mark.parametrize("call", OVER_PAGES + [_select])
def test_sound_arguments_still_need_a_context(call):
    assert call() == sc.E_NULL


def test_more_sound_arguments():
    assert _write(q=None, g=0, qs=0, qo=None, qos=0) == sc.E_NULL            # no q: nothing of it is looked at
    assert _write(qo=2 * A, qos=520) == sc.E_NULL
    assert _keep(kh=1, to=_seqs(d_table=2 * A), w_in=A, w_out=A, ws=4) == sc.E_NULL
    assert _weigh(w_in=None) == sc.E_NULL


# ---- the binding: the current device is taken to be -1, which is where torch says that host tensors are

CTX = SimpleNamespace(handle=None)
HEADS, D, ROWS, G, WS = 2, 64, 5, 3, 20


@pytest.fixture
def host(monkeypatch):
    monkeypatch.setattr(sc, "_here", lambda: (-1, None))


def _z(*shape, dtype=torch.float32):
    return torch.zeros(shape, dtype=dtype)


def _arguments():
    """Every call of the binding with tensors that fit, by the names of those."""
    pages = lambda: sc.Pages(d_data=A, d_scale=A, n_pages=4, page=16, heads=HEADS, head_dim=D, format=sc.INT8, dtype=sc.F16)
    seqs = lambda: _seqs(n_rows=ROWS)
    rows = lambda n: _z(ROWS, n * D, dtype=torch.float16)
    i32 = torch.int32
    q = HEADS * G
    return [
        (lambda t, **kw: sc.salicache_paged_write_rotary(CTX, pages(), seqs(), sc.Rotary([0.1] * 8, [0] * 8, 2), t["pos"], t["q"], q * D, G, t["q_out"], q * D,
                                                         t["k"], t["v"], HEADS * D, HEADS * D, **kw),
         dict(pos=_z(ROWS, 2, dtype=i32), q=rows(q), q_out=rows(q), k=rows(HEADS), v=rows(HEADS))),
        (lambda t, **kw: sc.salicache_paged_attend_tree(CTX, pages(), seqs(), t["tree"], 2, t["q"], q * D, G, 0.1, 0, 0, t["out"], q * D, t["lse"], t["work"], 64,
                                                        **kw),
         dict(tree=_z(ROWS, 2, dtype=torch.int64), q=rows(q), out=rows(q), lse=_z(ROWS, q), work=_z(64, dtype=torch.uint8))),
        (lambda t, **kw: sc.salicache_paged_weigh(CTX, pages(), seqs(), t["q"], q * D, G, 0.1, t["lse"], 1.0, t["w_in"], t["w_out"], WS, t["work"], 64, **kw),
         dict(q=rows(q), lse=_z(ROWS, q), w_in=_z(2, HEADS, WS), w_out=_z(2, HEADS, WS), work=_z(64, dtype=torch.uint8))),
        (lambda t, **kw: sc.salicache_select_heavy(CTX, t["w"], WS, HEADS, 2, t["len"], 8, 1, 1, t["keep"], t["kept"], **kw),
         dict(w=_z(2, HEADS, WS), len=_z(2, dtype=i32), keep=_z(2, HEADS, 8, dtype=i32), kept=_z(2, dtype=i32))),
        (lambda t, **kw: sc.salicache_paged_keep(CTX, pages(), seqs(), t["keep"], HEADS, 8, t["first"], t["kept"], None, t["w_in"], t["w_out"], WS, **kw),
         dict(keep=_z(2, HEADS, 8, dtype=i32), first=_z(2, dtype=i32), kept=_z(2, dtype=i32), w_in=_z(2, HEADS, WS), w_out=_z(2, HEADS, WS))),
    ]


@pytest.mark.parametrize("which", range(5))
def test_the_binding_compares_types_sizes_and_devices(host, which):
    call, tensors = _arguments()[which]
    with pytest.raises(sc.SalicacheError) as e:
        call(tensors)
    assert e.value.status == sc.E_NULL           # all of it fits: the library is asked, and misses the context
    for name, t in tensors.items():
        if name != "work":
            with pytest.raises(ValueError, match="type"):
                call({**tensors, name: t.to(torch.float64)})
        with pytest.raises(ValueError, match="memory"):
            call({**tensors, name: t.flatten()[:-1].clone()})
        with pytest.raises(ValueError, match="cuda"):
            call({**tensors, name: SimpleNamespace(get_device=lambda: 1, device="cuda:1")})
    with pytest.raises(ValueError, match="cuda:1"):
        call(tensors, stream=SimpleNamespace(device_index=1, cuda_stream=0))


def test_the_rotary_struct():
    r = sc.Rotary([1.0, 0.5], [0, 1], 2, sc.NEIGHBOURS)
    assert (r.pairs, r.n_axes, r.pairing, r.freq[1], r.axis[1]) == (2, 2, 1, 0.5, 1)
    assert C.sizeof(sc.Rotary) == 592
    for bad in (([1.0] * 65,), ([1.0], [0, 1]), ([1.0], [256]), ([1.0], [-1])):
        with pytest.raises(ValueError):
            sc.Rotary(*bad)
