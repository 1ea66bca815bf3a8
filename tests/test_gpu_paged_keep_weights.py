"""GPU tests of the weights that move along with kept rows: a weight moves where its row does, and stays where that stays.  Whole
rows of bytes and copies of numbers, compared for equality."""
import numpy as np
import pytest

import paged_util as pu
from paper_2602_14236_b200 import binding as sc
from test_gpu_paged_keep import _i32, _raw, _t, moved

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    return sc.Context(sc.salicache_default_params(max_batch=1, chunk_frames=1, L=1))


def weights(w, wt, behind, table_to, keep, first, kept):
    """The weights after the move, from those before; `behind`: what the output held."""
    out, S = behind.copy(), wt.shape[2]
    for b in range(len(w.lens)):
        for h in range(w.heads):
            row = keep[b, h if keep.shape[1] > 1 else 0]
            for k in range(min(max(kept[b], 0), keep.shape[2])):
                e, t = row[k], (first[b] if first is not None else 0) + k
                if not 0 <= e < w.lens[b] or e >= S or t >= S:
                    continue
                src = w.table[b, e // w.page]
                dst = table_to[b, t // w.page] if t < table_to.shape[1] * w.page else -1
                if 0 <= src < w.n_pages and 0 <= dst < w.n_pages:
                    out[b, h, t] = wt[b, h, e]
    return out


def run(ctx, w, keep, first, kept, table_to, S, bad):
    """table_to None: in place."""
    import torch
    pages, seqs = w.device()
    to = None if table_to is None else sc.Seqs(seqs.row_start, seqs.length, _i32(table_to), 0)
    raws = [_raw(pages.data), _raw(pages.scale)]
    to_table = w.table if table_to is None else table_to
    want, missed = moved(w, raws, to_table, keep, first, kept)
    assert missed == bad
    wt = np.random.default_rng(2).random((len(w.lens), w.heads, S)).astype(np.float32)
    w_in = torch.from_numpy(wt).cuda()
    w_out = w_in if to is None else torch.full_like(w_in, 7.0)
    want_w = weights(w, wt, w_out.cpu().numpy(), to_table, keep, first, kept)
    sc.salicache_paged_keep(ctx, pages.c, seqs.c, _i32(keep), keep.shape[1], keep.shape[2], None if first is None else _i32(first), _i32(np.array(kept)),
                            None if to is None else to.c, w_in, w_out, S)
    assert sc.salicache_poll_status(ctx) == (sc.E_CAPACITY if bad else 0)
    assert np.array_equal(_raw(pages.data), want[0]) and (want[1] is None or np.array_equal(_raw(pages.scale), want[1]))
    assert np.array_equal(w_out.cpu().numpy(), want_w)


@pytest.mark.parametrize("fmt", ["fp16", "int8"])
@pytest.mark.parametrize("S", [110, 45])
@pytest.mark.parametrize("first", [None, [5, 30], [2 ** 31 - 1, 16]])
def test_missing_pages_elsewhere(ctx, fmt, S, first):
    w = pu.World(1, fmt, _t("f16"), 2, 128, 16, [100, 50], [0, 0], spare=12)
    free = np.setdiff1d(np.arange(w.n_pages), np.concatenate([w.table[0, :7], w.table[1, :4]]))
    keep = np.array([[[0, 3, 99, 40, 7, 100, -1, 2 ** 31 - 1] + list(range(50, 74))], [[-5, 49, 50, 17, 18, 19, 20, 21] + list(range(22, 46))]])
    w.table[0, 0] = -1                                   # positions 0 .. 15 are gone
    run(ctx, w, keep, None if first is None else np.array(first), [32, 32], np.array([[free[0], free[1]], [free[2], w.n_pages]]), S, True)


@pytest.mark.parametrize("fmt", ["fp16", "int4"])
@pytest.mark.parametrize("per_head", [True, False])
@pytest.mark.parametrize("gone", [[(0, 2)], [(0, 0), (1, 1)], [(0, 4), (0, 5), (1, 2)]])
def test_missing_pages_in_place(ctx, fmt, per_head, gone):
    """A page that is none is both where rows come from and where they go."""
    w = pu.World(1, fmt, _t("bf16"), 3, 64, 16, [100, 50], [0, 0])
    rng = np.random.default_rng(3)
    keep = np.full((2, 3 if per_head else 1, 60), -1)
    kept = [60, 30]
    for b, n in enumerate([100, 50]):
        for h in range(keep.shape[1]):
            keep[b, h, :kept[b]] = np.sort(rng.choice(n, kept[b], replace=False))
    for i, (b, p) in enumerate(gone):
        w.table[b, p] = -1 if i % 2 else w.n_pages
    run(ctx, w, keep, None, kept, None, 100, True)


@pytest.mark.parametrize("where", ["elsewhere", "in place"])
def test_many_tiles_of_weights(ctx, where):
    """Lists longer than what a block's threads hold at a time; in place every weight moves by one."""
    n = 9500
    w = pu.World(1, "int4", _t("f16"), 2, 64, 128, [n, 4200], [0, 0], spare=120)
    keep = np.full((2, 1, n - 1), -1)
    keep[0, 0], keep[1, 0, :4199] = np.arange(1, n), np.arange(1, 4200)
    table_to = None
    if where == "elsewhere":
        free = np.setdiff1d(np.arange(w.n_pages), w.table[w.table < w.n_pages])
        table_to = np.full((2, 75), -1)
        table_to[0], table_to[1, :33] = free[:75], free[75:108]
    run(ctx, w, keep, None, [n - 1, 4199], table_to, n, False)
