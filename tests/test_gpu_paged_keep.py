"""GPU tests of what a budget keeps and of moving it together: whole numbers and bytes, compared for equality."""
import numpy as np
import pytest

import paged_util as pu
from paper_2602_14236_b200 import binding as sc

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    return sc.Context(sc.salicache_default_params(max_batch=1, chunk_frames=1, L=1))


def _t(name):
    import torch
    return {"f16": torch.float16, "bf16": torch.bfloat16}[name]


def _i32(a):
    import torch
    return torch.from_numpy(np.ascontiguousarray(a)).to(torch.int32).cuda()


def select(weight, lens, budget, sinks, recent):
    """numpy: lists padded with -1."""
    B, H, _ = weight.shape
    keep = np.full((B, H, budget), -1, np.int64)
    for b, n in enumerate(lens):
        for h in range(H):
            if n <= budget:
                keep[b, h, :n] = np.arange(n)
                continue
            p = np.arange(sinks, n - recent)
            x = weight[b, h, p].astype(np.float64)
            nan = np.isnan(x)
            order = np.lexsort((p, -np.where(nan, 0.0, x), nan))          # numbers first, heaviest first, then the lowest position
            mid = np.sort(p[order[:budget - sinks - recent]])
            keep[b, h] = np.concatenate([np.arange(sinks), mid, np.arange(n - recent, n)])
    return keep


def run_select(ctx, weight, lens, budget, sinks, recent, status=0, clip=None):
    import torch
    B, H, S = weight.shape
    keep = torch.full((B, H, budget), 7, dtype=torch.int32, device="cuda")
    kept = torch.full((B,), 7, dtype=torch.int32, device="cuda")
    sc.salicache_select_heavy(ctx, torch.from_numpy(weight).cuda(), S, H, B, _i32(np.array(lens)), budget, sinks, recent, keep, kept)
    assert sc.salicache_poll_status(ctx) == status
    lens = [max(0, min(n, S)) for n in lens]
    assert kept.tolist() == [min(n, budget) for n in lens]
    assert np.array_equal(keep.cpu().numpy(), select(weight, lens, budget, sinks, recent))
    return keep, kept


def _weights(kind, shape, seed=0):
    rng = np.random.default_rng(seed)
    w = rng.random(shape) ** 4 * 100
    if kind == "ties":
        w = rng.integers(0, 3, shape).astype(float)
    if kind == "one":
        w = np.full(shape, 0.25)
    if kind == "odd":
        w = rng.standard_normal(shape)
        w = np.where(rng.random(shape) < 0.3, rng.choice([np.nan, np.inf, -np.inf, 0.0, -0.0, 1e-42, -1e-42, 3.4e38], shape), w)
    if kind == "near":                                   # neighbours in binary32
        w = 1.0 + rng.integers(0, 5, shape) * 2.0 ** -23
    return w.astype(np.float32)


@pytest.mark.parametrize("kind", ["any", "ties", "one", "odd", "near"])
@pytest.mark.parametrize("lens,budget,sinks,recent", [
    ([0, 1, 7, 8, 9, 300], 8, 2, 3), ([1000, 31, 997], 100, 0, 0), ([1000, 31, 997], 100, 50, 50), ([500], 1, 0, 0), ([500], 1, 1, 0), ([500], 1, 0, 1),
    ([5000, 4097], 4096, 4, 64), ([4096], 4096, 4, 64), ([70000], 333, 4, 100), ([70001, 65], 60000, 0, 1),
])
def test_selection(ctx, kind, lens, budget, sinks, recent):
    run_select(ctx, _weights(kind, (len(lens), 2, max(lens) + 3)), lens, budget, sinks, recent)


def test_selection_of_many_and_of_lengths_past_the_array(ctx):
    run_select(ctx, _weights("ties", (300, 7, 90)), [i % 91 for i in range(300)], 40, 3, 5)
    run_select(ctx, _weights("any", (3, 2, 50)), [60, 50, -4], 20, 2, 2, status=sc.E_CAPACITY)


def test_a_captured_selection(ctx):
    import torch
    w = torch.zeros((2, 3, 900), device="cuda")
    ln, keep, kept = _i32(np.zeros(2)), torch.zeros((2, 3, 64), dtype=torch.int32, device="cuda"), torch.zeros(2, dtype=torch.int32, device="cuda")
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            sc.salicache_select_heavy(ctx, w, 900, 3, 2, ln, 64, 4, 10, keep, kept)
    for seed, lens in enumerate(([900, 40], [65, 899])):
        x = _weights("any", (2, 3, 900), seed)
        w.copy_(torch.from_numpy(x))
        ln.copy_(torch.tensor(lens))
        g.replay()
        torch.cuda.synchronize()
        assert np.array_equal(keep.cpu().numpy(), select(x, lens, 64, 4, 10)) and kept.tolist() == [min(n, 64) for n in lens]


# ---- moving

def _raw(x):
    import torch
    return x.contiguous().view(torch.uint8).cpu().numpy().reshape(tuple(x.shape[:4]) + (-1,)) if x is not None else None


def moved(w, raws, table_to, keep, first, kept, missing=()):
    """The pages' bytes after the move, entry by entry from the bytes before."""
    out = [None if r is None else r.copy() for r in raws]
    bad = False
    for b in range(len(w.lens)):
        for h in range(w.heads):
            row = keep[b, h if keep.shape[1] > 1 else 0]
            for k in range(min(max(kept[b], 0), keep.shape[2])):
                e, t = row[k], (first[b] if first is not None else 0) + k
                src = w.table[b, e // w.page] if 0 <= e < w.lens[b] else -1
                dst = table_to[b, t // w.page] if t < table_to.shape[1] * w.page else -1
                if not (0 <= src < w.n_pages and 0 <= dst < w.n_pages):
                    bad = True
                    continue
                for o, r in zip(out, raws):
                    if r is not None:
                        o[dst, :, h, t % w.page] = r[src, :, h, e % w.page]
    return out, bad


def _lists(rng, lens, heads, width, per_head=True, first=None):
    """Ascending lists with entry k at least first + k, padded with -1; and their lengths."""
    keep = np.full((len(lens), heads if per_head else 1, width), -1, np.int64)
    kept = []
    for b, n in enumerate(lens):
        f = 0 if first is None else first[b]
        m = int(min(width, max(n - f, 0) * 2 // 3))
        kept.append(m)
        for h in range(keep.shape[1]):
            keep[b, h, :m] = np.sort(rng.choice(np.arange(f, n), m, replace=False))
    return keep, np.array(kept)


CASES = [
    (2, 128, 16, [130, 9, 0, 300], 100), (5, 64, 32, [700, 40], 450), (1, 128, 128, [300], 300), (3, 64, 64, [17, 1000, 129], 600), (8, 128, 64, [500], 129),
]


@pytest.mark.parametrize("fmt", ["fp16", "int8", "int4"])
@pytest.mark.parametrize("case", range(len(CASES)))
@pytest.mark.parametrize("where", ["elsewhere", "in place"])
@pytest.mark.parametrize("per_head", [True, False])
@pytest.mark.parametrize("weights", [True, False])
def test_moving(ctx, fmt, case, where, per_head, weights):
    import torch
    heads, D, page, lens, width = CASES[case]
    rng = np.random.default_rng(case)
    counts = [-(-n // page) for n in lens]
    w = pu.World(case, fmt, _t("bf16" if case % 2 else "f16"), heads, D, page, lens, [0] * len(lens), spare=sum(counts) + 2)
    pages, seqs = w.device()
    first = np.array([min(n, 5 * b) for b, n in enumerate(lens)]) if case % 2 else None
    keep, kept = _lists(rng, lens, heads, width, per_head, first)
    to, table_to = None, w.table
    if where == "elsewhere":
        free = np.setdiff1d(np.arange(w.n_pages), np.concatenate([w.table[b, :c] for b, c in enumerate(counts)]))
        table_to = np.full((len(lens), w.width + 1), -1, np.int64)
        at = 0
        for b, c in enumerate(counts):
            table_to[b, :c] = free[at:at + c]
            at += c
        to = sc.Seqs(seqs.row_start, seqs.length, _i32(table_to), 0)
    raws = [_raw(pages.data), _raw(pages.scale)]
    want, bad = moved(w, raws, table_to, keep, first, kept)
    assert not bad
    S = max(lens) + 3
    wt = rng.random((len(lens), heads, S)).astype(np.float32)
    w_in = torch.from_numpy(wt).cuda()
    w_out = w_in if where == "in place" else torch.full_like(w_in, 7.0)
    want_w = w_out.cpu().numpy().copy()
    for b in range(len(lens)):
        for h in range(heads):
            f = 0 if first is None else first[b]
            want_w[b, h, f:f + kept[b]] = wt[b, h, keep[b, h if per_head else 0, :kept[b]]]
    sc.salicache_paged_keep(ctx, pages.c, seqs.c, _i32(keep), keep.shape[1], width, None if first is None else _i32(first), _i32(kept),
                            None if to is None else to.c, w_in if weights else None, w_out if weights else None, S)
    assert sc.salicache_poll_status(ctx) == 0
    assert np.array_equal(_raw(pages.data), want[0])
    assert want[1] is None or np.array_equal(_raw(pages.scale), want[1])
    if weights:
        assert np.array_equal(w_out.cpu().numpy(), want_w)


@pytest.mark.parametrize("fmt", ["fp16", "int4"])
@pytest.mark.parametrize("kept", ["all but the first", "all", "all but the last", "the last"])
def test_long_lists_in_place(ctx, fmt, kept):
    """Every row moves by one, through many tiles of a list, or none does."""
    import torch
    n = 3000
    w = pu.World(1, fmt, _t("f16"), 3, 64, 16, [n, n], [0, 0])
    pages, seqs = w.device()
    keep = {"all but the first": np.arange(1, n), "all": np.arange(n), "all but the last": np.arange(n - 1), "the last": np.array([n - 1])}[kept]
    keep = np.broadcast_to(keep, (2, 1, keep.size))
    raws = [_raw(pages.data), _raw(pages.scale)]
    want, _ = moved(w, raws, w.table, keep, None, [keep.shape[2], 0])
    wt = torch.rand((2, 3, n), device="cuda")
    ww = wt.clone()
    sc.salicache_paged_keep(ctx, pages.c, seqs.c, _i32(keep), 1, keep.shape[2], None, _i32(np.array([keep.shape[2] + 9, -3])), None, ww, ww, n)
    assert sc.salicache_poll_status(ctx) == 0
    assert np.array_equal(_raw(pages.data), want[0]) and (want[1] is None or np.array_equal(_raw(pages.scale), want[1]))
    wt[0, :, :keep.shape[2]] = wt[0][:, torch.from_numpy(keep[0, 0].copy()).cuda()]
    assert torch.equal(ww, wt)


def test_entries_and_pages_that_are_none(ctx):
    w = pu.World(1, "int8", _t("f16"), 2, 128, 16, [100, 50], [0, 0], spare=12)
    free = np.setdiff1d(np.arange(w.n_pages), np.concatenate([w.table[0, :7], w.table[1, :4]]))
    keep = np.array([[[0, 3, 99, 40, 7, 100, -1, 2 ** 31 - 1] + list(range(50, 74))], [[-5, 49, 50, 17, 18, 19, 20, 21] + list(range(22, 46))]])
    w.table[0, 0] = -1                                   # positions 0 .. 15 are gone
    table_to = np.array([[free[0], free[1]], [free[2], w.n_pages]])
    pages, seqs = w.device()
    to = sc.Seqs(seqs.row_start, seqs.length, _i32(table_to), 0)
    for first in (None, np.array([5, 30]), np.array([2 ** 31 - 1, 16])):
        raws = [_raw(pages.data), _raw(pages.scale)]
        want, bad = moved(w, raws, table_to, keep, first, [32, 32])
        assert bad
        sc.salicache_paged_keep(ctx, pages.c, seqs.c, _i32(keep), 1, 32, None if first is None else _i32(first), _i32(np.array([32, 32])), to.c)
        assert sc.salicache_poll_status(ctx) == sc.E_CAPACITY
        assert np.array_equal(_raw(pages.data), want[0]) and np.array_equal(_raw(pages.scale), want[1])
