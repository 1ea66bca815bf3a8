"""GPU tests of the calls for trees, weights, eviction and positions where they can go wrong: waits given up, what lies in rows and
pages that nobody owns, byte offsets past 2^32, other streams, graphs side by side."""
import numpy as np
import pytest

import paged_util as pu
import test_gpu_paged_tree as tr
import test_gpu_paged_weigh as wg
from paper_2602_14236_b200 import binding as sc

pytestmark = pytest.mark.gpu

ORDINARY = 1 << 24


@pytest.fixture()
def ctx():
    return sc.Context(sc.salicache_default_params(max_batch=1, chunk_frames=1, L=1))


def _t(name):
    import torch
    return {"f16": torch.float16, "bf16": torch.bfloat16}[name]


# ---- waits inside the kernels that are given up

class Weigh:
    def __init__(self, ctx, fmt, dt, heads, G, D, page, lens, news):
        import torch
        self.ctx, self.G = ctx, G
        self.w = w = pu.World(3, fmt, _t(dt), heads, D, page, lens, news)
        self.pages, self.seqs = w.device()
        self.q = torch.from_numpy(np.random.default_rng(4).standard_normal((w.rows, heads * G * D))).to(w.t).cuda()
        qn = self.q.double().cpu().numpy().reshape(w.rows, -1, D)
        self.lse = wg.softmax_sums(w, qn, G, D ** -0.5)
        self.had = np.random.default_rng(5).random((len(lens), heads, max(lens))).astype(np.float32)
        self.want, self.tol = wg.expect(w, qn, self.lse, G, D ** -0.5, 0.5, self.had.astype(np.float64), max(lens))
        self.work = torch.full((sc.salicache_paged_work_bytes(ctx, self.pages.c, G),), 255, dtype=torch.uint8, device="cuda")

    def run(self, limit):
        import torch
        w = self.w
        out = torch.full(self.had.shape, 7.0, device="cuda")
        sc.salicache_paged_wait_limit(self.ctx, limit)
        sc.salicache_paged_weigh(self.ctx, self.pages.c, self.seqs.c, self.q, self.q.shape[1], self.G, w.D ** -0.5, torch.from_numpy(self.lse).float().cuda(),
                                 0.5, torch.from_numpy(self.had).cuda(), out, max(w.lens), self.work, self.work.numel())
        status = sc.salicache_poll_status(self.ctx)
        torch.cuda.synchronize()
        got, held = out.double().cpu().numpy(), ~np.isnan(self.want)
        assert (got[~held] == 7).all()
        if status == 0:
            pu.check(got[held], self.want[held], self.tol[held], "weight")
        return status


class Tree:
    def __init__(self, ctx, fmt, dt, heads, G, D, page, lens, news):
        import torch
        self.ctx, self.G = ctx, G
        self.w = w = pu.World(3, fmt, _t(dt), heads, D, page, lens, news)
        self.pages, self.seqs = w.device()
        self.q = torch.from_numpy(np.random.default_rng(4).standard_normal((w.rows, heads * G * D))).to(w.t).cuda()
        mats = tr.trees(np.random.default_rng(6), news, "branch")
        self.bits = torch.from_numpy(tr.words(mats, 1, w.rows).view(np.int64)).cuda()
        self.want = tr.expect(w, self.q.double().cpu().numpy().reshape(w.rows, -1, D), G, D ** -0.5, mats, 1, 0, 0)
        self.work = torch.full((sc.salicache_paged_work_bytes(ctx, self.pages.c, G),), 255, dtype=torch.uint8, device="cuda")

    def run(self, limit):
        import torch
        w = self.w
        out, lse = torch.full_like(self.q, 7.0), torch.full((w.rows, w.heads * self.G), 7.0, device="cuda")
        sc.salicache_paged_wait_limit(self.ctx, limit)
        sc.salicache_paged_attend_tree(self.ctx, self.pages.c, self.seqs.c, self.bits, 1, self.q, self.q.shape[1], self.G, w.D ** -0.5, 0, 0, out,
                                       self.q.shape[1], lse, self.work, self.work.numel())
        status = sc.salicache_poll_status(self.ctx)
        torch.cuda.synchronize()
        if status == 0:
            o, l, tol, ltol = self.want
            pu.check(out.double().cpu().numpy().reshape(o.shape), o, tol, "out")
            pu.check(lse.double().cpu().numpy(), l, ltol, "lse")
        return status


CALLS = [
    (Weigh, "fp16", "f16", 2, 4, 128, 64, [3000, 700, 0, 129], [1, 1, 0, 1]),        # a few rows per sequence
    (Weigh, "int8", "bf16", 2, 4, 64, 16, [3000, 700, 0, 129], [1, 1, 0, 1]),
    (Weigh, "int4", "f16", 2, 4, 128, 32, [3000, 700, 5], [4, 3, 4]),
    (Weigh, "fp16", "bf16", 2, 2, 128, 128, [2500, 300], [300, 300]),                 # many
    (Weigh, "int8", "f16", 2, 3, 64, 16, [2500, 300], [300, 300]),
    (Weigh, "int4", "bf16", 1, 4, 128, 64, [2500, 300], [200, 300]),
    (Tree, "fp16", "f16", 2, 4, 128, 64, [3000, 700, 0, 129], [2, 1, 0, 1]),
    (Tree, "int8", "bf16", 2, 4, 128, 32, [2500, 300], [60, 64]),
]


@pytest.mark.parametrize("args", CALLS, ids=lambda a: f"{a[0].__name__}-{a[1]}-{a[2]}-{sum(a[8])}")
def test_waits_given_up(ctx, args):
    c = args[0](ctx, *args[1:])
    for _ in range(2):
        assert c.run(0) == sc.E_CUDA
        assert c.run(ORDINARY) == 0
    for limit in (1, 2, 3, 5, 8, 13, 21, 55, 200):
        assert c.run(limit) in (0, sc.E_CUDA)
    assert c.run(ORDINARY) == 0


# ---- what nobody owns

@pytest.mark.parametrize("news", [[1, 1, 1], [70, 33, 150]])
@pytest.mark.parametrize("fmt", ["fp16", "int4"])
def test_rows_of_nobody_may_hold_anything(ctx, news, fmt):
    """NaN and infinities in q behind the last sequence and before the first, next to rows that a block takes with them."""
    import torch
    lens, G, D = [700, 33, 150], 4, 128
    w = pu.World(3, fmt, _t("bf16"), 2, D, 32, lens, news)
    pages, _ = w.device()
    lead, tail, Hq = 5, 9, 8
    i32 = lambda a: torch.from_numpy(np.ascontiguousarray(a)).to(torch.int32).cuda()
    R = lead + w.rows + tail
    seqs = sc.Seqs(i32(w.start + lead), i32(np.array(lens)), i32(w.table), R)
    q = torch.from_numpy(np.random.default_rng(4).standard_normal((R, Hq * D))).to(w.t)
    q[:lead], q[lead + w.rows:] = float("nan"), float("inf")
    qn = q[lead:lead + w.rows].double().numpy().reshape(w.rows, Hq, D)
    lse = wg.softmax_sums(w, qn, G, D ** -0.5)
    full = np.full((R, Hq), np.nan)
    full[lead:lead + w.rows] = lse
    out = torch.full((3, 2, 700), 7.0, device="cuda")
    wk = torch.empty(sc.salicache_paged_work_bytes(ctx, pages.c, G), dtype=torch.uint8, device="cuda")
    sc.salicache_paged_weigh(ctx, pages.c, seqs.c, q.cuda(), Hq * D, G, D ** -0.5, torch.from_numpy(full).float().cuda(), 1.0, None, out, 700, wk, wk.numel())
    assert sc.salicache_poll_status(ctx) == 0
    want, tol = wg.expect(w, qn, lse, G, D ** -0.5, 1.0, None, 700)
    got, held = out.double().cpu().numpy(), ~np.isnan(want)
    pu.check(got[held], want[held], tol[held], "weight")
    # the tree's rows likewise
    mats = tr.trees(np.random.default_rng(2), news, "branch")
    bits = np.full((R, 3), 2 ** 63 + 12345, np.uint64)
    bits[lead:lead + w.rows] = tr.words(mats, 3, w.rows)
    o, l = torch.full((R, Hq * D), 7.0, dtype=w.t, device="cuda"), torch.full((R, Hq), 7.0, device="cuda")
    sc.salicache_paged_attend_tree(ctx, pages.c, seqs.c, torch.from_numpy(bits.view(np.int64)).cuda(), 3, q.cuda(), Hq * D, G, D ** -0.5, 0, 0, o, Hq * D, l,
                                   wk, wk.numel())
    assert sc.salicache_poll_status(ctx) == 0
    eo, el, etol, eltol = tr.expect(w, qn, G, D ** -0.5, mats, 3, 0, 0)
    pu.check(o[lead:lead + w.rows].double().cpu().numpy().reshape(eo.shape), eo, etol, "out")
    pu.check(l[lead:lead + w.rows].double().cpu().numpy(), el, eltol, "lse")
    assert (o[:lead] == 7).all() and (o[lead + w.rows:] == 7).all() and (l[:lead] == 7).all() and (l[lead + w.rows:] == 7).all()


@pytest.mark.parametrize("news", [[1, 2], [40, 64]])
def test_a_tree_under_a_window_reads_nothing_behind_it(ctx, news):
    """Pages that slid out of the window: their table entries are stale, what they hold is NaN."""
    import torch
    lens, G, D, window, sinks = [900, 500], 4, 128, 100, 3
    w = pu.World(3, "fp16", _t("f16"), 2, D, 16, lens, news)
    pages, seqs = w.device()
    table = w.table.copy()
    for b in range(2):
        before = lens[b] - news[b]
        for p in range(sinks, before - window + 1):
            pages.data[w.table[b, p // 16], :, :, p % 16] = float("nan")
        for i in range(1, (before - window + 1) // 16):
            table[b, i] = -7 if i % 2 else 2 ** 30
    seqs = sc.Seqs(seqs.row_start, seqs.length, torch.from_numpy(table).to(torch.int32).cuda(), w.rows)
    Hq = 8
    q = torch.from_numpy(np.random.default_rng(4).standard_normal((w.rows, Hq * D))).to(w.t)
    mats = tr.trees(np.random.default_rng(2), news, "branch")
    out, lse = torch.empty((w.rows, Hq * D), dtype=w.t, device="cuda"), torch.empty((w.rows, Hq), device="cuda")
    wk = torch.empty(sc.salicache_paged_work_bytes(ctx, pages.c, G), dtype=torch.uint8, device="cuda")
    sc.salicache_paged_attend_tree(ctx, pages.c, seqs.c, torch.from_numpy(tr.words(mats, 1, w.rows).view(np.int64)).cuda(), 1, q.cuda(), Hq * D, G, D ** -0.5,
                                   window, sinks, out, Hq * D, lse, wk, wk.numel())
    assert sc.salicache_poll_status(ctx) == 0
    o, l, tol, ltol = tr.expect(w, q.double().numpy().reshape(w.rows, Hq, D), G, D ** -0.5, mats, 1, window, sinks)
    pu.check(out.double().cpu().numpy().reshape(o.shape), o, tol, "out")
    pu.check(lse.double().cpu().numpy(), l, ltol, "lse")


@pytest.mark.parametrize("news", [[1, 1], [100, 64]])
@pytest.mark.parametrize("fmt", ["fp16", "int8"])
def test_rows_that_see_nothing_weigh_nothing(ctx, news, fmt):
    """A row whose logarithm is minus infinity, among others and as all there are; and K that is no number where nobody sees it."""
    import torch
    lens, G, D = [400, 64], 2, 64
    w = pu.World(3, fmt, _t("f16"), 2, D, 16, lens, news)
    pages, seqs = w.device()
    q = torch.from_numpy(np.random.default_rng(4).standard_normal((w.rows, 4 * D))).to(w.t)
    qn = q.double().numpy().reshape(w.rows, 4, D)
    wk = torch.empty(sc.salicache_paged_work_bytes(ctx, pages.c, G), dtype=torch.uint8, device="cuda")
    lse = wg.softmax_sums(w, qn, G, D ** -0.5)
    some = lse.copy()
    some[np.random.default_rng(5).random(some.shape) < 0.3] = -np.inf
    for case in (some, np.full_like(lse, -np.inf)):
        out = torch.full((2, 2, 400), 7.0, device="cuda")
        sc.salicache_paged_weigh(ctx, pages.c, seqs.c, q.cuda(), 4 * D, G, D ** -0.5, torch.from_numpy(case).float().cuda(), 1.0, None, out, 400, wk, wk.numel())
        assert sc.salicache_poll_status(ctx) == 0
        want, tol = wg.expect(w, qn, case, G, D ** -0.5, 1.0, None, 400)
        got, held = out.double().cpu().numpy(), ~np.isnan(want)
        pu.check(got[held], want[held], tol[held], "weight")


@pytest.mark.parametrize("fmt,news", [("fp16", [1, 1]), ("fp16", [70, 64]), ("int8", [3, 4]), ("int8", [70, 64])])
def test_numbers_that_are_none_and_sums_that_overflow(ctx, fmt, news):
    """A row of q that is no number makes none of all that it sees, whichever row it is, and touches nothing else; logarithms far
    below the scores give infinities, whichever column they come from."""
    import torch
    lens, G, D = [300, 200], 2, 64
    w = pu.World(3, fmt, _t("f16"), 1, D, 16, lens, news)
    pages, seqs = w.device()
    clean = torch.from_numpy(np.random.default_rng(4).standard_normal((w.rows, G * D))).to(w.t)
    qn = clean.double().numpy().reshape(w.rows, G, D)
    lse = wg.softmax_sums(w, qn, G, D ** -0.5)
    want, tol = wg.expect(w, qn, lse, G, D ** -0.5, 1.0, None, 300)
    wk = torch.empty(sc.salicache_paged_work_bytes(ctx, pages.c, G), dtype=torch.uint8, device="cuda")

    def weigh(q, sums):
        out = torch.full((2, 1, 300), 7.0, device="cuda")
        sc.salicache_paged_weigh(ctx, pages.c, seqs.c, q.cuda(), G * D, G, D ** -0.5, torch.from_numpy(sums).float().cuda(), 1.0, None, out, 300, wk, wk.numel())
        assert sc.salicache_poll_status(ctx) == 0
        return out.double().cpu().numpy()

    for r in range(0, news[0], max(1, news[0] // 17)):
        q = clean.clone()
        q[r, D + 3] = float("nan")
        got = weigh(q, lse)
        sees = lens[0] - news[0] + r + 1
        assert np.isnan(got[0, 0, :sees]).all()
        pu.check(got[0, 0, sees:300], want[0, 0, sees:300], tol[0, 0, sees:300], "weight")
        pu.check(got[1, 0, :200], want[1, 0, :200], tol[1, 0, :200], "weight")
    for r in range(0, news[0], max(1, news[0] // 17)):
        far = lse.copy()
        far[r, 1] = -300.0
        got = weigh(clean, far)
        sees = lens[0] - news[0] + r + 1
        assert np.isposinf(got[0, 0, :sees]).all()
        pu.check(got[0, 0, sees:300], want[0, 0, sees:300], tol[0, 0, sees:300], "weight")


# ---- byte offsets past 2^32

def test_a_cache_beyond_four_gigabytes(ctx):
    """Pages whose bytes lie on both sides of 2^32 and 2^33: written with positions, weighed, gathered, read."""
    import torch
    t, heads, D, page, G = _t("bf16"), 8, 128, 128, 2
    n_pages = 20000                                      # 524,288 bytes each
    pages = sc.PageSet(n_pages, page, heads, D, sc.FP16, t)
    ids = np.array([[8191, 8192, 16383, 16384, 19999, 3]])
    i32 = lambda a: torch.from_numpy(np.ascontiguousarray(a)).to(torch.int32).cuda()
    n = 5 * page + 77
    seqs = sc.Seqs(i32(np.array([0, n])), i32(np.array([n])), i32(ids), n)
    rng = np.random.default_rng(0)
    HD = heads * D
    x = torch.from_numpy(rng.standard_normal((3, n, HD))).to(t).cuda()
    q = torch.from_numpy(rng.standard_normal((n, G * HD))).to(t).cuda()
    pos = torch.arange(n, dtype=torch.int32, device="cuda")[:, None].contiguous()
    sc.salicache_paged_write_rotary(ctx, pages.c, seqs.c, sc.Rotary(10000.0 ** (-np.arange(64) / 64)), pos, x[0], HD, 1, x[2], HD, x[0], x[1], HD, HD)
    k, v = torch.empty_like(x[0]), torch.empty_like(x[0])
    sc.salicache_paged_read(ctx, pages.c, seqs.c, k, v, HD, HD)
    assert torch.equal(k, x[2]) and torch.equal(v, x[1])
    # attention, its weights, and the same over a copy of the cache in pages below 2^32
    low = sc.PageSet(6, page, heads, D, sc.FP16, t, data=pages.data[torch.from_numpy(ids[0]).cuda()].contiguous())
    low_seqs = sc.Seqs(seqs.row_start, seqs.length, i32(np.arange(6)[None]), n)
    wk = torch.empty(sc.salicache_paged_work_bytes(ctx, pages.c, G), dtype=torch.uint8, device="cuda")
    for first in (0, n - 3):                             # many rows, and three
        res = []
        for pg, table in ((pages, i32(ids)), (low, i32(np.arange(6)[None]))):
            s = sc.Seqs(i32(np.array([0, n - first])), i32(np.array([n])), table, n - first)
            qq, out, lse = q[first:], torch.empty_like(q[first:]), torch.empty((n - first, heads * G), device="cuda")
            sc.salicache_paged_attend(ctx, pg.c, s.c, qq, G * HD, G, D ** -0.5, 0, 0, out, G * HD, lse, wk, wk.numel())
            weight = torch.zeros((1, heads, n), device="cuda")
            sc.salicache_paged_weigh(ctx, pg.c, s.c, qq, G * HD, G, D ** -0.5, lse, 1.0, None, weight, n, wk, wk.numel())
            res.append((out, lse, weight))
        assert all(torch.equal(a, b) for a, b in zip(*res)) and res[0][2].min() > 0
    # gathered from the far pages into near ones and back
    keep = torch.from_numpy(np.sort(rng.choice(n, 300, replace=False))).to(torch.int32).cuda()
    to = sc.Seqs(seqs.row_start, seqs.length, i32(np.array([[100, 18000, 7]])), 0)
    kept = i32(np.array([300]))
    sc.salicache_paged_keep(ctx, pages.c, seqs.c, keep, 1, 300, None, kept, to.c)
    back = sc.Seqs(i32(np.array([0, 300])), kept, i32(np.array([[100, 18000, 7]])), 300)
    sc.salicache_paged_read(ctx, pages.c, back.c, k, v, HD, HD)
    assert torch.equal(k[:300], x[2][keep.long()]) and torch.equal(v[:300], x[1][keep.long()])
    assert sc.salicache_poll_status(ctx) == 0


# ---- streams and graphs

def test_graphs_side_by_side_on_streams_of_their_own():
    """Weights and trees captured for two sequences' batches, replayed at the same time, each with a workspace of its own."""
    import torch
    ctx = sc.Context(sc.salicache_default_params(max_batch=1, chunk_frames=1, L=1))
    pairs = []
    for k in range(2):
        c = Weigh(ctx, "int8", "f16", 2, 4, 128, 32, [2500, 300 + k], [200, 100])
        d = Tree(ctx, "fp16", "bf16", 2, 4, 128, 64, [1500 + k, 300], [40, 64])
        lse, had = torch.from_numpy(c.lse).float().cuda(), torch.from_numpy(c.had).cuda()
        weight, out, l = torch.zeros_like(had), torch.empty_like(d.q), torch.empty((d.w.rows, 8), device="cuda")
        s = torch.cuda.Stream()
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.stream(s), torch.cuda.graph(g, stream=s):
            sc.salicache_paged_weigh(ctx, c.pages.c, c.seqs.c, c.q, c.q.shape[1], 4, 128 ** -0.5, lse, 0.5, had, weight, had.shape[2], c.work, c.work.numel())
            sc.salicache_paged_attend_tree(ctx, d.pages.c, d.seqs.c, d.bits, 1, d.q, d.q.shape[1], 4, 128 ** -0.5, 0, 0, out, d.q.shape[1], l, d.work,
                                           d.work.numel())
        pairs.append((s, g, c, d, weight, out, l, lse, had))      # a graph holds addresses only
    for _ in range(5):
        for s, g, *_ in pairs:
            with torch.cuda.stream(s):
                g.replay()
    torch.cuda.synchronize()
    assert sc.salicache_poll_status(ctx) == 0
    for _, _, c, d, weight, out, l, *_ in pairs:
        held = ~np.isnan(c.want)
        pu.check(weight.double().cpu().numpy()[held], c.want[held], c.tol[held], "weight")
        pu.check(out.double().cpu().numpy().reshape(d.want[0].shape), d.want[0], d.want[2], "out")
        pu.check(l.double().cpu().numpy(), d.want[1], d.want[3], "lse")


def test_a_stream_that_is_given(ctx):
    import torch
    s = torch.cuda.Stream()
    w = torch.rand((2, 3, 500), device="cuda")
    ln = torch.tensor([500, 77], dtype=torch.int32, device="cuda")
    keep, kept = torch.empty((2, 3, 50), dtype=torch.int32, device="cuda"), torch.empty(2, dtype=torch.int32, device="cuda")
    torch.cuda.synchronize()
    sc.salicache_select_heavy(ctx, w, 500, 3, 2, ln, 50, 2, 9, keep, kept, stream=s)
    s.synchronize()
    from test_gpu_paged_keep import select
    assert np.array_equal(keep.cpu().numpy(), select(w.cpu().numpy(), [500, 77], 50, 2, 9)) and kept.tolist() == [50, 50]
    assert sc.salicache_poll_status(ctx, s) == 0
