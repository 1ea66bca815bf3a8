"""GPU tests of the paged cache and of the attention over it, against plain 64-bit forms (tests/paged_util.py)."""
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


def _np(x):
    return x.double().cpu().numpy()


def _work(ctx, pages, G):
    import torch
    return torch.full((sc.salicache_paged_work_bytes(ctx, pages.c, G),), 255, dtype=torch.uint8, device="cuda")


def _attend(ctx, w, G, window=0, sinks=0, seed=1, q_scale=1.0, extra=0, pad=0, table=None, work=None, status=0, missing=(), scale=None):
    """Runs the kernel over the world, with `extra` rows behind the last sequence and `pad` elements between rows; checks
    outputs, sums and untouched memory."""
    import torch
    pages, seqs = w.device(extra)
    if table is not None:
        seqs = sc.Seqs(seqs.row_start, seqs.length, torch.from_numpy(table).to(torch.int32).cuda(), w.rows + extra)
    Hq, R = w.heads * G, w.rows + extra
    stride = Hq * w.D + pad
    scale = w.D ** -0.5 if scale is None else scale
    rng = np.random.default_rng(seed)
    qf = torch.from_numpy(q_scale * rng.standard_normal((R, stride))).to(w.t)
    out = torch.full((R, stride), 7.0, dtype=w.t, device="cuda")
    lse = torch.full((R, Hq), 7.0, dtype=torch.float32, device="cuda")
    wk = _work(ctx, pages, G) if work is None else work
    sc.salicache_paged_attend(ctx, pages.c, seqs.c, qf.cuda(), stride, G, scale, window, sinks, out, stride, lse, wk, wk.numel())
    assert sc.salicache_poll_status(ctx) == status
    q = qf[:, :Hq * w.D].double().numpy().reshape(R, Hq, w.D)
    want, wl, tol, ltol = w.expect(q, G, scale, window, sinks, missing=missing)
    got, gl = _np(out), _np(lse)
    assert (got[:, Hq * w.D:] == 7).all() and (got[w.rows:] == 7).all() and (gl[w.rows:] == 7).all()
    pu.check(got[:w.rows, :Hq * w.D].reshape(w.rows, Hq, w.D), want, tol, "out")
    pu.check(gl[:w.rows], wl, ltol, "lse")


# ---- the store

@pytest.mark.parametrize("fmt", ["fp16", "int8", "int4"])
@pytest.mark.parametrize("dt", ["f16", "bf16"])
@pytest.mark.parametrize("heads,D,page,lens,news", [
    (2, 128, 16, [5, 16, 33, 0, 40], [5, 1, 17, 0, 3]),
    (5, 64, 32, [70, 1], [37, 1]),
    (8, 128, 128, [300], [300]),
    (1, 64, 16, [1], [1]),
])
def test_write_then_read(ctx, fmt, dt, heads, D, page, lens, news):
    import torch
    t = _t(dt)
    w = pu.World(11, fmt, t, heads, D, page, lens, news)
    pages, seqs = w.device(extra_rows=3)
    R, HD, pad = w.rows + 3, heads * D, 24
    rng = np.random.default_rng(5)
    x = rng.standard_normal((2, R, heads, D))
    x = np.where(rng.random(x.shape) < 0.02, 8 * x, x)
    x[:, 0] = 0.0                                    # a row of zeros, one of equal values, one tiny, one large
    x[1, -4] = -3.0
    x[0, -4] *= 1e-6
    x = pu.to_t(x, t)
    # rows as slices of one wider array
    rows = torch.full((R, 2 * HD + pad), float("nan"), dtype=t)
    rows[:, :HD] = torch.from_numpy(x[0].reshape(R, HD)).to(t)
    rows[:, HD:2 * HD] = torch.from_numpy(x[1].reshape(R, HD)).to(t)
    rows = rows.cuda()
    before = pages.data.clone(), None if pages.scale is None else pages.scale.clone()
    sc.salicache_paged_write(ctx, pages.c, seqs.c, rows, rows[:, HD:], 2 * HD + pad, 2 * HD + pad)
    assert sc.salicache_poll_status(ctx) == 0
    codes, s, z = pu.encode(x[:, :w.rows], fmt, t)
    want = pu.decode(codes, s, z, fmt, t)
    # slots: the new ones hold the codes, every other byte is as before
    data, scale = pu.as_tensors(codes, s, z, fmt, t)
    exp_d, exp_s = before[0].cpu(), None if before[1] is None else before[1].cpu()
    for b in range(len(lens)):
        for i in range(news[b]):
            r, p = int(w.start[b]) + i, lens[b] - news[b] + i
            exp_d[w.table[b, p // page], :, :, p % page] = data[:, r]
            if exp_s is not None:
                exp_s[w.table[b, p // page], :, :, p % page] = scale[:, r]
    # as values: the sign of a zero is not compared
    eq = lambda a, b: torch.equal(torch.nan_to_num(a.cpu().float(), nan=-12345.0), torch.nan_to_num(b.float(), nan=-12345.0))
    assert eq(pages.data, exp_d)
    assert exp_s is None or eq(pages.scale, exp_s)
    out = torch.full((2, R, HD + pad), 7.0, dtype=t, device="cuda")
    sc.salicache_paged_read(ctx, pages.c, seqs.c, out[0], out[1], HD + pad, HD + pad)
    assert sc.salicache_poll_status(ctx) == 0
    got = _np(out)
    assert (got[:, w.rows:] == 7).all() and (got[:, :, HD:] == 7).all()
    assert np.array_equal(got[:, :w.rows, :HD].reshape(2, w.rows, heads, D), want)


def test_rows_without_a_page_are_dropped_and_read_as_zeros(ctx):
    import torch
    w = pu.World(3, "int8", _t("f16"), 2, 128, 16, [40, 20, 2], [40, 20, 5])      # the last has three rows before position 0
    pages, seqs = w.device()
    table = seqs.table.clone()
    table[0, 1], table[1, 0] = -1, w.n_pages
    length = seqs.length.clone()
    length[1] = 60                                   # past the table: width 3 pages of 16
    bad = sc.Seqs(seqs.row_start, length, table, w.rows)
    x = torch.randn((2, w.rows, 256), device="cuda").half()
    before = pages.data.clone()
    sc.salicache_paged_write(ctx, pages.c, bad.c, x[0], x[1], 256, 256)
    assert sc.salicache_poll_status(ctx) == sc.E_CAPACITY
    gone = torch.zeros(w.rows, dtype=torch.bool)
    gone[16:32] = True                               # page 1 of sequence 0
    gone[48:60] = True                               # sequence 1: positions 40 .. 59; 48 and up are past the table
    gone[60:63] = True                               # negative positions of sequence 2
    table1 = [w.table[0, 0], w.table[0, 2], w.table[2, 0]] + ([w.table[1, 2]] if w.table[1, 2] < w.n_pages else [])
    touched = (pages.data != before).flatten(1).any(1).nonzero().flatten().tolist()
    assert set(touched) <= set(int(i) for i in table1)
    out = torch.full((2, w.rows, 256), 7.0, dtype=torch.float16, device="cuda")
    sc.salicache_paged_read(ctx, pages.c, bad.c, out[0], out[1], 256, 256)
    assert sc.salicache_poll_status(ctx) == sc.E_CAPACITY
    assert (out[:, gone] == 0).all()
    err = (out[:, 0:16] - x[:, 0:16]).abs()
    assert (err <= x[:, 0:16].abs().amax(-1, keepdim=True) / 127 * 0.51 + 1e-3).all()


# ---- attention: single rows

STEP_LENS = [1, 16, 17, 127, 128, 129, 700, 2049]


@pytest.mark.parametrize("fmt", ["fp16", "int8", "int4"])
@pytest.mark.parametrize("dt", ["f16", "bf16"])
@pytest.mark.parametrize("heads,G,D,page", [(2, 1, 128, 16), (2, 4, 128, 64), (1, 8, 64, 128), (3, 3, 64, 32)])
def test_one_new_token_per_sequence(ctx, fmt, dt, heads, G, D, page):
    w = pu.World(21, fmt, _t(dt), heads, D, page, STEP_LENS, [1] * len(STEP_LENS))
    _attend(ctx, w, G)


@pytest.mark.parametrize("fmt,dt", [("fp16", "f16"), ("int8", "bf16"), ("int4", "f16")])
@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (64, 4), (100, 300), (128, 128), (5000, 7)])
def test_one_new_token_under_a_window(ctx, fmt, dt, window, sinks):
    w = pu.World(22, fmt, _t(dt), 2, 128, 16, STEP_LENS, [1] * len(STEP_LENS))
    _attend(ctx, w, 4, window, sinks)


def test_one_sequence_split_over_many_blocks(ctx):
    w = pu.World(23, "fp16", _t("f16"), 1, 128, 64, [9001], [1], spare=0)
    _attend(ctx, w, 2)


def test_many_short_sequences(ctx):
    rng = np.random.default_rng(0)
    lens = rng.integers(0, 90, 300).tolist()
    w = pu.World(24, "int8", _t("f16"), 2, 64, 32, lens, [1 if n else 0 for n in lens])
    _attend(ctx, w, 2, extra=5)


# ---- attention: chunks of new rows

CHUNKS = [
    ([1], [1]), ([40], [40]), ([300], [64]), ([513], [129]), ([129, 5, 0, 260, 31], [2, 5, 0, 200, 1]), ([640, 64], [300, 64]),
]


@pytest.mark.parametrize("fmt", ["fp16", "int8", "int4"])
@pytest.mark.parametrize("dt", ["f16", "bf16"])
@pytest.mark.parametrize("heads,G,D,page", [(2, 4, 128, 64), (1, 1, 128, 16), (1, 3, 64, 32), (2, 8, 64, 128)])
def test_chunks_of_new_rows(ctx, fmt, dt, heads, G, D, page):
    for k, (lens, news) in enumerate(CHUNKS):
        w = pu.World(30 + k, fmt, _t(dt), heads, D, page, lens, news)
        _attend(ctx, w, G)


@pytest.mark.parametrize("fmt,dt", [("fp16", "bf16"), ("int8", "f16"), ("int4", "bf16")])
@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (17, 3), (128, 128), (200, 130), (10000, 2)])
def test_chunks_under_a_window(ctx, fmt, dt, window, sinks):
    for k, (lens, news) in enumerate([([700], [300]), ([129, 5, 0, 513, 31], [2, 5, 0, 513, 1])]):
        w = pu.World(40 + k, fmt, _t(dt), 2, 128, 16, lens, news)
        _attend(ctx, w, 2, window, sinks)


@pytest.mark.parametrize("G", [5, 7, 20, 33, 48])
def test_groups_that_do_not_divide_a_tile(ctx, G):
    """Rows of a tile are whole tokens: 125, 126, 120, 99 and 96 of 128."""
    for fmt, dt in (("fp16", "f16"), ("int4", "bf16")):
        w = pu.World(45 + G, fmt, _t(dt), 1, 64, 32, [333, 90], [29, 11])
        _attend(ctx, w, G)
        _attend(ctx, w, G, 100, 5)


@pytest.mark.parametrize("fmt,dt,D", [("fp16", "f16", 128), ("int8", "bf16", 64)])
def test_chunks_of_many_sequences(ctx, fmt, dt, D):
    """More sequences than a warp has lanes, some without rows, some without positions."""
    rng = np.random.default_rng(46)
    lens = rng.integers(0, 200, 75).tolist()
    news = [int(rng.integers(0, n + 1)) if i % 3 else 0 for i, n in enumerate(lens)]
    news[4] = lens[4] + 3
    w = pu.World(47, fmt, _t(dt), 1, D, 16, lens, news)
    _attend(ctx, w, 2, extra=7)
    _attend(ctx, w, 2, 50, 60)


def test_a_prompt_of_many_tiles(ctx):
    """Enough tiles that every block of the grid has some, with items cut in two and more."""
    w = pu.World(48, "fp16", _t("bf16"), 2, 64, 64, [1500], [1500])
    _attend(ctx, w, 2)
    w = pu.World(49, "int8", _t("f16"), 1, 128, 128, [9000], [40])
    _attend(ctx, w, 4)


def test_largest_group_of_query_heads(ctx):
    _attend(ctx, pu.World(50, "fp16", _t("f16"), 1, 128, 16, [200, 33], [3, 1]), 64)


def test_strided_rows_and_rows_behind_the_last_sequence(ctx):
    for news in ([1, 1, 1], [7, 0, 130]):
        w = pu.World(51, "int8", _t("bf16"), 2, 128, 32, [300, 1, 140], news)
        _attend(ctx, w, 4, extra=9, pad=72)


def test_rows_that_see_nothing(ctx):
    """More rows than positions (the first ones lie before position 0), and an empty sequence with rows."""
    for lens, news in (([2, 0, 5], [5, 3, 1]), ([0, 0], [1, 1]), ([100, 0], [300, 2])):
        w = pu.World(52, "fp16", _t("f16"), 2, 64, 16, lens, news)
        _attend(ctx, w, 2)


@pytest.mark.parametrize("q_scale", [30.0, 0.0, 200.0])
def test_peaked_and_flat_softmax(ctx, q_scale):
    for news in ([1, 1], [130, 20]):
        w = pu.World(53, "fp16", _t("f16"), 2, 128, 16, [400, 129], news, outliers=False)
        _attend(ctx, w, 2, q_scale=q_scale)


def test_rising_scores_move_the_maximum_every_tile(ctx):
    """Keys that grow along the sequence: every tile raises the running maximum far beyond the one before."""
    import torch
    for news in ([1], [200]):
        w = pu.World(54, "fp16", _t("f16"), 1, 128, 16, [1000], news, outliers=False)
        ramp = np.linspace(0.0, 12.0, 1000)
        for p in range(1000):
            w.values[w.table[0, p // 16], 0, 0, p % 16] = pu.to_t(np.full(128, ramp[p]), w.t)
        live = w.data.isnan().logical_not()
        w.data = torch.where(live, torch.from_numpy(w.values).to(w.t), w.data)
        w_q = 0.2
        _attend(ctx, w, 2, q_scale=w_q, scale=1.0)


def test_pages_outside_every_window_may_be_gone(ctx):
    for news in ([1], [140]):
        w = pu.World(55, "int8", _t("f16"), 2, 128, 16, [1500], news)
        table = w.table.copy()
        first = 1500 - news[0] - 256 + 1              # the first row's first position inside the window
        table[0, 2:first // 16] = -7
        _attend(ctx, w, 2, 256, 20, table=table)


@pytest.mark.parametrize("news", [[1, 1], [150, 3]])
def test_pages_that_are_missing_are_left_out(ctx, news):
    w = pu.World(56, "int4", _t("f16"), 2, 128, 32, [600, 40], news)
    table = w.table.copy()
    table[0, 3], table[0, 9], table[1, 0] = -1, w.n_pages, 2 ** 31 - 1
    _attend(ctx, w, 2, table=table, status=sc.E_CAPACITY, missing=[(0, 3), (0, 9), (1, 0)])


@pytest.mark.parametrize("fmt", ["fp16", "int4"])
def test_a_shared_prefix(ctx, fmt):
    """Two sequences whose tables name the same pages."""
    w = pu.World(57, fmt, _t("f16"), 2, 128, 16, [200, 200], [1, 40])
    w.table[1, :8] = w.table[0, :8]
    _attend(ctx, w, 4)


def test_offsets_beyond_32_bits(ctx):
    """Pages past 2^32 bytes of one layer's cache."""
    import torch
    w = pu.World(58, "fp16", _t("f16"), 8, 128, 128, [200], [3], spare=0)
    n = 2 ** 33 // (2 * 8 * 128 * 128 * 2) + 8
    data = torch.zeros((n, 2, 8, 128, 128), dtype=torch.float16, device="cuda")
    data[n - 2], data[n - 1] = w.data[int(w.table[0, 0])].cuda(), w.data[int(w.table[0, 1])].cuda()
    pages = sc.PageSet(n, 128, 8, 128, sc.FP16, torch.float16, data=data)
    i32 = lambda a: torch.tensor(a, dtype=torch.int32, device="cuda")
    q = torch.randn((3, 8, 128)).half()
    want, wl, tol, ltol = w.expect(q.double().numpy(), 1, 0.1, 0, 0)
    for seqs in (sc.Seqs(i32([0, 3]), i32([200]), i32([[n - 2, n - 1]]), 3),):
        out = torch.zeros((3, 8, 128), dtype=torch.float16, device="cuda")
        lse = torch.zeros((3, 8), device="cuda")
        wk = _work(ctx, pages, 1)
        sc.salicache_paged_attend(ctx, pages.c, seqs.c, q.cuda(), 1024, 1, 0.1, 0, 0, out, 1024, lse, wk, wk.numel())
        pu.check(_np(out), want, tol, "out")
        k = torch.zeros((2, 3, 1024), dtype=torch.float16, device="cuda")
        sc.salicache_paged_read(ctx, pages.c, seqs.c, k[0], k[1], 1024, 1024)
        assert np.array_equal(_np(k[0]).reshape(3, 8, 128), np.stack([w.kv(0, h, 0)[197:200] for h in range(8)], 1))
        x = torch.randn((2, 3, 1024), device="cuda").half()
        sc.salicache_paged_write(ctx, pages.c, seqs.c, x[0], x[1], 1024, 1024)
        sc.salicache_paged_read(ctx, pages.c, seqs.c, k[0], k[1], 1024, 1024)
        assert torch.equal(k, x)
        assert sc.salicache_poll_status(ctx) == 0


# ---- as they are used

@pytest.mark.parametrize("fmt", ["fp16", "int8", "int4"])
def test_prompt_then_steps_equals_the_definition(ctx, fmt):
    """A ragged prompt is written and attended, then tokens one by one; every output against the definition over the rows
    as the cache holds them."""
    import torch
    t = torch.float16
    heads, G, D, page, width = 2, 3, 128, 16, 9
    prompts, steps = [37, 1, 90], 5
    pages = sc.PageSet(32, page, heads, D, pu.FMT[fmt], t)
    table = torch.randperm(32)[:27].view(3, 9).to(torch.int32).cuda()
    i32 = lambda a: torch.tensor(a, dtype=torch.int32, device="cuda")
    work = _work(ctx, pages, G)
    seen = [[], [], []]
    g = torch.Generator().manual_seed(9)
    lens = [0, 0, 0]
    for it in range(1 + steps):
        news = prompts if it == 0 else [1, 1, 1]
        lens = [a + b for a, b in zip(lens, news)]
        R = sum(news)
        start = np.concatenate([[0], np.cumsum(news)])
        qkv = torch.randn((R, heads * (G + 2) * D), generator=g).to(t)
        d = qkv.cuda()
        seqs = sc.Seqs(i32(start.tolist()), i32(lens), table, R)
        row = d.shape[1]
        sc.salicache_paged_write(ctx, pages.c, seqs.c, d[:, heads * G * D:], d[:, heads * (G + 1) * D:], row, row)
        out = torch.empty((R, heads * G * D), dtype=t, device="cuda")
        sc.salicache_paged_attend(ctx, pages.c, seqs.c, d, row, G, D ** -0.5, 0, 0, out, heads * G * D, None, work, work.numel())
        assert sc.salicache_poll_status(ctx) == 0
        got = _np(out).reshape(R, heads * G, D)
        x = qkv.double().numpy()
        kv = x[:, heads * G * D:].reshape(R, 2, heads, D)
        held = pu.decode(*pu.encode(kv, fmt, t), fmt, t)
        for b in range(3):
            for i in range(news[b]):
                r = int(start[b]) + i
                seen[b].append(held[r])
                all_kv = np.stack(seen[b])
                for hq in range(heads * G):
                    h = hq // G
                    q = x[r, hq * D:(hq + 1) * D]
                    want, _, tol, _ = pu.attend(q, all_kv[:, 0, h], all_kv[:, 1, h], D ** -0.5, t, fmt)
                    pu.check(got[r, hq], want, tol, f"step {it} sequence {b} row {i} head {hq}")


@pytest.mark.parametrize("news", [[1, 1], [70, 3]])
def test_captured_and_replayed_with_other_lengths(ctx, news):
    """A captured write + attend replays on new contents of the same buffers, also side by side with another graph."""
    import torch
    t = _t("f16")
    ws = [pu.World(60 + i, "int8", t, 2, 128, 16, lens, news) for i, lens in enumerate([[200, 90], [333, 3], [90, 77]])]
    G, Hq, D = 2, 4, 128
    n_pages, width = max(w.n_pages for w in ws), max(w.width for w in ws)
    R = ws[0].rows

    class Lane:
        def __init__(self):
            self.pages = sc.PageSet(n_pages, 16, 2, D, sc.INT8, t)
            z = lambda *s: torch.zeros(s, dtype=torch.int32, device="cuda")
            self.seqs = sc.Seqs(z(3), z(2), z(2, width), R)
            self.q = torch.zeros((R, Hq * D), dtype=t, device="cuda")
            self.out = torch.zeros((R, Hq * D), dtype=t, device="cuda")
            self.lse = torch.zeros((R, Hq), device="cuda")
            self.work = _work(ctx, self.pages, G)

        def call(self):
            sc.salicache_paged_attend(ctx, self.pages.c, self.seqs.c, self.q, Hq * D, G, D ** -0.5, 0, 0, self.out, Hq * D, self.lse,
                                      self.work, self.work.numel())

        def fill(self, w, seed):
            self.pages.data[:w.n_pages].copy_(w.data)
            self.pages.scale[:w.n_pages].copy_(w.scale)
            self.seqs.row_start.copy_(torch.from_numpy(w.start))
            self.seqs.length.copy_(torch.tensor(w.lens))
            self.seqs.table[:, :w.width].copy_(torch.from_numpy(w.table))
            self.qh = torch.from_numpy(np.random.default_rng(seed).standard_normal((R, Hq * D))).to(t)
            self.q.copy_(self.qh)
            self.w = w

        def verify(self):
            want, wl, tol, ltol = self.w.expect(self.qh.double().numpy().reshape(R, Hq, D), G, D ** -0.5, 0, 0)
            pu.check(_np(self.out).reshape(R, Hq, D), want, tol, "out")
            pu.check(_np(self.lse), wl, ltol, "lse")

    lanes, graphs, streams = [Lane(), Lane()], [], [torch.cuda.Stream(), torch.cuda.Stream()]
    for ln in lanes:
        ln.fill(ws[0], 0)
        ln.call()
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            ln.call()
        graphs.append(g)
    for turn in range(2):
        for i, ln in enumerate(lanes):
            ln.fill(ws[(turn + i + 1) % 3], 10 * turn + i)
        torch.cuda.synchronize()
        for i in range(2):
            with torch.cuda.stream(streams[i]):
                for _ in range(3):
                    graphs[i].replay()
        torch.cuda.synchronize()
        for ln in lanes:
            ln.verify()
    assert sc.salicache_poll_status(ctx) == 0


_FIRST = """
import sys
sys.path.insert(0, {root!r})
sys.path.insert(0, {tests!r})
import numpy as np, torch
import paged_util as pu
from paper_2602_14236_b200 import binding as sc
ctx = sc.Context(sc.salicache_default_params(max_batch=1, chunk_frames=1, L=1))
for news in ([1, 1], [60, 3]):
    w = pu.World(61, "int8", torch.float16, 2, 128, 16, [200, 90], news)
    pages, seqs = w.device()
    qh = torch.from_numpy(np.random.default_rng(1).standard_normal((w.rows, 4 * 128))).half()
    q, x = qh.cuda(), torch.empty((2, w.rows, 256), dtype=torch.float16, device="cuda")
    out, lse = torch.zeros_like(q), torch.zeros((w.rows, 4), device="cuda")
    work = torch.empty(sc.salicache_paged_work_bytes(ctx, pages.c, 2), dtype=torch.uint8, device="cuda")
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        sc.salicache_paged_read(ctx, pages.c, seqs.c, x[0], x[1], 256, 256)
        sc.salicache_paged_write(ctx, pages.c, seqs.c, x[0], x[1], 256, 256)
        sc.salicache_paged_attend(ctx, pages.c, seqs.c, q, 512, 2, 0.09, 0, 0, out, 512, lse, work, work.numel())
    g.replay()
    torch.cuda.synchronize()
    assert sc.salicache_poll_status(ctx) == 0
    assert torch.isfinite(out).all() and (out != 0).any(1).all()
    held = np.stack([np.concatenate([w.kv(b, h, 0)[w.lens[b] - n:] for b, n in enumerate(news)]) for h in range(2)], 1)
    assert np.array_equal(x[0].double().cpu().numpy().reshape(held.shape), held)
print("captured")
"""


def test_the_first_call_of_a_process_may_be_captured(ctx):
    import os
    import subprocess
    import sys
    tests = os.path.dirname(os.path.abspath(__file__))
    r = subprocess.run([sys.executable, "-c", _FIRST.format(root=os.path.dirname(tests), tests=tests)], capture_output=True, text=True,
                       timeout=300)
    assert r.returncode == 0 and "captured" in r.stdout, r.stderr[-2000:]


def test_repeated_calls_give_the_same_bits(ctx):
    import torch
    for news in ([1] * 3, [64, 200, 9]):
        w = pu.World(70, "int4", _t("f16"), 2, 128, 64, [3000, 900, 77], news)
        pages, seqs = w.device()
        q = torch.randn((w.rows, 8 * 128), device="cuda").half()
        wk = _work(ctx, pages, 4)
        outs = []
        for _ in range(4):
            out = torch.zeros_like(q)
            sc.salicache_paged_attend(ctx, pages.c, seqs.c, q, 1024, 4, 0.088, 0, 0, out, 1024, None, wk, wk.numel())
            outs.append(out)
        assert all(torch.equal(outs[0], o) for o in outs[1:])


def test_nothing_to_do_and_too_small_a_workspace(ctx):
    import torch
    w = pu.World(71, "fp16", _t("f16"), 1, 64, 16, [3], [1])
    pages, seqs = w.device()
    q = torch.zeros((1, 64), dtype=torch.float16, device="cuda")
    wk = _work(ctx, pages, 1)
    none = sc.Seqs(torch.zeros(1, dtype=torch.int32, device="cuda"), torch.zeros(0, dtype=torch.int32, device="cuda"),
                   torch.zeros((0, 1), dtype=torch.int32, device="cuda"), 0)
    sc.salicache_paged_attend(ctx, pages.c, none.c, q, 64, 1, 1.0, 0, 0, q, 64, None, wk, wk.numel())
    with pytest.raises(sc.SalicacheError) as e:
        sc.salicache_paged_attend(ctx, pages.c, seqs.c, q, 64, 1, 1.0, 0, 0, q, 64, None, wk, wk.numel() - 1)
    assert e.value.status == sc.E_SHAPE
