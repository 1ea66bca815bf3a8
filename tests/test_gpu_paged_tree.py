"""GPU tests of attention for drafted tokens that form a tree, against the plain 64-bit form and its bounds (paged_util.attend)."""
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


def trees(rng, news, kind):
    """Per sequence a boolean matrix [n][n]: what row i sees of the rows."""
    out = []
    for n in news:
        m = np.zeros((n, n), bool)
        if kind == "any":                                # any bits: later rows, not its own, none at all
            m = rng.random((n, n)) < 0.4
            m[rng.random(n) < 0.2] = False
        else:
            for i in range(n):
                parent = i - 1 if kind == "chain" else int(rng.integers(max(-1, i - 6), i))
                if parent >= 0:
                    m[i] = m[parent]
                m[i, i] = True
            if kind == "shuffled":                       # nodes in any order
                p = rng.permutation(n)
                m = m[np.ix_(p, p)]
        out.append(m)
    return out


def words(mats, n_words, rows):
    """uint64 [rows][n_words], with bits past a sequence's rows set at random: they mean nothing."""
    rng = np.random.default_rng(9)
    out = rng.integers(0, 2 ** 63, (rows, n_words), dtype=np.uint64)
    r = 0
    for m in mats:
        n = m.shape[0]
        for i in range(n):
            for c in range(min(n, 64 * n_words)):
                bit = np.uint64(1) << np.uint64(c % 64)
                out[r, c // 64] = out[r, c // 64] | bit if m[i, c] else out[r, c // 64] & ~bit
            r += 1
    return out


def expect(w, q, G, scale, mats, n_words, window, sinks, missing=()):
    Hq = w.heads * G
    out, tol = np.zeros((w.rows, Hq, w.D)), np.zeros((w.rows, Hq, w.D))
    lse, ltol = np.full((w.rows, Hq), -np.inf), np.zeros((w.rows, Hq))
    for b, m in enumerate(mats):
        n, before = w.news[b], w.lens[b] - w.news[b]
        for i in range(n):
            named = m[i].copy()
            named[64 * n_words:] = False
            at = before + max(int(named.sum()), 1) - 1
            j = np.arange(max(before, 0))
            if window:
                j = j[(j > at - window) | (j < sinks)]
            own = before + np.flatnonzero(named)
            j = np.concatenate([j, own[own >= 0]]).astype(int)
            j = j[[(b, x // w.page) not in missing for x in j]] if j.size else j
            r = int(w.start[b]) + i
            for h in range(w.heads):
                k, v = w.kv(b, h, 0), w.kv(b, h, 1)
                for g in range(G):
                    hq = h * G + g
                    out[r, hq], lse[r, hq], tol[r, hq], ltol[r, hq] = pu.attend(q[r, hq], k[j], v[j], scale, w.t, w.fmt)
    return out, lse, tol, ltol


def run(ctx, w, G, mats, n_words=1, window=0, sinks=0, extra=2, pad=8, q_scale=1.0, status=0, table=None, missing=()):
    import torch
    pages, seqs = w.device(extra)
    if table is not None:
        seqs = sc.Seqs(seqs.row_start, seqs.length, torch.from_numpy(table).to(torch.int32).cuda(), w.rows + extra)
    Hq, R = w.heads * G, w.rows + extra
    stride, scale = Hq * w.D + pad, w.D ** -0.5
    qf = torch.from_numpy(q_scale * np.random.default_rng(1).standard_normal((R, stride))).to(w.t)
    bits = torch.from_numpy(words(mats, n_words, R).view(np.int64)).cuda()
    out = torch.full((R, stride), 7.0, dtype=w.t, device="cuda")
    lse = torch.full((R, Hq), 7.0, dtype=torch.float32, device="cuda")
    wk = torch.full((sc.salicache_paged_work_bytes(ctx, pages.c, G),), 255, dtype=torch.uint8, device="cuda")
    sc.salicache_paged_attend_tree(ctx, pages.c, seqs.c, bits, n_words, qf.cuda(), stride, G, scale, window, sinks, out, stride, lse, wk, wk.numel())
    assert sc.salicache_poll_status(ctx) == status
    q = qf[:, :Hq * w.D].double().numpy().reshape(R, Hq, w.D)
    want, wl, tol, ltol = expect(w, q, G, scale, mats, n_words, window, sinks, missing)
    got, gl = out.double().cpu().numpy(), lse.double().cpu().numpy()
    assert (got[:, Hq * w.D:] == 7).all() and (got[w.rows:] == 7).all() and (gl[w.rows:] == 7).all()
    pu.check(got[:w.rows, :Hq * w.D].reshape(w.rows, Hq, w.D), want, tol, "out")
    pu.check(gl[:w.rows], wl, ltol, "lse")


LAYOUTS = [                                              # rows of q per sequence: a few; up to 16; many
    (2, 1, 128, 16, [130, 9, 300], [4, 5, 3]),
    (2, 4, 128, 64, [700, 40, 0, 129], [2, 1, 0, 7]),
    (1, 8, 64, 32, [257, 33], [2, 1]),
    (2, 4, 128, 128, [500, 70, 64, 0], [64, 33, 64, 0]),
    (3, 6, 64, 16, [300, 21], [17, 21]),
    (1, 3, 128, 32, [200], [100]),
]


@pytest.mark.parametrize("fmt", ["fp16", "int8", "int4"])
@pytest.mark.parametrize("dt", ["f16", "bf16"])
@pytest.mark.parametrize("layout", range(len(LAYOUTS)))
def test_trees(ctx, fmt, dt, layout):
    heads, G, D, page, lens, news = LAYOUTS[layout]
    rng = np.random.default_rng(layout)
    w = pu.World(layout, fmt, _t(dt), heads, D, page, lens, news)
    run(ctx, w, G, trees(rng, news, ["branch", "shuffled", "any"][(layout + (dt == "f16")) % 3]), n_words=2)


@pytest.mark.parametrize("fmt", ["fp16", "int8", "int4"])
@pytest.mark.parametrize("window,sinks", [(1, 0), (17, 3), (128, 4), (100, 200), (4096, 4)])
@pytest.mark.parametrize("heads,G,D,page,lens,news", [(2, 2, 128, 32, [600, 300, 20], [3, 4, 4]), (1, 4, 64, 64, [900, 300, 40], [40, 64, 40])])
def test_windows(ctx, fmt, window, sinks, heads, G, D, page, lens, news):
    rng = np.random.default_rng(5)
    w = pu.World(8, fmt, _t("bf16"), heads, D, page, lens, news)
    run(ctx, w, G, trees(rng, news, "branch"), window=window, sinks=sinks)


@pytest.mark.parametrize("fmt", ["fp16", "int4"])
@pytest.mark.parametrize("G,news", [(1, [4, 1]), (4, [60, 64])])
def test_rows_that_see_nothing(ctx, fmt, G, news):
    """No position before the call's, and bits that name none, or only others."""
    w = pu.World(6, fmt, _t("f16"), 2, 128, 16, news, news)
    run(ctx, w, G, trees(np.random.default_rng(2), news, "any"))
    run(ctx, w, G, [np.zeros((n, n), bool) for n in news])


@pytest.mark.parametrize("fmt", ["fp16", "int8", "int4"])
@pytest.mark.parametrize("heads,G,D,lens,news", [(2, 4, 128, [500, 300], [2, 2]), (2, 4, 128, [1500, 300], [100, 256]), (1, 1, 64, [70], [70])])
def test_a_chain_is_causal_attention_bit_for_bit(ctx, fmt, heads, G, D, lens, news):
    import torch
    t = _t("bf16")
    w = pu.World(4, fmt, t, heads, D, 32, lens, news)
    pages, seqs = w.device()
    Hq = heads * G
    q = torch.from_numpy(np.random.default_rng(3).standard_normal((w.rows, Hq * D))).to(t).cuda()
    wk = torch.empty(sc.salicache_paged_work_bytes(ctx, pages.c, G), dtype=torch.uint8, device="cuda")
    a, b = (torch.empty_like(q) for _ in range(2))
    la, lb = (torch.empty((w.rows, Hq), device="cuda") for _ in range(2))
    bits = torch.from_numpy(words(trees(None, news, "chain"), 4, w.rows).view(np.int64)).cuda()
    sc.salicache_paged_attend(ctx, pages.c, seqs.c, q, Hq * D, G, 0.1, 0, 0, a, Hq * D, la, wk, wk.numel())
    sc.salicache_paged_attend_tree(ctx, pages.c, seqs.c, bits, 4, q, Hq * D, G, 0.1, 0, 0, b, Hq * D, lb, wk, wk.numel())
    assert sc.salicache_poll_status(ctx) == 0
    assert torch.equal(a, b) and torch.equal(la, lb)


@pytest.mark.parametrize("n_words", [1, 2, 16])
def test_many_words(ctx, n_words):
    """Rows past the words are named by none, and see what was there before the call."""
    news = [150, 64, 65]
    w = pu.World(5, "fp16", _t("bf16"), 1, 64, 64, [400, 64, 100], news)
    run(ctx, w, 2, trees(np.random.default_rng(3), news, "any"), n_words=n_words)


def test_missing_pages_and_more_rows_than_positions(ctx):
    w = pu.World(5, "int8", _t("f16"), 2, 128, 16, [300, 40], [30, 20])
    table = w.table.copy()
    table[0, 3], table[0, 17] = -1, 10 ** 6
    run(ctx, w, 2, trees(np.random.default_rng(3), [30, 20], "branch"), table=table, missing={(0, 3), (0, 17)}, status=sc.E_CAPACITY)
    for G in (1, 4):
        w = pu.World(5, "fp16", _t("f16"), 2, 64, 16, [5, 3], [8, 3])       # three rows at negative positions
        run(ctx, w, G, trees(np.random.default_rng(4), [8, 3], "any"))


def test_captured_with_trees_and_lengths_that_change(ctx):
    import torch
    t, G = _t("f16"), 4
    w = pu.World(5, "int4", t, 2, 128, 64, [600, 300], [24, 20])
    pages, seqs = w.device()
    Hq, D = 8, 128
    q = torch.from_numpy(np.random.default_rng(3).standard_normal((w.rows, Hq * D))).to(t).cuda()
    bits = torch.zeros((w.rows, 1), dtype=torch.int64, device="cuda")
    wk = torch.empty(sc.salicache_paged_work_bytes(ctx, pages.c, G), dtype=torch.uint8, device="cuda")
    out, lse = torch.empty_like(q), torch.empty((w.rows, Hq), device="cuda")
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            sc.salicache_paged_attend_tree(ctx, pages.c, seqs.c, bits, 1, q, Hq * D, G, D ** -0.5, 0, 0, out, Hq * D, lse, wk, wk.numel())
    for k, lens in enumerate(([600, 300], [333, 20])):
        w.lens = lens
        mats = trees(np.random.default_rng(k), w.news, "branch")
        seqs.length.copy_(torch.tensor(lens))
        bits.copy_(torch.from_numpy(words(mats, 1, w.rows).view(np.int64)))
        g.replay()
        assert sc.salicache_poll_status(ctx) == 0
        want, wl, tol, ltol = expect(w, q.double().cpu().numpy().reshape(-1, Hq, D), G, D ** -0.5, mats, 1, 0, 0)
        pu.check(out.double().cpu().numpy().reshape(-1, Hq, D), want, tol, "out")
        pu.check(lse.double().cpu().numpy(), wl, ltol, "lse")
