"""GPU tests of the weights that attention gave each position, against a plain 64-bit form.

Bounds, with s = scale q.k and p = e^(s - lse), per term: the score as in paged_util.attend, (D + 2) 2^-24 scale sum|q k|, and
for INT4 a step of the 16-bit type in a value of K; scale and lse are taken times log2(e) in binary32, and their difference
is rounded: 2^-23 (|s| + |lse|) + 2^-24 |s - lse|; the exponential 2^-21.  The sum over the rows is binary32: its terms times
2^-24, which is far more than their order can matter; decay * in and the last addition are one rounding each."""
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


def expect(w, q, lse, G, scale, decay, had, stride, missing=()):
    """Weights [seqs][heads][stride] and bounds; `had` None: zeros.  NaN where nothing is to be written."""
    out, tol = np.full((len(w.lens), w.heads, stride), np.nan), np.zeros((len(w.lens), w.heads, stride))
    for b, (ln, n) in enumerate(zip(w.lens, w.news)):
        held, before, r0 = min(ln, stride), ln - n, int(w.start[b])
        p = before + np.arange(n)
        for h in range(w.heads):
            old = np.zeros(held)
            m = held if n == 0 else min(max(before, 0), held)
            if had is not None:
                old[:m] = had[b, h, :m] * (decay if n else 1.0)
            x, e, terms = np.zeros(held), np.zeros(held), np.zeros(held)
            if n:
                k = w.kv(b, h, 0)[:held]
                for g in range(G):
                    qq, l = q[r0:r0 + n, h * G + g], lse[r0:r0 + n, h * G + g][:, None]
                    s = scale * (qq @ k.T)
                    sees = (p[:, None] >= np.arange(held)[None]) & np.isfinite(l)
                    pr = np.where(sees, np.exp(np.where(sees, s - np.where(np.isfinite(l), l, 0), 0)), 0)
                    a = scale * (np.abs(qq) @ np.abs(k).T) * (w.D + 2) * 2.0 ** -24
                    if w.fmt == "int4":
                        a += scale * pu.eps(w.t) * np.array([(np.abs(k) * np.abs(v)).max(-1) for v in qq])
                    la = np.abs(np.where(np.isfinite(l), l, 0))
                    a += 2.0 ** -23 * (np.abs(s) + la) + 2.0 ** -24 * np.abs(s - la) + 2.0 ** -21
                    x += pr.sum(0)
                    e += (pr * a).sum(0)
                    terms += sees.sum(0)
            for bb, i in missing:
                if bb == b:
                    x[i * w.page:(i + 1) * w.page] = e[i * w.page:(i + 1) * w.page] = 0
            out[b, h, :held] = old + x
            tol[b, h, :held] = (e + terms * 2.0 ** -24 * x) * 1.01 + 2.0 ** -23 * (np.abs(old) + x)
    return out, tol


def softmax_sums(w, q, G, scale):
    """lse of every row, as binary32 values: what attention returns."""
    lse = np.full((w.rows, w.heads * G), -np.inf)
    for b, n in enumerate(w.news):
        for h in range(w.heads):
            k = w.kv(b, h, 0)
            for i in range(n):
                p = w.lens[b] - n + i
                if p >= 0:
                    for g in range(G):
                        s = scale * (k[:p + 1] @ q[int(w.start[b]) + i, h * G + g])
                        lse[int(w.start[b]) + i, h * G + g] = s.max() + np.log(np.exp(s - s.max()).sum())
    return lse.astype(np.float32).astype(np.float64)


def run(ctx, w, G, decay=1.0, given=True, alias=False, extra=2, pad=8, stride=None, q_scale=1.0, status=0, table=None, missing=(), times=1):
    import torch
    pages, seqs = w.device(extra)
    if table is not None:
        seqs = sc.Seqs(seqs.row_start, seqs.length, torch.from_numpy(table).to(torch.int32).cuda(), w.rows + extra)
    Hq, R, B = w.heads * G, w.rows + extra, len(w.lens)
    row, scale = Hq * w.D + pad, w.D ** -0.5
    stride = max(w.lens) + 5 if stride is None else stride
    rng = np.random.default_rng(1)
    qf = torch.from_numpy(q_scale * rng.standard_normal((R, row))).to(w.t)
    q = qf[:, :Hq * w.D].double().numpy().reshape(R, Hq, w.D)
    lse = np.concatenate([softmax_sums(w, q, G, scale), np.full((extra, Hq), np.nan)])
    had = rng.random((B, w.heads, stride)).astype(np.float32) * 3
    for b, n in enumerate(w.news):                       # what a new position had, and what lies behind the end, is not read
        had[b, :, max(w.lens[b] - n, 0) if n else w.lens[b]:] = np.nan
    dev_had = torch.from_numpy(had).cuda()
    out = dev_had if alias else torch.full((B, w.heads, stride), 7.0, device="cuda")
    behind = out.clone()
    wk = torch.full((sc.salicache_paged_work_bytes(ctx, pages.c, G),), 255, dtype=torch.uint8, device="cuda")
    dl = torch.from_numpy(lse).float().cuda()
    for _ in range(times):
        sc.salicache_paged_weigh(ctx, pages.c, seqs.c, qf.cuda(), row, G, scale, dl, decay, dev_had if given else None, out, stride, wk, wk.numel())
        got = out.clone()
    assert sc.salicache_poll_status(ctx) == status
    want, tol = expect(w, q, lse, G, scale, decay, had.astype(np.float64) if given else None, stride, missing)
    g = out.double().cpu().numpy()
    held = ~np.isnan(want)
    pu.check(g[held], want[held], tol[held], "weight")
    assert np.array_equal(g[~held], behind.double().cpu().numpy()[~held], equal_nan=True)
    return got


LAYOUTS = [                                              # rows of q per sequence: single tokens; a few; many
    (2, 4, 128, 16, [130, 9, 1, 300], [1, 1, 1, 1]),
    (2, 8, 64, 64, [700, 40, 0, 129], [1, 1, 0, 0]),
    (3, 1, 128, 32, [257, 33, 50], [5, 8, 9]),
    (1, 64, 64, 16, [100, 17], [1, 1]),
    (2, 4, 128, 128, [500, 70, 64, 31, 0], [64, 33, 64, 0, 0]),
    (1, 6, 64, 16, [700, 21], [301, 21]),
    (1, 3, 128, 32, [900], [900]),
    (2, 1, 128, 64, [1300, 260], [129, 260]),
    (1, 16, 64, 128, [640], [130]),
]


@pytest.mark.parametrize("fmt", ["fp16", "int8", "int4"])
@pytest.mark.parametrize("dt", ["f16", "bf16"])
@pytest.mark.parametrize("layout", range(len(LAYOUTS)))
def test_weights(ctx, fmt, dt, layout):
    heads, G, D, page, lens, news = LAYOUTS[layout]
    w = pu.World(layout, fmt, _t(dt), heads, D, page, lens, news)
    run(ctx, w, G, decay=[1.0, 0.75, 0.0][layout % 3], given=layout % 4 != 3, alias=layout % 4 == 1)


@pytest.mark.parametrize("fmt", ["fp16", "int8", "int4"])
@pytest.mark.parametrize("layout", [0, 4, 7])
def test_large_scores(ctx, fmt, layout):
    heads, G, D, page, lens, news = LAYOUTS[layout]
    run(ctx, pu.World(layout, fmt, _t("bf16"), heads, D, page, lens, news), G, q_scale=8.0)


@pytest.mark.parametrize("G,lens,news", [(2, [5, 3, 40], [8, 3, 1]), (4, [60, 300], [90, 200])])
def test_more_rows_than_positions(ctx, G, lens, news):
    run(ctx, pu.World(5, "fp16", _t("f16"), 2, 64, 16, lens, news), G)


@pytest.mark.parametrize("news", [[1, 1], [70, 40]])
def test_missing_pages_and_a_short_array(ctx, news):
    w = pu.World(5, "int8", _t("f16"), 2, 128, 16, [300, 40], news)
    table = w.table.copy()
    table[0, 3], table[0, 17] = -1, 10 ** 6
    run(ctx, w, 2, table=table, missing={(0, 3), (0, 17)}, status=sc.E_CAPACITY)
    run(ctx, w, 2, stride=201, status=sc.E_CAPACITY)
    w = pu.World(5, "int8", _t("f16"), 2, 128, 16, [300, 40], news)
    run(ctx, w, 2)


def test_no_rows_at_all_is_a_copy(ctx):
    w = pu.World(5, "int4", _t("f16"), 2, 128, 16, [300, 0, 17], [0, 0, 0])
    run(ctx, w, 2, decay=0.5)


@pytest.mark.parametrize("fmt,news", [("fp16", [1] * 40), ("int4", [1] * 40), ("int8", [30] * 40)])
def test_many_sequences(ctx, fmt, news):
    lens = [30 + 7 * (i % 13) if i % 11 else 30 for i in range(40)]
    run(ctx, pu.World(5, fmt, _t("f16"), 1, 64, 16, lens, news), 2)


@pytest.mark.parametrize("fmt", ["fp16", "int8", "int4"])
@pytest.mark.parametrize("heads,G,D,page,lens,news", [
    (2, 4, 128, 32, [300, 900, 17, 40, 700, 33, 5], [1, 400, 1, 0, 5, 33, 4]),       # single tokens, drafts and prompts
    (1, 2, 64, 16, [300] * 40, [1] * 20 + [200] + [1] * 19),
    (1, 1, 128, 64, [90, 500, 64], [0, 3, 0]),                                       # as many rows as sequences, all in one
    (1, 2, 64, 16, [200, 300, 50, 70], [0, 0, 4, 0]),
    (1, 40, 64, 16, [200, 30], [1, 1]),                                              # many query heads
    (1, 12, 64, 16, [200, 30, 60], [2, 1, 0]),
])
def test_batches_of_every_kind(ctx, fmt, heads, G, D, page, lens, news):
    w = pu.World(6, fmt, _t("f16"), heads, D, page, lens, news)
    run(ctx, w, G)
    run(ctx, w, G, decay=0.5, alias=True)


@pytest.mark.parametrize("layout", [0, 2, 4, 6])
def test_the_same_bits_on_every_call(ctx, layout):
    import torch
    heads, G, D, page, lens, news = LAYOUTS[layout]
    w = pu.World(layout, "fp16", _t("bf16"), heads, D, page, lens, news)
    a = run(ctx, w, G)
    for _ in range(3):
        assert torch.equal(torch.nan_to_num(a), torch.nan_to_num(run(ctx, w, G)))


def test_attention_and_its_weights_add_up(ctx):
    """With the sums that attention returns, the weights of a call's rows add up to one per row and query head."""
    import torch
    t, G, D = _t("bf16"), 4, 128
    for lens, news in (([1000, 300], [1, 1]), ([1000, 300], [500, 300])):
        w = pu.World(9, "int8", t, 2, D, 64, lens, news)
        pages, seqs = w.device()
        q = torch.from_numpy(np.random.default_rng(1).standard_normal((w.rows, 8 * D))).to(t).cuda()
        out, lse = torch.empty_like(q), torch.empty((w.rows, 8), device="cuda")
        wk = torch.empty(sc.salicache_paged_work_bytes(ctx, pages.c, G), dtype=torch.uint8, device="cuda")
        weight = torch.zeros((2, 2, 1000), device="cuda")
        sc.salicache_paged_attend(ctx, pages.c, seqs.c, q, 8 * D, G, D ** -0.5, 0, 0, out, 8 * D, lse, wk, wk.numel())
        sc.salicache_paged_weigh(ctx, pages.c, seqs.c, q, 8 * D, G, D ** -0.5, lse, 1.0, None, weight, 1000, wk, wk.numel())
        assert sc.salicache_poll_status(ctx) == 0
        total = weight.double().sum(-1).cpu().numpy()
        # a row's weights add up to 1 within the errors of its scores, twice (the sum's and the weights'): 4e-5 for |s| < 8, D = 128
        assert np.allclose(total, G * np.array(news)[:, None], rtol=5e-5, atol=0)


def test_captured_with_lengths_that_change(ctx):
    import torch
    t, G, D = _t("f16"), 4, 128
    for news in ([1, 1], [64, 40]):
        w = pu.World(9, "fp16", t, 2, D, 64, [700, 300], news)
        pages, seqs = w.device()
        q = torch.from_numpy(np.random.default_rng(1).standard_normal((w.rows, 8 * D))).to(t).cuda()
        qn = q.double().cpu().numpy().reshape(-1, 8, D)
        lse, weight = torch.zeros((w.rows, 8), device="cuda"), torch.full((2, 2, 700), 7.0, device="cuda")
        wk = torch.empty(sc.salicache_paged_work_bytes(ctx, pages.c, G), dtype=torch.uint8, device="cuda")
        s = torch.cuda.Stream()
        with torch.cuda.stream(s):
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g, stream=s):
                sc.salicache_paged_weigh(ctx, pages.c, seqs.c, q, 8 * D, G, D ** -0.5, lse, 1.0, None, weight, 700, wk, wk.numel())
        for lens in ([700, 300], [333, 40], [64, 700 // 64 * 64 - 400]):
            w.lens = lens
            sums = softmax_sums(w, qn, G, D ** -0.5)
            lse.copy_(torch.from_numpy(sums))
            seqs.length.copy_(torch.tensor(lens))
            weight.fill_(7.0)
            g.replay()
            assert sc.salicache_poll_status(ctx) == 0
            want, tol = expect(w, qn, sums, G, D ** -0.5, 1.0, None, 700)
            got, held = weight.double().cpu().numpy(), ~np.isnan(want)
            pu.check(got[held], want[held], tol[held], "weight")
            assert (got[~held] == 7).all()
