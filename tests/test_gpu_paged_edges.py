"""GPU tests of the attention over the paged cache: tiles in which little or nothing is to be read, scores that keep rising, in
every format, type and kernel."""
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


def _run(ctx, w, G, window=0, sinks=0, table=None, q=None, scale=None, calls=1):
    """Outputs of the world's rows, and q as float64; `table` replaces the world's."""
    import torch
    pages, seqs = w.device()
    if table is not None:
        seqs = sc.Seqs(seqs.row_start, seqs.length, torch.from_numpy(table).to(torch.int32).cuda(), w.rows)
    Hq = w.heads * G
    if q is None:
        q = np.random.default_rng(3).standard_normal((w.rows, Hq, w.D))
    qt = torch.from_numpy(q.reshape(w.rows, Hq * w.D)).to(w.t)
    qd = qt.cuda()
    out, lse = torch.full_like(qd, 7.0), torch.full((w.rows, Hq), 7.0, device="cuda")
    work = torch.full((sc.salicache_paged_work_bytes(ctx, pages.c, G),), 255, dtype=torch.uint8, device="cuda")
    for _ in range(calls):
        sc.salicache_paged_attend(ctx, pages.c, seqs.c, qd, Hq * w.D, G, w.D ** -0.5 if scale is None else scale, window, sinks, out,
                                  Hq * w.D, lse, work, work.numel())
    f = lambda x: x.double().cpu().numpy()
    return f(out).reshape(w.rows, Hq, w.D), f(lse), f(qt).reshape(w.rows, Hq, w.D)


@pytest.mark.parametrize("fmt,dt", [("fp16", "bf16"), ("int8", "f16"), ("int4", "f16")])
@pytest.mark.parametrize("news", [[1, 1], [2, 2], [40, 3]])
def test_warps_with_nothing_to_read_pass_many_tiles(ctx, fmt, dt, news):
    """Pages of 16 positions, most of them missing in a pattern that changes from tile to tile: of a tile's eight groups of
    keys some are there, some are not, and the ring goes round many times."""
    w = pu.World(90, fmt, _t(dt), 1, 64, 16, [9000, 2200], news)
    table, missing = w.table.copy(), []
    rng = np.random.default_rng(7)
    for b, n in enumerate(w.lens):
        for i in range(-(-n // 16)):
            if rng.random() < 0.8:
                table[b, i] = (-1, w.n_pages, -2 ** 31)[i % 3]
                missing.append((b, i))
    got, lse, q = _run(ctx, w, 4, table=table, calls=3)
    assert sc.salicache_poll_status(ctx) == sc.E_CAPACITY
    want, wl, tol, ltol = w.expect(q, 4, 0.125, 0, 0, missing=missing)
    pu.check(got, want, tol, "out")
    pu.check(lse, wl, ltol, "lse")


@pytest.mark.parametrize("G", [4, 20])
def test_the_stride_of_a_single_row_does_not_matter(ctx, G):
    import torch
    w = pu.World(91, "fp16", _t("f16"), 1, 64, 16, [300], [1])
    pages, seqs = w.device()
    q = torch.randn((1, G * 64)).half()
    out, lse = torch.zeros_like(q).cuda(), torch.zeros((1, G), device="cuda")
    work = torch.empty(sc.salicache_paged_work_bytes(ctx, pages.c, G), dtype=torch.uint8, device="cuda")
    want, wl, tol, ltol = w.expect(q.double().numpy().reshape(1, G, 64), G, 0.125, 0, 0)
    for stride in (G * 64, 2 ** 40, 2 ** 62):
        out.fill_(7.0)
        sc.salicache_paged_attend(ctx, pages.c, seqs.c, q.cuda(), stride, G, 0.125, 0, 0, out, stride, lse, work, work.numel())
        assert sc.salicache_poll_status(ctx) == 0
        pu.check(out.double().cpu().numpy().reshape(1, G, 64), want, tol, "out")
        pu.check(lse.double().cpu().numpy(), wl, ltol, "lse")


@pytest.mark.parametrize("fmt,dt", [("fp16", "f16"), ("int8", "bf16"), ("int4", "f16")])
def test_rows_before_the_first_sequence(ctx, fmt, dt):
    """row_start need not begin at 0: the rows before it belong to nobody either."""
    import torch
    for news in ([1, 1], [90, 4]):
        w = pu.World(92, fmt, _t(dt), 2, 64, 16, [300, 45], news)
        pages, seqs = w.device()
        skip, R = 5, w.rows + 8
        seqs = sc.Seqs(seqs.row_start + skip, seqs.length, seqs.table, R)
        q = torch.randn((R, 4 * 64)).to(w.t)
        out, lse = torch.full((R, 4 * 64), 7.0, dtype=w.t, device="cuda"), torch.full((R, 4), 7.0, device="cuda")
        work = torch.empty(sc.salicache_paged_work_bytes(ctx, pages.c, 2), dtype=torch.uint8, device="cuda")
        sc.salicache_paged_attend(ctx, pages.c, seqs.c, q.cuda(), 256, 2, 0.125, 0, 0, out, 256, lse, work, work.numel())
        mine = slice(skip, skip + w.rows)
        want, wl, tol, ltol = w.expect(q[mine].double().numpy().reshape(w.rows, 4, 64), 2, 0.125, 0, 0)
        pu.check(out[mine].double().cpu().numpy().reshape(w.rows, 4, 64), want, tol, "out")
        pu.check(lse[mine].double().cpu().numpy(), wl, ltol, "lse")
        x = torch.full((2, R, 128), 7.0, dtype=w.t, device="cuda")
        sc.salicache_paged_read(ctx, pages.c, seqs.c, x[0], x[1], 128, 128)
        before = pages.data.clone()
        x[:, :skip], x[:, skip + w.rows:] = 3.0, 3.0
        held = x.clone()
        sc.salicache_paged_read(ctx, pages.c, seqs.c, x[0], x[1], 128, 128)
        assert torch.equal(held, x)
        if fmt == "fp16":
            sc.salicache_paged_write(ctx, pages.c, seqs.c, x[0], x[1], 128, 128)
            assert torch.equal(torch.nan_to_num(before, nan=-9.0), torch.nan_to_num(pages.data, nan=-9.0))
        assert sc.salicache_poll_status(ctx) == 0
        for y in (out, lse):
            assert (y[:skip] == 7).all() and (y[skip + w.rows:] == 7).all()


def test_more_sequences_than_threads_in_a_block(ctx):
    rng = np.random.default_rng(93)
    lens = rng.integers(1, 70, 1300).tolist()
    lens[700] = 900
    news = [min(n, int(rng.integers(0, 9))) for n in lens]
    news[700] = 400
    for fmt, dt in (("fp16", "bf16"), ("int4", "f16")):
        w = pu.World(94, fmt, _t(dt), 1, 64, 16, lens, news)
        got, lse, q = _run(ctx, w, 4)
        want, wl, tol, ltol = w.expect(q, 4, 0.125, 0, 0)
        pu.check(got, want, tol, "out")
        pu.check(lse, wl, ltol, "lse")
    w = pu.World(95, "int8", _t("f16"), 1, 64, 16, lens, [1] * len(lens))
    got, lse, q = _run(ctx, w, 4)
    want, wl, tol, ltol = w.expect(q, 4, 0.125, 0, 0)
    pu.check(got, want, tol, "out")
    pu.check(lse, wl, ltol, "lse")
    assert sc.salicache_poll_status(ctx) == 0


@pytest.mark.parametrize("fmt", ["fp16", "int8", "int4"])
@pytest.mark.parametrize("dt", ["f16", "bf16"])
def test_repeated_calls_give_the_same_bits_in_every_format(ctx, fmt, dt):
    import torch
    for news in ([1] * 4, [64, 200, 9, 0]):
        w = pu.World(96, fmt, _t(dt), 2, 128, 32, [5000, 900, 77, 40], news)
        first = _run(ctx, w, 4)
        for _ in range(5):
            again = _run(ctx, w, 4)
            assert all(np.array_equal(x, y) for x, y in zip(first, again))
