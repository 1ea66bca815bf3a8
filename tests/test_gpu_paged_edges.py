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
