"""GPU tests of attention weights of batches whose rows are in a few of many sequences: values, against a plain 64-bit form with the
bounds of test_gpu_paged_weigh.py, and which kernels run."""
import numpy as np
import pytest

import paged_util as pu
import test_gpu_paged_weigh as wg
from paper_2602_14236_b200 import binding as sc

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    return sc.Context(sc.salicache_default_params(max_batch=1, chunk_frames=1, L=1))


def _one(n, at, rows):
    return [rows if b == at else 0 for b in range(n)]


BATCHES = [                                              # heads, G, D, page, lengths, rows
    (1, 4, 64, 16, [40] * 20 + [500] + [17] * 79, _one(100, 20, 60)),         # fewer rows than sequences, all in one
    (1, 2, 64, 32, [40] * 39 + [600], _one(40, 39, 40)),                      # as many
    (2, 3, 128, 16, [700] + [30] * 31, _one(32, 0, 32)),
    (1, 4, 64, 16, [90] * 30, [4 if b % 3 == 0 else 0 for b in range(30)]),   # two tiles of columns in some
    (1, 4, 64, 16, [90] * 12, [3 if b % 3 == 0 else 0 for b in range(12)]),
    (1, 8, 64, 64, [200, 100, 300, 50], [2, 0, 2, 0]),                        # as many rows as sequences, 16 rows of q in each
    (1, 1, 64, 16, [200, 100, 300, 50, 60, 70, 80, 90, 10, 20, 30], [0, 0, 11, 0, 0, 0, 0, 0, 0, 0, 0]),
    (1, 4, 64, 16, [50 + b for b in range(300)], [1] * 200 + [0] * 99 + [70]),
]


@pytest.mark.parametrize("fmt", ["fp16", "int8", "int4"])
@pytest.mark.parametrize("batch", range(len(BATCHES)))
def test_rows_in_a_few_of_many_sequences(ctx, fmt, batch):
    heads, G, D, page, lens, news = BATCHES[batch]
    w = pu.World(batch, fmt, wg._t("bf16" if batch % 2 else "f16"), heads, D, page, lens, news)
    wg.run(ctx, w, G, decay=0.5)
    wg.run(ctx, w, G, given=False)


@pytest.mark.parametrize("news,launches", [(_one(100, 3, 60), 3), (_one(40, 3, 40), 3), ([1] * 40, 3), ([1, 1, 1, 0], 1), ([4, 0], 1)])
def test_long_sequences_are_the_other_kernels(ctx, news, launches):
    """Whatever the number of sequences: only a batch that cannot have one goes without it."""
    w = pu.World(1, "fp16", wg._t("f16"), 1, 64, 16, [90] * len(news), news)
    n = ctx.launch_count()
    wg.run(ctx, w, 4, extra=0)                           # rows of nobody count too
    assert ctx.launch_count() - n == launches


def test_a_captured_call_whose_rows_move(ctx):
    """Single tokens in one replay, all rows in one sequence in the next, none at all in a third."""
    import torch
    t, G, D, n = wg._t("f16"), 2, 64, 24
    lens = [150 + 7 * b for b in range(n)]
    w = pu.World(2, "int8", t, 1, D, 16, lens, [1] * n)
    pages, seqs = w.device()
    q = torch.from_numpy(np.random.default_rng(1).standard_normal((n, G * D))).to(t).cuda()
    qn = q.double().cpu().numpy().reshape(n, G, D)
    lse, out = torch.zeros((n, G), device="cuda"), torch.full((n, 1, max(lens)), 7.0, device="cuda")
    wk = torch.full((sc.salicache_paged_work_bytes(ctx, pages.c, G),), 255, dtype=torch.uint8, device="cuda")
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            sc.salicache_paged_weigh(ctx, pages.c, seqs.c, q, G * D, G, D ** -0.5, lse, 1.0, None, out, max(lens), wk, wk.numel())
    for news in ([1] * n, _one(n, 5, n), [0] * n, [2 * (b % 2) for b in range(n)], _one(n, 0, n), [1] * n):
        w.news, w.start, w.rows = news, np.concatenate([[0], np.cumsum(news)]).astype(np.int64), int(sum(news))
        sums = wg.softmax_sums(w, qn, G, D ** -0.5)
        lse[:w.rows] = torch.from_numpy(sums).float().cuda()
        seqs.row_start.copy_(torch.from_numpy(w.start))
        out.fill_(7.0)
        g.replay()
        assert sc.salicache_poll_status(ctx) == 0
        want, tol = wg.expect(w, qn, sums, G, D ** -0.5, 1.0, None, max(lens))
        got, held = out.double().cpu().numpy(), ~np.isnan(want)
        pu.check(got[held], want[held], tol[held], "weight")
        assert (got[~held] == 7).all()
