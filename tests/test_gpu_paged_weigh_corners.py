"""GPU tests of the attention weights where an operand is not finite: rows that count as none, keys whose scores are all minus
infinity, sums that overflow beside numbers that are none.  Bounds as in test_gpu_paged_weigh.py."""
import numpy as np
import pytest

import paged_util as pu
import test_gpu_paged_weigh as wg
from paper_2602_14236_b200 import binding as sc

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    return sc.Context(sc.salicache_default_params(max_batch=1, chunk_frames=1, L=1))


class Call:
    """A call of salicache_paged_weigh whose q, sums and pages a test changes before it runs."""

    def __init__(self, ctx, fmt, t, heads, G, D, page, lens, news, seed=3):
        import torch
        self.ctx, self.G, self.scale = ctx, G, D ** -0.5
        self.w = w = pu.World(seed, fmt, t, heads, D, page, lens, news)
        self.q = torch.from_numpy(np.random.default_rng(4).standard_normal((w.rows, heads * G, D))).to(t)
        self.lse = wg.softmax_sums(w, self.q.double().numpy(), G, self.scale)

    def expect(self, lse=None):
        w = self.w
        return wg.expect(w, self.q.double().numpy(), self.lse if lse is None else lse, self.G, self.scale, 1.0, None, max(w.lens))

    def run(self, q=None, lse=None):
        import torch
        w, row = self.w, self.w.heads * self.G * self.w.D
        pages, seqs = w.device()
        out = torch.full((len(w.lens), w.heads, max(w.lens)), 7.0, device="cuda")
        wk = torch.empty(sc.salicache_paged_work_bytes(self.ctx, pages.c, self.G), dtype=torch.uint8, device="cuda")
        sc.salicache_paged_weigh(self.ctx, pages.c, seqs.c, (self.q if q is None else q).contiguous().cuda(), row, self.G, self.scale,
                                 torch.from_numpy(self.lse if lse is None else lse).float().cuda(), 1.0, None, out, max(w.lens), wk, wk.numel())
        assert sc.salicache_poll_status(self.ctx) == 0
        return out.double().cpu().numpy()


def _same(got, want, tol):
    held = ~np.isnan(want)
    pu.check(got[held], want[held], tol[held], "weight")


# few rows per sequence (single tokens, two tiles of columns, all rows in one sequence), and many
SHAPES = [("fp16", "bf16", 2, 4, 64, [200, 33], [1, 1]), ("int8", "f16", 1, 3, 128, [200, 77], [5, 4]), ("fp16", "f16", 2, 2, 64, [200, 9, 40, 17], [0, 0, 4, 0]),
          ("int4", "bf16", 1, 1, 64, [300], [14]), ("fp16", "bf16", 2, 4, 128, [900, 300], [70, 150]), ("int8", "f16", 1, 3, 64, [700, 90], [300, 60]),
          ("int4", "bf16", 1, 6, 64, [700], [200])]


@pytest.mark.parametrize("shape", SHAPES, ids=str)
@pytest.mark.parametrize("value", [float("nan"), float("inf"), float("-inf")])
def test_a_row_that_counts_as_none_may_hold_anything(ctx, shape, value):
    """-infinity in d_lse takes a row out, whatever its q holds."""
    fmt, dt, heads, G, D, lens, news = shape
    c = Call(ctx, fmt, wg._t(dt), heads, G, D, 16, lens, news)
    out = np.random.default_rng(5).random(c.lse.shape) < 0.3
    out[0, 0] = True
    lse = np.where(out, -np.inf, c.lse)
    q = c.q.clone()
    import torch
    q[torch.from_numpy(out)] = value
    _same(c.run(q, lse), *c.expect(lse))


@pytest.mark.parametrize("fmt", ["fp16", "int8"])
@pytest.mark.parametrize("G,lens,news", [(3, [300, 50], [1, 1]), (3, [300, 50], [5, 5]), (3, [900, 300], [130, 200]), (6, [900], [60]), (40, [300], [40]), (4, [900], [60])])
def test_a_key_whose_scores_are_minus_infinity_weighs_nothing(ctx, fmt, G, lens, news):
    """An element of K that is infinite, against rows of q of the other sign: no row gives it anything, nor do columns that are no
    row."""
    D, t = 64, wg._t("f16")
    c = Call(ctx, fmt, t, 2, G, D, 16, lens, news)
    c.q[:, :, 7] = -c.q[:, :, 7].abs() - 0.5
    want, tol = c.expect()
    w = c.w
    for b, j in ((0, 0), (0, 133), (0, lens[0] - news[0]), (len(lens) - 1, 17)):
        pid, slot = w.table[b, j // 16], j % 16
        for h in range(2):
            w.data[pid, 0, h, slot] = 0
            if fmt == "fp16":
                w.data[pid, 0, h, slot, 7] = float("inf")
            else:                                        # 127 * 60000 is past f16's largest number
                w.data[pid, 0, h, slot, 7] = 127
                w.scale[pid, 0, h, slot] = 60000.0
            want[b, h, j] = tol[b, h, j] = 0
    _same(c.run(), want, tol)


@pytest.mark.parametrize("fmt", ["fp16", "int8"])
@pytest.mark.parametrize("G", [1, 2, 3])
def test_none_and_infinite_together(ctx, fmt, G):
    """One row is no number, another one's sums lie far below its scores: what both see is no number, whichever columns they are."""
    n, length, D = 150, 500, 64
    c = Call(ctx, fmt, wg._t("f16"), 1, G, D, 16, [length], [n])
    want, tol = c.expect()
    before = length - n
    for none in range(20, 29):
        for far in range(30, 39):
            q, lse = c.q.clone(), c.lse.copy()
            q[none, G - 1, 3] = float("nan")
            lse[far, 0] = -300.0
            got = c.run(q, lse)[0, 0]
            assert np.isnan(got[:before + none + 1]).all()
            assert np.isposinf(got[before + none + 1:before + far + 1]).all()
            pu.check(got[before + far + 1:], want[0, 0, before + far + 1:], tol[0, 0, before + far + 1:], "weight")
