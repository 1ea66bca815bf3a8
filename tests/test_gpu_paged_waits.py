"""GPU tests of the way out of the paged attention when a wait between a block's parts is given up: the limit is set so low
that waits run out, some or all of them, and the call has to end, say so, and leave everything usable."""
import numpy as np
import pytest

import paged_util as pu
from paper_2602_14236_b200 import binding as sc

pytestmark = pytest.mark.gpu

ORDINARY = 1 << 24


@pytest.fixture()
def ctx():
    return sc.Context(sc.salicache_default_params(max_batch=1, chunk_frames=1, L=1))


class Call:
    def __init__(self, ctx, fmt, dt, heads, G, D, page, lens, news, window=0, sinks=0):
        import torch
        t = {"f16": torch.float16, "bf16": torch.bfloat16}[dt]
        self.ctx, self.G, self.window, self.sinks = ctx, G, window, sinks
        self.w = pu.World(100, fmt, t, heads, D, page, lens, news)
        self.pages, self.seqs = self.w.device(extra_rows=4)
        self.Hq = heads * G
        self.q = torch.from_numpy(np.random.default_rng(4).standard_normal((self.w.rows + 4, self.Hq * D))).to(t).cuda()
        self.work = torch.full((sc.salicache_paged_work_bytes(ctx, self.pages.c, G),), 255, dtype=torch.uint8, device="cuda")
        qn = self.q.double().cpu().numpy().reshape(-1, self.Hq, D)
        self.want = self.w.expect(qn, G, D ** -0.5, window, sinks, rows=self.w.rows)

    def run(self, limit):
        """The status; outputs that come without an error are right, and rows of no sequence stay in any case."""
        import torch
        D, R = self.w.D, self.w.rows
        out, lse = torch.full_like(self.q, 7.0), torch.full((R + 4, self.Hq), 7.0, device="cuda")
        sc.salicache_paged_wait_limit(self.ctx, limit)
        sc.salicache_paged_attend(self.ctx, self.pages.c, self.seqs.c, self.q, self.Hq * D, self.G, D ** -0.5, self.window, self.sinks,
                                  out, self.Hq * D, lse, self.work, self.work.numel())
        status = sc.salicache_poll_status(self.ctx)
        torch.cuda.synchronize()
        assert (out[R:] == 7).all() and (lse[R:] == 7).all()
        if status == 0:
            want, wl, tol, ltol = self.want
            pu.check(out[:R].double().cpu().numpy().reshape(R, self.Hq, D), want, tol, "out")
            pu.check(lse[:R].double().cpu().numpy(), wl, ltol, "lse")
        return status


CALLS = [
    ("fp16", "f16", 2, 4, 128, 64, [3000, 700, 0, 129], [1, 1, 0, 1]),               # a few rows per sequence
    ("int8", "bf16", 2, 4, 128, 16, [3000, 700, 0, 129], [1, 1, 0, 1]),
    ("int4", "f16", 4, 4, 64, 32, [3000, 700, 5], [4, 3, 4]),
    ("fp16", "bf16", 2, 2, 128, 128, [2500, 300], [300, 300]),                        # many
    ("fp16", "f16", 1, 3, 64, 16, [1500, 31], [200, 31]),
    ("int8", "f16", 2, 2, 128, 32, [2500, 300], [300, 300]),
    ("int4", "bf16", 2, 4, 128, 64, [2500, 300], [200, 300]),
    ("int4", "f16", 1, 1, 64, 16, [2000], [500]),
]


@pytest.mark.parametrize("args", CALLS, ids=lambda a: f"{a[0]}-{a[1]}-{a[4]}-{sum(a[7])}")
def test_every_wait_given_up(ctx, args):
    c = Call(ctx, *args)
    for _ in range(3):
        assert c.run(0) == sc.E_CUDA
        assert c.run(ORDINARY) == 0


@pytest.mark.parametrize("args", CALLS, ids=lambda a: f"{a[0]}-{a[1]}-{a[4]}-{sum(a[7])}")
def test_some_waits_given_up(ctx, args):
    """Which ones depends on the moment: either the outputs are right or the status says that they are not."""
    c = Call(ctx, *args)
    for limit in (1, 2, 3, 5, 8, 13, 21, 34, 55, 89, 200, 1000):
        assert c.run(limit) in (0, sc.E_CUDA)
    assert c.run(ORDINARY) == 0


def test_a_window_with_waits_given_up(ctx):
    for news in ([1, 1], [150, 60]):
        c = Call(ctx, "fp16", "f16", 2, 4, 128, 16, [2500, 300], news, 400, 20)
        for limit in (0, 1, 2, 4, 16, 64):
            assert c.run(limit) in ((sc.E_CUDA,) if limit == 0 else (0, sc.E_CUDA))
        assert c.run(ORDINARY) == 0


def test_calls_after_one_that_gave_up_are_not_held_up(ctx):
    """Calls in a row without a look at the status between them, then another context on the same pages."""
    import torch
    c = Call(ctx, "int8", "f16", 2, 2, 128, 32, [2500, 300], [300, 300])
    out = torch.zeros_like(c.q)
    for limit in (0, 3, ORDINARY, 0, ORDINARY):
        sc.salicache_paged_wait_limit(ctx, limit)
        sc.salicache_paged_attend(ctx, c.pages.c, c.seqs.c, c.q, c.Hq * 128, 2, 128 ** -0.5, 0, 0, out, c.Hq * 128, None, c.work, c.work.numel())
    assert sc.salicache_poll_status(ctx) == sc.E_CUDA
    pu.check(out[:c.w.rows].double().cpu().numpy().reshape(c.w.rows, c.Hq, 128), c.want[0], c.want[2], "out")
    c.ctx = sc.Context(sc.salicache_default_params(max_batch=1, chunk_frames=1, L=1))
    assert c.run(ORDINARY) == 0


@pytest.mark.parametrize("news", [[1, 1], [150, 60]])
def test_a_missing_page_does_not_hide_that_a_wait_was_given_up(ctx, news):
    """Before or after it, in the same call or another one."""
    c = Call(ctx, "int4", "f16", 2, 4, 128, 32, [2500, 300], news)
    whole = c.seqs
    table = whole.table.clone()
    table[0, 3], table[1, 0] = -1, c.w.n_pages
    holes = sc.Seqs(whole.row_start, whole.length, table, c.w.rows + 4)

    def call(seqs, limit):
        import torch
        sc.salicache_paged_wait_limit(ctx, limit)
        sc.salicache_paged_attend(ctx, c.pages.c, seqs.c, c.q, c.Hq * 128, 4, 0.1, 0, 0, torch.empty_like(c.q), c.Hq * 128, None, c.work,
                                  c.work.numel())

    call(holes, ORDINARY)
    assert sc.salicache_poll_status(ctx) == sc.E_CAPACITY
    for run in ([(holes, 0)], [(holes, ORDINARY), (whole, 0)], [(whole, 0), (holes, ORDINARY)], [(holes, 0), (holes, ORDINARY)]):
        for seqs, limit in run:
            call(seqs, limit)
        assert sc.salicache_poll_status(ctx) == sc.E_CUDA
        assert sc.salicache_poll_status(ctx) == 0
