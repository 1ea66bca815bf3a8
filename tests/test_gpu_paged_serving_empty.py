"""GPU tests of calls without rows, sequences or entries, by empty tensors: whole numbers and copies, compared for equality."""
import numpy as np
import pytest

import paged_util as pu
from paper_2602_14236_b200 import binding as sc

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    return sc.Context(sc.salicache_default_params(max_batch=1, chunk_frames=1, L=1))


def _empty(dtype, *shape):
    import torch
    return torch.empty((0, *shape), dtype=dtype, device="cuda")


@pytest.mark.parametrize("given", [True, False])
def test_no_rows(ctx, given):
    """Weights are copied, or zeros where there were none; everything else stays as it is."""
    import torch
    t, G, D = torch.float16, 2, 64
    w = pu.World(3, "int8", t, 2, D, 16, [300, 0, 40], [0, 0, 0])
    pages, seqs = w.device()
    q, kv = _empty(t, 4 * D), _empty(t, 2 * D)
    work = torch.empty(sc.salicache_paged_work_bytes(ctx, pages.c, G), dtype=torch.uint8, device="cuda")
    had, out = torch.rand((3, 2, 305), device="cuda"), torch.full((3, 2, 305), 7.0, device="cuda")
    data, n = pages.data.clone(), ctx.launch_count()
    sc.salicache_paged_write(ctx, pages.c, seqs.c, kv, kv, 2 * D, 2 * D)
    sc.salicache_paged_read(ctx, pages.c, seqs.c, kv, kv, 2 * D, 2 * D)
    sc.salicache_paged_write_rotary(ctx, pages.c, seqs.c, sc.Rotary([0.1] * 8), _empty(torch.int32, 1), q, 4 * D, G, q, 4 * D, kv, kv, 2 * D, 2 * D)
    sc.salicache_paged_attend(ctx, pages.c, seqs.c, q, 4 * D, G, 0.1, 0, 0, q, 4 * D, _empty(torch.float32, 4), work, work.numel())
    sc.salicache_paged_attend_tree(ctx, pages.c, seqs.c, _empty(torch.int64, 1), 1, q, 4 * D, G, 0.1, 0, 0, q, 4 * D, _empty(torch.float32, 4), work, work.numel())
    assert ctx.launch_count() == n
    sc.salicache_paged_weigh(ctx, pages.c, seqs.c, q, 4 * D, G, 0.1, _empty(torch.float32, 4), 0.5, had if given else None, out, 305, work, work.numel())
    assert sc.salicache_poll_status(ctx) == 0
    want = torch.full_like(out, 7.0)
    for b, held in enumerate(w.lens):
        want[b, :, :held] = had[b, :, :held] if given else 0
    assert torch.equal(out, want) and torch.equal(pages.data, data)


def test_no_sequences_and_no_entries(ctx):
    import torch
    i32, f32 = torch.int32, torch.float32
    pages = sc.PageSet(4, 16, 2, 64, sc.FP16, torch.float16)
    none = sc.Seqs(torch.zeros(1, dtype=i32, device="cuda"), _empty(i32), _empty(i32, 3), 0)
    n = ctx.launch_count()
    sc.salicache_select_heavy(ctx, _empty(f32, 2, 20), 20, 2, 0, _empty(i32), 8, 1, 1, _empty(i32, 2, 8), _empty(i32))
    sc.salicache_paged_keep(ctx, pages.c, none.c, _empty(i32, 2, 8), 2, 8, None, _empty(i32), None, _empty(f32, 2, 20), _empty(f32, 2, 20), 20)
    work = torch.empty(sc.salicache_paged_work_bytes(ctx, pages.c, 1), dtype=torch.uint8, device="cuda")
    sc.salicache_paged_weigh(ctx, pages.c, none.c, _empty(torch.float16, 128), 128, 1, 0.1, _empty(f32, 2), 1.0, None, _empty(f32, 2, 20), 20, work, work.numel())
    one = sc.Seqs(torch.zeros(2, dtype=i32, device="cuda"), torch.full((1,), 9, dtype=i32, device="cuda"), torch.zeros((1, 3), dtype=i32, device="cuda"), 0)
    sc.salicache_paged_keep(ctx, pages.c, one.c, torch.empty((1, 1, 0), dtype=i32, device="cuda"), 1, 0, None, torch.zeros(1, dtype=i32, device="cuda"), None)
    assert ctx.launch_count() == n and sc.salicache_poll_status(ctx) == 0


def test_moving_without_the_offsets_that_it_does_not_use(ctx):
    import torch
    w = pu.World(3, "fp16", torch.float16, 2, 64, 16, [100], [0], spare=8)
    pages, seqs = w.device()
    free = np.setdiff1d(np.arange(w.n_pages), w.table[0])
    i32 = lambda a: torch.from_numpy(np.ascontiguousarray(a)).to(torch.int32).cuda()
    keep, kept, table = i32(np.arange(0, 100, 3)[None, None]), i32(np.array([34])), i32(free[None, :3])
    source = sc.SeqsC(1, w.width, 0, None, seqs.length.data_ptr(), seqs.table.data_ptr())
    target = sc.SeqsC(1, 3, 0, None, None, table.data_ptr())
    sc.salicache_paged_keep(ctx, pages.c, source, keep, 1, 34, None, kept, target)
    assert sc.salicache_poll_status(ctx) == 0
    raw = pages.data.cpu()
    for k, j in enumerate(range(0, 100, 3)):
        assert torch.equal(raw[free[k // 16], :, :, k % 16], raw[w.table[0, j // 16], :, :, j % 16])
