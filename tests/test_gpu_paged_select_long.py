"""GPU tests of selection over lists longer than a block's shared memory holds keys of, and of the longest ones: whole numbers,
compared for equality."""
import numpy as np
import pytest

from paper_2602_14236_b200 import binding as sc
from test_gpu_paged_keep import _i32, _weights, run_select

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    return sc.Context(sc.salicache_default_params(max_batch=1, chunk_frames=1, L=1))


def test_lengths_past_two_to_the_thirtieth(ctx):
    """2^30 positions count, whatever the length says."""
    import torch
    most, budget, sinks, recent = 2 ** 30, 40, 2, 3
    stride = most + 9000
    w = torch.zeros((1, 1, stride), device="cuda")
    heavy = np.sort(np.random.default_rng(0).choice(most - 100, budget - sinks - recent - 4, replace=False)) + 50
    w[0, 0, torch.from_numpy(heavy).cuda()] = 1.0
    w[0, 0, most:] = 5.0                                 # held by nobody
    keep, kept = torch.empty((1, 1, budget), dtype=torch.int32, device="cuda"), torch.empty(1, dtype=torch.int32, device="cuda")
    for length in (2 ** 31 - 1, most + 1):
        sc.salicache_select_heavy(ctx, w, stride, 1, 1, _i32(np.array([length])), budget, sinks, recent, keep, kept)
        assert sc.salicache_poll_status(ctx) == sc.E_CAPACITY and kept.tolist() == [budget]
        ties = [x for x in range(sinks, 60) if x not in heavy][:4]                    # among zeros the lowest
        assert keep.flatten().tolist() == [0, 1] + sorted(ties + heavy.tolist()) + [most - 3, most - 2, most - 1]


@pytest.mark.parametrize("kind", ["any", "ties", "odd"])
@pytest.mark.parametrize("seqs,heads,longest,budget,recent", [
    (80, 1, 60000, 5000, 7), (40, 2, 51000, 50500, 0),   # a block per list
    (1, 1, 120000, 100, 100), (2, 1, 101500, 90001, 1),  # two blocks per list
])
def test_lists_that_shared_memory_does_not_hold(ctx, kind, seqs, heads, longest, budget, recent):
    lens = [longest - 13 * b for b in range(seqs)]
    run_select(ctx, _weights(kind, (seqs, heads, longest + 3)), lens, budget, 0, recent)
