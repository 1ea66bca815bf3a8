"""GPU tests of frequencies of any magnitude, whose turns a double or a long double does not hold: expected angles by integer
arithmetic, bounds as in test_gpu_paged_rotary.py; what the fraction of a turn lacks, 2^-62 turns a position, adds 2 pi 2^-31 < 3e-9 to its
1.47e-7 radians at most."""
import math
from fractions import Fraction

import numpy as np
import pytest

import paged_util as pu
from paper_2602_14236_b200 import binding as sc
from test_paged_serving_refusals import _rotary, _write

BITS = 400


def _pi():
    """pi 2^BITS by Machin's formula."""
    one = 1 << BITS + 20

    def arctan(n):
        total, term, k = 0, one // n, 1
        while term:
            total += term // k if k % 4 == 1 else -(term // k)
            term //= n * n
            k += 2
        return total
    return 4 * (4 * arctan(5) - arctan(239)) >> 20


PI = Fraction(_pi(), 1 << BITS)


def angle(pos, freq):
    turns = Fraction(int(pos)) * Fraction(freq) / (2 * PI)
    return float((turns - math.floor(turns)) * 2 * PI)


FREQS = [1.0, -0.1, 3.5, 1e3 + 0.1, 1e6 / 7, -1e9 / 3, 1e12 / 7, 2.0 ** 53 + 2, -1.7e19 / 9, 2.0 ** 64, -2.0 ** 64, 1e-9, 1e-18, 5e-324, 0.0, 2 * math.pi]


def test_magnitudes_that_are_refused():
    for x in (2.0 ** 64 * (1 + 2.0 ** -52), -1e20, 1e300, float("inf"), float("nan")):
        assert _write(rotary=_rotary(freq=(5, x))) == sc.E_PARAM
    assert _write(rotary=_rotary(freq=(5, -2.0 ** 64)), k=None) == sc.E_NULL


@pytest.mark.gpu
def test_frequencies_of_any_magnitude():
    import torch
    ctx = sc.Context(sc.salicache_default_params(max_batch=1, chunk_frames=1, L=1))
    t, D = torch.float16, 64
    pos = np.array([0, 1, -1, 2, 7, 1000, 12345, 999983, -10 ** 6, 2 ** 30, 2 ** 31 - 1, -2 ** 31])
    n = len(pos)
    i32 = lambda a: torch.from_numpy(np.ascontiguousarray(a)).to(torch.int32).cuda()
    pages = sc.PageSet(2, 16, 1, D, sc.FP16, t)
    seqs = sc.Seqs(i32(np.array([0, n])), i32(np.array([n])), i32(np.array([[1]])), n)
    x = torch.from_numpy(np.random.default_rng(0).standard_normal((n, D))).to(t)
    xd, out = x.cuda(), torch.empty((n, D), dtype=t, device="cuda")
    axis, both = np.arange(16) % 2, np.stack([pos, pos[::-1]], 1)
    sc.salicache_paged_write_rotary(ctx, pages.c, seqs.c, sc.Rotary(FREQS, axis, 2, sc.NEIGHBOURS), i32(both), xd, D, 1, out, D, xd, xd, D, D)
    assert sc.salicache_poll_status(ctx) == 0
    phi = np.array([[angle(both[r, axis[i]], FREQS[i]) for i in range(16)] for r in range(n)])
    v = x.double().numpy()
    a, b = v[:, 0:32:2], v[:, 1:32:2]
    want, off = v.copy(), np.zeros_like(v)
    want[:, 0:32:2], want[:, 1:32:2] = a * np.cos(phi) - b * np.sin(phi), b * np.cos(phi) + a * np.sin(phi)
    off[:, 0:32:2] = off[:, 1:32:2] = 2.7e-7 * (np.abs(a) + np.abs(b))
    tol = np.where(off > 0, off + pu.eps(t) / 2 * (np.abs(want) + off) + 2.0 ** -25, 0)
    pu.check(out.double().cpu().numpy(), want, tol, "q")
    k, vv = torch.empty_like(out), torch.empty_like(out)
    sc.salicache_paged_read(ctx, pages.c, seqs.c, k, vv, D, D)
    assert torch.equal(k, out) and torch.equal(vv.cpu(), x)
