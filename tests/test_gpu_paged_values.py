"""GPU tests of what the paged cache does with extreme values: both ends of the types' ranges."""
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


def _i32(a):
    import torch
    return torch.tensor(a, dtype=torch.int32, device="cuda")


def _stored(ctx, x, fmt, t, page=16):
    """Writes x float64 [2][R][heads][D] as one sequence of R positions and reads it back: float64, same shape."""
    import torch
    _, R, heads, D = x.shape
    n = -(-R // page)
    pages = sc.PageSet(n, page, heads, D, pu.FMT[fmt], t)
    seqs = sc.Seqs(_i32([0, R]), _i32([R]), _i32([list(range(n))]), R)
    d = torch.from_numpy(x.reshape(2, R, heads * D)).to(t).cuda()
    out = torch.full_like(d, 7.0)
    sc.salicache_paged_write(ctx, pages.c, seqs.c, d[0], d[1], heads * D, heads * D)
    sc.salicache_paged_read(ctx, pages.c, seqs.c, out[0], out[1], heads * D, heads * D)
    assert sc.salicache_poll_status(ctx) == 0
    return out.double().cpu().numpy().reshape(x.shape)


# Largest magnitudes (INT4 groups span twice that, which has to stay below binary32's 3.4e38), and smallest ones: their
# scales are the type's smallest normal numbers, whose reciprocals are still below binary32's largest.
@pytest.mark.parametrize("fmt,dt,largest", [
    ("int8", "bf16", 3.0e38), ("int8", "bf16", 1.0e33), ("int8", "bf16", 3.0e-36), ("int8", "f16", 6.0e4), ("int8", "f16", 9.0e-3),
    ("int4", "bf16", 1.6e38), ("int4", "bf16", 4.0e36), ("int4", "bf16", 3.0e35), ("int4", "bf16", 2.0e34), ("int4", "bf16", 1.0e33),
    ("int4", "bf16", 2.0e32), ("int4", "bf16", 3.0e-37), ("int4", "f16", 6.4e4), ("int4", "f16", 1.0e-3),
])
@pytest.mark.parametrize("D", [64, 128])
def test_written_and_read_at_the_ends_of_the_range(ctx, fmt, dt, largest, D):
    t = _t(dt)
    rng = np.random.default_rng(80)
    x = pu.to_t(rng.uniform(-largest, largest, (2, 21, 3, D)), t)
    x[..., 5], x[..., D - 3] = pu.to_t(np.array(largest), t), pu.to_t(np.array(-largest), t)
    want = pu.decode(*pu.encode(x, fmt, t), fmt, t)
    assert np.isfinite(want).all()
    assert np.array_equal(_stored(ctx, x, fmt, t), want)


@pytest.mark.parametrize("fmt", ["fp16", "int8", "int4"])
@pytest.mark.parametrize("dt", ["f16", "bf16"])
@pytest.mark.parametrize("D", [64, 128])
def test_a_group_that_is_not_finite_is_read_as_nan(ctx, fmt, dt, D):
    """All of it, wherever in it the NaN or the infinity stands, and none of its neighbours; 16-bit pages hold a copy."""
    t = _t(dt)
    rng = np.random.default_rng(81)
    x = pu.to_t(rng.standard_normal((2, 40, 5, D)), t)
    want = pu.decode(*pu.encode(x, fmt, t), fmt, t)
    at = 0
    for r, v in enumerate([[np.nan], [np.inf], [-np.inf], [np.inf, -np.inf], [np.nan, np.inf], [np.nan, np.nan]] * 6):
        for kv, h in ((0, 1), (1, 4)) if r % 2 else ((0, 3), (1, 0)):
            for a in v:
                at = (at * 5 + 3) % D
                x[kv, r, h, at] = a
            want[kv, r, h] = x[kv, r, h] if fmt == "fp16" else np.nan
    assert np.array_equal(_stored(ctx, x, fmt, t), want, equal_nan=True)


def test_a_span_past_binary32_is_read_as_nan(ctx):
    t = _t("bf16")
    x = pu.to_t(np.random.default_rng(82).standard_normal((2, 3, 2, 128)), t)
    x[0, 1, 0, 3], x[0, 1, 0, 90] = 3.0e38, -3.0e38
    x = pu.to_t(x, t)
    ordinary = x.copy()
    ordinary[0, 1, 0] = 0.0
    want = pu.decode(*pu.encode(ordinary, "int4", t), "int4", t)
    want[0, 1, 0] = np.nan
    assert np.array_equal(_stored(ctx, x, "int4", t), want, equal_nan=True)


def test_positions_from_two_to_the_thirtieth_on_are_in_no_page(ctx):
    """A table that reaches past them: they are dropped, come back as zeros and are left out, with E_CAPACITY each time."""
    import torch
    t, D, page, n = torch.float16, 64, 128, 10
    width = 2 ** 30 // page + 1
    table = torch.full((1, width), -1, dtype=torch.int32, device="cuda")
    table[0, -2:] = torch.tensor([1, 0], dtype=torch.int32)
    pages = sc.PageSet(2, page, 1, D, sc.FP16, t)
    seqs = sc.Seqs(_i32([0, n]), _i32([2 ** 30 + 4]), table, n)         # rows 0 .. 5 below 2^30
    x = torch.randn((3, n, D), device="cuda").to(t)
    sc.salicache_paged_write(ctx, pages.c, seqs.c, x[0], x[1], D, D)
    assert sc.salicache_poll_status(ctx) == sc.E_CAPACITY
    assert (pages.data[0] == 0).all()
    assert torch.equal(pages.data[1, :, 0, page - 6:], x[:2, :6])
    out = torch.full((2, n, D), 7.0, dtype=t, device="cuda")
    sc.salicache_paged_read(ctx, pages.c, seqs.c, out[0], out[1], D, D)
    assert sc.salicache_poll_status(ctx) == sc.E_CAPACITY
    assert torch.equal(out[:, :6], x[:2, :6]) and (out[:, 6:] == 0).all()
    # window 3: the row at position p sees p - 2 .. p, below 2^30
    work = torch.empty(sc.salicache_paged_work_bytes(ctx, pages.c, 1), dtype=torch.uint8, device="cuda")
    o, lse = torch.empty((n, D), dtype=t, device="cuda"), torch.empty((n, 1), device="cuda")
    sc.salicache_paged_attend(ctx, pages.c, seqs.c, x[2], D, 1, 0.125, 3, 0, o, D, lse, work, work.numel())
    assert sc.salicache_poll_status(ctx) == sc.E_CAPACITY
    q, k, v = (y.double().cpu().numpy() for y in (x[2], x[0], x[1]))
    for i in range(n):
        j = np.arange(max(0, i - 2), min(i + 1, 6))
        # positions before row 0 hold zeros: rows 0 and 1 see two and one of them
        z = np.zeros((max(0, 2 - i), D))
        kk, vv = (np.concatenate([z, y[j]]) for y in (k, v))
        want, wl, tol, ltol = pu.attend(q[i], kk, vv, 0.125, t, "fp16")
        pu.check(o[i].double().cpu().numpy(), want, tol, f"row {i}")
        pu.check(lse[i, 0].item(), wl, ltol, f"lse {i}")


@pytest.mark.parametrize("fmt", ["int8", "int4"])
def test_the_largest_f16_numbers_are_read_as_the_rounded_scale_makes_them(ctx, fmt):
    t = _t("f16")
    x = pu.to_t(np.random.default_rng(83).uniform(-6.0e4, 6.0e4, (2, 5, 2, 128)), t)
    x[:, 1:3, :, 9], x[:, 1:3, :, 70] = 65504.0, -65504.0
    with np.errstate(over="ignore"):
        want = pu.decode(*pu.encode(x, fmt, t), fmt, t)
    assert np.isinf(want[:, 1:3]).any(-1).all() and np.isfinite(want[:, [0, 3, 4]]).all()
    assert np.array_equal(_stored(ctx, x, fmt, t), want)
