"""GPU tests of the attention over the paged cache that are sharp where test_gpu_paged.py has to leave room: the values an INT4
page stands for, and the correction of sums that are not empty."""
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


def _round(x, t):
    """float64 to the nearest value of the 16-bit type, ties to even, in one step (torch goes through binary32)."""
    import torch
    bits, low = (11, -14) if t is torch.float16 else (8, -126)
    e = np.maximum(np.frexp(x)[1] - 1, low)                     # |x| in [2^e, 2^(e+1)), or below the normal numbers
    step = np.ldexp(1.0, e - (bits - 1))
    return np.rint(x / step) * step


def _int4_values(data, scale, t):
    """What attention takes an INT4 page's codes for: T(q * s + zero), rounded once."""
    q = data.numpy()
    q = np.stack([q & 15, q >> 4], -1).reshape(q.shape[:-1] + (-1,)).astype(np.float64)
    sz = scale.double().numpy()
    return _round(q * sz[..., :1] + sz[..., 1:], t)


class World(pu.World):
    """As in paged_util, with INT4 values rounded once, so that their bounds need no room for another rounding."""

    def __init__(self, seed, fmt, t, *a, **kw):
        super().__init__(seed, fmt, t, *a, **kw)
        self.set_values()

    def set_values(self):
        if self.fmt == "int4":
            self.values = np.nan_to_num(_int4_values(self.data, self.scale, self.t), nan=0.0, posinf=0.0, neginf=0.0)

    def expect(self, *a, **kw):
        fmt, self.fmt = self.fmt, "fp16" if self.fmt == "int4" else self.fmt
        try:
            return super().expect(*a, **kw)
        finally:
            self.fmt = fmt


def _call(ctx, pages, seqs, q, G, D, scale, window=0, sinks=0):
    """q: device [rows][heads * G * D]."""
    import torch
    out, lse = torch.full_like(q, 7.0), torch.full((q.shape[0], q.shape[1] // D), 7.0, device="cuda")
    work = torch.full((sc.salicache_paged_work_bytes(ctx, pages.c, G),), 255, dtype=torch.uint8, device="cuda")
    sc.salicache_paged_attend(ctx, pages.c, seqs.c, q, q.shape[1], G, scale, window, sinks, out, q.shape[1], lse, work, work.numel())
    assert sc.salicache_poll_status(ctx) == 0
    return out, lse


@pytest.mark.parametrize("dt,s,zero,code", [("f16", 4.36328125, -7.0e-7, 12), ("bf16", 1.0078125, -2.0 ** -30, 3)])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("G", [1, 12, 20])
def test_int4_values_are_rounded_once_in_attention_and_twice_when_read(ctx, dt, s, zero, code, D, G):
    """A row that sees one position gets its V as it is.  q * s lies midway between two values of the type, which a zero below
    binary32's last place decides where it is not rounded away first.  The groups beside it are random, small zeros among them."""
    import torch
    t = _t(dt)
    rng = np.random.default_rng(110)
    heads, page = 16, 16
    codes = rng.integers(0, 16, (1, 2, heads, page, D))
    codes[:, :, 0] = code
    scale = np.stack([rng.uniform(0.5, 8.0, codes.shape[:4]), -np.exp2(rng.uniform(-40, 3, codes.shape[:4]))], -1)
    scale[:, :, 0] = s, zero
    scale = torch.from_numpy(scale).to(t)
    data = torch.from_numpy((codes[..., 0::2] | codes[..., 1::2] << 4).astype(np.uint8))
    once = _int4_values(data, scale, t)
    sz = scale.double().numpy()
    twice = pu.decode(codes, sz[..., 0], sz[..., 1], "int4", t)
    assert (once[0, 1, 0, 0] != twice[0, 1, 0, 0]).all() and np.mean(once != twice) < 0.2
    i32 = lambda a: torch.tensor(a, dtype=torch.int32, device="cuda")
    pages = sc.PageSet(1, page, heads, D, sc.INT4, t, data=data.cuda(), scale=scale.cuda())
    seqs = sc.Seqs(i32([0, 1]), i32([1]), i32([[0]]), 1)
    q = torch.from_numpy(rng.standard_normal((1, heads * G * D)) * 0.1).to(t).cuda()
    out, _ = _call(ctx, pages, seqs, q, G, D, 0.1)
    got = out.double().cpu().numpy().reshape(heads, G, D)
    assert np.array_equal(got, np.repeat(once[0, 1, :, 0][:, None], G, 1))
    kv = torch.zeros((2, 1, heads * D), dtype=t, device="cuda")
    sc.salicache_paged_read(ctx, pages.c, seqs.c, kv[0], kv[1], heads * D, heads * D)
    assert np.array_equal(kv.double().cpu().numpy().reshape(2, heads, D), twice[0, :, :, 0])


@pytest.mark.parametrize("dt", ["f16", "bf16"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("G,lens,news,window,sinks", [
    (1, [1, 17, 129, 700], [1, 1, 1, 1], 0, 0), (4, [700, 2049], [1, 1], 300, 20), (4, [300, 900], [4, 3], 0, 0),
    (2, [513, 129, 5], [129, 40, 5], 0, 0), (5, [640], [300], 200, 130),
])
def test_int4_pages_at_the_bounds_of_values_rounded_once(ctx, dt, D, G, lens, news, window, sinks):
    import torch
    t = _t(dt)
    w = World(111, "int4", t, 2, D, 32, lens, news)
    pages, seqs = w.device()
    q = torch.from_numpy(np.random.default_rng(112).standard_normal((w.rows, 2 * G * D))).to(t)
    out, lse = _call(ctx, pages, seqs, q.cuda(), G, D, D ** -0.5, window, sinks)
    want, wl, tol, ltol = w.expect(q.double().numpy().reshape(w.rows, 2 * G, D), G, D ** -0.5, window, sinks)
    pu.check(out.double().cpu().numpy().reshape(want.shape), want, tol, "out")
    pu.check(lse.double().cpu().numpy(), wl, ltol, "lse")


def _bounds(q, k, v, seen, scale, t):
    """Rows of one head: q [R][D], k, v [n][D], seen [R][n] -> out, lse and their bounds, by the terms of paged_util.attend."""
    D, n, E = q.shape[1], k.shape[0], pu.eps(t)
    a = np.where(seen, scale * (q @ k.T), -np.inf)
    m = a.max(-1, keepdims=True)
    wts = np.exp(a - m)
    l = wts.sum(-1, keepdims=True)
    out, lse = wts @ v / l, (m + np.log(l))[:, 0]
    a_err = (scale * (np.abs(q) @ np.abs(k).T)).max(-1, keepdims=True) * (D + 2) * 2.0 ** -24
    rel = 2 * a_err + 2.0 ** -20 + (n + 8) * 2.0 ** -24
    tiny = n * 2.0 ** -25 * np.abs(v).max(0) if E < 2e-3 else 0.0
    tol = E / 2 * np.abs(out) * (1 + rel) + wts @ np.abs(v) / l * (E / 2 + rel) * 1.01 + tiny + 2.0 ** -24
    return out, lse, tol, a_err[:, 0] + 2.0 ** -20 + (n + 8) * 2.0 ** -24 + 2.0 ** -22 * np.abs(lse), a


# As many (sequence, head) items of eight tiles as there are blocks or more, so that a block works on most of an item: the scores
# of the first tiles are alike, and then single ones, in the groups of 16 keys of different warps, exceed them by more than the
# 2^8 (in powers of two) up to which the running maximum stays.  What was summed before keeps about half of the weight, so
# that its correction shows.
@pytest.mark.parametrize("fmt", ["fp16", "int8", "int4"])
@pytest.mark.parametrize("dt", ["f16", "bf16"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("G,new,B", [(2, 1, 50), (4, 4, 20), (2, 30, 20), (7, 30, 20)])
def test_a_jump_of_the_scores_corrects_what_was_summed(ctx, fmt, dt, D, G, new, B):
    import torch
    t = _t(dt)
    n, heads, page = 1000, 8, 16
    rng = np.random.default_rng(113)
    w = World(114, fmt, t, heads, D, page, [n], [new], spare=0)
    base = np.zeros(n)
    base[[128 * 4 + 50, 128 * 5 + 3, 128 * 6 + 115]] = 9.0 * np.log(2.0)
    k = pu.to_t(0.3 * rng.standard_normal((heads, n, D)) + base[:, None], t)
    codes, s, z = pu.encode(k, fmt, t)
    data, scale = pu.as_tensors(codes, s, z, fmt, t)
    held = pu.decode(codes, s, z, fmt, t)
    p = np.arange(n)
    at = (w.table[0, p // page], 0, slice(None), p % page)
    w.values[at] = held.transpose(1, 0, 2)
    w.data[at] = data.transpose(0, 1)
    if scale is not None:
        w.scale[at] = scale.transpose(0, 1)
    w.set_values()
    i32 = lambda a: torch.from_numpy(np.ascontiguousarray(a)).to(torch.int32).cuda()
    pages = sc.PageSet(w.n_pages, page, heads, D, pu.FMT[fmt], t, data=w.data.cuda(), scale=None if w.scale is None else w.scale.cuda())
    seqs = sc.Seqs(i32(np.arange(B + 1) * new), i32(np.full(B, n)), i32(np.repeat(w.table, B, 0)), B * new)
    q = pu.to_t((1.0 + 0.1 * rng.standard_normal((B * new, heads, G, D))) / D, t)
    out, lse = _call(ctx, pages, seqs, torch.from_numpy(q.reshape(B * new, -1)).to(t).cuda(), G, D, 1.0)
    got, gl = out.double().cpu().numpy().reshape(q.shape), lse.double().cpu().numpy().reshape(B * new, heads, G)
    pos = n - new + np.arange(B * new) % new
    seen = np.repeat(p[None] <= pos[:, None], G, 0)
    for h in range(heads):
        want, wl, tol, ltol, a = _bounds(q[:, h].reshape(-1, D), w.kv(0, h, 0), w.kv(0, h, 1), seen, 1.0, t)
        a = a / np.log(2.0)
        assert (a[:, 512:640].max(-1) > a[:, :512].max(-1) + 8.0).all()
        old = np.exp2(a[:, :512]).sum(-1) / np.exp2(a).sum(-1)
        assert ((old > 0.1) & (old < 0.6)).all()
        pu.check(got[:, h].reshape(-1, D), want, tol, f"out, head {h}")
        pu.check(gl[:, h].reshape(-1), wl, ltol, f"lse, head {h}")
