"""Plain 64-bit forms of the paged cache and of the attention over it, and the bounds the kernels are held to.

The cache is built here on the host (numpy float32 steps in the order the header states, values in float64) and copied to
the device, so the attention tests do not rest on the library's own store."""
from __future__ import annotations

import numpy as np

FMT = {"fp16": 4, "int8": 3, "int4": 2}


def to_t(x, t):
    """float -> the 16-bit type and back, as float64 (numpy has no bf16: torch rounds)."""
    import torch
    return torch.from_numpy(np.ascontiguousarray(x, np.float64)).to(torch.float32).to(t).double().numpy()


def eps(t):
    import torch
    return float(torch.finfo(t).eps)


def encode(x, fmt, t):
    """x float64 [..., D] holding values of type t -> (codes, scale or None, zero or None), float64 / int."""
    f = x.astype(np.float32)
    if fmt == "fp16":
        return x, None, None
    if fmt == "int8":
        s = to_t((np.abs(f).max(-1) / np.float32(127)).astype(np.float32), t)
        s[s == 0] = 1.0
        inv = (np.float32(1) / s.astype(np.float32)).astype(np.float32)
        q = np.clip(np.rint((f * inv[..., None]).astype(np.float32)), -127, 127)
        return q.astype(np.int64), s, None
    z = f.min(-1)
    s = to_t(((f.max(-1) - z).astype(np.float32) / np.float32(15)).astype(np.float32), t)
    s[s == 0] = 1.0
    inv = (np.float32(1) / s.astype(np.float32)).astype(np.float32)
    d = (f - z[..., None]).astype(np.float32)
    q = np.clip(np.rint((d * inv[..., None]).astype(np.float32)), 0, 15)
    return q.astype(np.int64), s, z.astype(np.float64)


def decode(codes, s, z, fmt, t):
    if fmt == "fp16":
        return codes
    y = (codes.astype(np.float32) * s.astype(np.float32)[..., None]).astype(np.float32)
    if fmt == "int4":
        y = (y + z.astype(np.float32)[..., None]).astype(np.float32)
    return to_t(y, t)


def as_tensors(codes, s, z, fmt, t):
    """Host arrays of encode() -> (data, scale) tensors in the documented layout."""
    import torch
    if fmt == "fp16":
        return torch.from_numpy(codes).to(t), None
    if fmt == "int8":
        return torch.from_numpy(codes.astype(np.int8)), torch.from_numpy(s).to(t)
    packed = (codes[..., 0::2] | (codes[..., 1::2] << 4)).astype(np.uint8)
    return torch.from_numpy(packed), torch.stack([torch.from_numpy(s), torch.from_numpy(z)], -1).to(t)


def visible(p, length, window, sinks):
    """Positions the row at position p sees."""
    j = np.arange(max(0, min(p + 1, length)))
    return j[(j > p - window) | (j < sinks)] if window else j


def attend(q, k, v, scale, t, fmt):
    """One row of one head: q [D], k, v [n][D] -> out [D], lse, and the bounds of both.

    With E the 16-bit type's eps: a rounding to it is off by E/2 of the value, one to binary32 by 2^-24.
      scores   a 128-term binary32 sum of exact products, then the scale: (D + 2) 2^-24 sum|q k| scale each; the INT4
               values come from one fused step on the device and two here, which can differ by one step (E) of a value
      weights  their relative error is twice the score's, plus 2^-20 for the exponential (its argument, a product of up to
               2^7 in magnitude, is rounded to binary32), plus E/2 for the rounding to the 16-bit type; below the f16
               normals that rounding is 2^-25 absolute against a denominator of at least 1
      sums     n terms in binary32; the output's own rounding
    """
    D, n = q.shape[0], k.shape[0]
    E = eps(t)
    if n == 0:
        return np.zeros(D), -np.inf, np.zeros(D), 0.0
    a = scale * (k @ q)
    m = a.max()
    w = np.exp(a - m)
    l = w.sum()
    out, lse = (w @ v) / l, m + np.log(l)
    a_err = (scale * (np.abs(k) @ np.abs(q))).max() * (D + 2) * 2.0 ** -24
    if fmt == "int4":
        a_err += scale * (np.abs(k) * np.abs(q)).max() * E
    wabs = (w @ np.abs(v)) / l
    tiny = n * 2.0 ** -25 * np.abs(v).max(0) if E < 2e-3 else 0.0
    rel = 2 * a_err + 2.0 ** -20 + (n + 8) * 2.0 ** -24
    out_tol = E / 2 * np.abs(out) * (1 + rel) + wabs * (E / 2 + rel + (E if fmt == "int4" else 0.0)) * 1.01 + tiny + 2.0 ** -24
    return out, lse, out_tol, a_err + 2.0 ** -20 + (n + 8) * 2.0 ** -24 + 2.0 ** -22 * abs(lse)


class World:
    """Random sequences over shuffled pages, on the host, with what no row may read filled with NaN (16-bit pages) or
    wild scales."""

    def __init__(self, seed, fmt, t, heads, D, page, lens, news, spare=2, outliers=True):
        import torch
        rng = np.random.default_rng(seed)
        self.rng, self.fmt, self.t, self.heads, self.D, self.page = rng, fmt, t, heads, D, page
        self.lens, self.news = list(lens), list(news)
        B = len(lens)
        counts = [-(-n // page) for n in lens]
        self.width = max(max(counts + [0]), 1)
        self.n_pages = sum(counts) + spare
        order = rng.permutation(self.n_pages)
        self.table = np.full((B, self.width), 2 ** 31 - 1, np.int64)       # behind the end: no valid id
        at = 0
        for b, c in enumerate(counts):
            self.table[b, :c] = order[at:at + c]
            at += c
        x = rng.standard_normal((self.n_pages, 2, heads, page, D))
        if outliers:
            x = np.where(rng.random(x.shape) < 0.01, 8 * x, x)
        codes, s, z = encode(to_t(x, t), fmt, t)
        self.values = decode(codes, s, z, fmt, t)                          # [n_pages][2][heads][page][D]
        free = np.ones((self.n_pages, page), bool)
        for b, n in enumerate(lens):
            for p in range(n):
                free[self.table[b, p // page], p % page] = False
        if fmt == "fp16":
            codes = codes.copy()
            codes.transpose(0, 3, 1, 2, 4)[free] = np.nan
        else:
            s = s.copy()
            s.transpose(0, 3, 1, 2)[free] = np.nan
            if z is not None:
                z = z.copy()
                z.transpose(0, 3, 1, 2)[free] = np.inf
        self.data, self.scale = as_tensors(codes, s, z, fmt, t)
        self.start = np.concatenate([[0], np.cumsum(self.news)]).astype(np.int64)
        self.rows = int(self.start[-1])

    def kv(self, b, h, kv):
        """[len][D] float64: what the pages stand for."""
        p = np.arange(self.lens[b])
        return self.values[self.table[b, p // self.page], kv, h, p % self.page]

    def device(self, extra_rows=0):
        import torch
        from paper_2602_14236_b200 import binding as sc
        i32 = lambda a: torch.from_numpy(np.ascontiguousarray(a)).to(torch.int32).cuda()
        pages = sc.PageSet(self.n_pages, self.page, self.heads, self.D, FMT[self.fmt], self.t, data=self.data.cuda(),
                           scale=None if self.scale is None else self.scale.cuda())
        return pages, sc.Seqs(i32(self.start), i32(np.array(self.lens)), i32(self.table), self.rows + extra_rows)

    def expect(self, q, G, scale, window, sinks, rows=None, missing=()):
        """Every row's (out, lse, bounds) for q float64 [rows][heads * G][D]; `missing`: (sequence, page index) without a page."""
        R = self.rows if rows is None else rows
        Hq = self.heads * G
        out, tol = np.zeros((R, Hq, self.D)), np.zeros((R, Hq, self.D))
        lse, ltol = np.full((R, Hq), -np.inf), np.zeros((R, Hq))
        gone = {}
        for b, i in missing:
            gone.setdefault(b, set()).add(i)
        for b in range(len(self.lens)):
            for h in range(self.heads):
                k, v = self.kv(b, h, 0), self.kv(b, h, 1)
                for i in range(self.news[b]):
                    r, p = int(self.start[b]) + i, self.lens[b] - self.news[b] + i
                    j = visible(p, self.lens[b], window, sinks)
                    if b in gone:
                        j = j[[x // self.page not in gone[b] for x in j]] if j.size else j
                    for g in range(G):
                        hq = h * G + g
                        out[r, hq], lse[r, hq], tol[r, hq], ltol[r, hq] = attend(q[r, hq], k[j], v[j], scale, self.t, self.fmt)
        return out, lse, tol, ltol


def check(got, want, tol, what):
    got = np.asarray(got, np.float64)
    same = (got == want) | (np.abs(got - want) <= tol)
    assert same.all(), f"{what}: {(~same).sum()} of {same.size} beyond the bound, worst ratio " \
                       f"{np.nanmax(np.where(same, 0, np.abs(got - want) / np.maximum(tol, 1e-300))):.3g}, first at {np.argwhere(~same)[0]}"
