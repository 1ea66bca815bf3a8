"""GPU tests of rows that are turned by their positions on their way into the pages, against a plain form with 64-bit angles.

Bounds: the angle is right to 2^-27 half turns (within a quarter of a half turn it goes through binary32) and 2^-32 turns (what
is cut off), cosine and sine to 2 units in the last place, 2^-23, so that both are off by at most pi 2^-27 + pi 2^-31 + 2^-23 <
1.5e-7; one product and one fused step in binary32 add 2^-23 (|a| + |b|): together 2.7e-7 (|a| + |b|), and then the rounding to
the 16-bit type, half a step of the value, or of f16's subnormals."""
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


def turned(x, pos, freq, axis, pairing, t):
    """x float64 [rows][heads][D] -> what the rows become, and the bound; angles in numpy's long double."""
    n = len(freq)
    ld = np.longdouble
    turns = pos[:, axis].astype(ld) * (np.asarray(freq, ld) / (2 * ld("3.14159265358979323846264338327950288")))
    phi = ((turns - np.floor(turns)) * 2 * ld("3.14159265358979323846264338327950288")).astype(np.float64)[:, None]
    one, two = (slice(0, n), slice(n, 2 * n)) if pairing == sc.HALVES else (slice(0, 2 * n, 2), slice(1, 2 * n, 2))
    a, b = x[..., one], x[..., two]
    y, tol = x.copy(), np.zeros_like(x)
    y[..., one], y[..., two] = a * np.cos(phi) - b * np.sin(phi), b * np.cos(phi) + a * np.sin(phi)
    off = 2.7e-7 * (np.abs(a) + np.abs(b))
    for s in (one, two):
        tol[..., s] = off + pu.eps(t) / 2 * (np.abs(y[..., s]) + off) + (2.0 ** -25 if pu.eps(t) < 2e-3 else 0.0)
    return y, tol


def _positions(rng, kind, rows, axes):
    if kind == "near":
        return rng.integers(0, 4096, (rows, axes))
    if kind == "far":
        return rng.integers(10 ** 6, 10 ** 9, (rows, axes))
    x = rng.choice([0, 1, -1, 2 ** 31 - 1, -2 ** 31, 2 ** 30, -12345], (rows, axes))
    return x


def _bits(x):
    import torch
    return x.contiguous().view(torch.int16 if x.element_size() == 2 else torch.uint8)


@pytest.mark.parametrize("fmt", ["fp16", "int8", "int4"])
@pytest.mark.parametrize("dt", ["f16", "bf16"])
@pytest.mark.parametrize("heads,G,D,page,lens,news,pairs,axes,pairing,kind", [
    (2, 4, 128, 16, [5, 16, 33, 0, 40], [5, 1, 17, 0, 3], 64, 3, sc.HALVES, "near"),
    (5, 1, 64, 32, [70, 1], [37, 1], 32, 1, sc.NEIGHBOURS, "far"),
    (8, 3, 128, 128, [300], [300], 48, 2, sc.HALVES, "far"),
    (1, 7, 64, 16, [1], [1], 8, 4, sc.HALVES, "ends"),
    (3, 2, 128, 64, [90, 7], [33, 7], 8, 4, sc.NEIGHBOURS, "ends"),
    (12, 0, 64, 64, [40], [21], 24, 3, sc.HALVES, "near"),
])
def test_rows_are_turned(ctx, fmt, dt, heads, G, D, page, lens, news, pairs, axes, pairing, kind):
    import torch
    t, rng = _t(dt), np.random.default_rng(7)
    w = pu.World(3, fmt, t, heads, D, page, lens, news)
    pages, seqs = w.device(extra_rows=3)
    R, HD, pad = w.rows + 3, heads * D, 24
    freq = 10.0 ** rng.uniform(-4, 0.3, pairs) * rng.choice([1, 1, -1], pairs)
    axis = rng.integers(0, axes, pairs)
    pos = _positions(rng, kind, R, axes)
    x = torch.from_numpy(rng.standard_normal((R, 2 * HD + pad)) * 2).to(t).cuda()
    rotary = sc.Rotary(freq, axis, axes, pairing)
    dpos = torch.from_numpy(pos).to(torch.int32).cuda()
    q = q_out = None
    if G:
        q = torch.from_numpy(rng.standard_normal((R, HD * G + pad))).to(t).cuda()
        q_out = torch.full((R, HD * G + 8), 7.0, dtype=t, device="cuda")
    # K's rows turned by the call itself: as the q of a call into pages nobody looks at
    other, _ = w.device(extra_rows=3)
    k_turned = torch.zeros((R, HD), dtype=t, device="cuda")
    sc.salicache_paged_write_rotary(ctx, other.c, seqs.c, rotary, dpos, x, 2 * HD + pad, 1, k_turned, HD, x, x[:, HD:], 2 * HD + pad, 2 * HD + pad)
    sc.salicache_paged_write_rotary(ctx, pages.c, seqs.c, rotary, dpos, q, HD * G + pad, G, q_out, HD * G + 8, x, x[:, HD:], 2 * HD + pad, 2 * HD + pad)
    assert sc.salicache_poll_status(ctx) == 0
    n = w.rows
    want, tol = turned(x[:n, :HD].double().cpu().numpy().reshape(n, heads, D), pos[:n], freq, axis, pairing, t)
    pu.check(k_turned[:n].double().cpu().numpy().reshape(n, heads, D), want, tol, "k")
    assert (k_turned[n:] == 0).all()
    if G:
        want, tol = turned(q[:n, :HD * G].double().cpu().numpy().reshape(n, heads * G, D), pos[:n], freq, axis, pairing, t)
        pu.check(q_out[:n, :HD * G].double().cpu().numpy().reshape(n, heads * G, D), want, tol, "q")
        assert (q_out[n:] == 7).all() and (q_out[:, HD * G:] == 7).all()
    # what the pages hold is what the store makes of the turned rows
    plain, _ = w.device(extra_rows=3)
    sc.salicache_paged_write(ctx, plain.c, seqs.c, k_turned, x[:, HD:], HD, 2 * HD + pad)
    assert torch.equal(_bits(pages.data), _bits(plain.data))
    assert pages.scale is None or torch.equal(_bits(pages.scale), _bits(plain.scale))


@pytest.mark.parametrize("pairing", [sc.HALVES, sc.NEIGHBOURS])
def test_what_is_not_turned_keeps_its_bits(ctx, pairing):
    """Infinities and NaN beyond the pairs stay where they are and touch nothing; position 0 turns nothing."""
    import torch
    t = torch.float16
    w = pu.World(3, "fp16", t, 2, 128, 16, [20], [20])
    pages, seqs = w.device()
    rng = np.random.default_rng(1)
    x = torch.from_numpy(rng.standard_normal((20, 2, 128))).to(t).cuda()
    x[:, :, 32:] = torch.tensor([float("inf"), float("nan"), -0.0, 1.5], dtype=t, device="cuda").repeat(24)
    out = torch.empty_like(x)
    pos = torch.zeros((20, 1), dtype=torch.int32, device="cuda")
    pos[10:] = 5
    sc.salicache_paged_write_rotary(ctx, pages.c, seqs.c, sc.Rotary([0.3] * 16, pairing=pairing), pos, x, 256, 1, out, 256, x, x, 256, 256)
    assert sc.salicache_poll_status(ctx) == 0
    assert torch.equal(_bits(out[:, :, 32:]), _bits(x[:, :, 32:]))
    assert torch.equal(_bits(out[:10]), _bits(x[:10])) and torch.isfinite(out[:, :, :32]).all()
    assert not torch.equal(out[10:, :, :32], x[10:, :, :32])


def test_q_in_place_and_turned_back(ctx):
    """In place; and negated frequencies turn back, which is also what a gradient of the rows takes: up to two roundings."""
    import torch
    t = torch.bfloat16
    w = pu.World(3, "int8", t, 4, 64, 32, [100], [77])
    pages, seqs = w.device()
    rng = np.random.default_rng(2)
    q = torch.from_numpy(rng.standard_normal((77, 4 * 2 * 64))).to(t).cuda()
    k = torch.from_numpy(rng.standard_normal((77, 256))).to(t).cuda()
    pos = torch.from_numpy(rng.integers(0, 10 ** 6, (77, 2))).to(torch.int32).cuda()
    freq, axis = 10.0 ** rng.uniform(-4, 0, 32), rng.integers(0, 2, 32)
    fwd, back = sc.Rotary(freq, axis, 2), sc.Rotary(-freq, axis, 2)
    apart, same = torch.empty_like(q), q.clone()
    for out, src in ((apart, q), (same, same)):
        sc.salicache_paged_write_rotary(ctx, pages.c, seqs.c, fwd, pos, src, 512, 2, out, 512, k, k, 256, 256)
    assert torch.equal(apart, same)
    sc.salicache_paged_write_rotary(ctx, pages.c, seqs.c, back, pos, same, 512, 2, same, 512, k, k, 256, 256)
    assert sc.salicache_poll_status(ctx) == 0
    norm = torch.hypot(*[x.double() for x in q.view(77, 8, 2, 32).unbind(2)])
    err = (same.double() - q.double()).abs().view(77, 8, 2, 32)
    # each way rounds a pair's two values by half a step of at most its length; the second way turns the first's error along
    assert (err <= (norm * (2.0 ** -8 * (1 + 2 ** 0.5) * 1.01 + 2e-6))[:, :, None]).all()


def test_rows_without_a_page_and_before_the_first_sequence(ctx):
    import torch
    t = torch.float16
    w = pu.World(3, "fp16", t, 2, 64, 16, [40, 30], [20, 10])
    pages, seqs = w.device()
    table = w.table.copy()
    table[0, 1] = -1                                     # positions 16 .. 31 of the first sequence
    i32 = lambda a: torch.from_numpy(np.ascontiguousarray(a)).to(torch.int32).cuda()
    seqs = sc.Seqs(i32(w.start + 4), i32(np.array([40, 6])), i32(table), 36)      # four rows before the first; the second: 10 rows, 6 positions
    rng = np.random.default_rng(2)
    x = torch.from_numpy(rng.standard_normal((36, 128))).to(t).cuda()
    out = torch.full_like(x, 7.0)
    before = pages.data.clone()
    pos = torch.arange(36, dtype=torch.int32, device="cuda")[:, None].contiguous()
    freq = 10.0 ** rng.uniform(-3, 0, 32)
    sc.salicache_paged_write_rotary(ctx, pages.c, seqs.c, sc.Rotary(freq), pos, x, 128, 1, out, 128, x, x, 128, 128)
    assert sc.salicache_poll_status(ctx) == sc.E_CAPACITY
    assert (out[:4] == 7).all() and (out[34:] == 7).all()
    want, tol = turned(x[4:34].double().cpu().numpy().reshape(30, 2, 64), pos[4:34].cpu().numpy(), freq, np.zeros(32, int), sc.HALVES, t)
    pu.check(out[4:34].double().cpu().numpy().reshape(30, 2, 64), want, tol, "q")
    changed = (_bits(pages.data) != _bits(before)).view(before.shape).any(-1).any(1).any(1)            # [pages][slot]
    should = np.zeros((w.n_pages, 16), bool)
    for p in range(32, 40):
        should[w.table[0, p // 16], p % 16] = True
    for p in range(6):
        should[w.table[1, p // 16], p % 16] = True
    assert np.array_equal(changed.cpu().numpy(), should)


def test_captured_and_replayed_with_other_lengths_and_positions(ctx):
    import torch
    t = torch.bfloat16
    w = pu.World(3, "int4", t, 2, 128, 16, [64, 64], [3, 1])
    pages, seqs = w.device()
    rng = np.random.default_rng(2)
    x = torch.from_numpy(rng.standard_normal((4, 256))).to(t).cuda()
    pos, out = torch.zeros((4, 1), dtype=torch.int32, device="cuda"), torch.empty_like(x)
    rotary = sc.Rotary(10.0 ** rng.uniform(-3, 0, 64))
    call = lambda: sc.salicache_paged_write_rotary(ctx, pages.c, seqs.c, rotary, pos, x, 256, 1, out, 256, x, x, 256, 256)
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            call()
    again = sc.Rotary(list(rotary.freq)[:64])
    rotary.freq[0] = 99.0                                # read during the call, not at the replay
    for lens in ([64, 64], [50, 17]):
        seqs.length.copy_(torch.tensor(lens))
        pos.copy_(torch.tensor([[lens[0] - 3], [lens[0] - 2], [5], [lens[1]]]))
        g.replay()
        torch.cuda.synchronize()
        a, b, c = out.clone(), pages.data.clone(), pages.scale.clone()
        out.zero_()
        pages.data.zero_()
        sc.salicache_paged_write_rotary(ctx, pages.c, seqs.c, again, pos, x, 256, 1, out, 256, x, x, 256, 256)
        torch.cuda.synchronize()
        assert torch.equal(_bits(a), _bits(out)) and not (a == 0).all()
        new = pages.data != 0
        assert new.any() and torch.equal(b[new], pages.data[new]) and torch.equal(_bits(c), _bits(pages.scale))
    assert sc.salicache_poll_status(ctx) == 0
