"""Positions, drafted trees and eviction for the paged K/V cache.

A batch of sequences shares pages.  Sequence b's position p lives in slot p % page of page table[b][p // page]; the rows
row_start[b] .. row_start[b+1] of the caller's arrays are the last positions of its length[b].

  rotate   new rows' q and K are turned by their positions on several axes (time, height, width), and K and V go into the pages
  tree     softmax attention of drafted tokens that form a tree: a row sees what was cached before and, of the rows of its own
           call, those that its bits name (its ancestors and itself)
  weigh    what attention gave each cached position, summed over the rows and the query heads of a key/value head, is added
           to what it had before: the weight that eviction goes by
  evict    of every key/value head the heaviest positions are selected, with the first and the last ones kept in any case,
           and gathered into other pages

Lengths are texts ("old" = positions cached before, "new" = rows of this call, one number per sequence).
"""
import math
import random

import torch

own = False
DEVICE = "cuda"

TYPES = {"f16": torch.float16, "bf16": torch.bfloat16}
BYTES = {"fp16": 2.0, "int8": 1.0, "int4": 0.5}           # a stored element
META = {"fp16": 0, "int8": 2, "int4": 4}                  # scale (and zero) of one head of one token


def _case(name, kind, fmt, dtype, heads, q_per_kv, head_dim, page, old, new, **more):
    return dict(name=name, kind=kind, format=fmt, dtype=dtype, heads=heads, q_per_kv=q_per_kv, head_dim=head_dim, page=page,
                old=old, new=new, **more)


def listed():
    return [
        # one token of each of 32 streams, its question after the frames: launch latency
        _case("rotate_step_bf16", "rotate", "fp16", "bf16", 8, 4, 128, 64,
              "611,1187,16383,9000,12012,15001,577,2303,90,576,16,4031,14400,13824,11111,1,8191,10001,15555,6912,5184,16000,"
              "12345,3456,7777,100,9999,14001,8640,13579,2880,11520", ",".join(["1"] * 32),
              axes=3, sections="16,24,24", rotary_dim=128, pairing="halves", base=1e6, far=0),
        # four 672x672 frames (2880 visual tokens each) of four streams, quantised, and what attention is to see of them
        _case("rotate_frames_int4", "rotate", "int4", "f16", 8, 4, 128, 64, "2880,0,5760,61", "2880,2880,2880,2880",
              axes=3, sections="16,24,24", rotary_dim=128, pairing="halves", base=1e6, far=0),
        # ragged prompts, one of them empty; small heads of which a half turns, neighbouring pairs, far positions on one axis
        _case("rotate_prompts_f16", "rotate", "fp16", "f16", 12, 1, 64, 32, "0,300,17,0,1000,5", "1153,0,37,577,2,4095",
              axes=1, sections="16", rotary_dim=32, pairing="neighbours", base=1e4, far=1000000),
        # a draft of nine tokens for one stream after one frame and a short question: latency
        _case("tree_draft_f16", "tree", "fp16", "f16", 8, 4, 128, 16, "611", "9", window=0, sinks=0),
        # drafts of very different sizes for streams that keep a window and the first tokens; small heads
        _case("tree_window_int8", "tree", "int8", "bf16", 4, 6, 64, 64, "32767,20001,4099,577,31999,28800,0,4100,17280,30000,25001,8191",
              "17,64,1,33,8,0,12,26,5,48,63,31", window=4096, sinks=4),
        # drafts of up to 64 tokens for eight streams with long videos behind them
        _case("tree_streams_bf16", "tree", "fp16", "bf16", 8, 4, 128, 64, "16128,8000,11520,14400,17280,9216,12672,15001", "64,25,60,48,26,64,31,57",
              window=0, sinks=0),
        # one token of each of 32 streams
        _case("weigh_step_int4", "weigh", "int4", "f16", 8, 4, 128, 64,
              "611,1187,16383,9000,12012,15001,577,2303,90,576,16,4031,14400,13824,11111,1,8191,10001,15555,6912,5184,16000,"
              "12345,3456,7777,100,9999,14001,8640,13579,2880,11520", ",".join(["1"] * 32), decay=1.0),
        # four more frames of two streams over what was kept of the earlier ones; a stream with nothing new
        _case("weigh_frames_int8", "weigh", "int8", "f16", 8, 4, 128, 64, "20736,577,6912", "2304,0,2304", decay=0.9),
        # a whole prompt at once
        _case("weigh_prompt_bf16", "weigh", "fp16", "bf16", 8, 4, 128, 128, "0", "8192", decay=1.0),
        # two short streams that have outgrown a frame's worth of tokens, and one that has not: latency
        _case("evict_short_f16", "evict", "fp16", "f16", 8, 1, 128, 16, "640,611,90", "0,0,0", budget=576, sinks=4, recent=64),
        # eight streams go back to their budget; quantised pages, and what attention is to see of them
        _case("evict_streams_int4", "evict", "int4", "f16", 8, 1, 128, 64, "4352,4300,2304,4099,4352,5760,8640,4097", "0,0,0,0,0,0,0,0",
              budget=4096, sinks=4, recent=512),
        # prompts of whole videos are cut down after they have been read
        _case("evict_prompts_bf16", "evict", "fp16", "bf16", 8, 1, 128, 128, "32768,17280,28800,8192", "0,0,0,0", budget=8192, sinks=64, recent=1024),
    ]


def _log(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    while True:
        kind = rng.choice(["rotate", "tree", "tree", "weigh", "weigh", "evict"])
        seqs = _log(rng, 1, 32)
        old = [0 if rng.random() < 0.05 else _log(rng, 1, 32768) for _ in range(seqs)]
        few = rng.random() < 0.4
        most = {"rotate": 1 if few else 8192, "tree": 64, "weigh": 1 if few else 8192, "evict": 0}[kind]
        new = [0 if most == 0 or rng.random() < 0.05 else _log(rng, 1, most) for _ in range(seqs)]
        if kind == "evict":
            old[0] = max(old[0], 1)
        else:
            new[0] = max(new[0], 1)
        case = dict(kind=kind, format=rng.choice(["fp16", "int8", "int4"]), dtype=rng.choice(["f16", "bf16"]),
                    heads=rng.choice([1, 2, 4, 5, 8, 12, 16, 32]), q_per_kv=1 if kind == "evict" else rng.choice([1, 1, 2, 3, 4, 4, 6, 8]),
                    head_dim=rng.choice([64, 128, 128]), page=rng.choice([16, 32, 64, 128]), old=",".join(map(str, old)),
                    new=",".join(map(str, new)))
        D = case["head_dim"]
        if kind == "rotate":
            turned = rng.choice([D, D, D // 2, D // 4 * 3])
            axes = rng.choice([1, 2, 3, 3, 4])
            cuts = sorted(rng.sample(range(1, turned // 2), axes - 1))
            case |= dict(axes=axes, sections=",".join(str(b - a) for a, b in zip([0] + cuts, cuts + [turned // 2])), rotary_dim=turned,
                         pairing=rng.choice(["halves", "neighbours"]), base=rng.choice([1e4, 5e5, 1e6]), far=rng.choice([0, 0, 1000000]))
        if kind == "tree":
            window = rng.random() < 0.3
            case |= dict(window=_log(rng, 16, 8192) if window else 0, sinks=rng.choice([0, 1, 4, 64, 200]) if window else 0)
        if kind == "weigh":
            case |= dict(decay=rng.choice([1.0, 1.0, 0.9, 0.0]))
        if kind == "evict":
            budget = _log(rng, 32, 16384)
            case |= dict(budget=budget, sinks=rng.choice([0, 1, 4, budget // 8]), recent=rng.choice([0, 1, budget // 8, budget // 2]))
        longest = max(o + n for o, n in zip(old, new))
        scores = seqs * case["heads"] * case["q_per_kv"] * max(new) * longest if kind in ("tree", "weigh") else 0
        cells = seqs * longest * case["heads"] * D
        w = work(case)
        if scores <= 3.0e9 and cells <= 5.4e8 and w["bytes"] <= 2.8e8 and w["flops"] <= 5.0e11:
            return case


def _lengths(case):
    return tuple([int(x) for x in case[k].split(",")] for k in ("old", "new"))


def work(case):
    old, new = _lengths(case)
    H, D, G = case["heads"], case["head_dim"], case["q_per_kv"]
    stored = 2 * H * (D * BYTES[case["format"]] + META[case["format"]])      # bytes of a token in the pages, K and V
    dense = 2 * H * D * 2                                                    # ... in the caller's arrays
    back = 0 if case["format"] == "fp16" else stored + dense                 # codes are read back
    n = sum(new)
    if case["kind"] == "rotate":
        turned = (H * G + H) * case["rotary_dim"] // 2
        return {"bytes": n * (2 * H * G * D * 2 + dense + stored + back + 4 * case["axes"]), "flops": n * (6 * turned + 2 * H * D * 4)}
    if case["kind"] == "evict":
        kept = sum(min(o, case["budget"]) for o in old)
        return {"bytes": 4 * H * sum(old) + H * kept * (4 + 8) + kept * (2 * stored + back), "flops": H * sum(old)}
    pairs = keys = 0
    for o, m in zip(old, new):
        if m == 0:
            continue
        if case["kind"] == "weigh":
            pairs += m * o + m * (m + 1) // 2
            keys += o + m
        else:
            W, S = case["window"], case["sinks"]
            first = max(0, o - W + 1) if W else 0                            # the first position inside the first row's window
            keys += min(S, first) + (o + m - first)
            pairs += m * (min(S, first) + o - first + (1 + m) // 2)
    if case["kind"] == "weigh":
        return {"bytes": keys * stored / 2 + n * H * G * (2 * D + 4) + 8 * H * (sum(old) + n), "flops": 2 * pairs * H * G * D}
    return {"bytes": keys * stored + n * H * G * (4 * D + 4) + 8 * n, "flops": 4 * pairs * H * G * D}


# ---- the quantisers, one group = the last dimension: binary32 steps, stored scale (and zero) in the 16-bit type

def _encode(x, fmt):
    """16-bit rows -> (codes, scale or (scale, zero) or None) as the pages hold them."""
    t = x.dtype
    if fmt == "fp16":
        return x, None
    f = x.float()
    if fmt == "int8":
        s = (f.abs().amax(-1) / 127.0).to(t)
        s = torch.where(s == 0, torch.ones_like(s), s)
        q = torch.round(f * (1.0 / s.float())[..., None]).clamp(-127, 127)
        return q.to(torch.int8), s
    z = f.amin(-1)
    s = ((f.amax(-1) - z) / 15.0).to(t)
    s = torch.where(s == 0, torch.ones_like(s), s)
    q = torch.round((f - z[..., None]) * (1.0 / s.float())[..., None]).clamp(0, 15).to(torch.uint8)
    return q[..., 0::2] | (q[..., 1::2] << 4), torch.stack([s, z.to(t)], -1)


def _decode(data, scale, fmt, t):
    """What the pages stand for, in the 16-bit type."""
    if fmt == "fp16":
        return data
    if fmt == "int8":
        return (data.float() * scale.float()[..., None]).to(t)
    q = torch.stack([data & 15, data >> 4], -1).flatten(-2).float()
    return (q * scale[..., 0].float()[..., None] + scale[..., 1].float()[..., None]).to(t)


# ---- inputs

def _values(shape, t, g):
    """Normal values with one element in a hundred eight times as large."""
    x = torch.randn(shape, generator=g, device=DEVICE, dtype=torch.float32)
    x = torch.where(torch.rand(shape, generator=g, device=DEVICE) < 0.01, 8.0 * x, x)
    return x.to(t)


def _frequencies(case):
    """Radians per position of every pair, and the axis whose position turns it."""
    turned = case["rotary_dim"]
    sections = [int(x) for x in case["sections"].split(",")]
    return ([case["base"] ** (-2.0 * i / turned) for i in range(turned // 2)], [a for a, n in enumerate(sections) for _ in range(n)])


def _positions(case, old, new):
    """A frame's tokens stand on a grid of 24 x 24; on further axes, and where there is one, positions go on one by one."""
    p = torch.cat([torch.arange(o, o + n) for o, n in zip(old, new)])
    axes = {1: [p], 2: [p // 24, p % 24], 3: [p // 576, p // 24 % 24, p % 24]}.get(case["axes"], [p // 576, p // 24 % 24, p % 24, p])
    return (torch.stack(axes, -1) + case["far"]).to(torch.int32).to(DEVICE)


def _trees(new, seed):
    """Every row's ancestors and itself as bits of a 64-bit word: some drafts are chains, most branch at their last tokens."""
    rng, bits = random.Random(seed), []
    for n in new:
        mine = []
        for i in range(n):
            parent = rng.randint(max(-1, i - 1 - 2 ** rng.randint(0, 4)), i - 1)
            mine.append((mine[parent] if parent >= 0 else 0) | 1 << i)
        bits += mine
    return torch.tensor([b - (1 << 64) if b >> 63 else b for b in bits], dtype=torch.int64, device=DEVICE)


def _sums(state, old, new):
    """The logarithm of every row's softmax sum, as attention over the pages returns it: [rows][heads * q_per_kv]."""
    case = state["case"]
    H, D, G, page = (case[k] for k in ("heads", "head_dim", "q_per_kv", "page"))
    lse = torch.empty((sum(new), H * G), device=DEVICE)
    first = 0
    for b, (o, n) in enumerate(zip(old, new)):
        if n:
            ids = state["table"][b, : -(-(o + n) // page)].long()
            k = _decode(state["data"][ids, 0], None if state["scale"] is None else state["scale"][ids, 0], case["format"], TYPES[case["dtype"]])
            k = k.transpose(1, 2).reshape(-1, H, D)[: o + n].float().permute(1, 2, 0)
            j = torch.arange(o + n, device=DEVICE)
            for i0 in range(0, n, 512):
                i1 = min(n, i0 + 512)
                q = state["q"][first + i0:first + i1].float().view(i1 - i0, H, G, D).transpose(0, 1)
                a = torch.matmul(q.reshape(H, -1, D), k).view(H, i1 - i0, G, -1) * D ** -0.5
                a.masked_fill_((j > torch.arange(o + i0, o + i1, device=DEVICE)[:, None])[None, :, None], -math.inf)
                lse[first + i0:first + i1] = torch.logsumexp(a, -1).permute(1, 0, 2).reshape(i1 - i0, -1)
        first += n
    return lse


def prepare(case, seed):
    old, new = _lengths(case)
    H, D, G, page, fmt, kind = (case[k] for k in ("heads", "head_dim", "q_per_kv", "page", "format", "kind"))
    t = TYPES[case["dtype"]]
    g = torch.Generator(device=DEVICE).manual_seed(seed)
    length = [o + n for o, n in zip(old, new)]
    kept = [min(n, case["budget"]) for n in length] if kind == "evict" else []
    counts, counts_out = [-(-n // page) for n in length], [-(-n // page) for n in kept]
    used, n_pages = sum(counts), sum(counts) + sum(counts_out) + 3
    order = torch.randperm(n_pages, generator=g, device=DEVICE).to(torch.int32)
    rows = sum(new)
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device=DEVICE)

    def table_of(n, ids):
        width = max(max(n), 1)
        table = torch.full((len(n), width), -1, dtype=torch.int32, device=DEVICE)
        table[torch.arange(width, device=DEVICE)[None] < torch.tensor(n, device=DEVICE)[:, None]] = ids
        return table

    state = dict(case=case, table=table_of(counts, order[:used]), start=i32([0] + new).cumsum(0, dtype=torch.int32), length=i32(length),
                 rows=rows, most=max(length), wide=max(new))
    state["data"], state["scale"] = _encode(_values((n_pages, 2, H, page, D), t, g), fmt)
    if kind != "evict":
        state["q"] = torch.randn((rows, H * G, D), generator=g, device=DEVICE).to(t)
    if kind == "rotate":
        state["k"], state["v"] = (_values((rows, H, D), t, g) for _ in range(2))
        state["pos"] = _positions(case, old, new)
        freq, axis = _frequencies(case)
        state["freq"], state["axis"] = torch.tensor(freq, dtype=torch.float64, device=DEVICE), torch.tensor(axis, device=DEVICE)
        state["q_out"], state["k_out"], state["v_out"] = (torch.empty_like(state[x]) for x in ("q", "k", "v"))
    if kind == "tree":
        state["tree"] = _trees(new, seed)
        state["out"] = torch.empty_like(state["q"])
        state["lse"] = torch.empty((rows, H * G), dtype=torch.float32, device=DEVICE)
    if kind == "weigh":
        state["lse"] = _sums(state, old, new)
    if kind in ("weigh", "evict"):
        # what the rows before have given each position: a few positions draw much of it, the first ones most
        w = torch.rand((len(length), H, max(length)), generator=g, device=DEVICE).pow_(8).mul_(20.0)
        w[:, :, :4] += 100.0
        state["weight"], state["weight_out"] = w, torch.zeros_like(w)
    if kind == "evict":
        state["table_out"], state["length_out"] = table_of(counts_out, order[used:used + sum(counts_out)]), i32(kept)
        state["keep"] = torch.empty((len(length), H, case["budget"]), dtype=torch.int32, device=DEVICE)
        state["kept"] = torch.empty(len(length), dtype=torch.int32, device=DEVICE)
        state["rows_out"], state["start_out"] = sum(kept), i32([0] + kept).cumsum(0, dtype=torch.int32)
        state["k_out"], state["v_out"] = (torch.empty((sum(kept), H, D), dtype=t, device=DEVICE) for _ in range(2))
    if own:
        from paper_2602_14236_b200 import binding as sc
        state["ctx"] = sc.Context(sc.salicache_default_params(max_batch=1, chunk_frames=1, L=1))
        state["pages"] = sc.PageSet(n_pages, page, H, D, {"fp16": sc.FP16, "int8": sc.INT8, "int4": sc.INT4}[fmt], t,
                                    data=state["data"], scale=state["scale"])
        state["seqs"] = sc.Seqs(state["start"], state["length"], state["table"], rows)
        if kind == "rotate":
            state["rotary"] = sc.Rotary(freq, axis, case["axes"], {"halves": sc.HALVES, "neighbours": sc.NEIGHBOURS}[case["pairing"]])
        if kind == "evict":
            state["seqs_out"] = sc.Seqs(state["start_out"], state["length_out"], state["table_out"], state["rows_out"])
        if kind in ("tree", "weigh"):
            state["work"] = torch.empty(sc.salicache_paged_work_bytes(state["ctx"], state["pages"].c, G), dtype=torch.uint8, device=DEVICE)
    return state


def run(state):
    return _run_own(state) if own else globals()["_plain_" + state["case"]["kind"]](state)


# ---- the framework's calls

def _run_own(state):
    from paper_2602_14236_b200 import binding as sc
    case, ctx, pages, seqs = state["case"], state["ctx"], state["pages"].c, state["seqs"].c
    H, D, G = case["heads"], case["head_dim"], case["q_per_kv"]
    if case["kind"] == "rotate":
        sc.salicache_paged_write_rotary(ctx, pages, seqs, state["rotary"], state["pos"], state["q"], H * G * D, G, state["q_out"], H * G * D,
                                        state["k"], state["v"], H * D, H * D)
        if case["format"] == "fp16":
            return [state["q_out"], state["data"]]
        sc.salicache_paged_read(ctx, pages, seqs, state["k_out"], state["v_out"], H * D, H * D)
        return [state["q_out"], state["k_out"], state["v_out"]]
    if case["kind"] == "tree":
        sc.salicache_paged_attend_tree(ctx, pages, seqs, state["tree"], 1, state["q"], H * G * D, G, D ** -0.5, case["window"], case["sinks"],
                                       state["out"], H * G * D, state["lse"], state["work"], state["work"].numel())
        return [state["out"], state["lse"]]
    if case["kind"] == "weigh":
        sc.salicache_paged_weigh(ctx, pages, seqs, state["q"], H * G * D, G, D ** -0.5, state["lse"], case["decay"], state["weight"],
                                 state["weight_out"], state["most"], state["work"], state["work"].numel())
        return [state["weight_out"]]
    sc.salicache_select_heavy(ctx, state["weight"], state["most"], H, len(state["kept"]), state["length"], case["budget"], case["sinks"],
                              case["recent"], state["keep"], state["kept"])
    sc.salicache_paged_keep(ctx, pages, seqs, state["keep"], H, case["budget"], None, state["kept"], state["seqs_out"].c, state["weight"],
                            state["weight_out"], state["most"])
    if case["format"] == "fp16":
        return [state["keep"], state["kept"], state["weight_out"], state["data"]]
    sc.salicache_paged_read(ctx, pages, state["seqs_out"].c, state["k_out"], state["v_out"], H * D, H * D)
    return [state["keep"], state["kept"], state["weight_out"], state["k_out"], state["v_out"]]


# ---- the plain forms

def _rows(start, length, table, rows, page):
    """Sequence, position, page and slot of every row of a call."""
    start, length = start.long(), length.long()
    r = torch.arange(rows, device=DEVICE)
    b = torch.searchsorted(start, r, right=True) - 1
    pos = length[b] - start[b + 1] + r
    return b, pos, table[b, pos // page].long(), pos % page


def _read(state, pid, slot):
    fmt, scale = state["case"]["format"], state["scale"]
    x = _decode(state["data"][pid, :, :, slot], None if scale is None else scale[pid, :, :, slot], fmt, TYPES[state["case"]["dtype"]])
    return [x[:, 0].contiguous(), x[:, 1].contiguous()]


def _turn(x, cos, sin, pairing):
    """x [rows][heads][D] turned in its first 2 * pairs dimensions, in binary32, rounded once."""
    n = 2 * cos.shape[-1]
    y, c, s = x.float().clone(), cos[:, None], sin[:, None]
    one, two = (slice(0, n // 2), slice(n // 2, n)) if pairing == "halves" else (slice(0, n, 2), slice(1, n, 2))
    a, b = x[..., one].float(), x[..., two].float()
    y[..., one] = a * c - b * s
    y[..., two] = b * c + a * s
    return y.to(x.dtype)


def _plain_rotate(state):
    case = state["case"]
    _, _, pid, slot = _rows(state["start"], state["length"], state["table"], state["rows"], case["page"])
    angle = state["pos"][:, state["axis"]].double() * state["freq"]            # far positions: 64 bits
    cos, sin = angle.cos().float(), angle.sin().float()
    q = _turn(state["q"], cos, sin, case["pairing"])
    k = _turn(state["k"], cos, sin, case["pairing"])
    codes, meta = _encode(torch.stack([k, state["v"]], 1), case["format"])     # [rows][2][H][...]
    state["data"][pid, :, :, slot] = codes
    if meta is None:
        return [q, state["data"]]
    state["scale"][pid, :, :, slot] = meta
    return [q] + _read(state, pid, slot)


def _padded(state):
    """Every sequence's keys and values side by side, padded to the longest, and its rows of q, padded to the most new ones."""
    case = state["case"]
    H, D, G, page = (case[k] for k in ("heads", "head_dim", "q_per_kv", "page"))
    seqs, most, wide = state["table"].shape[0], state["most"], state["wide"]
    b = _rows(state["start"], state["length"], state["table"], state["rows"], page)[0]
    p = torch.arange(most, device=DEVICE)
    ids = state["table"][:, p // page].long()                                  # [seqs][most], -1 behind the end
    there = p[None] < state["length"][:, None]
    ids = torch.where(there, ids, torch.zeros_like(ids))
    parts = 2 if case["kind"] == "tree" else 1
    data, scale = state["data"][:, :parts], None if state["scale"] is None else state["scale"][:, :parts]
    kv = _decode(data[ids, :, :, p % page], None if scale is None else scale[ids, :, :, p % page], case["format"], TYPES[case["dtype"]])
    kv = torch.where(there[:, :, None, None, None], kv, torch.zeros_like(kv)).float()                        # [seqs][most][parts][H][D]
    i = torch.arange(state["rows"], device=DEVICE) - state["start"].long()[b]
    q = torch.zeros((seqs, wide, H, G, D), device=DEVICE)
    q[b, i] = state["q"].float().view(-1, H, G, D)
    before = (state["length"] - state["start"].diff()).long()
    return kv, q, p, there, before, b, i


def _plain_tree(state):
    case = state["case"]
    H, D, G, W = case["heads"], case["head_dim"], case["q_per_kv"], case["window"]
    kv, q, p, there, before, b, i = _padded(state)
    bits = (state["tree"][:, None] >> torch.arange(64, device=DEVICE)) & 1                                   # [rows][64]
    named = torch.zeros((q.shape[0], q.shape[1], 64), dtype=torch.bool, device=DEVICE)
    named[b, i] = bits.bool()
    at = before[:, None] + named.sum(-1) - 1                                                                 # [seqs][wide]
    k = p[None] - before[:, None]                                                                            # [seqs][most]: row of the call
    seen = named.gather(2, k.clamp(0, 63)[:, None].expand(-1, q.shape[1], -1)) & ((k >= 0) & (k < 64) & there)[:, None]
    old = (k < 0)[:, None].expand_as(seen)
    if W:
        old = old & ((p[None, None] > at[:, :, None] - W) | (p < case["sinks"])[None, None])
    seen = seen | old
    a = torch.einsum("sihgd,sjhd->shgij", q, kv[:, :, 0]) * D ** -0.5
    a.masked_fill_(~seen[:, None, None], -math.inf)
    m = a.amax(-1, keepdim=True)
    m = torch.where(m == -math.inf, torch.zeros_like(m), m)
    a = a.sub_(m).exp_()
    l = a.sum(-1)
    o = torch.einsum("shgij,sjhd->sihgd", a, kv[:, :, 1])
    l = l.permute(0, 3, 1, 2)                                                                                # [seqs][wide][H][G]
    o = torch.where(l[..., None] > 0, o / l[..., None], torch.zeros_like(o))
    lse = torch.log(l) + m[..., 0].permute(0, 3, 1, 2)
    return [o[b, i].reshape(-1, H * G, D).to(TYPES[case["dtype"]]), lse[b, i].reshape(-1, H * G)]


def _plain_weigh(state):
    case = state["case"]
    H, D, G = case["heads"], case["head_dim"], case["q_per_kv"]
    kv, q, p, there, before, b, i = _padded(state)
    lse = torch.full((q.shape[0], q.shape[1], H, G), math.inf, device=DEVICE)                                # rows that are none weigh nothing
    lse[b, i] = state["lse"].view(-1, H, G)
    a = torch.einsum("sihgd,sjhd->shgij", q, kv[:, :, 0]).mul_(D ** -0.5)
    a.sub_(lse.permute(0, 2, 3, 1)[..., None]).exp_()
    at = before[:, None] + torch.arange(q.shape[1], device=DEVICE)[None]
    a.masked_fill_((p[None, None] > at[:, :, None])[:, None, None], 0.0)
    had = torch.where((p[None] < before[:, None])[:, None], state["weight"], torch.zeros_like(state["weight"]))
    decay = torch.where(state["start"].diff() > 0, case["decay"], 1.0)                                       # nothing new, nothing forgotten
    w = a.sum((2, 3)) + had * decay[:, None, None]
    state["weight_out"].copy_(torch.where(there[:, None], w, state["weight_out"]))
    return [state["weight_out"]]


def _plain_evict(state):
    case = state["case"]
    H, page, budget = case["heads"], case["page"], case["budget"]
    w, length = state["weight"], state["length"].long()
    p = torch.arange(state["most"], device=DEVICE)
    there = (p[None] < length[:, None])[:, None]
    always = (p < case["sinks"])[None, None] | (p[None] >= length[:, None] - case["recent"])[:, None]
    order = torch.where(there, torch.where(always, math.inf, w), -math.inf)
    order = torch.sort(order, dim=-1, descending=True, stable=True).indices[..., :budget]
    short = torch.arange(order.shape[-1], device=DEVICE)
    kept = length.clamp(max=budget)
    order = torch.where((short[None] < kept[:, None])[:, None], order, state["most"]).sort(-1).values        # ascending, nothing behind
    there = short[None] < kept[:, None]
    keep = state["keep"]
    keep.fill_(-1)
    keep[..., : order.shape[-1]] = torch.where(there[:, None], order, -1).to(torch.int32)
    state["kept"].copy_(kept)
    b, h, k = torch.nonzero(there[:, None].expand(-1, H, -1), as_tuple=True)
    src = order[b, h, k]
    state["weight_out"][b, h, k] = w[b, h, src]
    pid, to = state["table"][b, src // page].long(), state["table_out"][b, k // page].long()
    state["data"][to, :, h, k % page] = state["data"][pid, :, h, src % page]
    if state["scale"] is None:
        return [keep, state["kept"], state["weight_out"], state["data"]]
    state["scale"][to, :, h, k % page] = state["scale"][pid, :, h, src % page]
    _, _, pid, slot = _rows(state["start_out"], state["length_out"], state["table_out"], state["rows_out"], page)
    return [keep, state["kept"], state["weight_out"]] + _read(state, pid, slot)


# ---- the definition in 64 bits, written apart from the above; one sequence, one head, a block of rows at a time

def _exact_group(x, fmt, t):
    """A stored group's values: the steps that the definition rounds to binary32 or the 16-bit type are rounded, the rest is not."""
    r32 = lambda y: y.to(torch.float32).double()
    if fmt == "fp16":
        return x
    lo = x.min(-1, keepdim=True).values if fmt == "int4" else torch.zeros_like(x[..., :1])
    span = r32(x.max(-1, keepdim=True).values - lo) if fmt == "int4" else x.abs().max(-1, keepdim=True).values
    top, low = (15, 0) if fmt == "int4" else (127, -127)
    s = r32(span / top).to(t).double()
    s[s == 0] = 1.0
    q = torch.round(r32(r32(x - lo) * r32(1.0 / s))).clamp(low, top)
    return (q * s + lo).to(t).double()


def _exact_pages(state):
    """The values of all pages, in 64 bits, rounded to the 16-bit type as reading them back does: [n_pages][2][H][page][D]."""
    case, t = state["case"], TYPES[state["case"]["dtype"]]
    data, scale = state["data"], state["scale"]
    if case["format"] == "fp16":
        return data
    if case["format"] == "int8":
        return (data.double() * scale.double().unsqueeze(-1)).to(t)
    out = torch.empty(data.shape[:-1] + (2 * data.shape[-1],), dtype=t, device=DEVICE)
    s, z = scale[..., :1].double(), scale[..., 1:].double()
    out[..., 0::2] = ((data % 16).double() * s + z).to(t)
    out[..., 1::2] = (data.div(16, rounding_mode="floor").double() * s + z).to(t)
    return out


def _exact_rotate(state, case, old, new):
    t, D, page = TYPES[case["dtype"]], case["head_dim"], case["page"]
    freq, axis = _frequencies(case)
    pairs = len(freq)
    first = [i if case["pairing"] == "halves" else 2 * i for i in range(pairs)]
    second = [i + pairs if case["pairing"] == "halves" else 2 * i + 1 for i in range(pairs)]
    angle = torch.stack([state["pos"][:, a].double() * f for f, a in zip(freq, axis)], -1)
    unit = torch.polar(torch.ones_like(angle), angle)[:, None]
    def turned(x):
        y = x.double()
        z = torch.complex(y[..., first], y[..., second]) * unit
        y[..., first], y[..., second] = z.real, z.imag
        return y
    q, k, v = turned(state["q"]), turned(state["k"]), state["v"].double()
    if case["format"] != "fp16":
        return [q, _exact_group(k.to(t).double(), case["format"], t), _exact_group(v, case["format"], t)]
    data, r = state["data"].double(), 0
    for b, (o, n) in enumerate(zip(old, new)):
        p = torch.arange(o, o + n, device=DEVICE)
        ids = state["table"][b][torch.div(p, page, rounding_mode="floor")].long()
        data[ids, 0, :, p.remainder(page)], data[ids, 1, :, p.remainder(page)] = k[r:r + n], v[r:r + n]
        r += n
    return [q, data]


def _exact_evict(state, case, old, new):
    H, D, page, budget = case["heads"], case["head_dim"], case["page"], case["budget"]
    keep = torch.full((len(old), H, budget), -1, dtype=torch.int64, device=DEVICE)
    kept = torch.tensor([min(n, budget) for n in old], device=DEVICE)
    values = _exact_pages(state)
    data, w, out = values.double(), state["weight"].double(), state["weight_out"].double()
    back = []
    for b, n in enumerate(old):
        m = min(n, budget)
        rows = torch.empty((m, 2, H, D), dtype=torch.float64, device=DEVICE)
        lo, hi = case["sinks"], n - case["recent"]
        for h in range(H):
            if n <= budget:
                mine = torch.arange(n, device=DEVICE)
            else:
                # the heaviest of the middle: all above the weight of the last that fits, then the lowest positions at that weight
                middle, take = w[b, h, lo:hi], budget - lo - case["recent"]
                edge = middle.sort().values[-take] if take else torch.tensor(math.inf, dtype=torch.float64, device=DEVICE)
                above, equal = (middle > edge).nonzero()[:, 0], (middle == edge).nonzero()[:, 0]
                mine = torch.cat([above, equal[: take - above.numel()]]).sort().values + lo
                mine = torch.cat([torch.arange(lo, device=DEVICE), mine, torch.arange(hi, n, device=DEVICE)])
            keep[b, h, :m], out[b, h, :m] = mine, w[b, h, mine]
            rows[:, :, h] = values[state["table"][b, mine // page].long(), :, h, mine % page].double()
        p = torch.arange(m, device=DEVICE)
        data[state["table_out"][b, p // page].long(), :, :, p % page] = rows
        back.append(rows)
    if case["format"] == "fp16":
        return [keep, kept, out, data]
    back = torch.cat(back)
    return [keep, kept, out, back[:, 0], back[:, 1]]


def exact(case, seed):
    state = prepare(case, seed)
    old, new = _lengths(case)
    H, D, G, page = (case[k] for k in ("heads", "head_dim", "q_per_kv", "page"))
    if case["kind"] == "rotate":
        return _exact_rotate(state, case, old, new)
    if case["kind"] == "evict":
        return _exact_evict(state, case, old, new)
    values = _exact_pages(state)
    weigh = case["kind"] == "weigh"
    out = torch.zeros((sum(new), H * G, D), dtype=torch.float64, device=DEVICE)
    lse = torch.full((sum(new), H * G), -math.inf, dtype=torch.float64, device=DEVICE)
    weight = state["weight_out"].double() if weigh else None
    first = 0
    for b, (o, n) in enumerate(zip(old, new)):
        if weigh:
            weight[b, :, :o] = state["weight"][b, :, :o].double() * (case["decay"] if n else 1.0)
        if n:
            kv = values[state["table"][b, : -(-(o + n) // page)].long()].permute(0, 3, 1, 2, 4).reshape(-1, 2, H, D)[: o + n]
            j = torch.arange(o + n, device=DEVICE)
            if not weigh:
                bits = [x % (1 << 64) for x in state["tree"][first:first + n].tolist()]
                hidden = torch.tensor([[not x >> c & 1 for c in range(n)] for x in bits], device=DEVICE)
                at = torch.tensor([[o + bin(x).count("1") - 1] for x in bits], device=DEVICE)
                far = (j[:o] <= at - case["window"]) & (j[:o] >= case["sinks"]) if case["window"] else torch.zeros((n, o), dtype=torch.bool, device=DEVICE)
                hidden = torch.cat([far, hidden], 1)
            for h in range(H):
                k = kv[:, 0, h].double()
                for i0 in range(0, n, 1024):
                    i1 = min(n, i0 + 1024)
                    q = state["q"][first + i0:first + i1, h * G:(h + 1) * G].double()
                    a = (q.reshape(-1, D) @ k.T).view(i1 - i0, G, -1) / math.sqrt(D)
                    if weigh:
                        a -= state["lse"][first + i0:first + i1, h * G:(h + 1) * G].double()[..., None]
                        a.masked_fill_((j > torch.arange(o + i0, o + i1, device=DEVICE)[:, None])[:, None], -math.inf)
                        weight[b, h, : o + n] += torch.exp(a).sum((0, 1))
                        continue
                    a.masked_fill_(hidden[i0:i1, None], -math.inf)
                    lse[first + i0:first + i1, h * G:(h + 1) * G] = torch.logsumexp(a, -1)
                    out[first + i0:first + i1, h * G:(h + 1) * G] = (torch.softmax(a, -1).view(-1, o + n) @ kv[:, 1, h].double()).view(i1 - i0, G, D)
        first += n
    return [weight] if weigh else [out, lse]
