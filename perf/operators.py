"""The paged K/V cache: quantising rows as they are written and reading them back, and attention of new tokens over it.

A batch of sequences shares pages.  Sequence b's position p lives in slot p % page of page table[b][p // page]; the rows
row_start[b] .. row_start[b+1] of the caller's arrays are the last positions of its length[b].

  store    the new rows' K and V go into the pages (16-bit, INT8 or INT4) and come back as the values the pages now hold,
           which is what attention over a quantised cache has to use for the prompt itself
  read     positions of a filled cache as dense 16-bit rows
  attend   softmax attention of the new rows (causal; optionally a sliding window with the first `sinks` tokens visible
           throughout) over the cache, with the logarithm of the softmax sum beside the output

Lengths are texts ("old" = positions cached before, "new" = rows of this call, one number per sequence).
"""
import math

import torch

own = False
DEVICE = "cuda"

TYPES = {"f16": torch.float16, "bf16": torch.bfloat16}
BYTES = {"fp16": 2.0, "int8": 1.0, "int4": 0.5}           # a stored element
META = {"fp16": 0, "int8": 2, "int4": 4}                  # scale (and zero) of one head of one token


def _case(name, kind, fmt, dtype, heads, q_per_kv, head_dim, page, old, new, window=0, sinks=0):
    return dict(name=name, kind=kind, format=fmt, dtype=dtype, heads=heads, q_per_kv=q_per_kv, head_dim=head_dim, page=page,
                old=old, new=new, window=window, sinks=sinks)


def listed():
    return [
        # one decode step of eight streams adds a token each: launch latency
        _case("store_step_int8", "store", "int8", "f16", 8, 1, 128, 16, "611,1187,2303,90,576,16,4031,0", "1,1,1,1,1,1,1,1"),
        # four 672x672 frames (2880 visual tokens each) of four streams, 32 key/value heads
        _case("store_frames_int4", "store", "int4", "f16", 32, 1, 128, 64, "2880,0,5760,61", "2880,2880,2880,2880"),
        # ragged prompts, one of them empty, kept in 16 bits; small heads
        _case("store_prompts_bf16", "store", "fp16", "bf16", 12, 1, 64, 32, "0,300,17,0,1000,5", "1153,0,37,577,2,4095"),
        # reading a few sequences back
        _case("read_int8", "read", "int8", "bf16", 8, 1, 128, 64, "0,0,0", "1,577,4111"),
        # reading two long ones back
        _case("read_long_int4", "read", "int4", "f16", 8, 1, 128, 128, "0,0", "31999,17280"),
        # one token of one stream after one frame and a short question: latency
        _case("attend_step_fp16", "attend", "fp16", "f16", 32, 1, 128, 16, "611", "1"),
        # one token of each of 32 streams of very different lengths
        _case("attend_step_int4", "attend", "int4", "f16", 8, 4, 128, 64,
              "611,1187,16383,9000,12012,15001,577,2303,90,576,16,4031,14400,13824,11111,1,8191,10001,15555,6912,5184,16000,"
              "12345,3456,7777,100,9999,14001,8640,13579,2880,11520", ",".join(["1"] * 32)),
        # long-running streams that keep a window of 4096 tokens and the first four
        _case("attend_step_window_int8", "attend", "int8", "bf16", 8, 4, 128, 64,
              "32767,20001,4099,577,31999,28800,4095,4100,17280,30000,25001,8191,12345,32001,29999,2880",
              ",".join(["1"] * 16), 4096, 4),
        # a question of 61 tokens about 30 frames (576 tokens each)
        _case("attend_question_fp16", "attend", "fp16", "f16", 8, 4, 128, 64, "17280", "61"),
        # a whole prompt at once
        _case("attend_prompt_bf16", "attend", "fp16", "bf16", 8, 4, 128, 128, "0", "8192"),
        # four more frames of two streams over what was kept of the earlier ones
        _case("attend_frames_int4", "attend", "int4", "f16", 8, 4, 128, 64, "20736,6912", "2304,2304"),
        # a ragged batch under a window: a step, a drafted answer, prompts, and a stream with nothing new; small heads
        _case("attend_ragged_window_int8", "attend", "int8", "bf16", 4, 6, 64, 16, "900,1300,0,64,5000", "1,5,300,0,1029", 1024, 16),
    ]


def _log(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    while True:
        kind = rng.choice(["store", "read", "attend", "attend", "attend"])
        seqs = _log(rng, 1, 32)
        step = kind == "attend" and rng.random() < 0.4
        old = [0 if kind == "read" else rng.choice([0, _log(rng, 1, 24000)]) if rng.random() < 0.3 else _log(rng, 1, 24000) for _ in range(seqs)]
        new = [1 if step else 0 if rng.random() < 0.05 else _log(rng, 1, 8192) for _ in range(seqs)]
        new[0] = max(new[0], 1)
        window = kind == "attend" and rng.random() < 0.4
        case = dict(kind=kind, format=rng.choice(["fp16", "int8", "int4"]), dtype=rng.choice(["f16", "bf16"]),
                    heads=rng.choice([1, 2, 4, 5, 8, 12, 16, 32]), q_per_kv=rng.choice([1, 1, 2, 3, 4, 4, 6, 8]) if kind == "attend" else 1,
                    head_dim=rng.choice([64, 128, 128]), page=rng.choice([16, 32, 64, 128]), old=",".join(map(str, old)),
                    new=",".join(map(str, new)), window=_log(rng, 16, 8192) if window else 0, sinks=rng.choice([0, 1, 4, 64, 200]) if window else 0)
        most = max(o + n for o, n in zip(old, new))
        scores = seqs * case["heads"] * case["q_per_kv"] * max(new) * most if kind == "attend" else 0
        cells = seqs * most * case["heads"] * case["head_dim"]
        w = work(case)
        if scores <= 3.4e9 and cells <= 5.4e8 and w["bytes"] <= 4.4e8 and w["flops"] <= 1.0e12:
            return case


def _lengths(case):
    old, new = ([int(x) for x in case[k].split(",")] for k in ("old", "new"))
    return old, new


def work(case):
    old, new = _lengths(case)
    H, D, G, W, S = case["heads"], case["head_dim"], case["q_per_kv"], case["window"], case["sinks"]
    stored = 2 * H * (D * BYTES[case["format"]] + META[case["format"]])      # bytes of a token in the pages, K and V
    dense = 2 * H * D * 2                                                    # ... in the caller's arrays
    n = sum(new)
    if case["kind"] == "store":
        return {"bytes": n * 2 * (dense + stored), "flops": n * 2 * H * D * 4}
    if case["kind"] == "read":
        return {"bytes": n * (dense + stored), "flops": n * 2 * H * D * 2}
    pairs = keys = 0
    for o, m in zip(old, new):
        if m == 0:
            continue
        if W == 0:
            pairs += m * o + m * (m + 1) // 2
            keys += o + m
        else:
            first = max(0, o - W + 1)                                        # the first position inside the first row's window
            keys += min(S, first) + (o + m - first)
            for p in range(o, o + m):
                lo = max(0, p - W + 1)
                pairs += p + 1 - lo + min(S, lo)
    return {"bytes": keys * stored + 2 * n * H * G * D * 2 + n * H * G * 4, "flops": 4 * pairs * H * G * D}


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


def _values(shape, t, g):
    """Normal values with one element in a hundred eight times as large."""
    x = torch.randn(shape, generator=g, device=DEVICE, dtype=torch.float32)
    x = torch.where(torch.rand(shape, generator=g, device=DEVICE) < 0.01, 8.0 * x, x)
    return x.to(t)


def prepare(case, seed):
    old, new = _lengths(case)
    H, D, G, page, fmt, t = (case[k] for k in ("heads", "head_dim", "q_per_kv", "page", "format", "dtype"))
    t = TYPES[t]
    g = torch.Generator(device=DEVICE).manual_seed(seed)
    length = [o + n for o, n in zip(old, new)]
    counts = [-(-n // page) for n in length]
    width, used = max(max(counts), 1), sum(counts)
    n_pages = used + 3
    order = torch.randperm(n_pages, generator=g, device=DEVICE)[:used].to(torch.int32)
    table = torch.full((len(old), width), -1, dtype=torch.int32, device=DEVICE)
    held = torch.arange(width, device=DEVICE)[None] < torch.tensor(counts, device=DEVICE)[:, None]
    table[held] = order
    rows = sum(new)
    start = torch.tensor([0] + new, dtype=torch.int32, device=DEVICE).cumsum(0, dtype=torch.int32)
    state = dict(case=case, table=table, start=start, length=torch.tensor(length, dtype=torch.int32, device=DEVICE), rows=rows,
                 most=max(length), wide=max(new))
    data, scale = _encode(_values((n_pages, 2, H, page, D), t, g), fmt)
    state["data"], state["scale"] = data, scale
    if case["kind"] == "store":
        state["k"], state["v"] = (_values((rows, H, D), t, g) for _ in range(2))
    if case["kind"] in ("store", "read"):
        state["k_out"], state["v_out"] = (torch.empty((rows, H, D), dtype=t, device=DEVICE) for _ in range(2))
    else:
        state["q"] = torch.randn((rows, H * G, D), generator=g, device=DEVICE).to(t)
        state["out"] = torch.empty((rows, H * G, D), dtype=t, device=DEVICE)
        state["lse"] = torch.empty((rows, H * G), dtype=torch.float32, device=DEVICE)
    if own:
        from paper_2602_14236_b200 import binding as sc
        state["ctx"] = sc.Context(sc.salicache_default_params(max_batch=1, chunk_frames=1, L=1))
        state["pages"] = sc.PageSet(n_pages, page, H, D, {"fp16": sc.FP16, "int8": sc.INT8, "int4": sc.INT4}[fmt], t, data=data, scale=scale)
        state["seqs"] = sc.Seqs(start, state["length"], table, rows)
        state["work"] = torch.empty(sc.salicache_paged_work_bytes(state["ctx"], state["pages"].c, G), dtype=torch.uint8, device=DEVICE)
    return state


def run(state):
    return _run_own(state) if own else _run_plain(state)


def _run_own(state):
    from paper_2602_14236_b200 import binding as sc
    case, ctx, pages, seqs = state["case"], state["ctx"], state["pages"].c, state["seqs"].c
    H, D, G = case["heads"], case["head_dim"], case["q_per_kv"]
    if case["kind"] == "store":
        sc.salicache_paged_write(ctx, pages, seqs, state["k"], state["v"], H * D, H * D)
    if case["kind"] in ("store", "read"):
        sc.salicache_paged_read(ctx, pages, seqs, state["k_out"], state["v_out"], H * D, H * D)
        return [state["k_out"], state["v_out"]]
    sc.salicache_paged_attend(ctx, pages, seqs, state["q"], H * G * D, G, D ** -0.5, case["window"], case["sinks"],
                              state["out"], H * G * D, state["lse"], state["work"], state["work"].numel())
    return [state["out"], state["lse"]]


def _rows(state):
    """Sequence, position, page and slot of every row of this call."""
    start, length = state["start"].long(), state["length"].long()
    r = torch.arange(state["rows"], device=DEVICE)
    b = torch.searchsorted(start, r, right=True) - 1
    pos = length[b] - start[b + 1] + r
    return b, pos, state["table"][b, pos // state["case"]["page"]].long(), pos % state["case"]["page"]


def _run_plain(state):
    case = state["case"]
    fmt, t = case["format"], TYPES[case["dtype"]]
    H, D, G, page = (case[k] for k in ("heads", "head_dim", "q_per_kv", "page"))
    data, scale = state["data"], state["scale"]
    b, pos, pid, slot = _rows(state)
    if case["kind"] == "store":
        codes, meta = _encode(torch.stack([state["k"], state["v"]], 1), fmt)         # [rows][2][H][...]
        data[pid, :, :, slot] = codes
        if meta is not None:
            scale[pid, :, :, slot] = meta
    if case["kind"] in ("store", "read"):
        x = _decode(data[pid, :, :, slot], None if scale is None else scale[pid, :, :, slot], fmt, t)
        return [x[:, 0].contiguous(), x[:, 1].contiguous()]
    # every sequence's keys and values side by side, padded to the longest; rows padded to the most new ones
    seqs, most, wide = state["table"].shape[0], state["most"], state["wide"]
    p = torch.arange(most, device=DEVICE)
    ids = state["table"][:, p // page].long()                                         # [seqs][most], -1 behind the end
    there = p[None] < state["length"][:, None]
    ids = torch.where(there, ids, torch.zeros_like(ids))
    kv = _decode(data[ids, :, :, p % page], None if scale is None else scale[ids, :, :, p % page], fmt, t)   # [seqs][most][2][H][D]
    kv = torch.where(there[:, :, None, None, None], kv, torch.zeros_like(kv)).float()
    i = torch.arange(state["rows"], device=DEVICE) - state["start"].long()[b]
    q = torch.zeros((seqs, wide, H, G, D), device=DEVICE)
    q[b, i] = state["q"].float().view(-1, H, G, D)
    a = torch.einsum("sihgd,sjhd->shgij", q, kv[:, :, 0]) * D ** -0.5
    at = (state["length"] - state["start"].diff())[:, None].long() + torch.arange(wide, device=DEVICE)[None]     # [seqs][wide]
    seen = (p[None, None] <= at[:, :, None]) & there[:, None]
    if case["window"]:
        seen &= (p[None, None] > at[:, :, None] - case["window"]) | (p < case["sinks"])[None, None]
    a.masked_fill_(~seen[:, None, None], -math.inf)
    m = a.amax(-1, keepdim=True)
    m = torch.where(m == -math.inf, torch.zeros_like(m), m)
    a = a.sub_(m).exp_()
    l = a.sum(-1)
    o = torch.einsum("shgij,sjhd->sihgd", a, kv[:, :, 1])
    l = l.permute(0, 3, 1, 2)                                                         # [seqs][wide][H][G]
    o = torch.where(l[..., None] > 0, o / l[..., None], torch.zeros_like(o))
    lse = torch.log(l) + m[..., 0].permute(0, 3, 1, 2)
    return [o[b, i].reshape(-1, H * G, D).to(t), lse[b, i].reshape(-1, H * G)]


# ---- the definition in 64 bits, written apart from the above; one sequence, one head, a block of rows at a time

def _exact_group(x, fmt, t):
    """A stored group's values: the steps that the definition rounds to binary32 or the 16-bit type are rounded, the rest is not."""
    r32 = lambda y: y.to(torch.float32).double()
    x = x.double()
    if fmt == "fp16":
        return x
    lo = x.min(-1, keepdim=True).values if fmt == "int4" else torch.zeros_like(x[..., :1])
    span = r32(x.max(-1, keepdim=True).values - lo) if fmt == "int4" else x.abs().max(-1, keepdim=True).values
    top, low = (15, 0) if fmt == "int4" else (127, -127)
    s = r32(span / top).to(t).double()
    s[s == 0] = 1.0
    q = torch.round(r32(r32(x - lo) * r32(1.0 / s))).clamp(low, top)
    return q * s + lo


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


def exact(case, seed):
    state = prepare(case, seed)
    old, new = _lengths(case)
    H, D, G, page, W, S = (case[k] for k in ("heads", "head_dim", "q_per_kv", "page", "window", "sinks"))
    t = TYPES[case["dtype"]]
    if case["kind"] == "store":
        return [_exact_group(state[k], case["format"], t).to(t).double() for k in ("k", "v")]
    values = _exact_pages(state)
    def sequence(b, n):                                                               # [n][2][H][D]
        x = values[state["table"][b, : -(-n // page)].long()]
        return x.permute(0, 3, 1, 2, 4).reshape(-1, 2, H, D)[:n]
    if case["kind"] == "read":
        x = torch.cat([sequence(b, n) for b, n in enumerate(new)]).double()
        return [x[:, 0], x[:, 1]]
    out = torch.zeros((sum(new), H * G, D), dtype=torch.float64, device=DEVICE)
    lse = torch.full((sum(new), H * G), -math.inf, dtype=torch.float64, device=DEVICE)
    first = 0
    for b, (o, n) in enumerate(zip(old, new)):
        if n:
            kv = sequence(b, o + n)
            j = torch.arange(o + n, device=DEVICE)
            for h in range(H):
                k, v = kv[:, 0, h].double(), kv[:, 1, h].double()
                for i0 in range(0, n, 1024):
                    i1 = min(n, i0 + 1024)
                    at = torch.arange(o + i0, o + i1, device=DEVICE)[:, None]
                    hidden = j > at
                    if W:
                        hidden |= (j <= at - W) & (j >= S)
                    q = state["q"][first + i0:first + i1, h * G:(h + 1) * G].double()
                    a = (q.reshape(-1, D) @ k.T).view(i1 - i0, G, -1) / math.sqrt(D)
                    a.masked_fill_(hidden[:, None], -math.inf)
                    lse[first + i0:first + i1, h * G:(h + 1) * G] = torch.logsumexp(a, -1)
                    out[first + i0:first + i1, h * G:(h + 1) * G] = (torch.softmax(a, -1).view(-1, o + n) @ v).view(i1 - i0, G, D)
        first += n
    return [out, lse]
