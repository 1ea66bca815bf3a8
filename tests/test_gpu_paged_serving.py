"""A run of the paged calls as a server makes them: a prompt with positions on three axes, the weights of its positions, an
eviction to a budget, a drafted tree, the accepted path moved up, and a single token after it.  Every attention is compared with
the plain 64-bit form over what the pages hold at that moment, read back before the call."""
import numpy as np
import pytest

import paged_util as pu
from paper_2602_14236_b200 import binding as sc
from test_gpu_paged_rotary import turned
from test_gpu_paged_tree import trees, words

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("fmt,dt", [("fp16", "bf16"), ("int8", "f16"), ("int4", "f16")])
def test_serving(fmt, dt):
    import torch
    ctx = sc.Context(sc.salicache_default_params(max_batch=1, chunk_frames=1, L=1))
    t = {"f16": torch.float16, "bf16": torch.bfloat16}[dt]
    H, G, D, page, B, budget = 2, 2, 64, 16, 3, 96
    Hq, HD = H * G, H * D
    rng = np.random.default_rng(0)
    n_pages, width = 80, 16
    pages = sc.PageSet(n_pages, page, H, D, pu.FMT[fmt], t)
    i32 = lambda a: torch.from_numpy(np.ascontiguousarray(a)).to(torch.int32).cuda()
    order = rng.permutation(n_pages)
    table = i32(order[:B * width].reshape(B, width))
    freq, axis = 10000.0 ** (-np.arange(32) / 32), np.repeat([0, 1, 2], [8, 12, 12])
    rotary = sc.Rotary(freq, axis, 3)
    weight = torch.zeros((B, H, 256), device="cuda")
    values = lambda n, heads: torch.from_numpy(rng.standard_normal((n, heads * D))).to(t).cuda()
    scale = D ** -0.5

    def seqs_of(lens, news):
        return sc.Seqs(i32(np.concatenate([[0], np.cumsum(news)])), i32(np.array(lens)), table, int(sum(news)))

    def held(lens):
        """[B][len][2][H][D] float64 of the pages."""
        s, n = seqs_of(lens, lens), int(sum(lens))
        k, v = (torch.empty((n, HD), dtype=t, device="cuda") for _ in range(2))
        sc.salicache_paged_read(ctx, pages.c, s.c, k, v, HD, HD)
        x = torch.stack([k, v], 1).double().cpu().numpy().reshape(n, 2, H, D)
        return np.split(x, np.cumsum(lens)[:-1])

    def check(q, out, lse, kv, sees):
        """sees(b, i): positions of row i of sequence b; [(out, lse)] against the plain form."""
        r = 0
        for b, x in enumerate(kv):
            for j in sees[b]:
                for hq in range(Hq):
                    o, l, tol, ltol = pu.attend(q[r, hq], x[j, 0, hq // G], x[j, 1, hq // G], scale, t, fmt)
                    pu.check(out[r, hq], o, tol, "out")
                    pu.check(lse[r, hq], np.array(l), ltol, "lse")
                r += 1

    def call(lens, news, tree=None):
        """New rows go in, attend and weigh; returns their sequences, turned q, output and sums."""
        s, n = seqs_of(lens, news), int(sum(news))
        q, k, v = values(n, Hq), values(n, H), values(n, H)
        pos = rng.integers(0, 5000, (n, 3))
        raw = q.double().cpu().numpy().reshape(n, Hq, D)
        sc.salicache_paged_write_rotary(ctx, pages.c, s.c, rotary, i32(pos), q, Hq * D, G, q, Hq * D, k, v, HD, HD)
        out, lse = torch.empty_like(q), torch.empty((n, Hq), device="cuda")
        wk = torch.empty(sc.salicache_paged_work_bytes(ctx, pages.c, G), dtype=torch.uint8, device="cuda")
        if tree is None:
            sc.salicache_paged_attend(ctx, pages.c, s.c, q, Hq * D, G, scale, 0, 0, out, Hq * D, lse, wk, wk.numel())
            sc.salicache_paged_weigh(ctx, pages.c, s.c, q, Hq * D, G, scale, lse, 1.0, weight, weight, 256, wk, wk.numel())
        else:
            bits = torch.from_numpy(words(tree, 1, n).view(np.int64)).cuda()
            sc.salicache_paged_attend_tree(ctx, pages.c, s.c, bits, 1, q, Hq * D, G, scale, 0, 0, out, Hq * D, lse, wk, wk.numel())
        f = lambda x: x.double().cpu().numpy()
        y, tol = turned(raw, pos, freq, axis, sc.HALVES, t)
        pu.check(f(q).reshape(n, Hq, D), y, tol, "q")
        return f(q).reshape(n, Hq, D), f(out).reshape(n, Hq, D), f(lse)

    # prompts
    lens = [200, 60, 131]
    q, out, lse = call(lens, lens)
    kv = held(lens)
    check(q, out, lse, kv, [[np.arange(i + 1) for i in range(n)] for n in lens])
    total = weight.double().sum(-1).cpu().numpy()
    assert np.allclose(total, G * np.array(lens)[:, None], rtol=5e-5)          # each row and query head gives one in all

    # back to the budget, in place
    keep, kept = torch.empty((B, H, budget), dtype=torch.int32, device="cuda"), torch.empty(B, dtype=torch.int32, device="cuda")
    sc.salicache_select_heavy(ctx, weight, 256, H, B, i32(np.array(lens)), budget, 4, 32, keep, kept)
    before_w = weight.clone()
    sc.salicache_paged_keep(ctx, pages.c, seqs_of(lens, [0] * B).c, keep, H, budget, None, kept, None, weight, weight, 256)
    assert sc.salicache_poll_status(ctx) == 0
    lists = keep.cpu().numpy()
    lens = kept.tolist()
    assert lens == [96, 60, 96]
    after = held(lens)
    for b, n in enumerate(lens):
        for h in range(H):
            assert np.array_equal(after[b][:, :, h], kv[b][lists[b, h, :n]][:, :, h])
            assert torch.equal(weight[b, h, :n], before_w[b, h, keep[b, h, :n].long()])

    # a draft for the first two
    news = [12, 7, 0]
    base, lens = lens, [n + m for n, m in zip(lens, news)]
    mats = trees(rng, news, "branch")
    q, out, lse = call(lens, news, mats)
    kv = held(lens)
    check(q, out, lse, kv, [[np.concatenate([np.arange(base[b]), base[b] + np.flatnonzero(m[i])]) for i in range(m.shape[0])] for b, m in enumerate(mats)])

    # the deepest path is accepted and moves up
    paths = [base[b] + np.flatnonzero(m[m.sum(1).argmax()]) if m.size else np.zeros(0, int) for b, m in enumerate(mats)]
    keep = np.full((B, 1, 12), -1)
    for b, p in enumerate(paths):
        keep[b, 0, :p.size] = p
    sc.salicache_paged_keep(ctx, pages.c, seqs_of(lens, [0] * B).c, i32(keep), 1, 12, i32(np.array(base)), i32(np.array([p.size for p in paths])), None)
    lens = [n + p.size for n, p in zip(base, paths)]
    after = held(lens)
    for b in range(B):
        assert np.array_equal(after[b], np.concatenate([kv[b][:base[b]], kv[b][paths[b]]]))

    # and a single token each
    lens = [n + 1 for n in lens]
    q, out, lse = call(lens, [1] * B)
    check(q, out, lse, held(lens), [[np.arange(n)] for n in lens])
    assert sc.salicache_poll_status(ctx) == 0
