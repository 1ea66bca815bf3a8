// Attention of new rows over the paged cache, many rows per sequence (prompts, questions, new frames): the products are
// the work, and they run on the fifth-generation tensor cores (tcgen05.mma, accumulators in tensor memory).
//
// One block per SM walks its stretch of the line of (256 rows x 128 keys) tiles (paged_plan.cuh).  A tile's rows are two
// halves of 128 = the lanes of tensor memory; scores S = Q K^T and sums O += P V of both halves stand in all 512 columns.
// Roles by warp group:
//   0, 1   one thread per row of half 0 / 1: maximum over the row's 128 scores, weights, row sum; P overwrites S as the
//          16-bit operand of the second product, handed on in two parts; also the output.  The row sum is of the unrounded
//          weights, in binary32; what P's rounding adds to the output's own is in paged_attend.cu
//   2      codes from a ring of raw stages to 16-bit operands; of 16-bit pages only the V tiles that hold positions no
//          row sees, which become zeros whatever the page holds there
//   3      one thread issues the matrix instructions; one warp feeds the rings with bulk copies, a lane per page: tensor
//          copies straight into the operand stages (16-bit pages), plain ones of codes and scales into the raw stages; and
//          Q, of the next item as soon as the last scores of the present one are done
// A half holds the query heads of 128 / G whole tokens, so that Q is one box of (64 dimensions, G heads, tokens) per copy.
// (Asynchronous 16-byte copies by the threads instead took 4.8 us for an item's 64 KB.)
// While one half's weights are formed, the tensor core works for the other: the products of a half are issued as
// P(t) V(t), then Q K(t+1).  Instructions of one thread run in order there, so S may be overwritten right behind the
// product that read P from the same columns, and whoever sees the scores of tile t knows the sums of tile t-1 complete.
// The reference maximum moves only when a row exceeds it by 2^8; then, and only then, O is rescaled, by the thread that
// found it and before it hands its weights on.
//
// Measured (bf16, 8192 new rows, 32 query and 8 key/value heads x 128): 560 us = 980 TFLOP/s, 0.58 of the cuBLAS burst rate;
// two streams' 2304 rows over 20736 and 6912 INT4 positions: 1150 us = 983 TFLOP/s.  A (256 x 128) tile takes some 3500
// clocks, of which the tensor core works 2050 (counted: 54 % of the kernel): the round of a half, S, weights, P V, is as
// long as that.  Without the weights (products and copies alone) a tile takes 2800, shared memory being read at its full
// rate for them.
//
// Both operands use the 128-byte swizzle: rows of 64 elements, eight rows to a 1024-byte atom.  K has the contracted
// dimension contiguous; V has it across rows, which the instruction descriptor's transpose bit covers, so neither is
// transposed in memory.  INT4 codes come out of their words in the order 0 4 1 5 2 6 3 7; Q is permuted alike when it is
// staged and the output back when it is written.
#include <math.h>
#include <type_traits>

#include "paged_plan.cuh"
#include "paged_tc.cuh"

namespace {

constexpr int CH_ROWS = 256, CH_THREADS = 512, CH_STAGES = 4;

constexpr int CH_RAW = 4;                    // raw stages at most

struct ChBars {
    uint64_t kv_full[CH_STAGES], kv_empty[CH_STAGES], raw_full[CH_RAW], raw_empty[CH_RAW], q_land[2], q_ready[2], q_empty[2], v_land[2], s_full[2], p_ready[2][2],
        o_done[2], left;
    uint32_t tmem;
    int gave_up;
    uint32_t pages[8];                       // per tile (in turn): bit g set: the page of keys 16 g .. 16 g + 15 exists
};

template <int FMT, int D>
struct ChSmem {
    static constexpr int TILE = 128 * D * 2;         // bytes of an operand tile
    static constexpr int RAW_CODES = 128 * pg_row_bytes<FMT, D>(), RAW = RAW_CODES + 128 * pg_meta_bytes<FMT>();
    static constexpr int N_RAW = FMT == PF_16 ? 0 : D == 64 ? 4 : FMT == PF_I4 ? 3 : 2;      // what 227 KB leave room for
    static constexpr int Q = 0, KV = 2 * TILE, RAWS = KV + CH_STAGES * TILE, BARS = RAWS + N_RAW * RAW;
    static constexpr int BYTES = BARS + (int)sizeof(ChBars) + 1024;
    static_assert(BYTES <= 227 * 1024, "shared memory");
};

// An item's fixed cost (Q, output) in tiles' time, as measured.
constexpr int CH_ITEM = 3;
using ChSeg = PtSeg<CH_ITEM>;

// INT4: a half's Q, which a copy has brought, into the order in which codes leave their words; a thread per row.
template <int D>
__device__ __noinline__ void permute_rows(uint32_t q_tile, uint32_t q_ready) {
    const int row = threadIdx.x & 127;
#pragma unroll 4
    for (int c = 0; c < D / 8; ++c) {
        uint32_t v[4];
        lds16(v, q_tile + swz(row, c));
        sts16(q_tile + swz(row, c), __byte_perm(v[0], v[2], 0x5410), __byte_perm(v[0], v[2], 0x7632), __byte_perm(v[1], v[3], 0x5410),
              __byte_perm(v[1], v[3], 0x7632));
    }
    fence_async();
    __syncwarp();
    if ((threadIdx.x & 31) == 0) bar_arrive(q_ready);
}

// TREE: the rows are a tree's, and see what their bits name of the call's own positions.
template <typename T, int FMT, int D, bool TREE>
__global__ void __launch_bounds__(CH_THREADS, 1)
k_paged_chunk(PtArgs a, const __grid_constant__ CUtensorMap map, const __grid_constant__ CUtensorMap q_map, int blocks) {
    using SM = ChSmem<FMT, D>;
    extern __shared__ uint8_t raw[];
    __shared__ PtShared plan;
    const uint32_t base = (smem_u32(raw) + 1023u) & ~1023u;
    ChBars& bars = *reinterpret_cast<ChBars*>(raw + (base - smem_u32(raw)) + SM::BARS);
    const int tid = threadIdx.x, wid = tid >> 5, lane = tid & 31;
    volatile int* gave_up = &bars.gave_up;

    if (tid == 0) {
        for (int i = 0; i < CH_STAGES; ++i) {
            bar_init(smem_u32(&bars.kv_full[i]), 4);       // the four warps of group 2, or four lanes of the feeder
            bar_init(smem_u32(&bars.kv_empty[i]), 1);
        }
        for (int i = 0; i < CH_RAW; ++i) {
            bar_init(smem_u32(&bars.raw_full[i]), 1);
            bar_init(smem_u32(&bars.raw_empty[i]), 4);
        }
        for (int i = 0; i < 2; ++i) {
            bar_init(smem_u32(&bars.q_land[i]), 1);
            bar_init(smem_u32(&bars.q_ready[i]), 4);      // a lane of each of the half's warps
            bar_init(smem_u32(&bars.q_empty[i]), 1);
            bar_init(smem_u32(&bars.v_land[i]), 1);
            bar_init(smem_u32(&bars.s_full[i]), 1);
            bar_init(smem_u32(&bars.p_ready[i][0]), 4);
            bar_init(smem_u32(&bars.p_ready[i][1]), 4);
            bar_init(smem_u32(&bars.o_done[i]), 1);
        }
        bar_init(smem_u32(&bars.left), 1);
        bars.gave_up = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (wid == 12) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_u32(&bars.tmem)) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    grid_wait();
    grid_release();
    tc_before();
    const PtPlace start = pt_start<CH_THREADS, CH_ITEM>(a, blockIdx.x, blocks, plan);
    PtWalk w = start.w;
    PgSeq s = start.s;
    __syncthreads();
    tc_after();
    const uint32_t tmem = bars.tmem;
    ChSeg g;
    const int HR = a.tile_rows >> 1;         // rows of a half
    auto wait = [&](uint64_t& bar, uint32_t parity) -> bool { return warp_wait_far(smem_u32(&bar), parity, a.wait_limit, gave_up); };

    if (wid < 8) {
        // ---------------- rows: softmax, Q, output
        const int half = wid >> 2, row = tid & 127;
        const uint32_t lane_base = (uint32_t)((wid & 3) * 32) << 16;
        const uint32_t S = tmem + 128 * half + lane_base, O = tmem + 256 + 128 * half + lane_base;
        const uint32_t q_ready = smem_u32(&bars.q_ready[half]), p_ready = smem_u32(&bars.p_ready[half][0]);
        const uint32_t q_tile = base + SM::Q + half * SM::TILE;
        uint32_t n_s = 0, n_o = 0, n_tile = 0;               // scores, outputs of this half and tiles seen so far
        int4 hd[2] = {make_int4(0, 0, 0, 0), make_int4(0, 0, 0, 0)};
        bool ok = true;
        uint32_t n_q = 0;
        auto hand_q = [&](const ChSeg& gg) -> bool {
            if (FMT != PF_I4 || gg.rows <= half * HR || gg.tiles == 0) return true;
            if (!wait(bars.q_land[half], n_q++ & 1)) return false;
            permute_rows<D>(q_tile, q_ready);
            return true;
        };
        if (w.left > 0) {
            g = ChSeg::of(a, w, s);
            ok = hand_q(g);
        }
        while (w.left > 0 && ok) {
            const bool first = g.t0 == 0, lastp = g.last, done = first && lastp;
            const int rows = min(HR, g.rows - half * HR);    // of this half
            if (tid == 0 && s.cut && s.pos0 + s.n > s.len) atomicMin(a.status, SALICACHE_E_CAPACITY);
            // the item after this one
            PtWalk wn = w;
            PgSeq sn = s;
            wn.left -= g.k1 - g.k0;
            if (wn.left > 0) pt_next_far(wn, sn, a);
            ChSeg gn;
            gn.rows = gn.tiles = 0;
            if (wn.left > 0) gn = ChSeg::of(a, wn, sn);
            bool handed = false;
            if (rows > 0) {
                const int rr = w.rt * a.tile_rows + half * HR + row;                 // this thread's row of the item
                const bool live = row < rows;
                const int own = (live ? rr : 0) / a.G, pos = s.pos0 + (TREE ? a.window ? pt_depth(a, s.row0 + own, s.n) : 0 : own);
                float m = PT_NONE, l = 0.0f;
                if (g.tiles > 0) {
                    // positions that every row of this half sees in full tiles need no mask
                    const PtSpan hs = pt_span(s, a.G, w.rt * a.tile_rows + half * HR, w.rt * a.tile_rows + half * HR + rows, a.window, a.sinks, TREE);
                    const int vis_hi = live ? max(0, min(TREE ? s.pos0 : pos + 1, s.len)) : 0;
                    const int vis_lo = a.window ? pos - a.window + 1 : 0;
                    for (int k = 0; k < g.tiles; ++k, ++n_tile) {
                        if (!wait(bars.s_full[half], n_s++ & 1)) {
                            ok = false;
                            break;
                        }
                        tc_after();
                        const int j0 = g.sp.tile(g.t0 + k) * PT_KEYS;
                        const uint32_t pages = *(volatile uint32_t*)&bars.pages[n_tile & 7];
                        uint32_t x[2][32];
                        if (!(j0 + PT_KEYS <= hs.all_hi && (j0 >= hs.all_lo || j0 + PT_KEYS <= a.sinks) && pages == 0xffu)) {
                            const int hi = vis_hi - j0, lo = vis_lo - j0, sk = a.sinks - j0;
#pragma unroll 1
                            for (int c = 0; c < 4; ++c) {        // 32 keys at a time as a word of visible ones
                                const uint32_t there = ((pages >> (2 * c) & 1u) ? 0xffffu : 0u) | ((pages >> (2 * c + 1) & 1u) ? 0xffff0000u : 0u);
                                uint32_t vis = below(hi - 32 * c) & (~below(lo - 32 * c) | below(sk - 32 * c));
                                if (TREE) {
                                    const int j = j0 + 32 * c;
                                    if (live && j + 32 > s.pos0) vis |= pt_bits(a, s.row0 + own, j - s.pos0, s.n) & below(s.len - j);
                                }
                                vis &= there;
                                tc_ld32(x[0], S + 32 * c);
                                tc_wait_ld(x[0]);
#pragma unroll
                                for (int i = 0; i < 32; ++i)
                                    if (!(vis & 1u << i)) x[0][i] = 0xff800000u;
                                tc_st32(S + 32 * c, x[0]);
                            }
                            tc_wait_st();
                        }
                        float mx[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
                        tc_ld32(x[0], S);
                        tc_wait_ld(x[0]);
#pragma unroll
                        for (int c = 0; c < 4; ++c) {
                            if (c < 3) tc_ld32(x[(c + 1) & 1], S + 32 * (c + 1));
#pragma unroll
                            for (int i = 0; i < 32; i += 2)
                                mx[(i >> 1) & 3] = fmaxf(mx[(i >> 1) & 3], fmaxf(__uint_as_float(x[c & 1][i]), __uint_as_float(x[c & 1][i + 1])));
                            if (c < 3) tc_wait_ld(x[(c + 1) & 1]);
                        }
                        tc_ld32(x[0], S);
                        const float top = live ? fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3])) * a.scale : PT_NONE;
                        if (k == 0) m = fmaxf(m, top);
                        else if (__any_sync(0xffffffffu, top > m + 8.0f)) {
                            const float nm = fmaxf(m, top), f = ex2(m - nm);
                            m = nm;
                            l *= f;
#pragma unroll 1
                            for (int c = 0; c < D; c += 16) {
                                uint32_t o[16];
                                tc_ld16(o, O + c);
                                tc_wait_ld16(o);
#pragma unroll
                                for (int i = 0; i < 16; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * f);
                                tc_st16(O + c, o);
                            }
                        }
                        tc_wait_ld(x[0]);
                        // P takes half the columns of S: what it overwrites has been read
                        float sum[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                        for (int c = 0; c < 4; ++c) {
                            if (c < 3) tc_ld32(x[(c + 1) & 1], S + 32 * (c + 1));
                            uint32_t pk[16];
#pragma unroll
                            for (int i = 0; i < 16; ++i) {
                                const float p0 = ex2(fmaf(__uint_as_float(x[c & 1][2 * i]), a.scale, -m));
                                const float p1 = ex2(fmaf(__uint_as_float(x[c & 1][2 * i + 1]), a.scale, -m));
                                sum[2 * (i & 1)] += p0;
                                sum[2 * (i & 1) + 1] += p1;
                                pk[i] = T::pack(p0, p1);
                            }
                            if (c < 3) tc_wait_ld(x[(c + 1) & 1]);
                            tc_st16(S + 16 * c, pk);
                            if (c & 1) {             // half of P: the product may start on it
                                tc_wait_st();
                                tc_before();
                                __syncwarp();
                                if (lane == 0) bar_arrive(p_ready + 8 * (c >> 1));
                            }
                        }
                        l += (sum[0] + sum[1]) + (sum[2] + sum[3]);
                    }
                    if (ok) {
                        ok = hand_q(gn);
                        handed = true;
                        ok = ok && wait(bars.o_done[half], n_o++ & 1);
                        tc_after();
                    }
                }
                if (ok && g.real) {
                    // the output, or the partial record: float4 [D / 4][256 rows]
                    const size_t slot = 2 * (size_t)blockIdx.x + (first ? 1 : 0);
                    const float inv = l > 0.0f ? 1.0f / l : 0.0f;
                    const int hq = w.h * a.G + rr % a.G;
                    const long long tok = s.row0 + rr / a.G;
                    uint16_t* dst = a.out + tok * a.out_stride + (long long)hq * D;
                    float4* part = reinterpret_cast<float4*>(a.part) + slot * (D / 4) * CH_ROWS + half * 128 + row;
#pragma unroll 1
                    for (int c = 0; c < D; c += 32) {
                        uint32_t o[32];
                        __syncwarp();
                        if (g.tiles > 0) {
                            tc_ld32(o, O + c);
                            tc_wait_ld(o);
                        } else {
#pragma unroll
                            for (int i = 0; i < 32; ++i) o[i] = 0u;
                        }
#pragma unroll
                        for (int e = 0; e < 32; e += 8) {
                            float f[8];
#pragma unroll
                            for (int i = 0; i < 8; ++i) f[i] = __uint_as_float(o[e + (FMT == PF_I4 ? (i < 4 ? 2 * i : 2 * i - 7) : i)]);
                            if (live && done) {
                                uint4 v = make_uint4(T::pack(f[0] * inv, f[1] * inv), T::pack(f[2] * inv, f[3] * inv),
                                                     T::pack(f[4] * inv, f[5] * inv), T::pack(f[6] * inv, f[7] * inv));
                                *reinterpret_cast<uint4*>(dst + c + e) = v;
                            } else if (live) {
                                part[(size_t)((c + e) / 4) * CH_ROWS] = make_float4(f[0], f[1], f[2], f[3]);
                                part[(size_t)((c + e) / 4 + 1) * CH_ROWS] = make_float4(f[4], f[5], f[6], f[7]);
                            }
                        }
                    }
                    tc_before();
                    if (live && done && a.lse) a.lse[tok * ((long long)a.pc.heads * a.G) + hq] = l > 0.0f ? (m + log2f(l)) * PT_LN2 : -INFINITY;
                    if (live && !done) a.stat[slot * CH_ROWS + half * 128 + row] = make_float2(m, l);
                }
            } else n_tile += g.tiles;
            if (ok && !handed) ok = hand_q(gn);
            if (!done && g.real && ok) {
                if (first) pt_tail(hd, w, s);
                else hd[0].x = lastp ? 2 : 1;
            }
            w = wn;
            s = sn;
            g = gn;
        }
        if (tid == 0) {
            a.head[2 * blockIdx.x] = hd[0];
            a.head[2 * blockIdx.x + 1] = hd[1];
        }
    } else if (wid < 12) {
        // ---------------- operands
        const Codes<T> cd;
        const int lw = wid - 8;                              // this warp's rows: 32 lw .. 32 lw + 31 of a tile
        uint32_t n_stage = 0, n_land = 0;
        bool ok = true;
        while (w.left > 0 && ok) {
            g = ChSeg::of(a, w, s);
            for (int k = g.t0; k < g.t0 + g.tiles && ok; ++k) {
                const int j0 = g.sp.tile(k) * PT_KEYS;
                const int pid = g.page_of(a, w, k, lane);
                const uint32_t bad = __ballot_sync(0xffffffffu, pid == -1);
                const bool clean = g.clean(a, k) && bad == 0;
                // whether some row sees key r of this warp's 32
                auto seen = [&](int r) -> bool {
                    const int j = j0 + lw * 32 + r;
                    return j < g.sp.hi && (j >= g.sp.lo || j < a.sinks) && !(bad >> (lw * 2 + (r >> 4)) & 1u);
                };
                for (int kv = 0; kv < 2; ++kv, ++n_stage) {
                    const uint32_t stage = n_stage % CH_STAGES, dst = base + SM::KV + stage * SM::TILE;
                    if (FMT == PF_16) {
                        if (kv == 0 || clean) continue;  // the feeder's copies are all there is to it
                        // the pages have been copied: zeros where no row sees them
                        if (!wait(bars.v_land[n_land & 1], n_land >> 1 & 1)) {
                            ok = false;
                            break;
                        }
                        ++n_land;
                        constexpr int LPR = D / 8, RPP = 32 / LPR;
                        const int c = lane % LPR;
#pragma unroll 1
                        for (int p = 0; p < 32 / RPP; ++p) {
                            const int r = p * RPP + lane / LPR;
                            if (!seen(r)) sts16(dst + swz(lw * 32 + r, c), 0u, 0u, 0u, 0u);
                        }
                        fence_async();
                        __syncwarp();
                    } else {
                        constexpr int N_RAW = SM::N_RAW > 0 ? SM::N_RAW : 1;
                        constexpr int LPR = pg_row_bytes<FMT, D>() >= 16 ? pg_row_bytes<FMT, D>() / 16 : 1, RPP = 32 / LPR;
                        const uint32_t rs = n_stage % N_RAW, raw0 = base + SM::RAWS + rs * SM::RAW;
                        if ((n_stage >= CH_STAGES && !wait(bars.kv_empty[stage], (n_stage / CH_STAGES - 1) & 1)) ||
                            !wait(bars.raw_full[rs], (n_stage / N_RAW) & 1)) {
                            ok = false;
                            break;
                        }
                        const int c = lane % LPR;
                        constexpr int BATCH = LPR < 4 ? LPR : 4;             // rows in flight
#pragma unroll
                        for (int p0 = 0; p0 < LPR; p0 += BATCH) {
                            uint32_t words[BATCH][4], meta[BATCH];
#pragma unroll
                            for (int p = 0; p < BATCH; ++p) {
                                const int row = lw * 32 + (p0 + p) * RPP + lane / LPR;
                                lds16(words[p], raw0 + row * pg_row_bytes<FMT, D>() + c * 16);
                                if (FMT == PF_I8) {
                                    uint16_t s16;
                                    asm volatile("ld.shared.u16 %0, [%1];" : "=h"(s16) : "r"(raw0 + SM::RAW_CODES + row * 2));
                                    meta[p] = s16;
                                } else asm volatile("ld.shared.u32 %0, [%1];" : "=r"(meta[p]) : "r"(raw0 + SM::RAW_CODES + row * 4));
                            }
#pragma unroll
                            for (int p = 0; p < BATCH; ++p) {
                                const int r = (p0 + p) * RPP + lane / LPR, row = lw * 32 + r;
                                if (!clean && !seen(r)) meta[p] = 0;      // scale and zero 0: the row becomes zeros
                                const uint32_t s2 = dup_lo(meta[p]), z2 = dup_hi(meta[p]);
                                const uint32_t* w4 = words[p];
                                if (FMT == PF_I8) {
#pragma unroll
                                    for (int i = 0; i < 2; ++i)
                                        sts16(dst + swz(row, 2 * c + i), mul2<T>(cd.bytes(w4[2 * i], 0x5140), s2),
                                              mul2<T>(cd.bytes(w4[2 * i], 0x5342), s2), mul2<T>(cd.bytes(w4[2 * i + 1], 0x5140), s2),
                                              mul2<T>(cd.bytes(w4[2 * i + 1], 0x5342), s2));
                                } else {
#pragma unroll
                                    for (int i = 0; i < 4; ++i) {
                                        const uint32_t y = w4[i] >> 8;
                                        sts16(dst + swz(row, 4 * c + i), fma2<T>(cd.nib_lo(w4[i]), s2, z2), fma2<T>(cd.nib_hi(w4[i]), s2, z2),
                                              fma2<T>(cd.nib_lo(y), s2, z2), fma2<T>(cd.nib_hi(y), s2, z2));
                                    }
                                }
                            }
                        }
                        fence_async();
                        __syncwarp();
                        if (lane == 0) bar_arrive(smem_u32(&bars.raw_empty[rs]));
                    }
                    if (lane == 0) bar_arrive(smem_u32(&bars.kv_full[stage]));
                }
            }
            w.left -= g.k1 - g.k0;
            if (w.left > 0) pt_next_far(w, s, a);
        }
    } else {
        if (wid == 12) {
            // ---------------- matrix instructions: the warp stays together (its values are uniform), one lane issues
            constexpr uint32_t ID_S = instr_desc<T>(128, false), ID_O = instr_desc<T>(D, true);
            uint32_t n_stage = 0, n_q[2] = {0, 0}, n_p[2] = {0, 0};
            bool ok = true;
            const uint32_t q_lo = desc_lo(base + SM::Q, 16), k_lo = desc_lo(base + SM::KV, 16), v_lo = desc_lo(base + SM::KV, 16384);
            auto scores = [&](int h, uint32_t st, bool last) {
                const uint32_t qa = q_lo + h * (SM::TILE >> 4), kb = k_lo + st * (SM::TILE >> 4);
                if (elect_one()) {
#pragma unroll
                    for (int i = 0; i < D / 16; ++i) {
                        const uint32_t off = (i >> 2) * 1024 + (i & 3) * 2;
                        mma_ss(tmem + 128 * h, desc(qa + off), desc(kb + off), ID_S, i > 0);
                    }
                    tc_commit(smem_u32(&bars.s_full[h]));
                    if (last) tc_commit(smem_u32(&bars.q_empty[h]));
                }
                __syncwarp();
            };
            auto sums = [&](int h, uint32_t st, int part, bool add, bool last) {         // keys 64 part .. 64 part + 63
                const uint32_t vb = v_lo + st * (SM::TILE >> 4);
                if (elect_one()) {
#pragma unroll
                    for (int i = 4 * part; i < 4 * part + 4; ++i) mma_ts(tmem + 256 + 128 * h, tmem + 128 * h + 8 * i, desc(vb + i * 128), ID_O, add || i > 0);
                    if (last) tc_commit(smem_u32(&bars.o_done[h]));
                }
                __syncwarp();
            };
            while (w.left > 0 && ok) {
                g = ChSeg::of(a, w, s);
                const int halves = g.rows > HR ? 2 : 1;
                for (int h = 0; h < halves && g.tiles > 0 && ok; ++h) ok = wait(FMT == PF_I4 ? bars.q_ready[h] : bars.q_land[h], n_q[h]++ & 1);
                for (int t = 0; t <= g.tiles && ok && g.tiles > 0; ++t) {
                    // stages in order: K(0), V(0), K(1), ...: V(t - 1) then K(t)
                    const uint32_t vs = n_stage, ks = t > 0 ? n_stage + 1 : n_stage;
                    if (t > 0) ok = wait(bars.kv_full[vs % CH_STAGES], (vs / CH_STAGES) & 1);
                    if (t < g.tiles && ok) ok = wait(bars.kv_full[ks % CH_STAGES], (ks / CH_STAGES) & 1);
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        if (h >= halves || !ok) break;
                        if (t > 0) {
                            ok = wait(bars.p_ready[h][0], n_p[h] & 1);
                            if (!ok) break;
                            tc_after();
                            sums(h, vs % CH_STAGES, 0, t > 1, false);
                            ok = wait(bars.p_ready[h][1], n_p[h]++ & 1);
                            if (!ok) break;
                            tc_after();
                            sums(h, vs % CH_STAGES, 1, true, t == g.tiles);
                        }
                        if (t < g.tiles) {
                            tc_after();
                            scores(h, ks % CH_STAGES, t == g.tiles - 1);
                        }
                    }
                    if (!ok) break;
                    if (elect_one()) {
                        if (t > 0) tc_commit(smem_u32(&bars.kv_empty[vs % CH_STAGES]));
                        if (t < g.tiles) tc_commit(smem_u32(&bars.kv_empty[ks % CH_STAGES]));
                    }
                    __syncwarp();
                    n_stage += (t > 0) + (t < g.tiles);
                }
                w.left -= g.k1 - g.k0;
                if (w.left > 0) pt_next_far(w, s, a);
            }
            // what the instructions' ends arrive at is there until they have: the last uses of the stages and of Q, which
            // nobody else waits for; after an early leave, all that is under way
            for (uint32_t i = n_stage > CH_STAGES ? n_stage - CH_STAGES : 0; i < n_stage && ok; ++i) ok = wait(bars.kv_empty[i % CH_STAGES], (i / CH_STAGES) & 1);
            for (int h = 0; h < 2 && ok; ++h)
                if (n_q[h] > 0) ok = wait(bars.q_empty[h], (n_q[h] - 1) & 1);
            if (!ok) {
                if (elect_one()) tc_commit(smem_u32(&bars.left));
                __syncwarp();
                bar_drain(smem_u32(&bars.left), 0);
            }
        }
        if (wid == 13) {
            // ---------------- feeder: lane i < 128 / page copies page i of a tile
            uint32_t n_stage = 0, n_tile = 0;
            uint32_t n_q[2] = {0, 0}, n_land = 0;
            uint32_t landed = 0;                     // bit i: the copies of the last stage but i arrive on kv_full
            bool ok = true;
            const int per_page = 1 << a.pc.page_shift, n_pages = PT_KEYS >> a.pc.page_shift;
            if (FMT == PF_16 && lane == 0) asm volatile("prefetch.tensormap [%0];" ::"l"(&map) : "memory");
            while (w.left > 0 && ok) {
                g = ChSeg::of(a, w, s);
                int pid16 = g.tiles > 0 ? g.page_of(a, w, g.t0, lane) : -2;
                for (int k = g.t0; k < g.t0 + g.tiles && ok; ++k, ++n_tile) {
                    const int pid16n = k + 1 < g.t0 + g.tiles ? g.page_of(a, w, k + 1, lane) : -2;
                    const uint32_t bad = __ballot_sync(0xffffffffu, pid16 == -1), need = __ballot_sync(0xffffffffu, pid16 >= 0);
                    const bool clean = g.clean(a, k) && bad == 0;
                    if (bad != 0 && lane == 0) atomicMin(a.status, SALICACHE_E_CAPACITY);
                    // the first group of 16 keys of this lane's page that is needed names the page
                    const uint32_t mine = lane < n_pages ? need >> (lane << (a.pc.page_shift - 4)) & ((1u << (per_page >> 4)) - 1u) : 0u;
                    const int from = mine ? (lane << (a.pc.page_shift - 4)) + __ffs(mine) - 1 : 0;
                    const int pid = __shfl_sync(0xffffffffu, pid16, from);
                    const uint32_t copies = (uint32_t)__popc(__ballot_sync(0xffffffffu, mine != 0));
                    for (int kv = 0; kv < 2; ++kv, ++n_stage) {
                        const size_t slot = pg_slot(a.pc, mine ? pid : 0, kv, w.h, 0);
                        if (FMT == PF_16) {
                            const uint32_t stage = n_stage % CH_STAGES, dst = base + SM::KV + stage * SM::TILE, bar = smem_u32(&bars.kv_full[stage]);
                            if (n_stage >= CH_STAGES && !wait(bars.kv_empty[stage], (n_stage / CH_STAGES - 1) & 1)) {
                                ok = false;
                                break;
                            }
                            // V with keys that no row sees goes through group 2, which waits for it by barriers of their own (two: as
                            // many V stages as the ring has)
                            const bool direct = kv == 0 || clean;
                            const uint32_t land = direct ? bar : smem_u32(&bars.v_land[n_land & 1]);
                            if (lane == 0) {
                                if (kv == 0) *(volatile uint32_t*)&bars.pages[n_tile & 7] = ~bad & 0xffu;
                                bar_expect(land, copies * (uint32_t)(per_page * D * 2));
                            } else if (direct && lane < 4) bar_arrive(bar);
                            n_land += !direct;
                            landed = landed << 1 | (uint32_t)direct;
                            __syncwarp();
                            if (mine) {
#pragma unroll
                                for (int x = 0; x < D; x += 64) tensor_copy(dst + x * 256 + lane * per_page * 128, &map, x, (int)slot, land);
                            }
                        } else {
                            constexpr int N_RAW = SM::N_RAW > 0 ? SM::N_RAW : 1;
                            const uint32_t rs = n_stage % N_RAW, dst = base + SM::RAWS + rs * SM::RAW, bar = smem_u32(&bars.raw_full[rs]);
                            if (n_stage >= N_RAW && !wait(bars.raw_empty[rs], (n_stage / N_RAW - 1) & 1)) {
                                ok = false;
                                break;
                            }
                            constexpr uint32_t RB = pg_row_bytes<FMT, D>(), MB = pg_meta_bytes<FMT>();
                            if (lane == 0) {
                                if (kv == 0) *(volatile uint32_t*)&bars.pages[n_tile & 7] = ~bad & 0xffu;
                                bar_expect(bar, copies * per_page * (RB + MB));
                            }
                            __syncwarp();
                            if (mine) {
                                bulk_copy(dst + lane * per_page * RB, a.pc.data + slot * RB, per_page * RB, bar);
                                bulk_copy(dst + SM::RAW_CODES + lane * per_page * MB, a.pc.scale + slot * MB, per_page * MB, bar);
                            }
                        }
                    }
                    pid16 = pid16n;
                    if (k == g.t0 && ok) {               // Q behind the first tile: a lane per half
                        for (int h = 0; h < 2; ++h) {
                            if (h > 0 && g.rows <= HR) break;
                            if (n_q[h] > 0 && !wait(bars.q_empty[h], (n_q[h] - 1) & 1)) {
                                ok = false;
                                break;
                            }
                            ++n_q[h];
                            if (lane == 0) {
                                const uint32_t bar = smem_u32(&bars.q_land[h]);
                                bar_expect(bar, (uint32_t)(HR * D * 2));
                                for (int x = 0; x < D; x += 64)
                                    tensor_copy3(base + SM::Q + h * SM::TILE + x * 256, &q_map, x, w.h * a.G, s.row0 + (w.rt * 2 + h) * (HR / a.G), bar);
                            }
                        }
                        __syncwarp();
                    }
                }
                w.left -= g.k1 - g.k0;
                if (w.left > 0) pt_next_far(w, s, a);
            }
            join_roles();
            // copies in flight end before the block does: who uses a stage waits for them, unless a role has left early
            if (*gave_up) {
                constexpr uint32_t N = FMT == PF_16 ? CH_STAGES : SM::N_RAW > 0 ? SM::N_RAW : 1;
                for (uint32_t x = 0; x < N && x < n_stage; ++x) {
                    const uint32_t i = n_stage - 1 - x;
                    if (FMT != PF_16) bar_drain(smem_u32(&bars.raw_full[i % N]), (i / N) & 1);
                    else if (landed >> x & 1u) bar_drain(smem_u32(&bars.kv_full[i % N]), (i / N) & 1);
                }
                for (int h = 0; h < 2; ++h)
                    if (n_q[h] > 0) bar_drain(smem_u32(&bars.q_land[h]), (n_q[h] - 1) & 1);
                for (uint32_t i = n_land > 2 ? n_land - 2 : 0; i < n_land; ++i) bar_drain(smem_u32(&bars.v_land[i & 1]), i >> 1 & 1);
            }
            return;
        }
        __syncwarp();
    }
    tc_before();
    join_roles();
    if (tid == 0 && *gave_up) atomicMin(a.status, SC_GAVE_UP);
    if (wid == 12) {
        tc_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tmem) : "memory");
    }
}

// Joins split items: a thread per row, four dimensions at a time.  The blocks, one wave of them, share out the (item,
// dimensions) pairs; a block per pair that might be would mostly find nothing to do, in several waves.  What the blocks
// said of their records is read at once, so that nothing but the records themselves has to be waited for after it.
template <typename T, int D>
__global__ void __launch_bounds__(CH_ROWS, 2)
k_paged_join_chunk(PtArgs a, int blocks) {
    constexpr int PARTS = D / 4;
    __shared__ int list[PT_MAX_BLOCKS + 1], tails[PT_MAX_BLOCKS], kind[PT_MAX_BLOCKS], in_warp[CH_ROWS / 32];
    __shared__ int4 item[PT_MAX_BLOCKS];     // head, row tile, first row, rows
    const int lane = threadIdx.x & 31, wid = threadIdx.x >> 5, row = threadIdx.x;
    grid_wait();
    int n_tails = 0;                         // the blocks that left a tail, in their order
    for (int c0 = 0; c0 < blocks; c0 += CH_ROWS) {
        const int c = c0 + threadIdx.x;
        int4 hd = make_int4(0, 0, 0, 0), sq = hd;
        if (c < blocks) {
            hd = a.head[2 * c];
            sq = a.head[2 * c + 1];
            kind[c] = hd.x;
        }
        const uint32_t has = __ballot_sync(0xffffffffu, hd.y != 0);
        if (lane == 0) in_warp[wid] = __popc(has);
        __syncthreads();
        int at = n_tails + __popc(has & ((1u << lane) - 1u));
        for (int i = 0; i < CH_ROWS / 32; ++i) {
            if (i < wid) at += in_warp[i];
            n_tails += in_warp[i];
        }
        if (hd.y != 0) {
            tails[at] = c;
            item[at] = make_int4(hd.y - 1, hd.z, sq.x, sq.y);
        }
        __syncthreads();
    }
    // A unit is one item's sums of P x 4 dimensions, AHEAD records under way at a time.
    auto units = [&](auto p_, auto ahead_) {
        constexpr int P = decltype(p_)::value, AHEAD = decltype(ahead_)::value, UNITS = PARTS / P;
        for (int unit = blockIdx.x; unit < n_tails * UNITS; unit += gridDim.x) {
            const int blk = tails[unit / UNITS], part = unit % UNITS * P;
            const int4 it = item[unit / UNITS];
            const int n = pt_records([&](int c) { return kind[c]; }, blk, blocks, list);
            const int HR = a.tile_rows >> 1, rr = it.y * a.tile_rows + (row >> 7) * HR + (row & 127);
            if ((row & 127) < HR && rr < it.w * a.G) {
                // the maximum moves along with the records: one pass over them
                float M = PT_NONE, l = 0.0f;
                float4 o[P];
#pragma unroll
                for (int x = 0; x < P; ++x) o[x] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
                for (int i0 = 0; i0 < n; i0 += AHEAD) {
                    float2 st[AHEAD];
                    float4 v[AHEAD][P];
#pragma unroll
                    for (int u = 0; u < AHEAD; ++u) {
                        const size_t t = (size_t)list[min(i0 + u, n - 1)];
                        st[u] = a.stat[t * CH_ROWS + row];
#pragma unroll
                        for (int x = 0; x < P; ++x)
                            v[u][x] = __ldcs(reinterpret_cast<const float4*>(a.part) + (t * PARTS + part + x) * CH_ROWS + row);
                    }
                    float nm = M;
#pragma unroll
                    for (int u = 0; u < AHEAD; ++u) nm = fmaxf(nm, st[u].x);
                    const float f = ex2(M - nm);
                    M = nm;
                    l *= f;
#pragma unroll
                    for (int x = 0; x < P; ++x) o[x] = make_float4(o[x].x * f, o[x].y * f, o[x].z * f, o[x].w * f);
#pragma unroll
                    for (int u = 0; u < AHEAD; ++u) {
                        const float e = i0 + u < n ? ex2(st[u].x - M) : 0.0f;
                        l += e * st[u].y;
#pragma unroll
                        for (int x = 0; x < P; ++x) {
                            o[x].x += e * v[u][x].x;
                            o[x].y += e * v[u][x].y;
                            o[x].z += e * v[u][x].z;
                            o[x].w += e * v[u][x].w;
                        }
                    }
                }
                const int hq = it.x * a.G + rr % a.G;
                const long long tok = it.z + rr / a.G;
                const float inv = l > 0.0f ? 1.0f / l : 0.0f;
                uint2* dst = reinterpret_cast<uint2*>(a.out + tok * a.out_stride + (long long)hq * D + part * 4);
#pragma unroll
                for (int x = 0; x < P; ++x) dst[x] = make_uint2(T::pack(o[x].x * inv, o[x].y * inv), T::pack(o[x].z * inv, o[x].w * inv));
                if (a.lse && part == 0) a.lse[tok * ((long long)a.pc.heads * a.G) + hq] = l > 0.0f ? (M + log2f(l)) * PT_LN2 : -INFINITY;
            }
            __syncthreads();                 // the list is used up
        }
    };
    // A few rows over a long cache leave few items of many records each, a long prompt one item of two or three records at
    // every block's edge.
    if (n_tails * PARTS <= 2 * (int)gridDim.x) units(std::integral_constant<int, 1>{}, std::integral_constant<int, 12>{});
    else units(std::integral_constant<int, 4>{}, std::integral_constant<int, 3>{});
}

template <typename T, int FMT, int D, bool TREE>
int launch_chunk(salicache_ctx* c, PtArgs a, char* work, cudaStream_t st) {
    constexpr int BYTES = ChSmem<FMT, D>::BYTES;
    a.tile_rows = 2 * (128 / a.G) * a.G;
    CUtensorMap map{}, q_map{};
    if (!rows_map(&q_map, a.q, a.q_stride, a.pc.heads, a.G, a.sq.n_rows, D, T::ONE == TypeBF16::ONE)) return SALICACHE_E_CUDA;
    if (FMT == PF_16 && !page_map(&map, a.pc, D, T::ONE == TypeBF16::ONE)) return SALICACHE_E_CUDA;
    SC_CHECK(cudaFuncSetAttribute(k_paged_chunk<T, FMT, D, TREE>, cudaFuncAttributeMaxDynamicSharedMemorySize, BYTES));
    const int blocks = min(c->sm_count, PT_MAX_BLOCKS);
    a.part = reinterpret_cast<float*>(work);
    a.stat = reinterpret_cast<float2*>(a.part + (size_t)2 * blocks * CH_ROWS * D);
    a.head = reinterpret_cast<int4*>(a.stat + (size_t)2 * blocks * CH_ROWS);
    SC_CHECK(pt_launch(k_paged_chunk<T, FMT, D, TREE>, dim3(blocks), CH_THREADS, BYTES, st, a, map, q_map, blocks));
    SC_CHECK(pt_launch(k_paged_join_chunk<T, D>, dim3(2 * blocks), CH_ROWS, 0, st, a, blocks));
    c->launches += 2;
    return SALICACHE_OK;
}

template <typename T, int FMT, int D>
int chunk_tree(salicache_ctx* c, const PtArgs& a, char* work, cudaStream_t st) {
    return a.tree ? launch_chunk<T, FMT, D, true>(c, a, work, st) : launch_chunk<T, FMT, D, false>(c, a, work, st);
}
template <typename T, int D>
int chunk_format(salicache_ctx* c, const PtArgs& a, int format, char* work, cudaStream_t st) {
    if (format == SALICACHE_FP16) return chunk_tree<T, PF_16, D>(c, a, work, st);
    if (format == SALICACHE_INT8) return chunk_tree<T, PF_I8, D>(c, a, work, st);
    return chunk_tree<T, PF_I4, D>(c, a, work, st);
}

}  // namespace

int sc_paged_chunk(salicache_ctx* c, const PtArgs& a, const salicache_pages* pg, char* work, cudaStream_t st) {
    if (pg->dtype == SALICACHE_F16)
        return pg->head_dim == 128 ? chunk_format<TypeF16, 128>(c, a, pg->format, work, st) : chunk_format<TypeF16, 64>(c, a, pg->format, work, st);
    return pg->head_dim == 128 ? chunk_format<TypeBF16, 128>(c, a, pg->format, work, st) : chunk_format<TypeBF16, 64>(c, a, pg->format, work, st);
}
