// Attention of new rows over the paged cache, many rows per sequence (prompts, questions, new frames): the products are
// the work, and they run on the fifth-generation tensor cores (tcgen05.mma, accumulators in tensor memory).
//
// One block per SM walks its stretch of the line of (256 rows x 128 keys) tiles (paged_plan.cuh).  A tile's rows are two
// halves of 128 = the lanes of tensor memory; scores S = Q K^T and sums O += P V of both halves stand in all 512 columns.
// Roles by warp group:
//   0, 1   one thread per row of half 0 / 1: maximum over the row's 128 scores, weights, row sum; P overwrites S as the
//          16-bit operand of the second product; also Q into shared memory before an item and the output after it
//   2      K and V of the next tiles into a ring of shared-memory stages: 16-bit pages by asynchronous copies, codes
//          through registers (the next stage's codes are requested before the present ones are expanded)
//   3      one thread issues the matrix instructions
// While one half's weights are formed, the tensor core works for the other: the products of a half are issued as
// P(t) V(t), then Q K(t+1).  Instructions of one thread run in order there, so S may be overwritten right behind the
// product that read P from the same columns, and whoever sees the scores of tile t knows the sums of tile t-1 complete.
// The reference maximum moves only when a row exceeds it by 2^8; then, and only then, O is rescaled, by the thread that
// found it and before it hands its weights on.
//
// Both operands use the 128-byte swizzle: rows of 64 elements, eight rows to a 1024-byte atom.  K has the contracted
// dimension contiguous; V has it across rows, which the instruction descriptor's transpose bit covers, so neither is
// transposed in memory.  INT4 codes come out of their words in the order 0 4 1 5 2 6 3 7; Q is permuted alike when it is
// staged and the output back when it is written.
#include <math.h>

#include "paged_plan.cuh"

namespace {

constexpr int CH_ROWS = 256, CH_THREADS = 512, CH_STAGES = 4;
constexpr int CH_WAIT_LIMIT = 1 << 22;       // tries (each suspends for up to about a microsecond) before a wait gives up

__device__ __forceinline__ uint32_t smem_u32(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }

// ---- mbarriers
__device__ __forceinline__ void bar_init(uint32_t bar, int count) { asm volatile("mbarrier.init.shared.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory"); }
__device__ __forceinline__ void bar_arrive(uint32_t bar) { asm volatile("mbarrier.arrive.shared.b64 _, [%0];" ::"r"(bar) : "memory"); }
__device__ __forceinline__ bool bar_try(uint32_t bar, uint32_t parity) {
    uint32_t ok;
    asm volatile("{ .reg .pred p; mbarrier.try_wait.parity.shared.b64 p, [%1], %2, %3; selp.b32 %0, 1, 0, p; }"
                 : "=r"(ok) : "r"(bar), "r"(parity), "r"(1000u) : "memory");
    return ok != 0;
}
// False when the wait was given up, here or by another role: the caller leaves its loops.
__device__ __forceinline__ bool bar_wait(uint32_t bar, uint32_t parity, volatile int* gave_up) {
    if (bar_try(bar, parity)) return true;
    for (int i = 0; i < CH_WAIT_LIMIT; ++i) {
        if (bar_try(bar, parity)) return true;
        if (*gave_up) return false;
    }
    *gave_up = 1;
    return false;
}

// ---- tensor memory and tcgen05
__device__ __forceinline__ void tc_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_commit(uint32_t bar) {
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void tc_ld32(uint32_t* r, uint32_t addr) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,"
        "%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]),
          "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]),
          "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]),
          "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
        : "r"(addr)
        : "memory");
}
__device__ __forceinline__ void tc_ld16(uint32_t* r, uint32_t addr) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]),
          "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
        : "r"(addr)
        : "memory");
}
__device__ __forceinline__ void tc_st16(uint32_t addr, const uint32_t* r) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};" ::"r"(addr),
        "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]),
        "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
        : "memory");
}
__device__ __forceinline__ void tc_wait_ld() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tc_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// Shared-memory operand: 128-byte swizzle; `lead` = bytes between blocks of 64 elements (only where those are the rows of
// the result), 1024 bytes between groups of eight rows.
__device__ __forceinline__ uint64_t smem_desc(uint32_t addr, uint32_t lead) {
    return (uint64_t)((addr >> 4) & 0x3fffu) | (uint64_t)((lead >> 4) & 0x3fffu) << 16 | (uint64_t)(1024 >> 4) << 32 | 1ull << 46 | 2ull << 61;
}
// kind::f16, binary32 accumulator, M = 128; `vt`: B has the contracted dimension across its rows.
template <typename T>
__device__ __forceinline__ constexpr uint32_t instr_desc(int n, bool vt);
template <>
__device__ __forceinline__ constexpr uint32_t instr_desc<TypeF16>(int n, bool vt) {
    return 1u << 4 | (vt ? 1u << 16 : 0u) | (uint32_t)(n >> 3) << 17 | (128u >> 4) << 24;
}
template <>
__device__ __forceinline__ constexpr uint32_t instr_desc<TypeBF16>(int n, bool vt) { return instr_desc<TypeF16>(n, vt) | 1u << 7 | 1u << 10; }

__device__ __forceinline__ void mma_ss(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, bool add) {
    asm volatile("{ .reg .pred p; setp.ne.b32 p, %4, 0; tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p; }" ::"r"(d), "l"(a), "l"(b),
                 "r"(idesc), "r"((uint32_t)add)
                 : "memory");
}
__device__ __forceinline__ void mma_ts(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, bool add) {
    asm volatile("{ .reg .pred p; setp.ne.b32 p, %4, 0; tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p; }" ::"r"(d), "r"(a), "l"(b),
                 "r"(idesc), "r"((uint32_t)add)
                 : "memory");
}

// Byte offset of 16-byte piece `c` of row `r` in an operand tile of 128 rows.
__device__ __forceinline__ uint32_t swz(int r, int c) { return (uint32_t)((c >> 3) * 16384 + r * 128 + ((c ^ r) & 7) * 16); }
__device__ __forceinline__ void sts16(uint32_t addr, uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
    asm volatile("st.shared.v4.b32 [%0], {%1,%2,%3,%4};" ::"r"(addr), "r"(a), "r"(b), "r"(c), "r"(d) : "memory");
}
__device__ __forceinline__ void fence_async() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }

struct ChBars {
    uint64_t kv_full[CH_STAGES], kv_empty[CH_STAGES], q_ready[2], s_full[2], p_ready[2], o_done[2];
    uint32_t tmem;
    int gave_up;
    uint32_t pages[4];                       // per tile (in turn): bit g set: the page of keys 16 g .. 16 g + 15 exists
};

template <int D>
struct ChSmem {
    static constexpr int TILE = 128 * D * 2;         // bytes of an operand tile
    static constexpr int Q = 0, KV = 2 * TILE, BARS = KV + CH_STAGES * TILE, BYTES = BARS + (int)sizeof(ChBars) + 1024;
};

// A walk over a block's segments that every role repeats for itself.
struct ChSeg {
    PtSpan sp;
    int k0, k1, rows, tiles;                 // item tiles [k0, k1), rows in it (at most 256), tiles with keys
    __device__ __forceinline__ void set(const PtArgs& a, const PtWalk& w, const PgSeq& s) {
        sp = pt_item<CH_ROWS>(s, a, w.rt);
        k0 = w.k;
        k1 = (int)min((long long)max(sp.n, 1), k0 + w.left);
        rows = min(CH_ROWS, s.n * a.G - w.rt * CH_ROWS);
        tiles = sp.n == 0 ? 0 : k1 - k0;
    }
};

// What a loader thread holds of a stage of codes: PASSES rows, 16 bytes of each.
template <int FMT, int D>
struct CodeRegs {
    static constexpr int LPR = pg_row_bytes<FMT, D>() / 16 > 0 ? pg_row_bytes<FMT, D>() / 16 : 1;      // lanes per row = passes
    uint4 c[LPR];
    uint32_t s[LPR];
};

template <typename T, int FMT, int D>
__global__ void __launch_bounds__(CH_THREADS, 1)
k_paged_chunk(PtArgs a, int blocks) {
    using SM = ChSmem<D>;
    extern __shared__ uint8_t raw[];
    const uint32_t base = (smem_u32(raw) + 1023u) & ~1023u;
    ChBars& bars = *reinterpret_cast<ChBars*>(raw + (base - smem_u32(raw)) + SM::BARS);
    const int tid = threadIdx.x, wid = tid >> 5, lane = tid & 31;
    volatile int* gave_up = &bars.gave_up;

    if (tid == 0) {
        for (int i = 0; i < CH_STAGES; ++i) {
            bar_init(smem_u32(&bars.kv_full[i]), 128);
            bar_init(smem_u32(&bars.kv_empty[i]), 1);
        }
        for (int i = 0; i < 2; ++i) {
            bar_init(smem_u32(&bars.q_ready[i]), 128);
            bar_init(smem_u32(&bars.s_full[i]), 1);
            bar_init(smem_u32(&bars.p_ready[i]), 128);
            bar_init(smem_u32(&bars.o_done[i]), 1);
        }
        bars.gave_up = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (wid == 12) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_u32(&bars.tmem)) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    tc_before();
    PtWalk w = pt_start<CH_ROWS, CH_THREADS>(a, blockIdx.x, blocks);
    __syncthreads();
    tc_after();
    const uint32_t tmem = bars.tmem;
    const uint32_t TS[2] = {tmem, tmem + 128}, TO[2] = {tmem + 256, tmem + 256 + 128};
    PgSeq s{};
    if (w.left > 0) s = pg_seq(a.sq, a.pc, w.b);
    ChSeg g;

    if (wid < 8) {
        // ---------------- rows: softmax, Q, output
        asm volatile("setmaxnreg.inc.sync.aligned.u32 184;");
        const int half = wid >> 2, row = tid & 127;
        const uint32_t lane_base = (uint32_t)((wid & 3) * 32) << 16;
        const uint32_t S = TS[half] + lane_base, O = TO[half] + lane_base;
        const uint32_t q_ready = smem_u32(&bars.q_ready[half]), s_full = smem_u32(&bars.s_full[half]);
        const uint32_t p_ready = smem_u32(&bars.p_ready[half]), o_done = smem_u32(&bars.o_done[half]);
        uint32_t n_s = 0, n_o = 0, n_tile = 0;               // scores, outputs of this half and tiles seen so far
        int4 hd = make_int4(0, 0, 0, 0);
        bool ok = true;
        while (w.left > 0 && ok) {
            g.set(a, w, s);
            const bool first = g.k0 == 0, lastp = g.k1 == max(g.sp.n, 1), done = first && lastp;
            const int rows = min(128, g.rows - half * 128);  // of this half
            if (tid == 0 && s.cut && s.pos0 + s.n > s.len) atomicMin(a.status, SALICACHE_E_CAPACITY);
            if (rows > 0) {
                const int rr = w.rt * CH_ROWS + half * 128 + row;                 // this thread's row of the item
                const bool live = row < rows;
                const int pos = s.pos0 + (live ? rr : 0) / a.G;
                float m = PT_NONE, l = 0.0f;
                if (g.tiles > 0) {
                    // Q: a row by D / 8 lanes, 16 bytes each
                    constexpr int LPR = D / 8, RPP = 32 / LPR;
#pragma unroll 4
                    for (int p = 0; p < 32 / RPP; ++p) {
                        const int qr = (wid & 3) * 32 + p * RPP + lane / LPR, c = lane % LPR;
                        uint4 v = make_uint4(0, 0, 0, 0);
                        if (qr < rows) {
                            const int x = w.rt * CH_ROWS + half * 128 + qr;
                            v = __ldg(reinterpret_cast<const uint4*>(a.q + (long long)(s.row0 + x / a.G) * a.q_stride +
                                                                     (long long)(w.h * a.G + x % a.G) * D) + c);
                        }
                        if (FMT == PF_I4)        // the order in which codes leave their words
                            v = make_uint4(__byte_perm(v.x, v.z, 0x5410), __byte_perm(v.x, v.z, 0x7632), __byte_perm(v.y, v.w, 0x5410),
                                           __byte_perm(v.y, v.w, 0x7632));
                        sts16(base + SM::Q + half * SM::TILE + swz(qr, c), v.x, v.y, v.z, v.w);
                    }
                    fence_async();
                    bar_arrive(q_ready);
                    // positions that every row of this half sees in full tiles need no mask
                    const PtSpan hs = pt_span(s, a.G, w.rt * CH_ROWS + half * 128, w.rt * CH_ROWS + half * 128 + rows, a.window, a.sinks);
                    const int vis_hi = live ? max(0, min(pos + 1, s.len)) : 0;
                    const int vis_lo = a.window ? pos - a.window + 1 : 0;
                    for (int k = g.k0; k < g.k1 && ok; ++k, ++n_tile) {
                        ok = __all_sync(0xffffffffu, bar_wait(s_full, n_s & 1, gave_up));
                        ++n_s;
                        if (!ok) break;
                        tc_after();
                        uint32_t x[128];
                        tc_ld32(x, S);
                        tc_ld32(x + 32, S + 32);
                        tc_ld32(x + 64, S + 64);
                        tc_ld32(x + 96, S + 96);
                        tc_wait_ld();
                        const int j0 = g.sp.tile(k) * PT_KEYS;
                        const uint32_t pages = *(volatile uint32_t*)&bars.pages[n_tile & 3];
                        if (!(j0 + PT_KEYS <= hs.all_hi && (j0 >= hs.all_lo || j0 + PT_KEYS <= a.sinks) && pages == 0xffu)) {
                            const int hi = vis_hi - j0, lo = vis_lo - j0, sk = a.sinks - j0;
#pragma unroll
                            for (int i = 0; i < 128; ++i)
                                if (i >= hi || (i < lo && i >= sk) || !(pages >> (i >> 4) & 1u)) x[i] = 0xff800000u;
                        }
                        float mx[4] = {__uint_as_float(x[0]), __uint_as_float(x[1]), __uint_as_float(x[2]), __uint_as_float(x[3])};
#pragma unroll
                        for (int i = 4; i < 128; ++i) mx[i & 3] = fmaxf(mx[i & 3], __uint_as_float(x[i]));
                        const float top = fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3])) * a.scale;
                        if (k == g.k0) m = fmaxf(m, top);
                        else if (__any_sync(0xffffffffu, top > m + 8.0f)) {
                            const float nm = fmaxf(m, top), f = ex2(m - nm);
                            m = nm;
                            l *= f;
#pragma unroll
                            for (int c = 0; c < D; c += 16) {
                                uint32_t o[16];
                                tc_ld16(o, O + c);
                                tc_wait_ld();
#pragma unroll
                                for (int i = 0; i < 16; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * f);
                                tc_st16(O + c, o);
                            }
                        }
                        float sum[2] = {0.0f, 0.0f};
#pragma unroll
                        for (int c = 0; c < 4; ++c) {
                            uint32_t pk[16];
#pragma unroll
                            for (int i = 0; i < 16; ++i) {
                                const float p0 = ex2(fmaf(__uint_as_float(x[32 * c + 2 * i]), a.scale, -m));
                                const float p1 = ex2(fmaf(__uint_as_float(x[32 * c + 2 * i + 1]), a.scale, -m));
                                sum[0] += p0;
                                sum[1] += p1;
                                pk[i] = T::pack(p0, p1);
                            }
                            tc_st16(S + 16 * c, pk);
                        }
                        l += sum[0] + sum[1];
                        tc_wait_st();
                        tc_before();
                        bar_arrive(p_ready);
                    }
                    if (ok) {
                        ok = __all_sync(0xffffffffu, bar_wait(o_done, n_o & 1, gave_up));
                        ++n_o;
                        tc_after();
                    }
                }
                if (ok) {
                    // the output, or the partial record: float4 [D / 4][256 rows]
                    const size_t slot = 2 * (size_t)blockIdx.x + (first ? 1 : 0);
                    const float inv = l > 0.0f ? 1.0f / l : 0.0f;
                    const int hq = w.h * a.G + rr % a.G;
                    const long long tok = s.row0 + rr / a.G;
                    uint16_t* dst = a.out + tok * a.out_stride + (long long)hq * D;
                    float4* part = reinterpret_cast<float4*>(a.part) + slot * (D / 4) * CH_ROWS + half * 128 + row;
#pragma unroll
                    for (int c = 0; c < D; c += 32) {
                        uint32_t o[32];
                        __syncwarp();
                        if (g.tiles > 0) {
                            tc_ld32(o, O + c);
                            tc_wait_ld();
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
            if (!done) {
                if (first) {
                    hd.y = w.h + 1;
                    hd.z = w.b;
                    hd.w = w.rt;
                } else hd.x = lastp ? 2 : 1;
            }
            w.left -= g.k1 - g.k0;
            if (w.left > 0) pt_next<CH_ROWS>(w, s, a);
        }
        if (tid == 0) a.head[blockIdx.x] = hd;
    } else if (wid < 12) {
        // ---------------- loaders
        asm volatile("setmaxnreg.dec.sync.aligned.u32 88;");
        const int lw = wid - 8;                              // this warp's rows: 32 lw .. 32 lw + 31 of a tile
        uint32_t n_stage = 0, n_tile = 0, n_arrived = 0;
        bool ok = true;
        while (w.left > 0 && ok) {
            g.set(a, w, s);
            const int* table = a.sq.table + (size_t)w.b * a.sq.width;
            // pages of this warp's two groups of 16 keys of tile k: -2 no row sees them, -1 there is no such page
            auto page_of = [&](int k, int grp) -> int {
                if (k >= g.k1) return -2;
                const int j = g.sp.tile(k) * PT_KEYS + lw * 32 + grp * 16;
                if (j >= g.sp.hi || (j + 16 <= g.sp.lo && j >= a.sinks)) return -2;
                const int p = table[j >> a.pc.page_shift];
                return p >= 0 && p < a.pc.n_pages ? p : -1;
            };
            const int tiles_end = g.k0 + g.tiles;
            int pg0 = -2, pg1 = -2;
            if (g.tiles > 0) {
                pg0 = page_of(g.k0, 0);
                pg1 = page_of(g.k0, 1);
            }
            for (int k = g.k0; k < tiles_end && ok; ++k, ++n_tile) {
                const int nx0 = page_of(k + 1, 0), nx1 = page_of(k + 1, 1);
                const int j0 = g.sp.tile(k) * PT_KEYS + lw * 32;
                if ((pg0 == -1 || pg1 == -1) && lane == 0) atomicMin(a.status, SALICACHE_E_CAPACITY);
                // which of the tile's keys any row sees: others are stored as zeros, whatever the page holds
                auto want = [&](int r) -> int {              // r: row of this warp's 32; page id or -1
                    const int j = j0 + r, p = r < 16 ? pg0 : pg1;
                    return p >= 0 && j < g.sp.hi && (j >= g.sp.lo || j < a.sinks) ? p : -1;
                };
                for (int kv = 0; kv < 2 && ok; ++kv, ++n_stage) {
                    const uint32_t stage = n_stage % CH_STAGES, dst = base + SM::KV + stage * SM::TILE;
                    if (FMT == PF_16) {
                        if (n_stage >= CH_STAGES) ok = bar_wait(smem_u32(&bars.kv_empty[stage]), (n_stage / CH_STAGES - 1) & 1, gave_up);
                        if (!ok) break;
                        constexpr int LPR = D / 8, RPP = 32 / LPR;
                        const int c = lane % LPR;
#pragma unroll
                        for (int p = 0; p < 32 / RPP; ++p) {
                            const int r = p * RPP + lane / LPR;
                            const int pid = want(r);
                            const size_t slot = pg_slot(a.pc, max(pid, 0), kv, w.h, (j0 + r) & ((1 << a.pc.page_shift) - 1));
                            asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst + swz(lw * 32 + r, c)),
                                         "l"(a.pc.data + slot * (2 * D) + c * 16), "r"(pid >= 0 ? 16 : 0)
                                         : "memory");
                        }
                        asm volatile("cp.async.commit_group;" ::: "memory");
                    } else {
                        constexpr int LPR = CodeRegs<FMT, D>::LPR, RPP = 32 / LPR;
                        CodeRegs<FMT, D> cr;
                        const int c = lane % LPR;
#pragma unroll
                        for (int p = 0; p < LPR; ++p) {
                            const int r = p * RPP + lane / LPR, pid = want(r);
                            const size_t slot = pg_slot(a.pc, max(pid, 0), kv, w.h, (j0 + r) & ((1 << a.pc.page_shift) - 1));
                            cr.c[p] = make_uint4(0, 0, 0, 0);
                            cr.s[p] = 0;
                            if (pid >= 0) {
                                cr.c[p] = __ldg(reinterpret_cast<const uint4*>(a.pc.data + slot * pg_row_bytes<FMT, D>()) + c);
                                cr.s[p] = FMT == PF_I8 ? __ldg(reinterpret_cast<const uint16_t*>(a.pc.scale) + slot)
                                                       : __ldg(reinterpret_cast<const uint32_t*>(a.pc.scale) + slot);
                            }
                        }
                        if (n_stage >= CH_STAGES) ok = bar_wait(smem_u32(&bars.kv_empty[stage]), (n_stage / CH_STAGES - 1) & 1, gave_up);
                        if (!ok) break;
#pragma unroll
                        for (int p = 0; p < LPR; ++p) {
                            const int r = lw * 32 + p * RPP + lane / LPR;
                            const uint32_t words[4] = {cr.c[p].x, cr.c[p].y, cr.c[p].z, cr.c[p].w};
                            const uint32_t s2 = dup_lo(cr.s[p]), z2 = dup_hi(cr.s[p]);
                            if (FMT == PF_I8) {
#pragma unroll
                                for (int i = 0; i < 2; ++i)
                                    sts16(dst + swz(r, 2 * c + i), mul2<T>(Codes<T>::bytes(words[2 * i], 0x5140), s2),
                                          mul2<T>(Codes<T>::bytes(words[2 * i], 0x5342), s2), mul2<T>(Codes<T>::bytes(words[2 * i + 1], 0x5140), s2),
                                          mul2<T>(Codes<T>::bytes(words[2 * i + 1], 0x5342), s2));
                            } else {
#pragma unroll
                                for (int i = 0; i < 4; ++i) {
                                    const uint32_t y = words[i] >> 8;
                                    sts16(dst + swz(r, 4 * c + i), fma2<T>(Codes<T>::nib_lo(words[i]), s2, z2), fma2<T>(Codes<T>::nib_hi(words[i]), s2, z2),
                                          fma2<T>(Codes<T>::nib_lo(y), s2, z2), fma2<T>(Codes<T>::nib_hi(y), s2, z2));
                                }
                            }
                        }
                    }
                    // which pages exist: read by the rows of this tile, whose scores come after this stage
                    if (kv == 0 && tid == 8 * 32) {
                        uint32_t mask = 0;
                        for (int i = 0; i < 8; ++i) {
                            const int j = g.sp.tile(k) * PT_KEYS + i * 16;
                            bool there = true;
                            if (j < g.sp.hi && !(j + 16 <= g.sp.lo && j >= a.sinks)) {
                                const int p = table[j >> a.pc.page_shift];
                                there = p >= 0 && p < a.pc.n_pages;
                            }
                            mask |= (there ? 1u : 0u) << i;
                        }
                        *(volatile uint32_t*)&bars.pages[n_tile & 3] = mask;
                    }
                    if (FMT == PF_16) {
                        // the copies of two stages may still be under way
                        if (n_stage >= 2) {
                            asm volatile("cp.async.wait_group 2;" ::: "memory");
                            fence_async();
                            bar_arrive(smem_u32(&bars.kv_full[n_arrived++ % CH_STAGES]));
                        }
                    } else {
                        fence_async();
                        bar_arrive(smem_u32(&bars.kv_full[stage]));
                    }
                }
                pg0 = nx0;
                pg1 = nx1;
            }
            w.left -= g.k1 - g.k0;
            if (w.left > 0) pt_next<CH_ROWS>(w, s, a);
        }
        if (FMT == PF_16) {
            asm volatile("cp.async.wait_all;" ::: "memory");
            fence_async();
            while (n_arrived < n_stage) bar_arrive(smem_u32(&bars.kv_full[n_arrived++ % CH_STAGES]));
        }
    } else {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 56;");
        if (wid == 12 && lane == 0) {
            // ---------------- matrix instructions
            constexpr uint32_t ID_S = instr_desc<T>(128, false), ID_O = instr_desc<T>(D, true);
            uint32_t n_stage = 0, n_q[2] = {0, 0}, n_p[2] = {0, 0};
            bool ok = true;
            auto scores = [&](int h, uint32_t st) {
                const uint32_t qa = base + SM::Q + h * SM::TILE, kb = base + SM::KV + st * SM::TILE;
#pragma unroll
                for (int i = 0; i < D / 16; ++i) {
                    const uint32_t off = (i >> 2) * 16384 + (i & 3) * 32;
                    mma_ss(TS[h], smem_desc(qa + off, 16), smem_desc(kb + off, 16), ID_S, i > 0);
                }
                tc_commit(smem_u32(&bars.s_full[h]));
            };
            auto sums = [&](int h, uint32_t st, bool add) {
                const uint32_t vb = base + SM::KV + st * SM::TILE;
#pragma unroll
                for (int i = 0; i < PT_KEYS / 16; ++i) mma_ts(TO[h], TS[h] + 8 * i, smem_desc(vb + i * 2048, 16384), ID_O, add || i > 0);
            };
            while (w.left > 0 && ok) {
                g.set(a, w, s);
                const int halves = g.rows > 128 ? 2 : 1;
                for (int h = 0; h < halves && ok && g.tiles > 0; ++h) ok = bar_wait(smem_u32(&bars.q_ready[h]), n_q[h]++ & 1, gave_up);
                for (int t = 0; t <= g.tiles && ok && g.tiles > 0; ++t) {
                    // stages in order: K(0), V(0), K(1), ...: V(t - 1) then K(t)
                    const uint32_t vs = n_stage, ks = t > 0 ? n_stage + 1 : n_stage;
                    if (t > 0) ok = bar_wait(smem_u32(&bars.kv_full[vs % CH_STAGES]), (vs / CH_STAGES) & 1, gave_up);
                    for (int h = 0; h < halves && ok; ++h) {
                        if (t > 0) {
                            ok = bar_wait(smem_u32(&bars.p_ready[h]), n_p[h]++ & 1, gave_up);
                            if (!ok) break;
                            tc_after();
                            sums(h, vs % CH_STAGES, t > 1);
                            if (t == g.tiles) tc_commit(smem_u32(&bars.o_done[h]));
                        }
                        if (t < g.tiles) {
                            if (h == 0) ok = bar_wait(smem_u32(&bars.kv_full[ks % CH_STAGES]), (ks / CH_STAGES) & 1, gave_up);
                            if (!ok) break;
                            tc_after();
                            scores(h, ks % CH_STAGES);
                        }
                    }
                    if (!ok) break;
                    if (t > 0) {
                        tc_commit(smem_u32(&bars.kv_empty[vs % CH_STAGES]));
                        ++n_stage;
                    }
                    if (t < g.tiles) {
                        tc_commit(smem_u32(&bars.kv_empty[ks % CH_STAGES]));
                        if (t == 0) ++n_stage;
                        else ++n_stage;
                    }
                }
                w.left -= g.k1 - g.k0;
                if (w.left > 0) pt_next<CH_ROWS>(w, s, a);
            }
        }
        __syncwarp();
    }
    tc_before();
    __syncthreads();
    if (tid == 0 && bars.gave_up) atomicMin(a.status, SALICACHE_E_CUDA);
    if (wid == 12) {
        if (bars.gave_up) {                  // a role left early: matrix instructions may be under way
            if (lane == 0) {
                bar_init(smem_u32(&bars.o_done[0]), 1);
                tc_commit(smem_u32(&bars.o_done[0]));
                for (int i = 0; i < CH_WAIT_LIMIT && !bar_try(smem_u32(&bars.o_done[0]), 0); ++i) {}
            }
            __syncwarp();
        }
        tc_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tmem) : "memory");
    }
}

// Joins the records of the item that block blockIdx.x left as its tail: a thread per row, grid.y over 32 dimensions each.
template <typename T, int D>
__global__ void __launch_bounds__(CH_ROWS)
k_paged_join_chunk(PtArgs a, int blocks) {
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int4 hd = a.head[blockIdx.x];
    if (hd.y == 0) return;
    const int row = threadIdx.x, b = hd.z, h = hd.y - 1, rt = hd.w;
    const PgSeq s = pg_seq(a.sq, a.pc, b);
    const int rr = rt * CH_ROWS + row;
    if (rr >= s.n * a.G) return;
    const size_t t0 = 2 * (size_t)blockIdx.x + 1;
    float M = a.stat[t0 * CH_ROWS + row].x;
    int last = blockIdx.x;
    for (int c = blockIdx.x + 1; c < blocks; ++c) {
        const int f = a.head[c].x;
        if (f == 0) continue;
        M = fmaxf(M, a.stat[(size_t)(2 * c) * CH_ROWS + row].x);
        last = c;
        if (f == 2) break;
    }
    float4 o[8];
    float l = 0.0f;
#pragma unroll
    for (int i = 0; i < 8; ++i) o[i] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    for (int c = blockIdx.x; c <= last; ++c) {
        if (c != blockIdx.x && a.head[c].x == 0) continue;
        const size_t t = c == blockIdx.x ? t0 : 2 * (size_t)c;
        const float2 st = a.stat[t * CH_ROWS + row];
        const float e = ex2(st.x - M);
        l += e * st.y;
        const float4* src = reinterpret_cast<const float4*>(a.part) + (t * (D / 4) + blockIdx.y * 8) * CH_ROWS + row;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float4 v = __ldcs(src + i * CH_ROWS);
            o[i].x += e * v.x;
            o[i].y += e * v.y;
            o[i].z += e * v.z;
            o[i].w += e * v.w;
        }
    }
    const int hq = h * a.G + rr % a.G;
    const long long tok = s.row0 + rr / a.G;
    const float inv = l > 0.0f ? 1.0f / l : 0.0f;
    uint4* dst = reinterpret_cast<uint4*>(a.out + tok * a.out_stride + (long long)hq * D + blockIdx.y * 32);
#pragma unroll
    for (int i = 0; i < 4; ++i)
        dst[i] = make_uint4(T::pack(o[2 * i].x * inv, o[2 * i].y * inv), T::pack(o[2 * i].z * inv, o[2 * i].w * inv),
                            T::pack(o[2 * i + 1].x * inv, o[2 * i + 1].y * inv), T::pack(o[2 * i + 1].z * inv, o[2 * i + 1].w * inv));
    if (a.lse && blockIdx.y == 0) a.lse[tok * ((long long)a.pc.heads * a.G) + hq] = l > 0.0f ? (M + log2f(l)) * PT_LN2 : -INFINITY;
}

template <typename T, int FMT, int D>
int launch_chunk(salicache_ctx* c, PtArgs a, char* work, cudaStream_t st) {
    constexpr int BYTES = ChSmem<D>::BYTES;
    SC_CHECK(cudaFuncSetAttribute(k_paged_chunk<T, FMT, D>, cudaFuncAttributeMaxDynamicSharedMemorySize, BYTES));
    const int blocks = c->sm_count;
    a.part = reinterpret_cast<float*>(work);
    a.stat = reinterpret_cast<float2*>(a.part + (size_t)2 * blocks * CH_ROWS * D);
    a.head = reinterpret_cast<int4*>(a.stat + (size_t)2 * blocks * CH_ROWS);
    k_paged_chunk<T, FMT, D><<<blocks, CH_THREADS, BYTES, st>>>(a, blocks);
    SC_CHECK(cudaGetLastError());
    cudaLaunchConfig_t cfg{};
    cudaLaunchAttribute at{};
    at.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at.val.programmaticStreamSerializationAllowed = 1;
    cfg.gridDim = dim3(blocks, D / 32);
    cfg.blockDim = dim3(CH_ROWS);
    cfg.stream = st;
    cfg.attrs = &at;
    cfg.numAttrs = 1;
    SC_CHECK(cudaLaunchKernelEx(&cfg, k_paged_join_chunk<T, D>, a, blocks));
    c->launches += 2;
    return SALICACHE_OK;
}

template <typename T, int D>
int chunk_format(salicache_ctx* c, const PtArgs& a, int format, char* work, cudaStream_t st) {
    if (format == SALICACHE_FP16) return launch_chunk<T, PF_16, D>(c, a, work, st);
    if (format == SALICACHE_INT8) return launch_chunk<T, PF_I8, D>(c, a, work, st);
    return launch_chunk<T, PF_I4, D>(c, a, work, st);
}

}  // namespace

int sc_paged_chunk(salicache_ctx* c, const PtArgs& a, const salicache_pages* pg, char* work, cudaStream_t st) {
    if (pg->dtype == SALICACHE_F16)
        return pg->head_dim == 128 ? chunk_format<TypeF16, 128>(c, a, pg->format, work, st) : chunk_format<TypeF16, 64>(c, a, pg->format, work, st);
    return pg->head_dim == 128 ? chunk_format<TypeBF16, 128>(c, a, pg->format, work, st) : chunk_format<TypeBF16, 64>(c, a, pg->format, work, st);
}
