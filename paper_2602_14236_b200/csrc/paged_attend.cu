// Attention of new rows over the paged cache (Eq. 2 with the dequantisation of Sec. III-C fused in).
//
//   a_j = scale q . K^_j over the visible j,  m = max_j a_j,  l = sum_j e^(a_j - m),  out = sum_j e^(a_j - m) V^_j / l
//
// This file: few rows per sequence (single tokens, short drafts), where reading the pages is the work.
//
// A warp takes 16 keys of one head at a time, and both products are m16n8k16 matrix instructions with the keys as the
// long side, since there are few rows: scores = K (16 keys x 16 dimensions) times up to 8 rows of q as columns; values =
// V transposed (16 dimensions x 16 keys) times the weights, transposed in registers by movmatrix.  Any order of the
// dimensions that q and K share will do, as will any that V and the output share, and any of the keys: a lane reads up to
// 16 contiguous bytes wherever the rows have them, straight into the registers that hold its operands; codes become the
// 16-bit type there.
// One more warp feeds a ring of tiles in shared memory by bulk copies of whole pages, so that some 130 to 200 KB per SM are
// under way whatever the registers hold.  (Loading each lane's next operands into registers instead: 32 ragged streams
// over INT4 pages took 149 us.)
// Measured: 16-bit pages, 16 sequences of 8000 positions: 99 us = 5.3 TB/s, 0.83 of the copy bandwidth, bound by memory;
// INT8: 65 us = 4.1 TB/s; INT4, 32 ragged streams, 270 MB: 94 us = 2.9 TB/s = 0.45.  Over codes neither memory nor the issue
// slots are full (60 % of them for INT4, 51 % for INT8): a warp's load, expansion, products, maximum, expansion and products
// follow one another, with nothing of the next keys under way, and 4.2 warps a scheduler do not cover that.  The ninth
// warp leaves two blocks 96 registers a thread, of which codes at head_dim 128 spill some (184 bytes for f16 INT4, 268 for
// INT8).  446 instructions go into 16 INT4 keys of a head; 192 of them turn codes into numbers (and, subtract,
// multiply-add per pair of them: the values attended to are of the 16-bit type, so the scales stay inside the sums).
// The weights' reference maximum moves only when a score exceeds it by 2^8 (in powers of two): until then no lane needs
// another's, weights stay below 2^8, and the sums are joined across lanes once at the end of an item.
#include <math.h>

#include "paged_plan.cuh"

namespace {

constexpr int ST_WARPS = 8, ST_THREADS = 32 * (ST_WARPS + 1);        // eight that compute, one that feeds
constexpr int ST_ROUND = 4;                  // rows joined across the warps at a time
static_assert(ST_WARPS * 16 == PT_KEYS, "a warp per 16 keys of a tile");

// A stage of the ring: 128 keys' K and V rows, then their scales.
template <int FMT, int D, int NT>
struct StSmem {
    static constexpr int ROWS = 128 * pg_row_bytes<FMT, D>(), META = 128 * pg_meta_bytes<FMT>(), STAGE = 2 * (ROWS + META);
    static constexpr int K = 0, V = ROWS, KM = 2 * ROWS, VM = 2 * ROWS + META;
    static constexpr int ACC = ST_WARPS * ST_ROUND * (D + 4) * 4, Q = 8 * NT * D * 2;       // Q: rows of an item
    // two blocks per SM where a ring of two stages leaves room for them, and the registers of 8 rows do
    static constexpr int BLOCKS = NT == 1 && 2 * STAGE + ACC + 2 * Q <= 110 * 1024 ? 2 : 1;
    static constexpr int ROOM = (BLOCKS == 2 ? 110 * 1024 : 222 * 1024) - ACC - 2 * Q;
    static constexpr int STAGES = ROOM / STAGE < 8 ? ROOM / STAGE : 8;
    static constexpr int BYTES = STAGES * STAGE + ACC + 2 * Q;
    // an item's fixed cost (its rows of q, joining the warps, the output) in tiles' time, as measured
    static constexpr int ITEM = FMT == PF_I4 ? 3 : 2;
};

template <typename T>
__device__ __forceinline__ void mma16816(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1);
template <>
__device__ __forceinline__ void mma16816<TypeF16>(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
template <>
__device__ __forceinline__ void mma16816<TypeBF16>(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// Joins the computing warps; whether any of their threads says so.
__device__ __forceinline__ bool any_of(bool x) {
    uint32_t r;
    asm volatile("{ .reg .pred p, q; setp.ne.b32 p, %1, 0; barrier.cta.red.or.pred q, 1, %2, p; selp.b32 %0, 1, 0, q; }"
                 : "=r"(r) : "r"((uint32_t)x), "n"(ST_WARPS * 32) : "memory");
    return r != 0;
}
__device__ __forceinline__ uint32_t transpose8(uint32_t x) {
    uint32_t d;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(d) : "r"(x));
    return d;
}
// Key of row slot r of the fragments: the keys 2 c, 2 c + 1 that a lane multiplies are c and c + 4, which lie in
// different banks.
__device__ __forceinline__ int key_of(int g8) { return (g8 >> 1) + 4 * (g8 & 1); }

// What a lane (g8 = lane / 4, c4 = lane % 4) takes of 16 keys: the shares of the keys of slots g8 and g8 + 8 of K that make
// its A fragments, and its share of slots 2 c4, 2 c4 + 1, 2 c4 + 8, 2 c4 + 9 of V.
template <int FMT, int D>
struct KTile {
    static constexpr int W = pg_row_bytes<FMT, D>() / 16;       // words of a key row per lane
    uint32_t k[2][W];
    uint32_t s[2];                                              // scale, or (scale, zero)
    static constexpr int RB = pg_row_bytes<FMT, D>(), MB = pg_meta_bytes<FMT>();
    // this lane's first bytes of 16 keys' rows, and of their scales
    static __device__ __forceinline__ uint32_t at(int g8, int c4) { return key_of(g8) * RB + (RB >= 64 ? 16 : 8) * c4; }
    static __device__ __forceinline__ uint32_t meta_at(int g8) { return key_of(g8) * MB; }
    __device__ __forceinline__ void load(uint32_t rows, uint32_t meta) {
#pragma unroll
        for (int r = 0; r < 2; ++r) {
            if (RB >= 64) {
#pragma unroll
                for (int i = 0; i < RB / 64; ++i) lds16(&k[r][4 * i], rows + 8 * r * RB + 64 * i);
            } else lds_words<2>(&k[r][0], rows + 8 * r * RB);
            if (FMT == PF_I8) s[r] = lds_u16(meta + 8 * r * MB);
            if (FMT == PF_I4) lds_words<1>(&s[r], meta + 8 * r * MB);
        }
    }
};
template <int FMT, int D>
struct VTile {
    static constexpr int W = pg_row_bytes<FMT, D>() / 32;       // words of a value row per lane
    uint32_t v[4][W];
    uint32_t s[2][FMT == PF_I4 ? 2 : 1];                        // per pair of keys: their scales in one word, or (scale, zero) each
    static constexpr int RB = pg_row_bytes<FMT, D>(), MB = pg_meta_bytes<FMT>();
    static __device__ __forceinline__ uint32_t at(int g8, int c4) { return c4 * RB + (W == 8 ? 16 : 4 * W) * g8; }
    static __device__ __forceinline__ uint32_t meta_at(int c4) { return c4 * MB; }
    __device__ __forceinline__ void load(uint32_t rows, uint32_t meta) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int key = 4 * (j & 1) + 8 * (j >> 1);          // from this lane's first
            const uint32_t p = rows + key * RB;
            if (W == 8) {
                lds16(&v[j][0], p);
                lds16(&v[j][W == 8 ? 4 : 0], p + 128);
            } else lds_words<W == 8 ? 4 : W>(&v[j][0], p);
            if (FMT == PF_I4) lds_words<1>(&s[j >> 1][FMT == PF_I4 ? j & 1 : 0], meta + key * MB);
            if (FMT == PF_I8) {
                const uint32_t x = lds_u16(meta + key * MB);
                s[j >> 1][0] = (j & 1) ? s[j >> 1][0] | x << 16 : x;
            }
        }
    }
};

// K fragments of matrix instruction st: registers (a0, a2) of one key row.
template <typename T, int FMT, int D>
__device__ __forceinline__ void key_frag(const Codes<T>& cd, const uint32_t (&k)[KTile<FMT, D>::W], uint32_t s, int st, uint32_t& x, uint32_t& y) {
    if (FMT == PF_16) {
        x = k[2 * st];
        y = k[2 * st + 1];
    } else if (FMT == PF_I8) {
        const uint32_t s2 = dup_lo(s);
        x = mul2<T>(cd.bytes(k[st], 0x5140), s2);
        y = mul2<T>(cd.bytes(k[st], 0x5342), s2);
    } else {
        const uint32_t s2 = dup_lo(s), z2 = dup_hi(s), w = k[st >> 1] >> (8 * (st & 1));
        x = fma2<T>(cd.nib_lo(w), s2, z2);
        y = fma2<T>(cd.nib_hi(w), s2, z2);
    }
}
// The dimension pairs that instruction st multiplies in a lane's registers b0 and b1.
template <int FMT>
__device__ __forceinline__ void q_dims(int st, int c4, int D, int (&d)[4]) {
    if (FMT == PF_16) {
        const int base = (st >> 1) * 32 + c4 * 8 + (st & 1) * 4;
        d[0] = base; d[1] = base + 1; d[2] = base + 2; d[3] = base + 3;
    } else if (FMT == PF_I8) {
        const int base = (st >> 2) * 64 + c4 * 16 + (st & 3) * 4;
        d[0] = base; d[1] = base + 1; d[2] = base + 2; d[3] = base + 3;
    } else {
        const int base = c4 * (D / 4) + (st >> 1) * 8 + (st & 1) * 2;      // nibbles 2 (st & 1) and + 4; then + 1 and + 5
        d[0] = base; d[1] = base + 4; d[2] = base + 1; d[3] = base + 5;
    }
}
// V fragments of dimension tile t: rows g8 (half 0) and g8 + 8 (half 1) of V transposed, key pairs 0 and 1.
template <typename T, int FMT, int D>
__device__ __forceinline__ uint32_t value_frag(const Codes<T>& cd, const VTile<FMT, D>& v, int t, int half, int pair) {
    constexpr int NT = D / 16;
    const int x = half * NT + t;                        // which of the lane's D / 8 dimensions
    const uint32_t *A = v.v[2 * pair], *B = v.v[2 * pair + 1];
    if (FMT == PF_16) return __byte_perm(A[x >> 1], B[x >> 1], (x & 1) ? 0x7632 : 0x5410);
    if (FMT == PF_I8) {
        const uint32_t ab = __byte_perm(A[x >> 2], B[x >> 2], (x & 2) ? 0x7632 : 0x5410);      // bytes A, A+1, B, B+1
        return mul2<T>(cd.bytes(ab, (x & 1) ? 0x5341 : 0x5240), v.s[pair][0]);
    }
    const uint32_t ab = __byte_perm(A[x >> 3], B[x >> 3], (x & 4) ? 0x7632 : 0x5410);          // 4 nibbles of A, 4 of B
    const uint32_t w = (x & 2) ? ab >> 8 : ab;
    const uint32_t s2 = __byte_perm(v.s[pair][0], v.s[pair][FMT == PF_I4 ? 1 : 0], 0x5410);
    const uint32_t z2 = __byte_perm(v.s[pair][0], v.s[pair][FMT == PF_I4 ? 1 : 0], 0x7632);
    return fma2<T>((x & 1) ? cd.nib_hi(w) : cd.nib_lo(w), s2, z2);
}
template <int FMT, int D>
__device__ __forceinline__ int value_dim(int t, int half, int g8) {
    if (FMT == PF_16 && D == 128) return 64 * half + 8 * g8 + t;
    return g8 * (D / 8) + half * (D / 16) + t;
}

// NT: 8-row column tiles per item.
template <typename T, int FMT, int D, int NT>
__global__ void __launch_bounds__(ST_THREADS, StSmem<FMT, D, NT>::BLOCKS)
k_paged_step(PtArgs a, int blocks) {
    using SM = StSmem<FMT, D, NT>;
    constexpr int RT = 8 * NT, KS = D / 16, VS = D / 16, STAGES = SM::STAGES;
    static_assert(STAGES >= 2, "ring");
    extern __shared__ __align__(128) uint8_t ring[];
    __shared__ uint64_t full[STAGES], empty[STAGES], q_full[2], q_empty[2];
    __shared__ uint32_t kinds[STAGES];       // per stage: bit g: some row sees keys 16 g .. and their page exists
    __shared__ float2 sh_stat[ST_WARPS][ST_ROUND];
    __shared__ PtShared sh_plan;
    __shared__ int sh_gave_up;
    using Seg = PtSeg<SM::ITEM>;
    const uint32_t q_ring = smem_u32(ring) + STAGES * SM::STAGE + SM::ACC;
    float (*sh_acc)[ST_ROUND][D + 4] = reinterpret_cast<float (*)[ST_ROUND][D + 4]>(ring + STAGES * SM::STAGE);
    volatile int* gave_up = &sh_gave_up;
    const int lane = threadIdx.x & 31, wid = threadIdx.x >> 5, g8 = lane >> 2, c4 = lane & 3;
    const int c = blockIdx.x;
    if (threadIdx.x == 0) {
        for (int i = 0; i < STAGES; ++i) {
            bar_init(smem_u32(&full[i]), 1);
            bar_init(smem_u32(&empty[i]), ST_WARPS);
        }
        for (int i = 0; i < 2; ++i) {
            bar_init(smem_u32(&q_full[i]), 1);
            bar_init(smem_u32(&q_empty[i]), ST_WARPS);
        }
        sh_gave_up = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    grid_wait();
    grid_release();
    const PtPlace start = pt_start<ST_THREADS, SM::ITEM>(a, c, blocks, sh_plan);
    PtWalk w = start.w;
    PgSeq s = start.s;
    __syncthreads();
    int4 hd[2] = {make_int4(0, 0, 0, 0), make_int4(0, 0, 0, 0)};
    uint32_t n_stage = 0, n_q = 0;
    bool ok = true;
    Seg g;

    if (wid == ST_WARPS) {
        // ---------------- feeder: a lane per (page of the tile, K rows | V rows | K scales | V scales)
        const int per_page = 1 << a.pc.page_shift, n_pages = PT_KEYS >> a.pc.page_shift;
        constexpr int PIECES = FMT == PF_16 ? 2 : 4;
        const int page = lane / PIECES, piece = lane % PIECES;
        constexpr uint32_t RB = pg_row_bytes<FMT, D>(), MB = pg_meta_bytes<FMT>();
        while (w.left > 0 && ok) {
            g.set(a, w, s);
            if (g.tiles > 0) {               // the item's rows of q, a lane per row
                const uint32_t qb = n_q & 1, bar = smem_u32(&q_full[qb]);
                if (n_q >= 2 && !warp_wait(smem_u32(&q_empty[qb]), (n_q / 2 - 1) & 1, a.wait_limit, gave_up)) break;
                __syncwarp();
                if (lane == 0) bar_expect(bar, (uint32_t)g.rows * (D * 2));
                __syncwarp();
                if (lane < g.rows) {
                    const int rr = w.rt * RT + lane;
                    bulk_copy(q_ring + qb * SM::Q + lane * (D * 2),
                              a.q + (long long)(s.row0 + rr / a.G) * a.q_stride + (long long)(w.h * a.G + rr % a.G) * D, D * 2, bar);
                }
                ++n_q;
            }
            int next = g.tiles > 0 ? g.page_of(a, w, g.t0, lane) : -2;
            for (int k = g.t0; k < g.t0 + g.tiles; ++k, ++n_stage) {
                const int pid16 = next;
                next = k + 1 < g.t0 + g.tiles ? g.page_of(a, w, k + 1, lane) : -2;
                const uint32_t bad = __ballot_sync(0xffffffffu, pid16 == -1), need = __ballot_sync(0xffffffffu, pid16 >= 0);
                if (bad != 0 && lane == 0) atomicMin(a.status, SALICACHE_E_CAPACITY);
                const uint32_t mine = page < n_pages ? need >> (page << (a.pc.page_shift - 4)) & ((1u << (per_page >> 4)) - 1u) : 0u;
                const int from = mine ? (page << (a.pc.page_shift - 4)) + __ffs(mine) - 1 : 0;
                const int pid = __shfl_sync(0xffffffffu, pid16, from);
                const uint32_t copies = (uint32_t)__popc(__ballot_sync(0xffffffffu, mine != 0 && piece == 0));
                const uint32_t st = n_stage % STAGES, bar = smem_u32(&full[st]), dst = smem_u32(ring) + st * SM::STAGE;
                if (n_stage >= STAGES && !warp_wait(smem_u32(&empty[st]), (n_stage / STAGES - 1) & 1, a.wait_limit, gave_up)) {
                    ok = false;
                    break;
                }
                __syncwarp();
                if (lane == 0) {
                    *(volatile uint32_t*)&kinds[st] = need;
                    bar_expect(bar, copies * per_page * 2 * (RB + MB));
                }
                __syncwarp();
                if (mine) {
                    const size_t slot = pg_slot(a.pc, pid, piece & 1, w.h, 0);
                    const uint32_t at = (uint32_t)(page << a.pc.page_shift);
                    if (piece < 2) bulk_copy(dst + (piece ? SM::V : SM::K) + at * RB, a.pc.data + slot * RB, per_page * RB, bar);
                    else bulk_copy(dst + (piece == 3 ? SM::VM : SM::KM) + at * MB, a.pc.scale + slot * MB, per_page * MB, bar);
                }
            }
            w.left -= g.k1 - g.k0;
            if (w.left > 0) pt_next(w, s, a);
        }
        join_roles();
        if (*gave_up) {                      // copies in flight end before the block does
            for (uint32_t i = n_stage > STAGES ? n_stage - STAGES : 0; i < n_stage; ++i) bar_drain(smem_u32(&full[i % STAGES]), (i / STAGES) & 1);
            for (uint32_t i = n_q > 2 ? n_q - 2 : 0; i < n_q; ++i) bar_drain(smem_u32(&q_full[i & 1]), (i / 2) & 1);
        }
        return;
    }

    const Codes<T> cd;
    uint32_t stage = 0, phase = 0;
    // this lane's places in a stage
    constexpr uint32_t RB16 = 16 * pg_row_bytes<FMT, D>(), MB16 = 16 * pg_meta_bytes<FMT>();
    const uint32_t k_at = SM::K + wid * RB16 + KTile<FMT, D>::at(g8, c4), km_at = SM::KM + wid * MB16 + KTile<FMT, D>::meta_at(g8);
    const uint32_t v_at = SM::V + wid * RB16 + VTile<FMT, D>::at(g8, c4), vm_at = SM::VM + wid * MB16 + VTile<FMT, D>::meta_at(c4);
    while (w.left > 0 && ok) {
        g.set(a, w, s);
        const PtSpan& sp = g.sp;
        const int rows = g.rows;
        if (s.cut && threadIdx.x == 0 && s.pos0 + s.n > s.len) atomicMin(a.status, SALICACHE_E_CAPACITY);

        // q as B fragments: column g8 of column tile n is row 8 n + g8
        uint32_t qf[NT][KS][2];
        bool on = true;                      // no wait of this warp has been given up in this item
        if (g.tiles > 0) {
            const uint32_t qb = n_q & 1;
            on = warp_wait(smem_u32(&q_full[qb]), (n_q / 2) & 1, a.wait_limit, gave_up);
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                const uint32_t src = q_ring + qb * SM::Q + (8 * n + g8) * (D * 2);
                const bool in = on && 8 * n + g8 < rows;
#pragma unroll
                for (int st = 0; st < KS; ++st) {
                    int d[4];
                    q_dims<FMT>(st, c4, D, d);
                    uint32_t x0 = 0, x1 = 0;
                    if (in) {                // (b, b + 1) and (b + 2, b + 3), or (b, b + 4) and (b + 1, b + 5)
                        lds_words<1>(&x0, src + 2 * d[0]);
                        lds_words<1>(&x1, src + 2 * (FMT == PF_I4 ? d[1] : d[2]));
                    }
                    qf[n][st][0] = FMT == PF_I4 ? __byte_perm(x0, x1, 0x5410) : x0;
                    qf[n][st][1] = FMT == PF_I4 ? __byte_perm(x0, x1, 0x7632) : x1;
                }
            }
            __syncwarp();
            if (lane == 0 && on) bar_arrive(smem_u32(&q_empty[qb]));
            ++n_q;
        }
        float acc[NT][VS][4], m[NT][2], l[NT][2];
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            m[n][0] = m[n][1] = PT_NONE;
            l[n][0] = l[n][1] = 0.0f;
#pragma unroll
            for (int t = 0; t < VS; ++t) acc[n][t][0] = acc[n][t][1] = acc[n][t][2] = acc[n][t][3] = 0.0f;
        }

        for (int k = g.t0; on && k < g.t0 + g.tiles; ++k) {
            const uint32_t st = stage, src = smem_u32(ring) + st * SM::STAGE;
            on = warp_wait(smem_u32(&full[st]), phase, a.wait_limit, gave_up);
            if (!on) break;
            if (++stage == STAGES) {
                stage = 0;
                phase ^= 1;
            }
            const int j0 = sp.tile(k) * PT_KEYS + wid * 16;
            if (!(*(volatile uint32_t*)&kinds[st] >> wid & 1u)) {
                __syncwarp();                // every lane has read it: the feeder may write the next one
                if (lane == 0) bar_arrive(smem_u32(&empty[st]));
                continue;
            }
            float sc[NT][4];
#pragma unroll
            for (int n = 0; n < NT; ++n) sc[n][0] = sc[n][1] = sc[n][2] = sc[n][3] = 0.0f;
            {
                KTile<FMT, D> kt;
                kt.load(src + k_at, src + km_at);
#pragma unroll
                for (int i = 0; i < KS; ++i) {
                    uint32_t a0, a1, a2, a3;
                    key_frag<T, FMT, D>(cd, kt.k[0], kt.s[0], i, a0, a2);
                    key_frag<T, FMT, D>(cd, kt.k[1], kt.s[1], i, a1, a3);
#pragma unroll
                    for (int n = 0; n < NT; ++n) mma16816<T>(sc[n], a0, a1, a2, a3, qf[n][i][0], qf[n][i][1]);
                }
            }
            VTile<FMT, D> vt;
            vt.load(src + v_at, src + vm_at);
            __syncwarp();
            if (lane == 0) bar_arrive(smem_u32(&empty[st]));
            {
                // sc[n][i]: key key_of(g8) + 8 (i >> 1), row 8 n + 2 c4 + (i & 1)
                const bool whole = j0 + 16 <= sp.all_hi && (j0 >= sp.all_lo || j0 + 16 <= a.sinks);
                if (!whole) {
#pragma unroll
                    for (int n = 0; n < NT; ++n)
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const int j = j0 + key_of(g8) + 8 * (i >> 1), rr = w.rt * RT + 8 * n + 2 * c4 + (i & 1);
                            if (j >= s.len || !pt_sees(s.pos0 + rr / a.G, j, a.window, a.sinks)) sc[n][i] = -INFINITY;
                        }
                    // values that no row sees may be anything: keep them out of the product
#pragma unroll
                    for (int x = 0; x < 4; ++x) {
                        const int j = j0 + c4 + 4 * (x & 1) + 8 * (x >> 1);
                        if (j >= sp.hi || (j < sp.lo && j >= a.sinks)) {
#pragma unroll
                            for (int i = 0; i < VTile<FMT, D>::W; ++i) vt.v[x][i] = 0u;
                            if (FMT == PF_I8) vt.s[x >> 1][0] &= (x & 1) ? 0x0000ffffu : 0xffff0000u;
                            if (FMT == PF_I4) vt.s[x >> 1][(x & 1) && FMT == PF_I4 ? 1 : 0] = 0u;
                        }
                    }
                }
                uint32_t pf[NT][2];
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                    float p[4];                              // in powers of two, less the reference
#pragma unroll
                    for (int i = 0; i < 4; ++i) p[i] = fmaf(sc[n][i], a.scale, -m[n][i & 1]);
                    if (__any_sync(0xffffffffu, fmaxf(fmaxf(p[0], p[1]), fmaxf(p[2], p[3])) > 8.0f)) {
#pragma unroll
                        for (int i = 0; i < 2; ++i) {
                            float y = fmaxf(sc[n][i], sc[n][2 + i]) * a.scale;
#pragma unroll
                            for (int o = 4; o < 32; o <<= 1) y = fmaxf(y, __shfl_xor_sync(0xffffffffu, y, o));
                            y = fmaxf(y, m[n][i]);
                            const float f = ex2(m[n][i] - y);
                            m[n][i] = y;
                            l[n][i] *= f;
#pragma unroll
                            for (int t = 0; t < VS; ++t) {
                                acc[n][t][i] *= f;
                                acc[n][t][2 + i] *= f;
                            }
                            p[i] = fmaf(sc[n][i], a.scale, -y);
                            p[2 + i] = fmaf(sc[n][2 + i], a.scale, -y);
                        }
                    }
#pragma unroll
                    for (int i = 0; i < 4; ++i) p[i] = ex2(p[i]);
                    l[n][0] += p[0] + p[2];
                    l[n][1] += p[1] + p[3];
                    pf[n][0] = transpose8(T::pack(p[0], p[1]));
                    pf[n][1] = transpose8(T::pack(p[2], p[3]));
                }
#pragma unroll
                for (int t = 0; t < VS; ++t) {
                    const uint32_t a0 = value_frag<T, FMT, D>(cd, vt, t, 0, 0), a1 = value_frag<T, FMT, D>(cd, vt, t, 1, 0);
                    const uint32_t a2 = value_frag<T, FMT, D>(cd, vt, t, 0, 1), a3 = value_frag<T, FMT, D>(cd, vt, t, 1, 1);
#pragma unroll
                    for (int n = 0; n < NT; ++n) mma16816<T>(acc[n][t], a0, a1, a2, a3, pf[n][0], pf[n][1]);
                }
            }
        }

        // join the warps: acc[n][t][i] is dimension value_dim(t, i >> 1), row 8 n + 2 c4 + (i & 1)
        const bool first = g.t0 == 0, done = first && g.last;
        const size_t slot = 2 * (size_t)c + (first ? 1 : 0);
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int o = 4; o < 32; o <<= 1) l[n][i] += __shfl_xor_sync(0xffffffffu, l[n][i], o);
        for (int r0 = 0; r0 < rows && ok && g.real; r0 += ST_ROUND) {          // rows r0 .. r0 + 3: columns of lanes c4 = (r0 & 7) / 2 and + 1
            const bool holds = (c4 >> 1) == ((r0 >> 2) & 1);
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                if (n != r0 >> 3 || !holds) continue;
                const int lr = 2 * (c4 & 1);
                if (g8 == 0) {
                    sh_stat[wid][lr] = make_float2(m[n][0], l[n][0]);
                    sh_stat[wid][lr + 1] = make_float2(m[n][1], l[n][1]);
                }
#pragma unroll
                for (int t = 0; t < VS; ++t)
#pragma unroll
                    for (int i = 0; i < 4; ++i) sh_acc[wid][lr + (i & 1)][value_dim<FMT, D>(t, i >> 1, g8)] = acc[n][t][i];
            }
            ok = !any_of(!on);
            const int r = r0 + (wid >> 1), d0 = (wid & 1) * (D / 2) + lane * (D / 64);        // two warps per row
            if (r < rows && ok) {
                float M = PT_NONE, L = 0.0f, o[D / 64];
                const int lr = wid >> 1;
#pragma unroll
                for (int x = 0; x < ST_WARPS; ++x) M = fmaxf(M, sh_stat[x][lr].x);
#pragma unroll
                for (int i = 0; i < D / 64; ++i) o[i] = 0.0f;
#pragma unroll
                for (int x = 0; x < ST_WARPS; ++x) {
                    const float2 st = sh_stat[x][lr];
                    const float f = ex2(st.x - M);
                    L += f * st.y;
#pragma unroll
                    for (int i = 0; i < D / 64; ++i) o[i] += f * sh_acc[x][lr][d0 + i];
                }
                if (done) {
                    const int rr = w.rt * RT + r, hq = w.h * a.G + rr % a.G;
                    const long long tok = s.row0 + rr / a.G;
                    const float inv = L > 0.0f ? 1.0f / L : 0.0f;
                    uint16_t* dst = a.out + tok * a.out_stride + (long long)hq * D + d0;
                    if (D == 128) *reinterpret_cast<uint32_t*>(dst) = T::pack(o[0] * inv, o[D / 64 - 1] * inv);
                    else *dst = T::round(o[0] * inv);
                    if (a.lse && lane == 0 && (wid & 1) == 0) a.lse[tok * ((long long)a.pc.heads * a.G) + hq] = L > 0.0f ? (M + log2f(L)) * PT_LN2 : -INFINITY;
                } else {
                    float* dst = a.part + (slot * RT + r) * D + d0;
#pragma unroll
                    for (int i = 0; i < D / 64; ++i) dst[i] = o[i];
                    if (lane == 0 && (wid & 1) == 0) a.stat[slot * RT + r] = make_float2(M, L);
                }
            }
            any_of(false);
        }
        if (!done && g.real && ok) {
            if (first) {
                pt_tail(hd, w, s);
            } else hd[0].x = g.last ? 2 : 1;
        }
        w.left -= g.k1 - g.k0;
        if (w.left > 0) pt_next(w, s, a);
    }
    join_roles();
    if (threadIdx.x == 0) {
        a.head[2 * c] = hd[0];
        a.head[2 * c + 1] = hd[1];
        if (*gave_up) atomicMin(a.status, SC_GAVE_UP);
    }
}

template <typename T, int FMT, int D, int NT>
int launch_step(salicache_ctx* c, PtArgs a, char* work, cudaStream_t st) {
    using SM = StSmem<FMT, D, NT>;
    constexpr int RT = 8 * NT;
    SC_CHECK(cudaFuncSetAttribute(k_paged_step<T, FMT, D, NT>, cudaFuncAttributeMaxDynamicSharedMemorySize, SM::BYTES));
    // no more blocks than there can be tiles of work: rows of q times heads times the table's tiles
    const long long most = (long long)a.sq.n_rows * a.pc.heads * ((((long long)a.sq.width << a.pc.page_shift) + PT_KEYS - 1) / PT_KEYS);
    const int blocks = (int)max(1ll, min(min(most, (long long)PT_MAX_BLOCKS), (long long)c->sm_count * SM::BLOCKS));
    a.tile_rows = RT;
    a.part = reinterpret_cast<float*>(work);
    a.stat = reinterpret_cast<float2*>(a.part + (size_t)2 * blocks * RT * D);
    a.head = reinterpret_cast<int4*>(a.stat + (size_t)2 * blocks * RT);
    SC_CHECK(pt_launch(k_paged_step<T, FMT, D, NT>, dim3(blocks), ST_THREADS, SM::BYTES, st, a, blocks));
    SC_CHECK(pt_launch(k_paged_join<T, RT, D>, dim3(blocks, NT), 256, 0, st, a, blocks));
    c->launches += 2;
    SC_CHECK(cudaGetLastError());
    return SALICACHE_OK;
}

template <typename T, int FMT, int D>
int launch_attend(salicache_ctx* c, const PtArgs& a, char* work, cudaStream_t st) {
    // one column tile of 8 rows, or two of them: codes are expanded once for both, at half the blocks per SM
    if constexpr (FMT != PF_16)
        if ((long long)a.sq.n_rows * a.G > 8ll * a.sq.n_seqs) return launch_step<T, FMT, D, 2>(c, a, work, st);
    return launch_step<T, FMT, D, 1>(c, a, work, st);
}

}  // namespace

int64_t sc_paged_work_bytes(const salicache_ctx* c, int head_dim) { return 2ll * c->sm_count * (256 * (head_dim + 2) * 4 + 32); }

int sc_paged_attend(salicache_ctx* c, const salicache_pages* pg, const salicache_seqs* q, const void* d_q, int64_t q_stride,
                    int q_per_kv, float softmax_scale, int window, int sinks, void* d_out, int64_t out_stride, float* d_lse,
                    void* d_work, cudaStream_t st) {
    PtArgs a{};
    a.pc = pg_cache(pg);
    a.sq = pg_seqs(q);
    a.q = (const uint16_t*)d_q;
    a.out = (uint16_t*)d_out;
    a.lse = d_lse;
    a.q_stride = q_stride;
    a.out_stride = out_stride;
    a.G = q_per_kv;
    a.window = min(window, 1 << 30);
    a.sinks = window ? sinks : 0;
    a.scale = softmax_scale * PT_LOG2E;
    a.status = c->d_status;
    a.wait_limit = c->paged_wait;
    char* work = (char*)d_work;
    // Rows (of q, times the query heads of a group) per sequence up to which reading the pages is the work: 8 of 16-bit
    // pages, 16 of codes.  Measured with 16 sequences of 8000 positions, 8 key/value heads, this kernel against
    // paged_chunk.cu's: 16-bit 8 rows 101 / 115 us, 16 rows 176 / 116; INT8 16 rows 94 / 124, 32 rows 164 / 125; INT4 16 rows
    // 89 / 125, 32 rows 158 / 126.  The mean over all sequences decides, as the host knows no other number, and a batch whose
    // sequences differ much pays for it: 64 single tokens over 4000 positions beside 900 rows over 16000 (INT8, one query
    // head a group) take 620 us here, 326 there; 63 single tokens and 193 rows (four) 542 / 320.  A caller that knows its
    // batch is better off with a call for each kind.
    const long long few = pg->format == SALICACHE_FP16 ? 8 : 16;
    if ((long long)a.sq.n_rows * a.G > few * a.sq.n_seqs) return sc_paged_chunk(c, a, pg, work, st);
#define GO(T, F, D) return launch_attend<T, F, D>(c, a, work, st)
#define GO_FORMAT(T, D)                                      \
    do {                                                     \
        if (pg->format == SALICACHE_FP16) GO(T, PF_16, D);   \
        if (pg->format == SALICACHE_INT8) GO(T, PF_I8, D);   \
        GO(T, PF_I4, D);                                     \
    } while (0)
    if (pg->dtype == SALICACHE_F16) {
        if (pg->head_dim == 128) GO_FORMAT(TypeF16, 128);
        GO_FORMAT(TypeF16, 64);
    }
    if (pg->head_dim == 128) GO_FORMAT(TypeBF16, 128);
    GO_FORMAT(TypeBF16, 64);
#undef GO_FORMAT
#undef GO
}
