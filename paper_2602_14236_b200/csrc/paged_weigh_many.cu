// What attention gave each cached position, many rows per sequence: the scores' product is the work, and runs on the
// fifth-generation tensor cores; then every score costs one exponential.
//
// One block per SM walks its stretch of the line of (256 keys x 128 rows) tiles.  An item is 256 keys of one head, and its
// tiles those of rows (new tokens times query heads of a group) that see some of the keys.  The scores stand transposed in
// tensor memory, S^T = K Q^T: a lane is a key, a column a row of q, so that a thread sums its own key's weights over all rows in
// a register and nothing is exchanged.  Two tiles' scores (2 x 2 x 128 columns) fill tensor memory: one is summed while the
// other is multiplied.
// Roles by warp group:
//   0 .. 3 two threads per key, one for odd tiles and one for even ones: e^(s - lse) over the columns, and at the item's end the
//          weight.  The two groups of a half never wait for one another within an item, so that one has exponentials to do while
//          the other waits for its scores
//   4      codes from the pages to 16-bit operands, an item's keys at a time
//   5      one thread issues the matrix instructions; one warp feeds K of 16-bit pages and the rows of q by tensor copies, another
//          one the rows' sums
// K is double-buffered, and read once per item; the rows of q come once per tile, from the L2.
//
// Measured: a prompt of 8192 rows, 32 query and 8 key/value heads x 128: 298 us, 333 us once the clocks have settled under load,
// = 825 to 925 TFLOP/s of the products.  A tile takes 2200 clocks: 2048 its 32768 exponentials would take on the special-function unit
// alone (69 % of it used, an eighth of them being elsewhere), 1024 the products (39 % of the tensor pipe).  Tried: 8 warps for the
// weights, which wait for the tensor memory at the same time (361 us with three stages of rows, 513 with two), two keys a thread
// (424), both halves of the warps on every tile (368).  A sequence's few rows over a long cache (64 to 256 of them over 8000
// positions) cost an item's fixed time per 256 keys: 2.7 us over 16-bit pages, 4.5 over codes, of which each role's walk and waits are more
// than half.
//
// An item that the ends of blocks' stretches cut leaves partial sums, which a second kernel adds in the
// order of the blocks.
#include <math.h>
#include <type_traits>

#include "paged_tc.cuh"
#include "paged_weigh.cuh"

namespace {

constexpr int WM_KEYS = 256, WM_K = 2, WM_Q = 3;
// The pairs of columns of which the first takes its exponentials on the FMA pipe instead of the special-function unit: one column in
// eight.  A prompt of 8192 rows with none, one, two of eight, before the last columns' masks: 314, 290, 298 us; one call after the other,
// until the clocks have settled: 339, 330, 343.
__device__ __forceinline__ constexpr bool WM_POLY(int pair) { return (pair & 3) == 0; }
// An item's fixed cost (its keys) in tiles' time.
constexpr int WM_ITEM = 2;

// A block's place in the line.
struct WmWalk {
    long long left;                          // units still to do
    int b, h, kt, k;                         // sequence, head, tile of keys, unit within the item
    PgSeq s;
    int held, rows;                          // its positions with a weight, and tiles of rows
};
// Tiles of the sequence's rows, and the first one that sees some key from j0 on.  A tile has `tok` whole tokens, by which a
// product with 2^38 / tok rounded up divides: x is at most a call's tokens, below 2^30 / G, and tok = 128 / G rounded down, so
// that the product fits and is less than x / 2^38, which is less than 1 / tok, too large.
__device__ __forceinline__ int wm_by_tok(int x, const WgArgs& a) { return (int)((uint64_t)x * a.per_tok >> 38); }
__device__ __forceinline__ int wm_rows(const PgSeq& s, const WgArgs& a) { return wm_by_tok(s.n + a.tok - 1, a); }
__device__ __forceinline__ int wm_first(const PgSeq& s, const WgArgs& a, int j0) { return wm_by_tok(max(0, j0 - s.pos0), a); }
// Its positions with a weight; none, if the sequence is the other kernel's.
__device__ __forceinline__ int wm_held(const PgSeq& s, const WgArgs& a) { return s.n * a.G > WG_FEW ? wg_held(s, a) : 0; }
__device__ __forceinline__ int wm_items(const PgSeq& s, const WgArgs& a) { return (wm_held(s, a) + WM_KEYS - 1) / WM_KEYS; }
// Units of an item: its fixed cost and its tiles, of which there are some, since the last row sees every position.
__device__ __forceinline__ int wm_units(const PgSeq& s, const WgArgs& a, int kt) {
    return WM_ITEM + wm_rows(s, a) - wm_first(s, a, kt * WM_KEYS);
}
// Items at the front that all rows see.
__device__ __forceinline__ int wm_whole(const PgSeq& s, const WgArgs& a) {
    return min(wm_items(s, a), s.pos0 >= 0 ? s.pos0 / WM_KEYS + 1 : 0);
}
// Units of one head of the sequence that each lane of a warp has; the warp sums the items of long ones together.
__device__ __forceinline__ long long wm_per_head(const WgArgs& a, const PgSeq& s) {
    constexpr int ALONE = 2;
    const int lane = threadIdx.x & 31, n = wm_items(s, a), whole = wm_whole(s, a);
    long long w = whole > 0 ? (long long)whole * wm_units(s, a, 0) : 0;
    if (n - whole <= ALONE)
#pragma unroll 1
        for (int kt = whole; kt < n; ++kt) w += wm_units(s, a, kt);
    for (uint32_t many = __ballot_sync(0xffffffffu, n - whole > ALONE); many; many &= many - 1) {
        const int from = __ffs(many) - 1;
        const PgSeq o = pt_seq_of(s, from);
        long long x = 0;
#pragma unroll 1
        for (int kt = __shfl_sync(0xffffffffu, whole, from) + lane; kt < __shfl_sync(0xffffffffu, n, from) + lane; kt += 32)
            if (kt < wm_items(o, a)) x += wm_units(o, a, kt);
#pragma unroll
        for (int d = 16; d; d >>= 1) x += __shfl_xor_sync(0xffffffffu, x, d);
        if (lane == from) w += x;
    }
    return w;
}
__device__ __forceinline__ void wm_enter(WmWalk& w, const WgArgs& a) {
    w.held = wm_held(w.s, a);
    w.rows = wm_rows(w.s, a);
}
// Where the block starts; the same for every thread, each warp for itself.
__device__ __noinline__ WmWalk wm_start(const WgArgs& a, int block, int blocks) {
    const int lane = threadIdx.x & 31;
    auto seq = [&](int b) -> PgSeq {
        PgSeq s{};
        if (b < a.sq.n_seqs) s = pg_seq(a.sq, a.pc, b);
        return s;
    };
    const PgSeq s0 = seq(lane);
    const long long mine = wm_per_head(a, s0) * a.pc.heads;
    long long total = 0;
    for (int b0 = 0; b0 < a.sq.n_seqs; b0 += 32)
        total += __shfl_sync(0xffffffffu, pt_scan(b0 == 0 ? mine : wm_per_head(a, seq(b0 + lane)) * a.pc.heads), 31);
    WmWalk w{};
    long long beg, end, before = 0;
    pt_share(total, block, blocks, beg, end);
    if (beg == end) return w;
    for (int b0 = 0; b0 < a.sq.n_seqs; b0 += 32) {
        const PgSeq s = b0 == 0 ? s0 : seq(b0 + lane);
        const long long n = b0 == 0 ? mine : wm_per_head(a, s) * a.pc.heads, incl = before + pt_scan(n);
        const uint32_t hit = __ballot_sync(0xffffffffu, beg >= incl - n && beg < incl);
        before = __shfl_sync(0xffffffffu, incl, 31);
        if (!hit) continue;
        const int from = __ffs(hit) - 1;
        w.s = pt_seq_of(s, from);
        wm_enter(w, a);
        w.b = b0 + from;
        w.left = end - beg;
        const long long at = __shfl_sync(0xffffffffu, beg - (incl - n), from), per = __shfl_sync(0xffffffffu, n, from) / a.pc.heads;
        w.h = (int)(at / per);
        long long rem = at - w.h * per;
        const int items = wm_items(w.s, a), whole = wm_whole(w.s, a), each = wm_units(w.s, a, 0);
        if (rem < (long long)whole * each) {
            w.kt = (int)(rem / each);
            w.k = (int)(rem - (long long)w.kt * each);
            return w;
        }
        rem -= (long long)whole * each;
#pragma unroll 1
        for (int k0 = whole;; k0 += 32) {
            const int u = k0 + lane < items ? wm_units(w.s, a, k0 + lane) : 0;
            const long long upto = pt_scan(u);
            const uint32_t in = __ballot_sync(0xffffffffu, rem >= upto - u && rem < upto);
            if (in || k0 + 32 >= items) {
                const int f = in ? __ffs(in) - 1 : 0;
                w.kt = k0 + f;
                w.k = __shfl_sync(0xffffffffu, (int)(rem - (upto - u)), f);
                return w;
            }
            rem -= __shfl_sync(0xffffffffu, upto, 31);
        }
    }
    w.left = 0;
    return w;
}
// On to another head.
__device__ __noinline__ WmWalk wm_after(const WgArgs& a, WmWalk w) {
    w.kt = 0;
    if (++w.h < a.pc.heads) return w;
    w.h = 0;
#pragma unroll 1
    do {
        if (++w.b >= a.sq.n_seqs) return w;  // cannot happen while units are left
        w.s = pg_seq(a.sq, a.pc, w.b);
    } while (wm_items(w.s, a) == 0);
    wm_enter(w, a);
    return w;
}
// On to the next item.  The keys after these of the same head need no more than their number: every role walks for itself, and over
// few rows that is what an item's time goes into (four rows over INT4 pages 137 us with all of it in the function above, 117 so).
__device__ __forceinline__ void wm_next(WmWalk& w, const WgArgs& a) {
    w.k = 0;
    if ((++w.kt) * WM_KEYS >= w.held) w = wm_after(a, w);
}

// A block's share of one item.
struct WmSeg {
    int k0, k1, tiles, rt, j0;               // units [k0, k1); tiles of rows from rt on; first key
    bool first, last;                        // the item begins, ends here
    __device__ __forceinline__ WmSeg(const WgArgs& a, const WmWalk& w) {
        j0 = w.kt * WM_KEYS;
        const int f = j0 <= w.s.pos0 ? 0 : wm_first(w.s, a, j0), units = WM_ITEM + w.rows - f;
        k0 = w.k;
        k1 = (int)min((long long)units, k0 + w.left);
        const int t0 = max(0, k0 - WM_ITEM), t1 = max(0, k1 - WM_ITEM);
        first = t0 == 0;
        last = k1 == units;
        tiles = t1 - t0;
        rt = f + t0;
    }
    // Page of keys 16 grp .. of the item: -2 there are none (or grp > 15), -1 there is no such page.
    __device__ __forceinline__ int page_of(const WgArgs& a, const WmWalk& w, int grp) const {
        const int j = j0 + grp * 16;
        if (grp > 15 || j >= w.held) return -2;
        const int p = a.sq.table[(size_t)w.b * a.sq.width + (j >> a.pc.page_shift)];
        return p >= 0 && p < a.pc.n_pages ? p : -1;
    }
};

// 2^x without the special-function unit, to 2.2e-7: x = n + f, n the nearest integer, which 1.5 * 2^23 + x holds in its low bits;
// a polynomial of degree 5 for 2^f on [-1/2, 1/2] (least largest relative error, by the Remez exchange); n goes into the
// exponent.  Below -126 the result is some number below 2^-126; from 128 on, and of what is no number, it is anything, which `top`,
// the largest argument so far, tells.
__device__ __forceinline__ float ex2_fma(float x, float& top) {
    asm("max.NaN.f32 %0, %0, %1;" : "+f"(top) : "f"(x));
    const float y = fmaxf(x, -127.0f), t = y + 12582912.0f, f = y - (t - 12582912.0f);
    float p = fmaf(0x1.5c08e6p-10f, f, 0x1.3d0c52p-7f);
    p = fmaf(p, f, 0x1.c6b6e4p-5f);
    p = fmaf(p, f, 0x1.ebf918p-3f);
    p = fmaf(p, f, 0x1.62e428p-1f);
    p = fmaf(p, f, 0x1.000002p+0f);
    return __uint_as_float((__float_as_uint(t) << 23) + __float_as_uint(p));
}

__device__ __forceinline__ uint64_t pair2(float lo, float hi) {
    uint64_t d;
    asm("mov.b64 %0, {%1, %2};" : "=l"(d) : "f"(lo), "f"(hi));
    return d;
}
__device__ __forceinline__ void split2(uint64_t x, float& lo, float& hi) { asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(x)); }
__device__ __forceinline__ uint64_t fma2x(uint64_t a, uint64_t b, uint64_t c) {
    uint64_t d;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a), "l"(b), "l"(c));
    return d;
}
__device__ __forceinline__ uint64_t add2x(uint64_t a, uint64_t b) {
    uint64_t d;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
    return d;
}
struct WmBars {
    uint64_t k_full[WM_K], k_empty[WM_K], q_full[WM_Q], q_empty[WM_Q], l_full[2], s_full[2][2], s_free[2][2], o_full, o_empty, left;
    int4 hd[2];                              // what the block says of its records
    uint32_t tmem;
    int gave_up;
    uint32_t counts[2][4];                   // even and odd tiles: bit c set: column c is a row, and one that counts
    int all[2];                              // ... which all but those behind the last whole token are
    uint32_t pages[8];                       // per item with tiles (in turn): bit g set: the page of keys 16 g .. 16 g + 15 exists
};
template <int D>
struct WmSmem {
    static constexpr int TILE = 128 * D * 2;         // bytes of an operand tile
    static constexpr int K = 0, Q = K + WM_K * 2 * TILE, LSE = Q + WM_Q * TILE, OTHER = LSE + 2 * 128 * 4, BARS = OTHER + WM_KEYS * 4;
    static constexpr int BYTES = BARS + (int)sizeof(WmBars);
    static_assert(BYTES <= 227 * 1024, "shared memory");
};

// Warps: 16 for the weights, 4 for codes where there are any, 4 more.
template <int FMT> __host__ __device__ constexpr int wm_threads() { return FMT == PF_16 ? 640 : 768; }

template <typename T, int FMT, int D>
__global__ void __launch_bounds__(wm_threads<FMT>(), 1)
k_weigh_many(const __grid_constant__ WgArgs a, const __grid_constant__ CUtensorMap map, const __grid_constant__ CUtensorMap q_map, int blocks) {
    using SM = WmSmem<D>;
    constexpr int WM_THREADS = wm_threads<FMT>(), LAST = WM_THREADS / 32 - 4;           // first warp of the last group
    extern __shared__ __align__(1024) uint8_t mem[];         // the swizzle's atoms; there is no room to align by hand
    const uint32_t base = smem_u32(mem);
    WmBars& bars = *reinterpret_cast<WmBars*>(mem + SM::BARS);
    const int tid = threadIdx.x, wid = tid >> 5, lane = tid & 31;
    volatile int* gave_up = &bars.gave_up;
    grid_wait();
    grid_release();
    if (!*a.some) return;
    if (tid == 0) {
        for (int i = 0; i < WM_K; ++i) {
            bar_init(smem_u32(&bars.k_full[i]), FMT == PF_16 ? 1 : 4);       // the feeder, or the warps of group 4
            bar_init(smem_u32(&bars.k_empty[i]), 1);
        }
        for (int i = 0; i < WM_Q; ++i) {
            bar_init(smem_u32(&bars.q_full[i]), 1);
            bar_init(smem_u32(&bars.q_empty[i]), 1);
        }
        for (int i = 0; i < 2; ++i) {
            bar_init(smem_u32(&bars.l_full[i]), 1);
            for (int h = 0; h < 2; ++h) {
                bar_init(smem_u32(&bars.s_full[i][h]), 1);
                bar_init(smem_u32(&bars.s_free[i][h]), 4);   // a lane of each warp that reads them
            }
        }
        bar_init(smem_u32(&bars.o_full), 8);
        bar_init(smem_u32(&bars.o_empty), 8);
        bar_init(smem_u32(&bars.left), 1);
        bars.gave_up = 0;
        bars.hd[0] = bars.hd[1] = make_int4(0, 0, 0, 0);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (wid == LAST) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_u32(&bars.tmem)) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    // rows of a tile that no copy fills (128 is no multiple of G) are zeros
    const int HR = a.tok * a.G;
    for (int i = tid; i < WM_Q * (128 - HR) * (D / 8); i += WM_THREADS) {
        const int c = i % (D / 8), r = i / (D / 8) % (128 - HR), q = i / (D / 8) / (128 - HR);
        sts16(base + SM::Q + q * SM::TILE + swz(HR + r, c), 0u, 0u, 0u, 0u);
    }
    fence_async();
    tc_before();
    WmWalk w = wm_start(a, blockIdx.x, blocks);
    __syncthreads();
    tc_after();
    const uint32_t tmem = bars.tmem;
    auto wait = [&](uint64_t& bar, uint32_t parity) -> bool { return warp_wait_far(smem_u32(&bar), parity, a.wait_limit, gave_up); };
    auto next = [&](const WmSeg& g) {
        w.left -= g.k1 - g.k0;
        if (w.left > 0) wm_next(w, a);
    };

    if (wid < 16) {
        // ---------------- weights
        const int half = wid >> 2 & 1, part = wid >> 3, key = tid & 255;         // keys; tiles with odd numbers, or even ones
        const uint32_t S = tmem + 256 * part + 128 * half + ((uint32_t)((wid & 3) * 32) << 16);
        const ulonglong2* const ls = reinterpret_cast<const ulonglong2*>(mem + SM::LSE) + 32 * part;
        float* const other = reinterpret_cast<float*>(mem + SM::OTHER) + key;
        uint32_t n = 0, n_item = 0, n_two = 0;   // tiles, items with tiles, with two or more of them so far
        bool ok = true;
        while (w.left > 0 && ok) {
            const WmSeg g(a, w);
            if (tid == 0 && (w.s.cut || w.s.len > a.w_stride)) atomicMin(a.status, SALICACHE_E_CAPACITY);
            const int j = g.j0 + key;
            float sum = 0.0f;
            const bool mine = j < w.held;
            const bool writes = g.tiles > 0 && (int)((n + g.tiles - 1) & 1) == part;       // the group that has the last tile
            if (writes && mine && a.in)      // what the key had is looked at when the tiles are through: no register holds it until then
                asm volatile("prefetch.global.L2 [%0];" ::"l"(a.in + ((size_t)w.b * a.pc.heads + w.h) * a.w_stride + j));
            for (int t = 0; t < g.tiles; ++t, ++n) {
                if ((int)(n & 1) != part) continue;
                if (!(wait(bars.l_full[part], n >> 1 & 1) && wait(bars.s_full[part][half], n >> 1 & 1))) {
                    ok = false;
                    break;
                }
                tc_after();
                const int r0 = (g.rt + t) * HR;
                const bool whole = HR >= 112 && *(volatile int*)&bars.all[part] && (long long)(g.j0 + half * 128 + 127 - w.s.pos0) * a.G <= r0;
                const int c_lo = max(0, min(128, max(0, j - w.s.pos0) * a.G - r0));          // rows before this column do not see the key
                // A column that is no row has the sum WG_NONE, which leaves nothing of a finite score, and is masked where it may meet
                // another one: the zeros behind a tile's rows under a key that is not finite, a row that counts as none.  `whole` tiles have
                // the former, where 128 is no multiple of G, among the last 16 columns, and none of the latter.  (The last 16 columns masked
                // in every tile: a prompt of 8192 rows 308 us instead of 298.  Such tiles in a third copy of this code: 5 % more for
                // 64 rows a sequence, whose time goes into walks and waits.)
                uint64_t acc[2] = {0ull, 0ull};  // the first one's lower half has the polynomial's columns alone
                float top = -INFINITY;
                const uint64_t scale2 = pair2(a.scale, a.scale);
                auto columns = [&](auto whole_) {
                    constexpr bool WHOLE = decltype(whole_)::value;
                    uint32_t x[2][16];
                    tc_ld16(x[0], S);
                    tc_wait_ld16(x[0]);
#pragma unroll
                    for (int c = 0; c < 8; ++c) {
                        if (c < 7) tc_ld16(x[(c + 1) & 1], S + 16 * (c + 1));
                        const uint32_t(&y)[16] = x[c & 1];
                        ulonglong2 l[4];
#pragma unroll
                        for (int i = 0; i < 4; ++i) l[i] = ls[4 * c + i];
                        auto sixteen = [&](auto masked_) {
                            constexpr bool MASKED = decltype(masked_)::value;
                            uint32_t sees = MASKED ? *(volatile uint32_t*)&bars.counts[part][c >> 1] >> (16 * (c & 1)) : 0u;
                            if (!WHOLE) sees &= ~below(c_lo - 16 * c);
                            if (c == 7) {        // the scores and their rows' sums are in registers
                                tc_before();
                                __syncwarp();
                                if (lane == 0) bar_arrive(smem_u32(&bars.s_free[part][half]));
                            }
#pragma unroll
                            for (int i = 0; i < 8; ++i) {
                                float lo, hi;
                                const uint64_t minus = i & 1 ? l[i >> 1].y : l[i >> 1].x;
                                split2(fma2x(pair2(__uint_as_float(y[2 * i]), __uint_as_float(y[2 * i + 1])), scale2, minus), lo, hi);
                                lo = !MASKED && WM_POLY(i) ? ex2_fma(lo, top) : ex2(lo);
                                hi = ex2(hi);
                                if (MASKED) {
                                    lo = sees & 1u << (2 * i) ? lo : 0.0f;
                                    hi = sees & 2u << (2 * i) ? hi : 0.0f;
                                }
                                acc[!WM_POLY(i)] = add2x(acc[!WM_POLY(i)], pair2(lo, hi));
                            }
                        };
                        if (WHOLE && (c < 7 || HR == 128)) sixteen(std::false_type{});
                        else sixteen(std::true_type{});
                        if (c < 7) tc_wait_ld16(x[(c + 1) & 1]);
                    }
                };
                if (whole) columns(std::true_type{});
                else columns(std::false_type{});
                float s[4];
                split2(acc[0], s[0], s[1]);
                split2(acc[1], s[2], s[3]);
                sum += (top < 128.0f ? s[0] : top == top ? INFINITY : top) + ((s[1] + s[2]) + s[3]);
            }
            if (!ok) break;
            const float had = writes && mine && g.first && g.last ? wg_had(a, w.s, w.b, w.h, j) : 0.0f;
            if (g.tiles > 0) {
                // the even and the odd tiles come together where the last one was; the other group has been done before it
                if (g.tiles > 1) {
                    if (!writes) {
                        if (n_two > 0 && !wait(bars.o_empty, (n_two - 1) & 1)) break;
                        *other = sum;
                        __syncwarp();
                        if (lane == 0) bar_arrive(smem_u32(&bars.o_full));
                    } else {
                        if (!wait(bars.o_full, n_two & 1)) break;
                        sum += *other;
                        __syncwarp();
                        if (lane == 0) bar_arrive(smem_u32(&bars.o_empty));
                    }
                    ++n_two;
                }
                // what lies in no page is not a weight, nor is what is left of exponentials of minus infinity
                if (writes && (!(*(volatile uint32_t*)&bars.pages[n_item & 7] >> (key >> 4) & 1u) || sum < 1e-33f)) sum = 0.0f;
                ++n_item;
            }
            if (writes) {
                if (g.first && g.last) {
                    if (mine) wg_put(a, w.b, w.h, j, had, sum);
                } else {
                    a.part[(2 * (size_t)blockIdx.x + (g.first ? 1 : 0)) * WM_KEYS + key] = sum;
                    if (key == 0) {
                        if (g.first) {
                            bars.hd[0].y = 1;
                            bars.hd[0].z = w.b;
                            bars.hd[0].w = w.h;
                            bars.hd[1].x = w.kt;
                        } else bars.hd[0].x = g.last ? 2 : 1;
                    }
                }
            }
            next(g);
        }
    } else if (wid < LAST) {
        // ---------------- codes to operands: 64 keys a warp
        if (FMT != PF_16) {
            constexpr int RB = pg_row_bytes<FMT, D>(), MB = pg_meta_bytes<FMT>(), LPR = RB / 16, RPP = 32 / LPR, P = 16 / RPP;
            static_assert(P >= 1, "16 keys at a time");
            constexpr int BATCH = FMT == PF_I4 ? 4 : 2;          // groups of 16 keys under way at a time, as the registers allow
            const Codes<T> cd;
            const int lw = wid - 16, c = lane % LPR;
            uint32_t n_item = 0;
            int pid16 = w.left > 0 ? WmSeg(a, w).page_of(a, w, lane) : -2;
            while (w.left > 0) {
                const WmSeg g(a, w);
                // the next item's pages are looked up meanwhile
                WmWalk wn = w;
                wn.left -= g.k1 - g.k0;
                if (wn.left > 0) wm_next(wn, a);
                const int pid16n = wn.left > 0 ? WmSeg(a, wn).page_of(a, wn, lane) : -2;
                if (g.tiles > 0) {
                    const uint32_t kb = n_item % WM_K;
                    uint4 words[BATCH][P];
                    uint32_t meta[BATCH][P];
                    int pid[BATCH];
                    auto load = [&](int grp0) {
#pragma unroll
                        for (int e = 0; e < BATCH; ++e) {
                            pid[e] = __shfl_sync(0xffffffffu, pid16, lw * 4 + grp0 + e);
                            const size_t slot = pg_slot(a.pc, max(pid[e], 0), 0, w.h, (g.j0 + lw * 64 + (grp0 + e) * 16) & ((1 << a.pc.page_shift) - 1));
                            if (pid[e] >= 0)
#pragma unroll
                                for (int p = 0; p < P; ++p) {
                                    const int r = p * RPP + lane / LPR;
                                    words[e][p] = __ldcs(reinterpret_cast<const uint4*>(a.pc.data + (slot + r) * RB) + c);
                                    const uint8_t* m = a.pc.scale + (slot + r) * MB;
                                    meta[e][p] = FMT == PF_I8 ? *reinterpret_cast<const uint16_t*>(m) : *reinterpret_cast<const uint32_t*>(m);
                                }
                        }
                    };
                    load(0);                 // before there is a place for them
                    if (n_item >= WM_K && !wait(bars.k_empty[kb], (n_item / WM_K - 1) & 1)) break;
                    if (lw == 0) {
                        const uint32_t there = __ballot_sync(0xffffffffu, pid16 >= 0), bad = __ballot_sync(0xffffffffu, pid16 == -1);
                        if (lane == 0) {
                            *(volatile uint32_t*)&bars.pages[n_item & 7] = there;
                            if (bad) atomicMin(a.status, SALICACHE_E_CAPACITY);
                        }
                    }
                    const uint32_t dst = base + SM::K + kb * 2 * SM::TILE + (lw >> 1) * SM::TILE;
#pragma unroll
                    for (int grp = 0; grp < 4; ++grp) {
                        const int e = grp % BATCH;
                        if (pid[e] >= 0)                         // what lies in no page is not looked at
#pragma unroll
                            for (int p = 0; p < P; ++p) {
                                const int row = (lw & 1) * 64 + grp * 16 + p * RPP + lane / LPR;
                                const uint32_t s2 = dup_lo(meta[e][p]), z2 = dup_hi(meta[e][p]), w4[4] = {words[e][p].x, words[e][p].y, words[e][p].z, words[e][p].w};
                                if (FMT == PF_I8) {
#pragma unroll
                                    for (int i = 0; i < 2; ++i)
                                        sts16(dst + swz(row, 2 * c + i), mul2<T>(cd.bytes(w4[2 * i], 0x5140), s2), mul2<T>(cd.bytes(w4[2 * i], 0x5342), s2),
                                              mul2<T>(cd.bytes(w4[2 * i + 1], 0x5140), s2), mul2<T>(cd.bytes(w4[2 * i + 1], 0x5342), s2));
                                } else {
#pragma unroll
                                    for (int i = 0; i < 4; ++i) {                // elements 0 4, 1 5, 2 6, 3 7 in their words: put in order
                                        const uint32_t y = w4[i] >> 8, e04 = fma2<T>(cd.nib_lo(w4[i]), s2, z2), e15 = fma2<T>(cd.nib_hi(w4[i]), s2, z2);
                                        const uint32_t e26 = fma2<T>(cd.nib_lo(y), s2, z2), e37 = fma2<T>(cd.nib_hi(y), s2, z2);
                                        sts16(dst + swz(row, 4 * c + i), __byte_perm(e04, e15, 0x5410), __byte_perm(e26, e37, 0x5410),
                                              __byte_perm(e04, e15, 0x7632), __byte_perm(e26, e37, 0x7632));
                                    }
                                }
                            }
                        if (e == BATCH - 1 && grp < 3) load(grp + 1);
                    }
                    fence_async();
                    __syncwarp();
                    if (lane == 0) bar_arrive(smem_u32(&bars.k_full[kb]));
                    ++n_item;
                }
                w = wn;
                pid16 = pid16n;
            }
        }
    } else {
        if (wid == LAST) {
            // ---------------- matrix instructions: the warp stays together, one lane issues
            constexpr uint32_t ID = instr_desc<T>(128, false);
            const uint32_t k_lo = desc_lo(base + SM::K, 16), q_lo = desc_lo(base + SM::Q, 16);
            uint32_t n = 0, n_item = 0;
            bool ok = true;
            while (w.left > 0 && ok) {
                const WmSeg g(a, w);
                const uint32_t kb = n_item % WM_K;
                const int halves = w.held - g.j0 > 128 ? 2 : 1;
                if (g.tiles > 0) ok = wait(bars.k_full[kb], n_item / WM_K & 1);
                for (int t = 0; t < g.tiles && ok; ++t, ++n) {
                    const uint32_t buf = n & 1, st = n % WM_Q;
                    ok = wait(bars.q_full[st], n / WM_Q & 1);
                    for (int h = 0; h < 2; ++h) {
                        if (ok && n >= 2) ok = wait(bars.s_free[buf][h], (n / 2 - 1) & 1);
                        if (!ok) break;
                        tc_after();
                        if (elect_one()) {
                            const uint32_t ka = k_lo + (kb * 2 + h) * (SM::TILE >> 4), qb = q_lo + st * (SM::TILE >> 4);
                            if (h < halves)
#pragma unroll
                                for (int i = 0; i < D / 16; ++i) {
                                    const uint32_t off = (i >> 2) * 1024 + (i & 3) * 2;
                                    mma_ss(tmem + 256 * buf + 128 * h, desc(ka + off), desc(qb + off), ID, i > 0);
                                }
                            tc_commit(smem_u32(&bars.s_full[buf][h]));
                            if (h == 1) {
                                tc_commit(smem_u32(&bars.q_empty[st]));
                                if (t == g.tiles - 1) tc_commit(smem_u32(&bars.k_empty[kb]));
                            }
                        }
                        __syncwarp();
                    }
                    if (!ok) break;
                }
                n_item += g.tiles > 0;
                next(g);
            }
            // what the instructions' ends arrive at is there until they have
            for (uint32_t i = n > WM_Q ? n - WM_Q : 0; i < n && ok; ++i) ok = wait(bars.q_empty[i % WM_Q], i / WM_Q & 1);
            for (uint32_t i = n_item > WM_K ? n_item - WM_K : 0; i < n_item && ok; ++i) ok = wait(bars.k_empty[i % WM_K], i / WM_K & 1);
            if (!ok) {
                if (elect_one()) tc_commit(smem_u32(&bars.left));
                __syncwarp();
                bar_drain(smem_u32(&bars.left), 0);
            }
        }
        if (wid == LAST + 1) {
            // ---------------- feeder
            uint32_t n = 0, n_item = 0;
            bool ok = true;
            const int per_page = 1 << a.pc.page_shift;
            if (lane == 0) asm volatile("prefetch.tensormap [%0];" ::"l"(&q_map) : "memory");
            // the keys of an item, those of 16-bit pages: group 4 brings the others
            auto feed_keys = [&](const WmWalk& x, const WmSeg& g) -> bool {
                const uint32_t kb = n_item % WM_K, bar = smem_u32(&bars.k_full[kb]);
                const int pid16 = g.page_of(a, x, lane);
                const uint32_t bad = __ballot_sync(0xffffffffu, pid16 == -1), there = __ballot_sync(0xffffffffu, pid16 >= 0);
                // the first group of 16 keys of this lane's page names the page
                const int pid = __shfl_sync(0xffffffffu, pid16, (lane << (a.pc.page_shift - 4)) & 31);
                const bool mine = lane < WM_KEYS >> a.pc.page_shift && pid >= 0;
                const uint32_t copies = (uint32_t)__popc(__ballot_sync(0xffffffffu, mine));
                if (n_item >= WM_K && !wait(bars.k_empty[kb], (n_item / WM_K - 1) & 1)) return false;
                if (lane == 0) {
                    *(volatile uint32_t*)&bars.pages[n_item & 7] = there;
                    if (bad) atomicMin(a.status, SALICACHE_E_CAPACITY);
                    bar_expect(bar, copies * (uint32_t)(per_page * D * 2));
                }
                __syncwarp();
                if (mine) {
                    const size_t slot = pg_slot(a.pc, pid, 0, x.h, 0);
                    const int key = lane << a.pc.page_shift;
                    const uint32_t dst = base + SM::K + (kb * 2 + (key >> 7)) * SM::TILE + (key & 127) * 128;
#pragma unroll
                    for (int y = 0; y < D; y += 64) tensor_copy(dst + y * 256, &map, y, (int)slot, bar);
                }
                __syncwarp();
                ++n_item;
                return true;
            };
            if (FMT == PF_16 && w.left > 0) {
                const WmSeg g(a, w);
                if (g.tiles > 0) ok = feed_keys(w, g);
            }
            while (w.left > 0 && ok) {
                const WmSeg g(a, w);
                WmWalk wn = w;
                wn.left -= g.k1 - g.k0;
                if (wn.left > 0) wm_next(wn, a);
                for (int t = 0; t < g.tiles; ++t, ++n) {
                    const uint32_t st = n % WM_Q, bar = smem_u32(&bars.q_full[st]);
                    if (n >= WM_Q && !wait(bars.q_empty[st], (n / WM_Q - 1) & 1)) {
                        ok = false;
                        break;
                    }
                    if (lane == 0) {
                        bar_expect(bar, (uint32_t)(HR * D * 2));
                        for (int x = 0; x < D; x += 64)
                            tensor_copy3(base + SM::Q + st * SM::TILE + x * 256, &q_map, x, w.h * a.G, w.s.row0 + (g.rt + t) * a.tok, bar);
                    }
                    __syncwarp();
                    // the next item's keys, once the rows' ring has gone past the item before, whose keys they replace
                    if (FMT == PF_16 && t == min(WM_Q, g.tiles) - 1 && wn.left > 0) {
                        const WmSeg gn(a, wn);
                        if (gn.tiles > 0 && !feed_keys(wn, gn)) {
                            ok = false;
                            ++n;
                            break;
                        }
                    }
                }
                if (FMT == PF_16 && g.tiles == 0 && wn.left > 0 && ok) {
                    const WmSeg gn(a, wn);
                    if (gn.tiles > 0) ok = feed_keys(wn, gn);
                }
                w = wn;
            }
            join_roles();
            // copies in flight end before the block does: who uses a stage waits for them, unless a role has left early
            if (*gave_up) {
                for (uint32_t i = n > WM_Q ? n - WM_Q : 0; i < n; ++i) bar_drain(smem_u32(&bars.q_full[i % WM_Q]), i / WM_Q & 1);
                if (FMT == PF_16)
                    for (uint32_t i = n_item > WM_K ? n_item - WM_K : 0; i < n_item; ++i) bar_drain(smem_u32(&bars.k_full[i % WM_K]), i / WM_K & 1);
            }
            return;
        }
        if (wid == LAST + 2) {
            // ---------------- the rows' sums: minus their logarithms, in powers of two; -WG_NONE for what is none.  A lane has four columns
            const int Hq = a.pc.heads * a.G;
            int off[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) off[i] = (4 * lane + i) / a.G * Hq + (4 * lane + i) % a.G;
            uint32_t n = 0;
            bool ok = true;
            while (w.left > 0 && ok) {
                const WmSeg g(a, w);
                for (int t = 0; t < g.tiles; ++t, ++n) {
                    const float* p = a.lse + (long long)(w.s.row0 + (g.rt + t) * a.tok) * Hq + w.h * a.G;
                    const int cols = min(HR, w.s.n * a.G - (g.rt + t) * HR);
                    float l[4];
                    uint32_t there = 0;          // this lane's columns that count
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const float y = 4 * lane + i < cols ? __ldg(p + off[i]) : -INFINITY;
                        l[i] = y == -INFINITY ? -WG_NONE : -y * PT_LOG2E;
                        there |= (y == -INFINITY ? 0u : 1u << i) << 4 * (lane & 7);
                    }
                    const bool all = __reduce_add_sync(0xffffffffu, __popc(there)) == HR;
#pragma unroll
                    for (int d = 1; d < 8; d <<= 1) there |= __shfl_xor_sync(0xffffffffu, there, d);
                    // who frees tile n - 2 has read its sums
                    if (n >= 2 && !(wait(bars.s_free[n & 1][0], (n / 2 - 1) & 1) && wait(bars.s_free[n & 1][1], (n / 2 - 1) & 1))) {
                        ok = false;
                        break;
                    }
                    reinterpret_cast<float4*>(mem + SM::LSE)[(n & 1) * 32 + lane] = make_float4(l[0], l[1], l[2], l[3]);
                    if ((lane & 7) == 0) *(volatile uint32_t*)&bars.counts[n & 1][lane >> 3] = there;
                    if (lane == 0) *(volatile int*)&bars.all[n & 1] = all;
                    __syncwarp();
                    if (lane == 0) bar_arrive(smem_u32(&bars.l_full[n & 1]));
                }
                next(g);
            }
        }
        __syncwarp();
    }
    tc_before();
    join_roles();
    if (tid == 0) {
        a.head[2 * blockIdx.x] = bars.hd[0];
        a.head[2 * blockIdx.x + 1] = bars.hd[1];
        if (*gave_up) atomicMin(a.status, SC_GAVE_UP);
    }
    if (wid == LAST) {
        tc_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tmem) : "memory");
    }
}

// Joins split items: block c that item whose tail block c of the first kernel left; a thread per key.
__global__ void __launch_bounds__(WM_KEYS)
k_weigh_join(WgArgs a, int blocks) {
    __shared__ int list[PT_MAX_BLOCKS + 1];
    grid_wait();
    if (!*a.some) return;
    const int4 hd = a.head[2 * blockIdx.x];
    if (hd.y == 0) return;
    const int b = hd.z, h = hd.w, j = a.head[2 * blockIdx.x + 1].x * WM_KEYS + threadIdx.x;
    const int n = pt_records([&](int c) { return a.head[2 * c].x; }, blockIdx.x, blocks, list);
    const PgSeq s = pg_seq(a.sq, a.pc, b);
    float sum = 0.0f;
    for (int i = 0; i < n; ++i) sum += a.part[(size_t)list[i] * WM_KEYS + threadIdx.x];
    if (j < wm_held(s, a)) wg_put(a, b, h, j, wg_had(a, s, b, h, j), sum);
}

template <typename T, int FMT, int D>
int launch_many(salicache_ctx* c, WgArgs a, char* work, cudaStream_t st) {
    constexpr int BYTES = WmSmem<D>::BYTES;
    CUtensorMap map{}, q_map{};
    const bool bf16 = T::ONE == TypeBF16::ONE;
    if (!rows_map(&q_map, a.q, a.q_stride, a.pc.heads, a.G, a.sq.n_rows, D, bf16)) return SALICACHE_E_CUDA;
    if (FMT == PF_16 && !page_map(&map, a.pc, D, bf16)) return SALICACHE_E_CUDA;
    SC_CHECK(cudaFuncSetAttribute(k_weigh_many<T, FMT, D>, cudaFuncAttributeMaxDynamicSharedMemorySize, BYTES));
    const int blocks = min(c->sm_count, PT_MAX_BLOCKS);
    a.tok = 128 / a.G;
    a.per_tok = ((1ull << 38) + a.tok - 1) / a.tok;
    a.part = reinterpret_cast<float*>(work + 16);        // behind a.some
    a.head = reinterpret_cast<int4*>(a.part + (size_t)2 * blocks * WM_KEYS);
    SC_CHECK(pt_launch(k_weigh_many<T, FMT, D>, dim3(blocks), wm_threads<FMT>(), BYTES, st, a, map, q_map, blocks));
    SC_CHECK(pt_launch(k_weigh_join, dim3(blocks), WM_KEYS, 0, st, a, blocks));
    c->launches += 2;
    SC_CHECK(cudaGetLastError());
    return SALICACHE_OK;
}
template <typename T, int D>
int many_format(salicache_ctx* c, const WgArgs& a, int format, char* work, cudaStream_t st) {
    if (format == SALICACHE_FP16) return launch_many<T, PF_16, D>(c, a, work, st);
    if (format == SALICACHE_INT8) return launch_many<T, PF_I8, D>(c, a, work, st);
    return launch_many<T, PF_I4, D>(c, a, work, st);
}

}  // namespace

int sc_weigh_many(salicache_ctx* c, const WgArgs& a, const salicache_pages* pg, char* work, cudaStream_t st) {
    if (pg->dtype == SALICACHE_F16)
        return pg->head_dim == 128 ? many_format<TypeF16, 128>(c, a, pg->format, work, st) : many_format<TypeF16, 64>(c, a, pg->format, work, st);
    return pg->head_dim == 128 ? many_format<TypeBF16, 128>(c, a, pg->format, work, st) : many_format<TypeBF16, 64>(c, a, pg->format, work, st);
}
