// Paged K/V cache: rows quantised as they are written, and read back (quantisers of Sec. IV-B).
//
// Bound by memory: a row is read once and its codes written once.  A CTA takes a tile of consecutive rows of the caller's
// arrays and a share of the (K|V, head) pairs; for a pair, groups of head_dim / 8 lanes take one row each (16 bytes a
// lane), and the rows of a tile fill neighbouring slots of a page (their codes and their 2- or 4-byte scales meet in whole
// sectors).  Four pairs are under way at a time, the first four before the rows' places are known: looking those up takes
// three dependent loads.
// Issue slots come next: at the copy bandwidth an SM has 28 clocks for 512 bytes of rows.  So the four pairs' extremes go
// through one transposing butterfly (5 exchanges instead of 16), after which a quarter of the lanes each divides for one of
// the four, integers are found in the mantissa bits of 1.5 * 2^23 + x instead of by the conversion unit, and a row's place
// is one pointer and a step per pair.
// Measured: 11520 rows of 32 x 128 into INT4 pages and back, 478 MB: 85 us = 5.6 TB/s, 0.87 of the copy bandwidth (116 us
// before the above); 49279 INT4 rows of 8 x 128 read back, 255 MB: 45 us = 5.7 TB/s; a token each of eight streams into
// INT8 pages and back: 6.2 us in a graph, two launches.
#include "paged_async.cuh"
#include "paged.cuh"

namespace {

constexpr int PM_THREADS = 256;
constexpr int PM_AHEAD = 4;          // (K|V, head) pairs in flight per lane

__device__ __forceinline__ uint4 ld16(const uint8_t* p) {
    uint4 v;
    asm volatile("ld.global.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
    return v;
}

// Where the tile's rows live: page id (or -1) and slot, one entry per row.
template <int ROWS>
struct RowMap {
    int pid[ROWS];
    int slot[ROWS];       // -2: the row belongs to no sequence
};

// Sequence of row r = number of sequences that end at or before it (d_row_start is non-decreasing).
template <int ROWS>
__device__ __forceinline__ void map_rows(RowMap<ROWS>& m, const PgSeqs& sq, const PgCache& pc, int r0, int* status) {
    constexpr int WARPS = PM_THREADS / 32;
    const int lane = threadIdx.x & 31, wid = threadIdx.x >> 5;
    for (int i = wid; i < ROWS; i += WARPS) {
        const int r = r0 + i;
        int b = 0;
        for (int base = 0; base < sq.n_seqs; base += 32) {
            const int k = base + lane;
            const bool before = k < sq.n_seqs && sq.start[k + 1] <= r;
            b += __popc(__ballot_sync(0xffffffffu, before));
        }
        if (lane == 0) {
            int pid = -1, slot = -2;
            if (r < sq.n_rows && b < sq.n_seqs) {
                const PgSeq s = pg_seq(sq, pc, b);
                const int pos = s.pos0 + (r - s.row0);
                if (r >= s.row0 && r < s.row0 + s.n) {
                    slot = -1;
                    if (pos >= 0) {
                        if (pos < s.len) pid = sq.table[(size_t)b * sq.width + (pos >> pc.page_shift)];
                        if (pid >= 0 && pid < pc.n_pages) slot = pos & ((1 << pc.page_shift) - 1);
                        else {
                            pid = -1;
                            atomicMin(status, SALICACHE_E_CAPACITY);
                        }
                    }
                }
            }
            m.pid[i] = pid;
            m.slot[i] = slot;
        }
    }
}

// Nearest integer (ties to even) of the product, as bits on top of those of 1.5 * 2^23: |product| < 2^22.
__device__ __forceinline__ uint32_t rint_bits(float d, float inv) {
    return __float_as_uint(__fadd_rn(__fmul_rn(d, inv), 12582912.0f));
}
// A NaN among the two is the result.
template <typename T>
__device__ __forceinline__ uint32_t max2(uint32_t a, uint32_t b) { return as_word(__hmax2_nan(as_pair<T>(a), as_pair<T>(b))); }
template <typename T>
__device__ __forceinline__ uint32_t min2(uint32_t a, uint32_t b) { return as_word(__hmin2_nan(as_pair<T>(a), as_pair<T>(b))); }

// Four words per lane, each the two halves' maximum to be taken over a group of LPG lanes: quarter u of the group's lanes
// (lane / (LPG / 4)) gets word u's.
template <typename T, int LPG>
__device__ __forceinline__ uint32_t quarter_max(const uint32_t (&w)[4], int gl) {
    const bool up = gl & (LPG / 2), up2 = gl & (LPG / 4);
    const uint32_t x0 = max2<T>(up ? w[2] : w[0], __shfl_xor_sync(0xffffffffu, up ? w[0] : w[2], LPG / 2));
    const uint32_t x1 = max2<T>(up ? w[3] : w[1], __shfl_xor_sync(0xffffffffu, up ? w[1] : w[3], LPG / 2));
    uint32_t y = max2<T>(up2 ? x1 : x0, __shfl_xor_sync(0xffffffffu, up2 ? x0 : x1, LPG / 4));
#pragma unroll
    for (int o = LPG / 8; o; o >>= 1) y = max2<T>(y, __shfl_xor_sync(0xffffffffu, y, o));
    return y;
}

// Where a row's codes (this lane's share) and scales lie for pair 0; a pair is one page's worth of slots further on.
struct RowPlace {
    uint8_t* data;
    uint8_t* scale;
    uint32_t data_step, scale_step;
};
template <int FMT, int D>
__device__ __forceinline__ RowPlace row_place(const PgCache& pc, int pid, int slot, int gl) {
    constexpr int RB = pg_row_bytes<FMT, D>(), MB = pg_meta_bytes<FMT>(), LPG = D / 8;
    const size_t at = pg_slot(pc, max(pid, 0), 0, 0, max(slot, 0));
    return RowPlace{pc.data + at * RB + gl * (RB / LPG), pc.scale + at * MB, (uint32_t)RB << pc.page_shift, (uint32_t)MB << pc.page_shift};
}

// A lane's 8 elements of four groups (pairs p0 .. p0 + 3 of a row, those below p1) -> codes and scales in the pages.
template <typename T, int FMT, int D>
__device__ __forceinline__ void store_groups(const uint4 (&v)[PM_AHEAD], const RowPlace& rp, int p0, int p1, int gl, bool live) {
    constexpr int LPG = D / 8, Q = LPG / 4;
    if (FMT == PF_16) {
#pragma unroll
        for (int u = 0; u < PM_AHEAD; ++u)
            if (live && p0 + u < p1) *reinterpret_cast<uint4*>(rp.data + (p0 + u) * rp.data_step) = v[u];
        return;
    }
    uint32_t e[PM_AHEAD];
#pragma unroll
    for (int u = 0; u < PM_AHEAD; ++u) {
        const uint32_t w[4] = {v[u].x, v[u].y, v[u].z, v[u].w};
        if (FMT == PF_I8) {
            const uint32_t m = max2<T>(max2<T>(as_word(__habs2(as_pair<T>(w[0]))), as_word(__habs2(as_pair<T>(w[1])))),
                                       max2<T>(as_word(__habs2(as_pair<T>(w[2]))), as_word(__habs2(as_pair<T>(w[3])))));
            e[u] = m;
        } else {                             // (maximum, -minimum)
            const uint32_t hi = max2<T>(max2<T>(w[0], w[1]), max2<T>(w[2], w[3]));
            const uint32_t lo = as_word(__hneg2(as_pair<T>(min2<T>(min2<T>(w[0], w[1]), min2<T>(w[2], w[3])))));
            e[u] = max2<T>(__byte_perm(hi, lo, 0x5410), __byte_perm(hi, lo, 0x7632));
        }
    }
    uint32_t x = quarter_max<T, LPG>(e, gl);
    if (FMT == PF_I8) x = max2<T>(x, __byte_perm(x, 0u, 0x1032));
    const int mine = gl / Q;                 // the group whose scale this lane forms
    const float zero = FMT == PF_I4 ? -T::hi(x) : 0.0f;
    const float span = FMT == PF_I4 ? __fsub_rn(T::lo(x), zero) : T::lo(x);
    uint16_t s16 = T::round(__fdiv_rn(span, FMT == PF_I4 ? 15.0f : 127.0f));
    float inv = __frcp_rn(T::lo(s16));
    if (!(inv < INFINITY)) {                 // zero, and what has no reciprocal in binary32
        s16 = (uint16_t)T::ONE;
        inv = 1.0f;
    }
    if (!(span < INFINITY)) s16 = (uint16_t)T::NOT_A_NUMBER;         // whatever the codes: every value of the group is read as NaN
    if (live && gl % Q == 0 && p0 + mine < p1) {
        uint8_t* at = rp.scale + (p0 + mine) * rp.scale_step;
        if (FMT == PF_I8) *reinterpret_cast<uint16_t*>(at) = s16;
        else *reinterpret_cast<uint32_t*>(at) = (uint32_t)s16 | (uint32_t)T::round(zero) << 16;
    }
    // A normal scale is within half a step of the quotient, so no code can leave its range; a subnormal one has fewer bits.
    const bool clamp = __any_sync(0xffffffffu, (s16 & 0x7fffu) < T::NORMAL);
    const int first = (threadIdx.x & 31) - gl;
#pragma unroll
    for (int u = 0; u < PM_AHEAD; ++u) {
        const float iu = __shfl_sync(0xffffffffu, inv, first + u * Q);
        const float zu = FMT == PF_I4 ? __shfl_sync(0xffffffffu, zero, first + u * Q) : 0.0f;
        const uint32_t w[4] = {v[u].x, v[u].y, v[u].z, v[u].w};
        uint32_t q[8];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            q[2 * i] = rint_bits(FMT == PF_I4 ? __fsub_rn(T::lo(w[i]), zu) : T::lo(w[i]), iu);
            q[2 * i + 1] = rint_bits(FMT == PF_I4 ? __fsub_rn(T::hi(w[i]), zu) : T::hi(w[i]), iu);
        }
        if (clamp) {
            constexpr int TOP = FMT == PF_I4 ? 15 : 127, LOW = FMT == PF_I4 ? 0 : -127;
#pragma unroll
            for (int i = 0; i < 8; ++i) q[i] = (uint32_t)max(LOW, min(TOP, (int)q[i] - 0x4B400000));
        }
        const bool put = live && p0 + u < p1;
        uint8_t* dst = rp.data + (p0 + u) * rp.data_step;
        if (FMT == PF_I8) {
            const uint32_t a = __byte_perm(__byte_perm(q[0], q[1], 0x0040), __byte_perm(q[2], q[3], 0x0040), 0x5410);
            const uint32_t b = __byte_perm(__byte_perm(q[4], q[5], 0x0040), __byte_perm(q[6], q[7], 0x0040), 0x5410);
            if (put) *reinterpret_cast<uint2*>(dst) = make_uint2(a, b);
        } else {
            const uint32_t b0 = q[0] + (q[1] << 4), b1 = q[2] + (q[3] << 4), b2 = q[4] + (q[5] << 4), b3 = q[6] + (q[7] << 4);
            const uint32_t o = __byte_perm(__byte_perm(b0, b1, 0x0040), __byte_perm(b2, b3, 0x0040), 0x5410);
            if (put) *reinterpret_cast<uint32_t*>(dst) = o;
        }
    }
}

// What a lane fetches of a stored group: its 8 elements' codes and the group's scale.
template <int FMT>
struct Fetched {
    uint4 c;
    uint32_t meta;
};
template <int FMT>
__device__ __forceinline__ void fetch_group(Fetched<FMT>& f, const RowPlace& rp, int p, bool get) {
    const uint8_t* src = rp.data + p * rp.data_step;
    const uint8_t* meta = rp.scale + p * rp.scale_step;
    f.c = make_uint4(0, 0, 0, 0);
    f.meta = 0;
    if (!get) return;
    if (FMT == PF_16) f.c = __ldcs(reinterpret_cast<const uint4*>(src));
    else if (FMT == PF_I8) {
        const uint2 x = __ldcs(reinterpret_cast<const uint2*>(src));
        f.c.x = x.x;
        f.c.y = x.y;
        f.meta = *reinterpret_cast<const uint16_t*>(meta);
    } else {
        f.c.x = __ldcs(reinterpret_cast<const uint32_t*>(src));
        f.meta = *reinterpret_cast<const uint32_t*>(meta);
    }
}
// Codes to numbers by putting them into the mantissa of 2^23, which is then taken off: exact, and before the scale, whose
// product with 2^23 need not be finite.  A nibble i places up stands for 16^i times its value, which the scale, divided by
// the same power of two, makes good exactly (its last place, 2^-133 or more, leaves room for 12 bits); q * s fits binary32,
// so that the fused step that adds the zero rounds as a multiplication and an addition do.
template <typename T, int FMT>
__device__ __forceinline__ uint4 expand_group(const Fetched<FMT>& f) {
    if (FMT == PF_16) return f.c;
    uint32_t o[4];
    const float s = T::lo(f.meta), z = T::hi(f.meta);
    if (FMT == PF_I8) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t w = (i < 2 ? f.c.x : f.c.y) ^ 0x80808080u;
            const float a = __uint_as_float(__byte_perm(w, 0x4B000000u, (i & 1) ? 0x7442 : 0x7440)) - 8388736.0f;
            const float b = __uint_as_float(__byte_perm(w, 0x4B000000u, (i & 1) ? 0x7443 : 0x7441)) - 8388736.0f;
            o[i] = T::pack(__fmul_rn(a, s), __fmul_rn(b, s));
        }
    } else {
        float x[8];
        const uint32_t w1 = f.c.x >> 16, big = held<0x4B000000u>();
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float si = s * (1.0f / (float)(1 << (4 * (i & 3))));
            const uint32_t w = i < 4 ? f.c.x : w1;
            const uint32_t b = (i & 3) == 0 ? and_or<0xfu>(w, big) : (i & 3) == 1 ? and_or<0xf0u>(w, big) : (i & 3) == 2 ? and_or<0xf00u>(w, big) : and_or<0xf000u>(w, big);
            x[i] = __fmaf_rn(__fsub_rn(__uint_as_float(b), 8388608.0f), si, z);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) o[i] = T::pack(x[2 * i], x[2 * i + 1]);
    }
    return make_uint4(o[0], o[1], o[2], o[3]);
}

// grid.x: tiles of rows; grid.y: shares of `per` consecutive (K|V, head) pairs (pair = kv * heads + head).
template <typename T, int FMT, int D, bool WRITE>
__global__ void __launch_bounds__(PM_THREADS)
k_paged_move(PgCache pc, PgSeqs sq, uint16_t* K, uint16_t* V, long long ks, long long vs, int per,
             int* status) {
    constexpr int LPG = D / 8, ROWS = PM_THREADS / LPG;
    __shared__ RowMap<ROWS> map;
    const int row = threadIdx.x / LPG, gl = threadIdx.x % LPG;
    const long long r = (long long)blockIdx.x * ROWS + row;
    const int p1 = min(2 * pc.heads, (int)(blockIdx.y + 1) * per);
    grid_wait();
    grid_release();
    // this lane's share of pair p: K's or V's row, the latter from pair `heads` on
    uint16_t* const k0 = K + r * ks + gl * 8;
    uint16_t* const v0 = V + r * vs + gl * 8 - (long long)pc.heads * D;
    auto dense = [&](int p) -> uint4* { return reinterpret_cast<uint4*>((p >= pc.heads ? v0 : k0) + p * D); };
    int p0 = blockIdx.y * per;
    if (WRITE) {
        auto load = [&](uint4 (&v)[PM_AHEAD], int q0) {
#pragma unroll
            for (int u = 0; u < PM_AHEAD; ++u) {
                v[u] = make_uint4(0, 0, 0, 0);
                if (r < sq.n_rows && q0 + u < p1) v[u] = ld16(reinterpret_cast<const uint8_t*>(dense(q0 + u)));
            }
        };
        uint4 v[PM_AHEAD], next[PM_AHEAD];
        load(v, p0);
        map_rows<ROWS>(map, sq, pc, blockIdx.x * ROWS, status);
        __syncthreads();
        const bool live = map.slot[row] >= 0;
        const RowPlace rp = row_place<FMT, D>(pc, map.pid[row], map.slot[row], gl);
        for (; p0 < p1; p0 += PM_AHEAD) {
            load(next, p0 + PM_AHEAD);
            store_groups<T, FMT, D>(v, rp, p0, p1, gl, live);
#pragma unroll
            for (int u = 0; u < PM_AHEAD; ++u) v[u] = next[u];
        }
    } else {
        map_rows<ROWS>(map, sq, pc, blockIdx.x * ROWS, status);
        __syncthreads();
        const int slot = map.slot[row];
        const RowPlace rp = row_place<FMT, D>(pc, map.pid[row], slot, gl);
        Fetched<FMT> f[PM_AHEAD], next[PM_AHEAD];
#pragma unroll
        for (int u = 0; u < PM_AHEAD; ++u) fetch_group(f[u], rp, p0 + u, slot >= 0 && p0 + u < p1);
        for (; p0 < p1; p0 += PM_AHEAD) {
#pragma unroll
            for (int u = 0; u < PM_AHEAD; ++u) fetch_group(next[u], rp, p0 + PM_AHEAD + u, slot >= 0 && p0 + PM_AHEAD + u < p1);
#pragma unroll
            for (int u = 0; u < PM_AHEAD; ++u)
                if (slot >= -1 && p0 + u < p1)          // rows in no page come back as zeros, rows of no sequence stay
                    __stcs(dense(p0 + u), expand_group<T, FMT>(f[u]));
#pragma unroll
            for (int u = 0; u < PM_AHEAD; ++u) f[u] = next[u];
        }
    }
}

template <typename T, int FMT, int D>
int launch_move(salicache_ctx* c, const PgCache& pc, const PgSeqs& sq, void* K, void* V, int64_t ks, int64_t vs, bool write,
                cudaStream_t st) {
    constexpr int ROWS = PM_THREADS / (D / 8);
    const long long tiles = ((long long)sq.n_rows + ROWS - 1) / ROWS;
    const int pairs = 2 * pc.heads;
    int per = pairs;
    while (per > PM_AHEAD && tiles * ((pairs + per - 1) / per) < 8ll * c->sm_count) per = (per + 1) / 2;
    per = (per + PM_AHEAD - 1) / PM_AHEAD * PM_AHEAD;
    const dim3 grid((unsigned)tiles, (unsigned)((pairs + per - 1) / per));
    if (write) SC_CHECK(pt_launch(k_paged_move<T, FMT, D, true>, grid, PM_THREADS, 0, st, pc, sq, (uint16_t*)K, (uint16_t*)V, (long long)ks, (long long)vs, per, c->d_status));
    else SC_CHECK(pt_launch(k_paged_move<T, FMT, D, false>, grid, PM_THREADS, 0, st, pc, sq, (uint16_t*)K, (uint16_t*)V, (long long)ks, (long long)vs, per, c->d_status));
    c->launches++;
    SC_CHECK(cudaGetLastError());
    return SALICACHE_OK;
}

template <typename T, int D>
int move_format(salicache_ctx* c, int format, const PgCache& pc, const PgSeqs& sq, void* K, void* V, int64_t ks, int64_t vs,
                bool write, cudaStream_t st) {
    if (format == SALICACHE_FP16) return launch_move<T, PF_16, D>(c, pc, sq, K, V, ks, vs, write, st);
    if (format == SALICACHE_INT8) return launch_move<T, PF_I8, D>(c, pc, sq, K, V, ks, vs, write, st);
    return launch_move<T, PF_I4, D>(c, pc, sq, K, V, ks, vs, write, st);
}

}  // namespace

int sc_paged_move(salicache_ctx* c, const salicache_pages* pg, const salicache_seqs* q, void* d_K, void* d_V, int64_t k_stride,
                  int64_t v_stride, bool write, cudaStream_t st) {
    const PgCache pc = pg_cache(pg);
    const PgSeqs sq = pg_seqs(q);
    if (pg->dtype == SALICACHE_F16) {
        if (pg->head_dim == 128) return move_format<TypeF16, 128>(c, pg->format, pc, sq, d_K, d_V, k_stride, v_stride, write, st);
        return move_format<TypeF16, 64>(c, pg->format, pc, sq, d_K, d_V, k_stride, v_stride, write, st);
    }
    if (pg->head_dim == 128) return move_format<TypeBF16, 128>(c, pg->format, pc, sq, d_K, d_V, k_stride, v_stride, write, st);
    return move_format<TypeBF16, 64>(c, pg->format, pc, sq, d_K, d_V, k_stride, v_stride, write, st);
}
