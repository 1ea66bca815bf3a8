// Rows of the caller's arrays on their way into pages: where they live, and the quantisers.  Shared by the store (paged.cu)
// and by the store that turns rows by their positions (paged_rotary.cu).
#pragma once
#include "paged.cuh"

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

// Sequence of row r = number of sequences that end at or before it (d_row_start is non-decreasing).  A warp has ROWS / WARPS
// rows, whose look-ups go side by side: three dependent loads for all of them (one row after the other: 10.6 us instead of
// 7.5 for writing prompts of 5864 rows).
template <int ROWS>
__device__ __forceinline__ void map_rows(RowMap<ROWS>& m, const PgSeqs& sq, const PgCache& pc, int r0, int* status) {
    constexpr int WARPS = PM_THREADS / 32, EACH = ROWS / WARPS;
    static_assert(EACH >= 1 && EACH * WARPS == ROWS, "rows of a warp");
    const int lane = threadIdx.x & 31, i0 = (threadIdx.x >> 5) * EACH;
    int b = 0;                               // of this lane's row, i0 + lane
    for (int base = 0; base < sq.n_seqs; base += 32) {
        const int k = base + lane, end = k < sq.n_seqs ? sq.start[k + 1] : 0;
#pragma unroll
        for (int e = 0; e < EACH; ++e) {
            const int n = __popc(__ballot_sync(0xffffffffu, k < sq.n_seqs && end <= r0 + i0 + e));
            if (lane == e) b += n;
        }
    }
    if (lane < EACH) {
        const int i = i0 + lane, r = r0 + i;
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
