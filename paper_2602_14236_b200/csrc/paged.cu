// Paged K/V cache: rows quantised as they are written, and read back (quantisers of Sec. IV-B).
//
// Bound by memory: a row is read once and its codes written once.  A CTA takes a tile of consecutive rows of the caller's
// arrays and a share of the (K|V, head) pairs; for a pair, groups of head_dim / 8 lanes take one row each (16 bytes a
// lane), so that the group's extremes need only a few shuffles, and the rows of a tile fill neighbouring slots of a page
// (their codes and their 2- or 4-byte scales meet in whole sectors).  Several pairs are loaded before the first is
// quantised.
#include "paged.cuh"

namespace {

constexpr int PM_THREADS = 256;
constexpr int PM_AHEAD = 4;          // (K|V, head) pairs in flight per lane

__device__ __forceinline__ uint4 ld16(const uint8_t* p) {
    uint4 v;
    asm volatile("ld.global.nc.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
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
                        const int pg = pos >> pc.page_shift;
                        if (pg < sq.width) pid = sq.table[(size_t)b * sq.width + pg];
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

// The largest value of both halves over the LPG lanes of a group.
template <typename T, int LPG>
__device__ __forceinline__ uint32_t group_max2(uint32_t w) {
#pragma unroll
    for (int o = LPG / 2; o; o >>= 1) w = as_word(__hmax2(as_pair<T>(w), as_pair<T>(__shfl_xor_sync(0xffffffffu, w, o))));
    return w;
}

// Nearest integer (ties to even) of the product, as bits: |product| < 2^22.
__device__ __forceinline__ uint32_t rint_bits(float d, float inv) {
    return __float_as_uint(__fadd_rn(__fmul_rn(d, inv), 12582912.0f));
}

// The reciprocal of a stored scale; a scale whose reciprocal is not finite, zero among them, becomes 1.
template <typename T>
__device__ __forceinline__ float scale_inv(uint16_t& s16) {
    float inv = __fdiv_rn(1.0f, T::lo(s16));
    if (!(inv < INFINITY)) {
        s16 = (uint16_t)T::ONE;
        inv = 1.0f;
    }
    return inv;
}

// One lane's 8 elements of a group -> codes and scale in the pages.
template <typename T, int FMT, int D>
__device__ __forceinline__ void store_group(const uint4& v, const PgCache& pc, size_t slot, int gl, bool put) {
    constexpr int LPG = D / 8;
    uint8_t* dst = pc.data + slot * pg_row_bytes<FMT, D>();
    if (FMT == PF_16) {
        if (put) reinterpret_cast<uint4*>(dst)[gl] = v;
        return;
    }
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
    if (FMT == PF_I8) {
        uint32_t m = as_word(__hmax2(__hmax2(__habs2(as_pair<T>(w[0])), __habs2(as_pair<T>(w[1]))),
                                     __hmax2(__habs2(as_pair<T>(w[2])), __habs2(as_pair<T>(w[3])))));
        m = group_max2<T, LPG>(m);
        uint16_t s16 = T::round(__fdiv_rn(fmaxf(T::lo(m), T::hi(m)), 127.0f));
        const float inv = scale_inv<T>(s16);
        uint32_t q[8];
#pragma unroll
        for (int i = 0; i < 4; ++i) {       // a scale rounded down may put the extreme half a step past 127: clamp
            q[2 * i] = rint_bits(T::lo(w[i]), inv);
            q[2 * i + 1] = rint_bits(T::hi(w[i]), inv);
        }
        uint32_t o[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            uint32_t b = 0;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int c = min(127, max(-127, (int)q[4 * i + j] - 0x4B400000));
                b |= (uint32_t)(c & 0xff) << (8 * j);
            }
            o[i] = b;
        }
        if (put) {
            reinterpret_cast<uint2*>(dst)[gl] = make_uint2(o[0], o[1]);
            if (gl == 0) reinterpret_cast<uint16_t*>(pc.scale)[slot] = s16;
        }
    } else {
        const uint32_t hi2 = as_word(__hmax2(__hmax2(as_pair<T>(w[0]), as_pair<T>(w[1])), __hmax2(as_pair<T>(w[2]), as_pair<T>(w[3]))));
        const uint32_t lo2 = as_word(__hmin2(__hmin2(as_pair<T>(w[0]), as_pair<T>(w[1])), __hmin2(as_pair<T>(w[2]), as_pair<T>(w[3]))));
        const uint32_t a = as_word(__hmax2(as_pair<T>(hi2), as_pair<T>(__byte_perm(hi2, 0, 0x1032))));       // max in both halves
        const uint32_t n = as_word(__hneg2(__hmin2(as_pair<T>(lo2), as_pair<T>(__byte_perm(lo2, 0, 0x1032)))));
        const uint32_t e = group_max2<T, LPG>((a & 0xffffu) | (n << 16));                                    // (max, -min)
        const float z = -T::hi(e);
        uint16_t s16 = T::round(__fdiv_rn(__fsub_rn(T::lo(e), z), 15.0f));
        const float inv = scale_inv<T>(s16);
        uint32_t o = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int q0 = min(15, (int)rint_bits(__fsub_rn(T::lo(w[i]), z), inv) - 0x4B400000);
            const int q1 = min(15, (int)rint_bits(__fsub_rn(T::hi(w[i]), z), inv) - 0x4B400000);
            o |= (uint32_t)(q0 | q1 << 4) << (8 * i);
        }
        if (put) {
            reinterpret_cast<uint32_t*>(dst)[gl] = o;
            if (gl == 0) reinterpret_cast<uint32_t*>(pc.scale)[slot] = (uint32_t)s16 | (uint32_t)T::round(z) << 16;
        }
    }
}

// What a lane fetches of a stored group: its 8 elements' codes and the group's scale.
template <int FMT>
struct Fetched {
    uint4 c;
    uint32_t meta;
};
template <int FMT, int D>
__device__ __forceinline__ void fetch_group(Fetched<FMT>& f, const PgCache& pc, size_t slot, int gl, bool get) {
    const uint8_t* src = pc.data + slot * pg_row_bytes<FMT, D>();
    f.c = make_uint4(0, 0, 0, 0);
    f.meta = 0;
    if (!get) return;
    if (FMT == PF_16) f.c = __ldcs(reinterpret_cast<const uint4*>(src) + gl);
    else if (FMT == PF_I8) {
        const uint2 x = __ldcs(reinterpret_cast<const uint2*>(src) + gl);
        f.c.x = x.x;
        f.c.y = x.y;
        f.meta = reinterpret_cast<const uint16_t*>(pc.scale)[slot];
    } else {
        f.c.x = __ldcs(reinterpret_cast<const uint32_t*>(src) + gl);
        f.meta = reinterpret_cast<const uint32_t*>(pc.scale)[slot];
    }
}
template <typename T, int FMT>
__device__ __forceinline__ uint4 expand_group(const Fetched<FMT>& f) {
    if (FMT == PF_16) return f.c;
    uint32_t o[4];
    const float s = T::lo(f.meta), z = T::hi(f.meta);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        float a, b;
        if (FMT == PF_I8) {
            const uint32_t w = i < 2 ? f.c.x : f.c.y;
            a = __fmul_rn((float)(int8_t)(w >> (16 * (i & 1))), s);
            b = __fmul_rn((float)(int8_t)(w >> (16 * (i & 1) + 8)), s);
        } else {
            a = __fadd_rn(__fmul_rn((float)((f.c.x >> (8 * i)) & 15u), s), z);
            b = __fadd_rn(__fmul_rn((float)((f.c.x >> (8 * i + 4)) & 15u), s), z);
        }
        o[i] = T::pack(a, b);
    }
    return make_uint4(o[0], o[1], o[2], o[3]);
}

// grid.x: tiles of rows; grid.y: shares of `per` consecutive (K|V, head) pairs (pair = kv * heads + head).
template <typename T, int FMT, int D, bool WRITE>
__global__ void __launch_bounds__(PM_THREADS)
k_paged_move(PgCache pc, PgSeqs sq, uint16_t* __restrict__ K, uint16_t* __restrict__ V, long long ks, long long vs, int per,
             int* __restrict__ status) {
    constexpr int LPG = D / 8, ROWS = PM_THREADS / LPG;
    __shared__ RowMap<ROWS> map;
    map_rows<ROWS>(map, sq, pc, blockIdx.x * ROWS, status);
    __syncthreads();
    const int row = threadIdx.x / LPG, gl = threadIdx.x % LPG;
    const int pid = map.pid[row], slot = map.slot[row];
    const long long r = (long long)blockIdx.x * ROWS + row;
    const int p1 = min(2 * pc.heads, (int)(blockIdx.y + 1) * per);
    const bool live = slot >= 0;                       // the row has a place in the pages
    for (int p0 = blockIdx.y * per; p0 < p1; p0 += PM_AHEAD) {
        if (WRITE) {
            uint4 v[PM_AHEAD];
#pragma unroll
            for (int u = 0; u < PM_AHEAD; ++u) {
                const int p = p0 + u, kv = p >= pc.heads, h = p - (kv ? pc.heads : 0);
                v[u] = make_uint4(0, 0, 0, 0);
                if (live && p < p1) v[u] = ld16(reinterpret_cast<const uint8_t*>((kv ? V + r * vs : K + r * ks) + h * D + gl * 8));
            }
#pragma unroll
            for (int u = 0; u < PM_AHEAD; ++u) {
                const int p = p0 + u, kv = p >= pc.heads, h = p - (kv ? pc.heads : 0);
                store_group<T, FMT, D>(v[u], pc, pg_slot(pc, max(pid, 0), kv, h, max(slot, 0)), gl, live && p < p1);
            }
        } else {
            Fetched<FMT> f[PM_AHEAD];
#pragma unroll
            for (int u = 0; u < PM_AHEAD; ++u) {
                const int p = p0 + u, kv = p >= pc.heads, h = p - (kv ? pc.heads : 0);
                fetch_group<FMT, D>(f[u], pc, pg_slot(pc, max(pid, 0), kv, h, max(slot, 0)), gl, live && p < p1);
            }
#pragma unroll
            for (int u = 0; u < PM_AHEAD; ++u) {
                const int p = p0 + u, kv = p >= pc.heads, h = p - (kv ? pc.heads : 0);
                if (slot >= -1 && p < p1)               // rows in no page come back as zeros, rows of no sequence stay
                    __stcs(reinterpret_cast<uint4*>((kv ? V + r * vs : K + r * ks) + h * D + gl * 8), expand_group<T, FMT>(f[u]));
            }
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
    const dim3 grid((unsigned)tiles, (unsigned)((pairs + per - 1) / per));
    if (write) k_paged_move<T, FMT, D, true><<<grid, PM_THREADS, 0, st>>>(pc, sq, (uint16_t*)K, (uint16_t*)V, ks, vs, per, c->d_status);
    else k_paged_move<T, FMT, D, false><<<grid, PM_THREADS, 0, st>>>(pc, sq, (uint16_t*)K, (uint16_t*)V, ks, vs, per, c->d_status);
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
