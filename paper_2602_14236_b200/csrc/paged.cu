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
// INT8 pages and back: 4.7 us in a graph, two launches.
#include "paged_async.cuh"
#include "paged_rows.cuh"

namespace {

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
