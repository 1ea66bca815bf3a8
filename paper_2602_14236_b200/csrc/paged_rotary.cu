// Rows on their way into the paged cache with K turned by its positions (rotary positions on one to four axes), and the rows
// of q turned beside them:
//
//   phi = position[axis(i)] * freq(i),  first' = first cos phi - second sin phi,  second' = second cos phi + first sin phi
//
// The angle is needed modulo one turn, and its fraction is what a product in binary32 would lose first (a position of 10^6
// leaves an error of 0.06 radians).  So freq / 2 pi comes as a 64-bit fraction F of a turn, and position * F modulo 2^64 is
// exact: its upper half is the angle in units of 2^-32 turns.  No table of cosines is read.
//
// Bound by memory: every row is read once and written once.  A block takes a tile of rows and a share either of the
// (K|V, head) pairs, whose groups it quantises as the store does (paged_rows.cuh), or of the query heads; a lane has 8
// elements of a head, four heads under way.  The tile's cosines and sines are worked out once per block, into shared memory,
// then every lane keeps its 8 for all heads.  With halves an element's partner is in another lane of the group: four shuffles
// for 8 elements.
// Measured: four frames (11520 rows of 32 query and 8 key/value heads x 128) into INT4 pages, 248 MB: 47 to 49 us = 5.2 TB/s = 0.80
// of the copy bandwidth, 65 % of the issue slots used (K and V alone take 19, of which the turning 5); prompts of 5864 rows of 12
// heads x 64, 54 MB: 13 us (11 with the rows in the L2 from the pass before, as the variants below were timed), of which a third is
// look-ups and angles before the first row; a token each of 32 streams 4.2 us in a graph.
#include <math.h>

#include "paged_async.cuh"
#include "paged_rows.cuh"

namespace {

struct RtTurns {
    uint64_t f[64];          // turns per position as a fraction of 2^64, of which the last two bits name the axis
    int pairs, n_axes;
};

// A lane's share of the rotation: where its partner is, and the cosine and sine (with its sign) of each element.
template <bool HALVES>
struct Turn {
    static constexpr int N = HALVES ? 8 : 4;
    float c[N], s[N];
    int from;                // halves: the lane that has the partners
    bool on;                 // these dimensions are turned
    // `row`: (cos, sin) of the row's pairs; lane gl of a group has dimensions 8 gl .. 8 gl + 7
    __device__ __forceinline__ void set(const float2* row, int gl, int pairs) {
        const int lane = threadIdx.x & 31, lanes = pairs / 8;        // lanes of a half
        on = gl < 2 * lanes;
        from = !on ? lane : gl < lanes ? lane + lanes : lane - lanes;
        const int i0 = !on ? 0 : HALVES ? 8 * (gl < lanes ? gl : gl - lanes) : 4 * gl;
        const float sign = HALVES && gl < lanes ? -1.0f : 1.0f;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const float2 x = row[i0 + i];
            c[i] = x.x;
            s[i] = sign * x.y;
        }
    }
    template <typename T>
    __device__ __forceinline__ uint4 operator()(const uint4& v) const {
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
        uint32_t o[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float a = T::lo(w[i]), b = T::hi(w[i]);
            if constexpr (HALVES) {
                const uint32_t p = __shfl_sync(0xffffffffu, w[i], from);
                o[i] = T::pack(fmaf(a, c[2 * i], T::lo(p) * s[2 * i]), fmaf(b, c[2 * i + 1], T::hi(p) * s[2 * i + 1]));
            } else o[i] = T::pack(fmaf(a, c[i], -(b * s[i])), fmaf(b, c[i], a * s[i]));
        }
        return on ? make_uint4(o[0], o[1], o[2], o[3]) : v;
    }
};

// grid.x: tiles of rows, each with kv_shares shares of `per` (K|V, head) pairs, then shares of `per` query heads: side by side,
// since the former wait for issue slots and the latter for memory.  Three blocks per SM at head_dim 128: four frames into INT4
// pages 47 us instead of 53, four blocks 47; at 64 two: prompts of 5864 rows 10.9 us, three blocks 12.8.
template <typename T, int FMT, int D, bool HALVES>
__global__ void __launch_bounds__(PM_THREADS, D == 128 ? 3 : 2)
k_paged_write_rotary(PgCache pc, PgSeqs sq, const __grid_constant__ RtTurns rt, const int* pos, const uint16_t* q, uint16_t* q_out,
                     const uint16_t* K, const uint16_t* V, long long qs, long long qos, long long ks, long long vs, int q_heads,
                     int shares, int kv_shares, int per, int* status) {
    constexpr int LPG = D / 8, ROWS = PM_THREADS / LPG, PAIRS = D / 2;
    __shared__ RowMap<ROWS> map;
    __shared__ __align__(16) float2 turns[ROWS][PAIRS + 2];          // rows in other banks than the ones before
    const int row = threadIdx.x / LPG, gl = threadIdx.x % LPG;
    const int tile = blockIdx.x / shares, y = blockIdx.x - tile * shares;
    const long long r = (long long)tile * ROWS + row;
    const bool is_q = y >= kv_shares, there = r < sq.n_rows;
    const int share = is_q ? y - kv_shares : y, p1 = min(is_q ? q_heads : 2 * pc.heads, (share + 1) * per);
    int p0 = share * per;
    grid_wait();
    grid_release();
    const uint16_t* const a0 = (is_q ? q + r * qs : K + r * ks) + gl * 8;
    const uint16_t* const v0 = V + r * vs + gl * 8 - (long long)pc.heads * D;
    auto load = [&](uint4 (&v)[PM_AHEAD], int h0) {
#pragma unroll
        for (int u = 0; u < PM_AHEAD; ++u) {
            v[u] = make_uint4(0, 0, 0, 0);
            if (there && h0 + u < p1) v[u] = ld16(reinterpret_cast<const uint8_t*>((!is_q && h0 + u >= pc.heads ? v0 : a0) + (h0 + u) * D));
        }
    };
    uint4 v[PM_AHEAD], next[PM_AHEAD];
    load(v, p0);
    if (is_q || p0 < pc.heads) {             // a thread has one pair of several rows
        const int i = threadIdx.x % PAIRS;
        if (i < rt.pairs) {
            const uint64_t f = rt.f[i];
            const int axis = (int)(f & 3u);
#pragma unroll
            for (int k = threadIdx.x / PAIRS; k < ROWS; k += PM_THREADS / PAIRS) {
                const long long rr = (long long)tile * ROWS + k;
                const uint64_t phase = rr < sq.n_rows ? (uint64_t)(long long)pos[rr * rt.n_axes + axis] * f : 0ull;
                // in integers to an eighth of a turn on either side of the nearest quarter: as a binary32 number of half turns that
                // is off by 2^-27 at most
                const uint32_t at = (uint32_t)(phase >> 32), quarter = (at + 0x20000000u) >> 30;
                float s, c;
                sincospif((float)(int)(at - (quarter << 30)) * 0x1p-31f, &s, &c);
                const float x = quarter & 1u ? -s : c, y = quarter & 1u ? c : s;
                turns[k][i] = quarter & 2u ? make_float2(-x, -y) : make_float2(x, y);
            }
        }
    }
    map_rows<ROWS>(map, sq, pc, tile * ROWS, status);
    __syncthreads();
    Turn<HALVES> turn;
    turn.set(turns[row], gl, rt.pairs);
    if (is_q) {
        const bool mine = map.slot[row] >= -1;
        uint16_t* const dst = q_out + r * qos + gl * 8;
        for (; p0 < p1; p0 += PM_AHEAD) {
            load(next, p0 + PM_AHEAD);
#pragma unroll
            for (int u = 0; u < PM_AHEAD; ++u) {
                const uint4 y = turn.template operator()<T>(v[u]);
                if (mine && p0 + u < p1) __stcs(reinterpret_cast<uint4*>(dst + (p0 + u) * D), y);
            }
#pragma unroll
            for (int u = 0; u < PM_AHEAD; ++u) v[u] = next[u];
        }
    } else {
        const bool live = map.slot[row] >= 0;
        const RowPlace rp = row_place<FMT, D>(pc, map.pid[row], map.slot[row], gl);
        for (; p0 < p1; p0 += PM_AHEAD) {
            load(next, p0 + PM_AHEAD);
#pragma unroll
            for (int u = 0; u < PM_AHEAD; ++u)
                if (p0 + u < pc.heads) v[u] = turn.template operator()<T>(v[u]);
            store_groups<T, FMT, D>(v, rp, p0, p1, gl, live);
#pragma unroll
            for (int u = 0; u < PM_AHEAD; ++u) v[u] = next[u];
        }
    }
}

// freq / 2 pi modulo one as a fraction of 2^64, for frequencies up to 2^64: the frequency's 53 bits times 192 of 1 / 2 pi (from
// Machin's formula for pi), of which the whole turns fall off.  What is cut off is below 2^-64 turns, 2^-62 with the axis in the
// last two bits.
uint64_t turns_per_position(double freq) {
    static const uint64_t INV[3] = {0x36d8a5664f10e410ull, 0x7f09d5f47d4d3770ull, 0x28be60db9391054aull};    // least first
    int e;
    const uint64_t m = (uint64_t)ldexp(frexp(fabs(freq), &e), 53);
    uint64_t p[5] = {};                      // freq = m 2^(e - 53), freq / 2 pi = p 2^(e - 53 - 192)
    unsigned __int128 carry = 0;
    for (int i = 0; i < 3; ++i) {
        carry += (unsigned __int128)m * INV[i];
        p[i] = (uint64_t)carry;
        carry >>= 64;
    }
    p[3] = (uint64_t)carry;
    const int shift = 128 + 53 - e;          // at least 116
    if (shift >= 256) return 0;
    const int w = shift / 64, off = shift % 64;
    const uint64_t f = off ? p[w] >> off | p[w + 1] << (64 - off) : p[w];
    return freq < 0 ? 0 - f : f;
}

struct RtCall {
    PgCache pc;
    PgSeqs sq;
    RtTurns rt;
    const int* pos;
    const uint16_t *q, *K, *V;
    uint16_t* q_out;
    long long qs, qos, ks, vs;
    int q_heads;
};

template <typename T, int FMT, int D, bool HALVES>
int launch_rotary(salicache_ctx* c, const RtCall& a, cudaStream_t st) {
    constexpr int ROWS = PM_THREADS / (D / 8);
    const long long tiles = ((long long)a.sq.n_rows + ROWS - 1) / ROWS;
    const int pairs = 2 * a.pc.heads;
    auto shares = [&](int n, int per) { return (n + per - 1) / per; };
    // every block looks its rows up and works out their angles: no more blocks than fill the SMs (8 blocks per SM instead of 3:
    // prompts of 5864 rows 14.4 us instead of 10.9)
    int per = max(pairs, a.q_heads);
    while (per > PM_AHEAD && tiles * (shares(pairs, per) + shares(a.q_heads, per)) < 3ll * c->sm_count) per = (per + 1) / 2;
    per = (per + PM_AHEAD - 1) / PM_AHEAD * PM_AHEAD;
    const int kv_shares = shares(pairs, per), all = kv_shares + shares(a.q_heads, per);
    const dim3 grid((unsigned)(tiles * all));            // below 2^28: a tile has 16 rows at least, and many tiles have two shares each
    SC_CHECK(pt_launch(k_paged_write_rotary<T, FMT, D, HALVES>, grid, PM_THREADS, 0, st, a.pc, a.sq, a.rt, a.pos, a.q, a.q_out, a.K, a.V, a.qs,
                       a.qos, a.ks, a.vs, a.q_heads, all, kv_shares, per, c->d_status));
    c->launches++;
    SC_CHECK(cudaGetLastError());
    return SALICACHE_OK;
}

template <typename T, int D, bool HALVES>
int rotary_format(salicache_ctx* c, int format, const RtCall& a, cudaStream_t st) {
    if (format == SALICACHE_FP16) return launch_rotary<T, PF_16, D, HALVES>(c, a, st);
    if (format == SALICACHE_INT8) return launch_rotary<T, PF_I8, D, HALVES>(c, a, st);
    return launch_rotary<T, PF_I4, D, HALVES>(c, a, st);
}
template <typename T, bool HALVES>
int rotary_dim(salicache_ctx* c, const salicache_pages* pg, const RtCall& a, cudaStream_t st) {
    return pg->head_dim == 128 ? rotary_format<T, 128, HALVES>(c, pg->format, a, st) : rotary_format<T, 64, HALVES>(c, pg->format, a, st);
}

}  // namespace

int sc_paged_write_rotary(salicache_ctx* c, const salicache_pages* pg, const salicache_seqs* sq, const salicache_rotary* rotary,
                          const int32_t* d_pos, const void* d_q, int64_t q_stride, int q_per_kv, void* d_q_out, int64_t q_out_stride,
                          const void* d_K, const void* d_V, int64_t k_stride, int64_t v_stride, cudaStream_t st) {
    RtCall a{};
    a.pc = pg_cache(pg);
    a.sq = pg_seqs(sq);
    a.rt.pairs = rotary->pairs;
    a.rt.n_axes = rotary->n_axes;
    for (int i = 0; i < rotary->pairs; ++i) a.rt.f[i] = (turns_per_position(rotary->freq[i]) & ~3ull) | rotary->axis[i];
    a.pos = d_pos;
    a.q = (const uint16_t*)d_q;
    a.q_out = (uint16_t*)d_q_out;
    a.K = (const uint16_t*)d_K;
    a.V = (const uint16_t*)d_V;
    a.qs = q_stride;
    a.qos = q_out_stride;
    a.ks = k_stride;
    a.vs = v_stride;
    a.q_heads = pg->heads * q_per_kv;
    if (pg->dtype == SALICACHE_F16)
        return rotary->pairing == SALICACHE_HALVES ? rotary_dim<TypeF16, true>(c, pg, a, st) : rotary_dim<TypeF16, false>(c, pg, a, st);
    return rotary->pairing == SALICACHE_HALVES ? rotary_dim<TypeBF16, true>(c, pg, a, st) : rotary_dim<TypeBF16, false>(c, pg, a, st);
}
