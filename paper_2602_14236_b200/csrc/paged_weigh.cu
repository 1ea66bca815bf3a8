// What attention gave each cached position (the weight that eviction goes by):
//
//   out_j = decay in_j + sum_i e^(scale q_i . K^_j - lse_i)   over the call's rows i, and their query heads, that see j
//
// The logarithms of the softmax sums come from the attention, so every position stands for itself: no maximum, no division,
// and nothing to be joined.  Only K is read.
//
// This file's kernel: a warp has 16 keys of one head as the long side of m16n8k16 matrix instructions, straight from the pages
// into the registers of its operands, the next 16 under way meanwhile; rows of q are the columns, 8 at a time.  A lane sums its
// columns' weights, four lanes join at the end.  All groups of 16 keys stand in one line, of which every warp takes an equal
// stretch, so that lengths on the device decide the split and warps never wait for one another.
#include <math.h>

#include "paged_frags.cuh"
#include "paged_weigh.cuh"

namespace {

constexpr int WG_THREADS = 256, WG_WARPS = WG_THREADS / 32;

// A group of 16 keys: its sequence, head and first position.
struct WgPlace {
    int b, h, k, groups;                     // the k-th of `groups`
    PgSeq s;
    int held;                                // positions that have a weight
};
__device__ __forceinline__ void wg_enter(WgPlace& p, const WgArgs& a) {
    p.s = pg_seq(a.sq, a.pc, p.b);
    p.held = wg_held(p.s, a);
    p.groups = (p.held + 15) >> 4;
}
__device__ __forceinline__ void wg_next(WgPlace& p, const WgArgs& a) {
    if (++p.k < p.groups) return;
    p.k = 0;
    if (++p.h < a.pc.heads) return;
    p.h = 0;
    do {
        if (++p.b >= a.sq.n_seqs) return;
        wg_enter(p, a);
    } while (p.groups == 0);
}
// Where the warp's stretch of the line starts; `left` groups, none if that is 0.
__device__ __forceinline__ WgPlace wg_start(const WgArgs& a, int warp, int warps, long long& left) {
    const int lane = threadIdx.x & 31;
    auto units = [&](int b) -> long long {
        return b < a.sq.n_seqs ? (long long)((wg_held(pg_seq(a.sq, a.pc, b), a) + 15) >> 4) * a.pc.heads : 0ll;
    };
    long long total = 0;
    const long long mine = units(lane);
    for (int b0 = 0; b0 < a.sq.n_seqs; b0 += 32) total += __shfl_sync(0xffffffffu, pt_scan(b0 == 0 ? mine : units(b0 + lane)), 31);
    long long beg, end, before = 0;
    pt_share(total, warp, warps, beg, end);
    left = end - beg;
    WgPlace p{};
    if (left == 0) return p;
    for (int b0 = 0; b0 < a.sq.n_seqs; b0 += 32) {
        const long long n = b0 == 0 ? mine : units(b0 + lane), incl = before + pt_scan(n);
        const uint32_t hit = __ballot_sync(0xffffffffu, beg >= incl - n && beg < incl);
        if (hit) {
            const int from = __ffs(hit) - 1;
            const long long at = __shfl_sync(0xffffffffu, beg - (incl - n), from);
            p.b = b0 + from;
            wg_enter(p, a);
            p.h = (int)(at / p.groups);
            p.k = (int)(at - (long long)p.h * p.groups);
            return p;
        }
        before = __shfl_sync(0xffffffffu, incl, 31);
    }
    left = 0;
    return p;
}

// 16 keys' rows and scales from their page.
template <int FMT, int D>
__device__ __forceinline__ void fetch_keys(KTile<FMT, D>& t, const PgCache& pc, size_t slot, int g8, int c4) {
    using KT = KTile<FMT, D>;
    const uint8_t* p = pc.data + slot * KT::RB + KT::at(g8, c4);
    const uint8_t* m = pc.scale + slot * KT::MB + KT::meta_at(g8);
#pragma unroll
    for (int r = 0; r < 2; ++r) {
        if constexpr (KT::RB >= 64) {
#pragma unroll
            for (int i = 0; i < KT::RB / 64; ++i) {
                const uint4 v = __ldcs(reinterpret_cast<const uint4*>(p + 8 * r * KT::RB + 64 * i));
                t.k[r][4 * i] = v.x;
                t.k[r][4 * i + 1] = v.y;
                t.k[r][4 * i + 2] = v.z;
                t.k[r][4 * i + 3] = v.w;
            }
        } else {
            const uint2 v = __ldcs(reinterpret_cast<const uint2*>(p + 8 * r * KT::RB));
            t.k[r][0] = v.x;
            t.k[r][1] = v.y;
        }
        if (FMT == PF_I8) t.s[r] = *reinterpret_cast<const uint16_t*>(m + 8 * r * KT::MB);
        if (FMT == PF_I4) t.s[r] = *reinterpret_cast<const uint32_t*>(m + 8 * r * KT::MB);
    }
}

// Column tile n of a sequence's rows for one head: B fragments, and the columns' sums (as powers of two).
template <int FMT, int D>
struct Columns {
    uint32_t q[D / 16][2];
    float lse[2];                            // of rows 8 n + 2 c4 and the next; +inf for what is no row
    __device__ __forceinline__ void load(const WgArgs& a, const PgSeq& s, int h, int n, int rows, int g8, int c4) {
        const int rr = 8 * n + g8;
        const uint16_t* src = a.q + (long long)(s.row0 + rr / a.G) * a.q_stride + (long long)(h * a.G + rr % a.G) * D;
#pragma unroll
        for (int st = 0; st < D / 16; ++st) {
            int d[4];
            q_dims<FMT>(st, c4, D, d);
            uint32_t x0 = 0, x1 = 0;
            if (rr < rows) {
                x0 = __ldg(reinterpret_cast<const uint32_t*>(src + d[0]));
                x1 = __ldg(reinterpret_cast<const uint32_t*>(src + (FMT == PF_I4 ? d[1] : d[2])));
            }
            q[st][0] = FMT == PF_I4 ? __byte_perm(x0, x1, 0x5410) : x0;
            q[st][1] = FMT == PF_I4 ? __byte_perm(x0, x1, 0x7632) : x1;
        }
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int r = 8 * n + 2 * c4 + i;
            lse[i] = INFINITY;
            if (r < rows) {
                const float x = __ldg(a.lse + (long long)(s.row0 + r / a.G) * (a.pc.heads * a.G) + h * a.G + r % a.G);
                lse[i] = x == -INFINITY ? INFINITY : x * PT_LOG2E;
            }
        }
    }
};

template <typename T, int FMT, int D>
__global__ void __launch_bounds__(WG_THREADS)
k_weigh_few(WgArgs a) {
    const int lane = threadIdx.x & 31, g8 = lane >> 2, c4 = lane & 3;
    grid_wait();
    grid_release();
    long long left;
    WgPlace p = wg_start(a, blockIdx.x * WG_WARPS + (threadIdx.x >> 5), gridDim.x * WG_WARPS, left);
    if (left == 0) return;
    const Codes<T> cd;
    // the page of a group: -1 there is none, -2 no row needs it
    auto page_of = [&](const WgPlace& x) -> int {
        if (x.s.n == 0) return -2;
        const int pid = __ldg(a.sq.table + (size_t)x.b * a.sq.width + ((x.k << 4) >> a.pc.page_shift));
        return pid >= 0 && pid < a.pc.n_pages ? pid : -1;
    };
    auto fetch = [&](KTile<FMT, D>& t, const WgPlace& x, int pid) {
        if (pid >= 0) fetch_keys<FMT, D>(t, a.pc, pg_slot(a.pc, pid, 0, x.h, (x.k << 4) & ((1 << a.pc.page_shift) - 1)), g8, c4);
    };
    KTile<FMT, D> t{}, next{};
    int pid = page_of(p);
    fetch(t, p, pid);
    Columns<FMT, D> col;
    int have_b = -1, have_h = -1;            // what `col` holds column tile 0 of
    while (true) {
        WgPlace pn = p;
        int pid_n = -2;
        if (left > 1) {
            wg_next(pn, a);
            pid_n = page_of(pn);
            fetch(next, pn, pid_n);
        }
        const PgSeq& s = p.s;
        const int j0 = p.k << 4, rows = s.n * a.G;
        float had[2] = {0.0f, 0.0f}, sum[2] = {0.0f, 0.0f};
        if (c4 == 0) {
#pragma unroll
            for (int r = 0; r < 2; ++r)
                if (j0 + key_of(g8) + 8 * r < p.held) had[r] = wg_had(a, s, p.b, p.h, j0 + key_of(g8) + 8 * r);
        }
        if (lane == 0 && (pid == -1 || (p.k == 0 && (p.s.cut || p.s.len > a.w_stride)))) atomicMin(a.status, SALICACHE_E_CAPACITY);
        if (pid >= 0) {
            // the first row that sees the first key, and its column tile
            for (int n = max(0, j0 - s.pos0) * a.G / 8; 8 * n < rows; ++n) {
                if (n != 0 || have_b != p.b || have_h != p.h) {
                    col.load(a, s, p.h, n, rows, g8, c4);
                    have_b = n == 0 ? p.b : -1;
                    have_h = p.h;
                }
                float sc[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                for (int i = 0; i < D / 16; ++i) {
                    uint32_t a0, a1, a2, a3;
                    key_frag<T, FMT, D>(cd, t.k[0], t.s[0], i, a0, a2);
                    key_frag<T, FMT, D>(cd, t.k[1], t.s[1], i, a1, a3);
                    mma16816<T>(sc, a0, a1, a2, a3, col.q[i][0], col.q[i][1]);
                }
                float w[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) w[i] = ex2(fmaf(sc[i], a.scale, -col.lse[i & 1]));
                if (s.pos0 + 8 * n / a.G < j0 + 15 || 8 * n + 8 > rows) {
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int r = 8 * n + 2 * c4 + (i & 1);
                        if (r >= rows || s.pos0 + r / a.G < j0 + key_of(g8) + 8 * (i >> 1)) w[i] = 0.0f;
                    }
                }
                sum[0] += w[0] + w[1];
                sum[1] += w[2] + w[3];
            }
        }
#pragma unroll
        for (int r = 0; r < 2; ++r) {
            sum[r] += __shfl_xor_sync(0xffffffffu, sum[r], 1);
            sum[r] += __shfl_xor_sync(0xffffffffu, sum[r], 2);
            if (c4 == 0 && j0 + key_of(g8) + 8 * r < p.held) wg_put(a, s, p.b, p.h, j0 + key_of(g8) + 8 * r, had[r], sum[r]);
        }
        if (--left == 0) break;
        t = next;
        p = pn;
        pid = pid_n;
    }
}

template <typename T, int FMT, int D>
int launch_few(salicache_ctx* c, const WgArgs& a, cudaStream_t st) {
    SC_CHECK(pt_launch(k_weigh_few<T, FMT, D>, dim3((unsigned)(2 * c->sm_count)), WG_THREADS, 0, st, a));
    c->launches++;
    SC_CHECK(cudaGetLastError());
    return SALICACHE_OK;
}
template <typename T, int D>
int few_format(salicache_ctx* c, const WgArgs& a, int format, cudaStream_t st) {
    if (format == SALICACHE_FP16) return launch_few<T, PF_16, D>(c, a, st);
    if (format == SALICACHE_INT8) return launch_few<T, PF_I8, D>(c, a, st);
    return launch_few<T, PF_I4, D>(c, a, st);
}

}  // namespace

int sc_paged_weigh(salicache_ctx* c, const salicache_pages* pg, const salicache_seqs* sq, const void* d_q, int64_t q_stride,
                   int q_per_kv, float softmax_scale, const float* d_lse, float decay, const float* d_weight_in, float* d_weight_out,
                   int64_t weight_stride, void* d_work, cudaStream_t st) {
    WgArgs a{};
    a.pc = pg_cache(pg);
    a.sq = pg_seqs(sq);
    a.q = (const uint16_t*)d_q;
    a.lse = d_lse;
    a.in = d_weight_in;
    a.out = d_weight_out;
    a.q_stride = q_stride;
    a.w_stride = weight_stride;
    a.G = q_per_kv;
    a.scale = softmax_scale * PT_LOG2E;
    a.decay = decay;
    a.status = c->d_status;
    a.wait_limit = c->paged_wait;
    if ((long long)sq->n_rows * q_per_kv > 16ll * sq->n_seqs) return sc_weigh_many(c, a, pg, (char*)d_work, st);
    if (pg->dtype == SALICACHE_F16)
        return pg->head_dim == 128 ? few_format<TypeF16, 128>(c, a, pg->format, st) : few_format<TypeF16, 64>(c, a, pg->format, st);
    return pg->head_dim == 128 ? few_format<TypeBF16, 128>(c, a, pg->format, st) : few_format<TypeBF16, 64>(c, a, pg->format, st);
}
