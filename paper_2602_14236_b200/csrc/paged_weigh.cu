// What attention gave each cached position (the weight that eviction goes by):
//
//   out_j = decay in_j + sum_i e^(scale q_i . K^_j - lse_i)   over the call's rows i, and their query heads, that see j
//
// The logarithms of the softmax sums come from the attention, so every position stands for itself: no maximum, no division,
// and nothing to be joined.  Only K is read.
//
// This file's kernel, for few rows per sequence: a warp has 16 keys of one head as the long side of m16n8k16 matrix
// instructions, rows of q are the columns, 8 at a time, 16 at most.  A lane sums its columns' weights, four lanes join at the
// end.  Every warp has a ring of its own in shared memory, which its first lanes fill by bulk copies of 16 keys' rows and scales.  All
// groups of keys stand in one line, of which every warp takes an equal stretch, so that the lengths on the device decide the
// split, and warps never wait for one another.
// Measured, 16 sequences of 8000 positions, 8 heads x 128, one token and four query heads a group (four tokens), with the launches of
// the other kernel, which return at once: 16-bit pages 55 us (55) = 4.9 TB/s, bound by memory; INT8 39 us (45), INT4 38 us (47), bound
// by neither memory nor issue slots alone: some 320 instructions go into 16 INT4 keys of a head, 112 of them turn codes into numbers,
// and take 64 % of the issue slots; the rest is fixed latencies of one chain of products after the other.
#include <limits.h>
#include <math.h>

#include "paged_frags.cuh"
#include "paged_weigh.cuh"

namespace {

constexpr int WG_THREADS = 256, WG_WARPS = WG_THREADS / 32, WG_BLOCKS = 2;      // per SM: 128 registers a thread

// Keys of a group: 32, so that what a group costs beside its products is shared by two of them, unless the rings hold too few
// such groups (72 us with 16 keys for 32 single tokens over INT4 pages).
template <int FMT, int D> __host__ __device__ constexpr int wg_keys() { return FMT == PF_16 && D == 128 ? 16 : 32; }

// A warp's ring: stages of a group's rows and their scales.
template <int FMT, int D>
struct WgRing {
    static constexpr int ROWS = wg_keys<FMT, D>() * pg_row_bytes<FMT, D>(), META = wg_keys<FMT, D>() * pg_meta_bytes<FMT>(), STAGE = ROWS + META;
    static constexpr int ROOM = 108 * 1024 / WG_WARPS, STAGES = ROOM / STAGE < 6 ? ROOM / STAGE : 6;
    static constexpr int BYTES = WG_WARPS * STAGES * STAGE;
};

// Positions of a sequence that have a weight; none, if the sequence is the other kernel's.
__device__ __forceinline__ int wf_held(const PgSeq& s, const WgArgs& a) { return s.n * a.G <= a.rows_to ? wg_held(s, a) : 0; }
// A group of KEYS keys: its sequence, head and first position.
struct WgPlace {
    int b, h, k, groups;                     // the k-th of `groups`
    PgSeq s;
    int held;                                // positions that have a weight
};
template <int KEYS>
__device__ __forceinline__ void wg_enter(WgPlace& p, const WgArgs& a) {
    p.s = pg_seq(a.sq, a.pc, p.b);
    p.held = wf_held(p.s, a);
    p.groups = (p.held + KEYS - 1) / KEYS;
}
template <int KEYS>
__device__ __forceinline__ void wg_next(WgPlace& p, const WgArgs& a) {
    if (++p.k < p.groups) return;
    p.k = 0;
    if (++p.h < a.pc.heads) return;
    p.h = 0;
    do {
        if (++p.b >= a.sq.n_seqs) return;
        wg_enter<KEYS>(p, a);
    } while (p.groups == 0);
}
// Where the warp's stretch of the line starts; `left` groups, none if that is 0.
template <int KEYS>
__device__ __forceinline__ WgPlace wg_start(const WgArgs& a, int warp, int warps, long long& left) {
    const int lane = threadIdx.x & 31;
    auto units = [&](int b) -> long long {
        return b < a.sq.n_seqs ? (long long)((wf_held(pg_seq(a.sq, a.pc, b), a) + KEYS - 1) / KEYS) * a.pc.heads : 0ll;
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
            wg_enter<KEYS>(p, a);
            p.h = (int)(at / p.groups);
            p.k = (int)(at - (long long)p.h * p.groups);
            return p;
        }
        before = __shfl_sync(0xffffffffu, incl, 31);
    }
    left = 0;
    return p;
}

// Column tile n of a sequence's rows for one head: B fragments, and the columns' sums (as powers of two).
template <int FMT, int D>
struct Columns {
    uint32_t q[D / 16][2];
    float lse[2];                            // of rows 8 n + 2 c4 and the next; WG_NONE for what is no row
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
            lse[i] = WG_NONE;
            if (r < rows) {
                const float x = __ldg(a.lse + (long long)(s.row0 + r / a.G) * (a.pc.heads * a.G) + h * a.G + r % a.G);
                lse[i] = x == -INFINITY ? WG_NONE : x * PT_LOG2E;
            }
        }
    }
};

// NT: column tiles that stay in registers.
template <typename T, int FMT, int D, int NT>
__global__ void __launch_bounds__(WG_THREADS, WG_BLOCKS)
k_weigh_few(WgArgs a) {
    using R = WgRing<FMT, D>;
    constexpr int STAGES = R::STAGES, KEYS = wg_keys<FMT, D>(), U = KEYS / 16;
    constexpr uint32_t RB = pg_row_bytes<FMT, D>(), MB = pg_meta_bytes<FMT>();
    static_assert(STAGES >= 2, "ring");
    extern __shared__ __align__(128) uint8_t rings[];
    __shared__ uint64_t full[WG_WARPS][STAGES];
    __shared__ int sh_gave_up;
    volatile int* gave_up = &sh_gave_up;
    const int lane = threadIdx.x & 31, wid = threadIdx.x >> 5, g8 = lane >> 2, c4 = lane & 3;
    if (threadIdx.x == 0) {
        for (int i = 0; i < WG_WARPS * STAGES; ++i) bar_init(smem_u32(&full[0][0]) + 8 * i, 1);
        sh_gave_up = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    grid_wait();
    grid_release();
    long long left;
    WgPlace p = wg_start<KEYS>(a, blockIdx.x * WG_WARPS + wid, gridDim.x * WG_WARPS, left);
    if (a.some && blockIdx.x == 0 && wid == 0) {
        bool some = false;
        for (int b = lane; b < a.sq.n_seqs; b += 32) some = some || pg_seq(a.sq, a.pc, b).n * a.G > a.rows_to;
        some = __any_sync(0xffffffffu, some);
        if (lane == 0) *a.some = some;
    }
    __syncthreads();
    const uint32_t ring = smem_u32(rings) + wid * STAGES * R::STAGE, bars = smem_u32(&full[wid][0]);

    // What is fetched goes STAGES groups ahead of what is summed.  The first U lanes bring 16 keys each; a lane looks up the
    // page of one of the next 32 times 16 keys.  `pages` has U bits for each group under way, the newest lowest: its pages exist.
    WgPlace f = p;
    long long to_fetch = left;
    int ids = 0, ids_at = -1;                // pages of 16 keys each from group ids_at of sequence f.b on
    uint32_t put = 0, pages = 0;             // next stage to fill
    int under_way = 0;                       // stages filled or about to be
    auto fetch = [&]() {
        pages <<= U;
        if (to_fetch == 0) return;
        const uint32_t bar = bars + 8 * put, dst = ring + put * R::STAGE + lane * 16 * RB;
        if (f.s.n > 0) {
            if (ids_at < 0 || f.k >= ids_at + 32 / U || f.k < ids_at) {
                ids_at = f.k;
                const int j = f.k * KEYS + lane * 16;
                ids = j < f.held ? __ldg(a.sq.table + (size_t)f.b * a.sq.width + (j >> a.pc.page_shift)) : -2;
                if (j < f.held && (ids < 0 || ids >= a.pc.n_pages)) ids = -1;
            }
            const int pid = __shfl_sync(0xffffffffu, ids, U * (f.k - ids_at) + lane % U);
            const uint32_t there = __ballot_sync(0xffffffffu, pid >= 0) & ((1u << U) - 1u);
            pages |= there;
            if (lane == 0) bar_expect(bar, __popc(there) * 16 * (RB + MB));
            __syncwarp();
            if (lane < U) {
                if (pid >= 0) {
                    const size_t slot = pg_slot(a.pc, pid, 0, f.h, (f.k * KEYS + lane * 16) & ((1 << a.pc.page_shift) - 1));
                    bulk_copy(dst, a.pc.data + slot * RB, 16 * RB, bar);
                    if (MB > 0) bulk_copy(ring + put * R::STAGE + R::ROWS + lane * 16 * MB, a.pc.scale + slot * MB, 16 * MB, bar);
                } else if (pid == -1) atomicMin(a.status, SALICACHE_E_CAPACITY);
            }
        } else if (lane == 0) bar_arrive(bar);           // nothing to come
        put = put + 1 == STAGES ? 0 : put + 1;
        ++under_way;
        if (--to_fetch > 0) {
            const int b = f.b;
            wg_next<KEYS>(f, a);
            if (f.b != b) ids_at = -1;
        }
    };
#pragma unroll 1
    for (int i = 0; i < STAGES; ++i) fetch();

    const Codes<T> cd;
    uint32_t stage = 0, phase = 0;
    bool ok = true;
    while (left > 0 && ok) {                 // the groups of one head
        const PgSeq& s = p.s;
        const int rows = s.n * a.G, run = (int)min(left, (long long)(p.groups - p.k));
        const int jl = key_of(g8) + 8 * (c4 & 1) + 16 * (c4 >> 1);       // the key that this lane writes, if the group has it
        const size_t row = ((size_t)p.b * a.pc.heads + p.h) * a.w_stride + jl;
        float* const out = a.out + row;
        const float* const in = a.in + row;
        const float decay = s.n > 0 ? a.decay : 1.0f;
        // positions below had_to had a weight before, which is looked at some groups ahead
        const bool writes = jl < KEYS;
        const int had_to = !a.in || !writes ? 0 : s.n > 0 ? min(s.pos0, p.held) : p.held, put_to = writes ? p.held : 0;
        auto load_had = [&](int k) { return KEYS * k + jl < had_to && k < p.k + run ? in[KEYS * k] : 0.0f; };
        if (lane == 0 && p.k == 0 && (s.cut || s.len > a.w_stride)) atomicMin(a.status, SALICACHE_E_CAPACITY);
        float had[3] = {0.0f, load_had(p.k), load_had(p.k + 1)};
        Columns<FMT, D> col[NT];
#pragma unroll
        for (int n = 0; n < NT; ++n)
            if (8 * n < rows) col[n].load(a, s, p.h, n, rows, g8, c4);
        bool first_columns = true;           // `col[0]` holds column tile 0
#pragma unroll 1
        for (int t = 0; t < run; ++t) {
            const int j0 = (p.k + t) * KEYS;
            had[0] = had[1];
            had[1] = had[2];
            had[2] = load_had(p.k + t + 2);
            ok = warp_wait(bars + 8 * stage, phase, a.wait_limit, gave_up);
            if (!ok) break;
            --under_way;
            const uint32_t there = pages >> (U * (STAGES - 1));
            // 16 keys at a time: four lanes' sums of slots g8 and g8 + 8, of which a lane pair exchanges one for the other
            const bool odd = c4 & 1, high = c4 & 2;
            float y[U];
#pragma unroll 1
            for (int u = 0; u < U; ++u) {
                const uint32_t at = ring + stage * R::STAGE;
                KTile<FMT, D> kt;
                kt.load(at + 16 * u * RB + KTile<FMT, D>::at(g8, c4), at + R::ROWS + 16 * u * MB + KTile<FMT, D>::meta_at(g8));
                if (u == U - 1) {
                    __syncwarp();            // the stage has been read
                    fetch();
                }
                float sum[2] = {0.0f, 0.0f};
                auto columns = [&](const Columns<FMT, D>& x, int n) {
                    float sc[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                    for (int i = 0; i < D / 16; ++i) {
                        uint32_t a0, a1, a2, a3;
                        key_frag<T, FMT, D>(cd, kt.k[0], kt.s[0], i, a0, a2);
                        key_frag<T, FMT, D>(cd, kt.k[1], kt.s[1], i, a1, a3);
                        mma16816<T>(sc, a0, a1, a2, a3, x.q[i][0], x.q[i][1]);
                    }
                    float w[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) w[i] = ex2(fmaf(sc[i], a.scale, -x.lse[i & 1]));
                    if (j0 + KEYS - 1 > s.pos0) {        // some row may be before some key
#pragma unroll
                        for (int i = 0; i < 4; ++i)
                            if (s.pos0 + (8 * n + 2 * c4 + (i & 1)) / a.G < j0 + 16 * u + key_of(g8) + 8 * (i >> 1)) w[i] = 0.0f;
                    }
                    // what is no row gives nothing, whatever its score: q is 0 behind the last row, which a key that is not finite would
                    // turn into no number, and anything in a row that sees nothing
                    const bool l0 = x.lse[0] != WG_NONE, l1 = x.lse[1] != WG_NONE;
                    sum[0] += (l0 ? w[0] : 0.0f) + (l1 ? w[1] : 0.0f);
                    sum[1] += (l0 ? w[2] : 0.0f) + (l1 ? w[3] : 0.0f);
                };
                if (there >> u & 1u) {
                    if (NT > 1 || rows <= 8) {
                        columns(col[0], 0);
                        if (NT > 1 && rows > 8) columns(col[NT - 1], NT - 1);
                    } else
#pragma unroll 1
                        for (int n = 0; n < 2; ++n) {
                            if (n != 0 || !first_columns) col[0].load(a, s, p.h, n, rows, g8, c4);
                            first_columns = n == 0;
                            columns(col[0], n);
                        }
                }
                const float x = (odd ? sum[1] : sum[0]) + __shfl_xor_sync(0xffffffffu, odd ? sum[0] : sum[1], 1);
                if (u == 0) y[0] = x;
                else y[U - 1] = x;
            }
            if (++stage == STAGES) {
                stage = 0;
                phase ^= 1;
            }
            // ... and pairs of pairs
            float x = (high ? y[U - 1] : y[0]) + __shfl_xor_sync(0xffffffffu, high ? y[0] : y[U - 1], 2);
            if (!(there >> (c4 >> 1) & 1u)) x = 0.0f;            // its page is none
            if (j0 + jl < put_to) out[j0] = fmaf(decay, had[0], x);
        }
        left -= run;
        p.k += run - 1;
        if (left > 0) wg_next<KEYS>(p, a);
    }
    for (; !ok && under_way > 0; --under_way) {              // copies in flight end before the block does
        bar_drain(bars + 8 * stage, phase);
        if (++stage == STAGES) {
            stage = 0;
            phase ^= 1;
        }
    }
    join_roles();
    if (threadIdx.x == 0 && *gave_up) atomicMin(a.status, SC_GAVE_UP);
}

template <typename T, int FMT, int D, int NT>
int launch_few(salicache_ctx* c, const WgArgs& a, cudaStream_t st) {
    using R = WgRing<FMT, D>;
    SC_CHECK(cudaFuncSetAttribute(k_weigh_few<T, FMT, D, NT>, cudaFuncAttributeMaxDynamicSharedMemorySize, R::BYTES));
    // no more blocks than there can be groups of keys for: sequences times heads times the table's groups
    const long long most = (long long)a.sq.n_seqs * a.pc.heads * ((((long long)a.sq.width << a.pc.page_shift) + wg_keys<FMT, D>() - 1) / wg_keys<FMT, D>());
    const int blocks = (int)max(1ll, min((most + WG_WARPS - 1) / WG_WARPS, (long long)c->sm_count * WG_BLOCKS));
    SC_CHECK(pt_launch(k_weigh_few<T, FMT, D, NT>, dim3((unsigned)blocks), WG_THREADS, R::BYTES, st, a));
    c->launches++;
    SC_CHECK(cudaGetLastError());
    return SALICACHE_OK;
}
template <typename T, int FMT, int D>
int few_columns(salicache_ctx* c, const WgArgs& a, cudaStream_t st) {
    const bool one = (long long)a.sq.n_rows * a.G <= 8 || (a.G <= 8 && a.sq.n_rows == a.sq.n_seqs);      // single tokens
    return one ? launch_few<T, FMT, D, 1>(c, a, st) : launch_few<T, FMT, D, 2>(c, a, st);
}
template <typename T, int D>
int few_format(salicache_ctx* c, const WgArgs& a, int format, cudaStream_t st) {
    if (format == SALICACHE_FP16) return few_columns<T, PF_16, D>(c, a, st);
    if (format == SALICACHE_INT8) return few_columns<T, PF_I8, D>(c, a, st);
    return few_columns<T, PF_I4, D>(c, a, st);
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
    // Rows of q of a sequence up to which reading the keys is the work: what two tiles of columns hold.  (16 sequences of 8000 positions, 16
    // rows each, this kernel against the other: 16-bit pages 58 / 74 us, INT8 44 / 129, INT4 45 / 117; 32 rows 179 / 75, 174 / 129,
    // 296 / 117.)  Only the device knows how many a sequence has, so each kernel takes its own ones and a batch that may have both
    // kinds gets both launches: single tokens beside a prompt are the usual batch, and either kernel takes many times as long over
    // the other's.  (31 single tokens over 8000 INT4 positions and a prompt of 4096: 158 us, 318 in the other kernel alone; 63 over
    // 4000 INT8 positions and 193 rows over 16000: 128, in this one alone 5098.)  How many rows there are for a sequence on average says
    // nothing about that: of 256 slots one may have a chunk of 200 rows while the others are idle (16000 INT4 positions: 83 us, in this
    // kernel alone 1702).  This kernel goes first and tells the others whether there is such a sequence; a batch without one pays 2 to 3 us
    // for two launches that return at once (16 single tokens over 8000 INT4 positions 46 us, 43; 256 over 2000 134, 131; 5 to 13 us where
    // they look for themselves).  The other one cannot start beside this one's rings, and after it, doing the join as well, this one added
    // 20 us to a prompt of 8192 rows (313, 290).
    const bool many = (long long)sq->n_rows * q_per_kv > WG_FEW;
    a.rows_to = many ? WG_FEW : INT_MAX;
    a.some = many ? reinterpret_cast<int*>(d_work) : nullptr;
    int rc;
    if (pg->dtype == SALICACHE_F16)
        rc = pg->head_dim == 128 ? few_format<TypeF16, 128>(c, a, pg->format, st) : few_format<TypeF16, 64>(c, a, pg->format, st);
    else
        rc = pg->head_dim == 128 ? few_format<TypeBF16, 128>(c, a, pg->format, st) : few_format<TypeBF16, 64>(c, a, pg->format, st);
    return rc == SALICACHE_OK && many ? sc_weigh_many(c, a, pg, (char*)d_work, st) : rc;
}
