// Eviction from the paged cache: which positions a budget keeps, and moving them together.
//
// Selection.  Of every (sequence, key/value head) the first `sinks` and the last `recent` positions stay, and the heaviest of
// those between.  One block per (sequence, head) finds the weight of the last one that fits by its bits, eight at a time from
// the top (floats become unsigned numbers in the same order), counting in shared memory; then it writes the positions above
// that weight, and the lowest ones at it, in ascending order: every warp has a stretch of positions, whose counts are summed
// before the second look.
//
// Moving.  A block has the rows that 128 entries of a list name, K and V of one head, 16 bytes a lane.  Into other pages all
// tiles of a list move at once.  In place one block takes a list's tiles in turn, and reads a tile before it writes it: entry
// k of an ascending list is at least first + k, so what a tile writes lies below all that later tiles read.
#include "paged_async.cuh"
#include "paged.cuh"

namespace {

constexpr int SH_THREADS = 1024, SH_WARPS = SH_THREADS / 32;

// In the order of the weights; what is not a number comes first.
__device__ __forceinline__ uint32_t weight_key(float w) {
    if (w != w) return 0u;
    const uint32_t b = __float_as_uint(w + 0.0f);        // -0 is 0
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}

__global__ void __launch_bounds__(SH_THREADS)
k_select_heavy(const float* weight, long long stride, int heads, const int* len_, int budget, int sinks, int recent, int* keep, int* kept,
               int* status) {
    __shared__ uint32_t hist[256], warp_sum[SH_WARPS][2];
    __shared__ uint32_t s_digit, s_left;
    const int b = blockIdx.x / heads, h = blockIdx.x % heads, lane = threadIdx.x & 31, wid = threadIdx.x >> 5;
    grid_wait();
    grid_release();
    int len = max(len_[b], 0);
    if (len > stride) {
        len = (int)stride;
        if (threadIdx.x == 0) atomicMin(status, SALICACHE_E_CAPACITY);
    }
    const float* w = weight + (size_t)blockIdx.x * stride;
    int* out = keep + (size_t)blockIdx.x * budget;
    if (h == 0 && threadIdx.x == 0) kept[b] = min(len, budget);
    if (len <= budget) {
        for (int i = threadIdx.x; i < budget; i += SH_THREADS) out[i] = i < len ? i : -1;
        return;
    }
    for (int i = threadIdx.x; i < sinks; i += SH_THREADS) out[i] = i;
    for (int i = threadIdx.x; i < recent; i += SH_THREADS) out[budget - recent + i] = len - recent + i;
    const int lo = sinks, hi = len - recent, take = budget - sinks - recent;
    if (take == 0) return;
    // the take-th heaviest of [lo, hi): its key's bits from the top
    uint32_t prefix = 0, left = (uint32_t)take;
    for (int shift = 24; shift >= 0; shift -= 8) {
        if (threadIdx.x < 256) hist[threadIdx.x] = 0;
        __syncthreads();
        for (int i = lo + threadIdx.x; i < hi; i += SH_THREADS) {
            const uint32_t k = weight_key(w[i]);
            if (shift == 24 || k >> (shift + 8) == prefix >> (shift + 8)) atomicAdd(&hist[k >> shift & 255u], 1u);
        }
        __syncthreads();
        if (wid == 0) {                      // from the top: lane l has digits 255 - 8 l .. 248 - 8 l
            uint32_t c[8], sum = 0;
#pragma unroll
            for (int i = 0; i < 8; ++i) sum += c[i] = hist[255 - 8 * lane - i];
            uint32_t incl = sum;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const uint32_t t = __shfl_up_sync(0xffffffffu, incl, o);
                if (lane >= o) incl += t;
            }
            uint32_t above = incl - sum;
            if (above < left && incl >= left) {
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    if (above < left && above + c[i] >= left) {
                        s_digit = 255 - 8 * lane - i;
                        s_left = left - above;
                    }
                    above += c[i];
                }
            }
        }
        __syncthreads();
        prefix |= s_digit << shift;
        left = s_left;
        __syncthreads();
    }
    // positions above `prefix`, and the first `left` at it
    const int seg = ((hi - lo + SH_WARPS - 1) / SH_WARPS + 31) / 32 * 32, a = min(hi, lo + wid * seg), e = min(hi, a + seg);
    uint32_t n_above = 0, n_equal = 0;
    for (int i = a + lane; i < e; i += 32) {
        const uint32_t k = weight_key(w[i]);
        n_above += k > prefix;
        n_equal += k == prefix;
    }
    n_above = __reduce_add_sync(0xffffffffu, n_above);
    n_equal = __reduce_add_sync(0xffffffffu, n_equal);
    if (lane == 0) {
        warp_sum[wid][0] = n_above;
        warp_sum[wid][1] = n_equal;
    }
    __syncthreads();
    uint32_t above = lane < wid ? warp_sum[lane][0] : 0u, equal = lane < wid ? warp_sum[lane][1] : 0u;
    above = __reduce_add_sync(0xffffffffu, above);
    equal = __reduce_add_sync(0xffffffffu, equal);
    for (int i0 = a; i0 < e; i0 += 32) {
        const int i = i0 + lane;
        const uint32_t k = i < e ? weight_key(w[i]) : 0u;
        const uint32_t is_above = __ballot_sync(0xffffffffu, i < e && k > prefix), is_equal = __ballot_sync(0xffffffffu, i < e && k == prefix);
        const uint32_t before = (1u << lane) - 1u, eq = equal + __popc(is_equal & before);
        const bool mine = is_above >> lane & 1u || (is_equal >> lane & 1u && eq < left);
        if (mine) out[sinks + above + __popc(is_above & before) + min(eq, left)] = i;
        above += __popc(is_above);
        equal += __popc(is_equal);
    }
}

constexpr int KP_THREADS = 256, KP_TILE = 128;

struct KpArgs {
    PgCache pc;
    PgSeqs from, to;
    const int *keep, *first, *kept;
    const float* w_in;
    float* w_out;
    long long w_stride;
    int keep_heads, keep_width;
    int* status;
};

// Weights of one list in tiles of 16 entries a thread, read before they are written, so that they may move in place.
__device__ void keep_weights(const KpArgs& a, int b, int h, int n, int len, const int* list) {
    constexpr int E = 16;
    const long long first = a.first ? max(a.first[b], 0) : 0;
    const size_t row = ((size_t)b * a.pc.heads + h) * a.w_stride;
    for (int k0 = 0; k0 < n; k0 += E * KP_THREADS) {
        int src[E];
        float w[E];
#pragma unroll
        for (int i = 0; i < E; ++i) {
            const int k = k0 + i * KP_THREADS + threadIdx.x;
            src[i] = k < n ? list[k] : -1;
            if (src[i] < 0 || src[i] >= len || src[i] >= a.w_stride || first + k >= a.w_stride) src[i] = -1;
        }
#pragma unroll
        for (int i = 0; i < E; ++i) w[i] = src[i] >= 0 ? a.w_in[row + src[i]] : 0.0f;
        __syncthreads();
#pragma unroll
        for (int i = 0; i < E; ++i)
            if (src[i] >= 0) a.w_out[row + first + k0 + i * KP_THREADS + threadIdx.x] = w[i];
    }
}

// grid.y: (sequence, head); grid.x: a list's tiles (one block for all of them in place), and one more for the weights.
template <int FMT, int D, bool IN_PLACE>
__global__ void __launch_bounds__(KP_THREADS)
k_paged_keep(KpArgs a, int row_blocks) {
    constexpr int RB = pg_row_bytes<FMT, D>(), MB = pg_meta_bytes<FMT>(), LPR = RB / 16, PIECES = 2 * LPR;
    constexpr int EACH = KP_TILE * PIECES / KP_THREADS;          // 16-byte pieces of a thread
    __shared__ long long src[KP_TILE], dst[KP_TILE];             // slots of K, or -1
    const int b = blockIdx.y / a.pc.heads, h = blockIdx.y % a.pc.heads;
    grid_wait();
    grid_release();
    const int n = min(max(a.kept[b], 0), a.keep_width);
    const long long cap = min((long long)a.from.width << a.pc.page_shift, 1ll << 30);
    const int len = (int)min((long long)max(a.from.len[b], 0), cap);
    const int* list = a.keep + ((size_t)b * a.keep_heads + (a.keep_heads > 1 ? h : 0)) * a.keep_width;
    if ((int)blockIdx.x == row_blocks) {
        keep_weights(a, b, h, n, len, list);
        return;
    }
    const long long to_cap = min((long long)a.to.width << a.pc.page_shift, 1ll << 30), first = a.first ? max(a.first[b], 0) : 0;
    const int mask = (1 << a.pc.page_shift) - 1;
    const size_t v_step = (size_t)a.pc.heads << a.pc.page_shift;         // slots from K to V
    for (int k0 = blockIdx.x * KP_TILE; k0 < n; k0 += row_blocks * KP_TILE) {
        if (threadIdx.x < KP_TILE) {
            const int k = k0 + threadIdx.x;
            long long s = -1, d = -1;
            if (k < n) {
                const int e = list[k];
                const long long t = first + k;
                if (e >= 0 && e < len && t < to_cap) {
                    const int p = a.from.table[(size_t)b * a.from.width + (e >> a.pc.page_shift)];
                    const int q = a.to.table[(size_t)b * a.to.width + (t >> a.pc.page_shift)];
                    if (p >= 0 && p < a.pc.n_pages && q >= 0 && q < a.pc.n_pages) {
                        s = (long long)pg_slot(a.pc, p, 0, h, e & mask);
                        d = (long long)pg_slot(a.pc, q, 0, h, (int)t & mask);
                    }
                }
                if (s < 0) atomicMin(a.status, SALICACHE_E_CAPACITY);
                else if (s == d) s = -1;                         // stays where it is
            }
            src[threadIdx.x] = s;
            dst[threadIdx.x] = d;
        }
        __syncthreads();
        uint4 v[EACH];
        uint32_t meta = 0;
        const int mk = threadIdx.x >> 1, mkv = threadIdx.x & 1;  // a scale per thread
        static_assert(KP_THREADS == 2 * KP_TILE, "a scale per thread");
#pragma unroll
        for (int i = 0; i < EACH; ++i) {
            const int p = i * KP_THREADS + threadIdx.x, k = p / PIECES, kv = p / LPR & 1, c = p % LPR;
            if (src[k] >= 0) v[i] = __ldcs(reinterpret_cast<const uint4*>(a.pc.data + (src[k] + kv * v_step) * RB) + c);
        }
        if (MB > 0 && src[mk] >= 0) {
            const uint8_t* at = a.pc.scale + (src[mk] + mkv * v_step) * MB;
            meta = MB == 2 ? *reinterpret_cast<const uint16_t*>(at) : *reinterpret_cast<const uint32_t*>(at);
        }
        if (IN_PLACE) __syncthreads();                           // all of the tile is read
#pragma unroll
        for (int i = 0; i < EACH; ++i) {
            const int p = i * KP_THREADS + threadIdx.x, k = p / PIECES, kv = p / LPR & 1, c = p % LPR;
            if (src[k] >= 0) __stcs(reinterpret_cast<uint4*>(a.pc.data + (dst[k] + kv * v_step) * RB) + c, v[i]);
        }
        if (MB > 0 && src[mk] >= 0) {
            uint8_t* at = a.pc.scale + (dst[mk] + mkv * v_step) * MB;
            if (MB == 2) *reinterpret_cast<uint16_t*>(at) = (uint16_t)meta;
            else *reinterpret_cast<uint32_t*>(at) = meta;
        }
        __syncthreads();                                         // the slots are used up
    }
}

template <int FMT, int D, bool IN_PLACE>
int launch_keep(salicache_ctx* c, const KpArgs& a, cudaStream_t st) {
    const int tiles = (a.keep_width + KP_TILE - 1) / KP_TILE, lists = a.from.n_seqs * a.pc.heads;
    const int row_blocks = IN_PLACE ? 1 : tiles;
    const dim3 grid((unsigned)(row_blocks + (a.w_in ? 1 : 0)), (unsigned)lists);
    SC_CHECK(pt_launch(k_paged_keep<FMT, D, IN_PLACE>, grid, KP_THREADS, 0, st, a, row_blocks));
    c->launches++;
    SC_CHECK(cudaGetLastError());
    return SALICACHE_OK;
}
template <int FMT, int D>
int keep_place(salicache_ctx* c, const KpArgs& a, bool in_place, cudaStream_t st) {
    return in_place ? launch_keep<FMT, D, true>(c, a, st) : launch_keep<FMT, D, false>(c, a, st);
}
template <int D>
int keep_format(salicache_ctx* c, const KpArgs& a, int format, bool in_place, cudaStream_t st) {
    if (format == SALICACHE_FP16) return keep_place<PF_16, D>(c, a, in_place, st);
    if (format == SALICACHE_INT8) return keep_place<PF_I8, D>(c, a, in_place, st);
    return keep_place<PF_I4, D>(c, a, in_place, st);
}

}  // namespace

int sc_select_heavy(salicache_ctx* c, const float* d_weight, int64_t weight_stride, int heads, int n_seqs, const int32_t* d_len,
                    int budget, int sinks, int recent, int32_t* d_keep, int32_t* d_kept, cudaStream_t st) {
    SC_CHECK(pt_launch(k_select_heavy, dim3((unsigned)(n_seqs * heads)), SH_THREADS, 0, st, d_weight, (long long)weight_stride, heads,
                       (const int*)d_len, budget, sinks, recent, (int*)d_keep, (int*)d_kept, c->d_status));
    c->launches++;
    SC_CHECK(cudaGetLastError());
    return SALICACHE_OK;
}

int sc_paged_keep(salicache_ctx* c, const salicache_pages* pg, const salicache_seqs* sq, const int32_t* d_keep, int keep_heads,
                  int keep_width, const int32_t* d_first, const int32_t* d_kept, const salicache_seqs* to, const float* d_weight_in,
                  float* d_weight_out, int64_t weight_stride, cudaStream_t st) {
    KpArgs a{};
    a.pc = pg_cache(pg);
    a.from = pg_seqs(sq);
    a.to = to ? pg_seqs(to) : a.from;
    a.keep = d_keep;
    a.first = d_first;
    a.kept = d_kept;
    a.w_in = d_weight_in;
    a.w_out = d_weight_out;
    a.w_stride = weight_stride;
    a.keep_heads = keep_heads;
    a.keep_width = keep_width;
    a.status = c->d_status;
    return pg->head_dim == 128 ? keep_format<128>(c, a, pg->format, !to, st) : keep_format<64>(c, a, pg->format, !to, st);
}
