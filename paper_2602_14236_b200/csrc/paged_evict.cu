// Eviction from the paged cache: which positions a budget keeps, and moving them together.
//
// Selection.  Of every (sequence, key/value head) the first `sinks` and the last `recent` positions stay, and the heaviest of
// those between.  One block per (sequence, head) finds the weight of the last one that fits by its bits, 11, 11 and 10 of them
// from the top (floats become unsigned numbers in the same order), counting in shared memory, where the keys stay too; then it
// writes the positions above that weight, and the lowest ones at it, in ascending order: every warp has a stretch of positions,
// whose counts are summed before the second look.  Bound by the latency of its passes: 24 lists of 640 positions 5.2 us, 64 of
// up to 8640 9.8 us, 32 of up to 32768 17 us (a third of it the first look, at 50 bytes a clock and with counts that meet).
//
// Moving.  A block has the rows that a tile of a list's entries names, K and V of one head, 16 bytes a lane.  Into other pages all
// tiles of a list move at once.  In place one block takes a list's tiles in turn, and reads a tile before it writes it: entry
// k of an ascending list is at least first + k, so what a tile writes lies below all that later tiles read.
// Into other pages bound by memory: 32768 rows of 8 heads x 128 in 16 bits, 268 MB: 45 to 47 us = 5.7 to 6.0 TB/s, 0.89 to 0.93 of the
// copy bandwidth; 31127 rows of INT4 codes, 68 MB: 14 us.  In place, where a block per list has one tile after the other under way: 163
// and 32 us.
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

constexpr int SH_BINS = 2048, SH_KEYS = 49 * 1024;               // keys that shared memory holds at most

__device__ __forceinline__ uint32_t cluster_rank() {
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ void cluster_sync() {
    asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// A word of another block's shared memory.
__device__ __forceinline__ uint32_t ld_peer(const uint32_t* p, uint32_t rank) {
    uint32_t at, v;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"(smem_u32(p)), "r"(rank));
    asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(at) : "memory");
    return v;
}

// A block per (sequence, head), or a cluster of two with half of the positions each.  `held`: keys of a part that the block's
// shared memory holds; those behind are read again in every pass.
template <int BLOCKS>
__global__ void __launch_bounds__(SH_THREADS)
k_select_heavy(const float* weight, long long stride, int heads, const int* len_, int budget, int sinks, int recent, int* keep, int* kept,
               int* status, int held) {
    extern __shared__ uint32_t keys[];
    __shared__ uint32_t hist[3][SH_BINS], warp_sum[SH_WARPS][2], part_sum[2];
    __shared__ uint32_t s_digit, s_left;
    const int rank = BLOCKS > 1 ? (int)cluster_rank() : 0;
    const int list = blockIdx.x / BLOCKS, b = list / heads, tid = threadIdx.x, lane = tid & 31, wid = tid >> 5;
    const uint32_t before = (1u << lane) - 1u;
    grid_wait();
    grid_release();
    int len = max(len_[b], 0);
    const long long most = min(stride, 1ll << 30);       // sums of positions and strides of the loops below stay within 32 bits
    if (len > most) {
        len = (int)most;
        if (tid == 0) atomicMin(status, SALICACHE_E_CAPACITY);
    }
    int* out = keep + (size_t)list * budget;
    if (list % heads == 0 && rank == 0 && tid == 0) kept[b] = min(len, budget);
    constexpr int each = BLOCKS * SH_THREADS;
    const int me = rank * SH_THREADS + tid;
    auto sync_all = [&]() {
        if (BLOCKS > 1) cluster_sync();
        else __syncthreads();
    };
    if (len <= budget) {                     // the same for all blocks of the cluster, as is what follows
        for (int i = me; i < budget; i += each) out[i] = i < len ? i : -1;
        return;
    }
    for (int i = me; i < sinks; i += each) out[i] = i;
    for (int i = me; i < recent; i += each) out[budget - recent + i] = len - recent + i;
    const int take = budget - sinks - recent, all = len - recent - sinks;
    if (take == 0) return;
    // of positions sinks .. sinks + all - 1 this block has n from `from` on
    const int part = ((all + BLOCKS - 1) / BLOCKS + 31) / 32 * 32, from = min(all, rank * part), n = min(part, all - from);
    const float* w = weight + (size_t)list * stride + sinks + from;
    auto key = [&](int i) -> uint32_t { return i < held ? keys[i] : weight_key(w[i]); };
    for (int i = tid; i < 3 * SH_BINS; i += SH_THREADS) hist[0][i] = 0;
    __syncthreads();
    // the take-th heaviest: its key's bits from the top, 11, 11 and 10 of them
    uint32_t prefix = 0, left = (uint32_t)take;
#pragma unroll
    for (int pass = 0; pass < 3; ++pass) {
        const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0, bits = pass == 2 ? 10 : 11;
        if (pass == 0) {
            constexpr int E = 8;             // loads under way
            for (int i0 = wid * 32; i0 < n; i0 += E * SH_THREADS) {
                uint32_t k[E];
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    const int i = i0 + e * SH_THREADS + lane;
                    k[e] = i < n ? weight_key(w[i]) : 0u;
                }
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    const int i = i0 + e * SH_THREADS + lane;
                    if (i < n) {
                        if (i < held) keys[i] = k[e];
                        atomicAdd(&hist[0][k[e] >> shift], 1u);
                    }
                }
            }
        } else {
            auto count = [&](uint32_t k) {
                if (k >> (shift + bits) == prefix >> (shift + bits)) atomicAdd(&hist[pass][k >> shift & ((1u << bits) - 1u)], 1u);
            };
#pragma unroll 8
            for (int i = tid; i < min(n, held); i += SH_THREADS) count(keys[i]);
            for (int i = (held - tid + SH_THREADS - 1) / SH_THREADS * SH_THREADS + tid; i < n; i += SH_THREADS) count(weight_key(w[i]));
        }
        sync_all();
        // from the top: thread t has bins 2047 - 2 t and 2046 - 2 t of all blocks
        uint32_t c0 = hist[pass][SH_BINS - 1 - 2 * tid], c1 = hist[pass][SH_BINS - 2 - 2 * tid];
        if (BLOCKS > 1) {
            c0 += ld_peer(&hist[pass][SH_BINS - 1 - 2 * tid], rank ^ 1);
            c1 += ld_peer(&hist[pass][SH_BINS - 2 - 2 * tid], rank ^ 1);
        }
        uint32_t incl = c0 + c1;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const uint32_t t = __shfl_up_sync(0xffffffffu, incl, o);
            if (lane >= o) incl += t;
        }
        if (lane == 31) warp_sum[wid][0] = incl;
        __syncthreads();
        incl += __reduce_add_sync(0xffffffffu, lane < wid ? warp_sum[lane][0] : 0u);
        const uint32_t above = incl - c0 - c1;
        if (above < left && incl >= left) {
            const bool second = above + c0 < left;
            s_digit = SH_BINS - 1 - 2 * tid - second;
            s_left = left - above - (second ? c0 : 0u);
        }
        __syncthreads();
        prefix |= s_digit << shift;
        left = s_left;
    }
    // positions above `prefix`, and the first `left` at it: a stretch for every warp, counted, then written
    const int seg = ((n + SH_WARPS - 1) / SH_WARPS + 31) / 32 * 32, a = min(n, wid * seg), e = min(n, a + seg);
    uint32_t n_above = 0, n_equal = 0;
    if (e <= held) {
#pragma unroll 8
        for (int i = a + lane; i < e; i += 32) {
            n_above += keys[i] > prefix;
            n_equal += keys[i] == prefix;
        }
    } else
        for (int i = a + lane; i < e; i += 32) {
            n_above += key(i) > prefix;
            n_equal += key(i) == prefix;
        }
    n_above = __reduce_add_sync(0xffffffffu, n_above);
    n_equal = __reduce_add_sync(0xffffffffu, n_equal);
    __syncthreads();                         // the sums of the last scan have been read
    if (lane == 0) {
        warp_sum[wid][0] = n_above;
        warp_sum[wid][1] = n_equal;
    }
    __syncthreads();
    if (wid == 0) {
        const uint32_t x = __reduce_add_sync(0xffffffffu, warp_sum[lane][0]), y = __reduce_add_sync(0xffffffffu, warp_sum[lane][1]);
        if (lane == 0) {
            part_sum[0] = x;
            part_sum[1] = y;
        }
    }
    uint32_t above = __reduce_add_sync(0xffffffffu, lane < wid ? warp_sum[lane][0] : 0u);
    uint32_t equal = __reduce_add_sync(0xffffffffu, lane < wid ? warp_sum[lane][1] : 0u);
    sync_all();
    for (int r = 0; r < rank; ++r) {
        above += ld_peer(&part_sum[0], r);
        equal += ld_peer(&part_sum[1], r);
    }
    sync_all();                              // nobody reads another block's memory any more
    constexpr int E = 4;                     // times 32 positions at a time
    for (int i0 = a; i0 < e; i0 += 32 * E) {
        uint32_t is_above[E], is_equal[E];
#pragma unroll
        for (int x = 0; x < E; ++x) {
            const int i = i0 + 32 * x + lane;
            const uint32_t k = i < e ? key(i) : 0u;
            is_above[x] = __ballot_sync(0xffffffffu, i < e && k > prefix);
            is_equal[x] = __ballot_sync(0xffffffffu, i < e && k == prefix);
        }
#pragma unroll
        for (int x = 0; x < E; ++x) {
            const uint32_t eq = equal + __popc(is_equal[x] & before);
            const bool mine = is_above[x] >> lane & 1u || (is_equal[x] >> lane & 1u && eq < left);
            if (mine) out[sinks + above + __popc(is_above[x] & before) + min(eq, left)] = sinks + from + i0 + 32 * x + lane;
            above += __popc(is_above[x]);
            equal += __popc(is_equal[x]);
        }
    }
}

constexpr int KP_THREADS = 256;
// Rows of a tile: eight 16-byte pieces a thread, K and V (twice as many, 128 rows of 512 bytes, take a quarter longer); in place,
// where tiles follow one another, sixteen.
template <int FMT, int D, bool IN_PLACE> __host__ __device__ constexpr int kp_tile() {
    return (IN_PLACE ? 16 : 8) * KP_THREADS / (2 * (pg_row_bytes<FMT, D>() / 16));
}

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

// The pages that position e of sequence b comes from and position t goes to; false: one of them is in no page.
__device__ __forceinline__ bool kp_pages(const KpArgs& a, int b, int len, int e, long long t, int& from, int& to) {
    const bool held = e >= 0 && e < len && t < min((long long)a.to.width << a.pc.page_shift, 1ll << 30);
    from = held ? a.from.table[(size_t)b * a.from.width + (e >> a.pc.page_shift)] : -1;
    to = held ? a.to.table[(size_t)b * a.to.width + (t >> a.pc.page_shift)] : -1;
    return from >= 0 && from < a.pc.n_pages && to >= 0 && to < a.pc.n_pages;
}

// Weights of one list, each where its row moves, in tiles of 8 entries a thread, of which block `first_tile` of `blocks` takes its own.  A
// tile is read before it is written: one block moves a list's weights in place.
constexpr int KW_EACH = 8, KW_TILE = KW_EACH * KP_THREADS;
__device__ void keep_weights(const KpArgs& a, int b, int h, int n, int len, const int* list, int first_tile, int blocks) {
    const long long first = a.first ? max(a.first[b], 0) : 0;
    const size_t row = ((size_t)b * a.pc.heads + h) * a.w_stride;
    for (int k0 = first_tile * KW_TILE; k0 < n; k0 += blocks * KW_TILE) {
        int src[KW_EACH], p[KW_EACH], q[KW_EACH];
        float w[KW_EACH];
#pragma unroll
        for (int i = 0; i < KW_EACH; ++i) {
            const int k = k0 + i * KP_THREADS + threadIdx.x;
            src[i] = k < n ? list[k] : -1;
            if (src[i] >= a.w_stride || first + k >= a.w_stride) src[i] = -1;
        }
#pragma unroll
        for (int i = 0; i < KW_EACH; ++i)
            if (!kp_pages(a, b, len, src[i], first + k0 + i * KP_THREADS + threadIdx.x, p[i], q[i])) src[i] = -1;
#pragma unroll
        for (int i = 0; i < KW_EACH; ++i) w[i] = src[i] >= 0 ? a.w_in[row + src[i]] : 0.0f;
        __syncthreads();
#pragma unroll
        for (int i = 0; i < KW_EACH; ++i)
            if (src[i] >= 0) a.w_out[row + first + k0 + i * KP_THREADS + threadIdx.x] = w[i];
    }
}

// grid.y: (sequence, head); grid.x: blocks for the weights, if they move, then a list's tiles (one block for all of them in place).
template <int FMT, int D, bool IN_PLACE>
__global__ void __launch_bounds__(KP_THREADS)
k_paged_keep(KpArgs a, int weight_blocks, int row_blocks) {
    constexpr int RB = pg_row_bytes<FMT, D>(), MB = pg_meta_bytes<FMT>(), LPR = RB / 16, PIECES = 2 * LPR;
    constexpr int KP_TILE = kp_tile<FMT, D, IN_PLACE>(), EACH = KP_TILE * PIECES / KP_THREADS;      // 16-byte pieces of a thread
    constexpr int METAS = MB > 0 ? (2 * KP_TILE + KP_THREADS - 1) / KP_THREADS : 1;                 // scales of a thread
    __shared__ long long src[KP_TILE], dst[KP_TILE];             // slots of K, or -1
    const int b = blockIdx.y / a.pc.heads, h = blockIdx.y % a.pc.heads;
    grid_wait();
    grid_release();
    const int n = min(max(a.kept[b], 0), a.keep_width);
    const long long cap = min((long long)a.from.width << a.pc.page_shift, 1ll << 30);
    const int len = (int)min((long long)max(a.from.len[b], 0), cap);
    const int* list = a.keep + ((size_t)b * a.keep_heads + (a.keep_heads > 1 ? h : 0)) * a.keep_width;
    if ((int)blockIdx.x < weight_blocks) {
        keep_weights(a, b, h, n, len, list, blockIdx.x, weight_blocks);
        return;
    }
    const long long first = a.first ? max(a.first[b], 0) : 0;
    const int mask = (1 << a.pc.page_shift) - 1;
    const size_t v_step = (size_t)a.pc.heads << a.pc.page_shift;         // slots from K to V
    for (int k0 = ((int)blockIdx.x - weight_blocks) * KP_TILE; k0 < n; k0 += row_blocks * KP_TILE) {
        for (int i = threadIdx.x; i < KP_TILE; i += KP_THREADS) {
            const int k = k0 + i;
            long long s = -1, d = -1;
            if (k < n) {
                const int e = list[k];
                const long long t = first + k;
                int p, q;
                if (kp_pages(a, b, len, e, t, p, q)) {
                    s = (long long)pg_slot(a.pc, p, 0, h, e & mask);
                    d = (long long)pg_slot(a.pc, q, 0, h, (int)t & mask);
                }
                if (s < 0) atomicMin(a.status, SALICACHE_E_CAPACITY);
                else if (s == d) s = -1;                         // stays where it is
            }
            src[i] = s;
            dst[i] = d;
        }
        __syncthreads();
        uint4 v[EACH];
        uint32_t meta[METAS];
#pragma unroll
        for (int i = 0; i < EACH; ++i) {
            const int p = i * KP_THREADS + threadIdx.x, k = p / PIECES, kv = p / LPR & 1, c = p % LPR;
            if (src[k] >= 0) v[i] = __ldcs(reinterpret_cast<const uint4*>(a.pc.data + (src[k] + kv * v_step) * RB) + c);
        }
#pragma unroll
        for (int i = 0; i < METAS; ++i) {
            const int p = i * KP_THREADS + threadIdx.x, k = p >> 1;
            meta[i] = 0;
            if (MB > 0 && k < KP_TILE && src[k] >= 0) {
                const uint8_t* at = a.pc.scale + (src[k] + (p & 1) * v_step) * MB;
                meta[i] = MB == 2 ? *reinterpret_cast<const uint16_t*>(at) : *reinterpret_cast<const uint32_t*>(at);
            }
        }
        if (IN_PLACE) __syncthreads();                           // all of the tile is read
#pragma unroll
        for (int i = 0; i < EACH; ++i) {
            const int p = i * KP_THREADS + threadIdx.x, k = p / PIECES, kv = p / LPR & 1, c = p % LPR;
            if (src[k] >= 0) __stcs(reinterpret_cast<uint4*>(a.pc.data + (dst[k] + kv * v_step) * RB) + c, v[i]);
        }
#pragma unroll
        for (int i = 0; i < METAS; ++i) {
            const int p = i * KP_THREADS + threadIdx.x, k = p >> 1;
            if (MB > 0 && k < KP_TILE && src[k] >= 0) {
                uint8_t* at = a.pc.scale + (dst[k] + (p & 1) * v_step) * MB;
                if (MB == 2) *reinterpret_cast<uint16_t*>(at) = (uint16_t)meta[i];
                else *reinterpret_cast<uint32_t*>(at) = meta[i];
            }
        }
        __syncthreads();                                         // the slots are used up
    }
}

template <int FMT, int D, bool IN_PLACE>
int launch_keep(salicache_ctx* c, const KpArgs& a, cudaStream_t st) {
    constexpr int TILE = kp_tile<FMT, D, IN_PLACE>();
    const int tiles = (a.keep_width + TILE - 1) / TILE, lists = a.from.n_seqs * a.pc.heads;
    const int row_blocks = IN_PLACE ? 1 : tiles;
    const int weight_blocks = !a.w_in ? 0 : a.w_in == a.w_out ? 1 : (a.keep_width + KW_TILE - 1) / KW_TILE;
    const dim3 grid((unsigned)(weight_blocks + row_blocks), (unsigned)lists);
    SC_CHECK(pt_launch(k_paged_keep<FMT, D, IN_PLACE>, grid, KP_THREADS, 0, st, a, weight_blocks, row_blocks));
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
    // Two blocks where every one finds an SM and has 4096 positions at least: 32 lists of 32768 17.6 us instead of 22.6, while
    // a cluster's launch costs short lists 2 us.  (Clusters of four: 21 us; not all of them find their place at once.)
    const int blocks = (long long)n_seqs * heads * 2 <= c->sm_count && weight_stride >= 2 * 4096 ? 2 : 1;
    const int held = (int)min((weight_stride + blocks - 1) / blocks + 32, (int64_t)SH_KEYS);
    auto kernel = blocks == 2 ? k_select_heavy<2> : k_select_heavy<1>;
    // 48 KB, of which the counts take half, need no leave
    if (held > 5 * 1024) SC_CHECK(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, SH_KEYS * 4));
    cudaLaunchConfig_t cfg{};
    cudaLaunchAttribute at[2]{};
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    at[1].id = cudaLaunchAttributeClusterDimension;
    at[1].val.clusterDim.x = 2;
    at[1].val.clusterDim.y = at[1].val.clusterDim.z = 1;
    cfg.gridDim = dim3((unsigned)(n_seqs * heads * blocks));
    cfg.blockDim = dim3(SH_THREADS);
    cfg.dynamicSmemBytes = (size_t)held * 4;
    cfg.stream = st;
    cfg.attrs = at;
    cfg.numAttrs = blocks;
    SC_CHECK(cudaLaunchKernelEx(&cfg, kernel, d_weight, (long long)weight_stride, heads, (const int*)d_len, budget, sinks, recent,
                                (int*)d_keep, (int*)d_kept, c->d_status, held));
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
