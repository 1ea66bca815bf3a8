// How the attention kernels over the paged cache share their work, and how split results are joined.
//
// An item is (sequence, key/value head, tile of rows); rows are numbered i * G + g (new token i, query head g of the
// group), so that all query heads of a group meet a key in one tile.  An item's work is the tiles of 128 positions that
// any of its rows may see: tiles of the first `sinks` positions and those from the window's edge on.  All items' tiles
// stand in one line, and block c of C takes the c-th equal stretch of it, wherever items begin and end: a batch of very
// different lengths, or one long sequence, loads every SM alike, and the split follows the lengths on the device, so
// that a captured call adapts to new ones.
// A stretch that covers an item from its first to its last tile writes the output.  Else the block leaves unnormalised
// sums, running maxima and denominators in the caller's workspace: at most one item that began in an earlier block
// ("head") and one that goes on in a later block ("tail").  A second kernel joins tail and heads in the order of the
// blocks, so results do not depend on timing.
#pragma once
#include "paged.cuh"
#include "paged_async.cuh"

constexpr int PT_KEYS = 128;                 // positions per tile
constexpr float PT_NONE = -3.0e38f;          // running maximum of a row that has seen nothing
constexpr float PT_LOG2E = 1.4426950408889634f, PT_LN2 = 0.6931471805599453f;

struct PtArgs {
    PgCache pc;
    PgSeqs sq;
    const uint16_t* q;
    uint16_t* out;
    float* lse;
    long long q_stride, out_stride;
    int G, window, sinks;
    int tile_rows;                           // rows of an item at most
    float scale;                             // softmax scale * log2(e): the kernels work in powers of two
    float* part;                             // [2 * blocks][rows of a tile][D], tail records after head records of a block
    float2* stat;                            // [2 * blocks][rows of a tile]: running maximum (powers of two), denominator
    int4* head;                              // [2 * blocks]: per block: head record (0 none, 1 the item goes on, 2 it ends); tail record:
                                             // 1 + head or 0, row tile, -; then its sequence's first row, rows, -, -
    int* status;
    int wait_limit;                          // tries before a wait between a block's roles is given up
};

// paged_chunk.cu
int sc_paged_chunk(salicache_ctx* c, const PtArgs& a, const salicache_pages* pg, char* work, cudaStream_t st);

// The tiles an item's rows may see.
struct PtSpan {
    int n;                                   // tiles
    int sink_tiles, first;                   // tile k is k below sink_tiles, first + k - sink_tiles from there on
    int lo, hi;                              // [lo, hi): positions inside some row's window; below `sinks` seen by all
    int all_lo, all_hi;                      // positions in [all_lo, all_hi) or below min(sinks, all_hi) are seen by every row
    __device__ __forceinline__ int tile(int k) const { return k < sink_tiles ? k : first + (k - sink_tiles); }
};
__device__ __forceinline__ PtSpan pt_span(const PgSeq& s, int G, int r0, int r1, int window, int sinks) {
    PtSpan p;
    const int p0 = s.pos0 + r0 / G, p1 = s.pos0 + (r1 - 1) / G;      // first and last row's position
    p.hi = max(0, min(p1 + 1, s.len));
    p.all_hi = max(0, min(p0 + 1, s.len));
    p.lo = window ? max(0, p0 - window + 1) : 0;
    p.all_lo = window ? max(0, p1 - window + 1) : 0;
    p.first = p.lo / PT_KEYS;
    p.sink_tiles = min(p.first, (min(window ? sinks : 0, p.hi) + PT_KEYS - 1) / PT_KEYS);
    p.n = p.sink_tiles + max(0, (p.hi + PT_KEYS - 1) / PT_KEYS - p.first);
    return p;
}
// Whether the row at position `pos` sees position j (j < len is the caller's to check).
__device__ __forceinline__ bool pt_sees(int pos, int j, int window, int sinks) {
    return j <= pos && (window == 0 || j > pos - window || j < sinks);
}

__device__ __forceinline__ int pt_row_tiles(const PgSeq& s, const PtArgs& a) { return (s.n * a.G + a.tile_rows - 1) / a.tile_rows; }
__device__ __forceinline__ PtSpan pt_item(const PgSeq& s, const PtArgs& a, int rt) {
    const int r0 = rt * a.tile_rows, r1 = min(r0 + a.tile_rows, s.n * a.G);
    return pt_span(s, a.G, r0, r1, a.window, a.sinks);
}

// A block's place in the line of tiles.
struct PtWalk {
    long long left;                          // tiles still to do
    int b, h, rt, k;                         // the next one: item and tile within it
};
// ... and the sequence it is in.
struct PtPlace {
    PtWalk w;
    PgSeq s;
};

// A block's share of one item, which every role of a block works out for itself.  An item counts ITEM units before its
// tiles' for its fixed cost, so that a stretch of many short items is not longer than one long item's.
template <int ITEM>
struct PtSeg {
    PtSpan sp;
    int k0, k1, t0, tiles, rows;             // units [k0, k1), first tile, tiles with keys, rows in the item
    bool last, real;                         // the item's end is in here; some of its tiles are (an item without keys has one)
    static __device__ __noinline__ PtSeg of(const PtArgs& a, PtWalk w, PgSeq s) {
        PtSeg g;
        g.set(a, w, s);
        return g;
    }
    __device__ __forceinline__ void set(const PtArgs& a, const PtWalk& w, const PgSeq& s) {
        sp = pt_item(s, a, w.rt);
        const int units = ITEM + max(sp.n, 1);
        k0 = w.k;
        k1 = (int)min((long long)units, k0 + w.left);
        rows = min(a.tile_rows, s.n * a.G - w.rt * a.tile_rows);
        t0 = max(0, k0 - ITEM);
        const int t1 = max(0, k1 - ITEM);
        last = k1 == units;
        real = t1 > t0;
        tiles = sp.n == 0 ? 0 : t1 - t0;
    }
    // Page of keys 16 grp .. of tile k: -2 no row sees them (or grp > 7), -1 there is no such page.
    __device__ __forceinline__ int page_of(const PtArgs& a, const PtWalk& w, int k, int grp) const {
        const int j = sp.tile(k) * PT_KEYS + grp * 16;
        if (grp > 7 || j >= sp.hi || (j + 16 <= sp.lo && j >= a.sinks)) return -2;
        const int p = a.sq.table[(size_t)w.b * a.sq.width + (j >> a.pc.page_shift)];
        return p >= 0 && p < a.pc.n_pages ? p : -1;
    }
    // Whether some row sees each key of tile k (pages permitting).
    __device__ __forceinline__ bool clean(const PtArgs& a, int k) const {
        const int j0 = sp.tile(k) * PT_KEYS;
        return j0 + PT_KEYS <= sp.hi && (j0 >= sp.lo || j0 + PT_KEYS <= a.sinks);
    }
};

// Tiles (and fixed costs) of one head of the sequence that each lane of a warp has; a lane sums a few row tiles by itself,
// the warp sums them together where there are many.
template <int ITEM>
__device__ __forceinline__ long long pt_per_head(const PtArgs& a, PgSeq s) {
    constexpr int ALONE = 2;
    const int lane = threadIdx.x & 31, R = pt_row_tiles(s, a);
    long long w = 0;
    if (R <= ALONE)
#pragma unroll 1
        for (int rt = 0; rt < R; ++rt) w += ITEM + max(1, pt_item(s, a, rt).n);
    for (uint32_t many = __ballot_sync(0xffffffffu, R > ALONE); many; many &= many - 1) {
        const int from = __ffs(many) - 1;
        PgSeq o{};
        o.n = __shfl_sync(0xffffffffu, s.n, from);
        o.pos0 = __shfl_sync(0xffffffffu, s.pos0, from);
        o.len = __shfl_sync(0xffffffffu, s.len, from);
        const int Ro = pt_row_tiles(o, a);
        long long x = 0;
#pragma unroll 1
        for (int rt = lane; rt < Ro; rt += 32) x += ITEM + max(1, pt_item(o, a, rt).n);
#pragma unroll
        for (int d = 16; d; d >>= 1) x += __shfl_xor_sync(0xffffffffu, x, d);
        if (lane == from) w = x;
    }
    return w;
}
__device__ __forceinline__ long long pt_scan(long long v) {          // inclusive, over a warp
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const long long t = __shfl_up_sync(0xffffffffu, v, o);
        if (lane >= o) v += t;
    }
    return v;
}
__device__ __forceinline__ PgSeq pt_seq_of(const PgSeq& s, int from) {
    PgSeq o;
    o.row0 = __shfl_sync(0xffffffffu, s.row0, from);
    o.n = __shfl_sync(0xffffffffu, s.n, from);
    o.pos0 = __shfl_sync(0xffffffffu, s.pos0, from);
    o.len = __shfl_sync(0xffffffffu, s.len, from);
    o.cut = __shfl_sync(0xffffffffu, (int)s.cut, from);
    return o;
}
// The block's stretch [beg, end) of the line: 32-bit divisions unless it needs more.
__device__ __forceinline__ void pt_share(long long total, int block, int blocks, long long& beg, long long& end) {
    const long long each = total >> 32 ? total / blocks : (long long)((uint32_t)total / (uint32_t)blocks);
    const uint32_t over = (uint32_t)(total - each * blocks);
    beg = each * block + over * (uint32_t)block / (uint32_t)blocks;
    end = each * (block + 1) + over * (uint32_t)(block + 1) / (uint32_t)blocks;
}
// `at` units into sequence `s` (w units): head, row tile and unit within it.  Called by whole warps.
template <int ITEM>
__device__ __forceinline__ PtWalk pt_find(const PtArgs& a, PgSeq s, long long w, long long at, PtWalk walk) {
    const int lane = threadIdx.x & 31, R = pt_row_tiles(s, a);
    long long rem;
    if (w >> 32) {
        const long long ph = w / a.pc.heads;
        walk.h = (int)(at / ph);
        rem = at - walk.h * ph;
    } else {
        const uint32_t ph = (uint32_t)w / (uint32_t)a.pc.heads;
        walk.h = (int)((uint32_t)at / ph);
        rem = (uint32_t)at - walk.h * ph;
    }
#pragma unroll 1
    for (int r0 = 0;; r0 += 32) {
        const int n = r0 + lane < R ? ITEM + max(1, pt_item(s, a, r0 + lane).n) : 0;
        const long long incl = pt_scan(n);
        const uint32_t hit = __ballot_sync(0xffffffffu, rem >= incl - n && rem < incl);
        if (hit || r0 + 32 >= R) {
            const int from = hit ? __ffs(hit) - 1 : 0;
            walk.rt = r0 + from;
            walk.k = __shfl_sync(0xffffffffu, (int)(rem - (incl - n)), from);
            return walk;
        }
        rem -= __shfl_sync(0xffffffffu, incl, 31);
    }
}

// Where the block starts, and the sequence it starts in; the same for every thread.  Up to 32 sequences every warp works
// it out for itself, a lane per sequence, without a barrier (2.2 us after the start instead of 3.0); more of them are
// shared out over the block's threads, with scans through shared memory.
struct PtShared {
    long long wsum[32];
    long long left, at, w;
    int b;
    PgSeq s;
};
template <int THREADS, int ITEM>
__device__ __forceinline__ PtPlace pt_start(const PtArgs& a, int block, int blocks, PtShared& sh) {
    const int lane = threadIdx.x & 31, wid = threadIdx.x >> 5;
    PtPlace place{};
    PtWalk& walk = place.w;
    PgSeq& seq = place.s;
    long long beg, end;
    if (a.sq.n_seqs <= 32) {
        PgSeq s{};
        if (lane < a.sq.n_seqs) s = pg_seq(a.sq, a.pc, lane);
        const long long w = pt_per_head<ITEM>(a, s) * a.pc.heads, incl = pt_scan(w);
        pt_share(__shfl_sync(0xffffffffu, incl, 31), block, blocks, beg, end);
        if (beg == end) return place;
        const uint32_t hit = __ballot_sync(0xffffffffu, beg >= incl - w && beg < incl);
        const int from = __ffs(hit) - 1;
        seq = pt_seq_of(s, from);
        walk.b = from;
        walk.left = end - beg;
        walk = pt_find<ITEM>(a, seq, __shfl_sync(0xffffffffu, w, from), __shfl_sync(0xffffffffu, beg - (incl - w), from), walk);
        return place;
    }
    auto units = [&](int b, PgSeq& s) -> long long {
        s = PgSeq{};
        if (b < a.sq.n_seqs) s = pg_seq(a.sq, a.pc, b);
        return pt_per_head<ITEM>(a, s) * a.pc.heads;
    };
    PgSeq s0, s;
    const long long w0 = units(threadIdx.x, s0);
    long long mine = w0;
    for (int b0 = THREADS; b0 < a.sq.n_seqs; b0 += THREADS) mine += units(b0 + threadIdx.x, s);
#pragma unroll
    for (int o = 16; o; o >>= 1) mine += __shfl_xor_sync(0xffffffffu, mine, o);
    if (lane == 0) sh.wsum[wid] = mine;
    __syncthreads();
    long long total = 0;
#pragma unroll
    for (int i = 0; i < THREADS / 32; ++i) total += sh.wsum[i];
    __syncthreads();
    pt_share(total, block, blocks, beg, end);
    if (beg == end) return place;
    long long before = 0;                    // units of the sequences before this round's
    for (int b0 = 0; b0 < a.sq.n_seqs; b0 += THREADS) {
        const int b = b0 + threadIdx.x;
        const long long w = b0 == 0 ? w0 : units(b, s);
        if (b0 == 0) s = s0;
        const long long incl = pt_scan(w);
        if (lane == 31) sh.wsum[wid] = incl;
        __syncthreads();
        long long off = before;
        for (int i = 0; i < wid; ++i) off += sh.wsum[i];
        const long long at = beg - (off + incl - w);
        if (at >= 0 && at < w) {             // this thread's sequence holds the start
            sh.b = b;
            sh.at = at;
            sh.w = w;
            sh.s = s;
        }
        for (int i = 0; i < THREADS / 32; ++i) before += sh.wsum[i];
        __syncthreads();
        if (before > beg) break;
    }
    seq = sh.s;
    walk.b = sh.b;
    walk.left = end - beg;
    walk = pt_find<ITEM>(a, seq, sh.w, sh.at, walk);
    return place;
}

// On to the next item: row tiles, then heads, then sequences with rows.
__device__ __forceinline__ void pt_next(PtWalk& w, PgSeq& s, const PtArgs& a) {
    w.k = 0;
    if (++w.rt < pt_row_tiles(s, a)) return;
    w.rt = 0;
    if (++w.h < a.pc.heads) return;
    w.h = 0;
#pragma unroll 1
    do {
        ++w.b;
        if (w.b >= a.sq.n_seqs) return;      // cannot happen while tiles are left
        s = pg_seq(a.sq, a.pc, w.b);
    } while (s.n == 0);
}
// The same in a function, for a kernel of many roles: with a copy of all this at each call it had grown past the
// instruction cache (170 KB).
static __device__ __noinline__ PtPlace pt_after(const PtArgs& a, PtPlace p) {
    pt_next(p.w, p.s, a);
    return p;
}
__device__ __forceinline__ void pt_next_far(PtWalk& w, PgSeq& s, const PtArgs& a) {
    const PtPlace p = pt_after(a, PtPlace{w, s});
    w = p.w;
    s = p.s;
}

// The record slots of the item that block c left as its tail: its tail, then later blocks' heads until one ends.  All
// threads of the block get the count.  flag(c): the kind of block c's head record.
template <typename F>
__device__ __forceinline__ int pt_records(F flag, int c, int blocks, int* list) {
    __shared__ int count;
    if (threadIdx.x < 32) {
        const int lane = threadIdx.x;
        int n = 1;
        if (lane == 0) list[0] = 2 * c + 1;
        for (int c0 = c + 1; c0 < blocks; c0 += 32) {
            const int f = c0 + lane < blocks ? flag(c0 + lane) : 0;
            const uint32_t ends = __ballot_sync(0xffffffffu, f == 2);
            const uint32_t upto = ends ? (2u << (__ffs(ends) - 1)) - 1u : 0xffffffffu;       // lanes up to the first that ends
            const uint32_t has = __ballot_sync(0xffffffffu, f != 0) & upto;
            if (has >> lane & 1u) list[n + __popc(has & ((1u << lane) - 1u))] = 2 * (c0 + lane);
            n += __popc(has);
            if (ends) break;
        }
        if (lane == 0) count = n;
    }
    __syncthreads();
    return count;
}
constexpr int PT_MAX_BLOCKS = 1024;          // of the attention kernels

// What a block says of its records (see PtArgs::head).
__device__ __forceinline__ void pt_tail(int4 (&hd)[2], const PtWalk& w, const PgSeq& s) {
    hd[0].y = w.h + 1;
    hd[0].z = w.rt;
    hd[1].x = s.row0;
    hd[1].y = s.n;
}

// Joins split items.  grid.x: blocks of the first kernel, grid.y: groups of 8 rows, one warp per row.
template <typename T, int RT, int D>
__global__ void __launch_bounds__(256)
k_paged_join(PtArgs a, int blocks) {
    __shared__ int list[PT_MAX_BLOCKS + 1];
    grid_wait();
    constexpr int N = D / 32;
    const int4 hd = a.head[2 * blockIdx.x], sq = a.head[2 * blockIdx.x + 1];
    if (hd.y == 0) return;
    const int n = pt_records([&](int c) { return a.head[2 * c].x; }, blockIdx.x, blocks, list);
    const int lane = threadIdx.x & 31, row = blockIdx.y * 8 + (threadIdx.x >> 5);
    const int h = hd.y - 1, r = hd.z * RT + row;
    if (r >= sq.y * a.G) return;
    // the maximum moves along with the records, eight under way at a time
    constexpr int AHEAD = 8;
    float M = PT_NONE, o[N], l = 0.0f;
#pragma unroll
    for (int i = 0; i < N; ++i) o[i] = 0.0f;
    for (int i0 = 0; i0 < n; i0 += AHEAD) {
        float2 st[AHEAD];
        float v[AHEAD][N];
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) {
            const size_t t = (size_t)list[min(i0 + u, n - 1)] * RT + row;
            st[u] = a.stat[t];
#pragma unroll
            for (int x = 0; x < N; ++x) v[u][x] = a.part[t * D + lane * N + x];
        }
        float nm = M;
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) nm = fmaxf(nm, st[u].x);
        const float f = ex2(M - nm);
        M = nm;
        l *= f;
#pragma unroll
        for (int x = 0; x < N; ++x) o[x] *= f;
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) {
            const float e = i0 + u < n ? ex2(st[u].x - M) : 0.0f;
            l += e * st[u].y;
#pragma unroll
            for (int x = 0; x < N; ++x) o[x] += e * v[u][x];
        }
    }
    const int hq = h * a.G + r % a.G;
    const long long tok = sq.x + r / a.G;
    const float inv = l > 0.0f ? 1.0f / l : 0.0f;
    uint16_t* dst = a.out + tok * a.out_stride + (long long)hq * D + lane * N;
#pragma unroll
    for (int i = 0; i < N; i += 2) *reinterpret_cast<uint32_t*>(dst + i) = T::pack(o[i] * inv, o[i + 1] * inv);
    if (a.lse && lane == 0) a.lse[tok * ((long long)a.pc.heads * a.G) + hq] = l > 0.0f ? (M + log2f(l)) * PT_LN2 : -INFINITY;
}
