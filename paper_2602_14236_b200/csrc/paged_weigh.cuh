// What the two kernels of salicache_paged_weigh share.
#pragma once
#include "paged_plan.cuh"

constexpr int WM_KEYS = 256;                 // of a tile in the kernel for many rows
struct WgArgs {
    PgCache pc;
    PgSeqs sq;
    const uint16_t* q;
    const float *lse, *in;
    float* out;
    long long q_stride, w_stride;
    int G;
    float scale, decay;                      // scale * log2(e)
    int rows_over, rows_to;                  // sequences with more rows of q than the one and at most the other are this kernel's
    int* status;
    int wait_limit;                          // tries before a wait between a block's roles is given up
    int tok;                                 // many rows: tokens of a tile of rows, and 2^38 / tok
    uint64_t per_tok;
    float* part;                             // [2 * blocks][keys of a tile]: sums of a tile's rows so far, tail after head records of a block
    int join;                                // blocks whose records are still to be joined
    int4* head;                              // [2 * blocks]: per block: head record (0 none, 1 the tile goes on, 2 it ends), tail record
                                             // (0, 1), its sequence, its head; then its tile of keys, -, -, -
};

// Positions of a sequence that have a weight; none, if the sequence is the other kernel's.
__device__ __forceinline__ int wg_held(const PgSeq& s, const WgArgs& a) {
    const int rows = s.n * a.G;
    return rows > a.rows_over && rows <= a.rows_to ? (int)min((long long)s.len, a.w_stride) : 0;
}
// What position j of (sequence b, head h) had before, of which decay is left.
__device__ __forceinline__ float wg_had(const WgArgs& a, const PgSeq& s, int b, int h, int j) {
    if (!a.in || (s.n > 0 && j >= s.pos0)) return 0.0f;
    return a.in[((size_t)b * a.pc.heads + h) * a.w_stride + j];
}
__device__ __forceinline__ void wg_put(const WgArgs& a, const PgSeq& s, int b, int h, int j, float had, float sum) {
    a.out[((size_t)b * a.pc.heads + h) * a.w_stride + j] = fmaf(s.n > 0 ? a.decay : 1.0f, had, sum);
}

// Joins the tiles of keys that the ends of stretches have cut in the kernel for many rows: block c the one whose tail that kernel's
// block c left, a thread per key.
__device__ __forceinline__ void wg_join(const WgArgs& a) {
    __shared__ int list[PT_MAX_BLOCKS + 1];
    const int4 hd = a.head[2 * blockIdx.x];
    if (hd.y == 0) return;
    const int b = hd.z, h = hd.w, j = a.head[2 * blockIdx.x + 1].x * WM_KEYS + threadIdx.x;
    const int n = pt_records([&](int c) { return a.head[2 * c].x; }, blockIdx.x, a.join, list);
    const PgSeq s = pg_seq(a.sq, a.pc, b);
    float sum = 0.0f;
    for (int i = 0; i < n; ++i) sum += a.part[(size_t)list[i] * WM_KEYS + threadIdx.x];
    if (j < (int)min((long long)s.len, a.w_stride)) wg_put(a, s, b, h, j, wg_had(a, s, b, h, j), sum);
}

// paged_weigh_many.cu.  `join`: with a kernel of its own for what is left to be joined; without, `a` says what the next kernel has to
// join.
int sc_weigh_many(salicache_ctx* c, WgArgs& a, const salicache_pages* pg, char* work, bool join, cudaStream_t st);
