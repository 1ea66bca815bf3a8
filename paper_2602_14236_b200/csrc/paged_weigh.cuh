// What the two kernels of salicache_paged_weigh share.
#pragma once
#include "paged_plan.cuh"

constexpr int WG_FEW = 16;                   // rows of q of a sequence up to which it is the other kernel's
constexpr float WG_NONE = 3.4028235e38f;     // the sum of a row that counts as none: finite, so that it is not taken for a row's own infinity
struct WgArgs {
    PgCache pc;
    PgSeqs sq;
    const uint16_t* q;
    const float *lse, *in;
    float* out;
    long long q_stride, w_stride;
    int G;
    float scale, decay;                      // scale * log2(e)
    int rows_to;                             // few rows: sequences with more rows of q are the other kernel's
    int* status;
    int wait_limit;                          // tries before a wait between a block's roles is given up
    int tok;                                 // many rows: tokens of a tile of rows, and 2^38 / tok
    uint64_t per_tok;
    float* part;                             // [2 * blocks][keys of a tile]: sums of a tile's rows so far, tail after head records of a block
    int* some;                               // whether a sequence of many rows is in the batch: the kernel for few rows tells
    int4* head;                              // [2 * blocks]: per block: head record (0 none, 1 the tile goes on, 2 it ends), tail record
                                             // (0, 1), its sequence, its head; then its tile of keys, -, -, -
};

// Positions of a sequence that have a weight.
__device__ __forceinline__ int wg_held(const PgSeq& s, const WgArgs& a) { return (int)min((long long)s.len, a.w_stride); }
// What position j of (sequence b, head h), which has rows in the call, had before, of which decay is left.
__device__ __forceinline__ float wg_had(const WgArgs& a, const PgSeq& s, int b, int h, int j) {
    if (!a.in || j >= s.pos0) return 0.0f;
    return a.in[((size_t)b * a.pc.heads + h) * a.w_stride + j];
}
__device__ __forceinline__ void wg_put(const WgArgs& a, int b, int h, int j, float had, float sum) {
    a.out[((size_t)b * a.pc.heads + h) * a.w_stride + j] = fmaf(a.decay, had, sum);
}

// paged_weigh_many.cu
int sc_weigh_many(salicache_ctx* c, const WgArgs& a, const salicache_pages* pg, char* work, cudaStream_t st);
