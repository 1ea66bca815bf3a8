// Attention of new rows over the paged cache (Eq. 2 with the dequantisation of Sec. III-C fused in).
//
//   a_j = scale q . K^_j over the visible j,  m = max_j a_j,  l = sum_j e^(a_j - m),  out = sum_j e^(a_j - m) V^_j / l
//
// One warp per (row, query head) walks the visible positions with a running maximum and sum, head_dim / 32 dimensions a
// lane.
#include <math.h>

#include "paged.cuh"

namespace {

template <typename T, int FMT, int D>
__device__ __forceinline__ void load_dims(const PgCache& pc, size_t slot, int lane, float (&x)[D / 32]) {
    constexpr int N = D / 32;
    const uint8_t* src = pc.data + slot * pg_row_bytes<FMT, D>();
    if (FMT == PF_16) {
#pragma unroll
        for (int i = 0; i < N / 2; ++i) {
            const uint32_t w = reinterpret_cast<const uint32_t*>(src)[lane * (N / 2) + i];
            x[2 * i] = T::lo(w);
            x[2 * i + 1] = T::hi(w);
        }
        return;
    }
    float v[N];
    if (FMT == PF_I8) {
        const float s = T::lo(reinterpret_cast<const uint16_t*>(pc.scale)[slot]);
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = __fmul_rn((float)reinterpret_cast<const int8_t*>(src)[lane * N + i], s);
    } else {
        const uint32_t m = reinterpret_cast<const uint32_t*>(pc.scale)[slot];
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const uint32_t c = (src[(lane * N + i) / 2] >> (4 * (i & 1))) & 15u;
            v[i] = __fadd_rn(__fmul_rn((float)c, T::lo(m)), T::hi(m));
        }
    }
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = T::lo(T::round(v[i]));
}

template <typename T, int FMT, int D>
__global__ void __launch_bounds__(128)
k_paged_attend(PgCache pc, PgSeqs sq, const uint16_t* __restrict__ q, long long qs, int G, float scale, int window, int sinks,
               uint16_t* __restrict__ out, long long os, float* __restrict__ lse, int* __restrict__ status) {
    constexpr int N = D / 32;
    const int lane = threadIdx.x & 31, hq = blockIdx.y * 4 + (threadIdx.x >> 5), r = blockIdx.x;
    const int Hq = pc.heads * G;
    if (hq >= Hq) return;
    int b = 0;
    for (int base = 0; base < sq.n_seqs; base += 32) {
        const int k = base + lane;
        b += __popc(__ballot_sync(0xffffffffu, k < sq.n_seqs && sq.start[k + 1] <= r));
    }
    if (b >= sq.n_seqs) return;
    const PgSeq s = pg_seq(sq, pc, b);
    if (r < s.row0 || r >= s.row0 + s.n) return;
    const int pos = s.pos0 + (r - s.row0), h = hq / G;
    float qv[N], o[N], m = -INFINITY, l = 0.0f;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        qv[i] = T::lo(q[r * qs + (long long)hq * D + lane * N + i]);
        o[i] = 0.0f;
    }
    const int end = min(pos + 1, s.len);
    const int lo = window ? max(0, pos - window + 1) : 0;
    if (s.cut && pos >= s.len && lane == 0) atomicMin(status, SALICACHE_E_CAPACITY);
    for (int j = 0; j < end; ++j) {
        if (j < lo && j >= sinks) j = lo;
        if (j >= end) break;
        const int pid = sq.table[(size_t)b * sq.width + (j >> pc.page_shift)];
        if (pid < 0 || pid >= pc.n_pages) {
            if (lane == 0) atomicMin(status, SALICACHE_E_CAPACITY);
            continue;
        }
        float k[N], v[N], a = 0.0f;
        load_dims<T, FMT, D>(pc, pg_slot(pc, pid, 0, h, j & ((1 << pc.page_shift) - 1)), lane, k);
        load_dims<T, FMT, D>(pc, pg_slot(pc, pid, 1, h, j & ((1 << pc.page_shift) - 1)), lane, v);
#pragma unroll
        for (int i = 0; i < N; ++i) a += qv[i] * k[i];
#pragma unroll
        for (int x = 16; x; x >>= 1) a += __shfl_xor_sync(0xffffffffu, a, x);
        a *= scale;
        if (a > m) {
            const float f = __expf(m - a);
            l *= f;
#pragma unroll
            for (int i = 0; i < N; ++i) o[i] *= f;
            m = a;
        }
        const float p = __expf(a - m);
        l += p;
#pragma unroll
        for (int i = 0; i < N; ++i) o[i] += p * v[i];
    }
    const float inv = l > 0.0f ? 1.0f / l : 0.0f;
#pragma unroll
    for (int i = 0; i < N; ++i) out[r * os + (long long)hq * D + lane * N + i] = T::round(o[i] * inv);
    if (lse && lane == 0) lse[(long long)r * Hq + hq] = l > 0.0f ? m + logf(l) : -INFINITY;
}

template <typename T, int FMT, int D>
int launch_attend(salicache_ctx* c, const PgCache& pc, const PgSeqs& sq, const void* q, int64_t qs, int G, float scale, int window,
                  int sinks, void* out, int64_t os, float* lse, cudaStream_t st) {
    const dim3 grid((unsigned)sq.n_rows, (unsigned)((pc.heads * G + 3) / 4));
    k_paged_attend<T, FMT, D><<<grid, 128, 0, st>>>(pc, sq, (const uint16_t*)q, qs, G, scale, window, sinks, (uint16_t*)out, os, lse,
                                                  c->d_status);
    c->launches++;
    SC_CHECK(cudaGetLastError());
    return SALICACHE_OK;
}

}  // namespace

int64_t sc_paged_work_bytes(const salicache_ctx* c, int head_dim) { return 2ll * c->sm_count * 256 * (head_dim + 2) * 4; }

int sc_paged_attend(salicache_ctx* c, const salicache_pages* pg, const salicache_seqs* q, const void* d_q, int64_t q_stride,
                    int q_per_kv, float softmax_scale, int window, int sinks, void* d_out, int64_t out_stride, float* d_lse,
                    void* d_work, cudaStream_t st) {
    const PgCache pc = pg_cache(pg);
    const PgSeqs sq = pg_seqs(q);
#define GO(T, F, D) return launch_attend<T, F, D>(c, pc, sq, d_q, q_stride, q_per_kv, softmax_scale, window, sinks, d_out, out_stride, d_lse, st)
#define GO_FORMAT(T, D)                                      \
    do {                                                     \
        if (pg->format == SALICACHE_FP16) GO(T, PF_16, D);   \
        if (pg->format == SALICACHE_INT8) GO(T, PF_I8, D);   \
        GO(T, PF_I4, D);                                     \
    } while (0)
    if (pg->dtype == SALICACHE_F16) {
        if (pg->head_dim == 128) GO_FORMAT(TypeF16, 128);
        GO_FORMAT(TypeF16, 64);
    }
    if (pg->head_dim == 128) GO_FORMAT(TypeBF16, 128);
    GO_FORMAT(TypeBF16, 64);
#undef GO_FORMAT
#undef GO
}
