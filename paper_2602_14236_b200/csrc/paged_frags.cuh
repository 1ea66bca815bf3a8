// Sixteen keys of a head as the long side of m16n8k16 matrix instructions: what a lane (g8 = lane / 4, c4 = lane % 4) takes
// of them, and of the rows of q that they are multiplied with.  Shared by the attention over few rows (paged_attend.cu) and
// by the attention weights (paged_weigh.cu).
#pragma once
#include "paged.cuh"
#include "paged_async.cuh"

template <typename T>
__device__ __forceinline__ void mma16816(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1);
template <>
__device__ __forceinline__ void mma16816<TypeF16>(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
template <>
__device__ __forceinline__ void mma16816<TypeBF16>(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// Key of row slot r of the fragments: the keys 2 c, 2 c + 1 that a lane multiplies are c and c + 4, which lie in
// different banks.
__device__ __forceinline__ int key_of(int g8) { return (g8 >> 1) + 4 * (g8 & 1); }

// What a lane takes of 16 keys: the shares of the keys of slots g8 and g8 + 8 that make its A fragments.
template <int FMT, int D>
struct KTile {
    static constexpr int W = pg_row_bytes<FMT, D>() / 16;       // words of a key row per lane
    uint32_t k[2][W];
    uint32_t s[2];                                              // scale, or (scale, zero)
    static constexpr int RB = pg_row_bytes<FMT, D>(), MB = pg_meta_bytes<FMT>();
    // this lane's first bytes of 16 keys' rows, and of their scales
    static __device__ __forceinline__ uint32_t at(int g8, int c4) { return key_of(g8) * RB + (RB >= 64 ? 16 : 8) * c4; }
    static __device__ __forceinline__ uint32_t meta_at(int g8) { return key_of(g8) * MB; }
    __device__ __forceinline__ void load(uint32_t rows, uint32_t meta) {
#pragma unroll
        for (int r = 0; r < 2; ++r) {
            if (RB >= 64) {
#pragma unroll
                for (int i = 0; i < RB / 64; ++i) lds16(&k[r][4 * i], rows + 8 * r * RB + 64 * i);
            } else lds_words<2>(&k[r][0], rows + 8 * r * RB);
            if (FMT == PF_I8) s[r] = lds_u16(meta + 8 * r * MB);
            if (FMT == PF_I4) lds_words<1>(&s[r], meta + 8 * r * MB);
        }
    }
};
// K fragments of matrix instruction st: registers (a0, a2) of one key row.
template <typename T, int FMT, int D>
__device__ __forceinline__ void key_frag(const Codes<T>& cd, const uint32_t (&k)[KTile<FMT, D>::W], uint32_t s, int st, uint32_t& x, uint32_t& y) {
    if (FMT == PF_16) {
        x = k[2 * st];
        y = k[2 * st + 1];
    } else if (FMT == PF_I8) {
        const uint32_t s2 = dup_lo(s);
        x = mul2<T>(cd.bytes(k[st], 0x5140), s2);
        y = mul2<T>(cd.bytes(k[st], 0x5342), s2);
    } else {
        const uint32_t s2 = dup_lo(s), z2 = dup_hi(s), w = k[st >> 1] >> (8 * (st & 1));
        x = fma2<T>(cd.nib_lo(w), s2, z2);
        y = fma2<T>(cd.nib_hi(w), s2, z2);
    }
}
// The dimension pairs that instruction st multiplies in a lane's registers b0 and b1.
template <int FMT>
__device__ __forceinline__ void q_dims(int st, int c4, int D, int (&d)[4]) {
    if (FMT == PF_16) {
        const int base = (st >> 1) * 32 + c4 * 8 + (st & 1) * 4;
        d[0] = base; d[1] = base + 1; d[2] = base + 2; d[3] = base + 3;
    } else if (FMT == PF_I8) {
        const int base = (st >> 2) * 64 + c4 * 16 + (st & 3) * 4;
        d[0] = base; d[1] = base + 1; d[2] = base + 2; d[3] = base + 3;
    } else {
        const int base = c4 * (D / 4) + (st >> 1) * 8 + (st & 1) * 2;      // nibbles 2 (st & 1) and + 4; then + 1 and + 5
        d[0] = base; d[1] = base + 4; d[2] = base + 1; d[3] = base + 5;
    }
}
