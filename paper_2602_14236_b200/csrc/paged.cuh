// Device-side view of the paged cache, shared by its store (paged.cu) and its attention (paged_attend*.cu).
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "common.cuh"

// The 16-bit types.  Both kinds of arithmetic below are the plain IEEE operations of the type.
struct TypeF16 {
    using pair = __half2;
    static __device__ __forceinline__ float lo(uint32_t w) { return __half2float(__ushort_as_half((unsigned short)(w & 0xffffu))); }
    static __device__ __forceinline__ float hi(uint32_t w) { return __half2float(__ushort_as_half((unsigned short)(w >> 16))); }
    static __device__ __forceinline__ uint32_t pack(float a, float b) {           // (a, b) rounded, a in the low half
        __half2 h = __floats2half2_rn(a, b);
        return *reinterpret_cast<uint32_t*>(&h);
    }
    static __device__ __forceinline__ uint16_t round(float a) { return __half_as_ushort(__float2half_rn(a)); }
    static constexpr uint32_t ONE = 0x3c00u, NORMAL = 0x0400u, NOT_A_NUMBER = 0x7e00u;      // 1, the smallest normal number
};
struct TypeBF16 {
    using pair = __nv_bfloat162;
    static __device__ __forceinline__ float lo(uint32_t w) { return __uint_as_float(w << 16); }
    static __device__ __forceinline__ float hi(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }
    static __device__ __forceinline__ uint32_t pack(float a, float b) {
        __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
        return *reinterpret_cast<uint32_t*>(&h);
    }
    static __device__ __forceinline__ uint16_t round(float a) { return __bfloat16_as_ushort(__float2bfloat16_rn(a)); }
    static constexpr uint32_t ONE = 0x3f80u, NORMAL = 0x0080u, NOT_A_NUMBER = 0x7fc0u;
};
template <typename T>
__device__ __forceinline__ typename T::pair as_pair(uint32_t w) { return *reinterpret_cast<typename T::pair*>(&w); }
template <typename P>
__device__ __forceinline__ uint32_t as_word(P p) { return *reinterpret_cast<uint32_t*>(&p); }

constexpr int PF_16 = 0, PF_I8 = 1, PF_I4 = 2;      // page formats as template arguments

struct PgCache {
    uint8_t* data;
    uint8_t* scale;
    int n_pages, page_shift, heads;
};
struct PgSeqs {
    const int* start;
    const int* len;
    const int* table;
    int n_seqs, width, n_rows;
};

inline PgCache pg_cache(const salicache_pages* p) {
    int shift = 4;
    while ((1 << shift) < p->page) ++shift;
    return PgCache{(uint8_t*)p->d_data, (uint8_t*)p->d_scale, p->n_pages, shift, p->heads};
}
inline PgSeqs pg_seqs(const salicache_seqs* q) {
    return PgSeqs{q->d_row_start, q->d_len, q->d_table, q->n_seqs, q->table_width, q->n_rows};
}

// Bytes of one token's head in the pages, and of its scale (and zero).
template <int FMT, int D> __host__ __device__ constexpr int pg_row_bytes() { return FMT == PF_16 ? 2 * D : FMT == PF_I8 ? D : D / 2; }
template <int FMT> __host__ __device__ constexpr int pg_meta_bytes() { return FMT == PF_16 ? 0 : FMT == PF_I8 ? 2 : 4; }

// Slot index of (page id, K or V, head, slot): times pg_row_bytes it is the byte offset in `data`, times pg_meta_bytes in
// `scale`.  64 bits: a long cache passes 2^32 bytes.
__device__ __forceinline__ size_t pg_slot(const PgCache& c, int pid, int kv, int head, int slot) {
    return (((size_t)pid * 2 + kv) * c.heads + head << c.page_shift) + slot;
}

// Rows and positions of a sequence, clamped so that no offset the device finds reaches outside the caller's arrays.
struct PgSeq {
    int row0, n;        // first row in the caller's arrays, rows
    int pos0;           // position of row 0 (may be negative)
    int len;            // positions held, without those past the table
    bool cut;           // some lie past the table
};
__device__ __forceinline__ PgSeq pg_seq(const PgSeqs& s, const PgCache& c, int b) {
    PgSeq r;
    const int a = min(max(s.start[b], 0), s.n_rows), e = min(max(s.start[b + 1], a), s.n_rows);
    const int len = max(s.len[b], 0);
    const long long cap = min((long long)s.width << c.page_shift, 1ll << 30);        // sums of positions stay within 32 bits
    r.row0 = a;
    r.n = e - a;
    r.pos0 = len - r.n;
    r.cut = len > cap;
    r.len = (int)min((long long)len, cap);
    return r;
}

// (a & B) | c in one instruction, which takes one literal: c has to be in a register.
template <uint32_t B>
__device__ __forceinline__ uint32_t and_or(uint32_t a, uint32_t c) {
    uint32_t d;
    asm("lop3.b32 %0, %1, %2, %3, 0xEA;" : "=r"(d) : "r"(a), "n"(B), "r"(c));
    return d;
}
// A constant that the compiler does not know, so that it stays in its register.
template <uint32_t C>
__device__ __forceinline__ uint32_t held() {
    uint32_t d;
    asm volatile("mov.b32 %0, %1;" : "=r"(d) : "n"(C));
    return d;
}
// Codes to the 16-bit type: OR-ed into the mantissa of a power of two whose last place is 1 (f16: 1024, bf16: 128; for a
// nibble one place up, f16: 64), a code adds exactly its value; the power is then subtracted.
template <typename T>
struct Codes;
template <>
struct Codes<TypeF16> {
    uint32_t k1024 = held<0x64006400u>(), k64 = held<0x54005400u>(), k1152 = held<0x64806480u>();
    static __device__ __forceinline__ uint32_t sub(uint32_t a, uint32_t b) { return as_word(__hsub2(as_pair<TypeF16>(a), as_pair<TypeF16>(b))); }
    // two signed bytes of w (whose places PRMT's selector names, with the constant's byte above each)
    __device__ __forceinline__ uint32_t bytes(uint32_t w, uint32_t sel) const {
        return sub(__byte_perm(w ^ 0x80808080u, 0x64646464u, sel), k1152);
    }
    __device__ __forceinline__ uint32_t nib_lo(uint32_t x) const { return sub(and_or<0x000f000fu>(x, k1024), k1024); }
    __device__ __forceinline__ uint32_t nib_hi(uint32_t x) const { return sub(and_or<0x00f000f0u>(x, k64), k64); }
};
template <>
struct Codes<TypeBF16> {
    uint32_t k128 = held<0x43004300u>();
    static __device__ __forceinline__ uint32_t sub(uint32_t a, uint32_t b) { return as_word(__hsub2(as_pair<TypeBF16>(a), as_pair<TypeBF16>(b))); }
    // seven bits fit the mantissa of 128; the sign bit (-128) goes into the other operand, 256 instead of 128
    __device__ __forceinline__ uint32_t bytes(uint32_t w, uint32_t sel) const {
        const uint32_t h = __byte_perm(w, 0u, sel);
        return sub(and_or<0x007f007fu>(h, k128), and_or<0x00800080u>(h, k128));
    }
    __device__ __forceinline__ uint32_t nib_lo(uint32_t x) const { return sub(and_or<0x000f000fu>(x, k128), k128); }
    __device__ __forceinline__ uint32_t nib_hi(uint32_t x) const { return nib_lo(x >> 4); }
};
template <typename T>
__device__ __forceinline__ uint32_t mul2(uint32_t a, uint32_t s) { return as_word(__hmul2(as_pair<T>(a), as_pair<T>(s))); }
template <typename T>
__device__ __forceinline__ uint32_t fma2(uint32_t a, uint32_t s, uint32_t z) { return as_word(__hfma2(as_pair<T>(a), as_pair<T>(s), as_pair<T>(z))); }
__device__ __forceinline__ uint32_t dup_lo(uint32_t w) { return __byte_perm(w, 0, 0x1010); }
__device__ __forceinline__ uint32_t dup_hi(uint32_t w) { return __byte_perm(w, 0, 0x3232); }

__device__ __forceinline__ float ex2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
