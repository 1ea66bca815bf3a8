// Attention of new rows over the paged cache (Eq. 2 with the dequantisation of Sec. III-C fused in).
//
//   a_j = scale q . K^_j over the visible j,  m = max_j a_j,  l = sum_j e^(a_j - m),  out = sum_j e^(a_j - m) V^_j / l
//
// This file: few rows per sequence (single tokens, short drafts), where reading the pages is the work.
//
// A warp takes 16 keys of one head at a time, and both products are m16n8k16 matrix instructions with the keys as the
// long side, since there are few rows: scores = K (16 keys x 16 dimensions) times up to 8 rows of q as columns; values =
// V transposed (16 dimensions x 16 keys) times the weights, transposed in registers by movmatrix.  Any order of the
// dimensions that q and K share will do, as will any that V and the output share, so a lane loads 16 contiguous bytes
// wherever the rows have them, straight into the registers that hold its operands; codes become the 16-bit type there.
// The next tile's K is requested as soon as this tile's K is used up, V likewise.
// The weights' reference maximum moves only when a score exceeds it by 2^8 (in powers of two): until then no lane needs
// another's, weights stay below 2^8, and the sums are joined across lanes once at the end of an item.
#include <math.h>

#include "paged_plan.cuh"

namespace {

constexpr int ST_WARPS = 8, ST_THREADS = 32 * ST_WARPS;
static_assert(ST_WARPS * 16 == PT_KEYS, "a warp per 16 keys of a tile");

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
__device__ __forceinline__ uint32_t transpose8(uint32_t x) {
    uint32_t d;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(d) : "r"(x));
    return d;
}
template <int W>
__device__ __forceinline__ void ld_words(uint32_t* d, const uint8_t* p) {
    if (W == 4) asm volatile("ld.global.nc.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(d[0]), "=r"(d[1]), "=r"(d[2]), "=r"(d[3]) : "l"(p));
    if (W == 2) asm volatile("ld.global.nc.L1::no_allocate.v2.u32 {%0,%1}, [%2];" : "=r"(d[0]), "=r"(d[1]) : "l"(p));
    if (W == 1) asm volatile("ld.global.nc.L1::no_allocate.u32 %0, [%1];" : "=r"(d[0]) : "l"(p));
}

// What a lane (g8 = lane / 4, c4 = lane % 4) holds of 16 keys: the shares of rows g8 and g8 + 8 of K that make its A
// fragments, and its share of rows 2 c4, 2 c4 + 1, 2 c4 + 8, 2 c4 + 9 of V.
template <int FMT, int D>
struct KTile {
    static constexpr int W = pg_row_bytes<FMT, D>() / 16;       // words of a key row per lane
    uint32_t k[2][W];
    uint32_t s[2];                                              // scale, or (scale, zero)
    __device__ __forceinline__ void load(const PgCache& pc, size_t slot, int g8, int c4) {
        constexpr int RB = pg_row_bytes<FMT, D>();
#pragma unroll
        for (int r = 0; r < 2; ++r) {
            const size_t row = slot + g8 + 8 * r;
            const uint8_t* p = pc.data + row * RB;
            if (RB >= 64) {
#pragma unroll
                for (int i = 0; i < RB / 64; ++i) ld_words<4>(&k[r][4 * i], p + 64 * i + 16 * c4);
            } else ld_words<2>(&k[r][0], p + 8 * c4);
            if (FMT == PF_I8) s[r] = __ldg(reinterpret_cast<const uint16_t*>(pc.scale) + row);
            if (FMT == PF_I4) s[r] = __ldg(reinterpret_cast<const uint32_t*>(pc.scale) + row);
        }
    }
};
template <int FMT, int D>
struct VTile {
    static constexpr int W = pg_row_bytes<FMT, D>() / 32;       // words of a value row per lane
    uint32_t v[4][W];
    uint32_t s[2][FMT == PF_I4 ? 2 : 1];                        // per pair of keys: the scales (and zeros), key order
    __device__ __forceinline__ void load(const PgCache& pc, size_t slot, int g8, int c4) {
        constexpr int RB = pg_row_bytes<FMT, D>();
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const uint8_t* p = pc.data + (slot + 2 * c4 + (j & 1) + 8 * (j >> 1)) * RB;
            if (W == 8) {
                ld_words<4>(&v[j][0], p + 16 * g8);
                ld_words<4>(&v[j][4], p + 128 + 16 * g8);
            } else ld_words<W == 8 ? 4 : W>(&v[j][0], p + 4 * W * g8);
        }
#pragma unroll
        for (int r = 0; r < 2; ++r) {
            const size_t row = slot + 2 * c4 + 8 * r;
            if (FMT == PF_I8) s[r][0] = __ldg(reinterpret_cast<const uint32_t*>(pc.scale + row * 2));
            if (FMT == PF_I4) {
                const uint2 x = __ldg(reinterpret_cast<const uint2*>(pc.scale + row * 4));
                s[r][0] = x.x;
                s[r][FMT == PF_I4 ? 1 : 0] = x.y;
            }
        }
    }
};

// K fragments of matrix instruction st: registers (a0, a2) of one key row.
template <typename T, int FMT, int D>
__device__ __forceinline__ void key_frag(const uint32_t (&k)[KTile<FMT, D>::W], uint32_t s, int st, uint32_t& x, uint32_t& y) {
    if (FMT == PF_16) {
        x = k[2 * st];
        y = k[2 * st + 1];
    } else if (FMT == PF_I8) {
        const uint32_t s2 = dup_lo(s);
        x = mul2<T>(Codes<T>::bytes(k[st], 0x5140), s2);
        y = mul2<T>(Codes<T>::bytes(k[st], 0x5342), s2);
    } else {
        const uint32_t s2 = dup_lo(s), z2 = dup_hi(s), w = k[st >> 1] >> (8 * (st & 1));
        x = fma2<T>(Codes<T>::nib_lo(w), s2, z2);
        y = fma2<T>(Codes<T>::nib_hi(w), s2, z2);
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
// V fragments of dimension tile t: rows g8 (half 0) and g8 + 8 (half 1) of V transposed, key pairs 0 and 1.
template <typename T, int FMT, int D>
__device__ __forceinline__ uint32_t value_frag(const VTile<FMT, D>& v, int t, int half, int pair) {
    constexpr int NT = D / 16;
    const int x = half * NT + t;                        // which of the lane's D / 8 dimensions
    const uint32_t *A = v.v[2 * pair], *B = v.v[2 * pair + 1];
    if (FMT == PF_16) return __byte_perm(A[x >> 1], B[x >> 1], (x & 1) ? 0x7632 : 0x5410);
    if (FMT == PF_I8) {
        const uint32_t ab = __byte_perm(A[x >> 2], B[x >> 2], (x & 2) ? 0x7632 : 0x5410);      // bytes A, A+1, B, B+1
        return mul2<T>(Codes<T>::bytes(ab, (x & 1) ? 0x5341 : 0x5240), v.s[pair][0]);
    }
    const uint32_t ab = __byte_perm(A[x >> 3], B[x >> 3], (x & 4) ? 0x7632 : 0x5410);          // 4 nibbles of A, 4 of B
    const uint32_t w = (x & 2) ? ab >> 8 : ab;
    const uint32_t s2 = __byte_perm(v.s[pair][0], v.s[pair][FMT == PF_I4 ? 1 : 0], 0x5410);
    const uint32_t z2 = __byte_perm(v.s[pair][0], v.s[pair][FMT == PF_I4 ? 1 : 0], 0x7632);
    return fma2<T>((x & 1) ? Codes<T>::nib_hi(w) : Codes<T>::nib_lo(w), s2, z2);
}
template <int FMT, int D>
__device__ __forceinline__ int value_dim(int t, int half, int g8) {
    if (FMT == PF_16 && D == 128) return 64 * half + 8 * g8 + t;
    return g8 * (D / 8) + half * (D / 16) + t;
}

// Blocks per SM: two where the registers allow it.
template <int FMT, int D, int NT> constexpr int st_blocks() { return NT == 1 && !(FMT == PF_16 && D == 128) ? 2 : 1; }

// NT: 8-row column tiles per item.
template <typename T, int FMT, int D, int NT>
__global__ void __launch_bounds__(ST_THREADS, st_blocks<FMT, D, NT>())
k_paged_step(PtArgs a, int blocks) {
    constexpr int RT = 8 * NT, KS = D / 16, VS = D / 16;
    __shared__ float sh_acc[ST_WARPS][8][D + 4];
    __shared__ float2 sh_stat[ST_WARPS][8];
    const int lane = threadIdx.x & 31, wid = threadIdx.x >> 5, g8 = lane >> 2, c4 = lane & 3;
    const int c = blockIdx.x;
    PtWalk w = pt_start<RT, ST_THREADS, 0>(a, c, blocks);
    int4 hd = make_int4(0, 0, 0, 0);
    PgSeq s;
    if (w.left > 0) s = pg_seq(a.sq, a.pc, w.b);
    while (w.left > 0) {
        const PtSpan sp = pt_item<RT>(s, a, w.rt);
        const int k0 = w.k, k1 = (int)min((long long)max(sp.n, 1), k0 + w.left);
        const int rows = min(RT, s.n * a.G - w.rt * RT);
        const int* table = a.sq.table + (size_t)w.b * a.sq.width;
        if (s.cut && threadIdx.x == 0 && s.pos0 + s.n > s.len) atomicMin(a.status, SALICACHE_E_CAPACITY);

        // q as B fragments: column g8 of column tile n is row 8 n + g8
        uint32_t qf[NT][KS][2];
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            const int r = 8 * n + g8, rr = w.rt * RT + r;
            const bool in = r < rows;
            const uint16_t* src = a.q + (long long)(s.row0 + (in ? rr / a.G : 0)) * a.q_stride + (long long)(w.h * a.G + (in ? rr % a.G : 0)) * D;
#pragma unroll
            for (int st = 0; st < KS; ++st) {
                int d[4];
                q_dims<FMT>(st, c4, D, d);
                uint32_t x0 = 0, x1 = 0;
                if (in) {
                    if (FMT == PF_I4) {
                        x0 = src[d[0]] | (uint32_t)src[d[1]] << 16;
                        x1 = src[d[2]] | (uint32_t)src[d[3]] << 16;
                    } else {
                        x0 = *reinterpret_cast<const uint32_t*>(src + d[0]);
                        x1 = *reinterpret_cast<const uint32_t*>(src + d[2]);
                    }
                }
                qf[n][st][0] = x0;
                qf[n][st][1] = x1;
            }
        }
        float acc[NT][VS][4], m[NT][2], l[NT][2];
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            m[n][0] = m[n][1] = PT_NONE;
            l[n][0] = l[n][1] = 0.0f;
#pragma unroll
            for (int t = 0; t < VS; ++t) acc[n][t][0] = acc[n][t][1] = acc[n][t][2] = acc[n][t][3] = 0.0f;
        }

        // page of this warp's 16 keys of tile k: -2 behind the last position, -1 no such page
        auto page_of = [&](int k) -> int {
            if (k >= k1 || k >= sp.n) return -2;
            const int j = sp.tile(k) * PT_KEYS + wid * 16;
            if (j >= sp.hi || (j + 16 <= sp.lo && j >= a.sinks)) return -2;
            const int p = table[j >> a.pc.page_shift];
            return p >= 0 && p < a.pc.n_pages ? p : -1;
        };
        auto slot_of = [&](int k, int pid, int kv) -> size_t {
            const int j = sp.tile(k) * PT_KEYS + wid * 16;
            return pg_slot(a.pc, pid, kv, w.h, j & ((1 << a.pc.page_shift) - 1));
        };
        KTile<FMT, D> kt;
        VTile<FMT, D> vt;
        int pid = page_of(k0), pid1 = page_of(k0 + 1);
        if (pid >= 0) {
            kt.load(a.pc, slot_of(k0, pid, 0), g8, c4);
            vt.load(a.pc, slot_of(k0, pid, 1), g8, c4);
        }
        for (int k = k0; k < k1; ++k) {
            const int pid2 = page_of(k + 2);
            const int j0 = sp.tile(k) * PT_KEYS + wid * 16;
            float sc[NT][4];
            if (pid >= 0) {
#pragma unroll
                for (int n = 0; n < NT; ++n) sc[n][0] = sc[n][1] = sc[n][2] = sc[n][3] = 0.0f;
#pragma unroll
                for (int st = 0; st < KS; ++st) {
                    uint32_t a0, a1, a2, a3;
                    key_frag<T, FMT, D>(kt.k[0], kt.s[0], st, a0, a2);
                    key_frag<T, FMT, D>(kt.k[1], kt.s[1], st, a1, a3);
#pragma unroll
                    for (int n = 0; n < NT; ++n) mma16816<T>(sc[n], a0, a1, a2, a3, qf[n][st][0], qf[n][st][1]);
                }
            } else if (pid == -1 && lane == 0) atomicMin(a.status, SALICACHE_E_CAPACITY);
            if (pid1 >= 0) kt.load(a.pc, slot_of(k + 1, pid1, 0), g8, c4);
            if (pid >= 0) {
                // scores in powers of two; sc[n][i]: key g8 + 8 (i >> 1), row 8 n + 2 c4 + (i & 1)
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int i = 0; i < 4; ++i) sc[n][i] *= a.scale;
                const bool whole = j0 + 16 <= sp.all_hi && (j0 >= sp.all_lo || j0 + 16 <= a.sinks);
                if (!whole) {
#pragma unroll
                    for (int n = 0; n < NT; ++n)
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const int j = j0 + g8 + 8 * (i >> 1), rr = w.rt * RT + 8 * n + 2 * c4 + (i & 1);
                            if (j >= s.len || !pt_sees(s.pos0 + rr / a.G, j, a.window, a.sinks)) sc[n][i] = -INFINITY;
                        }
                    // values that no row sees may be anything: keep them out of the product
#pragma unroll
                    for (int x = 0; x < 4; ++x) {
                        const int j = j0 + 2 * c4 + (x & 1) + 8 * (x >> 1);
                        if (j >= sp.hi || (j < sp.lo && j >= a.sinks)) {
#pragma unroll
                            for (int i = 0; i < VTile<FMT, D>::W; ++i) vt.v[x][i] = 0u;
                            if (FMT == PF_I8) vt.s[x >> 1][0] &= (x & 1) ? 0x0000ffffu : 0xffff0000u;
                            if (FMT == PF_I4) vt.s[x >> 1][(x & 1) && FMT == PF_I4 ? 1 : 0] = 0u;
                        }
                    }
                }
                uint32_t pf[NT][2];
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                    const float x0 = fmaxf(sc[n][0], sc[n][2]), x1 = fmaxf(sc[n][1], sc[n][3]);
                    if (__any_sync(0xffffffffu, x0 > m[n][0] + 8.0f || x1 > m[n][1] + 8.0f)) {
                        float y[2] = {x0, x1};
#pragma unroll
                        for (int i = 0; i < 2; ++i) {
#pragma unroll
                            for (int o = 4; o < 32; o <<= 1) y[i] = fmaxf(y[i], __shfl_xor_sync(0xffffffffu, y[i], o));
                            y[i] = fmaxf(y[i], m[n][i]);
                            const float f = ex2(m[n][i] - y[i]);
                            m[n][i] = y[i];
                            l[n][i] *= f;
#pragma unroll
                            for (int t = 0; t < VS; ++t) {
                                acc[n][t][i] *= f;
                                acc[n][t][2 + i] *= f;
                            }
                        }
                    }
                    float p[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) p[i] = ex2(sc[n][i] - m[n][i & 1]);
                    l[n][0] += p[0] + p[2];
                    l[n][1] += p[1] + p[3];
                    pf[n][0] = transpose8(T::pack(p[0], p[1]));
                    pf[n][1] = transpose8(T::pack(p[2], p[3]));
                }
#pragma unroll
                for (int t = 0; t < VS; ++t) {
                    const uint32_t a0 = value_frag<T, FMT, D>(vt, t, 0, 0), a1 = value_frag<T, FMT, D>(vt, t, 1, 0);
                    const uint32_t a2 = value_frag<T, FMT, D>(vt, t, 0, 1), a3 = value_frag<T, FMT, D>(vt, t, 1, 1);
#pragma unroll
                    for (int n = 0; n < NT; ++n) mma16816<T>(acc[n][t], a0, a1, a2, a3, pf[n][0], pf[n][1]);
                }
            }
            if (pid1 >= 0) vt.load(a.pc, slot_of(k + 1, pid1, 1), g8, c4);
            pid = pid1;
            pid1 = pid2;
        }

        // join the warps: acc[n][t][i] is dimension value_dim(t, i >> 1), row 8 n + 2 c4 + (i & 1)
        const bool first = k0 == 0, lastp = k1 == max(sp.n, 1), done = first && lastp;
        const size_t slot = 2 * (size_t)c + (first ? 1 : 0);
#pragma unroll
        for (int n = 0; n < NT; ++n) {
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int o = 4; o < 32; o <<= 1) l[n][i] += __shfl_xor_sync(0xffffffffu, l[n][i], o);
            if (g8 == 0) {
                sh_stat[wid][2 * c4] = make_float2(m[n][0], l[n][0]);
                sh_stat[wid][2 * c4 + 1] = make_float2(m[n][1], l[n][1]);
            }
#pragma unroll
            for (int t = 0; t < VS; ++t)
#pragma unroll
                for (int i = 0; i < 4; ++i) sh_acc[wid][2 * c4 + (i & 1)][value_dim<FMT, D>(t, i >> 1, g8)] = acc[n][t][i];
            __syncthreads();
            const int r = 8 * n + wid;                  // a warp per row
            if (r < rows) {
                float M = PT_NONE, L = 0.0f, o[D / 32];
#pragma unroll
                for (int x = 0; x < ST_WARPS; ++x) M = fmaxf(M, sh_stat[x][wid].x);
#pragma unroll
                for (int i = 0; i < D / 32; ++i) o[i] = 0.0f;
#pragma unroll
                for (int x = 0; x < ST_WARPS; ++x) {
                    const float2 st = sh_stat[x][wid];
                    const float f = ex2(st.x - M);
                    L += f * st.y;
#pragma unroll
                    for (int i = 0; i < D / 32; ++i) o[i] += f * sh_acc[x][wid][lane * (D / 32) + i];
                }
                if (done) {
                    const int rr = w.rt * RT + r, hq = w.h * a.G + rr % a.G;
                    const long long tok = s.row0 + rr / a.G;
                    const float inv = L > 0.0f ? 1.0f / L : 0.0f;
                    uint16_t* dst = a.out + tok * a.out_stride + (long long)hq * D + lane * (D / 32);
#pragma unroll
                    for (int i = 0; i < D / 32; i += 2) *reinterpret_cast<uint32_t*>(dst + i) = T::pack(o[i] * inv, o[i + 1] * inv);
                    if (a.lse && lane == 0) a.lse[tok * ((long long)a.pc.heads * a.G) + hq] = L > 0.0f ? (M + log2f(L)) * PT_LN2 : -INFINITY;
                } else {
                    float* dst = a.part + (slot * RT + r) * D + lane * (D / 32);
#pragma unroll
                    for (int i = 0; i < D / 32; ++i) dst[i] = o[i];
                    if (lane == 0) a.stat[slot * RT + r] = make_float2(M, L);
                }
            }
            __syncthreads();
        }
        if (!done) {
            if (first) {
                hd.y = w.h + 1;
                hd.z = w.b;
                hd.w = w.rt;
            } else hd.x = lastp ? 2 : 1;
        }
        w.left -= k1 - k0;
        if (w.left > 0) pt_next<RT>(w, s, a);
    }
    if (threadIdx.x == 0) a.head[c] = hd;
}

template <typename T, int FMT, int D, int NT>
int launch_step(salicache_ctx* c, PtArgs a, char* work, cudaStream_t st) {
    constexpr int RT = 8 * NT;
    // no more blocks than there can be tiles of work: rows of q times heads times the table's tiles
    const long long most = (long long)a.sq.n_rows * a.pc.heads * ((((long long)a.sq.width << a.pc.page_shift) + PT_KEYS - 1) / PT_KEYS);
    const int blocks = (int)max(1ll, min(min(most, (long long)PT_MAX_BLOCKS), (long long)c->sm_count * st_blocks<FMT, D, NT>()));
    a.part = reinterpret_cast<float*>(work);
    a.stat = reinterpret_cast<float2*>(a.part + (size_t)2 * blocks * RT * D);
    a.head = reinterpret_cast<int4*>(a.stat + (size_t)2 * blocks * RT);
    k_paged_step<T, FMT, D, NT><<<blocks, ST_THREADS, 0, st>>>(a, blocks);
    cudaLaunchConfig_t cfg{};
    cudaLaunchAttribute at{};
    at.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at.val.programmaticStreamSerializationAllowed = 1;
    cfg.gridDim = dim3(blocks, NT);
    cfg.blockDim = dim3(256);
    cfg.stream = st;
    cfg.attrs = &at;
    cfg.numAttrs = 1;
    SC_CHECK(cudaLaunchKernelEx(&cfg, k_paged_join<T, RT, D>, a, blocks));
    c->launches += 2;
    SC_CHECK(cudaGetLastError());
    return SALICACHE_OK;
}

template <typename T, int FMT, int D>
int launch_attend(salicache_ctx* c, const PtArgs& a, char* work, cudaStream_t st) {
    if ((long long)a.sq.n_rows * a.G <= 8ll * a.sq.n_seqs) return launch_step<T, FMT, D, 1>(c, a, work, st);
    return launch_step<T, FMT, D, 2>(c, a, work, st);
}

}  // namespace

int64_t sc_paged_work_bytes(const salicache_ctx* c, int head_dim) { return 2ll * c->sm_count * (256 * (head_dim + 2) * 4 + 16); }

int sc_paged_attend(salicache_ctx* c, const salicache_pages* pg, const salicache_seqs* q, const void* d_q, int64_t q_stride,
                    int q_per_kv, float softmax_scale, int window, int sinks, void* d_out, int64_t out_stride, float* d_lse,
                    void* d_work, cudaStream_t st) {
    PtArgs a{};
    a.pc = pg_cache(pg);
    a.sq = pg_seqs(q);
    a.q = (const uint16_t*)d_q;
    a.out = (uint16_t*)d_out;
    a.lse = d_lse;
    a.q_stride = q_stride;
    a.out_stride = out_stride;
    a.G = q_per_kv;
    a.window = min(window, 1 << 30);
    a.sinks = window ? sinks : 0;
    a.scale = softmax_scale * PT_LOG2E;
    a.status = c->d_status;
    char* work = (char*)d_work;
    if ((long long)a.sq.n_rows * a.G > 16ll * a.sq.n_seqs) return sc_paged_chunk(c, a, pg, work, st);
#define GO(T, F, D) return launch_attend<T, F, D>(c, a, work, st)
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
