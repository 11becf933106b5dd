// Attention of single tokens, drafted tokens in a row and drafted trees over a paged cache in bf16 or in 8 bits.
//
// This kernel is for tiles of up to 16 lines (rows x query heads of a KV head's group), where the read of the cache is the bound.
//   work        equal shares of the list of units (draft.cuh), two CTAs per SM; an item that several CTAs share is joined by the one
//               that finds all other pieces done, always in the list's order
//   data path   a producer warp walks the share and keeps a ring of stages filled with tiled TMA loads of whole pages (a page's K or V of
//               one KV head is a contiguous block), whose swizzle is what both kinds of reads want: K is read as (two rows) x (four chunks
//               of 16 bytes), V as (rows 0, 2, 4, 6 or 1, 3, 5, 7) x (two chunks), each without a bank conflict
//   arithmetic  mma.sync m16n8k16 with the 16 lines as rows: S = Q K^T, O += P V, operands made in registers from 16-byte reads (the order
//               of channels inside a product is free).  Codes of 8 bits become fp16 exactly: int8 + 128 under the exponent of 1024, less
//               1152; e4m3 by the hardware's conversion.  Queries are bf16, or fp16 after a power of two that brings the line's largest
//               entry to [2^14, 2^15).
//   softmax     online, fp32, base 2, each warp with its own running state.  Of an 8-bit cache the weight of a code is p_j * scale_j, so
//               the running reference follows s_j + log2 scale_j, the weights enter the product in fp16 below 2^15, and their sum is
//               taken of weight / scale.  A reference moves only when a score outgrows it by 2^7.  Of a bf16 cache the weights are the
//               sum of two bf16 values.
//   masks       only pages that hold drafted tokens look at one
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <math.h>

#include "draft.cuh"
#include "internal.h"
#include "ptx.cuh"
#include "rows.cuh"

namespace aflex {

namespace {

constexpr int kLines = 16;                         // of a tile
constexpr int kComputeWarps = 4;
constexpr int kDraftThreads = (kComputeWarps + 2) * 32;      // compute warps, producer, epilogue
constexpr int kStages = 3;

template <int D, int F> struct DraftStage {
    static constexpr int kBytes = F == AFLEX_CACHE_BF16 ? 2 : 1;      // of an element
    static constexpr int kRow = D * kBytes;                           // of a token's head
    static constexpr int kBlock = kPageTokens * kRow;                 // K or V of a page
    static constexpr int kPerWarp = F == AFLEX_CACHE_BF16 ? 1 : 2;    // pages per warp: their place holds the warp's state at the end
    static constexpr int kPages = kComputeWarps * kPerWarp;
    static constexpr int kTokens = kPages * kPageTokens;
    static constexpr int kScales = F == AFLEX_CACHE_BF16 ? 0 : 2 * kPageTokens * 4;      // bytes of a page's scales
    static constexpr int kSize = kPages * (2 * kBlock + kScales);
    static_assert(kPerWarp * 2 * kBlock >= kLines * D * 4, "the state has to fit");
    static_assert(kSize % 1024 == 0, "swizzled blocks are aligned to their pattern");
};

enum : int { kFirst = 1, kLast = 2, kEnd = 4 };    // first, last unit of a piece; end of the share

struct UnitMeta {
    int flags, t0, sees, ctx;      // first token of the unit, tokens the tile's rows may see, earlier tokens of the sequence
    int row0, lines, i0, m, g;     // first row and lines of the tile, number of the first row and of all rows in the sequence, KV head
    int item, slot, whole;
    long long first, last;         // positions of the item's first and last unit with tokens
};

struct __align__(8) DraftShared {
    uint64_t full[kStages], empty[kStages], parked[kStages];
    UnitMeta meta[kStages];
    float m[kStages][kComputeWarps][kLines], l[kStages][kComputeWarps][kLines];
    DraftShare share;
    int merges;                    // items that this CTA has to join at the end
    UnitMeta merge[2];
    volatile int abort;
    int arrived;
};

__device__ __forceinline__ uint4 lds128(uint32_t addr) {
    uint4 v;
    asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(addr) : "memory");
    return v;
}
__device__ __forceinline__ uint2 lds64(uint32_t addr) {
    uint2 v;
    asm volatile("ld.shared.v2.u32 {%0, %1}, [%2];" : "=r"(v.x), "=r"(v.y) : "r"(addr) : "memory");
    return v;
}

// Byte offset of a token's 16-byte chunk inside a page's K or V block, as the tiled copies write it.
template <int kRow> __device__ __forceinline__ uint32_t chunk_at(int t, int ch) {
    if (kRow == 256) return (uint32_t)((ch >> 3) * (kPageTokens * 128) + t * 128 + (((ch & 7) ^ (t & 7)) << 4));
    if (kRow == 128) return (uint32_t)(t * 128 + ((ch ^ (t & 7)) << 4));
    return (uint32_t)(t * 64 + ((ch ^ ((t >> 1) & 3)) << 4));
}

// Four codes as two pairs of fp16, exactly.
template <int F> __device__ __forceinline__ void widen4(uint32_t w, uint32_t& lo, uint32_t& hi) {
    if (F == AFLEX_CACHE_INT8) {
        w ^= 0x80808080u;
        const __half2 off = __halves2half2(__ushort_as_half(0x6480), __ushort_as_half(0x6480));      // 1024 + 128
        const uint32_t a = __byte_perm(w, 0x64646464u, 0x4140), b = __byte_perm(w, 0x64646464u, 0x4342);
        const __half2 x = __hsub2(*reinterpret_cast<const __half2*>(&a), off), y = __hsub2(*reinterpret_cast<const __half2*>(&b), off);
        lo = *reinterpret_cast<const uint32_t*>(&x);
        hi = *reinterpret_cast<const uint32_t*>(&y);
    } else {
        asm("{\n\t.reg .b16 a, b;\n\tmov.b32 {a, b}, %2;\n\tcvt.rn.f16x2.e4m3x2 %0, a;\n\tcvt.rn.f16x2.e4m3x2 %1, b;\n\t}" : "=r"(lo), "=r"(hi) : "r"(w));
    }
}

template <int F>
__device__ __forceinline__ void mma_16816(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    if (F == AFLEX_CACHE_BF16) mma_bf16_16816(d, a[0], a[1], a[2], a[3], b0, b1);
    else mma_f16_16816(d, a[0], a[1], a[2], a[3], b0, b1);
}

template <int D> struct LineState {                // of a warp: lines lane / 4 and lane / 4 + 8
    float o[D / 8][4];
    float m[2], l[2];
    uint32_t q[D / 16][4];
    float c[2];                                    // what a product counts, in log2 units
    __device__ __forceinline__ void reset() {
#pragma unroll
        for (int i = 0; i < D / 8; ++i) o[i][0] = o[i][1] = o[i][2] = o[i][3] = 0.f;
        m[0] = m[1] = kLowest;
        l[0] = l[1] = 0.f;
    }
};

// Chunk c of a lane's part of a K row (or of a query).
template <int kRow> __device__ __forceinline__ int k_chunk(int c, int l4) { return kRow == 256 ? (c >> 1) * 8 + 2 * l4 + (c & 1) : kRow == 128 ? 2 * l4 + c : l4; }

template <int D, int F>
__device__ __forceinline__ void load_queries(LineState<D>& st, const DraftParams& p, const UnitMeta& u) {
    typedef DraftStage<D, F> S;
    const int lane = threadIdx.x & 31, hl = lane >> 2, l4 = lane & 3;
#pragma unroll
    for (int x = 0; x < 2; ++x) {
        const int line = hl + 8 * x;
        const bool there = line < u.lines;
        const uint4* src = reinterpret_cast<const uint4*>(p.q + ((size_t)(u.row0 + (there ? line / p.G : 0)) * p.Hq + (size_t)u.g * p.G + (there ? line % p.G : 0)) * D);
        if (F == AFLEX_CACHE_BF16) {
#pragma unroll
            for (int c = 0; c < S::kRow / 64; ++c) {
                uint4 v = fetch(src + k_chunk<S::kRow>(c, l4));
                if (!there) v = make_uint4(0, 0, 0, 0);
                st.q[2 * c][x] = v.x; st.q[2 * c][2 + x] = v.y;
                st.q[2 * c + 1][x] = v.z; st.q[2 * c + 1][2 + x] = v.w;
            }
            st.c[x] = p.scale_log2;
        } else {
            uint32_t v[D / 8], big = 0;            // this lane's quarter of the line
#pragma unroll
            for (int c = 0; c < S::kRow / 64; ++c) {
                const int ch = k_chunk<S::kRow>(c, l4);
                uint4 a = fetch(src + 2 * ch), b = fetch(src + 2 * ch + 1);
                if (!there) a = b = make_uint4(0, 0, 0, 0);
                v[8 * c] = a.x; v[8 * c + 1] = a.y; v[8 * c + 2] = a.z; v[8 * c + 3] = a.w;
                v[8 * c + 4] = b.x; v[8 * c + 5] = b.y; v[8 * c + 6] = b.z; v[8 * c + 7] = b.w;
            }
#pragma unroll
            for (int i = 0; i < D / 8; ++i) big = __vmaxu2(big, v[i] & 0x7fff7fffu);
            big = max(big & 0xffffu, big >> 16);
            big = max(big, __shfl_xor_sync(0xffffffffu, big, 1));
            big = max(big, __shfl_xor_sync(0xffffffffu, big, 2));
            // largest in [2^e, 2^(e + 1)): times 2^(14 - e); tiny lines by 2^126
            const int e = max((int)(big >> 7) - 127, -112);
            const float up = __uint_as_float((uint32_t)(127 + 14 - e) << 23);
            st.c[x] = big >= 0x7f80u ? __uint_as_float(0x7fc00000u) : p.scale_log2 * __uint_as_float((uint32_t)(127 - 14 + e) << 23);
#pragma unroll
            for (int i = 0; i < D / 8; ++i) {
                const __half2 h = __floats2half2_rn(__uint_as_float(v[i] << 16) * up, __uint_as_float(v[i] & 0xffff0000u) * up);
                st.q[i / 2][(i & 1) * 2 + x] = *reinterpret_cast<const uint32_t*>(&h);
            }
        }
    }
}

// Whether drafted token j (negative: an earlier token) is seen by row i of its sequence.
__device__ __forceinline__ bool sees_drafted(const DraftParams& p, int row, int i, int j, int m) {
    if (j < 0) return true;
    if (j >= m) return false;
    if (p.mask == nullptr) return j <= i;
    return (j >> 5) < p.mask_words && ((fetch(p.mask + (size_t)row * p.mask_words + (j >> 5)) >> (j & 31)) & 1u);
}

// One page for one warp: K at shared address kp, V at vp, its scales at sp; tokens tp .. of the sequence.
template <int D, int F>
__device__ __forceinline__ void attend_page(LineState<D>& st, const DraftParams& p, const UnitMeta& u, uint32_t kp, uint32_t vp, uint32_t sp, int tp) {
    typedef DraftStage<D, F> S;
    constexpr int kRow = S::kRow;
    const int lane = threadIdx.x & 31, hl = lane >> 2, l4 = lane & 3;
    float s[2][4];
#pragma unroll
    for (int r = 0; r < 2; ++r) {
        s[r][0] = s[r][1] = s[r][2] = s[r][3] = 0.f;
#pragma unroll
        for (int c = 0; c < kRow / 64; ++c) {
            const uint4 x = lds128(kp + chunk_at<kRow>(hl + 8 * r, k_chunk<kRow>(c, l4)));
            if (F == AFLEX_CACHE_BF16) {
                mma_16816<F>(s[r], st.q[2 * c], x.x, x.y);
                mma_16816<F>(s[r], st.q[2 * c + 1], x.z, x.w);
            } else {
                const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    uint32_t lo, hi;
                    widen4<F>(w[k], lo, hi);
                    mma_16816<F>(s[r], st.q[4 * c + k], lo, hi);
                }
            }
        }
    }
    // scores in log2 units, of token 2 l4 + (k & 1) + 8 (k >> 1) for line hl at x[0][k], for line hl + 8 at x[1][k]
    float x[2][4], inv[4];                         // inv: 1 / scale of the token's V
#pragma unroll
    for (int r = 0; r < 2; ++r) {
        float ks[2] = {1.f, 1.f}, lv[2] = {0.f, 0.f};
        inv[2 * r] = inv[2 * r + 1] = 1.f;
        if (F != AFLEX_CACHE_BF16) {
            const uint2 a = lds64(sp + (uint32_t)(2 * l4 + 8 * r) * 4), b = lds64(sp + (uint32_t)(kPageTokens + 2 * l4 + 8 * r) * 4);
            ks[0] = __uint_as_float(a.x); ks[1] = __uint_as_float(a.y);
            const float vs[2] = {__uint_as_float(b.x), __uint_as_float(b.y)};
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                lv[e] = __log2f(vs[e]);
                if (lv[e] < -64.f) lv[e] = -64.f;  // (a scale of 0; NaN stays)
                inv[2 * r + e] = fast_exp2(-lv[e]);
            }
        }
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            x[0][2 * r + e] = fmaf(s[r][e] * st.c[0], ks[e], lv[e]);
            x[1][2 * r + e] = fmaf(s[r][2 + e] * st.c[1], ks[e], lv[e]);
        }
    }
    const bool partial = tp + kPageTokens > u.sees, masked = tp + kPageTokens > u.ctx;
    bool poison[2] = {false, false};
    uint32_t dead = 0;                             // bit k: nothing of this lane's token k of V may enter the product
    if (partial || masked) {
        if (F == AFLEX_CACHE_BF16 && masked) {
            // tokens whose V holds an infinity or NaN: they enter no product, which would carry it to lines that do not see them
            uint32_t odd = 0;
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const int t = 2 * l4 + (k & 1) + 8 * (k >> 1);
                bool o = false;
#pragma unroll
                for (int h = 0; h < D / 64; ++h) {
                    const uint4 v = lds128(vp + chunk_at<kRow>(t, 8 * h + hl));
                    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
                    for (int i = 0; i < 4; ++i) o = o || (w[i] & 0x7f80u) == 0x7f80u || (w[i] & 0x7f800000u) == 0x7f800000u;
                }
                if (o && tp + t < u.sees) odd |= 1u << k;
            }
            odd |= __shfl_xor_sync(0xffffffffu, odd, 4);
            odd |= __shfl_xor_sync(0xffffffffu, odd, 8);
            odd |= __shfl_xor_sync(0xffffffffu, odd, 16);
            dead = odd;
        }
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const int t = tp + 2 * l4 + (k & 1) + 8 * (k >> 1);
            if (t >= u.sees) dead |= 1u << k;
#pragma unroll
            for (int y = 0; y < 2; ++y) {
                const int i = (hl + 8 * y) / p.G;
                const bool see = t < u.sees && hl + 8 * y < u.lines && sees_drafted(p, u.row0 + i, u.i0 + i, t - u.ctx, u.m);
                if (see && (dead >> k & 1)) poison[y] = true;
                if (!see) x[y][k] = -INFINITY;
            }
        }
    }
    float mx[2];
#pragma unroll
    for (int y = 0; y < 2; ++y) {
        mx[y] = fmaxf(fmaxf(x[y][0], x[y][1]), fmaxf(x[y][2], x[y][3]));
        mx[y] = fmaxf(mx[y], __shfl_xor_sync(0xffffffffu, mx[y], 1));
        mx[y] = fmaxf(mx[y], __shfl_xor_sync(0xffffffffu, mx[y], 2));
    }
    // weights are 2^(x - m), m the running maximum less 8; they stay below 2^15 until a score is 2^15 times the reference
    if (__any_sync(0xffffffffu, mx[0] > st.m[0] + 15.f || mx[1] > st.m[1] + 15.f)) {
        float corr[2];
#pragma unroll
        for (int y = 0; y < 2; ++y) {
            const float mn = fmaxf(st.m[y], mx[y] - 8.f);
            corr[y] = fast_exp2(st.m[y] - mn);
            st.m[y] = mn;
            st.l[y] *= corr[y];
        }
#pragma unroll
        for (int i = 0; i < D / 8; ++i) { st.o[i][0] *= corr[0]; st.o[i][1] *= corr[0]; st.o[i][2] *= corr[1]; st.o[i][3] *= corr[1]; }
    }
#pragma unroll
    for (int y = 0; y < 2; ++y) {
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const bool hidden = (partial || masked) && x[y][k] == -INFINITY;
            x[y][k] = fast_exp2(x[y][k] - st.m[y]);
            st.l[y] += F == AFLEX_CACHE_BF16 ? x[y][k] : hidden ? 0.f : x[y][k] * inv[k];
        }
        if (poison[y]) st.l[y] = __uint_as_float(0x7fc00000u);
    }
    uint32_t a[4], b[4];                           // weights as the product's operand; bf16: the rest of them in b
    if (F == AFLEX_CACHE_BF16) {
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const float w0 = x[k & 1][k & 2], w1 = x[k & 1][(k & 2) + 1];
            a[k] = pack_bf16x2(w0, w1);
            b[k] = pack_bf16x2(w0 - __uint_as_float(a[k] << 16), w1 - __uint_as_float(a[k] & 0xffff0000u));
        }
    } else {
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const __half2 h = __floats2half2_rn(x[k & 1][k & 2], x[k & 1][(k & 2) + 1]);
            a[k] = *reinterpret_cast<const uint32_t*>(&h);
        }
    }
    if (F == AFLEX_CACHE_BF16) {
#pragma unroll
        for (int h = 0; h < D / 64; ++h) {
            uint4 v[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                v[k] = lds128(vp + chunk_at<kRow>(2 * l4 + (k & 1) + 8 * (k >> 1), 8 * h + hl));
                if (dead >> k & 1) v[k] = make_uint4(0, 0, 0, 0);
            }
            const uint32_t* r0 = reinterpret_cast<const uint32_t*>(&v[0]);
            const uint32_t* r1 = reinterpret_cast<const uint32_t*>(&v[1]);
            const uint32_t* r2 = reinterpret_cast<const uint32_t*>(&v[2]);
            const uint32_t* r3 = reinterpret_cast<const uint32_t*>(&v[3]);
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                const uint32_t e0 = __byte_perm(r0[w], r1[w], 0x5410), e1 = __byte_perm(r2[w], r3[w], 0x5410);
                const uint32_t f0 = __byte_perm(r0[w], r1[w], 0x7632), f1 = __byte_perm(r2[w], r3[w], 0x7632);
                mma_16816<F>(st.o[8 * h + 2 * w], a, e0, e1);
                mma_16816<F>(st.o[8 * h + 2 * w + 1], a, f0, f1);
                mma_16816<F>(st.o[8 * h + 2 * w], b, e0, e1);
                mma_16816<F>(st.o[8 * h + 2 * w + 1], b, f0, f1);
            }
        }
    } else {
        constexpr int kWords = D / 32;             // 32-bit words of a lane's chunk: 16 channels, or 8
        uint32_t v[4][kWords];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const int t = 2 * l4 + (k & 1) + 8 * (k >> 1);
            if (D == 128) {
                const uint4 r = lds128(vp + chunk_at<kRow>(t, hl));
                v[k][0] = r.x; v[k][1] = r.y; v[k][2 % kWords] = r.z; v[k][3 % kWords] = r.w;
            } else {
                const uint2 r = lds64(vp + chunk_at<kRow>(t, hl >> 1) + (uint32_t)(hl & 1) * 8);
                v[k][0] = r.x; v[k][1] = r.y;
            }
            if (dead >> k & 1)
#pragma unroll
                for (int w = 0; w < kWords; ++w) v[k][w] = 0;
        }
#pragma unroll
        for (int w = 0; w < kWords; ++w) {
            uint32_t b0[4], b1[4];
            widen4<F>(__byte_perm(v[0][w], v[1][w], 0x5140), b0[0], b0[1]);
            widen4<F>(__byte_perm(v[0][w], v[1][w], 0x7362), b0[2], b0[3]);
            widen4<F>(__byte_perm(v[2][w], v[3][w], 0x5140), b1[0], b1[1]);
            widen4<F>(__byte_perm(v[2][w], v[3][w], 0x7362), b1[2], b1[3]);
#pragma unroll
            for (int i = 0; i < 4; ++i) mma_16816<F>(st.o[4 * w + i], a, b0[i], b1[i]);
        }
    }
}

// First channel of the four that a lane holds at n-tiles i .. i + 3 (i a multiple of 4), of accumulator column e.
template <int D, int F> __device__ __forceinline__ int channel_of(int i, int e, int l4) {
    return F == AFLEX_CACHE_BF16 ? 64 * (i >> 3) + 8 * (2 * l4 + e) + (i & 7) : (D / 8) * (2 * l4 + e) + i;
}
// Place of four channels of a line in a parked state: neighbouring lines' words in other banks.
template <int D> __device__ __forceinline__ uint32_t parked_at(int line, int run) { return (uint32_t)(line * (D * 4) + ((run ^ (line & 7)) << 4)); }

template <int D, int F>
__device__ __forceinline__ void park(const LineState<D>& st, uint8_t* to, float* m_to, float* l_to) {
    const int lane = threadIdx.x & 31, hl = lane >> 2, l4 = lane & 3;
#pragma unroll
    for (int y = 0; y < 2; ++y) {
        float l = st.l[y];
        l += __shfl_xor_sync(0xffffffffu, l, 1);
        l += __shfl_xor_sync(0xffffffffu, l, 2);
#pragma unroll
        for (int i = 0; i < D / 8; i += 4)
#pragma unroll
            for (int e = 0; e < 2; ++e)
                *reinterpret_cast<float4*>(to + parked_at<D>(hl + 8 * y, channel_of<D, F>(i, e, l4) / 4)) =
                    make_float4(st.o[i][2 * y + e], st.o[i + 1][2 * y + e], st.o[i + 2][2 * y + e], st.o[i + 3][2 * y + e]);
        if (l4 == 0) { m_to[hl + 8 * y] = st.m[y]; l_to[hl + 8 * y] = l; }
    }
}

struct RunSum {
    float M, L;
    float4 acc;
};
__device__ __forceinline__ void add_piece(RunSum& s, float m, float l, const float4& v) {
    const float f = fast_exp2(m - s.M);            // (s.M: the largest m of all pieces)
    s.L = fmaf(l, f, s.L);
    s.acc.x = fmaf(v.x, f, s.acc.x); s.acc.y = fmaf(v.y, f, s.acc.y); s.acc.z = fmaf(v.z, f, s.acc.z); s.acc.w = fmaf(v.w, f, s.acc.w);
}
template <int D>
__device__ __forceinline__ void store_run(const DraftParams& p, const UnitMeta& u, int line, int c, const RunSum& s) {
    const float inv = s.L == 0.f ? 0.f : 1.f / s.L;            // a line with nothing to attend to: zeros
    const size_t hq = (size_t)(u.row0 + line / p.G) * p.Hq + (size_t)u.g * p.G + line % p.G;
    reinterpret_cast<uint2*>(p.out + hq * D)[c] = make_uint2(pack_bf16x2(s.acc.x * inv, s.acc.y * inv), pack_bf16x2(s.acc.z * inv, s.acc.w * inv));
    if (p.lse != nullptr && c == 0) p.lse[hq] = s.L == 0.f ? -INFINITY : (s.M + log2f(s.L)) * 0.6931471805599453f;
}

template <int D, int F>
__global__ void __launch_bounds__(kDraftThreads, 2)
attn_draft_kernel(const __grid_constant__ CUtensorMap tmap_k, const __grid_constant__ CUtensorMap tmap_v, const __grid_constant__ DraftParams p) {
    typedef DraftStage<D, F> S;
    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
    __shared__ DraftShared sh;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (threadIdx.x == 0) {
        for (int s = 0; s < kStages; ++s) {
            mbar_init(&sh.full[s], 1);
            mbar_init(&sh.empty[s], kComputeWarps + 1);
            mbar_init(&sh.parked[s], kComputeWarps);
        }
        sh.abort = 0;
        sh.merges = 0;
        fence_mbar_init();
        prefetch_tmap(&tmap_k);
        prefetch_tmap(&tmap_v);
    }
    pdl_launch_dependents();
    pdl_wait();
    const DraftList<S::kTokens> list(p);
    draft_plan<S::kTokens, kDraftThreads>(p, list, sh.share);
    const DraftShare share = sh.share;

    if (warp == kComputeWarps) {
        // ------------------------------------------------------------------ producer
        int it = 0;
        bool ok = true;
        auto slot_free = [&]() {                   // the next stage, once everybody has left it
            ok = mbar_wait(&sh.empty[it % kStages], ((it / kStages) & 1) ^ 1);
            ok = __all_sync(0xffffffffu, ok) && !sh.abort;
            return ok;
        };
        // lane: a page of the unit, K or V, and half of a row or the scales
        const int page = lane % S::kPages, kv = (lane / S::kPages) & 1, part = lane / (2 * S::kPages);
        const bool copies = lane < (F == AFLEX_CACHE_BF16 ? 2 * S::kPages * (S::kRow / 128) : 4 * S::kPages);
        DraftWalk<S::kTokens> w;
        if (share.x0 < share.x1) w.start(p, list, share.x0, share.seq, share.seq_first, share.seq_tiles);
        else w.pos = share.x1;
        while (ok && w.pos < share.x1) {
            if (w.u == 0 && w.nu > 1) { w.advance(p, list, 1, share.total); continue; }
            const int u0 = w.u, u1 = (int)min((long long)w.nu, w.u + (share.x1 - w.pos));       // (u0 = 0: an item without tokens)
            UnitMeta meta;
            meta.sees = list.sees(w.s, w.tile); meta.ctx = w.s.ctx;
            meta.i0 = w.tile * p.rpt; meta.row0 = w.s.o0 + meta.i0; meta.m = w.s.m; meta.g = w.g;
            meta.lines = min(p.rpt, w.s.m - meta.i0) * p.G;
            meta.item = w.id + w.g; meta.slot = u0 > 1 ? 0 : 1; meta.whole = u0 <= 1 && u1 == w.nu;
            meta.first = w.pos - u0 + 1; meta.last = w.pos - u0 + w.nu - 1;
            const int32_t* table = p.page_table + (size_t)w.b * p.max_pages;
            auto page_id = [&](int u) -> int {
                const int i = (u - 1) * S::kPages + page;
                return copies && u >= 1 && i * kPageTokens < meta.sees ? fetch(table + i) : 0;
            };
            int id = page_id(u0);
            for (int u = u0; u < u1; ++u, ++it) {
                const int id_next = u + 1 < u1 ? page_id(u + 1) : 0;
                if (!slot_free()) break;
                const int st = it % kStages;
                meta.t0 = (u - 1) * S::kTokens;
                meta.flags = (u == u0 ? kFirst : 0) | (u == u1 - 1 ? kLast : 0);
                const int np = u == 0 ? 0 : min(S::kPages, (meta.sees - meta.t0 + kPageTokens - 1) / kPageTokens);
                if (copies && page < np && (id < 0 || id >= p.num_pages)) { atomicExch(p.status, AFLEX_ERR_BOUNDS); id = 0; }
                if (lane == 0) {
                    sh.meta[st] = meta;
                    mbar_expect_tx(&sh.full[st], (uint32_t)(np * (2 * S::kBlock + S::kScales)));
                }
                __syncwarp();
                if (copies && page < np) {
                    uint8_t* stage = smem + st * S::kSize;
                    uint8_t* dst = stage + (page * 2 + kv) * S::kBlock;
                    const int slab = id * p.Hkv + w.g;
                    if (F == AFLEX_CACHE_BF16) tma_load_2d(dst + part * (kPageTokens * 128), kv ? &tmap_v : &tmap_k, part * 64, slab * kPageTokens, &sh.full[st]);
                    else if (part == 0) tma_load_2d(dst, kv ? &tmap_v : &tmap_k, 0, slab * kPageTokens, &sh.full[st]);
                    else bulk_load_1d(stage + S::kPages * 2 * S::kBlock + page * S::kScales + kv * (S::kScales / 2), (kv ? p.v_scales : p.k_scales) + (size_t)slab * kPageTokens,
                                      S::kScales / 2, &sh.full[st]);
                }
                id = id_next;
            }
            if (ok) w.advance(p, list, u1 - u0, share.total);
        }
        if (ok && slot_free()) {
            if (lane == 0) {
                sh.meta[it % kStages].flags = kEnd;
                mbar_arrive(&sh.full[it % kStages]);
            }
        }
        if (!ok && lane == 0) { sh.abort = 1; atomicExch(p.status, AFLEX_ERR_TIMEOUT); }
    } else if (warp < kComputeWarps) {
        // ------------------------------------------------------------------ compute
        LineState<D> st;
        for (int it = 0;; ++it) {
            const int stage = it % kStages;
            bool ok = mbar_wait(&sh.full[stage], (it / kStages) & 1);
            ok = __all_sync(0xffffffffu, ok) && !sh.abort;
            if (!ok) { if (lane == 0 && !sh.abort) { sh.abort = 1; atomicExch(p.status, AFLEX_ERR_TIMEOUT); } break; }
            const UnitMeta& u = sh.meta[stage];
            const int flags = u.flags;
            if (flags & kEnd) break;
            if (flags & kFirst) {
                st.reset();
                load_queries<D, F>(st, p, u);
            }
            uint8_t* base = smem + stage * S::kSize;
            uint8_t* mine = base + warp * S::kPerWarp * 2 * S::kBlock;
#pragma unroll
            for (int k = 0; k < S::kPerWarp; ++k) {
                const int page = warp * S::kPerWarp + k, tp = u.t0 + page * kPageTokens;
                const uint32_t kp = smem_u32(mine) + (uint32_t)(k * 2 * S::kBlock);
                if (tp < u.sees && tp >= 0)
                    attend_page<D, F>(st, p, u, kp, kp + S::kBlock, smem_u32(base) + (uint32_t)(S::kPages * 2 * S::kBlock + page * S::kScales), tp);
            }
            __syncwarp();
            if (flags & kLast) {
                park<D, F>(st, mine, sh.m[stage][warp], sh.l[stage][warp]);
                fence_proxy_async();               // (the stage's next copies come behind these stores)
                __syncwarp();
                if (lane == 0) mbar_arrive(&sh.parked[stage]);
            } else if (lane == 0) {
                mbar_arrive(&sh.empty[stage]);
            }
        }
    } else {
        // ------------------------------------------------------------------ epilogue: joins the warps of a piece
        constexpr int kRuns = D / 4;               // a line's outputs in runs of four channels
        uint32_t phases = 0;                       // of sh.parked
        for (int it = 0;; ++it) {
            const int stage = it % kStages;
            bool ok = mbar_wait(&sh.full[stage], (it / kStages) & 1);
            ok = __all_sync(0xffffffffu, ok) && !sh.abort;
            if (!ok) { if (lane == 0 && !sh.abort) { sh.abort = 1; atomicExch(p.status, AFLEX_ERR_TIMEOUT); } break; }
            const int flags = sh.meta[stage].flags;
            if (flags & kEnd) break;
            if (!(flags & kLast)) {
                if (lane == 0) mbar_arrive(&sh.empty[stage]);
                continue;
            }
            ok = mbar_wait(&sh.parked[stage], (phases >> stage) & 1);
            ok = __all_sync(0xffffffffu, ok) && !sh.abort;
            if (!ok) { if (lane == 0 && !sh.abort) { sh.abort = 1; atomicExch(p.status, AFLEX_ERR_TIMEOUT); } break; }
            phases ^= 1u << stage;
            const UnitMeta u = sh.meta[stage];
            const uint8_t* base = smem + stage * S::kSize;
            const size_t part = ((size_t)blockIdx.x * 2 + u.slot) * kLines;
            for (int i = lane; i < u.lines * kRuns; i += 32) {
                const int line = i / kRuns, c = i % kRuns;
                RunSum s = {kLowest, 0.f, make_float4(0.f, 0.f, 0.f, 0.f)};
#pragma unroll
                for (int w = 0; w < kComputeWarps; ++w) s.M = fmaxf(s.M, sh.m[stage][w][line]);
#pragma unroll
                for (int w = 0; w < kComputeWarps; ++w)
                    add_piece(s, sh.m[stage][w][line], sh.l[stage][w][line],
                              *reinterpret_cast<const float4*>(base + w * S::kPerWarp * 2 * S::kBlock + parked_at<D>(line, c)));
                if (u.whole) store_run<D>(p, u, line, c, s);
                else {
                    __stcg(reinterpret_cast<float4*>(p.o_part + (part + line) * D) + c, s.acc);
                    if (c == 0) __stcg(reinterpret_cast<float2*>(p.ml_part) + part + line, make_float2(s.M, s.L));
                }
            }
            fence_proxy_async();
            __syncwarp();
            if (lane == 0) mbar_arrive_n(&sh.empty[stage], kComputeWarps + 1);
            if (!u.whole) {
                // the last of the item's CTAs to get here joins the pieces
                __threadfence();
                __syncwarp();
                // (offsets that decrease could name more items than there are counters)
                if (u.item >= kAttnCounterCap) {
                    if (lane == 0) atomicExch(p.status, AFLEX_ERR_BOUNDS);
                } else if (lane == 0) {
                    const int pieces = draft_cta_of(u.last, share.total, share.ctas) - draft_cta_of(u.first, share.total, share.ctas) + 1;
                    if (atomicAdd(p.counters + u.item, 1) == pieces - 1) {
                        p.counters[u.item] = 0;
                        sh.merge[sh.merges++] = u;
                    }
                }
                __syncwarp();
            }
        }
    }
    __syncthreads();
    if (sh.abort || sh.merges == 0) return;
    __threadfence();
    for (int j = 0; j < sh.merges; ++j) {
        constexpr int kRuns = D / 4;
        const UnitMeta& u = sh.merge[j];
        const int c0 = draft_cta_of(u.first, share.total, share.ctas), c1 = draft_cta_of(u.last, share.total, share.ctas);
        for (int i = threadIdx.x; i < u.lines * kRuns; i += kDraftThreads) {
            const int line = i / kRuns, c = i % kRuns;
            auto part = [&](int cta) -> size_t { return ((size_t)cta * 2 + (cta == c0 ? 1 : 0)) * kLines + line; };
            RunSum s = {kLowest, 0.f, make_float4(0.f, 0.f, 0.f, 0.f)};
            for (int k = c0; k <= c1; ++k) s.M = fmaxf(s.M, __ldcg(p.ml_part + 2 * part(k)));
#pragma unroll 4
            for (int k = c0; k <= c1; ++k) {
                const float2 ml = __ldcg(reinterpret_cast<const float2*>(p.ml_part) + part(k));
                add_piece(s, ml.x, ml.y, __ldcg(reinterpret_cast<const float4*>(p.o_part + part(k) * D) + c));
            }
            store_run<D>(p, u, line, c, s);
        }
    }
}

template <int D, int F>
aflex_status launch_t(aflex_ctx* ctx, const aflex_cache* cache, int grid, const DraftParams& p, cudaStream_t st) {
    typedef DraftStage<D, F> S;
    CUtensorMap tk, tv;
    const uint64_t rows = (uint64_t)cache->kv.num_pages * p.Hkv * kPageTokens;
    const bool made = F == AFLEX_CACHE_BF16
        ? encode_tmap_2d_bf16(&tk, cache->kv.k_cache, rows, D, (uint64_t)D * 2, kPageTokens, 64, true) && encode_tmap_2d_bf16(&tv, cache->kv.v_cache, rows, D, (uint64_t)D * 2, kPageTokens, 64, true)
        : encode_tmap_rows_u8(&tk, cache->kv.k_cache, rows, D, kPageTokens) && encode_tmap_rows_u8(&tv, cache->kv.v_cache, rows, D, kPageTokens);
    if (!made) return set_error(ctx, AFLEX_ERR_CUDA, "draft attention: cuTensorMapEncodeTiled failed");
    const size_t smem = (size_t)kStages * S::kSize + 1024;
    if (!ctx->draft_attr_set[D == 128][F]) {
        cudaError_t e = cudaFuncSetAttribute(attn_draft_kernel<D, F>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
        if (e != cudaSuccess) return check_cuda(ctx, e, "cudaFuncSetAttribute(draft attention)");
        ctx->draft_attr_set[D == 128][F] = true;
    }
    KernelScope scope(ctx, kKAttnDraft, st);
    return check_cuda(ctx, launch_pdl(attn_draft_kernel<D, F>, dim3((unsigned)grid), dim3(kDraftThreads), smem, st, tk, tv, p), "attn_draft_kernel launch");
}

}  // namespace

// ------------------------------------------------------------------------------------------ host
static int draft_grid(int num_sms) { return 2 * num_sms; }

size_t attn_draft_workspace_bytes(const aflex_attn_desc* d, int num_sms) {
    const size_t pieces = 2 * (size_t)draft_grid(num_sms) * kLines;
    return align256(pieces * d->head_dim * sizeof(float)) + align256(pieces * 2 * sizeof(float));
}

aflex_status attn_draft_launch(aflex_ctx* ctx, const aflex_attn_desc* d, const void* q, const aflex_cache* cache, int batch,
                               const aflex_draft* draft, int rows, void* out, float* lse, char* ws, size_t ws_bytes, cudaStream_t st) {
    DraftParams p;
    const aflex_kv* kv = &cache->kv;
    const int D = d->head_dim, grid = draft_grid(ctx->num_sms);
    p.q = (const __nv_bfloat16*)q;
    p.k_scales = cache->k_scales; p.v_scales = cache->v_scales;
    p.page_table = kv->page_table; p.seq_lens = kv->seq_lens;
    p.q_offsets = draft ? draft->q_offsets : nullptr;
    p.mask = draft ? draft->mask : nullptr; p.mask_words = draft ? draft->mask_words : 0;
    p.batch = batch; p.rows = rows; p.max_pages = kv->max_pages_per_seq;
    p.Hq = d->num_q_heads; p.Hkv = d->num_kv_heads; p.G = p.Hq / p.Hkv; p.num_pages = kv->num_pages;
    p.rpt = kLines / p.G;
    const float scale = d->sm_scale != 0.f ? d->sm_scale : 1.0f / sqrtf((float)D);
    p.scale_log2 = scale * 1.4426950408889634f;
    p.out = (__nv_bfloat16*)out; p.lse = lse; p.status = ctx->dev_status;
    p.counters = ctx->counters_attn;
    Arena arena(ws, ws_bytes);
    const size_t pieces = 2 * (size_t)grid * kLines;
    p.o_part = arena.take<float>(pieces * D);
    p.ml_part = arena.take<float>(pieces * 2);
    if (arena.overflow)
        return set_error(ctx, AFLEX_ERR_WORKSPACE, "draft attention: need %zu workspace bytes, have %zu", attn_draft_workspace_bytes(d, ctx->num_sms), ws_bytes);
    // m rows of a sequence are at most (m + rpt - 1) / rpt tiles
    const long long items = ((long long)rows / p.rpt + batch) * p.Hkv;
    if (items > kAttnCounterCap) return set_error(ctx, AFLEX_ERR_UNSUPPORTED, "draft attention: %d rows of %d sequences (supported: up to 2^20 tiles of %d rows x KV heads)", rows, batch, p.rpt);
    const int f = cache->format;
    if (D == 128)
        return f == AFLEX_CACHE_BF16 ? launch_t<128, AFLEX_CACHE_BF16>(ctx, cache, grid, p, st)
             : f == AFLEX_CACHE_INT8 ? launch_t<128, AFLEX_CACHE_INT8>(ctx, cache, grid, p, st) : launch_t<128, AFLEX_CACHE_E4M3>(ctx, cache, grid, p, st);
    return f == AFLEX_CACHE_BF16 ? launch_t<64, AFLEX_CACHE_BF16>(ctx, cache, grid, p, st)
         : f == AFLEX_CACHE_INT8 ? launch_t<64, AFLEX_CACHE_INT8>(ctx, cache, grid, p, st) : launch_t<64, AFLEX_CACHE_E4M3>(ctx, cache, grid, p, st);
}

}  // namespace aflex
