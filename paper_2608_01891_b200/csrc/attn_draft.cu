// Attention of single tokens, drafted tokens in a row and drafted trees over a paged cache in bf16 or in 8 bits.
//
// This kernel is for tiles of up to 8 or 16 lines (rows x query heads of a KV head's group), where the read of the cache is the bound.
//   work        equal shares of the list of units (draft.cuh), two CTAs per SM; an item that several CTAs share is joined by the one
//               that finds all other pieces done, always in the list's order
//   data path   a producer warp walks the share and keeps a ring of stages filled with tiled TMA loads of whole pages (a page's K or V of
//               one KV head is a contiguous block), whose swizzle is what both kinds of reads want: K is read as (two rows) x (four chunks
//               of 16 bytes), V as (rows 0, 2, 4, 6 or 1, 3, 5, 7) x (two chunks), each without a bank conflict
//   arithmetic  mma.sync m16n8k16 with the 16 tokens of a page, or 16 channels, as rows and 8 lines as columns, so that single tokens of
//               groups of 8 waste nothing: S^T = K Q^T, O^T += V^T P^T, P^T from S^T by movmatrix; operands made in registers from 16-byte
//               reads (the order of channels inside a product is free).  Codes of 8 bits become fp16 exactly: int8 + 128 under the exponent
//               of 1024, less 1152; e4m3 by the hardware's conversion.  Queries are bf16, or fp16 after a power of two
//               that brings the line's largest entry to [2^14, 2^15).
//   softmax     online, fp32, base 2, each warp with its own running state.  Of an 8-bit cache the weight of a code is p_j * scale_j, so
//               the running reference follows s_j + log2 scale_j, the weights enter the product in fp16 below 2^15, and their sum is
//               taken of p_j, with the same reference.  A reference moves only when a score outgrows it by 2^7.  Of a bf16 cache the weights are the
//               sum of two bf16 values.
//   masks       only pages that hold drafted tokens look at one
//
// Bound: the read of the cache; for few or short sequences the chain plan -> page ids -> pages -> join, some 12 us of a single long context's.
// 256 rows (32 / 8 heads of 128) over up to 8192 int8 tokens 402 us (5.9 TB/s) repeated over one cache, 459 over another one at every call; one row
// over 131072 55 us (5.0 TB/s), 13 chains of up to 5 (16 / 4 heads of 64) over up to 6000 bf16 tokens 21 us.
//
// Weights of an 8-bit cache are rounded to fp16 once: off by at most 2^-11 of each, an eighth of what the output's rounding to bf16 may be off, and at
// random over the tokens; outputs are as far from the definition in 64 bits as those of weights in 32 bits.  A second fp16 part took 2 % more for
// single tokens, 4 - 10 % for 9 - 32 lines and 10 - 35 % in attn_draft_wide.cu.
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <math.h>

#include "draft.cuh"
#include "internal.h"
#include "ptx.cuh"
#include "rows.cuh"

namespace aflex {

namespace {

constexpr int kMaxLines = 16;                      // of a tile
constexpr int kStages = 3;

// F: the cache's format; NT: eights of lines.  Four compute warps, each with one page (bf16) or two (8 bits) of a unit, which are the place of its
// state at the end.  Two pages are worked on together where 8 lines leave the registers for it: one row over 131072 tokens 55.1 us against 55.8 with
// one at a time; no gain for many rows (256 rows of up to 8192 403 against 400).  Tiles of 16 lines of heads of 128 spill 112 - 120 bytes a thread.
template <int D, int F, int NT> struct DraftForm {
    static constexpr int kLines = 8 * NT;
    static constexpr int kBytes = F == AFLEX_CACHE_BF16 ? 2 : 1;      // of an element
    static constexpr int kRow = D * kBytes;                           // of a token's head
    static constexpr int kBlock = kPageTokens * kRow;                 // K or V of a page
    static constexpr int kWarps = 4;
    static constexpr int kPerWarp = F != AFLEX_CACHE_BF16 ? 2 : 1;
    static constexpr int kTogether = NT == 1 ? kPerWarp : 1;          // pages worked on together
    static constexpr int kPages = kWarps * kPerWarp;
    static constexpr int kTokens = kPages * kPageTokens;
    static constexpr int kThreads = (kWarps + 1) * 32;                // and the producer
    static constexpr int kScales = F == AFLEX_CACHE_BF16 ? 0 : 2 * kPageTokens * 4;      // bytes of a page's scales
    static constexpr int kSize = kPages * (2 * kBlock + kScales);     // of a stage
    static_assert(kPerWarp * 2 * kBlock >= kLines * D * 4, "the state has to fit");
    static_assert(kSize % 1024 == 0, "swizzled blocks are aligned to their pattern");
};

template <int W> struct __align__(8) DraftShared {            // W: compute warps
    uint64_t told[kStages], full[kStages], empty[kStages];     // told: the unit's description is there
    uint64_t meet, pieces;         // the compute warps; copies of pieces to be joined
    DraftPiece meta[kStages];
    float m[2][W][kMaxLines], l[2][W][kMaxLines];              // of pieces in turn
    float3 carry[kMaxLines];       // while pieces are joined: reference and sum so far, and what the sums before are to be multiplied by
    DraftShare share;
    int merges, units;             // items that this CTA has to join at the end; units that the producer brought
    DraftPiece merge[2];
    volatile int abort;
};

// Byte offset of a token's 16-byte chunk inside a page's K or V block, as the tiled copies write it.
template <int kRow> __device__ __forceinline__ uint32_t chunk_at(int t, int ch) {
    if (kRow == 256) return (uint32_t)((ch >> 3) * (kPageTokens * 128) + t * 128 + (((ch & 7) ^ (t & 7)) << 4));
    if (kRow == 128) return (uint32_t)(t * 128 + ((ch ^ (t & 7)) << 4));
    return (uint32_t)(t * 64 + ((ch ^ ((t >> 1) & 3)) << 4));
}

// D(16x8, fp32) += A(16x16) * B(16x8).  (Not volatile, like the loads around it: what a page's products wait for may be done in any order.)
template <int F>
__device__ __forceinline__ void mma_16816(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    if (F == AFLEX_CACHE_BF16)
        asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
            : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
    else
        asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
            : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

template <int D, int NT> struct LineState {        // of a warp: a lane's lines are 8 nt + 2 (lane % 4), + 1
    float o[D / 16][NT][4];                        // channels of n-tiles' pairs (channel_of 2 j, 2 j + 1) x the two lines
    float m[NT][2], l[NT][2];
    uint32_t q[D / 16][NT][2];                     // operand: line 8 nt + lane / 4
    float c[NT][2];                                // what a product counts, in log2 units
    __device__ __forceinline__ void reset() {
#pragma unroll
        for (int n = 0; n < NT; ++n) {
#pragma unroll
            for (int j = 0; j < D / 16; ++j) o[j][n][0] = o[j][n][1] = o[j][n][2] = o[j][n][3] = 0.f;
            m[n][0] = m[n][1] = kLowest;
            l[n][0] = l[n][1] = 0.f;
        }
    }
};

// Chunk c of a lane's part of a K row (or of a query).
template <int kRow> __device__ __forceinline__ int k_chunk(int c, int l4) { return kRow == 256 ? (c >> 1) * 8 + 2 * l4 + (c & 1) : kRow == 128 ? 2 * l4 + c : l4; }

template <int D, int F, int NT>
__device__ __forceinline__ void load_queries(LineState<D, NT>& st, const DraftParams& p, const DraftPiece& u) {
    constexpr int kRow = DraftForm<D, F, NT>::kRow;
    const int lane = threadIdx.x & 31, hl = lane >> 2, l4 = lane & 3;
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        const int line = hl + 8 * n;
        const bool there = line < u.lines;
        const uint4* src = reinterpret_cast<const uint4*>(p.q + ((size_t)(u.row0 + (there ? line >> p.g_shift : 0)) * p.Hq + (size_t)u.g * p.G + (there ? line & (p.G - 1) : 0)) * D);
        float c = p.scale_log2;
        if (F == AFLEX_CACHE_BF16) {
#pragma unroll
            for (int k = 0; k < kRow / 64; ++k) {
                uint4 v = fetch(src + k_chunk<kRow>(k, l4));
                if (!there) v = make_uint4(0, 0, 0, 0);
                st.q[2 * k][n][0] = v.x; st.q[2 * k][n][1] = v.y;
                st.q[2 * k + 1][n][0] = v.z; st.q[2 * k + 1][n][1] = v.w;
            }
        } else {
            uint32_t v[D / 8], big = 0;            // this lane's quarter of the line
#pragma unroll
            for (int k = 0; k < kRow / 64; ++k) {
                const int ch = k_chunk<kRow>(k, l4);
                uint4 a = fetch(src + 2 * ch), b = fetch(src + 2 * ch + 1);
                if (!there) a = b = make_uint4(0, 0, 0, 0);
                v[8 * k] = a.x; v[8 * k + 1] = a.y; v[8 * k + 2] = a.z; v[8 * k + 3] = a.w;
                v[8 * k + 4] = b.x; v[8 * k + 5] = b.y; v[8 * k + 6] = b.z; v[8 * k + 7] = b.w;
            }
#pragma unroll
            for (int i = 0; i < D / 8; ++i) big = __vmaxu2(big, v[i] & 0x7fff7fffu);
            big = max(big & 0xffffu, big >> 16);
            big = max(big, __shfl_xor_sync(0xffffffffu, big, 1));
            big = max(big, __shfl_xor_sync(0xffffffffu, big, 2));
            // largest in [2^e, 2^(e + 1)): times 2^(14 - e); tiny lines by 2^126
            const int e = max((int)(big >> 7) - 127, -112);
            const float up = __uint_as_float((uint32_t)(127 + 14 - e) << 23);
            c = big >= 0x7f80u ? __uint_as_float(0x7fc00000u) : p.scale_log2 * __uint_as_float((uint32_t)(127 - 14 + e) << 23);
#pragma unroll
            for (int i = 0; i < D / 8; ++i) {
                const __half2 h = __floats2half2_rn(__uint_as_float(v[i] << 16) * up, __uint_as_float(v[i] & 0xffff0000u) * up);
                st.q[i / 2][n][i & 1] = *reinterpret_cast<const uint32_t*>(&h);
            }
        }
        // from the lanes that loaded a line to those that hold its scores
#pragma unroll
        for (int e = 0; e < 2; ++e) st.c[n][e] = __shfl_sync(0xffffffffu, c, l4 * 8 + 4 * e);
    }
}

// N pages for one warp: K of the first at kp and its V behind it, the scales at sp; tokens tp .. of the sequence, of which the first `seen` count.
template <int D, int F, int NT, int N>
__device__ __forceinline__ void attend_pages(LineState<D, NT>& st, const DraftParams& p, const DraftPiece& u, const uint8_t* kp, const float* sp, int tp, int seen, bool masked) {
    typedef DraftForm<D, F, NT> S;
    constexpr int kRow = S::kRow, kPageBytes = 2 * S::kBlock, kPageScales = S::kScales / 4;
    const int lane = threadIdx.x & 31, hl = lane >> 2, l4 = lane & 3;
    float s[N][NT][4];                             // token hl: lines 2 l4, 2 l4 + 1; token hl + 8: the same
#pragma unroll
    for (int g = 0; g < N; ++g)
#pragma unroll
        for (int n = 0; n < NT; ++n) s[g][n][0] = s[g][n][1] = s[g][n][2] = s[g][n][3] = 0.f;
#pragma unroll
    for (int c = 0; c < kRow / 64; ++c) {
        uint4 x[N], y[N];
#pragma unroll
        for (int g = 0; g < N; ++g) {
            x[g] = *reinterpret_cast<const uint4*>(kp + g * kPageBytes + chunk_at<kRow>(hl, k_chunk<kRow>(c, l4)));
            y[g] = *reinterpret_cast<const uint4*>(kp + g * kPageBytes + chunk_at<kRow>(hl + 8, k_chunk<kRow>(c, l4)));
        }
        if (F == AFLEX_CACHE_BF16) {
#pragma unroll
            for (int g = 0; g < N; ++g) {
                const uint32_t a[2][4] = {{x[g].x, y[g].x, x[g].y, y[g].y}, {x[g].z, y[g].z, x[g].w, y[g].w}};
#pragma unroll
                for (int k = 0; k < 2; ++k)
#pragma unroll
                    for (int n = 0; n < NT; ++n) mma_16816<F>(s[g][n], a[k], st.q[2 * c + k][n][0], st.q[2 * c + k][n][1]);
            }
        } else {
#pragma unroll
            for (int k = 0; k < 4; ++k)
#pragma unroll
                for (int g = 0; g < N; ++g) {
                    uint32_t a[4];
                    widen4<F>(reinterpret_cast<const uint32_t*>(&x[g])[k], a[0], a[2]);
                    widen4<F>(reinterpret_cast<const uint32_t*>(&y[g])[k], a[1], a[3]);
#pragma unroll
                    for (int n = 0; n < NT; ++n) mma_16816<F>(s[g][n], a, st.q[4 * c + k][n][0], st.q[4 * c + k][n][1]);
                }
        }
    }
    // ---- scores in log2 units, of the lane's lines: x[g][n][r][e] for token hl + 8 r, with lv of the token's V (log2_scale)
    float x[N][NT][2][2], lv[N][2];
#pragma unroll
    for (int g = 0; g < N; ++g)
#pragma unroll
        for (int r = 0; r < 2; ++r) {
            float ks = 1.f;
            if (F != AFLEX_CACHE_BF16) {
                ks = sp[g * kPageScales + hl + 8 * r];
                lv[g][r] = log2_scale(sp[g * kPageScales + kPageTokens + hl + 8 * r]);
            }
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    float& v = x[g][n][r][e];
                    v = s[g][n][2 * r + e] * st.c[n][e];
                    if (F != AFLEX_CACHE_BF16) v = fmaf(v, ks, lv[g][r]);
                }
        }
    uint32_t dead = 0;                             // bit 4 g + k: nothing of token 2 l4 + (k & 1) + 8 (k >> 1) of V may enter the product
    if (masked) {
        bool poison[NT][2];
#pragma unroll
        for (int n = 0; n < NT; ++n) poison[n][0] = poison[n][1] = false;
#pragma unroll
        for (int g = 0; g < N; ++g) {
            const int first = tp + g * kPageTokens;
            // slots behind the last token may hold anything; and an infinity or NaN of a drafted token (int8 has neither) must not enter the
            // product, which would carry it to the lines that do not see it
            uint32_t here = 0;
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const int t = 2 * l4 + (k & 1) + 8 * (k >> 1);
                bool odd = first + t >= seen;
                // (the words that this lane is to multiply; of e4m3 not where a single row sees itself and there is nobody to be kept from it)
                if (F == AFLEX_CACHE_E4M3 && p.mask == nullptr && u.m == 1) {
                } else if (F == AFLEX_CACHE_E4M3 && D == 64) {
                    const uint2 v = *reinterpret_cast<const uint2*>(kp + g * kPageBytes + S::kBlock + chunk_at<kRow>(t, hl >> 1) + (hl & 1) * 8);
                    odd = odd || odd_e4m3(v.x) || odd_e4m3(v.y);
                } else if (F != AFLEX_CACHE_INT8) {
#pragma unroll
                    for (int h = 0; h < (F == AFLEX_CACHE_BF16 ? D / 64 : 1); ++h) {
                        const uint4 v = *reinterpret_cast<const uint4*>(kp + g * kPageBytes + S::kBlock + chunk_at<kRow>(t, 8 * h + hl));
                        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
                        for (int i = 0; i < 4; ++i) odd = odd || (F == AFLEX_CACHE_BF16 ? odd_bf16(w[i]) : odd_e4m3(w[i]));
                    }
                }
                if (odd) here |= 1u << k;
            }
            uint32_t all = (here & 3u) << (2 * l4) | (here >> 2) << (2 * l4 + 8);         // bit t: token t
            if (F != AFLEX_CACHE_INT8) {
                all = __reduce_or_sync(0xffffffffu, all);
                here = (all >> (2 * l4) & 3u) | (all >> (2 * l4 + 8) & 3u) << 2;
            }
            dead |= here << (4 * g);
#pragma unroll
            for (int r = 0; r < 2; ++r) {
                const int t = first + hl + 8 * r;
                bool bad = F != AFLEX_CACHE_INT8 && (all >> (hl + 8 * r) & 1u);
                if (F != AFLEX_CACHE_BF16) bad = bad || !(lv[g][r] == lv[g][r]);      // (a scale that is no number)
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const int line = 8 * n + 2 * l4 + e, i = line >> p.g_shift;
                        const bool see = t < seen && line < u.lines && sees_drafted(p, u.row0 + i, u.i0 + i, t - u.ctx, u.m);
                        if (see && bad) poison[n][e] = true;
                        if (!see) x[g][n][r][e] = -INFINITY;
                    }
                if (F != AFLEX_CACHE_BF16 && bad) lv[g][r] = 0.f;       // (for the lines that do not see it, whose x is -infinity)
            }
        }
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int e = 0; e < 2; ++e) if (poison[n][e]) st.l[n][e] = __uint_as_float(0x7fc00000u);
    }
    float mx[NT][2];
    bool grow = false;
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            mx[n][e] = fmaxf(x[0][n][0][e], x[0][n][1][e]);
#pragma unroll
            for (int g = 1; g < N; ++g) mx[n][e] = fmaxf(mx[n][e], fmaxf(x[g][n][0][e], x[g][n][1][e]));
            grow = grow || mx[n][e] > st.m[n][e] + (kBelow<F> + 7.f);
        }
    // (m is the same for all lanes of a line)
    if (__any_sync(0xffffffffu, grow)) {
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            float corr[2];
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                float& v = mx[n][e];
                v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, 4));
                v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, 8));
                v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, 16));
                const float mn = v > st.m[n][e] + (kBelow<F> + 7.f) ? v - kBelow<F> : st.m[n][e];          // (a line's bits do not depend on who else's moves)
                corr[e] = fast_exp2(st.m[n][e] - mn);
                st.l[n][e] = scale_sum(st.l[n][e], st.m[n][e] - mn);
                st.m[n][e] = mn;
            }
#pragma unroll
            for (int j = 0; j < D / 16; ++j) { st.o[j][n][0] *= corr[0]; st.o[j][n][1] *= corr[1]; st.o[j][n][2] *= corr[0]; st.o[j][n][3] *= corr[1]; }
        }
    }
    uint32_t a[N][NT][2], b[N][NT][2];             // weights as the product's operand; bf16: the rest of them in b
#pragma unroll
    for (int g = 0; g < N; ++g)
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int r = 0; r < 2; ++r) {
                const float w0 = fast_exp2(x[g][n][r][0] - st.m[n][0]), w1 = fast_exp2(x[g][n][r][1] - st.m[n][1]);
                if (F == AFLEX_CACHE_BF16) {
                    st.l[n][0] += w0;
                    st.l[n][1] += w1;
                    const uint32_t hi = pack_bf16x2(w0, w1);
                    a[g][n][r] = movmatrix_trans(hi);
                    b[g][n][r] = movmatrix_trans(pack_bf16x2(w0 - __uint_as_float(hi << 16), w1 - __uint_as_float(hi & 0xffff0000u)));
                } else {
                    st.l[n][0] += fast_exp2(x[g][n][r][0] - st.m[n][0] - lv[g][r]);
                    st.l[n][1] += fast_exp2(x[g][n][r][1] - st.m[n][1] - lv[g][r]);
                    const __half2 h = __floats2half2_rn(w0, w1);
                    a[g][n][r] = movmatrix_trans(*reinterpret_cast<const uint32_t*>(&h));
                }
            }
    // ---- V: tokens 2 l4, 2 l4 + 1, 2 l4 + 8, 2 l4 + 9 of the lane's channels
    constexpr int kParts = F == AFLEX_CACHE_BF16 ? D / 64 : 1;      // chunks of a lane per token
    constexpr int kWords = F == AFLEX_CACHE_BF16 ? 4 : D / 32;      // 32-bit words of one
#pragma unroll
    for (int g = 0; g < N; ++g) {
        const uint8_t* vp = kp + g * kPageBytes + S::kBlock;
#pragma unroll
        for (int h = 0; h < kParts; ++h) {
            uint32_t w[4][kWords];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const int t = 2 * l4 + (k & 1) + 8 * (k >> 1);
                if (kWords == 4) {
                    const uint4 v = *reinterpret_cast<const uint4*>(vp + chunk_at<kRow>(t, 8 * h + hl));
                    w[k][0] = v.x; w[k][1] = v.y; w[k][2 % kWords] = v.z; w[k][3 % kWords] = v.w;
                } else {
                    const uint2 v = *reinterpret_cast<const uint2*>(vp + chunk_at<kRow>(t, hl >> 1) + (hl & 1) * 8);
                    w[k][0] = v.x; w[k][1] = v.y;
                }
            }
            if (masked) {
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    if (dead >> (4 * g + k) & 1)
#pragma unroll
                        for (int i = 0; i < kWords; ++i) w[k][i] = 0;
            }
#pragma unroll
            for (int i = 0; i < kWords; ++i) {
                // channels of the word: two of bf16 (one product), four codes (two products)
                uint32_t v[4][2];
#pragma unroll
                for (int y = 0; y < 2; ++y) {
                    if (F == AFLEX_CACHE_BF16) {
                        v[0][y] = __byte_perm(w[2 * y][i], w[2 * y + 1][i], 0x5410);
                        v[1][y] = __byte_perm(w[2 * y][i], w[2 * y + 1][i], 0x7632);
                    } else {
                        widen4<F>(__byte_perm(w[2 * y][i], w[2 * y + 1][i], 0x5140), v[0][y], v[1][y]);
                        widen4<F>(__byte_perm(w[2 * y][i], w[2 * y + 1][i], 0x7362), v[2][y], v[3][y]);
                    }
                }
#pragma unroll
                for (int z = 0; z < (F == AFLEX_CACHE_BF16 ? 1 : 2); ++z) {
                    const uint32_t av[4] = {v[2 * z][0], v[2 * z + 1][0], v[2 * z][1], v[2 * z + 1][1]};
                    const int j = F == AFLEX_CACHE_BF16 ? 4 * h + i : 2 * i + z;
#pragma unroll
                    for (int n = 0; n < NT; ++n) {
                        mma_16816<F>(st.o[j][n], av, a[g][n][0], a[g][n][1]);
                        if (F == AFLEX_CACHE_BF16) mma_16816<F>(st.o[j][n], av, b[g][n][0], b[g][n][1]);
                    }
                }
            }
        }
    }
}

// Place of four channels of a line in a parked state: neighbouring lines' words in other banks.
template <int D> __device__ __forceinline__ uint32_t parked_at(int line, int run) { return (uint32_t)(line * (D * 4) + ((run ^ (line & 7)) << 4)); }

template <int D, int F, int NT>
__device__ __forceinline__ void park(const LineState<D, NT>& st, uint8_t* to, float* m_to, float* l_to) {
    const int lane = threadIdx.x & 31, hl = lane >> 2, l4 = lane & 3;
#pragma unroll
    for (int n = 0; n < NT; ++n) {
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const int line = 8 * n + 2 * l4 + e;
            float l = st.l[n][e];
#pragma unroll
            for (int off = 4; off < 32; off <<= 1) l += __shfl_xor_sync(0xffffffffu, l, off);
#pragma unroll
            for (int j = 0; j < D / 16; j += 2) {
                // the lane's 2 j-th channel and the three behind it
                const int ch = F == AFLEX_CACHE_BF16 ? 64 * (j >> 2) + 8 * hl + 2 * (j & 3) : (D / 8) * hl + 2 * j;
                *reinterpret_cast<float4*>(to + parked_at<D>(line, ch / 4)) = make_float4(st.o[j][n][e], st.o[j][n][2 + e], st.o[j + 1][n][e], st.o[j + 1][n][2 + e]);
            }
            if (hl == 0) { m_to[line] = st.m[n][e]; l_to[line] = l; }
        }
    }
}

constexpr int kCarry = 2 * kMaxLines;                 // references and sums before a slot's lines
template <int D> constexpr int kSlot = kCarry + kMaxLines * D;      // floats of a piece's slot

template <int D, int F, int NT>
__global__ void __launch_bounds__(DraftForm<D, F, NT>::kThreads, 2)
attn_draft_kernel(const __grid_constant__ CUtensorMap tmap_k, const __grid_constant__ CUtensorMap tmap_v, const __grid_constant__ DraftParams p) {
    typedef DraftForm<D, F, NT> S;
    constexpr int W = S::kWarps, kThreads = S::kThreads;
    constexpr int kRuns = D / 4;                   // a line's outputs in runs of four channels
    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
    __shared__ DraftShared<W> sh;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (threadIdx.x == 0) {
        for (int s = 0; s < kStages; ++s) {
            mbar_init(&sh.full[s], F == AFLEX_CACHE_BF16 ? 1 : 33);       // (8 bits: and the producer's lanes, for the scales)
            mbar_init(&sh.told[s], 1);
            mbar_init(&sh.empty[s], W);
        }
        mbar_init(&sh.meet, W);
        mbar_init(&sh.pieces, 1);
        sh.abort = 0;
        sh.merges = 0;
        fence_mbar_init();
        prefetch_tmap(&tmap_k);
        prefetch_tmap(&tmap_v);
    }
    pdl_launch_dependents();
    // The lengths, the row offsets and the page table are inputs of the step, never written by a kernel of this library, so the plan and the
    // first page ids are made while the preceding kernel is still draining; what it may have written (q, the cache, partial results,
    // counters) waits for it, per role.
    const DraftList<S::kTokens, 1> list(p);
    draft_plan<kThreads>(p, list, sh.share);

    if (warp == W) {
        // ------------------------------------------------------------------ producer
        const DraftShare share = sh.share;
        int it = 0;
        bool ok = true;
        auto slot_free = [&]() {                   // the next stage, once everybody has left it
            ok = mbar_wait(&sh.empty[it % kStages], ((it / kStages) & 1) ^ 1);
            ok = __all_sync(0xffffffffu, ok) && !sh.abort;
            return ok;
        };
        // lane: a page of the unit, K or V, and half of a row or the scales
        const int page = lane % S::kPages, kv = (lane / S::kPages) & 1, part = lane / (2 * S::kPages);
        const bool copies = lane < 2 * S::kPages * (F == AFLEX_CACHE_BF16 ? S::kRow / 128 : 1);
        const uint64_t policy = policy_evict_first();                  // (the cache is read once)
        DraftWalk<S::kTokens, 1> w;
        if (share.x0 < share.x1) w.start(p, list, share.x0, share.seq, share.seq_first, share.seq_tiles);
        else w.pos = share.x1;
        while (ok && w.pos < share.x1) {
            if (w.u == 0 && w.nu > 1) { w.advance(p, list, 1, share.total); continue; }
            const DraftPiece meta = draft_piece(p, list, w, share.x1);
            const int u0 = w.u, u1 = w.until(share.x1);
            const int32_t* table = p.page_table + (size_t)w.b * p.max_pages;
            auto page_id = [&](int u) -> int {
                const int i = (u - 1) * S::kPages + page;
                return copies && u >= 1 && i * kPageTokens < meta.sees ? fetch(table + i) : 0;
            };
            int id = page_id(u0);
            for (int u = u0; u < u1; ++u, ++it) {
                const int id_next = u + 1 < u1 ? page_id(u + 1) : 0;
                if (it == 0) pdl_wait();
                if (!slot_free()) break;
                const int st = it % kStages;
                const int t0 = (u - 1) * S::kTokens;
                const int np = u == 0 ? 0 : min(S::kPages, (meta.sees - t0 + kPageTokens - 1) / kPageTokens);
                if (copies && page < np && (id < 0 || id >= p.num_pages)) { atomicExch(p.status, AFLEX_ERR_BOUNDS); id = 0; }
                if (lane == 0) {
                    sh.meta[st] = meta;            // (with every unit: the last one's is read when the piece ends)
                    mbar_arrive(&sh.told[st]);
                    mbar_expect_tx(&sh.full[st], (uint32_t)(np * 2 * S::kBlock));
                }
                __syncwarp();
                if (copies && page < np) {
                    uint8_t* stage = smem + st * S::kSize;
                    uint8_t* dst = stage + (page * 2 + kv) * S::kBlock;
                    const int slab = id * p.Hkv + w.g;
                    if (F == AFLEX_CACHE_BF16) tma_load_2d_hint(dst + part * (kPageTokens * 128), kv ? &tmap_v : &tmap_k, part * 64, slab * kPageTokens, &sh.full[st], policy);
                    else {
                        tma_load_2d_hint(dst, kv ? &tmap_v : &tmap_k, 0, slab * kPageTokens, &sh.full[st], policy);
                        // 64 bytes of scales, too small for a bulk copy each
                        const float* from = (kv ? p.v_scales : p.k_scales) + (size_t)slab * kPageTokens;
                        const uint32_t to = smem_u32(stage) + (uint32_t)(S::kPages * 2 * S::kBlock + page * S::kScales + kv * (S::kScales / 2));
#pragma unroll
                        for (int i = 0; i < 4; ++i) copy16(to + i * 16, from + i * 4);
                    }
                }
                if (F != AFLEX_CACHE_BF16) copies_arrive(&sh.full[st]);
                id = id_next;
            }
            if (ok) w.advance(p, list, u1 - u0, share.total);
        }
        if (ok && slot_free()) {
            if (lane == 0) {
                sh.meta[it % kStages].units = 0;
                mbar_arrive(&sh.told[it % kStages]);
                mbar_arrive_n(&sh.full[it % kStages], F == AFLEX_CACHE_BF16 ? 1 : 33);
            }
            ++it;
        }
        if (lane == 0) sh.units = it;
        if (!ok && lane == 0) { sh.abort = 1; atomicExch(p.status, AFLEX_ERR_TIMEOUT); }
    } else if (warp < W) {
        // ------------------------------------------------------------------ compute
        LineState<D, NT> st;
        int pieces = 0;
        uint32_t met = 0;
        auto meet = [&]() -> bool {                // the compute warps (a bounded wait: a warp that has given up does not come)
            __syncwarp();
            if (lane == 0) mbar_arrive(&sh.meet);
            const bool came = mbar_wait(&sh.meet, met & 1);
            ++met;
            return __all_sync(0xffffffffu, came);
        };
        pdl_wait();
        int stage = 0, parity = 0, left = 0, tp = 0, seen = 0, plain = 0;       // of the piece: units to come, the warp's next token ..
        for (;;) {
            if (left == 0) {                       // a new piece: its description, and the queries while its pages are on their way
                bool ok = mbar_wait(&sh.told[stage], parity);
                ok = __all_sync(0xffffffffu, ok);
                if (!ok) { if (lane == 0) { sh.abort = 1; atomicExch(p.status, AFLEX_ERR_TIMEOUT); } break; }
                const DraftPiece& u = sh.meta[stage];
                left = u.units;
                if (left == 0) break;              // the end of the share
                seen = u.sees;
                plain = min(u.ctx, seen);
                tp = u.t0 + warp * S::kPerWarp * kPageTokens;
                st.reset();
                load_queries<D, F, NT>(st, p, u);
            }
            const bool ok = mbar_wait(&sh.full[stage], parity);
            if (!__all_sync(0xffffffffu, ok)) { if (lane == 0) { sh.abort = 1; atomicExch(p.status, AFLEX_ERR_TIMEOUT); } break; }
            uint8_t* base = smem + stage * S::kSize;
            uint8_t* mine = base + warp * S::kPerWarp * 2 * S::kBlock;
#pragma unroll 1
            for (int k = 0; k < S::kPerWarp; k += S::kTogether) {
                // (a page of them that the unit does not have is masked like one that ends early)
                const int t = tp + k * kPageTokens;
                if (t < seen && t >= 0)
                    attend_pages<D, F, NT, S::kTogether>(st, p, sh.meta[stage], mine + k * 2 * S::kBlock,
                                                         reinterpret_cast<const float*>(base + S::kPages * 2 * S::kBlock + (warp * S::kPerWarp + k) * S::kScales), t, seen,
                                                         t + S::kTogether * kPageTokens > plain);
            }
            tp += S::kTokens;
            __syncwarp();
            if (--left == 0) {
                // ---- the piece is done: the warps leave their states in their pages' place, and each joins a part of the lines.  (A warp that
                // is ahead leaves the next piece's references in the other half of sh.m and sh.l, and waits for the others there.)
                float(&pm)[W][kMaxLines] = sh.m[pieces & 1];
                float(&pl)[W][kMaxLines] = sh.l[pieces & 1];
                ++pieces;
                park<D, F, NT>(st, mine, pm[warp], pl[warp]);
                const DraftPiece piece = sh.meta[stage];
                if (!meet()) { if (lane == 0) { sh.abort = 1; atomicExch(p.status, AFLEX_ERR_TIMEOUT); } break; }
                float* slot = p.parts + ((size_t)blockIdx.x * 2 + piece.slot) * kSlot<D>;
#pragma unroll 1                                   // (here and below: code that runs once a piece is kept small, it is seldom in the instruction cache)
                for (int i = threadIdx.x; i < piece.lines * kRuns; i += W * 32) {
                    const int line = i / kRuns, c = i % kRuns;
                    RunSum s = {kLowest, 0.f, make_float4(0.f, 0.f, 0.f, 0.f)};
#pragma unroll
                    for (int w = 0; w < W; ++w) s.M = fmaxf(s.M, pm[w][line]);
#pragma unroll
                    for (int w = 0; w < W; ++w)
                        add_piece(s, pm[w][line], pl[w][line], *reinterpret_cast<const float4*>(base + w * S::kPerWarp * 2 * S::kBlock + parked_at<D>(line, c)));
                    if (piece.whole) store_run<D>(p, piece, line, c, s);
                    else {
                        __stcg(reinterpret_cast<float4*>(slot + kCarry + line * D) + c, s.acc);
                        if (c == 0) __stcg(reinterpret_cast<float2*>(slot) + line, make_float2(s.M, s.L));
                    }
                }
                fence_proxy_async();               // (the stage's next copies come behind these reads and stores)
                __syncwarp();
                if (lane == 0) mbar_arrive(&sh.empty[stage]);
                if (!piece.whole) {
                    // the last of the item's CTAs to get here joins the pieces (offsets that decrease could name more items than there are counters)
                    if (!meet()) { if (lane == 0) { sh.abort = 1; atomicExch(p.status, AFLEX_ERR_TIMEOUT); } break; }
                    if (threadIdx.x == 0) {
                        __threadfence();
                        if (piece.item >= kAttnCounterCap) atomicExch(p.status, AFLEX_ERR_BOUNDS);
                        else if (atomicAdd(p.counters + piece.item, 1) == sh.share.cta_of(piece.last) - sh.share.cta_of(piece.first)) {
                            p.counters[piece.item] = 0;
                            sh.merge[sh.merges++] = piece;
                        }
                    }
                }
            } else if (lane == 0) {
                mbar_arrive(&sh.empty[stage]);
            }
            if (++stage == kStages) { stage = 0; parity ^= 1; }
        }
    }
    __syncthreads();
    if (sh.abort) {                                // copies under way are waited for once more, since this memory will be another CTA's
        for (int i = max(0, sh.units - kStages); i < sh.units; ++i) mbar_wait(&sh.full[i % kStages], (i / kStages) & 1);
        return;
    }
    if (sh.merges == 0) return;
    __threadfence();
    fence_proxy_async_all();
    __syncthreads();
    // ---- join the pieces of the items that this CTA was the last one to work on, as many at a time as the ring holds behind the sums: it is
    // free, every copy has been waited for
    float4* sums = reinterpret_cast<float4*>(smem);                     // [line][run], and references and sums of weights in sh.carry
    uint8_t* slots = smem + S::kLines * D * 4;
    uint32_t phase = 0;
#pragma unroll 1
    for (int j = 0; j < sh.merges; ++j) {
        const DraftPiece u = sh.merge[j];
        const int c0 = sh.share.cta_of(u.first), n = sh.share.cta_of(u.last) - c0 + 1;
        const uint32_t bytes = (uint32_t)(kCarry + u.lines * D) * 4;
        const int at_once = (kStages * S::kSize - S::kLines * D * 4) / (int)bytes;
        auto weight = [&](int k, int line) -> float2* { return reinterpret_cast<float2*>(slots + (size_t)k * bytes) + line; };
#pragma unroll 1
        for (int k0 = 0; k0 < n; k0 += at_once) {
            const int here = min(at_once, n - k0);
            if (warp == 0) {
                if (lane == 0) mbar_expect_tx(&sh.pieces, bytes * here);
                __syncwarp();
#pragma unroll 1
                for (int k = lane; k < here; k += 32)                                   // (of the first CTA the second slot)
                    bulk_load_1d(slots + (size_t)k * bytes, p.parts + ((size_t)(c0 + k0 + k) * 2 + (k0 + k == 0 ? 1 : 0)) * kSlot<D>, bytes, &sh.pieces);
            }
            const bool ok = mbar_wait(&sh.pieces, phase);
            phase ^= 1;
            if (__syncthreads_or(!ok)) {
                if (threadIdx.x == 0) atomicExch(p.status, AFLEX_ERR_TIMEOUT);
                mbar_wait(&sh.pieces, phase ^ 1);
                return;
            }
            // factors of the pieces' sums, a warp for a line
#pragma unroll 1
            for (int line = warp; line < u.lines; line += kThreads / 32) {
                const float before = k0 > 0 ? sh.carry[line].x : kLowest;
                float M = before, L = 0.f;
#pragma unroll 1
                for (int k = lane; k < here; k += 32) M = fmaxf(M, weight(k, line)->x);
#pragma unroll
                for (int off = 16; off > 0; off >>= 1) M = fmaxf(M, __shfl_xor_sync(0xffffffffu, M, off));
#pragma unroll 1
                for (int k = lane; k < here; k += 32) {
                    float2* x = weight(k, line);
                    L += scale_sum(x->y, x->x - M);
                    x->x = fast_exp2(x->x - M);
                }
#pragma unroll
                for (int off = 16; off > 0; off >>= 1) L += __shfl_xor_sync(0xffffffffu, L, off);
                const float f = fast_exp2(before - M);
                if (lane == 0) sh.carry[line] = make_float3(M, k0 > 0 ? L + scale_sum(sh.carry[line].y, before - M) : L, f);
            }
            __syncthreads();
#pragma unroll 1
            for (int i = threadIdx.x; i < u.lines * kRuns; i += kThreads) {
                const int line = i / kRuns, c = i % kRuns;
                float4 a = make_float4(0.f, 0.f, 0.f, 0.f);
                if (k0 > 0) {
                    const float f = sh.carry[line].z;
                    a = sums[i];
                    a.x *= f; a.y *= f; a.z *= f; a.w *= f;
                }
#pragma unroll 4
                for (int k = 0; k < here; ++k) {
                    const float g = weight(k, line)->x;
                    const float4 v = *reinterpret_cast<const float4*>(slots + (size_t)k * bytes + (kCarry + line * D + 4 * c) * 4);
                    a.x = fmaf(v.x, g, a.x); a.y = fmaf(v.y, g, a.y); a.z = fmaf(v.z, g, a.z); a.w = fmaf(v.w, g, a.w);
                }
                if (k0 + here < n) sums[i] = a;
                else store_run<D>(p, u, line, c, RunSum{sh.carry[line].x, sh.carry[line].y, a});
            }
            fence_proxy_async();
            __syncthreads();
        }
    }
}

template <int D, int F, int NT>
aflex_status launch_t(aflex_ctx* ctx, const aflex_cache* cache, int grid, const DraftParams& p, cudaStream_t st) {
    typedef DraftForm<D, F, NT> S;
    CUtensorMap tk, tv;
    const uint64_t rows = (uint64_t)cache->kv.num_pages * p.Hkv * kPageTokens;
    const bool made = F == AFLEX_CACHE_BF16
        ? encode_tmap_2d_bf16(&tk, cache->kv.k_cache, rows, D, (uint64_t)D * 2, kPageTokens, 64, true) && encode_tmap_2d_bf16(&tv, cache->kv.v_cache, rows, D, (uint64_t)D * 2, kPageTokens, 64, true)
        : encode_tmap_rows_u8(&tk, cache->kv.k_cache, rows, D, kPageTokens) && encode_tmap_rows_u8(&tv, cache->kv.v_cache, rows, D, kPageTokens);
    if (!made) return set_error(ctx, AFLEX_ERR_CUDA, "draft attention: cuTensorMapEncodeTiled failed");
    const size_t smem = (size_t)kStages * S::kSize + 1024;
    if (!ctx->draft_attr_set[D == 128][F][NT - 1]) {
        cudaError_t e = cudaFuncSetAttribute(attn_draft_kernel<D, F, NT>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
        if (e != cudaSuccess) return check_cuda(ctx, e, "cudaFuncSetAttribute(draft attention)");
        ctx->draft_attr_set[D == 128][F][NT - 1] = true;
    }
    KernelScope scope(ctx, kKAttnDraft, st);
    return check_cuda(ctx, launch_pdl(attn_draft_kernel<D, F, NT>, dim3((unsigned)grid), dim3(S::kThreads), smem, st, tk, tv, p), "attn_draft_kernel launch");
}

template <int D, int F>
aflex_status launch_f(aflex_ctx* ctx, const aflex_cache* cache, int grid, const DraftParams& p, cudaStream_t st) {
    return p.rpt_shift + p.g_shift == 3 ? launch_t<D, F, 1>(ctx, cache, grid, p, st) : launch_t<D, F, 2>(ctx, cache, grid, p, st);
}

}  // namespace

// ------------------------------------------------------------------------------------------ host
static int draft_grid(int num_sms) { return 2 * num_sms; }
size_t attn_draft_wide_workspace_bytes(int head_dim, int num_sms);                    // attn_draft_wide.cu
aflex_status attn_draft_wide_launch(aflex_ctx* ctx, const aflex_cache* cache, int head_dim, const DraftParams& p, cudaStream_t st);

size_t attn_draft_workspace_bytes(const aflex_attn_desc* d, int num_sms) {
    const size_t narrow = align256((size_t)draft_grid(num_sms) * 2 * (kCarry + kMaxLines * d->head_dim) * sizeof(float));
    const size_t wide = attn_draft_wide_workspace_bytes(d->head_dim, num_sms);
    return narrow > wide ? narrow : wide;
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
    p.g_shift = p.G == 1 ? 0 : p.G == 2 ? 1 : p.G == 4 ? 2 : 3;
    // Lines per tile by the lines of an average sequence: 8, 16, or 256 on the tensor cores, whose step costs the same for any number of lines up to
    // 128 while tiles of 16 read the cache again.  Measured (us, tiles of 16 / tensor cores) with ragged sequences, by their average:
    //   heads of 128, 8 sequences   25 lines 73 / 83 in int8, 68 / 80 in e4m3, 88 / 83 in bf16;   33 lines 88 / 83, 81 / 81, 101 / 83
    //   64 sequences, int8          24 lines 449 / 473;   32 lines 620 / 475
    //   heads of 64, 13 sequences   31 lines 27 / 33 in int8, 29 / 32 in bf16;   37 lines 30 / 33, 31 / 32;   41 lines 35 / 32 in bf16
    //   64 sequences                36 lines 95 / 96 in int8, 109 / 94 in bf16
    // One rule for all formats and batches, which costs up to 30 % beside its border; and a batch of single tokens and a long chunk has one form.
    const long long lines = (long long)rows << p.g_shift;
    const int narrow = D == 64 ? 48 : 32;
    p.rpt_shift = (lines <= 8LL * batch ? 3 : lines <= (long long)narrow * batch ? 4 : 8) - p.g_shift;
    const float scale = d->sm_scale != 0.f ? d->sm_scale : 1.0f / sqrtf((float)D);
    p.scale_log2 = scale * 1.4426950408889634f;
    p.unit = cache->format == AFLEX_CACHE_BF16 ? 1.f : exp2f(kScaleShift);
    p.out = (__nv_bfloat16*)out; p.lse = lse; p.status = ctx->dev_status;
    p.counters = ctx->counters_attn;
    const size_t need = attn_draft_workspace_bytes(d, ctx->num_sms);
    if (ws_bytes < need) return set_error(ctx, AFLEX_ERR_WORKSPACE, "draft attention: need %zu workspace bytes, have %zu", need, ws_bytes);
    p.parts = reinterpret_cast<float*>(ws);
    // m rows of a sequence are at most m / 2^rpt_shift + 1 tiles
    const long long items = (((long long)rows >> p.rpt_shift) + batch) * p.Hkv;
    if (items > kAttnCounterCap) return set_error(ctx, AFLEX_ERR_UNSUPPORTED, "draft attention: %d rows of %d sequences (supported: up to 2^20 tiles of %d rows x KV heads)", rows, batch, 1 << p.rpt_shift);
    if (p.rpt_shift + p.g_shift == 8) return attn_draft_wide_launch(ctx, cache, D, p, st);
    typedef aflex_status (*Launch)(aflex_ctx*, const aflex_cache*, int, const DraftParams&, cudaStream_t);
    const Launch launch[2][3] = {{launch_f<64, AFLEX_CACHE_BF16>, launch_f<64, AFLEX_CACHE_INT8>, launch_f<64, AFLEX_CACHE_E4M3>},
                                 {launch_f<128, AFLEX_CACHE_BF16>, launch_f<128, AFLEX_CACHE_INT8>, launch_f<128, AFLEX_CACHE_E4M3>}};
    return launch[D == 128][cache->format](ctx, cache, grid, p, st);
}

}  // namespace aflex
