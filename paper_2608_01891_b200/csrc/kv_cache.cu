// A paged KV cache in bf16 or in 8 bits (a scale per token and KV head), written, converted and compacted:
//   cache_append_kernel    head norms, rotary embedding and K/V append of the rows of a call, quantised as they are written
//   cache_convert_kernel   a bf16 cache quantised, an 8-bit cache read back
//   cache_accept_kernel    the accepted path of every sequence's drafted tokens moved together, in the caches of all layers
//
// Quantisation of one token's head x[D] (bf16 values), every step in fp32 and rounded to nearest, halves to even:
//   a = max |x_d|,  scale = max(a * fl(1 / TOP), 2^-64),  code_d = round(x_d * fl(1 / scale))
// with TOP = 127 and whole numbers (int8), or TOP = 448 and e4m3 values.  |x_d| * fl(1 / scale) is at most TOP (1 + 2^-22), which
// rounds to TOP.  One scale per token makes an append independent of what the page held before, and costs 4 bytes beside 128.
// A head with an infinite or NaN entry gets the scale NaN and codes 0: whoever reads it gets NaN.
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <math.h>

#include "internal.h"
#include "ptx.cuh"
#include "rows.cuh"

namespace aflex {

namespace {

constexpr int kWarps = 8;
constexpr int kThreads = kWarps * 32;

// Larger of two pairs of magnitudes (bf16 bits without the sign): as whole numbers NaN > infinity > any number.
__device__ __forceinline__ uint32_t max_magnitudes(uint32_t a, uint32_t b) { return __vmaxu2(a & 0x7fff7fffu, b & 0x7fff7fffu); }

// Scale of a head and the factor of its codes, from the bits of its largest magnitude.
template <int F> __device__ __forceinline__ float head_scale(uint32_t bits, float& inv) {
    if (bits >= 0x7f80u) { inv = 0.f; return __uint_as_float(0x7fc00000u); }
    const float scale = fmaxf(__fmul_rn(__uint_as_float(bits << 16), F == AFLEX_CACHE_INT8 ? 1.f / 127.f : 1.f / 448.f), 5.421010862427522e-20f);
    inv = __frcp_rn(scale);
    return scale;
}
// Codes of four channels, in order.
template <int F> __device__ __forceinline__ uint32_t codes4(uint32_t x01, uint32_t x23, uint64_t inv) {
    float a, b, c, d;
    if (F == AFLEX_CACHE_INT8) {
        // adding 1.5 * 2^23 rounds to a whole number and leaves it in the low bits.  The product is rounded to fp32 first, as defined: the
        // additions are separate, since a packed one directly behind a packed product is joined with it into one rounding.
        unpack_f32x2(mul_f32x2(widen_bf16x2(x01), inv), a, b);
        unpack_f32x2(mul_f32x2(widen_bf16x2(x23), inv), c, d);
        a = __fadd_rn(a, 12582912.f); b = __fadd_rn(b, 12582912.f); c = __fadd_rn(c, 12582912.f); d = __fadd_rn(d, 12582912.f);
        const uint32_t lo = __byte_perm(__float_as_uint(a), __float_as_uint(b), 0x0040), hi = __byte_perm(__float_as_uint(c), __float_as_uint(d), 0x0040);
        return __byte_perm(lo, hi, 0x5410);
    }
    unpack_f32x2(mul_f32x2(widen_bf16x2(x01), inv), a, b);
    unpack_f32x2(mul_f32x2(widen_bf16x2(x23), inv), c, d);
    uint16_t lo, hi;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(lo) : "f"(b), "f"(a));
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(hi) : "f"(d), "f"(c));
    return (uint32_t)lo | ((uint32_t)hi << 16);
}
// The values of four codes times the scale, as bf16 pairs.
template <int F> __device__ __forceinline__ uint2 values4(uint32_t codes, float scale) {
    float x[4];
    if (F == AFLEX_CACHE_INT8) {
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = (float)(int8_t)(codes >> (8 * i));
    } else {
        uint32_t h[2];
        asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h[0]) : "h"((uint16_t)codes));
        asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h[1]) : "h"((uint16_t)(codes >> 16)));
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&h[i]));
            x[2 * i] = f.x;
            x[2 * i + 1] = f.y;
        }
    }
    return make_uint2(pack_bf16x2(x[0] * scale, x[1] * scale), pack_bf16x2(x[2] * scale, x[3] * scale));
}

// Stores one token's head, whose lanes (Lanes<D>) hold 16 channels each, into a cache of format F; `token` counts (page, KV head, slot).
// Every lane of the warp takes part; those with `store` false write nothing.
template <int D, int F>
__device__ __forceinline__ void store_head(void* codes, float* scales, size_t token, int l, const uint4& a, const uint4& b, bool store) {
    if (F == AFLEX_CACHE_BF16) {
        if (store) {
            uint4* dst = reinterpret_cast<uint4*>(codes) + token * (D / 8);
            dst[l] = a;
            dst[D / 16 + l] = b;
        }
        return;
    }
    uint32_t m = max_magnitudes(max_magnitudes(max_magnitudes(a.x, a.y), max_magnitudes(a.z, a.w)),
                                max_magnitudes(max_magnitudes(b.x, b.y), max_magnitudes(b.z, b.w)));
    m = max(m & 0xffffu, m >> 16);
#pragma unroll
    for (int off = 1; off < Lanes<D>::kPer; off <<= 1) m = max(m, __shfl_xor_sync(0xffffffffu, m, off));
    float inv;
    const float scale = head_scale<F>(m, inv);
    const uint64_t inv2 = pack_f32x2(inv, inv);
    uint2 ca = make_uint2(codes4<F>(a.x, a.y, inv2), codes4<F>(a.z, a.w, inv2)), cb = make_uint2(codes4<F>(b.x, b.y, inv2), codes4<F>(b.z, b.w, inv2));
    if (m >= 0x7f80u) ca = cb = make_uint2(0, 0);
    if (store) {
        uint2* dst = reinterpret_cast<uint2*>(reinterpret_cast<uint8_t*>(codes) + token * D);
        dst[l] = ca;
        dst[D / 16 + l] = cb;
        if (l == 0) scales[token] = scale;
    }
}

// ------------------------------------------------------------------------------------------ append
struct AppendParams {
    const __nv_bfloat16* qkv;      // [rows][(Hq + 2 Hkv) * D]
    const __nv_bfloat16* w_qn;     // [D] or null
    const __nv_bfloat16* w_kn;     // [D] or null
    const int32_t* page_table;
    const int32_t* seq_lens;
    const int32_t* q_offsets;      // null: one row per sequence
    const int32_t* positions;      // [rows] or null
    int batch, rows, max_pages, Hq, Hkv;
    long long num_pages;
    __nv_bfloat16* q_out;
    void* k_cache;
    void* v_cache;
    float* k_scales;
    float* v_scales;
    int tile, q_heads_per_cta, kv_ctas, groups;    // rows per CTA; head groups of a tile: kv_ctas for its K and V heads, the others for its query heads
    float eps;
    double inv_freq[64];           // theta^(-2 i / D), formed in double on the host
    double step_cos[64], step_sin[64];             // ... and the cosine and sine of that angle: one position's rotation
    int* status;
};
constexpr int kTile = 16;                          // most rows per CTA

// A CTA handles up to 16 rows of the call, whichever sequences they belong to, and a group of heads: 32 query heads, or eight key
// and value heads, a warp each.  Rows are independent of one another, since a scale belongs to one token.
//
// Bound: qkv read and q, K, V written once (7 chunks of up to 1171 rows, 64 + 16 heads of 128, norms, int8: 60 us, 4.9 TB/s; the key heads'
// doubles and the rotations out of shared memory keep it from more).  Two rotary halves of eight channels per lane make every access 16 bytes.
// Queries are rotated in fp32.  Keys are normalised and rotated in double and rounded to fp32 and then to bf16, so that the codes,
// which are whole numbers made from them, come out the same everywhere but for values within 1e-11 of a rounding border.
template <int D, int F>
__global__ void __launch_bounds__(kThreads, 3) cache_append_kernel(const AppendParams p) {
    // No early release of the dependents: an attention kernel may read the cache without waiting for the grid dependency, which is
    // sound only if the kernel that writes the cache has finished before anything later starts.
    typedef Lanes<D> L;
    constexpr int kHalf = D / 2;
    // A row's rotation per pair, the gains of the head norms multiplied in: x' = x A - y B, y' = y C + x E.  Stored so that
    // the lanes of a token read neighbouring words; queries' in pairs, for the packed arithmetic.
    __shared__ __align__(16) union Rotation {
        float4 q[kTile][4][2][L::kPer];            // pairs 8 l + 2 k, + 1: (A, A', -B, -B'), (C, C', E, E') at [row][k][0, 1][l]
        double2 k[kTile][8][2][L::kPer];           // (A, B), (C, E)
    } rot;
    __shared__ int s_pos[kTile];                   // position that the row's rotation goes by
    __shared__ long long s_slot[kTile];            // (page * Hkv) * 16 + slot: plus 16 g the place of the row's token; -1: bad page, -2: no place
    const int row0 = (int)(blockIdx.x / p.groups) * p.tile, group = (int)(blockIdx.x % p.groups);
    const int nrows = min(p.tile, p.rows - row0);
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const bool kv_part = group < p.kv_ctas;
    pdl_wait();
    for (int r = warp; r < nrows; r += kWarps) {
        const int row = row0 + r;
        const RowSeq at = locate_row(row, p.q_offsets, p.batch);
        long long slot = -2;
        int pos = 0;
        if (!at.padding) {
            const int len = fetch(p.seq_lens + at.b);
            const int o0 = p.q_offsets ? fetch(p.q_offsets + at.b) : row, m = p.q_offsets ? fetch(p.q_offsets + at.b + 1) - o0 : 1;
            const int t = row_position(at, len, p.max_pages);
            if (t < 0 || row < o0 || m > len || (long long)o0 + m > p.rows) {
                if (lane == 0) atomicExch(p.status, AFLEX_ERR_BOUNDS);
            } else {
                pos = p.positions ? fetch(p.positions + row) : t;
                const int page = fetch(p.page_table + (size_t)at.b * p.max_pages + t / kPageTokens);
                const bool ok = page >= 0 && page < p.num_pages;
                if (!ok && lane == 0) atomicExch(p.status, AFLEX_ERR_BOUNDS);
                slot = ok ? (long long)page * p.Hkv * kPageTokens + t % kPageTokens : -1;
            }
        }
        if (lane == 0) { s_slot[r] = slot; s_pos[r] = pos; }
    }
    __syncthreads();
    const int heads = p.Hq + 2 * p.Hkv;
    const int sub = lane / L::kPer, l = lane % L::kPer;
    // Rotations: angle and its reduction to [-pi, pi] in double (two-term 2 pi); a thread makes one pair's of four rows.
    const int c_rot = tid % kHalf, r_rot = 4 * (tid / kHalf);
    auto reduced = [&](int r, int c) -> double {
        const double ang = (double)s_pos[r] * p.inv_freq[c];
        const double turns = rint(ang * 0.15915494309189535);
        return fma(-turns, 2.4492935982947064e-16, fma(-turns, 6.283185307179586, ang));
    };
    if (!kv_part) {
        // ---- query heads.  The warps are dealt out over rows and heads, two times kTok heads of a row at once; the next ones
        // are loaded while these are rotated (the first ones while the rotations are made).
        const int h_lo = (group - p.kv_ctas) * p.q_heads_per_cta, h_hi = min(p.Hq, h_lo + p.q_heads_per_cta);
        const int along = nrows >= 8 ? 1 : nrows >= 4 ? 2 : nrows >= 2 ? 4 : 8;              // warps along the heads of a row
        const int h_first = h_lo + (warp & (along - 1)) * 2 * L::kTok + sub, h_step = along * 2 * L::kTok;
        const int r_first = warp / along, r_step = kWarps / along;
        uint4 xa[2], xb[2];
        auto load = [&](int r, int h) {
            const uint4* src = reinterpret_cast<const uint4*>(p.qkv + (size_t)(row0 + r) * heads * D) + l;
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const uint4* s = src + min(h + u * L::kTok, h_hi - 1) * (D / 8);
                xa[u] = fetch(s);
                xb[u] = fetch(s + D / 16);
            }
        };
        if (r_first < nrows) load(r_first, h_first);
        if (r_rot < nrows) {
            const int c = c_rot;
            const float ga = p.w_qn ? __bfloat162float(p.w_qn[c]) : 1.f, gc = p.w_qn ? __bfloat162float(p.w_qn[kHalf + c]) : 1.f;
            for (int r = r_rot; r < min(nrows, r_rot + 4); ++r) {
                float* z = reinterpret_cast<float*>(&rot.q[r][(c & 7) >> 1][0][c >> 3]) + (c & 1);
                float sn, cs;                      // (each row's from its own angle: it does not depend on which rows came with it)
                sincosf((float)reduced(r, c), &sn, &cs);
                z[0] = ga * cs; z[2] = -gc * sn;
                z += 4 * L::kPer;
                z[0] = gc * cs; z[2] = ga * sn;
            }
        }
        __syncthreads();
        for (int r = r_first; r < nrows; r += r_step) {
            const bool place = s_slot[r] != -2;
            // (h_first - sub is the same for the whole warp)
            for (int h = h_first; h - sub < h_hi; h += h_step) {
                uint32_t va[2][4], vc[2][4];
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    va[u][0] = xa[u].x; va[u][1] = xa[u].y; va[u][2] = xa[u].z; va[u][3] = xa[u].w;
                    vc[u][0] = xb[u].x; vc[u][1] = xb[u].y; vc[u][2] = xb[u].z; vc[u][3] = xb[u].w;
                }
                if (h - sub + h_step < h_hi) load(r, h + h_step);
                else if (r + r_step < nrows) load(r + r_step, h_first);
                uint64_t rinv[2];
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    float ri = 1.f;
                    if (p.w_qn) {
                        uint64_t s2 = 0;
#pragma unroll
                        for (int k = 0; k < 4; ++k) {
                            const uint64_t a = widen_bf16x2(va[u][k]), c = widen_bf16x2(vc[u][k]);
                            s2 = fma_f32x2(a, a, fma_f32x2(c, c, s2));
                        }
                        float s0, s1;
                        unpack_f32x2(s2, s0, s1);
                        float ss = s0 + s1;
#pragma unroll
                        for (int off = 1; off < L::kPer; off <<= 1) ss += __shfl_xor_sync(0xffffffffu, ss, off);
                        ri = rsqrtf(ss / (float)D + p.eps);
                    }
                    rinv[u] = pack_f32x2(ri, ri);
                }
                // the pair's rotation is read once for both heads, the result takes the input's place
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const ulonglong2 z0 = *reinterpret_cast<const ulonglong2*>(&rot.q[r][k][0][l]);
                    const ulonglong2 z1 = *reinterpret_cast<const ulonglong2*>(&rot.q[r][k][1][l]);
#pragma unroll
                    for (int u = 0; u < 2; ++u) {
                        const uint64_t a = widen_bf16x2(va[u][k]), c = widen_bf16x2(vc[u][k]);
                        float x0, x1, y0, y1;
                        unpack_f32x2(mul_f32x2(fma_f32x2(a, z0.x, mul_f32x2(c, z0.y)), rinv[u]), x0, x1);
                        unpack_f32x2(mul_f32x2(fma_f32x2(c, z1.x, mul_f32x2(a, z1.y)), rinv[u]), y0, y1);
                        va[u][k] = pack_bf16x2(x0, x1);
                        vc[u][k] = pack_bf16x2(y0, y1);
                    }
                }
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    if (place && h + u * L::kTok < h_hi) {
                        uint4* dst = reinterpret_cast<uint4*>(p.q_out + ((size_t)(row0 + r) * p.Hq + h + u * L::kTok) * D);
                        dst[l] = make_uint4(va[u][0], va[u][1], va[u][2], va[u][3]);
                        dst[D / 16 + l] = make_uint4(vc[u][0], vc[u][1], vc[u][2], vc[u][3]);
                    }
                }
            }
        }
        return;
    }
    // ---- a key or value head per warp, loaded before the rotations are made; values are stored as they are
    const int i = group * kWarps + warp, g = i < p.Hkv ? i : i - p.Hkv;
    const bool is_key = i < p.Hkv, works = i < 2 * p.Hkv;
    uint4 xa[L::kIter], xb[L::kIter];
    if (works) {
#pragma unroll
        for (int it = 0; it < L::kIter; ++it) {
            if (it * L::kTok >= nrows) break;
            const int t = min(it * L::kTok + sub, nrows - 1);
            const uint4* src = reinterpret_cast<const uint4*>(p.qkv + ((size_t)(row0 + t) * heads + p.Hq + i) * D);
            xa[it] = fetch(src + l);
            xb[it] = fetch(src + D / 16 + l);
        }
    }
    if (group * kWarps < p.Hkv) {                                   // (some of this CTA's heads are keys)
        if (r_rot < nrows) {
            const int c = c_rot;
            const double ga = p.w_kn ? __bfloat162float(p.w_kn[c]) : 1.f, gc = p.w_kn ? __bfloat162float(p.w_kn[kHalf + c]) : 1.f;
            double sn = 0.0, cs = 1.0;
            for (int r = r_rot; r < min(nrows, r_rot + 4); ++r) {
                // the row behind, one position on or at the same one, needs no sine of its own
                const long long on = r > r_rot ? (long long)s_pos[r] - s_pos[r - 1] : -1;
                if (on == 1) {
                    const double next = cs * p.step_cos[c] - sn * p.step_sin[c];
                    sn = sn * p.step_cos[c] + cs * p.step_sin[c];
                    cs = next;
                } else if (on != 0) {
                    sincos(reduced(r, c), &sn, &cs);
                }
                rot.k[r][c & 7][0][c >> 3] = make_double2(ga * cs, gc * sn);
                rot.k[r][c & 7][1][c >> 3] = make_double2(gc * cs, ga * sn);
            }
        }
        __syncthreads();
    }
    if (!works) return;
#pragma unroll
    for (int it = 0; it < L::kIter; ++it) {
        if (it * L::kTok >= nrows) break;
        const int t = min(it * L::kTok + sub, nrows - 1);
        if (is_key) {
            const __nv_bfloat16* pa = reinterpret_cast<const __nv_bfloat16*>(&xa[it]);
            const __nv_bfloat16* pb = reinterpret_cast<const __nv_bfloat16*>(&xb[it]);
            double rinv = 1.0;
            if (p.w_kn) {
                double ss = 0.0;
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    const double a = __bfloat162float(pa[k]), c = __bfloat162float(pb[k]);
                    ss = fma(a, a, fma(c, c, ss));
                }
#pragma unroll
                for (int off = 1; off < L::kPer; off <<= 1) ss += __shfl_xor_sync(0xffffffffu, ss, off);
                rinv = rsqrt(ss / (double)D + (double)p.eps);
            }
            uint4 oa, ob;
            __nv_bfloat16* qa = reinterpret_cast<__nv_bfloat16*>(&oa);
            __nv_bfloat16* qb = reinterpret_cast<__nv_bfloat16*>(&ob);
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const double a = __bfloat162float(pa[k]), c = __bfloat162float(pb[k]);
                const double2 z0 = rot.k[t][k][0][l], z1 = rot.k[t][k][1][l];
                qa[k] = __float2bfloat16_rn((float)((a * z0.x - c * z0.y) * rinv));
                qb[k] = __float2bfloat16_rn((float)((c * z1.x + a * z1.y) * rinv));
            }
            xa[it] = oa;
            xb[it] = ob;
        }
        const long long slot = s_slot[t];
        store_head<D, F>(is_key ? p.k_cache : p.v_cache, is_key ? p.k_scales : p.v_scales, (size_t)(slot + (long long)g * kPageTokens), l, xa[it], xb[it],
                         slot >= 0 && it * L::kTok + sub < nrows);
    }
}

// ------------------------------------------------------------------------------------------ conversion
struct ConvertParams {
    const void* src_k; const void* src_v;
    const float* src_ks; const float* src_vs;
    void* dst_k; void* dst_v;
    float* dst_ks; float* dst_vs;
    const int32_t* src_table; const int32_t* dst_table;
    const int32_t* seq_lens;
    const int32_t* first_token;    // [batch] or null
    int src_max, dst_max, Hkv, pages_per_cta;
    long long src_pages, dst_pages;
    int* status;
};

// A CTA takes a run of pages of one sequence (their ids are looked up once), a warp every eighth (page, KV head, K or V) of it and
// holds its 16 tokens in registers.  Bound: the read of one cache and the write of the other (32 caches of up to 4096 tokens, 8 heads of
// 128, to int8: 76 us, 6.1 TB/s).
template <int D, int F, bool kBack>                 // F: the format of the 8-bit cache; kBack: it is the source
__global__ void __launch_bounds__(kThreads) cache_convert_kernel(const ConvertParams p) {
    typedef Lanes<D> L;
    pdl_wait();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, b = blockIdx.y;
    const int first_page = blockIdx.x * p.pages_per_cta, my_page = first_page + lane;     // lane i holds the run's i-th page
    const int raw = fetch(p.seq_lens + b), most = min(p.src_max, p.dst_max);
    const int from = p.first_token ? max(0, fetch(p.first_token + b)) : 0;
    const bool mine = lane < p.pages_per_cta && my_page < most;
    const int src_id = mine ? fetch(p.src_table + (size_t)b * p.src_max + my_page) : 0;
    const int dst_id = mine ? fetch(p.dst_table + (size_t)b * p.dst_max + my_page) : 0;
    const bool bad_len = raw < 0 || raw > most * kPageTokens;
    if (bad_len && blockIdx.x == 0 && threadIdx.x == 0) atomicExch(p.status, AFLEX_ERR_BOUNDS);
    const int len = bad_len ? 0 : raw;
    const int pages = min(p.pages_per_cta, (len + kPageTokens - 1) / kPageTokens - first_page);
    if (pages <= 0) return;
    // Tokens [lo, hi) of this lane's page
    int lo = max(0, min(kPageTokens, from - my_page * kPageTokens)), hi = lane < pages ? min(kPageTokens, len - my_page * kPageTokens) : 0;
    if (lo < hi && (src_id < 0 || src_id >= p.src_pages || dst_id < 0 || dst_id >= p.dst_pages)) { atomicExch(p.status, AFLEX_ERR_BOUNDS); hi = lo; }
    const int sub = lane / L::kPer, l = lane % L::kPer;
    const int items = pages * 2 * p.Hkv;
    for (int i = warp; i < items; i += kWarps) {
        const int page = i / (2 * p.Hkv), head = i % (2 * p.Hkv), g = head % p.Hkv;
        const bool is_v = head >= p.Hkv;
        const int t0 = __shfl_sync(0xffffffffu, lo, page), t1 = __shfl_sync(0xffffffffu, hi, page);
        const size_t from_slab = (size_t)__shfl_sync(0xffffffffu, src_id, page) * p.Hkv + g, to_slab = (size_t)__shfl_sync(0xffffffffu, dst_id, page) * p.Hkv + g;
        if (t0 >= t1) continue;
        const void* src = is_v ? p.src_v : p.src_k;
        void* dst = is_v ? p.dst_v : p.dst_k;
        if (!kBack) {
            uint4 xa[L::kIter], xb[L::kIter];
#pragma unroll
            for (int it = 0; it < L::kIter; ++it) {
                const int t = max(t0, min(t1 - 1, it * L::kTok + sub));       // a token outside repeats one inside
                const uint4* x = reinterpret_cast<const uint4*>(src) + (from_slab * kPageTokens + t) * (D / 8) + l;
                xa[it] = fetch(x);
                xb[it] = fetch(x + D / 16);
            }
#pragma unroll
            for (int it = 0; it < L::kIter; ++it) {
                const int t = it * L::kTok + sub;
                store_head<D, F>(dst, is_v ? p.dst_vs : p.dst_ks, to_slab * kPageTokens + t, l, xa[it], xb[it], t >= t0 && t < t1);
            }
        } else {
            uint2 ca[L::kIter], cb[L::kIter];
            float s[L::kIter];
#pragma unroll
            for (int it = 0; it < L::kIter; ++it) {
                const size_t t = from_slab * kPageTokens + max(t0, min(t1 - 1, it * L::kTok + sub));
                const uint2* x = reinterpret_cast<const uint2*>(reinterpret_cast<const uint8_t*>(src) + t * D) + l;
                ca[it] = fetch(x);
                cb[it] = fetch(x + D / 16);
                s[it] = fetch((is_v ? p.src_vs : p.src_ks) + t);
            }
#pragma unroll
            for (int it = 0; it < L::kIter; ++it) {
                const int t = it * L::kTok + sub;
                const uint2 a0 = values4<F>(ca[it].x, s[it]), a1 = values4<F>(ca[it].y, s[it]);
                const uint2 b0 = values4<F>(cb[it].x, s[it]), b1 = values4<F>(cb[it].y, s[it]);
                if (t >= t0 && t < t1) {
                    uint4* out = reinterpret_cast<uint4*>(dst) + (to_slab * kPageTokens + t) * (D / 8) + l;
                    out[0] = make_uint4(a0.x, a0.y, a1.x, a1.y);
                    out[D / 16] = make_uint4(b0.x, b0.y, b1.x, b1.y);
                }
            }
        }
    }
}

// ------------------------------------------------------------------------------------------ acceptance
constexpr int kAcceptCaches = 64;                  // caches per launch
struct AcceptCache { uint8_t* k; uint8_t* v; float* ks; float* vs; const int32_t* table; const int32_t* lens; long long num_pages; int max_pages; };
template <int N> struct AcceptParams {             // of up to N caches: a launch copies all of its arguments
    AcceptCache cache[N];
    const int32_t* base; const int32_t* path; const int32_t* count;
    int batch, stride, Hkv, row_bytes;
    int* status;
};

// A warp moves one (sequence, KV head, K or V) of one cache, 16-byte words of four to sixteen tokens at a time.  The path ascends,
// so a token never moves up: a source that is still to be read lies behind every place that has been written, and within a step all
// reads come before the writes.  Bound: the chain of dependent loads (path -> page ids -> tokens); a tree's path is a few KB per head.  64 int8
// caches of 32 sequences, 64 of whose 128 path tokens move (17.4 MB read and written), take 13.8 us (1.3 TB/s).  Without the look at every page before
// the first move it was 12.9, and with 4, 6 or 8 CTAs per SM 13.5, 13.8 and 14.0 (the last two spill).
template <int N> __global__ void __launch_bounds__(kThreads, 5) cache_accept_kernel(const __grid_constant__ AcceptParams<N> p) {
    pdl_wait();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int per = (2 * p.Hkv + kWarps - 1) / kWarps, b = blockIdx.x / per, head = (int)(blockIdx.x % per) * kWarps + warp;
    const AcceptCache& c = p.cache[blockIdx.y];
    if (head >= 2 * p.Hkv) return;
    const int32_t* path = p.path + (size_t)b * p.stride;
    const int n = fetch(p.count + b), base = fetch(p.base + b), len = fetch(c.lens + b);
    auto from_path = [&](int k) -> int { return k < p.stride ? fetch(path + k) : 0; };
    const int first = from_path(lane);             // (whatever the length: no second trip to memory for most paths)
    const int g = head % p.Hkv;
    uint8_t* data = head < p.Hkv ? c.k : c.v;
    float* scales = head < p.Hkv ? c.ks : c.vs;
    const int words = p.row_bytes / 16, at_once = 32 / words, w = lane % words;         // 16-byte words of a token's head; tokens per access
    const int32_t* table = c.table + (size_t)b * c.max_pages;
    auto place = [&](int t) -> int {                                                       // of a token: (page, head, slot), below 2^31; -1 for a bad page id
        const int page = fetch(table + t / kPageTokens);
        return page >= 0 && page < c.num_pages ? (page * p.Hkv + g) * kPageTokens + t % kPageTokens : -1;
    };
    // the whole path is looked at before anything moves: it has to ascend inside the sequence, and every page of a move has to be one
    bool bad = n < 0 || n > p.stride || base < 0 || len < 0 || len > c.max_pages * kPageTokens;
    int before = -1, first_from = -1, first_to = -1;       // (places of the first 32 moves, which most paths do not exceed)
    for (int k0 = 0; k0 < n && !bad; k0 += 32) {
        const int k = k0 + lane, s = k0 == 0 ? first : from_path(k);
        int last = __shfl_up_sync(0xffffffffu, s, 1);
        if (lane == 0) last = before;
        before = __shfl_sync(0xffffffffu, s, 31);
        bad = __any_sync(0xffffffffu, k < n && (s <= last || (long long)base + s >= len));
        if (bad) break;
        int from = -1, to = -1;
        if (k < n && s != k) { from = place(base + s); to = place(base + k); }
        bad = __any_sync(0xffffffffu, k < n && s != k && (from < 0 || to < 0));
        if (k0 == 0) { first_from = from; first_to = to; }
    }
    if (bad) {
        if (lane == 0) atomicExch(p.status, AFLEX_ERR_BOUNDS);
        return;
    }
    for (int k0 = 0; k0 < n; k0 += 32) {
        // lane i knows the k0 + i-th move
        int from = first_from, to = first_to;
        if (k0 > 0) {
            const int k = k0 + lane, s = from_path(k);
            const bool moves = k < n && s != k;
            from = moves ? place(base + s) : -1;
            to = moves ? place(base + k) : -1;
        }
        const uint32_t moves = __ballot_sync(0xffffffffu, from >= 0);
        if (moves == 0) continue;
        float scale = 0.f;
        if (scales != nullptr && from >= 0) scale = scales[from];
        for (int i0 = 0; i0 < 32 && moves >> i0 != 0; i0 += 4 * at_once) {
            uint4 x[4];
            int dst[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const int i = i0 + u * at_once + lane / words;
                const int src = __shfl_sync(0xffffffffu, from, i);
                dst[u] = __shfl_sync(0xffffffffu, to, i);
                if (src >= 0) x[u] = *reinterpret_cast<const uint4*>(data + (size_t)src * p.row_bytes + w * 16);
            }
            __syncwarp();
#pragma unroll
            for (int u = 0; u < 4; ++u)
                if (dst[u] >= 0) *reinterpret_cast<uint4*>(data + (size_t)dst[u] * p.row_bytes + w * 16) = x[u];
            __syncwarp();
        }
        if (scales != nullptr && to >= 0) scales[to] = scale;
        __syncwarp();
    }
}

template <int D, int F> void (*append_of())(const AppendParams) { return cache_append_kernel<D, F>; }

}  // namespace

// ------------------------------------------------------------------------------------------ host
void rope_tables(aflex_ctx* ctx, float theta, int head_dim) {
    if (ctx->rope_theta == theta && ctx->rope_dim == head_dim) return;
    for (int i = 0; i < head_dim / 2; ++i) {
        ctx->rope_freq[i] = pow((double)theta, -2.0 * i / (double)head_dim);
        ctx->rope_step[0][i] = cos(ctx->rope_freq[i]);
        ctx->rope_step[1][i] = sin(ctx->rope_freq[i]);
    }
    ctx->rope_theta = theta;
    ctx->rope_dim = head_dim;
}

aflex_status cache_append_launch(aflex_ctx* ctx, const aflex_attn_desc* d, const void* qkv, const aflex_cache* cache, int batch,
                                 const aflex_draft* draft, int rows, const void* w_qn, const void* w_kn, float eps, float theta,
                                 void* q_out, cudaStream_t st) {
    AppendParams p;
    const aflex_kv* kv = &cache->kv;
    p.qkv = (const __nv_bfloat16*)qkv;
    p.w_qn = (const __nv_bfloat16*)w_qn; p.w_kn = (const __nv_bfloat16*)w_kn;
    p.page_table = kv->page_table; p.seq_lens = kv->seq_lens;
    p.q_offsets = draft ? draft->q_offsets : nullptr;
    p.positions = draft ? draft->positions : nullptr;
    p.batch = batch; p.rows = rows; p.max_pages = kv->max_pages_per_seq;
    p.Hq = d->num_q_heads; p.Hkv = d->num_kv_heads; p.num_pages = kv->num_pages;
    p.q_out = (__nv_bfloat16*)q_out;
    p.k_cache = const_cast<void*>(kv->k_cache); p.v_cache = const_cast<void*>(kv->v_cache);
    p.k_scales = cache->k_scales; p.v_scales = cache->v_scales;
    p.eps = eps;
    rope_tables(ctx, theta, d->head_dim);
    for (int i = 0; i < 64; ++i) { p.inv_freq[i] = ctx->rope_freq[i]; p.step_cos[i] = ctx->rope_step[0][i]; p.step_sin[i] = ctx->rope_step[1][i]; }
    p.status = ctx->dev_status;
    p.kv_ctas = (2 * p.Hkv + kWarps - 1) / kWarps;
    p.q_heads_per_cta = p.Hq < 32 ? p.Hq : 32;
    p.groups = p.kv_ctas + (p.Hq + p.q_heads_per_cta - 1) / p.q_heads_per_cta;
    // Rows per CTA: 16, which share what a CTA costs, or as few as still make two CTAs per SM.
    p.tile = kTile;
    while (p.tile > 1 && (long long)rows * p.groups < 2LL * ctx->num_sms * p.tile) p.tile /= 2;
    const long long ctas = ((long long)rows + p.tile - 1) / p.tile * p.groups;
    if (ctas > 0x7fffffffLL) return set_error(ctx, AFLEX_ERR_UNSUPPORTED, "cache append: rows = %d", rows);
    typedef void (*Kernel)(const AppendParams);
    const Kernel kernels[2][3] = {{append_of<64, AFLEX_CACHE_BF16>(), append_of<64, AFLEX_CACHE_INT8>(), append_of<64, AFLEX_CACHE_E4M3>()},
                                  {append_of<128, AFLEX_CACHE_BF16>(), append_of<128, AFLEX_CACHE_INT8>(), append_of<128, AFLEX_CACHE_E4M3>()}};
    KernelScope scope(ctx, kKCacheAppend, st);
    return check_cuda(ctx, launch_pdl(kernels[d->head_dim == 128][cache->format], dim3((unsigned)ctas), dim3(kThreads), 0, st, p),
                      "cache_append_kernel launch");
}

aflex_status cache_convert_launch(aflex_ctx* ctx, const aflex_attn_desc* d, const aflex_cache* src, const aflex_cache* dst, int batch,
                                  const int32_t* first_token, cudaStream_t st) {
    ConvertParams p;
    p.src_k = src->kv.k_cache; p.src_v = src->kv.v_cache; p.src_ks = src->k_scales; p.src_vs = src->v_scales;
    p.dst_k = const_cast<void*>(dst->kv.k_cache); p.dst_v = const_cast<void*>(dst->kv.v_cache); p.dst_ks = dst->k_scales; p.dst_vs = dst->v_scales;
    p.src_table = src->kv.page_table; p.dst_table = dst->kv.page_table;
    p.seq_lens = src->kv.seq_lens; p.first_token = first_token;
    p.src_max = src->kv.max_pages_per_seq; p.dst_max = dst->kv.max_pages_per_seq;
    p.Hkv = d->num_kv_heads; p.src_pages = src->kv.num_pages; p.dst_pages = dst->kv.num_pages;
    p.status = ctx->dev_status;
    const int most = p.src_max < p.dst_max ? p.src_max : p.dst_max;
    // Pages per CTA: one (page, head, K or V) per warp at least; up to four times that where four CTAs per SM are still left.
    const int least = (kWarps + 2 * p.Hkv - 1) / (2 * p.Hkv);
    p.pages_per_cta = least;
    while (p.pages_per_cta < 4 * least && p.pages_per_cta <= 16 && (long long)batch * most >= 2LL * p.pages_per_cta * 4 * ctx->num_sms)
        p.pages_per_cta *= 2;
    const bool back = src->format != AFLEX_CACHE_BF16;
    const int f = back ? src->format : dst->format;
    typedef void (*Kernel)(const ConvertParams);
    const Kernel kernels[2][2][2] = {
        {{cache_convert_kernel<64, AFLEX_CACHE_INT8, false>, cache_convert_kernel<64, AFLEX_CACHE_INT8, true>},
         {cache_convert_kernel<64, AFLEX_CACHE_E4M3, false>, cache_convert_kernel<64, AFLEX_CACHE_E4M3, true>}},
        {{cache_convert_kernel<128, AFLEX_CACHE_INT8, false>, cache_convert_kernel<128, AFLEX_CACHE_INT8, true>},
         {cache_convert_kernel<128, AFLEX_CACHE_E4M3, false>, cache_convert_kernel<128, AFLEX_CACHE_E4M3, true>}}};
    KernelScope scope(ctx, kKCacheConvert, st);
    return check_cuda(ctx, launch_pdl(kernels[d->head_dim == 128][f - 1][back], dim3((unsigned)((most + p.pages_per_cta - 1) / p.pages_per_cta), (unsigned)batch),
                                      dim3(kThreads), 0, st, p),
                      "cache_convert_kernel launch");
}

template <int N>
static aflex_status accept_launch(aflex_ctx* ctx, const aflex_attn_desc* d, const aflex_cache* caches, int num_caches, int batch,
                                  const int32_t* base, const int32_t* path, int path_stride, const int32_t* path_len, cudaStream_t st) {
    AcceptParams<N> p;
    p.base = base; p.path = path; p.count = path_len;
    p.batch = batch; p.stride = path_stride; p.Hkv = d->num_kv_heads;
    p.row_bytes = d->head_dim * (caches[0].format == AFLEX_CACHE_BF16 ? 2 : 1);
    p.status = ctx->dev_status;
    const long long ctas = (long long)batch * ((2 * p.Hkv + kWarps - 1) / kWarps);
    if (ctas > 0x7fffffffLL) return set_error(ctx, AFLEX_ERR_UNSUPPORTED, "cache accept: batch * Hkv");
    for (int l = 0; l < N; ++l) {
        const aflex_cache& c = caches[l < num_caches ? l : 0];
        p.cache[l] = {(uint8_t*)const_cast<void*>(c.kv.k_cache), (uint8_t*)const_cast<void*>(c.kv.v_cache), c.k_scales, c.v_scales,
                      c.kv.page_table, c.kv.seq_lens, (long long)c.kv.num_pages, c.kv.max_pages_per_seq};
    }
    KernelScope scope(ctx, kKCacheAccept, st);
    return check_cuda(ctx, launch_pdl(cache_accept_kernel<N>, dim3((unsigned)ctas, (unsigned)num_caches), dim3(kThreads), 0, st, p), "cache_accept_kernel launch");
}

aflex_status cache_accept_launch(aflex_ctx* ctx, const aflex_attn_desc* d, const aflex_cache* caches, int num_caches, int batch,
                                 const int32_t* base, const int32_t* path, int path_stride, const int32_t* path_len, cudaStream_t st) {
    aflex_status s = AFLEX_OK;
    for (int l0 = 0; l0 < num_caches && s == AFLEX_OK; l0 += kAcceptCaches) {
        const int n = num_caches - l0 < kAcceptCaches ? num_caches - l0 : kAcceptCaches;
        s = n <= 4 ? accept_launch<4>(ctx, d, caches + l0, n, batch, base, path, path_stride, path_len, st)
                   : accept_launch<kAcceptCaches>(ctx, d, caches + l0, n, batch, base, path, path_stride, path_len, st);
    }
    return s;
}

}  // namespace aflex
