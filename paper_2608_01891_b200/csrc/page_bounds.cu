// Key bounds of cache pages, the summary that page selection scores instead of the keys themselves:
//   rope_append_bounds_kernel  rotary embedding + K/V append of one token or a chunk per sequence, and the
//                              bounds of every page it touches, in one pass over q | k | v
//   page_bounds_kernel         the bounds of pages that something else filled
//
// For one page and KV head, over the keys stored so far (as stored, in bf16; NaN is ignored):
//   hi_d = max_j K_j[d], lo_d = min_j K_j[d]
// kept as 8-bit integers with one power-of-two scale per 32 channels: with a = max(|hi|, |lo|) over the block and
// e the smallest integer with a <= 127 * 2^e (within [-60, 50]),
//   HI_d = ceil(hi_d / 2^e), LO_d = floor(lo_d / 2^e), both within [-127, 127]
// so that HI * 2^e and LO * 2^e still bound the keys (unless e had to be clamped at 50).  A page's bounds are a function of
// its stored keys alone: they do not depend on how many calls appended them, which is why an append reads the page's older
// keys (4 KB per head, resident in L2 or one DRAM burst) instead of widening the old bounds.
// Layout [page][KV head][D / 8][HI, LO][8]: 16 bytes hold eight channels of both, which is what one lane of the scoring
// kernel's MMA takes, so it loads its operands straight into registers.
#include <cuda_bf16.h>
#include <math.h>

#include "internal.h"
#include "ptx.cuh"

namespace aflex {

namespace {

constexpr int kBoundsWarps = 8;
constexpr int kBoundsThreads = kBoundsWarps * 32;
constexpr int kPageTokens = 16;

// Lane layout of both kernels: D / 16 lanes hold one token's key, lane l the channels [8 l, 8 l + 8) and
// [D / 2 + 8 l, D / 2 + 8 l + 8) -- the two halves a rotary pair comes from; 32 / (D / 16) tokens per warp at a time.
template <int D> struct Lanes {
    static constexpr int kPer = D / 16;           // lanes per token
    static constexpr int kTok = 32 / kPer;        // tokens per warp at a time
    static constexpr int kIter = kPageTokens / kTok;
};

struct Range16 {                                  // running extremes of this lane's 16 channels, bf16 pairs
    __nv_bfloat162 hi[8], lo[8];
    __device__ __forceinline__ void reset() {
        const __nv_bfloat162 ninf = __halves2bfloat162(__ushort_as_bfloat16(0xff80), __ushort_as_bfloat16(0xff80));
        const __nv_bfloat162 pinf = __halves2bfloat162(__ushort_as_bfloat16(0x7f80), __ushort_as_bfloat16(0x7f80));
#pragma unroll
        for (int i = 0; i < 8; ++i) { hi[i] = ninf; lo[i] = pinf; }
    }
    __device__ __forceinline__ void add(const uint4& a, const uint4& b) {      // a: first half's channels, b: second half's
        const __nv_bfloat162* pa = reinterpret_cast<const __nv_bfloat162*>(&a);
        const __nv_bfloat162* pb = reinterpret_cast<const __nv_bfloat162*>(&b);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            hi[i] = __hmax2(hi[i], pa[i]);         // the other operand where one is NaN
            lo[i] = __hmin2(lo[i], pa[i]);
            hi[4 + i] = __hmax2(hi[4 + i], pb[i]);
            lo[4 + i] = __hmin2(lo[4 + i], pb[i]);
        }
    }
};

// Smallest e with a <= 127 * 2^e, within [-60, 50]; -60 for a == 0.
__device__ __forceinline__ int block_exponent(float a) {
    const int field = (int)((__float_as_uint(a) >> 23) & 255u);
    int e = field - 126 - 7;                       // a * 2^-e in [64, 128)
    // e is far below -60 for the small fields that would not make a normal power of two, far above 50 for infinity
    if (e >= -60 && e <= 50 && a * __uint_as_float((uint32_t)(127 - e) << 23) > 127.f) ++e;
    return max(-60, min(50, e));
}

__device__ __forceinline__ uint32_t pack4(int a, int b, int c, int d) {
    return (uint32_t)(a & 255) | ((uint32_t)(b & 255) << 8) | ((uint32_t)(c & 255) << 16) | ((uint32_t)d << 24);
}

// Joins the lanes' ranges of one (page, KV head) and writes its bounds.  All 32 lanes take part.
template <int D>
__device__ __forceinline__ void store_bounds(Range16& r, int lane, int8_t* codes, uint8_t* scales) {
    constexpr int kPer = Lanes<D>::kPer;
#pragma unroll
    for (int off = kPer; off < 32; off <<= 1) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            r.hi[i] = __hmax2(r.hi[i], __shfl_xor_sync(0xffffffffu, r.hi[i], off));
            r.lo[i] = __hmin2(r.lo[i], __shfl_xor_sync(0xffffffffu, r.lo[i], off));
        }
    }
    const int l = lane % kPer;
#pragma unroll
    for (int half = 0; half < 2; ++half) {
        float hi[8], lo[8], a = 0.f;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float2 h = __bfloat1622float2(r.hi[half * 4 + i]), w = __bfloat1622float2(r.lo[half * 4 + i]);
            hi[2 * i] = h.x; hi[2 * i + 1] = h.y;
            lo[2 * i] = w.x; lo[2 * i + 1] = w.y;
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            if (hi[i] < lo[i]) hi[i] = lo[i] = 0.f;           // no key was a number
            a = fmaxf(a, fmaxf(fabsf(hi[i]), fabsf(lo[i])));
        }
        a = fmaxf(a, __shfl_xor_sync(0xffffffffu, a, 1));      // the four lanes of a 32-channel block
        a = fmaxf(a, __shfl_xor_sync(0xffffffffu, a, 2));
        const int e = block_exponent(a);
        const float inv = __uint_as_float((uint32_t)(127 - e) << 23);
        int ih[8], il[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            ih[i] = (int)fminf(127.f, fmaxf(-127.f, ceilf(hi[i] * inv)));
            il[i] = (int)fminf(127.f, fmaxf(-127.f, floorf(lo[i] * inv)));
        }
        if (lane < kPer) {
            uint4 o;
            o.x = pack4(ih[0], ih[1], ih[2], ih[3]); o.y = pack4(ih[4], ih[5], ih[6], ih[7]);
            o.z = pack4(il[0], il[1], il[2], il[3]); o.w = pack4(il[4], il[5], il[6], il[7]);
            reinterpret_cast<uint4*>(codes)[half * kPer + l] = o;
            if ((l & 3) == 0) scales[half * (D / 64) + l / 4] = (uint8_t)(e + 127);
        }
    }
}

struct BoundsParams {
    const __nv_bfloat16* k_cache;
    int8_t* codes;
    uint8_t* scales;
    const int32_t* page_table;
    const int32_t* seq_lens;
    const int32_t* first_token;    // [batch] or null
    int max_pages, Hkv, heads_per_warp;
    long long num_pages;
    int* status;
};

// One warp per (sequence, page) and run of KV heads: a head's 16 keys are 8 sixteen-byte loads per lane (D = 128), and the next
// head's are in flight while one is reduced.  Bound: the read of the keys.
template <int D>
__global__ void __launch_bounds__(kBoundsThreads) page_bounds_kernel(const BoundsParams p) {
    pdl_launch_dependents();
    pdl_wait();
    typedef Lanes<D> L;
    const int lane = threadIdx.x & 31;
    const int runs = (p.Hkv + p.heads_per_warp - 1) / p.heads_per_warp;
    const int item = blockIdx.x * kBoundsWarps + (threadIdx.x >> 5);
    const int page_i = item / runs, b = blockIdx.y;
    if (page_i >= p.max_pages) return;
    const int page = p.page_table[(size_t)b * p.max_pages + page_i];
    const int raw = p.seq_lens[b];
    if (raw < 0 || raw > p.max_pages * kPageTokens) {
        if (item == 0 && lane == 0) atomicExch(p.status, AFLEX_ERR_BOUNDS);
    }
    const int len = max(0, min(raw, p.max_pages * kPageTokens));
    if (page_i * kPageTokens >= len) return;
    if (p.first_token && (page_i + 1) * kPageTokens <= p.first_token[b]) return;     // a page without a new token
    if (page < 0 || page >= p.num_pages) {
        if (lane == 0) atomicExch(p.status, AFLEX_ERR_BOUNDS);
        return;
    }
    const int valid = min(kPageTokens, len - page_i * kPageTokens);
    const int g0 = (item % runs) * p.heads_per_warp, g1 = min(p.Hkv, g0 + p.heads_per_warp);
    const int sub = lane / L::kPer, l = lane % L::kPer;
    uint4 a[L::kIter], c[L::kIter];
    auto load = [&](int g) {
        const uint4* k = reinterpret_cast<const uint4*>(p.k_cache + ((size_t)page * p.Hkv + g) * kPageTokens * D);
#pragma unroll
        for (int it = 0; it < L::kIter; ++it) {
            const int t = min(it * L::kTok + sub, valid - 1);       // a slot past the end repeats the last valid key
            a[it] = __ldg(k + t * (D / 8) + l);
            c[it] = __ldg(k + t * (D / 8) + D / 16 + l);
        }
    };
    load(g0);
    for (int g = g0; g < g1; ++g) {
        Range16 r;
        r.reset();
#pragma unroll
        for (int it = 0; it < L::kIter; ++it) r.add(a[it], c[it]);
        if (g + 1 < g1) load(g + 1);
        const size_t slab = (size_t)page * p.Hkv + g;
        store_bounds<D>(r, lane, p.codes + slab * 2 * D, p.scales + slab * (D / 32));
    }
}

struct AppendParams {
    const __nv_bfloat16* qkv;      // [rows][(Hq + 2 Hkv) * D]
    const __nv_bfloat16* w_qn;     // [D] or null
    const __nv_bfloat16* w_kn;     // [D] or null
    const int32_t* page_table;
    const int32_t* seq_lens;
    const int32_t* q_offsets;      // null: one row per sequence
    int batch, rows, max_pages, Hq, Hkv;
    long long num_pages;
    __nv_bfloat16* q_out;
    __nv_bfloat16* k_cache;
    __nv_bfloat16* v_cache;
    int8_t* codes;
    uint8_t* scales;
    int q_heads_per_cta, kv_ctas;  // blockIdx.y < kv_ctas: K and V heads, a share each; else query heads
    float eps;
    double inv_freq[64];           // theta^(-2 i / D), formed in double on the host
    int* status;
};

// A CTA handles the rows of ONE page of one sequence (1 to 16 rows), so that whoever rotates the page's keys holds all of
// them when the bounds are formed.  blockIdx.x: the page among the pages touched by the call (located by a scan over the
// sequences), blockIdx.y: a group of heads.
//
// Bound: qkv read and q, K, V written once.  Two rotary halves of eight channels per lane make every access 16 bytes.
// Queries are rotated in fp32.  Keys (one head in ten on the shapes served here) are normalised and rotated in double and
// rounded to fp32 and then to bf16: the stored key no longer depends on the order in which sums were formed (but for values
// within 1e-11 of a rounding border), and the bounds, which are integers made from it, come out the same everywhere.
// U: how many times kTok query heads a warp has in flight.
template <int D, int U>
__global__ void __launch_bounds__(kBoundsThreads, 3) rope_append_bounds_kernel(const AppendParams p) {
    // No early release of the dependents: the dense attention kernel reads the cache without waiting for the grid
    // dependency, which is sound only if the kernel that writes the cache has finished before anything later starts.
    typedef Lanes<D> L;
    constexpr int kHalf = D / 2;
    __shared__ int s_warp[kBoundsWarps];
    __shared__ int s_b, s_page;
    __shared__ __align__(16) float2 s_rot[kPageTokens][kHalf];      // (cos, sin), queries
    __shared__ double2 s_rotd[kPageTokens][kHalf];                  // keys
    pdl_wait();
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    int b, page_i, row0, nrows, slot0;                              // rows row0 .. of the call go to slots slot0 .. of the page
    if (p.q_offsets == nullptr) {
        b = blockIdx.x;
        const int len = p.seq_lens[b];
        if (len < 1 || len > p.max_pages * kPageTokens) {
            if (tid == 0) atomicExch(p.status, AFLEX_ERR_BOUNDS);
            return;                                                 // no position to write to
        }
        page_i = (len - 1) / kPageTokens;
        slot0 = (len - 1) % kPageTokens;
        row0 = b; nrows = 1;
    } else {
        // pages touched by sequence i: from that of its first new token to that of its last; thread t owns a run of sequences
        const int per = (p.batch + kBoundsThreads - 1) / kBoundsThreads;
        const int lo = min(p.batch, tid * per), hi = min(p.batch, lo + per);
        auto touched = [&](int i, int& first) -> int {
            const int o0 = p.q_offsets[i], o1 = p.q_offsets[i + 1], m = o1 - o0, len = p.seq_lens[i];
            first = 0;
            if (m == 0) return 0;
            if (m < 0 || o0 < 0 || o1 > p.rows || m > len || len > p.max_pages * kPageTokens) return -1;
            first = (len - m) / kPageTokens;
            return (len - 1) / kPageTokens - first + 1;
        };
        int local = 0, first;
        for (int i = lo; i < hi; ++i) {
            const int c = touched(i, first);
            if (c < 0) { if (blockIdx.x == 0 && blockIdx.y == 0) atomicExch(p.status, AFLEX_ERR_BOUNDS); }
            else local += c;
        }
        int incl = local;
#pragma unroll
        for (int off = 1; off < 32; off <<= 1) {
            const int v = __shfl_up_sync(0xffffffffu, incl, off);
            if (lane >= off) incl += v;
        }
        if (lane == 31) s_warp[warp] = incl;
        if (tid == 0) s_b = -1;
        __syncthreads();
        int before = incl - local;
        for (int w = 0; w < warp; ++w) before += s_warp[w];
        const int want = (int)blockIdx.x;
        if (want >= before && want < before + local) {
            int at = before;
            for (int i = lo; i < hi; ++i) {
                const int c = max(0, touched(i, first));
                if (want < at + c) { s_b = i; s_page = first + (want - at); break; }
                at += c;
            }
        }
        __syncthreads();
        b = s_b;
        if (b < 0) return;                                          // past the last touched page
        page_i = s_page;
        const int o0 = p.q_offsets[b], m = p.q_offsets[b + 1] - o0, len = p.seq_lens[b];
        const int begin = max(len - m, page_i * kPageTokens), end = min(len, (page_i + 1) * kPageTokens);
        slot0 = begin - page_i * kPageTokens;
        row0 = o0 + begin - (len - m);
        nrows = end - begin;
    }
    const int heads = p.Hq + 2 * p.Hkv;
    const bool kv_part = (int)blockIdx.y < p.kv_ctas;
    const int page = p.page_table[(size_t)b * p.max_pages + page_i];
    if (kv_part && (page < 0 || page >= p.num_pages)) {
        if (tid == 0) atomicExch(p.status, AFLEX_ERR_BOUNDS);
        return;
    }
    // the rows' rotations: angle and its reduction to [-pi, pi] in double (two-term 2 pi)
    for (int i = tid; i < nrows * kHalf; i += kBoundsThreads) {
        const int r = i / kHalf, c = i % kHalf;
        const double ang = (double)(page_i * kPageTokens + slot0 + r) * p.inv_freq[c];
        const double turns = rint(ang * 0.15915494309189535);
        const double red = fma(-turns, 2.4492935982947064e-16, fma(-turns, 6.283185307179586, ang));
        if (kv_part) {
            double sn, cs;
            sincos(red, &sn, &cs);
            s_rotd[r][c] = make_double2(cs, sn);
        } else {
            float sn, cs;
            sincosf((float)red, &sn, &cs);
            s_rot[r][c] = make_float2(cs, sn);
        }
    }
    __syncthreads();
    const int sub = lane / L::kPer, l = lane % L::kPer;
    if (!kv_part) {
        // ---- query heads.  A warp takes a row and U * kTok of its heads at a time: one rotation in registers, all loads first.
        const int h_lo = ((int)blockIdx.y - p.kv_ctas) * p.q_heads_per_cta, h_hi = min(p.Hq, h_lo + p.q_heads_per_cta);
        const int groups = (h_hi - h_lo + U * L::kTok - 1) / (U * L::kTok);
        float gn[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) gn[i] = 1.f;
        if (p.w_qn) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                gn[i] = __bfloat162float(p.w_qn[8 * l + i]);
                gn[8 + i] = __bfloat162float(p.w_qn[kHalf + 8 * l + i]);
            }
        }
        for (int task = warp; task < nrows * groups; task += kBoundsWarps) {
            const int r = task / groups, h0 = h_lo + (task % groups) * (U * L::kTok) + sub;
            const uint4* src = reinterpret_cast<const uint4*>(p.qkv + (size_t)(row0 + r) * heads * D) + l;
            uint4 xa[U], xb[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int h = min(h0 + u * L::kTok, h_hi - 1);
                xa[u] = __ldg(src + h * (D / 8));
                xb[u] = __ldg(src + h * (D / 8) + D / 16);
            }
            float4 cs[4];                                           // (cos, sin) of this lane's eight pairs
#pragma unroll
            for (int k = 0; k < 4; ++k) cs[k] = *reinterpret_cast<const float4*>(&s_rot[r][8 * l + 2 * k]);
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const __nv_bfloat162* pa = reinterpret_cast<const __nv_bfloat162*>(&xa[u]);
                const __nv_bfloat162* pb = reinterpret_cast<const __nv_bfloat162*>(&xb[u]);
                float a[8], c[8], ss = 0.f;
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const float2 x = __bfloat1622float2(pa[k]), y = __bfloat1622float2(pb[k]);
                    a[2 * k] = x.x; a[2 * k + 1] = x.y; c[2 * k] = y.x; c[2 * k + 1] = y.y;
                }
                if (p.w_qn) {
#pragma unroll
                    for (int k = 0; k < 8; ++k) ss = fmaf(a[k], a[k], fmaf(c[k], c[k], ss));
#pragma unroll
                    for (int off = 1; off < L::kPer; off <<= 1) ss += __shfl_xor_sync(0xffffffffu, ss, off);
                    const float rinv = rsqrtf(ss / (float)D + p.eps);
#pragma unroll
                    for (int k = 0; k < 8; ++k) { a[k] *= rinv * gn[k]; c[k] *= rinv * gn[8 + k]; }
                }
                uint4 oa, ob;
                __nv_bfloat162* qa = reinterpret_cast<__nv_bfloat162*>(&oa);
                __nv_bfloat162* qb = reinterpret_cast<__nv_bfloat162*>(&ob);
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    qa[k] = __floats2bfloat162_rn(a[2 * k] * cs[k].x - c[2 * k] * cs[k].y, a[2 * k + 1] * cs[k].z - c[2 * k + 1] * cs[k].w);
                    qb[k] = __floats2bfloat162_rn(c[2 * k] * cs[k].x + a[2 * k] * cs[k].y, c[2 * k + 1] * cs[k].z + a[2 * k + 1] * cs[k].w);
                }
                const int h = h0 + u * L::kTok;
                if (h < h_hi) {
                    uint4* dst = reinterpret_cast<uint4*>(p.q_out + ((size_t)(row0 + r) * p.Hq + h) * D);
                    dst[l] = oa;
                    dst[D / 16 + l] = ob;
                }
            }
        }
        return;
    }
    // ---- value heads: copied as they are; key heads: a warp each
    const int step = p.kv_ctas * kBoundsWarps;
    for (int i = (int)blockIdx.y * kBoundsWarps + warp; i < 2 * p.Hkv; i += step) {
        const int g = i < p.Hkv ? i : i - p.Hkv;
        const size_t slab = (size_t)page * p.Hkv + g;
        if (i >= p.Hkv) {
            const uint4* src = reinterpret_cast<const uint4*>(p.qkv + ((size_t)row0 * heads + p.Hq + p.Hkv + g) * D);
            uint4* dst = reinterpret_cast<uint4*>(p.v_cache + (slab * kPageTokens + slot0) * D);
            uint4 v[kPageTokens * D / 256];
#pragma unroll
            for (int k = 0; k < kPageTokens * D / 256; ++k) {
                const int j = k * 32 + lane, r = j / (D / 8);
                if (r < nrows) v[k] = __ldg(src + (size_t)r * heads * (D / 8) + j % (D / 8));
            }
#pragma unroll
            for (int k = 0; k < kPageTokens * D / 256; ++k) {
                const int j = k * 32 + lane;
                if (j / (D / 8) < nrows) dst[j] = v[k];
            }
            continue;
        }
        uint4* kd = reinterpret_cast<uint4*>(p.k_cache + slab * kPageTokens * D);
        const int end = slot0 + nrows;                              // slots [0, slot0) hold older keys, [slot0, end) are new
        uint4 xa[L::kIter], xb[L::kIter];
#pragma unroll
        for (int it = 0; it < L::kIter; ++it) {
            const int t = min(it * L::kTok + sub, end - 1);
            const uint4* src = t < slot0 ? kd + t * (D / 8)
                                         : reinterpret_cast<const uint4*>(p.qkv + ((size_t)(row0 + t - slot0) * heads + p.Hq + g) * D);
            xa[it] = src[l];
            xb[it] = src[D / 16 + l];
        }
        Range16 range;
        range.reset();
#pragma unroll
        for (int it = 0; it < L::kIter; ++it) {
            const int t0 = it * L::kTok;
            if (t0 >= end) break;
            const int t = min(t0 + sub, end - 1);
            if (t0 + L::kTok > slot0) {                             // some of these tokens are new (the same for the whole warp)
                const int r = max(0, t - slot0);
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
                    rinv = 1.0 / sqrt(ss / (double)D + (double)p.eps);
                }
                uint4 oa, ob;
                __nv_bfloat16* qa = reinterpret_cast<__nv_bfloat16*>(&oa);
                __nv_bfloat16* qb = reinterpret_cast<__nv_bfloat16*>(&ob);
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    double a = __bfloat162float(pa[k]), c = __bfloat162float(pb[k]);
                    if (p.w_kn) {
                        a *= rinv * (double)__bfloat162float(p.w_kn[8 * l + k]);
                        c *= rinv * (double)__bfloat162float(p.w_kn[kHalf + 8 * l + k]);
                    }
                    const double2 rot = s_rotd[r][8 * l + k];
                    qa[k] = __float2bfloat16_rn((float)(a * rot.x - c * rot.y));
                    qb[k] = __float2bfloat16_rn((float)(c * rot.x + a * rot.y));
                }
                if (t >= slot0) {
                    xa[it] = oa;
                    xb[it] = ob;
                    if (t0 + sub < end) {
                        kd[t * (D / 8) + l] = oa;
                        kd[t * (D / 8) + D / 16 + l] = ob;
                    }
                }
            }
            range.add(xa[it], xb[it]);
        }
        store_bounds<D>(range, lane, p.codes + slab * 2 * D, p.scales + slab * (D / 32));
    }
}

}  // namespace

// ------------------------------------------------------------------------------------------ host
aflex_status page_bounds_launch(aflex_ctx* ctx, const aflex_attn_desc* d, const aflex_kv* kv, const aflex_key_bounds* bounds,
                                int batch, const int32_t* first_token, cudaStream_t st) {
    BoundsParams p;
    p.k_cache = (const __nv_bfloat16*)kv->k_cache;
    p.codes = bounds->codes; p.scales = bounds->scales;
    p.page_table = kv->page_table; p.seq_lens = kv->seq_lens; p.first_token = first_token;
    p.max_pages = kv->max_pages_per_seq; p.Hkv = d->num_kv_heads; p.num_pages = kv->num_pages;
    p.status = ctx->dev_status;
    // all heads of a page on one warp where that still leaves 16 warps per SM, fewer of them where there are few pages
    const long long pages = (long long)batch * p.max_pages;
    p.heads_per_warp = 1;
    while (p.heads_per_warp < p.Hkv && pages * p.Hkv >= 2LL * p.heads_per_warp * 16 * ctx->num_sms) p.heads_per_warp *= 2;
    const long long items = (long long)p.max_pages * ((p.Hkv + p.heads_per_warp - 1) / p.heads_per_warp);
    const dim3 grid((unsigned)((items + kBoundsWarps - 1) / kBoundsWarps), (unsigned)batch);
    KernelScope scope(ctx, kKPageBounds, st);
    return check_cuda(ctx, launch_pdl(d->head_dim == 128 ? page_bounds_kernel<128> : page_bounds_kernel<64>, grid, dim3(kBoundsThreads), 0, st, p),
                      "page_bounds_kernel launch");
}

aflex_status rope_append_bounds_launch(aflex_ctx* ctx, const aflex_attn_desc* d, const void* qkv, const aflex_kv* kv,
                                       const aflex_key_bounds* bounds, int batch, const int32_t* q_offsets, int rows,
                                       const void* w_qn, const void* w_kn, float eps, float theta, void* q_out, cudaStream_t st) {
    AppendParams p;
    p.qkv = (const __nv_bfloat16*)qkv;
    p.w_qn = (const __nv_bfloat16*)w_qn; p.w_kn = (const __nv_bfloat16*)w_kn;
    p.page_table = kv->page_table; p.seq_lens = kv->seq_lens; p.q_offsets = q_offsets;
    p.batch = batch; p.rows = rows; p.max_pages = kv->max_pages_per_seq;
    p.Hq = d->num_q_heads; p.Hkv = d->num_kv_heads; p.num_pages = kv->num_pages;
    p.q_out = (__nv_bfloat16*)q_out;
    p.k_cache = (__nv_bfloat16*)const_cast<void*>(kv->k_cache);
    p.v_cache = (__nv_bfloat16*)const_cast<void*>(kv->v_cache);
    p.codes = bounds->codes; p.scales = bounds->scales;
    p.eps = eps;
    for (int i = 0; i < 64; ++i) p.inv_freq[i] = i < d->head_dim / 2 ? pow((double)theta, -2.0 * i / (double)d->head_dim) : 0.0;
    p.status = ctx->dev_status;
    // A page's K and V heads on one CTA per eight of them.  One row per sequence: 16 query heads per CTA, every warp a few of
    // them; chunks: 32 query heads per CTA, so that a warp keeps a row's rotation for several loads.
    p.kv_ctas = (2 * p.Hkv + kBoundsWarps - 1) / kBoundsWarps;
    const int per_cta = q_offsets ? 32 : 16;
    p.q_heads_per_cta = p.Hq < per_cta ? p.Hq : per_cta;
    const int q_ctas = (p.Hq + p.q_heads_per_cta - 1) / p.q_heads_per_cta;
    // m new tokens of a sequence touch at most (m + 14) / 16 + 1 pages
    const long long tasks = q_offsets ? ((long long)rows + 14LL * batch) / 16 + batch : batch;
    KernelScope scope(ctx, kKAppendBounds, st);
    typedef void (*Kernel)(const AppendParams);
    static const Kernel kernels[2][2] = {{rope_append_bounds_kernel<64, 1>, rope_append_bounds_kernel<64, 2>},
                                         {rope_append_bounds_kernel<128, 1>, rope_append_bounds_kernel<128, 4>}};
    return check_cuda(ctx, launch_pdl(kernels[d->head_dim == 128][q_offsets != nullptr],
                                      dim3((unsigned)tasks, (unsigned)(p.kv_ctas + q_ctas)), dim3(kBoundsThreads), 0, st, p),
                      "rope_append_bounds_kernel launch");
}

}  // namespace aflex
