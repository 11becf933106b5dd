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

// A plain load, for what a preceding kernel may have written (projections, lengths): these kernels may have started before that
// one was done and wait for it, so the read-only path (ld.global.nc) would not be bound to see its stores.
template <typename V> __device__ __forceinline__ V fetch(const V* p) { return *p; }

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

// Larger / smaller of two bf16 pairs; the other operand where one is NaN.
__device__ __forceinline__ uint32_t max_pair(uint32_t a, uint32_t b) {
    uint32_t d;
    asm("max.bf16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
    return d;
}
__device__ __forceinline__ uint32_t min_pair(uint32_t a, uint32_t b) {
    uint32_t d;
    asm("min.bf16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
    return d;
}

struct Range16 {                                  // running extremes of this lane's 16 channels, bf16 pairs
    uint32_t hi[8], lo[8];
    __device__ __forceinline__ void reset() {
#pragma unroll
        for (int i = 0; i < 8; ++i) { hi[i] = 0xff80ff80u; lo[i] = 0x7f807f80u; }      // -inf, +inf
    }
    __device__ __forceinline__ void add(const uint4& a, const uint4& b) {      // a: first half's channels, b: second half's
        const uint32_t v[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
#pragma unroll
        for (int i = 0; i < 8; ++i) { hi[i] = max_pair(hi[i], v[i]); lo[i] = min_pair(lo[i], v[i]); }
    }
};

// Two fp32 operations in one instruction.
__device__ __forceinline__ uint64_t pack_f32x2(float x, float y) {
    uint64_t d;
    asm("mov.b64 %0, {%1, %2};" : "=l"(d) : "f"(x), "f"(y));
    return d;
}
__device__ __forceinline__ void unpack_f32x2(uint64_t v, float& x, float& y) { asm("mov.b64 {%0, %1}, %2;" : "=f"(x), "=f"(y) : "l"(v)); }
__device__ __forceinline__ uint64_t widen_bf16x2(uint32_t v) { return pack_f32x2(__uint_as_float(v << 16), __uint_as_float(v & 0xffff0000u)); }
__device__ __forceinline__ uint64_t fma_f32x2(uint64_t a, uint64_t b, uint64_t c) {
    uint64_t d;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a), "l"(b), "l"(c));
    return d;
}
__device__ __forceinline__ uint64_t mul_f32x2(uint64_t a, uint64_t b) {
    uint64_t d;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
    return d;
}

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

// Joins the lanes' ranges of one (page, KV head) and writes its bounds.  All 32 lanes take part.  Each joining step hands half
// of a lane's channels to its partner, so that in the end every channel is quantised by one lane: lane bit 4 tells which half
// of the head, bits 3 (and 2, D = 64) which of the chunk's channels, the others the chunk.
template <int K>                                    // of 2 K pairs keep K, the first or (upper lanes) the last
__device__ __forceinline__ void join(Range16& r, int lane, int off) {
    const bool upper = (lane & off) != 0;
#pragma unroll
    for (int i = 0; i < K; ++i) {
        const uint32_t h0 = r.hi[i], h1 = r.hi[i + K], l0 = r.lo[i], l1 = r.lo[i + K];
        r.hi[i] = max_pair(upper ? h1 : h0, __shfl_xor_sync(0xffffffffu, upper ? h0 : h1, off));
        r.lo[i] = min_pair(upper ? l1 : l0, __shfl_xor_sync(0xffffffffu, upper ? l0 : l1, off));
    }
}
template <int D>
__device__ __forceinline__ void store_bounds(Range16& r, int lane, int8_t* codes, uint8_t* scales) {
    constexpr int kPer = Lanes<D>::kPer;
    constexpr int kPairs = D == 128 ? 2 : 1;       // channel pairs a lane ends up with
    join<4>(r, lane, 16);
    join<2>(r, lane, 8);
    if (D == 64) join<1>(r, lane, 4);
    float hi[2 * kPairs], lo[2 * kPairs], a = 0.f;
#pragma unroll
    for (int i = 0; i < kPairs; ++i) {
        hi[2 * i] = __uint_as_float(r.hi[i] << 16); hi[2 * i + 1] = __uint_as_float(r.hi[i] & 0xffff0000u);
        lo[2 * i] = __uint_as_float(r.lo[i] << 16); lo[2 * i + 1] = __uint_as_float(r.lo[i] & 0xffff0000u);
    }
#pragma unroll
    for (int i = 0; i < 2 * kPairs; ++i) {
        if (hi[i] < lo[i]) hi[i] = lo[i] = 0.f;               // no key was a number
        a = fmaxf(a, fmaxf(fabsf(hi[i]), fabsf(lo[i])));
    }
    // the lanes of a 32-channel block: four chunks, and the lanes that share a chunk
    a = fmaxf(a, __shfl_xor_sync(0xffffffffu, a, 1));
    a = fmaxf(a, __shfl_xor_sync(0xffffffffu, a, 2));
    a = fmaxf(a, __shfl_xor_sync(0xffffffffu, a, 8));
    if (D == 64) a = fmaxf(a, __shfl_xor_sync(0xffffffffu, a, 4));
    const int e = block_exponent(a);
    const float inv = __uint_as_float((uint32_t)(127 - e) << 23);
    int ih[2 * kPairs], il[2 * kPairs];
#pragma unroll
    for (int i = 0; i < 2 * kPairs; ++i) {                     // (conversions saturate, so infinity ends at the border)
        ih[i] = max(-127, min(127, __float2int_ru(hi[i] * inv)));
        il[i] = max(-127, min(127, __float2int_rd(lo[i] * inv)));
    }
    const int half = lane >> 4, l = lane & (kPer - 1);
    int8_t* chunk = codes + (half * kPer + l) * 16;
    if (D == 128) {
        const int q = (lane >> 3) & 1;
        reinterpret_cast<uint32_t*>(chunk)[q] = pack4(ih[0], ih[1], ih[2 * kPairs - 2], ih[2 * kPairs - 1]);
        reinterpret_cast<uint32_t*>(chunk)[2 + q] = pack4(il[0], il[1], il[2 * kPairs - 2], il[2 * kPairs - 1]);
        if ((lane & 11) == 0) scales[half * 2 + (l >> 2)] = (uint8_t)(e + 127);
    } else {
        const int q = ((lane >> 3) & 1) * 2 + ((lane >> 2) & 1);
        reinterpret_cast<uint16_t*>(chunk)[q] = (uint16_t)((ih[0] & 255) | (ih[1] << 8));
        reinterpret_cast<uint16_t*>(chunk)[4 + q] = (uint16_t)((il[0] & 255) | (il[1] << 8));
        if ((lane & 15) == 0) scales[half] = (uint8_t)(e + 127);
    }
}

struct BoundsParams {
    const __nv_bfloat16* k_cache;
    int8_t* codes;
    uint8_t* scales;
    const int32_t* page_table;
    const int32_t* seq_lens;
    const int32_t* first_token;    // [batch] or null
    int max_pages, Hkv, pages_per_cta;
    long long num_pages;
    int* status;
};

// A CTA takes a run of pages of one sequence (their ids are looked up once), a warp every eighth (page, KV head) of it.  A head's
// 16 keys go through a ring in shared memory by asynchronous copies, the next head's in flight while one is reduced; a lane copies
// exactly the 16-byte words that it will read, so nothing but its own copies has to be waited for.  Bound: the read of the keys.
constexpr int kBoundsStages = 2;
template <int D>
__global__ void __launch_bounds__(kBoundsThreads) page_bounds_kernel(const BoundsParams p) {
    typedef Lanes<D> L;
    constexpr int kWords = 2 * L::kIter;                            // 16-byte words of a head per lane
    extern __shared__ __align__(16) uint4 ring[];                   // [warp][stage][word][lane]
    pdl_launch_dependents();
    pdl_wait();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, b = blockIdx.y;
    const int first_page = blockIdx.x * p.pages_per_cta, my_page = first_page + lane;     // lane i holds the run's i-th page
    const int raw = fetch(p.seq_lens + b);
    const int from = p.first_token ? fetch(p.first_token + b) : 0;
    int id = lane < p.pages_per_cta && my_page < p.max_pages ? fetch(p.page_table + (size_t)b * p.max_pages + my_page) : 0;
    if ((raw < 0 || raw > p.max_pages * kPageTokens) && blockIdx.x == 0 && threadIdx.x == 0) atomicExch(p.status, AFLEX_ERR_BOUNDS);
    const int len = max(0, min(raw, p.max_pages * kPageTokens));
    const int pages = min(p.pages_per_cta, (len + kPageTokens - 1) / kPageTokens - first_page);
    if (pages <= 0) return;
    // Valid tokens of this lane's page; 0: nothing to do (a page before the first new token, or a bad id)
    int valid = lane < pages && (my_page + 1) * kPageTokens > from ? min(kPageTokens, len - my_page * kPageTokens) : 0;
    if (valid > 0 && (id < 0 || id >= p.num_pages)) { atomicExch(p.status, AFLEX_ERR_BOUNDS); valid = 0; }
    const int sub = lane / L::kPer, l = lane % L::kPer;
    uint4* mine = ring + (size_t)warp * kBoundsStages * kWords * 32 + lane;
    const int items = pages * p.Hkv;
    auto issue = [&](int i, int stage) {
        const int v = __shfl_sync(0xffffffffu, valid, i / p.Hkv);
        if (v > 0) {
            const size_t slab = (size_t)__shfl_sync(0xffffffffu, id, i / p.Hkv) * p.Hkv + i % p.Hkv;
            const uint4* k = reinterpret_cast<const uint4*>(p.k_cache + slab * kPageTokens * D) + l;
            const uint32_t to = smem_u32(mine + stage * kWords * 32);
#pragma unroll
            for (int w = 0; w < kWords; ++w) {
                const int t = (w >> 1) * L::kTok + sub;             // a slot past the end repeats the last valid key
                asm volatile("cp.async.cg.shared.global [%0], [%1], 16;"
                             ::"r"(to + w * 512), "l"(k + (v == kPageTokens ? t : min(t, v - 1)) * (D / 8) + (w & 1) * (D / 16)) : "memory");
            }
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
    int ahead = warp;                                               // next item to copy
#pragma unroll
    for (int s = 0; s < kBoundsStages - 1; ++s) {
        if (ahead < items) issue(ahead, s); else asm volatile("cp.async.commit_group;" ::: "memory");
        ahead += kBoundsWarps;
    }
    int stage = 0;
    for (int i = warp; i < items; i += kBoundsWarps) {
        const int to = stage == 0 ? kBoundsStages - 1 : stage - 1;  // the stage that was read last
        if (ahead < items) issue(ahead, to); else asm volatile("cp.async.commit_group;" ::: "memory");
        ahead += kBoundsWarps;
        asm volatile("cp.async.wait_group %0;" ::"n"(kBoundsStages - 1) : "memory");
        if (__shfl_sync(0xffffffffu, valid, i / p.Hkv) > 0) {
            Range16 r;
            r.reset();
#pragma unroll
            for (int it = 0; it < L::kIter; ++it) r.add(mine[(stage * kWords + 2 * it) * 32], mine[(stage * kWords + 2 * it + 1) * 32]);
            const size_t slab = (size_t)__shfl_sync(0xffffffffu, id, i / p.Hkv) * p.Hkv + i % p.Hkv;
            store_bounds<D>(r, lane, p.codes + slab * 2 * D, p.scales + slab * (D / 32));
        }
        stage = stage + 1 == kBoundsStages ? 0 : stage + 1;
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
    int q_heads_per_cta, kv_ctas, groups;  // head groups of a page: kv_ctas for its K and V heads, the others for its query heads
    float eps;
    double inv_freq[64];           // theta^(-2 i / D), formed in double on the host
    double step_cos[64], step_sin[64];             // ... and the cosine and sine of that angle: one position's rotation
    int* status;
};

// A CTA handles the rows of ONE page of one sequence (1 to 16 rows), so that whoever rotates the page's keys holds all of
// them when the bounds are formed: a page among the pages touched by the call (located by a scan over the sequences) and a
// group of heads.  In chunks a page's groups are neighbours, so that key CTAs (arithmetic in double) run next to query and
// value CTAs (bytes): 58.2 against 64.0 us for 7420 rows of 64 + 2 x 8 heads.  One row per page: all key CTAs, the longest, first.
//
// Bound: qkv read and q, K, V written once.  Two rotary halves of eight channels per lane make every access 16 bytes.
// Queries are rotated in fp32.  Keys (one head in ten on the shapes served here) are normalised and rotated in double and
// rounded to fp32 and then to bf16: the stored key no longer depends on the order in which sums were formed (but for values
// within 1e-11 of a rounding border), and the bounds, which are integers made from it, come out the same everywhere.
template <int D>
__global__ void __launch_bounds__(kBoundsThreads, 3) rope_append_bounds_kernel(const AppendParams p) {
    // No early release of the dependents: the dense attention kernel reads the cache without waiting for the grid
    // dependency, which is sound only if the kernel that writes the cache has finished before anything later starts.
    typedef Lanes<D> L;
    constexpr int kHalf = D / 2;
    __shared__ int s_warp[kBoundsWarps];
    __shared__ int s_b, s_page;
    // A row's rotation per pair, the gains of the head norms multiplied in: x' = x A - y B, y' = y C + x E.  Stored so that
    // the lanes of a token read neighbouring words; queries' in pairs, for the packed arithmetic.
    __shared__ __align__(16) union Rotation {
        float4 q[kPageTokens][4][2][L::kPer];      // pairs 8 l + 2 k, + 1: (A, A', -B, -B'), (C, C', E, E') at [slot][k][0, 1][l]
        double2 k[kPageTokens][8][2][L::kPer];     // (A, B), (C, E)
    } rot;
    const int task = (int)(p.q_offsets ? blockIdx.x / p.groups : blockIdx.x % p.batch);
    const int group = (int)(p.q_offsets ? blockIdx.x % p.groups : blockIdx.x / p.batch);
    pdl_wait();
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    int b, page_i, row0, nrows, slot0;                              // rows row0 .. of the call go to slots slot0 .. of the page
    if (p.q_offsets == nullptr) {
        b = task;
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
            if (c < 0) { if (blockIdx.x == 0) atomicExch(p.status, AFLEX_ERR_BOUNDS); }
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
        const int want = task;
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
    const bool kv_part = group < p.kv_ctas;
    const int page = p.page_table[(size_t)b * p.max_pages + page_i];
    if (kv_part && (page < 0 || page >= p.num_pages)) {
        if (tid == 0) atomicExch(p.status, AFLEX_ERR_BOUNDS);
        return;
    }
    const int sub = lane / L::kPer, l = lane % L::kPer;
    // Rotations, by slot of the page: angle and its reduction to [-pi, pi] in double (two-term 2 pi).  A thread makes the sine
    // and cosine of one pair at every fourth slot and steps to the next three by the pair's rotation of one position; the
    // steps start at fixed slots, so a position's rotation does not depend on which rows came with it.
    const int slot1 = slot0 + nrows, c_rot = tid % kHalf, s_rot = 4 * (tid / kHalf);
    const bool rotates = s_rot < slot1 && s_rot + 4 > slot0;
    auto reduced = [&](int slot, int c) -> double {
        const double ang = (double)(page_i * kPageTokens + slot) * p.inv_freq[c];
        const double turns = rint(ang * 0.15915494309189535);
        return fma(-turns, 2.4492935982947064e-16, fma(-turns, 6.283185307179586, ang));
    };
    if (!kv_part) {
        // ---- query heads.  The warps are dealt out over rows and heads, two times kTok heads of a row at once; the next ones
        // are loaded while these are rotated (the first ones while the rotations are made).
        const int h_lo = (group - p.kv_ctas) * p.q_heads_per_cta, h_hi = min(p.Hq, h_lo + p.q_heads_per_cta);
        const int along = nrows >= 8 ? 1 : nrows >= 4 ? 2 : nrows >= 2 ? 4 : 8;              // warps along the heads of a row
        const int h_first = h_lo + (warp & (along - 1)) * 2 * L::kTok + sub, h_step = along * 2 * L::kTok;
        const int r_first = warp / along, r_step = kBoundsWarps / along;
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
        if (rotates) {
            const int c = c_rot;
            const float ga = p.w_qn ? __bfloat162float(p.w_qn[c]) : 1.f, gc = p.w_qn ? __bfloat162float(p.w_qn[kHalf + c]) : 1.f;
            const float step_cs = (float)p.step_cos[c], step_sn = (float)p.step_sin[c];
            float sn, cs;
            sincosf((float)reduced(s_rot, c), &sn, &cs);
            for (int s = s_rot; s < min(slot1, s_rot + 4); ++s) {
                float* z = reinterpret_cast<float*>(&rot.q[s][(c & 7) >> 1][0][c >> 3]) + (c & 1);
                z[0] = ga * cs; z[2] = -gc * sn;
                z += 4 * L::kPer;
                z[0] = gc * cs; z[2] = ga * sn;
                const float next = cs * step_cs - sn * step_sn;
                sn = sn * step_cs + cs * step_sn;
                cs = next;
            }
        }
        __syncthreads();
        for (int r = r_first; r < nrows; r += r_step) {
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
                    const ulonglong2 z0 = *reinterpret_cast<const ulonglong2*>(&rot.q[slot0 + r][k][0][l]);
                    const ulonglong2 z1 = *reinterpret_cast<const ulonglong2*>(&rot.q[slot0 + r][k][1][l]);
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
                    if (h + u * L::kTok < h_hi) {
                        uint4* dst = reinterpret_cast<uint4*>(p.q_out + ((size_t)(row0 + r) * p.Hq + h + u * L::kTok) * D);
                        dst[l] = make_uint4(va[u][0], va[u][1], va[u][2], va[u][3]);
                        dst[D / 16 + l] = make_uint4(vc[u][0], vc[u][1], vc[u][2], vc[u][3]);
                    }
                }
            }
        }
        return;
    }
    // ---- a key or value head per warp, loaded before the rotations are made; values are copied as they are
    const int i = group * kBoundsWarps + warp, g = i < p.Hkv ? i : i - p.Hkv;
    const bool is_key = i < p.Hkv, is_value = !is_key && i < 2 * p.Hkv;
    const size_t slab = (size_t)page * p.Hkv + g;
    const int end = slot1;                                          // slots [0, slot0) hold older keys, [slot0, end) are new
    uint4* kd = reinterpret_cast<uint4*>(p.k_cache + slab * kPageTokens * D);
    uint4 xa[L::kIter], xb[L::kIter];
    if (is_key) {
#pragma unroll
        for (int it = 0; it < L::kIter; ++it) {
            const int t = min(it * L::kTok + sub, end - 1);
            const uint4* src = t < slot0 ? kd + t * (D / 8)
                                         : reinterpret_cast<const uint4*>(p.qkv + ((size_t)(row0 + t - slot0) * heads + p.Hq + g) * D);
            xa[it] = src[l];
            xb[it] = src[D / 16 + l];
        }
    }
    if (is_value) {
        const uint4* src = reinterpret_cast<const uint4*>(p.qkv + ((size_t)row0 * heads + p.Hq + i) * D);
        uint4* dst = reinterpret_cast<uint4*>(p.v_cache + (slab * kPageTokens + slot0) * D);
        uint4 v[kPageTokens * D / 256];
#pragma unroll
        for (int k = 0; k < kPageTokens * D / 256; ++k) {
            const int j = k * 32 + lane, r = j / (D / 8);
            if (r < nrows) v[k] = fetch(src + (size_t)r * heads * (D / 8) + j % (D / 8));
        }
#pragma unroll
        for (int k = 0; k < kPageTokens * D / 256; ++k) {
            const int j = k * 32 + lane;
            if (j / (D / 8) < nrows) dst[j] = v[k];
        }
    }
    if (group * kBoundsWarps >= p.Hkv) return;                      // values only
    if (rotates) {
        const int c = c_rot;
        const double ga = p.w_kn ? __bfloat162float(p.w_kn[c]) : 1.f, gc = p.w_kn ? __bfloat162float(p.w_kn[kHalf + c]) : 1.f;
        double sn, cs;
        sincos(reduced(s_rot, c), &sn, &cs);
        for (int s = s_rot; s < min(slot1, s_rot + 4); ++s) {
            rot.k[s][c & 7][0][c >> 3] = make_double2(ga * cs, gc * sn);
            rot.k[s][c & 7][1][c >> 3] = make_double2(gc * cs, ga * sn);
            const double next = cs * p.step_cos[c] - sn * p.step_sin[c];
            sn = sn * p.step_cos[c] + cs * p.step_sin[c];
            cs = next;
        }
    }
    __syncthreads();
    if (is_key) {
        Range16 range;
        range.reset();
#pragma unroll
        for (int it = 0; it < L::kIter; ++it) {
            const int t0 = it * L::kTok;
            if (t0 >= end) break;
            const int t = min(t0 + sub, end - 1);
            if (t0 + L::kTok > slot0) {                             // some of these tokens are new (the same for the whole warp)
                const int s = max(slot0, t);
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
                    const double2 z0 = rot.k[s][k][0][l], z1 = rot.k[s][k][1][l];
                    qa[k] = __float2bfloat16_rn((float)((a * z0.x - c * z0.y) * rinv));
                    qb[k] = __float2bfloat16_rn((float)((c * z1.x + a * z1.y) * rinv));
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
    // Pages per CTA: one (page, head) per warp at least; twice and four times that where four CTAs per SM are still left.
    // 32 sequences of up to 256 pages x 8 heads: 37.2 / 29.2 / 28.8 / 32.5 us with 1 / 2 / 4 / 8 heads per warp (a ring of
    // three: 48.4 / 34.7 / 29.9 / 31.7; every warp's 16 keys in registers: 35.3).
    const int least = (kBoundsWarps + p.Hkv - 1) / p.Hkv;
    p.pages_per_cta = least;
    while (p.pages_per_cta < 4 * least && p.pages_per_cta <= 16 && (long long)batch * p.max_pages >= 2LL * p.pages_per_cta * 4 * ctx->num_sms)
        p.pages_per_cta *= 2;
    const dim3 grid((unsigned)((p.max_pages + p.pages_per_cta - 1) / p.pages_per_cta), (unsigned)batch);
    const size_t smem = (size_t)kBoundsWarps * kBoundsStages * kPageTokens * d->head_dim * 2;
    const bool wide = d->head_dim == 128;
    if (!ctx->bounds_attr_set[wide]) {
        cudaError_t e = cudaFuncSetAttribute(wide ? page_bounds_kernel<128> : page_bounds_kernel<64>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
        if (e != cudaSuccess) return check_cuda(ctx, e, "cudaFuncSetAttribute(page bounds)");
        ctx->bounds_attr_set[wide] = true;
    }
    KernelScope scope(ctx, kKPageBounds, st);
    return check_cuda(ctx, launch_pdl(wide ? page_bounds_kernel<128> : page_bounds_kernel<64>, grid, dim3(kBoundsThreads), smem, st, p),
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
    // the frequencies of the last theta and head size (a few microseconds of host time for a launch of as many)
    if (ctx->rope_theta != theta || ctx->rope_dim != d->head_dim) {
        for (int i = 0; i < d->head_dim / 2; ++i) {
            ctx->rope_freq[i] = pow((double)theta, -2.0 * i / (double)d->head_dim);
            ctx->rope_step[0][i] = cos(ctx->rope_freq[i]);
            ctx->rope_step[1][i] = sin(ctx->rope_freq[i]);
        }
        ctx->rope_theta = theta;
        ctx->rope_dim = d->head_dim;
    }
    for (int i = 0; i < 64; ++i) { p.inv_freq[i] = ctx->rope_freq[i]; p.step_cos[i] = ctx->rope_step[0][i]; p.step_sin[i] = ctx->rope_step[1][i]; }
    p.status = ctx->dev_status;
    // A page's K and V heads on one CTA per eight of them; its query heads 32 per CTA (7420 rows: 79.2 / 63.0 / 58.2 / 59.6 us with
    // 8 / 16 / 32 / 64; 256 single rows: 10.0 / 7.3 / 6.7 / 6.7: every CTA locates its page and makes its rotations).
    // m new tokens of a sequence touch at most (m + 14) / 16 + 1 pages.
    const long long tasks = q_offsets ? ((long long)rows + 14LL * batch) / 16 + batch : batch;
    p.kv_ctas = (2 * p.Hkv + kBoundsWarps - 1) / kBoundsWarps;
    p.q_heads_per_cta = p.Hq < 32 ? p.Hq : 32;
    const int q_ctas = (p.Hq + p.q_heads_per_cta - 1) / p.q_heads_per_cta;
    p.groups = p.kv_ctas + q_ctas;
    if (tasks * p.groups > 0x7fffffffLL) return set_error(ctx, AFLEX_ERR_UNSUPPORTED, "rope_append_bounds: rows = %d", rows);
    KernelScope scope(ctx, kKAppendBounds, st);
    return check_cuda(ctx, launch_pdl(d->head_dim == 128 ? rope_append_bounds_kernel<128> : rope_append_bounds_kernel<64>,
                                      dim3((unsigned)(tasks * p.groups)), dim3(kBoundsThreads), 0, st, p),
                      "rope_append_bounds_kernel launch");
}

}  // namespace aflex
