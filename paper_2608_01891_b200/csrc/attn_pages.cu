// Page-sparse decode attention: which pages of the cache each row's queries should read, and attention over those pages only.
//   page_select_kernel        scores every page's key bounds against the row's queries and keeps the best
//   attn_decode_pages_kernel  attention of each row over its listed pages
// A row is one query token: the one being decoded, or one of the last few of its sequence (drafted tokens).
#include <cuda_bf16.h>
#include <math.h>

#include "internal.h"
#include "ptx.cuh"

namespace aflex {

namespace {

constexpr int kPageTokens = 16;
constexpr float kNegBig = -1.0e30f;

// Sequence and position of a row.  Returns false (and reports it) where the inputs give none; rows behind the last
// sequence's are not theirs to report: `padding`.
struct RowAt { int b, pos; bool padding; };
__device__ __forceinline__ bool locate_row(int row, const int32_t* q_offsets, const int32_t* seq_lens, int batch, int max_pages,
                                           RowAt& at) {
    int back = 0;
    at.b = row; at.padding = false;
    if (q_offsets != nullptr) {
        if (row >= q_offsets[batch]) { at.padding = true; return false; }
        int lo = 0, hi = batch;                    // largest b with q_offsets[b] <= row
        while (hi - lo > 1) {
            const int mid = (lo + hi) / 2;
            if (q_offsets[mid] <= row) lo = mid; else hi = mid;
        }
        at.b = lo;
        back = q_offsets[lo + 1] - 1 - row;
    }
    const int len = seq_lens[at.b];
    at.pos = len - 1 - back;
    return back >= 0 && at.pos >= 0 && len <= max_pages * kPageTokens;
}

__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }
__device__ __forceinline__ void st_cluster_u32(uint32_t addr, uint32_t v) {
    asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(addr), "r"(v) : "memory");
}
__device__ __forceinline__ uint32_t ld_cluster_u32(uint32_t addr) {
    uint32_t v;
    asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(addr) : "memory");
    return v;
}
__device__ __forceinline__ float ld_cluster_f32(uint32_t addr) {
    float v;
    asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(addr) : "memory");
    return v;
}

// D(16x8, s32) += A(16x32, s8, row) * B(32x8, s8, col)
__device__ __forceinline__ void mma_s8_16832(int (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm volatile(
        "mma.sync.aligned.m16n8k32.row.col.s32.s8.s8.s32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
        : "+r"(d[0]), "+r"(d[1]), "+r"(d[2]), "+r"(d[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// ------------------------------------------------------------------------------------------ selection
//
// Score of a page for query head h, per 32-channel block c:  f_c the smallest exponent with max|q| <= 127 * 2^f_c,
//   Q_d = rint(q_d / 2^f_c),  i_c = sum_d max(Q_d, 0) HI_d + min(Q_d, 0) LO_d
//   s_h = ((v_0 + v_1) + v_2) + v_3 in fp32,  v_c = i_c 2^e_c 2^f_c
// an upper bound (up to the rounding of q) of any key's product with the query.  The page's score is the largest over the
// group's heads.  i_c is an integer below 2^19 and v_c exact in fp32, so the score, and with it the selection, is the same
// bit for bit whatever computes it.
//
// One cluster of CTAs per (row, KV head); each warp scores tiles of 16 pages with integer MMAs, operands loaded from global
// memory straight into registers (the bounds' layout is the fragment's), and drops the scores as order-preserving keys into
// the first CTA's shared memory.  That CTA then finds the key of the last page to keep by radix selection and writes the list.
constexpr int kSelWarps = 8;
constexpr int kSelThreads = kSelWarps * 32;
constexpr int kSelTile = 16;
constexpr int kSelKeyCap = 48 * 1024;               // keys one CTA's shared memory holds; further ones go to the next CTA's
constexpr int kSelMaxCluster = 8;

struct SelectParams {
    const __nv_bfloat16* q;        // [rows][Hq][D]
    const int8_t* codes;
    const uint8_t* scales;
    const int32_t* page_table;
    const int32_t* seq_lens;
    const int32_t* q_offsets;
    int batch, max_pages, Hq, Hkv, G;
    long long num_pages;
    int top, sink, window;
    int cluster;                   // CTAs per (row, KV head)
    int cap;                       // keys per CTA
    int32_t* list;                 // [rows][Hkv][top]
    int32_t* count;                // [rows][Hkv]
    int* status;
};

struct SelectShared {
    int hist[256];
    int warp_a[kSelWarps], warp_b[kSelWarps];
    uint32_t all_or, all_and;
    int bin, need;
};

__device__ __forceinline__ int q_exponent(float a) {             // smallest e with a <= 127 * 2^e, within [-60, 50]
    const int field = (int)((__float_as_uint(a) >> 23) & 255u);
    int e = field - 133;
    if (e >= -60 && e <= 50 && a * __uint_as_float((uint32_t)(127 - e) << 23) > 127.f) ++e;
    return max(-60, min(50, e));
}

template <int D>
__global__ void __launch_bounds__(kSelThreads) page_select_kernel(const SelectParams p) {
    constexpr int kBlocks = D / 32;
    extern __shared__ __align__(16) uint8_t smem_raw[];
    uint32_t* keys = reinterpret_cast<uint32_t*>(smem_raw);
    __shared__ SelectShared sh;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int S = p.cluster, rank = (int)(blockIdx.x % S);
    const long long item = blockIdx.x / S;
    const int row = (int)(item / p.Hkv), g = (int)(item % p.Hkv);
    if (S > 1) cluster_arrive();                                  // the cluster's CTAs have started: waited for below
    pdl_launch_dependents();
    pdl_wait();
    RowAt at;
    const bool ok = locate_row(row, p.q_offsets, p.seq_lens, p.batch, p.max_pages, at);
    const int n = ok ? at.pos / kPageTokens + 1 : 0;
    if (!ok && !at.padding && tid == 0 && rank == 0) atomicExch(p.status, AFLEX_ERR_BOUNDS);
    int32_t* list = p.list + item * p.top;
    const int keep = p.top - p.sink - p.window;                   // scored pages to keep
    const int cand = n - p.sink - p.window;                       // scored pages
    if (n <= p.top || keep == 0) {                                // nothing to choose (the same for the whole cluster)
        if (S > 1) cluster_wait();
        if (rank != 0 || at.padding) return;
        for (int i = tid; i < p.top; i += kSelThreads) {
            int v = i < n ? i : -1;
            if (n > p.top && i >= p.sink) v = n - p.top + i;
            list[i] = v;
        }
        if (tid == 0) p.count[item] = min(n, p.top);
        return;
    }
    // ---- the group's queries as the MMA's B operand: lane holds head lane / 4, channels 8 (lane % 4) .. + 7 of every block
    const int hl = lane >> 2, l4 = lane & 3;
    uint32_t qp[kBlocks][2], qn[kBlocks][2];
    float fq[kBlocks][2];                                         // 2^f of this lane's two accumulator columns
    {
        const bool on = hl < p.G;
        const uint4* src = reinterpret_cast<const uint4*>(p.q + ((size_t)row * p.Hq + (size_t)g * p.G + (on ? hl : 0)) * D);
#pragma unroll
        for (int c = 0; c < kBlocks; ++c) {
            const uint4 x = src[c * 4 + l4];
            const __nv_bfloat162* px = reinterpret_cast<const __nv_bfloat162*>(&x);
            float v[8], a = 0.f;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float2 u = __bfloat1622float2(px[i]);
                v[2 * i] = u.x; v[2 * i + 1] = u.y;
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                if (!on || v[i] != v[i]) v[i] = 0.f;              // NaN counts as 0
                a = fmaxf(a, fabsf(v[i]));
            }
            a = fmaxf(a, __shfl_xor_sync(0xffffffffu, a, 1));
            a = fmaxf(a, __shfl_xor_sync(0xffffffffu, a, 2));
            const int e = q_exponent(a);
            const float inv = __uint_as_float((uint32_t)(127 - e) << 23);
            uint32_t pos[2] = {0, 0}, neg[2] = {0, 0};
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int z = (int)rintf(fminf(127.f, fmaxf(-127.f, v[i] * inv)));
                pos[i >> 2] |= (uint32_t)max(z, 0) << (8 * (i & 3));
                neg[i >> 2] |= (uint32_t)(min(z, 0) & 255) << (8 * (i & 3));
            }
            qp[c][0] = pos[0]; qp[c][1] = pos[1];
            qn[c][0] = neg[0]; qn[c][1] = neg[1];
            const float f = __uint_as_float((uint32_t)(127 + e) << 23);
            fq[c][0] = __shfl_sync(0xffffffffu, f, 8 * l4);       // columns 2 l4 and 2 l4 + 1 of the accumulator
            fq[c][1] = __shfl_sync(0xffffffffu, f, 8 * l4 + 4);
        }
    }
    if (S > 1) cluster_wait();
    // ---- scores
    const int32_t* table = p.page_table + (size_t)at.b * p.max_pages + p.sink;
    const int tiles = (cand + kSelTile - 1) / kSelTile;
    const uint32_t keys_addr = smem_u32(keys);
    for (int t = rank * kSelWarps + warp; t < tiles; t += S * kSelWarps) {
        size_t slab[2];
#pragma unroll
        for (int r = 0; r < 2; ++r) {
            const int j = t * kSelTile + hl + 8 * r;
            int id = table[min(j, cand - 1)];
            if (id < 0 || id >= p.num_pages) { atomicExch(p.status, AFLEX_ERR_BOUNDS); id = 0; }
            slab[r] = (size_t)id * p.Hkv + g;
        }
        uint4 x[2][kBlocks];
        uint32_t sc[2];
#pragma unroll
        for (int r = 0; r < 2; ++r) {
            const uint4* src = reinterpret_cast<const uint4*>(p.codes + slab[r] * (2 * D)) + l4;
#pragma unroll
            for (int c = 0; c < kBlocks; ++c) x[r][c] = __ldg(src + c * 4);
            if (kBlocks == 4) sc[r] = __ldg(reinterpret_cast<const uint32_t*>(p.scales) + slab[r]);
            else sc[r] = __ldg(reinterpret_cast<const uint16_t*>(p.scales) + slab[r]);
        }
        float s[4];
#pragma unroll
        for (int c = 0; c < kBlocks; ++c) {
            int d[4] = {0, 0, 0, 0};
            mma_s8_16832(d, x[0][c].x, x[1][c].x, x[0][c].y, x[1][c].y, qp[c][0], qp[c][1]);
            mma_s8_16832(d, x[0][c].z, x[1][c].z, x[0][c].w, x[1][c].w, qn[c][0], qn[c][1]);
            const float k0 = __uint_as_float(((sc[0] >> (8 * c)) & 255u) << 23), k1 = __uint_as_float(((sc[1] >> (8 * c)) & 255u) << 23);
            // the products are exact, so a fused multiply-add rounds like the sum alone
            s[0] = fmaf((float)d[0] * k0, fq[c][0], c ? s[0] : 0.f);
            s[1] = fmaf((float)d[1] * k0, fq[c][1], c ? s[1] : 0.f);
            s[2] = fmaf((float)d[2] * k1, fq[c][0], c ? s[2] : 0.f);
            s[3] = fmaf((float)d[3] * k1, fq[c][1], c ? s[3] : 0.f);
        }
        const bool h0 = 2 * l4 < p.G, h1 = 2 * l4 + 1 < p.G;
        float m0 = fmaxf(h0 ? s[0] : -INFINITY, h1 ? s[1] : -INFINITY);
        float m1 = fmaxf(h0 ? s[2] : -INFINITY, h1 ? s[3] : -INFINITY);
        m0 = fmaxf(m0, __shfl_xor_sync(0xffffffffu, m0, 1));
        m1 = fmaxf(m1, __shfl_xor_sync(0xffffffffu, m1, 1));
        m0 = fmaxf(m0, __shfl_xor_sync(0xffffffffu, m0, 2));
        m1 = fmaxf(m1, __shfl_xor_sync(0xffffffffu, m1, 2));
        if (l4 < 2) {
            const int j = t * kSelTile + hl + 8 * l4;
            if (j < cand) {
                uint32_t u = __float_as_uint((l4 ? m1 : m0) + 0.f);          // no negative zero
                u ^= (u >> 31) ? 0xffffffffu : 0x80000000u;                 // unsigned order = numeric order
                const int owner = j / p.cap;
                if (S == 1) keys[j] = u;
                else st_cluster_u32(cluster_map_shared(keys_addr + (uint32_t)(j - owner * p.cap) * 4, (uint32_t)owner), u);
            }
        }
    }
    const bool far = cand > p.cap;                                 // some keys are in another CTA's shared memory
    if (S > 1) {
        cluster_arrive();
        cluster_wait();
        if (rank != 0) {
            if (far) { cluster_arrive(); cluster_wait(); }
            return;
        }
    } else {
        __syncthreads();
    }
    auto key_at = [&](int j) -> uint32_t {
        if (!far) return keys[j];
        const int owner = j / p.cap;
        return ld_cluster_u32(cluster_map_shared(keys_addr + (uint32_t)(j - owner * p.cap) * 4, (uint32_t)owner));
    };
    // ---- radix selection of the keep-th largest key, eight bits at a time from the highest bit in which keys differ
    uint32_t o = 0, a = 0xffffffffu;
    for (int j = tid; j < cand; j += kSelThreads) { const uint32_t k = key_at(j); o |= k; a &= k; }
    o = __reduce_or_sync(0xffffffffu, o);
    a = __reduce_and_sync(0xffffffffu, a);
    if (tid == 0) { sh.all_or = 0; sh.all_and = 0xffffffffu; }
    __syncthreads();
    if (lane == 0) { atomicOr(&sh.all_or, o); atomicAnd(&sh.all_and, a); }
    __syncthreads();
    uint32_t prefix = sh.all_and, mask;                            // keys are compared in the bits of `mask`
    int need = keep;                                               // of the keys that equal prefix in those bits
    const uint32_t differ = sh.all_or ^ sh.all_and;
    int bits = differ ? 32 - __clz(differ) : 0;                    // unresolved low bits
    mask = bits == 32 ? 0u : ~((1u << bits) - 1u);
    prefix &= mask;
    while (bits > 0) {
        const int shift = max(bits - 8, 0);
        sh.hist[tid] = 0;
        __syncthreads();
        for (int j = tid; j < cand; j += kSelThreads) {
            const uint32_t k = key_at(j);
            if ((k & mask) == prefix) atomicAdd(&sh.hist[(k & ~mask) >> shift], 1);
        }
        __syncthreads();
        // thread t looks at bin 255 - t: keys in it and above it
        const int c = sh.hist[255 - tid];
        int incl = c;
#pragma unroll
        for (int off = 1; off < 32; off <<= 1) {
            const int v = __shfl_up_sync(0xffffffffu, incl, off);
            if (lane >= off) incl += v;
        }
        if (lane == 31) sh.warp_a[warp] = incl;
        __syncthreads();
        for (int w = 0; w < warp; ++w) incl += sh.warp_a[w];
        if (incl >= need && incl - c < need) { sh.bin = 255 - tid; sh.need = need - (incl - c); sh.warp_b[0] = c; }
        __syncthreads();
        prefix |= (uint32_t)sh.bin << shift;
        need = sh.need;
        bits = shift;
        mask = bits == 0 ? 0xffffffffu : ~((1u << bits) - 1u);
        const bool whole = sh.warp_b[0] == need;                   // the bin is kept whole: no need to look inside
        __syncthreads();
        if (whole) break;
    }
    // ---- the list, ascending: each warp places a contiguous run of the candidates
    const int run = ((cand + kSelThreads - 1) / kSelThreads) * 32;
    const int j0 = min(cand, warp * run), j1 = min(cand, j0 + run);
    int gt = 0, eq = 0;
    for (int j = j0 + lane; j < j1; j += 32) {
        const uint32_t k = key_at(j) & mask;
        gt += k > prefix;
        eq += k == prefix;
    }
    gt = __reduce_add_sync(0xffffffffu, gt);
    eq = __reduce_add_sync(0xffffffffu, eq);
    if (lane == 0) { sh.warp_a[warp] = gt; sh.warp_b[warp] = eq; }
    __syncthreads();
    int gt0 = 0, eq0 = 0;
    for (int w = 0; w < warp; ++w) { gt0 += sh.warp_a[w]; eq0 += sh.warp_b[w]; }
    for (int j = j0; j < j1; j += 32) {
        const bool in = j + lane < j1;
        const uint32_t k = in ? key_at(j + lane) & mask : 0u;
        const bool is_gt = in && k > prefix, is_eq = in && k == prefix;
        const unsigned bg = __ballot_sync(0xffffffffu, is_gt), be = __ballot_sync(0xffffffffu, is_eq);
        const unsigned below = (1u << lane) - 1u;
        const int g_at = gt0 + __popc(bg & below), e_at = eq0 + __popc(be & below);
        if (is_gt || (is_eq && e_at < need)) list[p.sink + g_at + min(e_at, need)] = p.sink + j + lane;
        gt0 += __popc(bg);
        eq0 += __popc(be);
    }
    for (int i = tid; i < p.sink; i += kSelThreads) list[i] = i;
    for (int i = tid; i < p.window; i += kSelThreads) list[p.top - p.window + i] = n - p.window + i;
    if (tid == 0) p.count[item] = p.top;
    if (far) { cluster_arrive(); cluster_wait(); }
}

// ------------------------------------------------------------------------------------------ attention over listed pages
//
// For row r at position t and query head h of KV head g, over the tokens j <= t of the listed pages:
//   s_j = sm_scale <q, K_j>,  out = sum_j softmax(s)_j V_j,  lse = ln sum_j exp(s_j)
//
// Bound: the K and V bytes of the listed pages.  Every page is 4 KB of K and 4 KB of V (D = 128) somewhere in HBM, read once
// by one warp straight into registers: with the channels of a row permuted alike for q and K (a sum does not mind), sixteen
// contiguous bytes per lane are MMA fragments as they are, S = Q K^T leaves P in the layout of the second product's A operand,
// and V's fragments are two rows' words interleaved.  No shared memory, no barrier, no copy engine in the loop: the next
// page's K is loaded as soon as the current one has been multiplied, the next V likewise.
// The MMA has 16 rows and a group at most 8 heads: the other 8 rows carry the low half of P (P = P_hi + P_lo, both bf16), so
// the second product loses nothing to the rounding of P.
// Lists are short (tens to a few hundred pages), so the work is split by (row, KV head) and, where those are few, the list is
// cut over a cluster's CTAs; warps and CTAs keep their own running maximum and sum and are joined through shared memory.
constexpr int kPagesWarps = 4;
constexpr int kPagesThreads = kPagesWarps * 32;

struct PagesParams {
    const __nv_bfloat16* q;
    const __nv_bfloat16* k_cache;
    const __nv_bfloat16* v_cache;
    const int32_t* page_table;
    const int32_t* seq_lens;
    const int32_t* q_offsets;
    const int32_t* list;           // [rows][Hkv][top]
    const int32_t* count;          // [rows][Hkv]
    int batch, max_pages, Hq, Hkv, G, top, cluster;
    long long num_pages;
    float scale_log2;
    __nv_bfloat16* out;
    float* lse;
    int* status;
};

template <int D> struct PagesShared {
    float o[kPagesWarps][8][D];
    float m[kPagesWarps][8], l[kPagesWarps][8];
};

__device__ __forceinline__ uint4 ld_stream(const uint4* p) {
    uint4 v;
    asm volatile("ld.global.nc.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
    return v;
}

template <int D>
__global__ void __launch_bounds__(kPagesThreads, 3) attn_decode_pages_kernel(const PagesParams p) {
    constexpr int kSteps = D / 32;                 // 16-byte loads per lane and K row
    constexpr int kHalves = D / 64;                // 16-byte loads per lane and V row
    __shared__ __align__(16) PagesShared<D> sh;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int hl = lane >> 2, l4 = lane & 3;
    const int S = p.cluster, rank = (int)(blockIdx.x % S);
    const long long item = blockIdx.x / S;
    const int row = (int)(item / p.Hkv), g = (int)(item % p.Hkv);
    pdl_launch_dependents();
    pdl_wait();
    RowAt at;
    const bool ok = locate_row(row, p.q_offsets, p.seq_lens, p.batch, p.max_pages, at);
    if (at.padding) return;                        // (the same for the whole cluster)
    int total = 0;
    if (ok) total = max(0, min(p.top, p.count[item]));
    else if (tid == 0) atomicExch(p.status, AFLEX_ERR_BOUNDS);
    const int lo = (int)((long long)total * rank / S), hi = (int)((long long)total * (rank + 1) / S);
    const int32_t* list = p.list + item * p.top;
    const int32_t* table = p.page_table + (size_t)at.b * p.max_pages;

    uint4 qf[kSteps];                              // head lane / 4, channels 32 step + 8 (lane % 4) .. + 7
    {
        const uint4* src = reinterpret_cast<const uint4*>(p.q + ((size_t)row * p.Hq + (size_t)g * p.G + (hl < p.G ? hl : 0)) * D);
#pragma unroll
        for (int c = 0; c < kSteps; ++c) {
            qf[c] = src[c * 4 + l4];
            if (hl >= p.G) qf[c] = make_uint4(0, 0, 0, 0);
        }
    }
    float o[kHalves][8][4];                        // [half][channel of the lane's chunk][rows 0-7: P_hi, rows 8-15: P_lo]
#pragma unroll
    for (int h = 0; h < kHalves; ++h)
#pragma unroll
        for (int c = 0; c < 8; ++c) o[h][c][0] = o[h][c][1] = o[h][c][2] = o[h][c][3] = 0.f;
    float m = kNegBig, l = 0.f;

    for (int i0 = lo + warp; i0 < hi; i0 += 32 * kPagesWarps) {
        // this warp's next 32 list entries, one per lane: physical page and valid tokens
        int phys = 0, valid = 0;
        const int ie = i0 + lane * kPagesWarps;
        if (ie < hi) {
            const int e = list[ie];
            if (e >= 0 && e <= at.pos / kPageTokens) {
                phys = table[e];
                valid = min(kPageTokens, at.pos - e * kPageTokens + 1);
            }
            if (valid == 0 || phys < 0 || phys >= p.num_pages) { atomicExch(p.status, AFLEX_ERR_BOUNDS); phys = 0; valid = 0; }
        }
        const int nb = min(32, (hi - i0 + kPagesWarps - 1) / kPagesWarps);
        uint4 kx[2][kSteps], vx[4][kHalves];
        auto load_k = [&](int j) {
            const size_t slab = (size_t)__shfl_sync(0xffffffffu, phys, j) * p.Hkv + g;
            const uint4* src = reinterpret_cast<const uint4*>(p.k_cache + slab * kPageTokens * D) + hl * (D / 8) + l4;
#pragma unroll
            for (int r = 0; r < 2; ++r)
#pragma unroll
                for (int c = 0; c < kSteps; ++c) kx[r][c] = ld_stream(src + r * D + c * 4);        // 8 rows are D sixteen-byte words
        };
        auto load_v = [&](int j) {
            const size_t slab = (size_t)__shfl_sync(0xffffffffu, phys, j) * p.Hkv + g;
            const int nv = __shfl_sync(0xffffffffu, valid, j);
            const uint4* src = reinterpret_cast<const uint4*>(p.v_cache + slab * kPageTokens * D) + hl;
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int t = 2 * l4 + (r & 1) + (r >> 1) * 8;
#pragma unroll
                for (int h = 0; h < kHalves; ++h) {
                    vx[r][h] = make_uint4(0, 0, 0, 0);                                             // slots past the end may hold NaN
                    if (t < nv) vx[r][h] = ld_stream(src + t * (D / 8) + h * 8);
                }
            }
        };
        load_k(0);
        load_v(0);
        for (int j = 0; j < nb; ++j) {
            const int nv = __shfl_sync(0xffffffffu, valid, j);
            float s[2][4];
#pragma unroll
            for (int r = 0; r < 2; ++r) {
                s[r][0] = s[r][1] = s[r][2] = s[r][3] = 0.f;
#pragma unroll
                for (int c = 0; c < kSteps; ++c) {
                    mma_bf16_16816(s[r], qf[c].x, 0u, qf[c].y, 0u, kx[r][c].x, kx[r][c].y);
                    mma_bf16_16816(s[r], qf[c].z, 0u, qf[c].w, 0u, kx[r][c].z, kx[r][c].w);
                }
            }
            if (j + 1 < nb) load_k(j + 1);
            if (nv > 0) {
                // tokens 2 l4, 2 l4 + 1 and those + 8 of head lane / 4
                float x0 = 2 * l4 < nv ? s[0][0] * p.scale_log2 : -INFINITY;
                float x1 = 2 * l4 + 1 < nv ? s[0][1] * p.scale_log2 : -INFINITY;
                float x2 = 2 * l4 + 8 < nv ? s[1][0] * p.scale_log2 : -INFINITY;
                float x3 = 2 * l4 + 9 < nv ? s[1][1] * p.scale_log2 : -INFINITY;
                float mx = fmaxf(fmaxf(x0, x1), fmaxf(x2, x3));
                mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 1));
                mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 2));
                if (__any_sync(0xffffffffu, mx > m)) {
                    const float mn = fmaxf(m, mx), corr = fast_exp2(m - mn);
                    m = mn;
                    l *= corr;
#pragma unroll
                    for (int h = 0; h < kHalves; ++h)
#pragma unroll
                        for (int c = 0; c < 8; ++c) { o[h][c][0] *= corr; o[h][c][1] *= corr; o[h][c][2] *= corr; o[h][c][3] *= corr; }
                }
                x0 = fast_exp2(x0 - m); x1 = fast_exp2(x1 - m); x2 = fast_exp2(x2 - m); x3 = fast_exp2(x3 - m);
                l += (x0 + x1) + (x2 + x3);
                const uint32_t a0 = pack_bf16x2(x0, x1), a2 = pack_bf16x2(x2, x3);
                const uint32_t a1 = pack_bf16x2(x0 - __uint_as_float(a0 << 16), x1 - __uint_as_float(a0 & 0xffff0000u));
                const uint32_t a3 = pack_bf16x2(x2 - __uint_as_float(a2 << 16), x3 - __uint_as_float(a2 & 0xffff0000u));
#pragma unroll
                for (int h = 0; h < kHalves; ++h) {
                    const uint32_t* r0 = reinterpret_cast<const uint32_t*>(&vx[0][h]);
                    const uint32_t* r1 = reinterpret_cast<const uint32_t*>(&vx[1][h]);
                    const uint32_t* r2 = reinterpret_cast<const uint32_t*>(&vx[2][h]);
                    const uint32_t* r3 = reinterpret_cast<const uint32_t*>(&vx[3][h]);
#pragma unroll
                    for (int w = 0; w < 4; ++w) {
                        mma_bf16_16816(o[h][2 * w], a0, a1, a2, a3, __byte_perm(r0[w], r1[w], 0x5410), __byte_perm(r2[w], r3[w], 0x5410));
                        mma_bf16_16816(o[h][2 * w + 1], a0, a1, a2, a3, __byte_perm(r0[w], r1[w], 0x7632), __byte_perm(r2[w], r3[w], 0x7632));
                    }
                }
            }
            if (j + 1 < nb) load_v(j + 1);
        }
    }
    // ---- join the warps, then the cluster's CTAs.  Lane: head lane / 4, channels 64 h + 16 l4 + 8 x + c at o[h][c][x].
    l += __shfl_xor_sync(0xffffffffu, l, 1);
    l += __shfl_xor_sync(0xffffffffu, l, 2);
#pragma unroll
    for (int h = 0; h < kHalves; ++h)
#pragma unroll
        for (int x = 0; x < 2; ++x) {
            float* dst = &sh.o[warp][hl][64 * h + 16 * l4 + 8 * x];
            *reinterpret_cast<float4*>(dst) = make_float4(o[h][0][x] + o[h][0][x + 2], o[h][1][x] + o[h][1][x + 2],
                                                          o[h][2][x] + o[h][2][x + 2], o[h][3][x] + o[h][3][x + 2]);
            *reinterpret_cast<float4*>(dst + 4) = make_float4(o[h][4][x] + o[h][4][x + 2], o[h][5][x] + o[h][5][x + 2],
                                                              o[h][6][x] + o[h][6][x + 2], o[h][7][x] + o[h][7][x + 2]);
        }
    if (l4 == 0) { sh.m[warp][hl] = m; sh.l[warp][hl] = l; }
    if (S > 1) { cluster_arrive(); cluster_wait(); } else __syncthreads();
    // The G * D outputs in runs of eight channels; CTA `rank` of the cluster makes its share of the runs
    for (int i = rank * kPagesThreads + tid; i < p.G * (D / 8); i += S * kPagesThreads) {
        const int h = i / (D / 8), c0 = (i % (D / 8)) * 8;
        float M = kNegBig, L = 0.f, acc[8];
#pragma unroll
        for (int c = 0; c < 8; ++c) acc[c] = 0.f;
        for (int s = 0; s < S; ++s) {
#pragma unroll
            for (int w = 0; w < kPagesWarps; ++w) {
                float pm, pl, v[8];
                if (S == 1) {
                    pm = sh.m[w][h]; pl = sh.l[w][h];
#pragma unroll
                    for (int c = 0; c < 8; ++c) v[c] = sh.o[w][h][c0 + c];
                } else {
                    pm = ld_cluster_f32(cluster_map_shared(smem_u32(&sh.m[w][h]), (uint32_t)s));
                    pl = ld_cluster_f32(cluster_map_shared(smem_u32(&sh.l[w][h]), (uint32_t)s));
                    const uint32_t base = cluster_map_shared(smem_u32(&sh.o[w][h][c0]), (uint32_t)s);
#pragma unroll
                    for (int c = 0; c < 8; ++c) v[c] = ld_cluster_f32(base + 4 * c);
                }
                const float mn = fmaxf(M, pm), ca = fast_exp2(M - mn), cb = fast_exp2(pm - mn);
                M = mn;
                L = L * ca + pl * cb;
#pragma unroll
                for (int c = 0; c < 8; ++c) acc[c] = acc[c] * ca + v[c] * cb;
            }
        }
        const float inv = L == 0.f ? 0.f : 1.f / L;           // a row with nothing to attend to: zeros
        uint4 y;
        y.x = pack_bf16x2(acc[0] * inv, acc[1] * inv); y.y = pack_bf16x2(acc[2] * inv, acc[3] * inv);
        y.z = pack_bf16x2(acc[4] * inv, acc[5] * inv); y.w = pack_bf16x2(acc[6] * inv, acc[7] * inv);
        const size_t hq = (size_t)row * p.Hq + (size_t)g * p.G + h;
        reinterpret_cast<uint4*>(p.out + hq * D)[c0 / 8] = y;
        if (p.lse != nullptr && c0 == 0) p.lse[hq] = L == 0.f ? -INFINITY : (M + log2f(L)) * 0.6931471805599453f;
    }
    if (S > 1) { cluster_arrive(); cluster_wait(); }          // the others' shared memory stays until everybody has read it
}

template <typename P>
cudaError_t launch_cluster(void (*kernel)(const P), long long ctas, int threads, size_t smem, int cluster, cudaStream_t st, const P& p) {
    cudaLaunchConfig_t lc = {};
    lc.gridDim = dim3((unsigned)ctas);
    lc.blockDim = dim3((unsigned)threads);
    lc.dynamicSmemBytes = smem;
    lc.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = (unsigned)cluster;
    attr[1].val.clusterDim.y = 1;
    attr[1].val.clusterDim.z = 1;
    lc.attrs = attr;
    lc.numAttrs = cluster > 1 ? 2 : 1;
    return cudaLaunchKernelEx(&lc, kernel, p);
}

}  // namespace

// ------------------------------------------------------------------------------------------ host
aflex_status page_select_launch(aflex_ctx* ctx, const aflex_attn_desc* d, const void* q, const aflex_kv* kv,
                                const aflex_key_bounds* bounds, const aflex_page_policy* policy, int batch, const int32_t* q_offsets,
                                int rows, int32_t* page_list, int32_t* page_count, cudaStream_t st) {
    SelectParams p;
    p.q = (const __nv_bfloat16*)q;
    p.codes = bounds->codes; p.scales = bounds->scales;
    p.page_table = kv->page_table; p.seq_lens = kv->seq_lens; p.q_offsets = q_offsets;
    p.batch = batch; p.max_pages = kv->max_pages_per_seq;
    p.Hq = d->num_q_heads; p.Hkv = d->num_kv_heads; p.G = p.Hq / p.Hkv; p.num_pages = kv->num_pages;
    p.top = policy->top_pages; p.sink = policy->sink_pages; p.window = policy->window_pages;
    p.list = page_list; p.count = page_count; p.status = ctx->dev_status;
    const long long items = (long long)rows * p.Hkv;
    int S = 1;
    while (S < kSelMaxCluster && (items * S < ctx->num_sms || p.max_pages > (long long)S * kSelKeyCap) && p.max_pages > S * kSelWarps * kSelTile) S *= 2;
    if (p.max_pages > (long long)S * kSelKeyCap)
        return set_error(ctx, AFLEX_ERR_UNSUPPORTED, "page select: max_pages_per_seq %d (supported: up to %d)", p.max_pages, kSelMaxCluster * kSelKeyCap);
    if (items * S > 0x7fffffffLL) return set_error(ctx, AFLEX_ERR_UNSUPPORTED, "page select: rows * Hkv = %lld", items);
    p.cluster = S;
    p.cap = kSelKeyCap < p.max_pages ? kSelKeyCap : p.max_pages;
    const size_t smem = (size_t)p.cap * 4;
    void (*kernel)(const SelectParams) = d->head_dim == 128 ? page_select_kernel<128> : page_select_kernel<64>;
    if (!ctx->select_attr_set[d->head_dim == 128]) {
        cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kSelKeyCap * 4);
        if (e != cudaSuccess) return check_cuda(ctx, e, "cudaFuncSetAttribute(page select)");
        ctx->select_attr_set[d->head_dim == 128] = true;
    }
    KernelScope scope(ctx, kKPageSelect, st);
    return check_cuda(ctx, launch_cluster(kernel, items * S, kSelThreads, smem, S, st, p), "page_select_kernel launch");
}

aflex_status attn_decode_pages_launch(aflex_ctx* ctx, const aflex_attn_desc* d, const void* q, const aflex_kv* kv,
                                      const int32_t* page_list, const int32_t* page_count, int top_pages, int batch,
                                      const int32_t* q_offsets, int rows, void* out, float* lse, cudaStream_t st) {
    PagesParams p;
    p.q = (const __nv_bfloat16*)q;
    p.k_cache = (const __nv_bfloat16*)kv->k_cache; p.v_cache = (const __nv_bfloat16*)kv->v_cache;
    p.page_table = kv->page_table; p.seq_lens = kv->seq_lens; p.q_offsets = q_offsets;
    p.list = page_list; p.count = page_count;
    p.batch = batch; p.max_pages = kv->max_pages_per_seq;
    p.Hq = d->num_q_heads; p.Hkv = d->num_kv_heads; p.G = p.Hq / p.Hkv; p.top = top_pages; p.num_pages = kv->num_pages;
    const float scale = d->sm_scale != 0.f ? d->sm_scale : 1.0f / sqrtf((float)d->head_dim);
    p.scale_log2 = scale * 1.4426950408889634f;
    p.out = (__nv_bfloat16*)out; p.lse = lse; p.status = ctx->dev_status;
    const long long items = (long long)rows * p.Hkv;
    int S = 1;
    while (S < 8 && items * S < 6LL * ctx->num_sms && top_pages > S * kPagesWarps) S *= 2;
    if (items * S > 0x7fffffffLL) return set_error(ctx, AFLEX_ERR_UNSUPPORTED, "attention over pages: rows * Hkv = %lld", items);
    p.cluster = S;
    void (*kernel)(const PagesParams) = d->head_dim == 128 ? attn_decode_pages_kernel<128> : attn_decode_pages_kernel<64>;
    KernelScope scope(ctx, kKAttnPages, st);
    return check_cuda(ctx, launch_cluster(kernel, items * S, kPagesThreads, 0, S, st, p), "attn_decode_pages_kernel launch");
}

}  // namespace aflex
