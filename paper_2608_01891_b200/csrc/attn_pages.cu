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

// A plain load, for what a preceding kernel may have written (queries, lists, lengths, bounds): these kernels may have started before that
// one was done and wait for it, so the read-only path (ld.global.nc) would not be bound to see its stores.
template <typename V> __device__ __forceinline__ V fetch(const V* p) { return *p; }

constexpr int kPageTokens = 16;
constexpr float kLowest = -3.402823466e38f;     // the lowest finite value: where running maxima start, so that no score lies below

// Sequence of a row, and how many of the sequence's rows follow it; every lane of a warp takes part.  Rows behind the last
// sequence's are padding: nothing is to be read, written or reported for them.
struct RowSeq { int b, back; bool padding; };
__device__ __forceinline__ RowSeq locate_row(int row, const int32_t* q_offsets, int batch) {
    RowSeq at;
    at.b = row; at.back = 0; at.padding = false;
    if (q_offsets != nullptr) {
        // largest b with q_offsets[b] <= row: the lanes look at 32 sequences at a time (one load's latency for up to 32)
        const int lane = threadIdx.x & 31, end = fetch(q_offsets + batch);
        int lo = 0, span = batch;
        while (span > 1) {
            const int step = (span + 31) / 32, i = lane * step;
            const unsigned le = __ballot_sync(0xffffffffu, i < span && fetch(q_offsets + lo + (i < span ? i : 0)) <= row);
            const int skip = max(__popc(le) - 1, 0) * step;
            lo += skip;
            span = min(step, span - skip);
        }
        at.b = lo;
        at.back = fetch(q_offsets + lo + 1) - 1 - row;
        at.padding = row >= end;
    }
    return at;
}
// Position of the row in its sequence of `len` tokens; -1 where the inputs give none.
__device__ __forceinline__ int row_position(const RowSeq& at, int len, int max_pages) {
    const int pos = len - 1 - at.back;
    return !at.padding && at.back >= 0 && pos >= 0 && len <= max_pages * kPageTokens ? pos : -1;
}

__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }
__device__ __forceinline__ void st_cluster_u32(uint32_t addr, uint32_t v) {
    asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(addr), "r"(v) : "memory");
}
__device__ __forceinline__ void st_cluster_v2(uint32_t addr, uint32_t x, uint32_t y) {
    asm volatile("st.shared::cluster.v2.u32 [%0], {%1, %2};" ::"r"(addr), "r"(x), "r"(y) : "memory");
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
__device__ __forceinline__ float4 ld_cluster_f32x4(uint32_t addr) {
    float4 v;
    asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(addr) : "memory");
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
// One CTA, or a cluster with a contiguous share of the candidate pages each, per (row, KV head); a warp scores tiles of 16 pages with
// integer MMAs, operands loaded from global memory straight into registers (the bounds' layout is the fragment's), and leaves
// the scores in shared memory.  A histogram of 256 equal intervals between the lowest and the highest score, summed over the
// cluster, tells the interval that holds the last page to keep, and the few pages of that interval are ranked by comparing all
// pairs (a crowded interval is divided again, by the scores' bits; a crowd of equal scores by page).  Every CTA draws the same
// conclusions and writes its share of the list.
//
// Bound: with hundreds of pages the chain of dependent steps (lengths and page ids -> bounds -> scores -> interval -> rank ->
// list), not the bytes; so as much as possible is loaded before it is known to be needed, and barriers are few.  A score
// takes some 60 instructions on its way through the selection, which is why a long row's selection is spread over the cluster.
constexpr int kSelTile = 16;
constexpr uint32_t kScaleMax = 127 + 50;            // largest exponent of the bounds, as stored
constexpr int kSelCap = 48 * 1024;                  // scores one CTA's shared memory holds
constexpr int kSelMaxCluster = 8;
constexpr size_t kSelRowsSmem = 190 * 1024;         // most dynamic shared memory of page_select_rows_kernel
constexpr int kSelRank = 64;                        // members of an interval that are ranked by comparing all pairs

struct SelectParams {
    const __nv_bfloat16* q;        // [rows][Hq][D]
    const int8_t* codes;
    const uint8_t* scales;
    const int32_t* page_table;
    const int32_t* seq_lens;
    const int32_t* q_offsets;
    int batch, rows, max_pages, Hq, Hkv, G;
    long long num_pages;
    int top, sink, window;
    int cluster;                   // CTAs per (row, KV head), or per group of rows and KV head
    int group, stride, row_warps;  // rows per group, floats per row of its scores, log2 of the warps that select for a row
    int32_t* list;                 // [rows][Hkv][top]
    int32_t* count;                // [rows][Hkv]
    int* status;
};

// What the (up to W) warps share that select for one row; CL: the most CTAs that they are spread over.
template <int W, int CL> struct SelectShared {
    __align__(16) int hist[256];   // this CTA's
    __align__(16) int sum[CL > 1 ? 256 : 4];       // the cluster's
    uint2 range[W];                // lowest and highest score of every warp, as ordered bits
    uint2 all_range[CL];
    int members;                   // of the interval that is ranked, in this CTA
    int all_members[CL];
    uint2 member[CL][kSelRank];    // (score, page) of every CTA's
    uint2 rank[CL > 1 ? kSelRank : 1];             // all of them in one piece
    float last_score;              // the last one to keep
    int last_page;
    int kept[W];                   // of every warp's run
    int all_kept[CL];              // of every CTA
};

__device__ __forceinline__ int q_exponent(float a) {             // smallest e with a <= 127 * 2^e, within [-60, 50]
    const int field = (int)((__float_as_uint(a) >> 23) & 255u);
    int e = field - 133;
    if (e >= -60 && e <= 50 && a * __uint_as_float((uint32_t)(127 - e) << 23) > 127.f) ++e;
    return max(-60, min(50, e));
}

// Quantises a 32-channel block of a group's queries: lane holds head lane / 4, channels 8 (lane % 4) .. + 7 in x.
__device__ __forceinline__ void quantise_block(uint4 x, int lane, uint4& out, float& f) {
    const uint32_t in[4] = {x.x, x.y, x.z, x.w};
    float v[8], a = 0.f;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        v[2 * i] = __uint_as_float(in[i] << 16); v[2 * i + 1] = __uint_as_float(in[i] & 0xffff0000u);
        a = fmaxf(a, fmaxf(fabsf(v[2 * i]), fabsf(v[2 * i + 1])));      // (a NaN is passed over)
    }
    a = fmaxf(a, __shfl_xor_sync(0xffffffffu, a, 1));
    a = fmaxf(a, __shfl_xor_sync(0xffffffffu, a, 2));
    const int e = q_exponent(a);
    const float inv = __uint_as_float((uint32_t)(127 - e) << 23);
    uint32_t w[2], neg[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        int z[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) z[k] = max(-127, min(127, __float2int_rn(v[4 * i + k] * inv)));        // NaN becomes 0
        w[i] = __byte_perm(__byte_perm(z[0], z[1], 0x0040), __byte_perm(z[2], z[3], 0x0040), 0x5410);
        neg[i] = w[i] & (((w[i] & 0x80808080u) >> 7) * 255u);                                               // bytes below zero
    }
    out = make_uint4(w[0] & ~neg[0], w[1] & ~neg[1], neg[0], neg[1]);
    f = __uint_as_float((uint32_t)(127 + e) << 23);
}

// The bounds of a tile's 16 pages as this lane's A operands: rows lane / 4 and + 8.  `ids`: page ids by lane, the tile's from
// lane `from` on; j: the candidate of row 0, of which those below `end` exist (of the others some page is loaded).
template <int D> struct Tile { uint4 x[2][D / 32]; uint32_t scale[2]; };
template <int D>
__device__ __forceinline__ void load_tile(Tile<D>& tile, const SelectParams& p, int g, int ids, int from, int j, int end) {
    const int lane = threadIdx.x & 31, hl = lane >> 2, l4 = lane & 3;
#pragma unroll
    for (int r = 0; r < 2; ++r) {
        int id = __shfl_sync(0xffffffffu, ids, from + hl + 8 * r);
        if (j + hl + 8 * r >= end) id = 0;
        if (id < 0 || id >= p.num_pages) { atomicExch(p.status, AFLEX_ERR_BOUNDS); id = 0; }
        const size_t slab = (size_t)id * p.Hkv + g;
        const uint4* src = reinterpret_cast<const uint4*>(p.codes + slab * (2 * D)) + l4;
#pragma unroll
        for (int c = 0; c < D / 32; ++c) tile.x[r][c] = fetch(src + c * 4);
        if (D == 128) tile.scale[r] = fetch(reinterpret_cast<const uint32_t*>(p.scales) + slab);
        else tile.scale[r] = fetch(reinterpret_cast<const uint16_t*>(p.scales) + slab);
    }
}
// Scores of a tile's pages: rows lane / 4 and + 8, MMA columns 2 (lane % 4) and + 1, in v as (row, column) 00, 01, 10, 11.
template <int D>
__device__ __forceinline__ void tile_scales(const Tile<D>& tile, float (&k0)[D / 32], float (&k1)[D / 32]) {
#pragma unroll
    for (int c = 0; c < D / 32; ++c) {
        // (bounds that nobody has made yet may hold any byte: none makes a score infinite or not a number)
        k0[c] = __uint_as_float(min((tile.scale[0] >> (8 * c)) & 255u, kScaleMax) << 23);
        k1[c] = __uint_as_float(min((tile.scale[1] >> (8 * c)) & 255u, kScaleMax) << 23);
    }
}
template <int D>
__device__ __forceinline__ void score_columns(const Tile<D>& tile, const float (&k0)[D / 32], const float (&k1)[D / 32],
                                              const uint4 (&qf)[D / 32], const float2 (&fq)[D / 32], float (&v)[4]) {
#pragma unroll
    for (int c = 0; c < D / 32; ++c) {
        int d[4] = {0, 0, 0, 0};
        mma_s8_16832(d, tile.x[0][c].x, tile.x[1][c].x, tile.x[0][c].y, tile.x[1][c].y, qf[c].x, qf[c].y);
        mma_s8_16832(d, tile.x[0][c].z, tile.x[1][c].z, tile.x[0][c].w, tile.x[1][c].w, qf[c].z, qf[c].w);
        // the products are exact, so a fused multiply-add rounds like the sum alone
        v[0] = fmaf((float)d[0] * k0[c], fq[c].x, c ? v[0] : 0.f);
        v[1] = fmaf((float)d[1] * k0[c], fq[c].y, c ? v[1] : 0.f);
        v[2] = fmaf((float)d[2] * k1[c], fq[c].x, c ? v[2] : 0.f);
        v[3] = fmaf((float)d[3] * k1[c], fq[c].y, c ? v[3] : 0.f);
    }
}
// The largest over a row's heads; lanes 4 i and 4 i + 1 return those of rows i and i + 8.
template <int D>
__device__ __forceinline__ float score_tile(const Tile<D>& tile, const uint4 (&qf)[D / 32], const float2 (&fq)[D / 32], int G) {
    const int l4 = threadIdx.x & 3;
    float k0[D / 32], k1[D / 32], s[4];
    tile_scales<D>(tile, k0, k1);
    score_columns<D>(tile, k0, k1, qf, fq, s);
    const bool h0 = 2 * l4 < G, h1 = 2 * l4 + 1 < G;
    float m0 = fmaxf(h0 ? s[0] : -INFINITY, h1 ? s[1] : -INFINITY);
    float m1 = fmaxf(h0 ? s[2] : -INFINITY, h1 ? s[3] : -INFINITY);
    m0 = fmaxf(m0, __shfl_xor_sync(0xffffffffu, m0, 1));
    m1 = fmaxf(m1, __shfl_xor_sync(0xffffffffu, m1, 1));
    m0 = fmaxf(m0, __shfl_xor_sync(0xffffffffu, m0, 2));
    m1 = fmaxf(m1, __shfl_xor_sync(0xffffffffu, m1, 2));
    return l4 ? m1 : m0;
}
// The list of a row that sees n pages of which nothing has to be chosen: all of them, or the first and the last ones.
__device__ __forceinline__ void list_without_choice(const SelectParams& p, long long item, int n, int tid, int threads) {
    int32_t* list = p.list + item * p.top;
    for (int i = tid; i < p.top; i += threads) {
        int v = i < n ? i : -1;
        if (n > p.top && i >= p.sink) v = n - p.top + i;
        list[i] = v;
    }
    if (tid == 0) p.count[item] = min(n, p.top);
}
// What is listed in any case of a row that sees n > top pages, by one warp.
__device__ __forceinline__ void list_forced(const SelectParams& p, long long item, int n) {
    const int lane = threadIdx.x & 31;
    int32_t* list = p.list + item * p.top;
    for (int i = lane; i < p.sink; i += 32) list[i] = i;
    for (int i = lane; i < p.window; i += 32) list[p.top - p.window + i] = n - p.window + i;
    if (lane == 0) p.count[item] = p.top;
}

// Keeps the `keep` best of a row's `cand` candidates and writes them to list[sink ..], ascending.  This CTA (of S in the
// cluster) holds the scores of [c0, c1); low and high are the extremes of what the thread has seen of them.  `share`: the most
// tiles that a CTA holds.  The histogram and the member count are zero on entry.  `warps` neighbouring warps work on it (this
// thread is number tid of theirs), which meet at hardware barrier `barrier`.
template <int W, int CL>
__device__ __forceinline__ void select_pages(SelectShared<W, CL>& sh, int tid, int warps, int barrier, const float* scores, int S, int rank, int cand, int c0, int c1, int share,
                                             float low, float high, int keep, int sink, int32_t* list) {
    const int threads = warps * 32, lane = tid & 31, warp = tid >> 5;
    const unsigned below = (1u << lane) - 1u;
    // ---- division.  What the CTAs tell one another goes through shared memory that is written before a barrier and read after.
    auto sync = [&]() { asm volatile("bar.sync %0, %1;" ::"r"(barrier), "r"(threads) : "memory"); };
    auto sync_all = [&]() {
        if (CL > 1 && S > 1) { cluster_arrive(); cluster_wait(); } else sync();
    };
    auto bits_of = [](float s) -> uint32_t { const uint32_t u = __float_as_uint(s + 0.f); return u ^ ((u >> 31) ? 0xffffffffu : 0x80000000u); };
    auto score_of = [](uint32_t u) -> float { return __uint_as_float(u ^ ((u >> 31) ? 0x80000000u : 0xffffffffu)); };
    uint32_t lo = __reduce_min_sync(0xffffffffu, bits_of(low)), hi = __reduce_max_sync(0xffffffffu, bits_of(high));
    if (lane == 0) sh.range[warp] = make_uint2(lo, hi);
    sync();
    uint2 r = sh.range[lane < warps ? lane : 0];
    lo = __reduce_min_sync(0xffffffffu, r.x); hi = __reduce_max_sync(0xffffffffu, r.y);
    if (CL > 1 && S > 1) {
        if (warp == 0 && lane < S) st_cluster_v2(cluster_map_shared(smem_u32(&sh.all_range[rank]), (uint32_t)lane), lo, hi);
        sync_all();
        r = sh.all_range[lane % S];
        lo = __reduce_min_sync(0xffffffffu, r.x); hi = __reduce_max_sync(0xffffffffu, r.y);
    }
    low = score_of(lo); high = score_of(hi);
    // 256 intervals of equal width.  (One fused operation rounds monotonically: a higher score is never in a lower interval.)
    const float per = 256.f / fmaxf(high - low, 1e-30f), shift_by = -low * per;
    auto interval = [&](float s) -> int { return max(0, min(255, (int)fmaf(s, per, shift_by))); };
    // f(candidate, its score, whether there is one) over the warp's run of the CTA's candidates, all lanes together
    const int steps = (share * kSelTile + threads - 1) / threads;
    const int j0 = c0 + warp * steps * 32 + lane, j1 = min(c1, c0 + (warp + 1) * steps * 32);
    auto each = [&](auto f) {
#pragma unroll 2
        for (int s = 0; s < steps; ++s) {
            const int j = j0 + 32 * s;
            f(j, j < j1 ? scores[j - c0] : 0.f, j < j1);
        }
    };
    // Sums the CTAs' histograms and counts from the top: the interval in which the need-th highest lies, what lies above it
    // (taken off need) and in it.  Every warp counts by itself: lane i has intervals 255 - 8 i .. 248 - 8 i.
    int need = keep, bin = 0, inside = 0;
    auto divide = [&]() {
        sync_all();                                                // the histograms are complete
        if (CL > 1 && S > 1) {
            for (int i = tid; i < 256; i += threads) {
                uint32_t v[CL], sum = 0;
#pragma unroll
                for (int s = 0; s < CL; ++s) v[s] = ld_cluster_u32(cluster_map_shared(smem_u32(&sh.hist[i]), (uint32_t)(s < S ? s : 0)));
#pragma unroll
                for (int s = 0; s < CL; ++s) sum += s < S ? v[s] : 0u;
                sh.sum[i] = (int)sum;
            }
            sync();
        }
        const int* h = CL > 1 && S > 1 ? sh.sum : sh.hist;
        const int4 a = *reinterpret_cast<const int4*>(h + 248 - 8 * lane), b = *reinterpret_cast<const int4*>(h + 252 - 8 * lane);
        const int sum = a.x + a.y + a.z + a.w + b.x + b.y + b.z + b.w;
        int incl = sum;
#pragma unroll
        for (int off = 1; off < 32; off <<= 1) {
            const int v = __shfl_up_sync(0xffffffffu, incl, off);
            if (lane >= off) incl += v;
        }
        const int from = __ffs(__ballot_sync(0xffffffffu, incl - sum < need && incl >= need)) - 1;     // (there is one: all are counted)
        need -= __shfl_sync(0xffffffffu, incl - sum, from);
        for (bin = 255 - 8 * from; bin > 248 - 8 * from && h[bin] < need; --bin) need -= h[bin];
        inside = h[bin];
    };
    each([&](int, float s, bool in) { if (in) atomicAdd(&sh.hist[interval(s)], 1); });
    divide();
    const int first_bin = bin;
    // A crowded interval is divided by the scores' bits (in numeric order) and, where a crowd of equal ones is left, by page.
    // Of the members in [lo, hi] -- bits, or once `by_page` is set mirrored pages -- the `need` largest are to be kept.
    uint32_t equal = 0;
    bool by_page = false;
    auto value = [&](int j, float s) -> uint32_t { return by_page ? (uint32_t)(cand - 1 - j) : bits_of(s); };
    auto member = [&](int j, float s) -> bool {
        if (interval(s) != first_bin) return false;
        const uint32_t v = value(j, s);
        return v >= lo && v <= hi && (!by_page || bits_of(s) == equal);
    };
    while (inside > kSelRank && inside > need) {
        sync_all();                                                // everybody has read the histograms
        for (int i = tid; i < 256; i += threads) sh.hist[i] = 0;
        sync();
        const int shift = max(0, 24 - __clz(hi - lo));
        each([&](int j, float s, bool in) { if (in && member(j, s)) atomicAdd(&sh.hist[(value(j, s) - lo) >> shift], 1); });
        divide();
        lo += (uint32_t)bin << shift;
        hi = min(hi, lo + ((1u << shift) - 1u));
        if (shift == 0 && !by_page && inside > kSelRank && inside > need) {
            by_page = true;                                        // equal scores: the lowest pages go first
            equal = lo;
            lo = 0;
            hi = (uint32_t)(cand - 1);
        }
    }
    // Kept are the candidates above the interval, and of its members those before (last bits, last page) in the order.
    uint32_t last;
    int last_page;
    if (inside > kSelRank) {                                       // (all members are kept)
        last = by_page ? equal : lo;
        last_page = by_page ? cand - 1 - (int)lo : 0x7fffffff;
    } else {
        // every member goes to every CTA's copy of its CTA's list
        each([&](int j, float s, bool in) {
            if (in && member(j, s)) {
                const int i = atomicAdd(&sh.members, 1);
                if (CL == 1 || S == 1) sh.member[0][i] = make_uint2(__float_as_uint(s), (uint32_t)j);       // (cluster or not: this CTA's)
                else for (int c = 0; c < S; ++c)
                    st_cluster_v2(cluster_map_shared(smem_u32(&sh.member[rank][i]), (uint32_t)c), __float_as_uint(s), (uint32_t)j);
            }
        });
        sync();
        if (CL > 1 && S > 1) {
            if (tid < S) st_cluster_u32(cluster_map_shared(smem_u32(&sh.all_members[rank]), (uint32_t)tid), (uint32_t)sh.members);
            sync_all();
            const int m = lane < S ? sh.all_members[lane] : 0;
            int end = m;
#pragma unroll
            for (int off = 1; off < CL; off <<= 1) {
                const int v = __shfl_up_sync(0xffffffffu, end, off);
                if (lane >= off) end += v;
            }
            // the warps pack the CTAs' lists in turn
            for (int c = warp; c < S; c += warps) {
                const int mc = __shfl_sync(0xffffffffu, m, c), to = __shfl_sync(0xffffffffu, end, c) - mc;
                for (int i = lane; i < mc; i += 32) sh.rank[to + i] = sh.member[c][i];
            }
            sync();
        }
        const uint2* members = CL > 1 && S > 1 ? sh.rank : sh.member[0];
        for (int m = tid; m < inside; m += threads) {              // (a row's one warp has fewer threads than there may be members)
            const float s = __uint_as_float(members[m].x);
            const uint32_t j = members[m].y;
            int before = 0;
#pragma unroll 4
            for (int i = 0; i < inside; ++i) {
                const uint2 o = members[i];
                before += __uint_as_float(o.x) > s || (__uint_as_float(o.x) == s && o.y < j);
            }
            if (before == need - 1) { sh.last_score = s; sh.last_page = (int)j; }
        }
        sync();
        last = bits_of(sh.last_score);
        last_page = sh.last_page;
    }
    auto keeps = [&](int j, float s) -> bool {
        const int i = interval(s);
        if (i != first_bin) return i > first_bin;
        const uint32_t u = bits_of(s);
        return u > last || (u == last && j <= last_page);
    };
    // ---- the list, ascending: each warp places its run's
    int kept = 0;
    each([&](int j, float s, bool in) { kept += in && keeps(j, s); });
    kept = __reduce_add_sync(0xffffffffu, kept);
    if (lane == 0) sh.kept[warp] = kept;
    sync();
    const int k = lane < warps ? sh.kept[lane] : 0;
    int base = __reduce_add_sync(0xffffffffu, lane < warp ? k : 0);
    if (CL > 1 && S > 1) {
        const uint32_t all = (uint32_t)__reduce_add_sync(0xffffffffu, k);
        if (tid < S) st_cluster_u32(cluster_map_shared(smem_u32(&sh.all_kept[rank]), (uint32_t)tid), all);
        sync_all();                                                // behind it nobody reads another CTA's shared memory
        base += __reduce_add_sync(0xffffffffu, lane < rank ? sh.all_kept[lane] : 0);
    }
    int32_t* to = list + sink;
    each([&](int j, float s, bool in) {
        const bool mine = in && keeps(j, s);
        const unsigned who = __ballot_sync(0xffffffffu, mine);
        const int at = base + __popc(who & below);
        if (mine && at < keep) to[at] = sink + j;                  // (exactly `keep` are kept; no store leaves their place in any case)
        base += __popc(who);
    });
}

template <int D, int W, int O>                      // W warps, O CTAs per SM
__global__ void __launch_bounds__(W * 32, O) page_select_kernel(const SelectParams p) {
    constexpr int kBlocks = D / 32;
    constexpr int kThreads = W * 32;
    constexpr int kTiles = W * O <= 16 ? 2 : 1;                    // tiles a warp has in flight (the lanes hold two tiles' page ids)
    extern __shared__ __align__(16) uint8_t smem_raw[];
    float* scores = reinterpret_cast<float*>(smem_raw);            // of this CTA's candidates
    __shared__ SelectShared<W, kSelMaxCluster> sh;
    __shared__ uint4 s_q[kBlocks][32];                            // quantised queries as the lanes' B operands: two words of positive parts, two of negative
    __shared__ float s_f[kBlocks][8];                             // 2^f per block and head
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int S = p.cluster, rank = (int)(blockIdx.x % S);
    const long long item = blockIdx.x / S;
    const int row = (int)(item / p.Hkv), g = (int)(item % p.Hkv);
    const int hl = lane >> 2, l4 = lane & 3;
    if (S > 1) cluster_arrive();                                  // the cluster's CTAs have started: waited for below
    for (int i = tid; i < 256; i += kThreads) sh.hist[i] = 0;
    if (tid == 0) sh.members = 0;
    pdl_launch_dependents();
    pdl_wait();
    // The first four warps quantise a block of the queries each: lane holds head lane / 4, channels 8 (lane % 4) .. + 7.
    const bool quantises = warp < kBlocks;
    uint4 qx = make_uint4(0, 0, 0, 0);
    if (quantises && hl < p.G)
        qx = fetch(reinterpret_cast<const uint4*>(p.q + ((size_t)row * p.Hq + (size_t)g * p.G + hl) * D) + warp * 4 + l4);
    const RowSeq at = locate_row(row, p.q_offsets, p.batch);
    const int len = fetch(p.seq_lens + at.b);
    const int32_t* table = p.page_table + (size_t)at.b * p.max_pages;
    // The lanes hold the page ids of two of the warp's tiles (lane / 16).  With one CTA the warp's tiles do not depend on the
    // length, so the first ids are loaded along with it (whatever the table's row holds beyond the sequence).
    auto page_ids = [&](int t) -> int {
        const long long j = p.sink + (long long)(t + (lane >> 4) * W) * kSelTile + (lane & 15);
        return fetch(table + min(j, (long long)p.max_pages - 1));
    };
    int t = warp, ids = S == 1 ? page_ids(t) : 0;
    const int pos = row_position(at, len, p.max_pages), n = pos >= 0 ? pos / kPageTokens + 1 : 0;
    if (pos < 0 && !at.padding && tid == 0 && rank == 0) atomicExch(p.status, AFLEX_ERR_BOUNDS);
    int32_t* list = p.list + item * p.top;
    const int keep = p.top - p.sink - p.window;                   // scored pages to keep
    const int cand = n - p.sink - p.window;                       // scored pages
    if (n <= p.top || keep == 0) {                                // nothing to choose (the same for the whole cluster)
        if (S > 1) cluster_wait();
        if (rank == 0 && !at.padding) list_without_choice(p, item, n, tid, kThreads);
        return;
    }
    if (quantises) {
        float f;
        quantise_block(qx, lane, s_q[warp][lane], f);
        if (l4 == 0) s_f[warp][hl] = f;
    }
    if (rank == 0 && warp == W - 1) list_forced(p, item, n);
    __syncthreads();
    uint4 qf[kBlocks];
    float2 fq[kBlocks];                                           // of this lane's two accumulator columns
#pragma unroll
    for (int c = 0; c < kBlocks; ++c) {
        qf[c] = s_q[c][lane];
        fq[c] = *reinterpret_cast<const float2*>(&s_f[c][2 * l4]);
    }
    if (S > 1) cluster_wait();
    // ---- scores of this CTA's candidates [c0, c1)
    const int tiles = (cand + kSelTile - 1) / kSelTile, share = (tiles + S - 1) / S;
    const int c0 = min(cand, rank * share * kSelTile), c1 = min(cand, c0 + share * kSelTile);
    const int t_end = min(tiles, (rank + 1) * share);
    float low = INFINITY, high = -INFINITY;
    if (S > 1) {
        t += rank * share;
        ids = page_ids(t);
    }
    while (t < t_end) {
        Tile<D> tile[kTiles];
#pragma unroll
        for (int k = 0; k < kTiles; ++k) load_tile<D>(tile[k], p, g, ids, k * 16, (t + k * W) * kSelTile, c1);
        const int t_now = t;
        t += kTiles * W;
        if (t < t_end) ids = page_ids(t);
#pragma unroll
        for (int k = 0; k < kTiles; ++k) {
            const float v = score_tile<D>(tile[k], qf, fq, p.G);
            const int j = (t_now + k * W) * kSelTile + hl + 8 * l4;
            if (l4 < 2 && j < c1) {
                low = fminf(low, v);
                high = fmaxf(high, v);
                scores[j - c0] = v;
            }
        }
    }
    select_pages(sh, tid, W, 0, scores, S, rank, cand, c0, c1, share, low, high, keep, p.sink, list);
}

// The same for several rows of one sequence (drafted tokens, a prompt chunk): a CTA, or a cluster of them, per group of `group`
// neighbouring rows and KV head.  Every warp scores a share of the pages for all of the rows, so that a page's bounds are read once
// for them -- read once per row they are what bounds the kernel above when rows are many: an SM takes some 32 bytes a cycle out of
// L2 -- with the columns of the MMA filled by as many rows as their heads fit.  The scores go to the shared memory of the CTA that
// selects for the row, WR warps for each of its W / WR rows.  Rows of different sequences in one group (the host can only guess
// where sequences end) are scored one after another by their own CTAs.
template <int D, int W, int O>                      // W warps, O CTAs per SM
__global__ void __launch_bounds__(W * 32, O) page_select_rows_kernel(const SelectParams p) {
    constexpr int kBlocks = D / 32, kSlots = kSelMaxCluster;
    extern __shared__ __align__(16) uint8_t smem_raw[];
    const int R = p.group, C = p.cluster;                                         // CTA i has rows i, i + C, ...
    const int per = 8 / p.G, all_sets = (R + per - 1) / per;                      // rows that fill the MMA's 8 columns; sets of them
    uint4* queries = reinterpret_cast<uint4*>(smem_raw);                          // [set][kBlocks][32]
    float* factors = reinterpret_cast<float*>(queries + all_sets * kBlocks * 32); // [set][kBlocks][8]
    float* scores = factors + all_sets * kBlocks * 8;                             // [slot][stride]
    __shared__ SelectShared<W, 1> sh[kSlots];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int hl = lane >> 2, l4 = lane & 3;
    const int rank = (int)(blockIdx.x % C), g = (int)(blockIdx.x / C % p.Hkv), row0 = (int)(blockIdx.x / C / p.Hkv) * R;
    const int nrows = min(R, p.rows - row0);
    const int WR = 1 << p.row_warps, row_threads = WR * 32;
    const int slot = warp >> p.row_warps, my_row = rank + slot * C, t_row = tid & (row_threads - 1);              // what this warp selects for
    if (C > 1) cluster_arrive();
    if (slot < kSlots) {
        for (int i = t_row; i < 256; i += row_threads) sh[slot].hist[i] = 0;
        if (t_row == 0) sh[slot].members = 0;
    }
    pdl_launch_dependents();
    pdl_wait();
    // A warp quantises up to kPairs (set, block) pairs of the group's queries; they are loaded before it is known which are needed.
    constexpr int kPairs = kSelMaxCluster * kBlocks / W;
    uint4 qx[kPairs];
#pragma unroll
    for (int k = 0; k < kPairs; ++k) {
        const int i = warp + k * W, r = i / kBlocks * per + hl / p.G;
        qx[k] = make_uint4(0, 0, 0, 0);
        if (r < nrows)
            qx[k] = fetch(reinterpret_cast<const uint4*>(p.q + ((size_t)(row0 + r) * p.Hq + (size_t)g * p.G + hl % p.G) * D) + (i % kBlocks) * 4 + l4);
    }
    const RowSeq first = locate_row(row0, p.q_offsets, p.batch);
    const bool shared = !first.padding && first.back >= nrows - 1;                // all rows of the group in one sequence
    const int first_len = fetch(p.seq_lens + first.b);
    const int keep = p.top - p.sink - p.window, forced = p.sink + p.window;
    auto visible = [&](const RowSeq& at, int len) -> int {                        // pages a row sees
        const int pos = row_position(at, len, p.max_pages);
        return pos >= 0 ? pos / kPageTokens + 1 : 0;
    };
    const uint32_t scores_addr = smem_u32(scores);
    // Scores of the first `cand` candidates of a sequence, tiles from t on, for the rows [ra, rb) of the group.
    auto score = [&](int b, int cand, int ra, int rb, int t, int step) {
        const int32_t* table = p.page_table + (size_t)b * p.max_pages;
        auto page_ids = [&](int t) -> int {
            const long long j = p.sink + (long long)t * kSelTile + (lane & 15);
            return fetch(table + min(j, (long long)p.max_pages - 1));
        };
        const int tiles = (cand + kSelTile - 1) / kSelTile;
        int ids = t < tiles ? page_ids(t) : 0;
        for (; t < tiles; t += step) {
            Tile<D> tile;
            load_tile<D>(tile, p, g, ids, 0, t * kSelTile, cand);
            if (t + step < tiles) ids = page_ids(t + step);
            const int j0 = t * kSelTile + hl;
            float k0[kBlocks], k1[kBlocks];
            tile_scales<D>(tile, k0, k1);
            for (int s = ra / per; s * per < rb; ++s) {
                float v[4];                                                       // (page, column): (hl, 2 l4), (hl, 2 l4 + 1), (hl + 8, ..)
                uint4 qf[kBlocks];
                float2 fq[kBlocks];
#pragma unroll
                for (int c = 0; c < kBlocks; ++c) {
                    qf[c] = queries[(s * kBlocks + c) * 32 + lane];
                    fq[c] = *reinterpret_cast<const float2*>(factors + (s * kBlocks + c) * 8 + 2 * l4);
                }
                score_columns<D>(tile, k0, k1, qf, fq, v);
                auto put = [&](int r, int j, float s) {
                    if (r < ra || r >= rb || j >= cand) return;
                    if (C == 1) scores[r * p.stride + j] = s;
                    else st_cluster_u32(cluster_map_shared(scores_addr + (uint32_t)(r / C * p.stride + j) * 4, (uint32_t)(r % C)), __float_as_uint(s));
                };
                if (p.G == 1) {
                    const int r = s * per + 2 * l4;
                    put(r, j0, v[0]); put(r + 1, j0, v[1]); put(r, j0 + 8, v[2]); put(r + 1, j0 + 8, v[3]);
                } else {
                    float m0 = fmaxf(v[0], v[1]), m1 = fmaxf(v[2], v[3]);
                    if (p.G == 2) { put(s * per + l4, j0, m0); put(s * per + l4, j0 + 8, m1); }
                    else {
                        m0 = fmaxf(m0, __shfl_xor_sync(0xffffffffu, m0, 1));
                        m1 = fmaxf(m1, __shfl_xor_sync(0xffffffffu, m1, 1));
                        if (p.G == 8) {
                            m0 = fmaxf(m0, __shfl_xor_sync(0xffffffffu, m0, 2));
                            m1 = fmaxf(m1, __shfl_xor_sync(0xffffffffu, m1, 2));
                        }
                        // lanes 0 and 1 of a row's two or four store
                        if (p.G == 4 || l4 < 2) put(s * per + (p.G == 4 ? l4 >> 1 : 0), j0 + 8 * (l4 & 1), l4 & 1 ? m1 : m0);
                    }
                }
            }
        }
    };
    RowSeq last = first;
    last.back -= nrows - 1;
    const int n_all = shared ? visible(last, first_len) : 0;                      // pages that the group's last row sees
#pragma unroll
    for (int k = 0; k < kPairs; ++k) {
        const int i = warp + k * W;
        if (i < all_sets * kBlocks) {
            float f;
            quantise_block(qx[k], lane, queries[i * 32 + lane], f);
            if (l4 == 0) factors[i * 8 + hl] = f;
        }
    }
    __syncthreads();
    if (C > 1) cluster_wait();                                                    // the group's CTAs have started
    RowSeq at = first;
    int len = first_len;
    if (shared) {
        at.back = first.back - my_row;
        if (n_all > p.top && keep > 0) score(first.b, n_all - forced, 0, nrows, rank * W + warp, C * W);
    } else {
        for (int r = rank; r < nrows; r += C) {
            const RowSeq here = locate_row(row0 + r, p.q_offsets, p.batch);
            const int here_len = fetch(p.seq_lens + here.b), n = visible(here, here_len);
            if (r == my_row) { at = here; len = here_len; }
            if (n > p.top && keep > 0) score(here.b, n - forced, r, r + 1, warp, W);
        }
    }
    if (C > 1) { cluster_arrive(); cluster_wait(); } else __syncthreads();        // behind it nobody writes another CTA's shared memory
    if (my_row >= nrows || at.padding) return;
    const int n = visible(at, len);
    if (n == 0 && t_row == 0) atomicExch(p.status, AFLEX_ERR_BOUNDS);
    const long long item = (long long)(row0 + my_row) * p.Hkv + g;
    if (n <= p.top || keep == 0) {
        list_without_choice(p, item, n, t_row, row_threads);
        return;
    }
    if (t_row < 32) list_forced(p, item, n);
    const int own = n - forced;                                                   // (an earlier row may see a page less)
    const float* mine = scores + slot * p.stride;
    float low = INFINITY, high = -INFINITY;
    for (int j = t_row; j < own; j += row_threads) { low = fminf(low, mine[j]); high = fmaxf(high, mine[j]); }
    select_pages(sh[slot], t_row, WR, 1 + slot, mine, 1, 0, own, 0, own, (own + kSelTile - 1) / kSelTile, low, high, keep, p.sink, p.list + item * p.top);
}

// ------------------------------------------------------------------------------------------ attention over listed pages
//
// For row r at position t and query head h of KV head g, over the tokens j <= t of the listed pages:
//   s_j = sm_scale <q, K_j>,  out = sum_j softmax(s)_j V_j,  lse = ln sum_j exp(s_j)
//
// Bound: the K and V bytes of the listed pages.  Every page is 4 KB of K and 4 KB of V (D = 128) somewhere in HBM, read once
// by one warp through a ring of pages of its own (asynchronous 16-byte copies, so what is in flight does not cost registers).
// Warps share nothing until the end: no barrier in the loop, only the warp's own copy groups.
// With the channels of a row permuted alike for q and K (a sum does not mind), sixteen contiguous bytes per lane are MMA
// fragments as they are, S = Q K^T leaves P in the layout of the second product's A operand, and V's fragments are two rows'
// words interleaved.  The copies swizzle the 16-byte chunks of a row so that both reads are free of bank conflicts.
// The MMA has 16 rows and a group at most 8 heads: the other 8 rows carry the low half of P (P = P_hi + P_lo, both bf16), so
// the second product loses nothing to the rounding of P.
// Lists are short (tens to a few hundred pages), so the work is split by (row, KV head) and, where those are few, the list is
// dealt out page by page over a cluster's CTAs and warps (which page is whose does not depend on the count, so the list entry
// is loaded along with it); each keeps its own running maximum and sum, joined at the end through shared memory.
constexpr int kPagesWarps = 4;
constexpr int kPagesThreads = kPagesWarps * 32;
constexpr int kPagesMaxCluster = 8;

struct PagesParams {
    const __nv_bfloat16* q;
    const __nv_bfloat16* k_cache;
    const __nv_bfloat16* v_cache;
    const int32_t* page_table;
    const int32_t* seq_lens;
    const int32_t* q_offsets;
    const int32_t* list;           // [rows][Hkv][top]
    const int32_t* count;          // [rows][Hkv]
    int batch, rows, max_pages, Hq, Hkv, G, top, cluster;
    long long num_pages;
    float scale_log2;
    __nv_bfloat16* out;
    float* lse;
    int* status;
};

// O CTAs per SM: two (D = 64: three) with a deep ring, or one more with a ring of two.
template <int D, int O> struct PagesRing {
    static constexpr int kStages = D == 128 ? (O == 2 ? 3 : 2) : (O == 3 ? 4 : 2);
    static constexpr int kPageBytes = kPageTokens * D * 2;            // of K; as many of V
    static constexpr int kWarpBytes = kStages * 2 * kPageBytes;       // holds the warp's state (8 heads x D floats) at the end
    static constexpr int kBytes = kPagesWarps * kWarpBytes;
};

struct PagesShared {
    float m[kPagesWarps][8], l[kPagesWarps][8];
    float cm[8], cl[8];            // the CTA's own, joined
    int valid[kPagesWarps][4];     // tokens of the page in each stage of the ring
};

__device__ __forceinline__ void copy16(uint32_t dst, const void* src, int bytes) {      // fewer than 16 bytes: the rest is zero
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}
__device__ __forceinline__ void copy_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void copy_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }
__device__ __forceinline__ uint4 lds128(uint32_t addr) {
    uint4 v;
    asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(addr) : "memory");
    return v;
}
// Place of a row's 16-byte chunk: K is read as (8 rows) x (4 neighbouring chunks) per instruction, V as (rows 0, 2, 4, 6 or
// 1, 3, 5, 7) x (8 chunks); either way the eight lanes of a bank cycle then touch eight different 16-byte banks.
__device__ __forceinline__ int swizzle(int row) { return (((row >> 1) & 3) << 1) ^ ((row & 1) << 2); }

// One page for one warp: K at shared address kp, V at vp (swizzled rows), the first nv > 0 tokens of it.
template <int D> struct PageState {
    float o[D / 64][8][4];                         // [half][channel of the lane's chunk][rows 0-7: P_hi, rows 8-15: P_lo]
    float m, l;
    __device__ __forceinline__ void reset() {
#pragma unroll
        for (int h = 0; h < D / 64; ++h)
#pragma unroll
            for (int c = 0; c < 8; ++c) o[h][c][0] = o[h][c][1] = o[h][c][2] = o[h][c][3] = 0.f;
        m = kLowest;
        l = 0.f;
    }
};
template <int D>
__device__ __forceinline__ void attend_page(PageState<D>& st, uint32_t kp, uint32_t vp, int nv, const uint4 (&qf)[D / 32], float scale_log2) {
    constexpr int kSteps = D / 32;                 // 16-byte reads per lane and K row
    constexpr int kHalves = D / 64;                // 16-byte reads per lane and V row
    const int lane = threadIdx.x & 31, hl = lane >> 2, l4 = lane & 3;
    auto& o = st.o;
    float& m = st.m;
    float& l = st.l;
                float s[2][4];
#pragma unroll
                for (int r = 0; r < 2; ++r) {
                    s[r][0] = s[r][1] = s[r][2] = s[r][3] = 0.f;
                    const int t = hl + 8 * r;
#pragma unroll
                    for (int c = 0; c < kSteps; ++c) {
                        const uint4 x = lds128(kp + (uint32_t)(t * (D * 2) + (((c * 4 + l4) ^ swizzle(t)) << 4)));
                        mma_bf16_16816(s[r], qf[c].x, 0u, qf[c].y, 0u, x.x, x.y);
                        mma_bf16_16816(s[r], qf[c].z, 0u, qf[c].w, 0u, x.z, x.w);
                    }
                }
                // tokens 2 l4, 2 l4 + 1 and those + 8 of head lane / 4
                float x0 = 2 * l4 < nv ? s[0][0] * scale_log2 : -INFINITY;
                float x1 = 2 * l4 + 1 < nv ? s[0][1] * scale_log2 : -INFINITY;
                float x2 = 2 * l4 + 8 < nv ? s[1][0] * scale_log2 : -INFINITY;
                float x3 = 2 * l4 + 9 < nv ? s[1][1] * scale_log2 : -INFINITY;
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
                    uint4 v[4];
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        const int t = 2 * l4 + (r & 1) + (r >> 1) * 8;
                        v[r] = lds128(vp + (uint32_t)(t * (D * 2) + (((h * 8 + hl) ^ swizzle(t)) << 4)));
                    }
                    const uint32_t* r0 = reinterpret_cast<const uint32_t*>(&v[0]);
                    const uint32_t* r1 = reinterpret_cast<const uint32_t*>(&v[1]);
                    const uint32_t* r2 = reinterpret_cast<const uint32_t*>(&v[2]);
                    const uint32_t* r3 = reinterpret_cast<const uint32_t*>(&v[3]);
#pragma unroll
                    for (int w = 0; w < 4; ++w) {
                        mma_bf16_16816(o[h][2 * w], a0, a1, a2, a3, __byte_perm(r0[w], r1[w], 0x5410), __byte_perm(r2[w], r3[w], 0x5410));
                        mma_bf16_16816(o[h][2 * w + 1], a0, a1, a2, a3, __byte_perm(r0[w], r1[w], 0x7632), __byte_perm(r2[w], r3[w], 0x7632));
                    }
                }
}
// Leaves a warp's state in shared memory: [8 heads][D] unnormalised sums at `to`, maximum and sum at m_to / l_to [8].
// Lane: head lane / 4, channels 64 h + 16 l4 + 8 x + c at o[h][c][x].
template <int D>
__device__ __forceinline__ void park_state(const PageState<D>& st, float* to, float* m_to, float* l_to) {
    const int lane = threadIdx.x & 31, hl = lane >> 2, l4 = lane & 3;
    float l = st.l;
    l += __shfl_xor_sync(0xffffffffu, l, 1);
    l += __shfl_xor_sync(0xffffffffu, l, 2);
    const auto& o = st.o;
#pragma unroll
    for (int h = 0; h < D / 64; ++h)
#pragma unroll
        for (int x = 0; x < 2; ++x) {
            float* dst = to + hl * D + 64 * h + 16 * l4 + 8 * x;
            *reinterpret_cast<float4*>(dst) = make_float4(o[h][0][x] + o[h][0][x + 2], o[h][1][x] + o[h][1][x + 2],
                                                          o[h][2][x] + o[h][2][x + 2], o[h][3][x] + o[h][3][x + 2]);
            *reinterpret_cast<float4*>(dst + 4) = make_float4(o[h][4][x] + o[h][4][x + 2], o[h][5][x] + o[h][5][x + 2],
                                                              o[h][6][x] + o[h][6][x + 2], o[h][7][x] + o[h][7][x + 2]);
        }
    if (l4 == 0) { m_to[hl] = st.m; l_to[hl] = l; }
}
// Joins pieces of one output run of four channels.
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
__device__ __forceinline__ void store_run(const PagesParams& p, int row, int g, int h, int c, const RunSum& s) {
    const float inv = s.L == 0.f ? 0.f : 1.f / s.L;            // a row with nothing to attend to: zeros
    const size_t hq = (size_t)row * p.Hq + (size_t)g * p.G + h;
    reinterpret_cast<uint2*>(p.out + hq * D)[c] = make_uint2(pack_bf16x2(s.acc.x * inv, s.acc.y * inv), pack_bf16x2(s.acc.z * inv, s.acc.w * inv));
    if (p.lse != nullptr && c == 0) p.lse[hq] = s.L == 0.f ? -INFINITY : (s.M + log2f(s.L)) * 0.6931471805599453f;
}

// Starts the copies of a page (slab: its K or V block's first element) to shared address dst, V behind K.
template <int D>
__device__ __forceinline__ void copy_page(const PagesParams& p, size_t slab, int nv, uint32_t dst) {
    constexpr int kChunks = D / 8;                 // 16-byte chunks of a row
    constexpr uint32_t kPageBytes = kPageTokens * D * 2;
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int k = 0; k < kPageTokens * kChunks / 32; ++k) {
        const int c = k * 32 + lane, r = c / kChunks, ch = c % kChunks;
        const uint32_t to = dst + (uint32_t)(r * (D * 2) + ((ch ^ swizzle(r)) << 4));
        // slots past the end may hold anything: K's scores are masked, V has to be zero
        copy16(to, p.k_cache + slab + c * 8, 16);
        copy16(to + kPageBytes, p.v_cache + slab + c * 8, r < nv ? 16 : 0);
    }
}

template <int D, int O>                             // O CTAs per SM
__global__ void __launch_bounds__(kPagesThreads, O) attn_decode_pages_kernel(const PagesParams p) {
    typedef PagesRing<D, O> R;
    constexpr int kSteps = D / 32;                 // 16-byte reads per lane and K row
    extern __shared__ __align__(128) uint8_t ring[];
    __shared__ PagesShared sh;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int hl = lane >> 2, l4 = lane & 3;
    const int S = p.cluster, rank = (int)(blockIdx.x % S);
    const long long item = blockIdx.x / S;
    const int row = (int)(item / p.Hkv), g = (int)(item % p.Hkv);
    pdl_launch_dependents();
    pdl_wait();
    // This warp's pages are list entries first, first + stride, ...; lane i holds the i-th of the next 32.
    const int first = rank * kPagesWarps + warp, stride = S * kPagesWarps;
    const int32_t* list = p.list + item * p.top;
    auto entry = [&](int i0) -> int {
        const long long i = first + (long long)(i0 + lane) * stride;
        return i < p.top ? fetch(list + i) : -1;
    };
    int next = entry(0);
    const int total = max(0, min(p.top, fetch(p.count + item)));
    uint4 qf[kSteps];                              // head lane / 4, channels 32 step + 8 (lane % 4) .. + 7
    {
        const uint4* src = reinterpret_cast<const uint4*>(p.q + ((size_t)row * p.Hq + (size_t)g * p.G + (hl < p.G ? hl : 0)) * D);
#pragma unroll
        for (int c = 0; c < kSteps; ++c) qf[c] = fetch(src + c * 4 + l4);
    }
    const RowSeq at = locate_row(row, p.q_offsets, p.batch);
    if (at.padding) return;                        // (the same for the whole cluster)
    const int pos = row_position(at, fetch(p.seq_lens + at.b), p.max_pages);
    if (pos < 0 && tid == 0) atomicExch(p.status, AFLEX_ERR_BOUNDS);
    const int n = pos >= 0 ? max(0, (total - first + stride - 1) / stride) : 0;        // this warp's pages
    const int32_t* table = p.page_table + (size_t)at.b * p.max_pages;
    if (hl >= p.G) {
#pragma unroll
        for (int c = 0; c < kSteps; ++c) qf[c] = make_uint4(0, 0, 0, 0);
    }
    const uint32_t base = smem_u32(ring) + (uint32_t)(warp * R::kWarpBytes);
    int phys = 0, valid = 0;
    // starts the copies of page i of this warp's into stage i % kStages
    auto issue = [&](int i) {
        if ((i & 31) == 0) {                       // look up the next 32 entries, and load the 32 after them
            phys = 0; valid = 0;
            if (i + lane < n) {
                if (next >= 0 && next <= pos / kPageTokens) {
                    phys = fetch(table + next);
                    valid = min(kPageTokens, pos - next * kPageTokens + 1);
                }
                if (valid == 0 || phys < 0 || phys >= p.num_pages) { atomicExch(p.status, AFLEX_ERR_BOUNDS); phys = 0; valid = 0; }
            }
            next = entry(i + 32);
        }
        const int nv = __shfl_sync(0xffffffffu, valid, i & 31);
        const size_t slab = ((size_t)__shfl_sync(0xffffffffu, phys, i & 31) * p.Hkv + g) * kPageTokens * D;
        const int stage = i % R::kStages;
        if (lane == 0) sh.valid[warp][stage] = nv;
        copy_page<D>(p, slab, nv, base + (uint32_t)(stage * 2 * R::kPageBytes));
    };
    PageState<D> st;
    st.reset();
#pragma unroll
    for (int i = 0; i < R::kStages - 1; ++i) {
        if (i < n) issue(i);
        copy_commit();
    }
    for (int i = 0; i < n; ++i) {
        if (i + R::kStages - 1 < n) issue(i + R::kStages - 1);
        copy_commit();
        copy_wait<R::kStages - 1>();
        __syncwarp();
        const int stage = i % R::kStages;
        const int nv = sh.valid[warp][stage];
        const uint32_t kp = base + (uint32_t)(stage * 2 * R::kPageBytes), vp = kp + R::kPageBytes;
        if (nv > 0) attend_page<D>(st, kp, vp, nv, qf, p.scale_log2);
        __syncwarp();                              // everybody has read the stage that the next copies overwrite
    }
    // ---- join the warps, then the cluster's CTAs.  Lane: head lane / 4, channels 64 h + 16 l4 + 8 x + c at o[h][c][x].
    // The copies that this warp started have all landed (a group is waited for before its page is used), so its ring is free.
    auto state = [&](int w) { return reinterpret_cast<float*>(ring + w * R::kWarpBytes); };       // [8][D]
    park_state<D>(st, state(warp), sh.m[warp], sh.l[warp]);
    __syncthreads();
    constexpr int kRuns = D / 4;                   // a head's outputs in runs of four channels
    for (int i = tid; i < p.G * kRuns; i += kPagesThreads) {
        const int h = i / kRuns, c = i % kRuns;
        RunSum s = {kLowest, 0.f, make_float4(0.f, 0.f, 0.f, 0.f)};
#pragma unroll
        for (int w = 0; w < kPagesWarps; ++w) s.M = fmaxf(s.M, sh.m[w][h]);
#pragma unroll
        for (int w = 0; w < kPagesWarps; ++w) add_piece(s, sh.m[w][h], sh.l[w][h], *reinterpret_cast<const float4*>(state(w) + h * D + 4 * c));
        if (S == 1) store_run<D>(p, row, g, h, c, s);
        else {
            *reinterpret_cast<float4*>(state(0) + h * D + 4 * c) = s.acc;      // read by nobody else in this loop
            if (c == 0) { sh.cm[h] = s.M; sh.cl[h] = s.L; }
        }
    }
    if (S == 1) return;
    // the cluster's CTAs: each makes its share of the runs, all pieces loaded before the first is used
    cluster_arrive();
    cluster_wait();
    for (int i = rank + S * tid; i < p.G * kRuns; i += S * kPagesThreads) {
        const int h = i / kRuns, c = i % kRuns;
        float pm[kPagesMaxCluster], pl[kPagesMaxCluster];
        float4 v[kPagesMaxCluster];
#pragma unroll
        for (int s = 0; s < kPagesMaxCluster; ++s) {
            const uint32_t from = (uint32_t)(s < S ? s : 0);
            pm[s] = ld_cluster_f32(cluster_map_shared(smem_u32(&sh.cm[h]), from));
            pl[s] = ld_cluster_f32(cluster_map_shared(smem_u32(&sh.cl[h]), from));
            v[s] = ld_cluster_f32x4(cluster_map_shared(smem_u32(state(0) + h * D + 4 * c), from));
        }
        RunSum sum = {kLowest, 0.f, make_float4(0.f, 0.f, 0.f, 0.f)};
#pragma unroll
        for (int s = 0; s < kPagesMaxCluster; ++s) if (s < S) sum.M = fmaxf(sum.M, pm[s]);
#pragma unroll
        for (int s = 0; s < kPagesMaxCluster; ++s) if (s < S) add_piece(sum, pm[s], pl[s], v[s]);
        store_run<D>(p, row, g, h, c, sum);
    }
    cluster_arrive();
    cluster_wait();                                // the others' shared memory stays until everybody has read it
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
typedef void (*SelectKernel)(const SelectParams);
static const SelectKernel kSelectKernels[2][5] = {
    {page_select_kernel<64, 16, 1>, page_select_kernel<64, 8, 2>, page_select_kernel<64, 4, 4>, page_select_kernel<64, 4, 6>, page_select_kernel<64, 4, 8>},
    {page_select_kernel<128, 16, 1>, page_select_kernel<128, 8, 2>, page_select_kernel<128, 4, 4>, page_select_kernel<128, 4, 6>,
     page_select_kernel<128, 4, 8>}};
static const SelectKernel kSelectRowsKernels[2][4] = {
    {page_select_rows_kernel<64, 16, 1>, page_select_rows_kernel<64, 8, 2>, page_select_rows_kernel<64, 8, 3>, page_select_rows_kernel<64, 8, 4>},
    {page_select_rows_kernel<128, 16, 1>, page_select_rows_kernel<128, 8, 2>, page_select_rows_kernel<128, 8, 3>, page_select_rows_kernel<128, 8, 4>}};

// Clusters of `cluster` CTAs that the current device holds at once.
template <typename P>
cudaError_t clusters_at_once(void (*kernel)(const P), int threads, size_t smem, int cluster, int* n) {
    cudaLaunchConfig_t lc = {};
    lc.gridDim = dim3((unsigned)cluster);
    lc.blockDim = dim3((unsigned)threads);
    lc.dynamicSmemBytes = smem;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = (unsigned)cluster;
    attr[0].val.clusterDim.y = 1;
    attr[0].val.clusterDim.z = 1;
    lc.attrs = attr;
    lc.numAttrs = 1;
    return cudaOccupancyMaxActiveClusters(n, kernel, &lc);
}

// Raises the kernels' shared-memory limits on the current device, and asks for the clusters that it holds.
static aflex_status select_attributes(aflex_ctx* ctx, int di) {
    cudaError_t e = cudaSuccess;
    for (int w = 0; w < 5 && e == cudaSuccess; ++w)
        e = cudaFuncSetAttribute(kSelectKernels[di][w], cudaFuncAttributeMaxDynamicSharedMemorySize, (kSelCap + 4) * (int)sizeof(float));
    for (int w = 0; w < 4 && e == cudaSuccess; ++w)
        e = cudaFuncSetAttribute(kSelectRowsKernels[di][w], cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kSelRowsSmem);
    for (int c = 2; c <= kSelMaxCluster && e == cudaSuccess; ++c) {
        e = clusters_at_once(kSelectRowsKernels[di][0], 512, kSelRowsSmem, c, &ctx->select_clusters[di][0][c]);
        if (e == cudaSuccess) e = clusters_at_once(kSelectRowsKernels[di][2], 256, 48 * 1024, c, &ctx->select_clusters[di][1][c]);
    }
    return check_cuda(ctx, e, "page select: kernel attributes");
}

aflex_status page_select_supported(aflex_ctx* ctx, const aflex_kv* kv) {
    if (kv->max_pages_per_seq > kSelMaxCluster * kSelCap)
        return set_error(ctx, AFLEX_ERR_UNSUPPORTED, "page select: max_pages_per_seq %d (supported: up to %d)", kv->max_pages_per_seq,
                         kSelMaxCluster * kSelCap);
    return AFLEX_OK;
}

aflex_status page_select_launch(aflex_ctx* ctx, const aflex_attn_desc* d, const void* q, const aflex_kv* kv,
                                const aflex_key_bounds* bounds, const aflex_page_policy* policy, int batch, const int32_t* q_offsets,
                                int rows, int32_t* page_list, int32_t* page_count, cudaStream_t st) {
    SelectParams p;
    p.q = (const __nv_bfloat16*)q;
    p.codes = bounds->codes; p.scales = bounds->scales;
    p.page_table = kv->page_table; p.seq_lens = kv->seq_lens; p.q_offsets = q_offsets;
    p.batch = batch; p.rows = rows; p.max_pages = kv->max_pages_per_seq;
    p.Hq = d->num_q_heads; p.Hkv = d->num_kv_heads; p.G = p.Hq / p.Hkv; p.num_pages = kv->num_pages;
    p.top = policy->top_pages; p.sink = policy->sink_pages; p.window = policy->window_pages;
    p.list = page_list; p.count = page_count; p.status = ctx->dev_status;
    const long long items = (long long)rows * p.Hkv;
    aflex_status ok = page_select_supported(ctx, kv);
    if (ok != AFLEX_OK) return ok;
    const int di = d->head_dim == 128;
    if (!ctx->select_attr_set[di]) {
        aflex_status s = select_attributes(ctx, di);
        if (s != AFLEX_OK) return s;
        ctx->select_attr_set[di] = true;
    }
    // Rows that share their sequence go in groups: as many as a sequence has (up to 8, a divisor of more), four where the
    // sequences' numbers of rows differ.  A group gets one CTA; more of them, as long as all clusters fit at once, where each
    // still has eight tiles of pages, or where the scores need the room.  Warps per CTA and CTAs per SM: the fewest of the latter (with
    // the most registers) that hold all CTAs at once; for long rows three CTAs of 8 warps where those are more warps (clusters of 3, 5,
    // 6 and 7 pay from 2048 pages: 128 groups 57 instead of 66 us at 4096, 14.1 instead of 11.2 at 512).  Alone against grouped, 32 query
    // on 8 KV heads: 16 x 5 rows of 128 / 256 / 512 pages 11.0 / 15.2 / 22.5 against 6.5 / 7.9 / 11.2 us, 32 x 4 rows 11.8 / 16.5 / 27.4
    // against 7.1 / 9.4 / 17.1, 64 x 5 rows of 64 / 256 / 1024 pages 26 / 43 / 100 against 9.6 / 21 / 60, 1 x 8 rows of 1024 / 4096 pages 9.0 /
    // 15.8 against 8.4 / 13.1.
    if (q_offsets != nullptr && rows >= 2LL * batch) {
        const int each = rows % batch == 0 ? rows / batch : 4;
        int R = each <= 8 ? each : 4;
        for (int r = 8; r >= 2 && each > 8; --r) if (each % r == 0) { R = r; break; }
        const long long groups = ((long long)rows + R - 1) / R * p.Hkv;
        const int per = 8 / p.G, sets = (R + per - 1) / per;
        p.group = R;
        p.stride = (p.max_pages + 3) / 4 * 4;
        auto smem_of = [&](int C) -> size_t {
            return (size_t)sets * (d->head_dim / 32) * (32 * sizeof(uint4) + 8 * sizeof(float)) + (size_t)((R + C - 1) / C) * p.stride * sizeof(float);
        };
        int C = 1, form = 0;
        while (C < kSelMaxCluster && ((groups <= ctx->select_clusters[di][0][2 * C] && p.max_pages >= 2 * C * 8 * kSelTile) || smem_of(C) > kSelRowsSmem)) C *= 2;
        if (C == 1 && groups > ctx->num_sms) form = groups <= 2 * ctx->num_sms ? 1 : groups <= 3 * ctx->num_sms ? 2 : 3;
        if (p.max_pages >= 32 * kSelTile) {                         // three CTAs of 8 warps per SM where those are more warps
            int more = 1;
            for (int c = 2; c <= kSelMaxCluster; c = p.max_pages >= 128 * kSelTile ? c + 1 : 2 * c) if (groups <= ctx->select_clusters[di][1][c]) more = c;
            if (more > 1 && more * 8 > C * (form ? 8 : 16)) { C = more; form = 2; }
        }
        // (few groups of short rows: a CTA per row and head is quicker)
        if (smem_of(C) <= kSelRowsSmem && (groups * 3 >= ctx->num_sms || p.max_pages >= 16 * kSelTile)) {
            if (groups * C > 0x7fffffffLL) return set_error(ctx, AFLEX_ERR_UNSUPPORTED, "page select: rows * Hkv = %lld", items);
            const int W = form == 0 ? 16 : 8, slots = (R + C - 1) / C, most = p.max_pages >= 16 * kSelTile ? W : 4;
            p.cluster = C;
            p.row_warps = 0;
            while ((2 << p.row_warps) <= most && (slots << (p.row_warps + 1)) <= W) ++p.row_warps;
            KernelScope scope(ctx, kKPageSelect, st);
            return check_cuda(ctx, launch_cluster(kSelectRowsKernels[di][form], groups * C, W * 32, smem_of(C), C, st, p), "page_select_rows_kernel launch");
        }
    }
    // A cluster per (row, KV head) where those are fewer than the SMs (and where the scores need the room), each CTA at least
    // eight tiles.  16 warps per CTA while an SM has no second one, 8 while two per SM hold all of them, else 4 (more CTAs at
    // once, and a selection that fewer warps have to agree on) and as many CTAs per SM as hold all of them, with the registers that are
    // left.  8 x 8192 pages: 34.0 / 22.6 / 11.5 us with 1 / 2 / 8 CTAs of 16 warps, 13.4 with 8 of 8; 192 x 256 pages: 6.0 and 7.8 us
    // with 8 and 4 warps, 320 x 256: 10.8 and 8.5; 4 warps with 4 / 6 / 8 CTAs per SM: 512 x 256 pages 10.6 / 12.4 / 17.5, 640 x 256 17.1 /
    // 13.4 / 18.0, 1024 x 64 10.7 / 9.6 / 7.8, 2560 x 64 28.9 / 19.5 / 21.4, 2560 x 256 50 / 42.5 / 50.
    int S = 1;
    while (S < kSelMaxCluster && (items * S < ctx->num_sms || p.max_pages > (long long)S * kSelCap) && p.max_pages > S * 8 * kSelTile) S *= 2;
    const long long per_sm = (items * S + ctx->num_sms - 1) / ctx->num_sms;
    const int form = per_sm <= 1 ? 0 : per_sm <= 2 ? 1 : per_sm <= 4 ? 2 : per_sm > 6 && per_sm <= 8 ? 4 : 3;
    const int share = ((p.max_pages + kSelTile - 1) / kSelTile + S - 1) / S * kSelTile;       // candidates per CTA at most
    if (items * S > 0x7fffffffLL) return set_error(ctx, AFLEX_ERR_UNSUPPORTED, "page select: rows * Hkv = %lld", items);
    p.cluster = S;
    const size_t smem = (size_t)(share + 4) * sizeof(float);
    KernelScope scope(ctx, kKPageSelect, st);
    return check_cuda(ctx, launch_cluster(kSelectKernels[di][form], items * S, form == 0 ? 512 : form == 1 ? 256 : 128, smem, S, st, p), "page_select_kernel launch");
}

aflex_status attn_decode_pages_launch(aflex_ctx* ctx, const aflex_attn_desc* d, const void* q, const aflex_kv* kv,
                                      const int32_t* page_list, const int32_t* page_count, int top_pages, int batch,
                                      const int32_t* q_offsets, int rows, void* out, float* lse, cudaStream_t st) {
    PagesParams p;
    p.q = (const __nv_bfloat16*)q;
    p.k_cache = (const __nv_bfloat16*)kv->k_cache; p.v_cache = (const __nv_bfloat16*)kv->v_cache;
    p.page_table = kv->page_table; p.seq_lens = kv->seq_lens; p.q_offsets = q_offsets;
    p.list = page_list; p.count = page_count;
    p.batch = batch; p.rows = rows; p.max_pages = kv->max_pages_per_seq;
    p.Hq = d->num_q_heads; p.Hkv = d->num_kv_heads; p.G = p.Hq / p.Hkv; p.top = top_pages; p.num_pages = kv->num_pages;
    const float scale = d->sm_scale != 0.f ? d->sm_scale : 1.0f / sqrtf((float)d->head_dim);
    p.scale_log2 = scale * 1.4426950408889634f;
    p.out = (__nv_bfloat16*)out; p.lse = lse; p.status = ctx->dev_status;
    const long long items = (long long)rows * p.Hkv;
    const bool wide = d->head_dim == 128;
    typedef void (*Kernel)(const PagesParams);
    const Kernel kernels[2] = {wide ? attn_decode_pages_kernel<128, 2> : attn_decode_pages_kernel<64, 3>,
                               wide ? attn_decode_pages_kernel<128, 3> : attn_decode_pages_kernel<64, 4>};
    const int smem[2] = {wide ? PagesRing<128, 2>::kBytes : PagesRing<64, 3>::kBytes, wide ? PagesRing<128, 3>::kBytes : PagesRing<64, 4>::kBytes};
    int* fit = ctx->pages_clusters[wide];          // clusters of 2, 3 .. 8 CTAs that the GPU holds at once
    if (!ctx->pages_attr_set[wide]) {
        cudaError_t e = cudaSuccess;
        for (int f = 0; f < 2 && e == cudaSuccess; ++f) e = cudaFuncSetAttribute(kernels[f], cudaFuncAttributeMaxDynamicSharedMemorySize, smem[f]);
        for (int s = 2; s <= kPagesMaxCluster && e == cudaSuccess; ++s) e = clusters_at_once(kernels[0], kPagesThreads, smem[0], s, &fit[s]);
        if (e != cudaSuccess) return check_cuda(ctx, e, "attention over pages: kernel attributes");
        ctx->pages_attr_set[wide] = true;
    }
    // CTAs per (row, KV head): as many as the GPU holds at once as clusters (fewer than the places that its SMs have, since a
    // cluster stays inside one group of them), down to one page per warp.  A CTA costs about 5 us beside its pages (three
    // dependent loads before the first page, the join), so a second wave costs more than an even split gains: 8 pairs of 128
    // pages 23.8 / 15.1 / 9.9 / 7.2 us with 1 / 2 / 4 / 8 CTAs each; 80 pairs 29.4 / 19.9 / 19.6 / 26.9 with 1 / 2 / 3 / 4; 256 of
    // up to 64 pages 26 / 32 / 43 with 1 / 2 / 4.  (Equal shares of all pairs' pages, cut anywhere and joined through global
    // memory: 60 against 57 us at 304 pairs of 128, 52 against 47 at 256, 93 against 84 at 512.)
    const int most = (top_pages + kPagesWarps - 1) / kPagesWarps;
    int S = 1;
    for (int s = 2; s <= kPagesMaxCluster && s <= most; ++s) if (items <= fit[s]) S = s;
    if (items * S > 0x7fffffffLL) return set_error(ctx, AFLEX_ERR_UNSUPPORTED, "attention over pages: rows * Hkv = %lld", items);
    p.cluster = S;
    // One CTA more per SM, with less of a ring, where an SM then takes no more turns x CTAs: 320 / 384 / 440 / 640 pairs of 128 pages 69.4 /
    // 71.7 / 73.8 / 111 us with two and 59.3 / 68.4 / 75.3 / 106 with three, but 296 pairs 52.4 and 56.1, 512 pairs 84 and 102; heads of 64,
    // 512 / 1024 pairs 55 / 88 with three and 44 / 83 with four.
    const long long deep = wide ? 2 : 3, places = deep * ctx->num_sms, more = (deep + 1) * ctx->num_sms;
    const int form = S == 1 && items > places && (items + more - 1) / more * (deep + 1) <= (items + places - 1) / places * deep;
    KernelScope scope(ctx, kKAttnPages, st);
    return check_cuda(ctx, launch_cluster(kernels[form], items * S, kPagesThreads, smem[form], S, st, p), "attn_decode_pages_kernel launch");
}

}  // namespace aflex
