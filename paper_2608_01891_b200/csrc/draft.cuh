// Work of the attention kernels for drafted tokens (attn_draft.cu): the list of units and its equal shares.
//
// A tile is a run of up to `rpt` rows of one sequence; its lines are the rows' queries of one KV head's group.  An item is a tile and a
// KV head; it has one unit of kTokens cached tokens after another, up to the last token that a row of the tile may see, and one empty
// unit in front (what starting and joining an item costs).  All items' units in a list, cut anywhere into equal shares, a share per CTA:
// no plan on the host, which does not know the lengths, and no CTA that is left with a long sequence.
#pragma once
#include <stdint.h>

#include "internal.h"
#include "rows.cuh"

namespace aflex {

struct DraftParams {
    const __nv_bfloat16* q;        // [rows][Hq][D]
    const float* k_scales;         // [pages][Hkv][16], null for bf16
    const float* v_scales;
    const int32_t* page_table;
    const int32_t* seq_lens;
    const int32_t* q_offsets;      // null: one row per sequence
    const uint32_t* mask;          // [rows][mask_words] or null
    int mask_words, batch, rows, max_pages, Hq, Hkv, G, g_shift, rpt_shift;      // G = 2^g_shift; rows per tile: 2^rpt_shift
    long long num_pages;
    float scale_log2;
    __nv_bfloat16* out;
    float* lse;
    float* parts;                  // [CTA][2][slot]: of an item's piece, [lines][2] reference of the weights (log2 units) and their sum, then
                                   // [lines][D] unnormalised sums
    int* counters;                 // [items] pieces done, zero on entry and on exit
    int* status;
};

// Rows of a sequence.  m = 0: none, or offsets that cannot be followed.  ok: false if its length does not go with them: its rows see nothing.
struct DraftSeq {
    int o0, m, len, ctx;
    bool ok, bad;
};
__device__ __forceinline__ DraftSeq draft_seq(const DraftParams& p, int b) {
    DraftSeq s;
    s.o0 = p.q_offsets ? fetch(p.q_offsets + b) : b;
    const long long m = p.q_offsets ? (long long)fetch(p.q_offsets + b + 1) - s.o0 : 1;
    s.len = fetch(p.seq_lens + b);
    s.bad = m < 0 || s.o0 < 0 || s.o0 + m > p.rows;
    s.m = s.bad ? 0 : (int)m;
    s.ok = s.len >= 1 && s.len >= s.m && s.len <= (long long)p.max_pages * kPageTokens;
    s.bad = s.bad || (s.m > 0 && !s.ok);
    if (!s.ok) s.len = 0;
    s.ctx = s.ok ? s.len - s.m : 0;
    return s;
}

template <int kTokens> struct DraftList {
    static constexpr int kShift = kTokens == 128 ? 7 : 6;
    static_assert(kTokens == 1 << kShift, "");
    int rpt_shift;
    bool causal;
    __device__ DraftList(const DraftParams& p) : rpt_shift(p.rpt_shift), causal(p.mask == nullptr) {}
    __device__ int tiles(const DraftSeq& s) const { return (s.m + (1 << rpt_shift) - 1) >> rpt_shift; }
    // tokens that the rows of a tile may see, units of one of its items (the empty one among them)
    __device__ int sees(const DraftSeq& s, int tile) const {
        return !s.ok ? 0 : causal ? s.ctx + (int)min((long long)s.m, (long long)(tile + 1) << rpt_shift) : s.len;
    }
    __device__ int units(const DraftSeq& s, int tile) const { return 1 + ((sees(s, tile) + kTokens - 1) >> kShift); }
    // sum over i = 1 .. x of ceil(i / q), q = tiles whose rows make a unit of tokens (a power of two)
    __device__ long long ramp(long long x) const {
        const int qs = kShift - rpt_shift;
        const long long y = x >> qs, z = x - (y << qs);
        return ((y * (y + 1)) << qs >> 1) + z * (y + 1);
    }
    // units of the sequence's first `n` tiles, for one KV head; all but a sequence's last tile are full, and with a = ceil(ctx / rows per tile)
    // a full tile t's tokens are ceil((a + t + 1) / q) units
    __device__ long long before(const DraftSeq& s, int n) const {
        if (n == 0) return 0;
        if (!causal || !s.ok || n == 1) return (long long)n * units(s, 0);
        const int full = min(n, tiles(s) - 1);
        const long long a = (s.ctx + (1 << rpt_shift) - 1) >> rpt_shift;
        return ramp(a + full) - ramp(a) + full + (n > full ? units(s, n - 1) : 0);
    }
};

// Quotients of whole numbers >= 0, which seldom need 64 bits.
__device__ __forceinline__ long long draft_div(long long a, long long b) {
    return (unsigned long long)(a | b) >> 32 ? a / b : (long long)((uint32_t)a / (uint32_t)b);
}

// A place in the list: unit u of the item (tile of sequence b, KV head g); position `pos` of all.
template <int kTokens> struct DraftWalk {
    long long pos;
    int b, tile, g, u, nu, id;     // id: number of the tile's first item
    DraftSeq s;
    __device__ void start(const DraftParams& p, const DraftList<kTokens>& list, long long x, int seq, long long seq_first, int seq_tiles) {
        pos = x; b = seq;
        s = draft_seq(p, b);
        const long long rel = x - seq_first;
        int lo = 0, hi = list.tiles(s) - 1;        // the last tile that starts at rel or before
        while (lo < hi) {
            const int mid = (lo + hi + 1) / 2;
            if (list.before(s, mid) * p.Hkv <= rel) lo = mid; else hi = mid - 1;
        }
        tile = lo;
        id = (seq_tiles + tile) * p.Hkv;
        nu = list.units(s, tile);
        const long long in = rel - list.before(s, tile) * p.Hkv;
        g = (int)draft_div(in, nu);
        u = (int)(in - (long long)g * nu);
    }
    // n units on, inside the item or to the start of the next one; `end`: the list's length
    __device__ void advance(const DraftParams& p, const DraftList<kTokens>& list, int n, long long end) {
        pos += n; u += n;
        if (u < nu || pos >= end) return;
        u = 0;
        if (++g < p.Hkv) return;
        g = 0;
        id += p.Hkv;
        if (++tile == list.tiles(s)) {
            tile = 0;
            do s = draft_seq(p, ++b); while (s.m == 0);      // (there is another, or pos would be the end)
        }
        nu = list.units(s, tile);
    }
};

// What a CTA finds out about the list before it starts: its share [x0, x1), and where x0 is.  The first `more` CTAs have each + 1 units,
// the others `each`.
struct DraftShare {
    long long total, each, x0, x1, seq_first;
    int more, ctas, seq, seq_tiles;
    __device__ long long begin(int c) const { return each * c + min(c, more); }
    __device__ int cta_of(long long x) const {
        const long long first = (each + 1) * more;
        return (int)(x < first ? draft_div(x, each + 1) : more + draft_div(x - first, each));
    }
};
// All kThreads threads of the CTA, thread t a run of sequences; returns after a barrier.
template <int kTokens, int kThreads>
__device__ __forceinline__ void draft_plan(const DraftParams& p, const DraftList<kTokens>& list, DraftShare& out) {
    __shared__ long long s_units[kThreads / 32];
    __shared__ int s_tiles[kThreads / 32];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int per = (p.batch + kThreads - 1) / kThreads;
    const int lo = min(p.batch, tid * per), hi = min(p.batch, lo + per);
    long long units = 0;
    int tiles = 0;
    for (int b = lo; b < hi; ++b) {
        const DraftSeq s = draft_seq(p, b);
        if (s.bad && blockIdx.x == 0) atomicExch(p.status, AFLEX_ERR_BOUNDS);
        const int n = list.tiles(s);
        tiles += n;
        units += list.before(s, n);
    }
    long long u_incl = units;
    int t_incl = tiles;
#pragma unroll
    for (int off = 1; off < 32; off <<= 1) {
        const long long u = __shfl_up_sync(0xffffffffu, u_incl, off);
        const int t = __shfl_up_sync(0xffffffffu, t_incl, off);
        if (lane >= off) { u_incl += u; t_incl += t; }
    }
    if (lane == 31) { s_units[warp] = u_incl; s_tiles[warp] = t_incl; }
    __syncthreads();
    long long u_before = u_incl - units, total = 0;
    int t_before = t_incl - tiles;
    for (int w = 0; w < kThreads / 32; ++w) {
        if (w < warp) { u_before += s_units[w]; t_before += s_tiles[w]; }
        total += s_units[w];
    }
    total *= p.Hkv;
    DraftShare share;
    share.total = total;
    share.ctas = (int)min((long long)gridDim.x, total);
    share.each = share.ctas > 0 ? draft_div(total, share.ctas) : 0;
    share.more = share.ctas > 0 ? (int)(total - share.each * share.ctas) : 0;
    const bool works = (int)blockIdx.x < share.ctas;
    const long long x0 = works ? share.begin(blockIdx.x) : 0;
    if (tid == 0) {
        out.total = total; out.each = share.each; out.more = share.more; out.ctas = share.ctas;
        out.x0 = x0;
        out.x1 = works ? share.begin(blockIdx.x + 1) : 0;
    }
    u_before *= p.Hkv;
    if (x0 >= u_before && x0 < u_before + units * p.Hkv) {
        for (int b = lo; b < hi; ++b) {
            const DraftSeq s = draft_seq(p, b);
            const int n = list.tiles(s);
            const long long here = list.before(s, n) * p.Hkv;
            if (x0 < u_before + here) { out.seq = b; out.seq_first = u_before; out.seq_tiles = t_before; break; }
            u_before += here;
            t_before += n;
        }
    }
    __syncthreads();
}

}  // namespace aflex
