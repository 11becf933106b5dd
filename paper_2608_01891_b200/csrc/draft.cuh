// Work of the attention kernels for drafted tokens (attn_draft.cu): the list of units and its equal shares.
//
// A tile is a run of up to `rpt` rows of one sequence; its lines are the rows' queries of one KV head's group.  An item is a tile and a
// KV head; it has one unit of kTokens cached tokens after another, up to the last token that a row of the tile may see, and one empty
// unit in front (what starting and joining an item costs).  In the kernel whose tiles are 256 lines, a unit of more than 128 lines takes two places.
// All items' units in a list, cut anywhere into equal shares, a share per CTA:
// no plan on the host, which does not know the lengths, and no CTA that is left with a long sequence.
#pragma once
#include <cuda_fp16.h>
#include <math.h>
#include <stdint.h>

#include "internal.h"
#include "ptx.cuh"
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
    float scale_log2, unit;        // unit: what the sums of weights times codes count (2^16 of an 8-bit cache)
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

template <int kTokens, int kFull> struct DraftList {        // kFull: places of a full tile's unit
    static constexpr int kShift = kTokens == 128 ? 7 : 6;
    static_assert(kTokens == 1 << kShift, "");
    int rpt_shift, g_shift;
    bool causal;
    __device__ DraftList(const DraftParams& p) : rpt_shift(p.rpt_shift), g_shift(p.g_shift), causal(p.mask == nullptr) {}
    __device__ int tiles(const DraftSeq& s) const { return (s.m + (1 << rpt_shift) - 1) >> rpt_shift; }
    // tokens that the rows of a tile may see, units of one of its items, places of a unit, places of the item (the empty one among them)
    __device__ int sees(const DraftSeq& s, int tile) const {
        return !s.ok ? 0 : causal ? s.ctx + (int)min((long long)s.m, (long long)(tile + 1) << rpt_shift) : s.len;
    }
    __device__ int units(const DraftSeq& s, int tile) const { return (sees(s, tile) + kTokens - 1) >> kShift; }
    __device__ int weight(const DraftSeq& s, int tile) const {
        return kFull == 1 || (min(1 << rpt_shift, s.m - (tile << rpt_shift)) << g_shift) <= 128 ? 1 : kFull;
    }
    __device__ int places(const DraftSeq& s, int tile) const { return 1 + weight(s, tile) * units(s, tile); }
    // sum over i = 1 .. x of ceil(i / q), q = tiles whose rows make a unit of tokens (a power of two); of k i where a tile's rows are k units
    __device__ long long ramp(long long x) const {
        const int qs = kShift - rpt_shift;
        if (qs < 0) return (x * (x + 1) / 2) << -qs;
        const long long y = x >> qs, z = x - (y << qs);
        return ((y * (y + 1)) << qs >> 1) + z * (y + 1);
    }
    // places of the sequence's first `n` tiles, for one KV head; all but a sequence's last tile are full, and with a = ceil(ctx / rows per tile)
    // a full tile t's tokens are ceil((a + t + 1) / q) units
    __device__ long long before(const DraftSeq& s, int n) const {
        if (n == 0) return 0;
        const int full = min(n, tiles(s) - 1);
        long long sum = 0;
        if (full > 0) {
            const long long a = (s.ctx + (1 << rpt_shift) - 1) >> rpt_shift;
            if (!s.ok) sum = 0;
            else if (!causal) sum = (long long)full * units(s, 0);
            else if (rpt_shift > kShift) sum = (long long)full * ((s.ctx + kTokens - 1) >> kShift) + ramp(full);
            else sum = ramp(a + full) - ramp(a);
        }
        return full + kFull * sum + (n > full ? places(s, n - 1) : 0);
    }
};

// Quotients of whole numbers >= 0, which seldom need 64 bits.
__device__ __forceinline__ long long draft_div(long long a, long long b) {
    return (unsigned long long)(a | b) >> 32 ? a / b : (long long)((uint32_t)a / (uint32_t)b);
}

// A place in the list: place u of the item (tile of sequence b, KV head g), of nu; position `pos` of all.
template <int kTokens, int kFull> struct DraftWalk {
    typedef DraftList<kTokens, kFull> List;
    long long pos;
    int b, tile, g, u, nu, id;     // id: number of the tile's first item
    DraftSeq s;
    __device__ void start(const DraftParams& p, const List& list, long long x, int seq, long long seq_first, int seq_tiles) {
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
        nu = list.places(s, tile);
        const long long in = rel - list.before(s, tile) * p.Hkv;
        g = (int)draft_div(in, nu);
        u = (int)(in - (long long)g * nu);
    }
    // n places on, inside the item or to the start of the next one; `end`: the list's length
    __device__ void advance(const DraftParams& p, const List& list, int n, long long end) {
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
        nu = list.places(s, tile);
    }
    __device__ int until(long long x1) const { return (int)min((long long)nu, u + (x1 - pos)); }      // the item's places before x1
};

// A piece: a run of units of one item.  A unit belongs to the CTA that has its first place.
struct DraftPiece {
    int units, t0, sees, ctx;      // units with tokens, or 1 for an item without (t0 < 0); first token, tokens the tile's rows may see, earlier tokens
    int row0, lines, i0, m, g;     // first row and lines of the tile, number of the first row and of all rows in the sequence, KV head
    int item, slot, whole, b;      // b: the sequence
    long long first, last;         // positions of the item's first and last unit with tokens
};
// The piece that starts at w (not at the empty place of an item that has tokens) and ends with the item or at x1; no units: nothing to do.
template <int kTokens, int kFull>
__device__ __forceinline__ DraftPiece draft_piece(const DraftParams& p, const DraftList<kTokens, kFull>& list, const DraftWalk<kTokens, kFull>& w, long long x1) {
    DraftPiece d;
    const int wt = list.weight(w.s, w.tile), all = list.units(w.s, w.tile);
    const int k0 = w.u == 0 ? -1 : (w.u - 1 + wt - 1) / wt, k1 = w.u == 0 ? 0 : (w.until(x1) - 1 + wt - 1) / wt;
    d.units = k1 - k0; d.t0 = k0 * kTokens;
    d.sees = list.sees(w.s, w.tile); d.ctx = w.s.ctx;
    d.i0 = w.tile << p.rpt_shift; d.row0 = w.s.o0 + d.i0; d.m = w.s.m; d.g = w.g;
    d.lines = min(1 << p.rpt_shift, w.s.m - d.i0) << p.g_shift;
    d.b = w.b; d.item = w.id + w.g; d.slot = k0 > 0 ? 0 : 1; d.whole = k0 <= 0 && k1 == all;
    d.first = w.pos - w.u + 1; d.last = d.first + (long long)wt * (all - 1);
    return d;
}

// Whether drafted token j (negative: an earlier token) is seen by row i of its sequence.
__device__ __forceinline__ bool sees_drafted(const DraftParams& p, int row, int i, int j, int m) {
    if (j < 0) return true;
    if (j >= m) return false;
    if (p.mask == nullptr) return j <= i;
    return (j >> 5) < p.mask_words && ((fetch(p.mask + (size_t)row * p.mask_words + (j >> 5)) >> (j & 31)) & 1u);
}

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
template <int kThreads, int kTokens, int kFull>
__device__ __forceinline__ void draft_plan(const DraftParams& p, const DraftList<kTokens, kFull>& list, DraftShare& out) {
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
    share.ctas = (int)min((long long)gridDim.x, max(total / kFull, min(total, 1LL)));       // (at least a unit's places each)
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

// Weights are 2^(x - m): m is the running maximum less kBelow, and moves when a weight would pass 2^(kBelow + 7).  In fp16 (8-bit caches) weights
// from 2^8 to 2^15 leave the most room below; bf16 has room enough anywhere, and weights from 2^-8 to 2^-1 keep the sums of weights times values
// finite where those of a softmax in 32 bits are.
template <int F> constexpr float kBelow = F == AFLEX_CACHE_BF16 ? -8.f : 8.f;

// Of an 8-bit cache x is the score plus lv = log2 of the token's V scale less 16 (at least -80: a scale of 0, or of a value of zeros), so that 2^(x - m) is
// what its codes count and 2^(x - m - lv) what the token counts in the sum L of all weights: by its score alone, whatever its value's size.  The 16
// leave L room below where V's scales are near 2^121 (terms of 2^-97) and above where they are the least (2^95); sums of codes are multiplied by 2^16 at the end.
constexpr float kScaleShift = 16.f, kLeastScale = -64.f - kScaleShift;
__device__ __forceinline__ float log2_scale(float scale) {
    const float lv = __log2f(scale) - kScaleShift;
    return lv < kLeastScale ? kLeastScale : lv;    // (NaN stays)
}
// l * 2^d where 2^d alone could be 0 and the product not: of pieces whose V's scales are far apart
__device__ __forceinline__ float scale_sum(float l, float d) {
    const float c = fmaxf(d, -100.f);
    return l * fast_exp2(c) * fast_exp2(d - c);
}

// Sums of one run of four channels of a line over pieces.
struct RunSum {
    float M, L;
    float4 acc;
};
__device__ __forceinline__ void add_piece(RunSum& s, float m, float l, const float4& v) {
    const float f = fast_exp2(m - s.M);            // (s.M: the largest m of all pieces)
    s.L += scale_sum(l, m - s.M);
    s.acc.x = fmaf(v.x, f, s.acc.x); s.acc.y = fmaf(v.y, f, s.acc.y); s.acc.z = fmaf(v.z, f, s.acc.z); s.acc.w = fmaf(v.w, f, s.acc.w);
}
template <int D>
__device__ __forceinline__ void store_run(const DraftParams& p, const DraftPiece& u, int line, int c, const RunSum& s) {
    const float inv = s.L == 0.f ? 0.f : __frcp_rn(s.L) * p.unit;      // a line with nothing to attend to: zeros
    const size_t hq = (size_t)(u.row0 + (line >> p.g_shift)) * p.Hq + (size_t)u.g * p.G + (line & (p.G - 1));
    reinterpret_cast<uint2*>(p.out + hq * D)[c] = make_uint2(pack_bf16x2(s.acc.x * inv, s.acc.y * inv), pack_bf16x2(s.acc.z * inv, s.acc.w * inv));
    if (p.lse != nullptr && c == 0) p.lse[hq] = s.L == 0.f ? -INFINITY : (s.M + __log2f(s.L)) * 0.6931471805599453f;
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

// Whether one of four e4m3 codes is a NaN (0x7f or 0xff); of two bf16 values whether one is an infinity or NaN.
__device__ __forceinline__ bool odd_e4m3(uint32_t w) { return (((w & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u) != 0; }
__device__ __forceinline__ bool odd_bf16(uint32_t w) { return (w & 0x7f80u) == 0x7f80u || (w & 0x7f800000u) == 0x7f800000u; }

// 16 bytes of scales (the L2 cache is told to fetch the neighbouring heads' with them), and one arrival when this thread's copies so far have landed.
__device__ __forceinline__ void copy16(uint32_t dst, const void* src) {
    asm volatile("cp.async.cg.shared.global.L2::256B [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void copies_arrive(uint64_t* bar) {
    asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(smem_u32(bar)) : "memory");
}

}  // namespace aflex
