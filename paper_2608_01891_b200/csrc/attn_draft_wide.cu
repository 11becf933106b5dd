// Attention of drafted tokens over a paged cache in bf16 or in 8 bits, for sequences with more lines (rows x query heads of a KV head's
// group) than attn_draft.cu is for: a page's K and V serve up to 256 lines, and the products run on the tcgen05 tensor cores.
//
//   work        as in attn_draft.cu: equal shares of the list of units, one CTA per SM, pieces joined by the CTA that is last
//   tiles       two S / P and two O accumulators in TMEM.  An item of more than 128 lines has two tiles of 128, both at every step of 128 cached
//               tokens; one of up to 128 has its one tile in both places, one for the even and one for the odd steps, so that one's softmax runs
//               under the other's products either way
//   data path   a producer warp brings pages; of an 8-bit cache they are widened to fp16 by a warp group of its own, exactly (the scales are the
//               softmax's business), into the swizzled layout that the tensor cores read; a bf16 cache's pages are copied into that layout by TMA
//               and the warp group only looks at the V of drafted tokens.  K is a K-major operand, V (as stored) an MN-major one
//   softmax     eight warps per place, sixteen lines each, read from TMEM as fragments (two lines x 32 tokens per thread), so that a token's
//               scales, which every line needs, are loaded once for two lines and by four lanes at a time (with a line per thread the loads of scales alone
//               took longer than the products); 64 tokens at a time, since all 128 did not fit the registers (329 against 267 us when it was made so); statistics,
//               references and weights as in attn_draft.cu.  The weights of an 8-bit cache are stored back over the scores they came from, in
//               fp16; those of a bf16 cache as two bf16 parts, which fill the place of the scores, and the second product is issued for each part
//
// Bound: neither the products (1024 cycles per 128 lines x 128 tokens, 1536 with two parts of weights) nor the exponentials (16 per cycle: 1024)
// but the chain from a place's scores to its weights and back, some 3400 cycles per 128 x 128 with two places under way.  (attn_prefill.cu is
// twice as fast with the same two places: its softmax has a line per thread and 216 registers, where 24 warps here have 80 each and spill 44 - 100 bytes
// a thread.)  8 trees of up to 61 tokens, 64 / 8 heads of 128, over up to 16384 tokens (120 GFLOP): 256 us in int8 (0.47 PFLOP/s), 237 in e4m3, 249
// in bf16; of up to 5 tokens 83 us (2.0 TB/s of int8, 3.9 of bf16).
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <math.h>

#include <type_traits>

#include "draft.cuh"
#include "internal.h"
#include "ptx.cuh"
#include "rows.cuh"

namespace aflex {

namespace {

constexpr int kBM = 128;                           // lines per tile
constexpr int kBN = 128;                           // cached tokens per step
constexpr int kUnitPages = kBN / kPageTokens;
constexpr int kWideLines = 2 * kBM;
constexpr int kSoftmaxWarps = 16;                  // [place][sixteen lines]
constexpr int kWideThreads = (kSoftmaxWarps + 8) * 32;       // and producer, issuer (and two idle), four that widen: 80 registers a thread
constexpr int kPieceRing = 4;

template <int D, int F> struct WideForm {
    static constexpr bool kWidens = F != AFLEX_CACHE_BF16;
    static constexpr int kHalves = D / 64;
    static constexpr int kHalf = kBN * 128;                           // 128 rows of 128 bytes: 64 channels of a tile of lines or of tokens
    static constexpr int kTile = kHalves * kHalf;                     // Q of a place, K or V of a step
    // bf16: a ring of K(0) V(0) K(1) V(1) ..  8 bits: two slots for K and one for V, widened in the order K(0) K(1) V(0) K(2) V(1) ..: the products
    // with K(t + 2) follow those with V(t), whose slot it must not wait for (one ring of three: 486 against 465 us, 64 trees of 5; 261 against 251, 8 of up to 61); V(t + 1) has the
    // softmax's time
    static constexpr int kSlots = kWidens ? 3 : 4;
    static constexpr int kRaws = kWidens ? 3 : 0;                     // ring of the same in 8 bits, in the same order
    static constexpr int kRawTile = kBN * D;
    static constexpr int kRaw = kRawTile + 2 * kBN * 4;               // and with K the scales of K and V
    static constexpr int kSmem = 2 * kTile + kSlots * kTile + kRaws * kRaw;
};

struct __align__(16) WideShared {
    float4 scale[4][kBN / 2];                      // by step: of two tokens, K's scales and lv of V's (log2_scale)
    float4 inv[4][kBN / 4];                        // 2^-lv, of four tokens
    float2 state[2][kBM];                          // by place: references and sums of a finished piece
    float factor[2][kBM];                          // by place: what a line's products count, in log2 units
    uint32_t bad[4][kBN / 32];                     // by step: tokens whose V holds an infinity or NaN (bf16)
    uint64_t told[kPieceRing], left[kPieceRing];   // a piece's description is there, everybody has read it
    uint64_t raw_full[4], raw_empty[3];            // pages have landed (bf16: in their slot), have been widened
    uint64_t full[4], empty[4];                    // a slot can be read by the products, has been
    uint64_t scaled[4];                            // by step: the scales are there
    uint64_t q_ready[2], s_ready[2], p_ready[2], pv_done[2], meet, spent;       // meet: the softmax warps; spent: after a wait that ran out, the products issued before
    DraftPiece piece[kPieceRing];
    DraftShare share;
    DraftPiece merge[2];
    int merges, tiles;             // tiles: K and V tiles that the producer brought
    uint32_t tmem_base;
    int far;                       // the first step with a token whose lv is above kNear
    int odd[kPieceRing];           // e4m3: number (from 1) of the last piece there with a NaN in V of a drafted token
    volatile int abort;
};

__device__ __forceinline__ float max3(float a, float b, float c) {
    float d;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
    return d;
}

// The largest lv up to which a token's part of the sum of weights may be formed as weight * 2^-lv: a weight that is lost (below 2^-126) is then one of
// less than 2^(-134 + kNear + 80) of the sum.  Behind a token with a larger one it takes an exponential of its own.
constexpr float kNear = 10.f;

// Two weights of a line as operand: fp16, or the two bf16 parts.
template <int F> __device__ __forceinline__ void pack_weights(float w0, float w1, uint32_t& hi, uint32_t& lo) {
    if (F == AFLEX_CACHE_BF16) {
        hi = pack_bf16x2(w0, w1);
        lo = pack_bf16x2(w0 - __uint_as_float(hi << 16), w1 - __uint_as_float(hi & 0xffff0000u));
    } else {
        const __half2 f = __floats2half2_rn(w0, w1);
        hi = *reinterpret_cast<const uint32_t*>(&f);
    }
}

template <int F> __device__ __forceinline__ uint32_t wide_idesc(uint32_t n) {
    const uint32_t d = umma_idesc_bf16(kBM, n);
    return F == AFLEX_CACHE_BF16 ? d : d & ~((1u << 7) | (1u << 10));                     // fp16 operands
}

// TMEM fragments: 16 lines x 32 columns (element 4 i + 2 y + e: line lane / 4 + 8 y, column 8 i + 2 (lane % 4) + e), and of 16 lines x 32 packed
// columns (element 2 i + y: line lane / 4 + 8 y, column 4 i + lane % 4): a pair of the one packed is an element of the other.
#define R4(a, i) "=r"(a[i]), "=r"(a[i + 1]), "=r"(a[i + 2]), "=r"(a[i + 3])
#define R16(a, i) R4(a, i), R4(a, i + 4), R4(a, i + 8), R4(a, i + 12)
#define I4(a, i) "r"(a[i]), "r"(a[i + 1]), "r"(a[i + 2]), "r"(a[i + 3])
#define I16(a, i) I4(a, i), I4(a, i + 4), I4(a, i + 8), I4(a, i + 12)
__device__ __forceinline__ void tmem_ld_16x256b_x4(uint32_t taddr, uint32_t (&r)[16]) {
    asm volatile("tcgen05.ld.sync.aligned.16x256b.x4.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];" : R16(r, 0) : "r"(taddr) : "memory");
}
__device__ __forceinline__ void tmem_st_16x256b_x4(uint32_t taddr, const uint32_t (&r)[16]) {
    asm volatile("tcgen05.st.sync.aligned.16x256b.x4.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};" ::"r"(taddr), I16(r, 0) : "memory");
}
__device__ __forceinline__ void tmem_ld_16x128b_x8(uint32_t taddr, uint32_t (&r)[16]) {
    asm volatile("tcgen05.ld.sync.aligned.16x128b.x8.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];" : R16(r, 0) : "r"(taddr) : "memory");
}
__device__ __forceinline__ void tmem_st_16x128b_x8(uint32_t taddr, const uint32_t (&r)[16]) {
    asm volatile("tcgen05.st.sync.aligned.16x128b.x8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};" ::"r"(taddr), I16(r, 0) : "memory");
}
#undef R4
#undef R16
#undef I4
#undef I16

// A drafted token of an e4m3 cache whose V (codes at `raw`) has a NaN becomes zeros in the widened tile, whose row is at `to`: it would spread to
// lines that do not see it.  Those that do are looked for when the piece is done.  (A thread per token: they share their banks, so each begins at a
// chunk of its own.  Not inlined: the loop that widens, which all wait for, was slower with this in its middle)
template <int D> __noinline__ __device__ bool zero_odd_token(const uint8_t* raw, uint8_t* to) {
    bool odd = false;
#pragma unroll 1
    for (int k = 0; k < D / 16; ++k) {
        const uint4 v = *reinterpret_cast<const uint4*>(raw + ((k + threadIdx.x) & (D / 16 - 1)) * 16);
        odd = odd || odd_e4m3(v.x) || odd_e4m3(v.y) || odd_e4m3(v.z) || odd_e4m3(v.w);
    }
#pragma unroll 1
    for (int k = 0; odd && k < D / 8; ++k) *reinterpret_cast<uint4*>(to + (k >> 3) * (kBN * 128) + (k & 7) * 16) = make_uint4(0, 0, 0, 0);
    return odd;
}

// Floats of a piece's slot in global memory: [line][2] reference and sum, then [run of four channels][line][4] sums.
constexpr int kWideCarry = 2 * kWideLines;
template <int D> constexpr int kWideSlot = kWideCarry + kWideLines * D;

template <int D, int F>
__global__ void __launch_bounds__(kWideThreads, 1)
attn_draft_wide_kernel(const __grid_constant__ CUtensorMap tmap_k, const __grid_constant__ CUtensorMap tmap_v, const __grid_constant__ DraftParams p,
                       const uint8_t* k_codes, const uint8_t* v_codes) {
    typedef WideForm<D, F> S;
    constexpr uint32_t kOCol = 2 * kBN;
    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
    uint8_t* sq = smem;
    uint8_t* skv = sq + 2 * S::kTile;
    uint8_t* sraw = skv + S::kSlots * S::kTile;
    WideShared& sh = *reinterpret_cast<WideShared*>(sraw + S::kRaws * S::kRaw);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, group = warp >> 2;

    if (threadIdx.x == 0) {
        for (int i = 0; i < kPieceRing; ++i) { mbar_init(&sh.told[i], 1); mbar_init(&sh.left[i], kSoftmaxWarps + 5); }       // softmax and widening warps, the issuer
        for (int i = 0; i < 4; ++i) {
            mbar_init(&sh.raw_full[i], S::kWidens ? 33 : 1);
            mbar_init(&sh.full[i], 4);
            mbar_init(&sh.empty[i], 1);
            mbar_init(&sh.scaled[i], 4);
        }
        for (int i = 0; i < 3; ++i) mbar_init(&sh.raw_empty[i], 4);
        for (int i = 0; i < 2; ++i) { mbar_init(&sh.q_ready[i], 8); mbar_init(&sh.s_ready[i], 1); mbar_init(&sh.p_ready[i], 8); mbar_init(&sh.pv_done[i], 1); }
        mbar_init(&sh.meet, kSoftmaxWarps);
        mbar_init(&sh.spent, 1);
        sh.abort = 0;
        sh.merges = 0;
        sh.far = 0x7fffffff;
        for (int i = 0; i < kPieceRing; ++i) sh.odd[i] = 0;
        fence_mbar_init();
        if (!S::kWidens) { prefetch_tmap(&tmap_k); prefetch_tmap(&tmap_v); }
    }
    if (warp == kSoftmaxWarps + 1) { tmem_alloc(&sh.tmem_base, 512); tmem_relinquish(); }
    pdl_launch_dependents();
    const DraftList<kBN, 2> list(p);                  // (lengths, offsets and page table are no kernel's output: the plan need not wait)
    tc_fence_before();
    draft_plan<kWideThreads>(p, list, sh.share);
    tc_fence_after();
    const uint32_t tmem = sh.tmem_base;

    auto give_up = [&]() { if (lane == 0) { sh.abort = 1; atomicExch(p.status, AFLEX_ERR_TIMEOUT); } };
    // wait of a whole warp; false: it has run out, here or elsewhere
    auto wait = [&](uint64_t* bar, uint32_t parity) -> bool {
        const bool ok = mbar_wait(bar, parity);
        return __all_sync(0xffffffffu, ok);
    };

    if (group == 4) {
        if (warp == kSoftmaxWarps) {
            // -------------------------------------------------------------- producer: pieces and their pages
            const uint64_t policy = policy_evict_first();
            int pieces = 0, tile_no = 0;           // (tile_no: K and V tiles so far, two a step)
            bool ok = true;
            DraftWalk<kBN, 2> w;
            const long long x1 = sh.share.x1, total = sh.share.total;
            if (sh.share.x0 < x1) w.start(p, list, sh.share.x0, sh.share.seq, sh.share.seq_first, sh.share.seq_tiles);
            else w.pos = x1;
            while (ok && w.pos < x1) {
                if (w.u == 0 && w.nu > 1) { w.advance(p, list, 1, total); continue; }
                const int places = w.until(x1) - w.u;
                int units, t0, sees;
                {
                    const DraftPiece d = draft_piece(p, list, w, x1);
                    units = d.units; t0 = d.t0; sees = d.sees;
                    if (units == 0) { w.advance(p, list, places, total); continue; }      // (the second place of the CTA's before)
                    if (pieces == kPieceRing) pdl_wait();      // (the softmax warps, which leave pieces, wait for the preceding kernel without a limit)
                    ok = wait(&sh.left[pieces % kPieceRing], ((pieces / kPieceRing) & 1) ^ 1);
                    if (!ok) break;
                    if (lane == 0) {
                        sh.piece[pieces % kPieceRing] = d;
                        mbar_arrive(&sh.told[pieces % kPieceRing]);
                    }
                    __syncwarp();
                }
                ++pieces;
                const int g = w.g;
                const int32_t* table = p.page_table + (size_t)w.b * p.max_pages;
                const int page = lane & 7, part = lane >> 3;              // bf16: one box per (half, page)
                auto page_id = [&](int t) -> int {                        // of the unit with tokens t ..
                    const int i = t / kPageTokens + page;
                    return t >= 0 && i * kPageTokens < sees ? fetch(table + i) : 0;
                };
                auto pages_of = [&](int t) -> int { return min(kUnitPages, (sees - t + kPageTokens - 1) / kPageTokens); };
                auto checked = [&](int t, int id) -> int {
                    if (page < pages_of(t) && (id < 0 || id >= p.num_pages)) { if (part == 0) atomicExch(p.status, AFLEX_ERR_BOUNDS); return 0; }
                    return id;
                };
                auto bring = [&](int isv, int t, int id) {                // K or V of the unit with tokens t ..
                    const int np = pages_of(t);
                    if (S::kWidens) {
                        const int r = tile_no % 3;
                        ok = ok && wait(&sh.raw_empty[r], ((tile_no / 3) & 1) ^ 1);
                        if (!ok) return;
                        uint8_t* raw = sraw + r * S::kRaw;
                        if (lane == 0) mbar_expect_tx(&sh.raw_full[r], (uint32_t)(np * kPageTokens * D));
                        __syncwarp();
                        if (lane < np)
                            bulk_load_1d(raw + lane * (kPageTokens * D), (isv ? v_codes : k_codes) + ((size_t)id * p.Hkv + g) * (kPageTokens * D), kPageTokens * D, &sh.raw_full[r]);
                        const int from = __shfl_sync(0xffffffffu, id, lane >> 2);            // four lanes bring a page's scales
                        if (!isv && (lane >> 2) < np) {
                            const size_t at = ((size_t)from * p.Hkv + g) * kPageTokens + (lane & 3) * 4;
                            copy16(smem_u32(raw) + (uint32_t)(S::kRawTile + lane * 16), p.k_scales + at);
                            copy16(smem_u32(raw) + (uint32_t)(S::kRawTile + kBN * 4 + lane * 16), p.v_scales + at);
                        }
                        copies_arrive(&sh.raw_full[r]);
                    } else {
                        const int s = tile_no % S::kSlots;
                        ok = ok && wait(&sh.empty[s], ((tile_no / S::kSlots) & 1) ^ 1);
                        if (!ok) return;
                        if (lane == 0) mbar_expect_tx(&sh.raw_full[s], (uint32_t)(np * S::kHalves * kPageTokens * 128));
                        __syncwarp();
                        if (part < S::kHalves && page < np)
                            tma_load_2d_hint(skv + s * S::kTile + part * S::kHalf + page * (kPageTokens * 128), isv ? &tmap_v : &tmap_k, part * 64,
                                             (id * p.Hkv + g) * kPageTokens, &sh.raw_full[s], policy);
                    }
                    ++tile_no;
                };
                if (t0 >= 0) {
                    int id = page_id(t0), id_next = units > 1 ? page_id(t0 + kBN) : 0;
                    if (tile_no == 0) pdl_wait();
                    id = checked(t0, id);
                    bring(0, t0, id);
                    for (int t = t0, left = units; left > 0 && ok; t += kBN, --left) {
                        const int id_then = left > 2 ? page_id(t + 2 * kBN) : 0;
                        if (left > 1) id_next = checked(t + kBN, id_next);
                        if (S::kWidens && left > 1) bring(0, t + kBN, id_next);
                        bring(1, t, id);
                        if (!S::kWidens && left > 1) bring(0, t + kBN, id_next);
                        id = id_next;
                        id_next = id_then;
                    }
                }
                if (ok) w.advance(p, list, places, total);
            }
            pdl_wait();            // (pieces without tokens have not come by it)
            if (ok) ok = wait(&sh.left[pieces % kPieceRing], ((pieces / kPieceRing) & 1) ^ 1);
            if (ok && lane == 0) {
                sh.piece[pieces % kPieceRing].units = 0;
                mbar_arrive(&sh.told[pieces % kPieceRing]);
            }
            if (lane == 0) sh.tiles = tile_no;
            if (!ok) give_up();
        } else if (warp == kSoftmaxWarps + 1) {
            // -------------------------------------------------------------- issuer of the products (one thread)
            pdl_wait();            // (the preceding kernel may run for longer than a wait's limit, which begins behind it)
            if (lane == 0) {
                constexpr uint32_t kTileLo = S::kTile >> 4;
                const uint32_t idesc_s = wide_idesc<F>(kBN);
                const uint32_t idesc_pv = wide_idesc<F>(D) | (1u << 16);  // B operand (V) is MN-major
                const uint32_t q_lo = desc_lo(smem_u32(sq), 16), k_lo = desc_lo(smem_u32(skv), 16), v_lo = desc_lo(smem_u32(skv), S::kHalf);
                // (everything kept by increments: between a place's weights and its next scores this thread is what all wait for)
                uint32_t ks = 0, kp = 0, vs = S::kWidens ? 2 : 1, vp = 0;             // slot and parity of the next K and V
                uint32_t p0 = 0, p1 = 0;                                  // parities of the places' weights
                bool ok = true;
                uint32_t pc = 0, loaded = 0;
                auto next_k = [&]() { ks ^= S::kWidens ? 1u : 2u; if (ks == 0) kp ^= 1; };
                auto next_v = [&]() { if (!S::kWidens) vs ^= 2u; if (S::kWidens || vs == 1) vp ^= 1; };
                auto issue_s = [&](uint32_t i) {                          // scores of place i with the next K
                    const uint32_t to = tmem + i * kBN, a = q_lo + i * kTileLo, bk = k_lo + ks * kTileLo;
#pragma unroll
                    for (int j = 0; j < D / 16; ++j)
                        umma_ss(to, a + (uint32_t)(((j / 4) * S::kHalf + (j % 4) * 32) >> 4), bk + (uint32_t)(((j / 4) * S::kHalf + (j % 4) * 32) >> 4), idesc_s, j > 0 ? 1u : 0u);
                    umma_commit(&sh.s_ready[i]);
                };
                auto issue_pv = [&](uint32_t i, bool first) {             // place i's weights with the next V
                    const uint32_t to = tmem + kOCol + i * D, a = tmem + i * kBN, bv = v_lo + vs * kTileLo;
#pragma unroll
                    for (int part = 0; part < (F == AFLEX_CACHE_BF16 ? 2 : 1); ++part)
#pragma unroll
                        for (int j = 0; j < kBN / 16; ++j)
                            umma_ts(to, a + (uint32_t)((j >> 2) * 64 + part * 32 + (j & 3) * 8), bv + (uint32_t)((j * 2048) >> 4), idesc_pv, part > 0 || j > 0 ? 1u : first ? 0u : 1u);
                    umma_commit(&sh.pv_done[i]);
                };
                auto have_k = [&]() { ok = ok && mbar_wait(&sh.full[ks], kp); tc_fence_after(); return ok; };
                auto done_k = [&]() { umma_commit(&sh.empty[ks]); next_k(); };
                for (; ok; ++pc) {
                    ok = mbar_wait(&sh.told[pc % kPieceRing], (pc / kPieceRing) & 1);
                    if (!ok) break;
                    const DraftPiece& d = sh.piece[pc % kPieceRing];
                    const int units = d.t0 < 0 ? 0 : d.units;             // (an item without tokens has no step)
                    const bool end = d.units == 0, two = d.lines > kBM;
                    mbar_arrive(&sh.left[pc % kPieceRing]);
                    if (end) break;
                    if (units == 0) continue;
                    ok = mbar_wait(&sh.q_ready[0], loaded & 1) && mbar_wait(&sh.q_ready[1], loaded & 1);
                    ++loaded;
                    // The pipe runs in order: a place's scores may be issued over its weights as soon as their product has been.
                    if (two) {
                        if (!have_k()) break;
                        issue_s(0);
                        issue_s(1);
                        done_k();
                        for (int t = 0; t < units; ++t) {
                            const bool more = t + 1 < units;
                            ok = ok && mbar_wait(&sh.full[vs], vp) && mbar_wait(&sh.p_ready[0], p0);
                            if (!ok) break;
                            p0 ^= 1;
                            tc_fence_after();
                            issue_pv(0, t == 0);
                            if (more) { if (!have_k()) break; issue_s(0); }
                            ok = mbar_wait(&sh.p_ready[1], p1);
                            if (!ok) break;
                            p1 ^= 1;
                            tc_fence_after();
                            issue_pv(1, t == 0);
                            umma_commit(&sh.empty[vs]);
                            next_v();
                            if (more) { issue_s(1); done_k(); }
                        }
                    } else {
                        for (uint32_t i = 0; i < 2 && (int)i < units; ++i) {
                            if (!have_k()) break;
                            issue_s(i);
                            done_k();
                        }
                        for (int t = 0; t < units && ok; ++t) {
                            const uint32_t i = t & 1;
                            ok = mbar_wait(&sh.full[vs], vp) && mbar_wait(&sh.p_ready[i], i ? p1 : p0);
                            if (!ok) break;
                            if (i) p1 ^= 1; else p0 ^= 1;
                            tc_fence_after();
                            issue_pv(i, t < 2);
                            umma_commit(&sh.empty[vs]);
                            next_v();
                            if (t + 2 < units) { if (!have_k()) break; issue_s(i); done_k(); }
                        }
                    }
                }
                if (!ok) {
                    sh.abort = 1;
                    atomicExch(p.status, AFLEX_ERR_TIMEOUT);
                    umma_commit(&sh.spent);
                    mbar_wait(&sh.spent, 0);
                }
            }
        }
    } else if (group == 5) {
        // ------------------------------------------------------------------ widening; bf16: a look at the V of drafted tokens
        const int tid = threadIdx.x - (kWideThreads - 128);
        int tile_no = 0, step = 0;
        bool ok = true;
        pdl_wait();                                // (as the issuer)
        for (int pc = 0; ok; ++pc) {
            ok = wait(&sh.told[pc % kPieceRing], (pc / kPieceRing) & 1);
            if (!ok) break;
            const int units = sh.piece[pc % kPieceRing].units, t0 = sh.piece[pc % kPieceRing].t0, sees = sh.piece[pc % kPieceRing].sees, ctx = sh.piece[pc % kPieceRing].ctx;
            __syncwarp();
            if (lane == 0) mbar_arrive(&sh.left[pc % kPieceRing]);
            if (units == 0) break;
            if (t0 < 0) continue;
            if constexpr (S::kWidens) {
                auto widen = [&](int isv, int t, auto look) {
                    const int here = sees - (t0 + t * kBN), at = step + t;                // tokens of the step that count; the step's number
                    const int s = isv ? 2 : at & 1;
                    uint8_t* to = skv + s * S::kTile;
                    const int r = tile_no % 3;
                    const uint8_t* raw = sraw + r * S::kRaw;
                    ok = ok && wait(&sh.raw_full[r], (tile_no / 3) & 1);
                    ok = ok && wait(&sh.empty[s], ((isv ? at : at >> 1) & 1) ^ 1);
                    if (!ok) return;
                    if (!isv) {                // this thread's token's scales (the buffer is the step's four back; the products of three back have been waited for)
                        const float* own = reinterpret_cast<const float*>(raw + S::kRawTile) + tid;
                        const float x = tid < here ? own[0] : 0.f, y = tid < here ? own[kBN] : 1.f;
                        float* pair = reinterpret_cast<float*>(&sh.scale[at & 3][tid >> 1]) + (tid & 1);
                        const float lv = log2_scale(y);               // (NaN makes the scores of who sees it NaN)
                        pair[0] = x;
                        pair[2] = lv;
                        const float n = fast_exp2(-lv);
                        reinterpret_cast<float*>(sh.inv[at & 3])[tid] = n == n ? n : 0.f;
                        if (lv > kNear && lv < INFINITY) atomicMin(&sh.far, at);
                    }
                    // Chunks of 16 codes become two of 16 bytes of the tile, in half c / 4.  Four lanes of eight take a chunk's second eight codes first,
                    // the other four in rows of the other parity: so both the 8-byte loads and the 16-byte stores of a warp meet every
                    // bank equally often.  Half of the thread's chunks are loaded before the first is widened
                    constexpr int kPer = D / 16, kRows = 128 / kPer, kTurns = kBN / kRows;      // chunks per token, tokens per turn of the group
                    const int c = tid % kPer, row = tid / kPer;       // (kRows is a multiple of 8: a token's last three bits are row's)
                    const uint32_t second = (uint32_t)((c >> 2) ^ row) & 1;
                    uint8_t* half = to + (c >> 2) * S::kHalf + row * 128;
                    const uint8_t* from = raw + row * D + c * 16 + second * 8;
                    const uint32_t at0 = (uint32_t)((((c & 3) * 2 + second) ^ (row & 7)) << 4), at1 = at0 ^ 16;
                    const int other = 8 - 16 * (int)second;
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        uint2 x[kTurns / 2], y[kTurns / 2];
#pragma unroll
                        for (int it = 0; it < kTurns / 2; ++it) {
                            const uint8_t* src = from + (h * (kTurns / 2) + it) * kRows * D;
                            x[it] = *reinterpret_cast<const uint2*>(src);
                            y[it] = *reinterpret_cast<const uint2*>(src + other);
                        }
#pragma unroll
                        for (int it = 0; it < kTurns / 2; ++it) {
                            const int turn = h * (kTurns / 2) + it;
                            uint4 a, b;
                            widen4<F>(x[it].x, a.x, a.y); widen4<F>(x[it].y, a.z, a.w);
                            widen4<F>(y[it].x, b.x, b.y); widen4<F>(y[it].y, b.z, b.w);
                            if (isv && turn * kRows + row >= here) a = b = make_uint4(0, 0, 0, 0);      // slots behind the last token may hold anything
                            *reinterpret_cast<uint4*>(half + turn * kRows * 128 + at0) = a;
                            *reinterpret_cast<uint4*>(half + turn * kRows * 128 + at1) = b;
                        }
                    }
                    if (look && isv) {
                        // (a thread per token, of those that the warp has widened)
                        __syncwarp();
                        const int mine = lane / (32 / kPer) * kRows + warp % 4 * (32 / kPer) + lane % (32 / kPer);
                        if (mine < here && t0 + t * kBN + mine >= ctx && zero_odd_token<D>(raw + mine * D, to + mine * 128)) sh.odd[pc % kPieceRing] = pc + 1;
                    }
                    fence_proxy_async();
                    __syncwarp();
                    if (lane == 0) { mbar_arrive(&sh.full[s]); mbar_arrive(&sh.raw_empty[r]); if (!isv) mbar_arrive(&sh.scaled[at & 3]); }
                    ++tile_no;
                };
                auto tile = [&](int i, auto look) {                       // the i-th of K(0) K(1) V(0) K(2) V(1) .. V(units - 1)
                    const bool k = i == 0 || ((i & 1) && i != 2 * units - 1);
                    widen(k ? 0 : 1, k ? (i + 1) / 2 : i == 2 * units - 1 ? units - 1 : i / 2 - 1, look);
                };
                // e4m3: from the first V with drafted tokens on they are looked at (8 trees of up to 61: 227 us without that, 230 with, 239 if the
                // first tiles went through the same loop)
                int i = 0;
                const int plain = F == AFLEX_CACHE_E4M3 ? min(max((min(ctx, sees) - t0) / kBN, 0), units) : units;       // units without drafted tokens
#pragma unroll 1
                for (; i < 2 * plain && ok; ++i) tile(i, std::false_type());
#pragma unroll 1
                for (; F == AFLEX_CACHE_E4M3 && i < 2 * units && ok; ++i) tile(i, std::bool_constant<F == AFLEX_CACHE_E4M3>());
                step += units;
            } else {
                for (int t = 0; t < units && ok; ++t, ++step) {
                    const int here = sees - (t0 + t * kBN);                   // tokens of the step that count
                    for (int isv = 0; isv < 2; ++isv, ++tile_no) {
                        const int s = tile_no % S::kSlots;
                        uint8_t* to = skv + s * S::kTile;
                        ok = wait(&sh.raw_full[s], (tile_no / S::kSlots) & 1);
                        if (!ok) break;
                        if (isv && t0 + (t + 1) * kBN > min(ctx, sees)) {
                            // a thread per token: rows behind the last are zeroed, and so are drafted tokens with an infinity or NaN, which
                            // would spread to lines that do not see them (those that do are told by sh.bad)
                            bool odd = false;
                            if (tid < here && t0 + t * kBN + tid >= ctx) {
#pragma unroll 4
                                for (int k = 0; k < S::kHalves * 8; ++k) {
                                    const uint4 v = *reinterpret_cast<const uint4*>(to + (k >> 3) * S::kHalf + tid * 128 + (k & 7) * 16);
                                    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
                                    for (int i = 0; i < 4; ++i) odd = odd || odd_bf16(w[i]);
                                }
                            }
                            if (odd || tid >= here) {
#pragma unroll 4
                                for (int k = 0; k < S::kHalves * 8; ++k) *reinterpret_cast<uint4*>(to + (k >> 3) * S::kHalf + tid * 128 + (k & 7) * 16) = make_uint4(0, 0, 0, 0);
                            }
                            const uint32_t word = __ballot_sync(0xffffffffu, odd);
                            if (lane == 0) sh.bad[step & 3][tid >> 5] = word;
                            fence_proxy_async();
                        }
                        __syncwarp();
                        if (lane == 0) mbar_arrive(&sh.full[s]);
                    }
                }
            }
        }
        if (!ok) give_up();
    } else {
        // ------------------------------------------------------------------ softmax: 16 lines per warp, two (and a quarter of the tokens) per thread.
        // A warp reaches only the rows 32 (warp % 4) .. + 31 of TMEM; sixteens of lines go round these quarters, so that few lines keep all four
        // of the SM's schedulers busy
        const int place = warp >> 3, row0 = (warp & 3) * 32 + ((warp >> 2) & 1) * 16, hl = lane >> 2, l4 = lane & 3;
        const uint32_t lane_base = tmem + ((uint32_t)row0 << 16);
        const uint32_t s_addr = lane_base + (uint32_t)(place * kBN), o_addr = lane_base + kOCol;
        int steps_before = 0;                      // of all pieces: the ring's position
        uint32_t done = 0;                         // steps of this place
        bool ok = true;
        uint32_t met = 0;
        auto meet = [&]() -> bool {                // all softmax warps (a bounded wait: a warp that has given up does not come)
            __syncwarp();
            if (lane == 0) mbar_arrive(&sh.meet);
            const bool came = wait(&sh.meet, met & 1);
            ++met;
            return came;
        };
        pdl_wait();
        for (int pc = 0; ok; ++pc) {
            ok = wait(&sh.told[pc % kPieceRing], (pc / kPieceRing) & 1);
            if (!ok) break;
            const DraftPiece& d = sh.piece[pc % kPieceRing];          // (left when the piece is done)
            if (d.units == 0) break;
            const int units = d.t0 < 0 ? 0 : d.units;
            const bool two = d.lines > kBM;
            const int line0 = (two ? place * kBM : 0) + (warp & 7) * 16;          // of the warp's first row
            const bool busy = line0 < d.lines;                        // (a warp without lines only keeps step)
            if (units > 0 && busy) {
                // ---- the warp's queries into the place's tile, two halves of 128 bytes, swizzled; D / 8 lanes for a line
                constexpr int kLanes = D / 8, kAtOnce = 32 / kLanes, kTurns = 16 / kAtOnce;
                const int sub = lane / kLanes, ch = lane % kLanes;
                uint4 v[kTurns];
#pragma unroll
                for (int it = 0; it < kTurns; ++it) {
                    const int line = line0 + it * kAtOnce + sub;
                    v[it] = make_uint4(0, 0, 0, 0);
                    if (line < d.lines)
                        v[it] = fetch(reinterpret_cast<const uint4*>(p.q + ((size_t)(d.row0 + (line >> p.g_shift)) * p.Hq + (size_t)d.g * p.G + (line & (p.G - 1))) * D) + ch);
                }
#pragma unroll
                for (int it = 0; it < kTurns; ++it) {
                    const int row = row0 + it * kAtOnce + sub;
                    float c = p.scale_log2;
                    if (S::kWidens) {
                        uint32_t* x = reinterpret_cast<uint32_t*>(&v[it]);
                        uint32_t big = __vmaxu2(__vmaxu2(x[0] & 0x7fff7fffu, x[1] & 0x7fff7fffu), __vmaxu2(x[2] & 0x7fff7fffu, x[3] & 0x7fff7fffu));
                        big = max(big & 0xffffu, big >> 16);
#pragma unroll
                        for (int off = 1; off < kLanes; off <<= 1) big = max(big, __shfl_xor_sync(0xffffffffu, big, off));
                        // largest in [2^e, 2^(e + 1)): times 2^(14 - e); tiny lines by 2^126
                        const int e = max((int)(big >> 7) - 127, -112);
                        const float up = __uint_as_float((uint32_t)(127 + 14 - e) << 23);
                        c = big >= 0x7f80u ? __uint_as_float(0x7fc00000u) : p.scale_log2 * __uint_as_float((uint32_t)(127 - 14 + e) << 23);
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const __half2 h = __floats2half2_rn(__uint_as_float(x[i] << 16) * up, __uint_as_float(x[i] & 0xffff0000u) * up);
                            x[i] = *reinterpret_cast<const uint32_t*>(&h);
                        }
                    }
                    *reinterpret_cast<uint4*>(sq + place * S::kTile + (ch >> 3) * S::kHalf + row * 128 + (((ch & 7) ^ (row & 7)) << 4)) = v[it];
                    if (ch == 0) sh.factor[place][row] = c;
                }
                fence_proxy_async();
            }
            __syncwarp();
            if (units > 0 && lane == 0) mbar_arrive(&sh.q_ready[place]);
            float m[2] = {kLowest, kLowest}, l[2] = {0.f, 0.f}, c[2] = {0.f, 0.f};
            if (units > 0 && busy) { c[0] = sh.factor[place][row0 + hl]; c[1] = sh.factor[place][row0 + hl + 8]; }
            const int plain = min(d.ctx, d.sees), t0 = d.t0;
            int mine_steps = 0;
            for (int t = two ? 0 : place; t < units && ok; t += two ? 1 : 2, ++done, ++mine_steps) {
                const int step = steps_before + t, jv = 2 * step + 1, sv = jv % S::kSlots;
                ok = wait(&sh.s_ready[place], done & 1);
                const bool masked = t0 + (t + 1) * kBN > plain;
                if (S::kWidens) ok = ok && wait(&sh.scaled[step & 3], (step >> 2) & 1);
                else if (masked) ok = ok && wait(&sh.full[sv], (jv / S::kSlots) & 1);               // (what is known of V)
                if (!ok) break;
                if (busy) {
                    const bool far = S::kWidens && step >= sh.far;      // (a later step's number may stand there already, and changes nothing)
                    tc_fence_after();
                    // Half of the tokens at a time, whose weights go where their scores were: both halves' scores would not fit the registers.
#pragma unroll 1
                    for (int half = 0; half < 2 && ok; ++half) {
                        uint32_t x0[16], x1[16];   // scores of 32 tokens each
                        tmem_ld_16x256b_x4(s_addr + (uint32_t)(half * 64), x0);
                        tmem_ld_16x256b_x4(s_addr + (uint32_t)(half * 64 + 32), x1);
                        const ulonglong2* scales = reinterpret_cast<const ulonglong2*>(sh.scale[step & 3]) + half * 32 + l4;
                        const uint64_t cc[2] = {pack_f32x2(c[0], c[0]), pack_f32x2(c[1], c[1])};
                        tmem_ld_wait();
                        auto scaled = [&](uint32_t (&x)[16], int first) {
#pragma unroll
                            for (int i = 0; i < 4; ++i) {
                                ulonglong2 sc;
                                if (S::kWidens) sc = scales[first + 4 * i];
#pragma unroll
                                for (int y = 0; y < 2; ++y) {
                                    uint64_t v = mul_f32x2(pack_f32x2(__uint_as_float(x[4 * i + 2 * y]), __uint_as_float(x[4 * i + 2 * y + 1])), cc[y]);
                                    if (S::kWidens) v = fma_f32x2(v, sc.x, sc.y);
                                    float a, b;
                                    unpack_f32x2(v, a, b);
                                    x[4 * i + 2 * y] = __float_as_uint(a);
                                    x[4 * i + 2 * y + 1] = __float_as_uint(b);
                                }
                            }
                        };
                        scaled(x0, 0);
                        scaled(x1, 16);
                        if (masked) {
#pragma unroll
                            for (int y = 0; y < 2; ++y) {
                                const int line = line0 + hl + 8 * y, mine = line >> p.g_shift, qi = d.i0 + mine;
                                const bool there = line < d.lines;
                                const uint32_t* mask = p.mask + (size_t)(d.row0 + mine) * p.mask_words;
#pragma unroll
                                for (int q = 0; q < 2; ++q) {
                                    // which of 32 tokens this line sees
                                    const int t32 = t0 + t * kBN + 64 * half + 32 * q, j0 = t32 - d.ctx;       // the first of them, its number among the drafted
                                    uint32_t see = 0xffffffffu;
                                    const int last = d.sees - t32;        // tokens behind the last do not count
                                    if (last < 32) see = last <= 0 ? 0u : (1u << last) - 1u;
                                    if (j0 + 31 >= 0 && see != 0) {
                                        uint32_t drafted;                 // bits of tokens j0 .. j0 + 31, earlier ones set
                                        const uint32_t early = j0 < 0 ? (1u << -j0) - 1u : 0u;
                                        if (p.mask == nullptr) {
                                            const int upto = qi - j0 + 1; // tokens 0 .. qi
                                            drafted = upto >= 32 ? 0xffffffffu : upto <= 0 ? 0u : (1u << upto) - 1u;
                                        } else {
                                            auto word = [&](int i) -> uint32_t { return there && i >= 0 && i < p.mask_words ? fetch(mask + i) : 0u; };
                                            const int wi = j0 >> 5, sft = j0 & 31;          // (arithmetic shift: -1 for tokens before the first)
                                            drafted = __funnelshift_r(word(wi), word(wi + 1), (uint32_t)sft);
                                            const int over = d.m - j0;    // bits of tokens that there are
                                            if (over < 32) drafted &= over <= 0 ? 0u : (1u << over) - 1u;
                                        }
                                        see &= drafted | early;
                                    }
                                    if (!there) see = 0;
                                    if (!S::kWidens && (see & sh.bad[step & 3][2 * half + q])) l[y] = __uint_as_float(0x7fc00000u);
                                    see >>= 2 * l4;
#pragma unroll
                                    for (int i = 0; i < 4; ++i)
#pragma unroll
                                        for (int e = 0; e < 2; ++e)
                                            if (!(see >> (8 * i + e) & 1u)) (q ? x1 : x0)[4 * i + 2 * y + e] = 0xff800000u;
                                }
                            }
                        }
                        float mx[2] = {-INFINITY, -INFINITY};
#pragma unroll
                        for (int i = 0; i < 4; ++i)
#pragma unroll
                            for (int y = 0; y < 2; ++y) {
                                mx[y] = max3(mx[y], __uint_as_float(x0[4 * i + 2 * y]), __uint_as_float(x0[4 * i + 2 * y + 1]));
                                mx[y] = max3(mx[y], __uint_as_float(x1[4 * i + 2 * y]), __uint_as_float(x1[4 * i + 2 * y + 1]));
                            }
                        constexpr float kRoom = kBelow<F> + 7.f;
                        if (__any_sync(0xffffffffu, mx[0] > m[0] + kRoom || mx[1] > m[1] + kRoom)) {
                            float corr[2];
#pragma unroll
                            for (int y = 0; y < 2; ++y) {
                                mx[y] = fmaxf(mx[y], __shfl_xor_sync(0xffffffffu, mx[y], 1));
                                mx[y] = fmaxf(mx[y], __shfl_xor_sync(0xffffffffu, mx[y], 2));
                                const float mn = mx[y] > m[y] + kRoom ? ceilf(mx[y]) - kBelow<F> : m[y];          // (whole: what was rounded is scaled exactly)
                                corr[y] = fast_exp2(m[y] - mn);
                                l[y] = scale_sum(l[y], m[y] - mn);
                                m[y] = mn;
                            }
                            tmem_st_wait();        // (in the second half: the first one's weights, and the sums if it moved the references too)
                            if (mine_steps > 0) {
                                ok = wait(&sh.pv_done[place], (done - 1) & 1);
                                if (!ok) break;
                                tc_fence_after();
#pragma unroll 1
                                for (int c0 = 0; c0 < D; c0 += 32) {
                                    uint32_t r[16];
                                    tmem_ld_16x256b_x4(o_addr + (uint32_t)(place * D + c0), r);
                                    tmem_ld_wait();
#pragma unroll
                                    for (int i = 0; i < 16; ++i) r[i] = __float_as_uint(__uint_as_float(r[i]) * corr[(i >> 1) & 1]);
                                    tmem_st_16x256b_x4(o_addr + (uint32_t)(place * D + c0), r);
                                }
                            }
                            if (half == 1) {       // and the weights of the first half
                                uint32_t hi[16], lo[16];
                                tmem_ld_16x128b_x8(s_addr, hi);
                                if (!S::kWidens) tmem_ld_16x128b_x8(s_addr + 32, lo);
                                tmem_ld_wait();
#pragma unroll
                                for (int i = 0; i < 16; ++i) {
                                    float w0, w1;
                                    if (S::kWidens) {
                                        const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&hi[i]));
                                        w0 = f.x; w1 = f.y;
                                    } else {
                                        w0 = __uint_as_float(hi[i] << 16) + __uint_as_float(lo[i] << 16);
                                        w1 = __uint_as_float(hi[i] & 0xffff0000u) + __uint_as_float(lo[i] & 0xffff0000u);
                                    }
                                    pack_weights<F>(w0 * corr[i & 1], w1 * corr[i & 1], hi[i], lo[i]);
                                }
                                tmem_st_16x128b_x8(s_addr, hi);
                                if (!S::kWidens) tmem_st_16x128b_x8(s_addr + 32, lo);
                            }
                        }
                        if (far) {                 // the sums by exponentials of their own (see kNear)
                            const float* lvs = reinterpret_cast<const float*>(&sh.scale[step & 3][half * 32 + l4]) + 2;
                            auto count = [&](const uint32_t (&x)[16], int first) {
#pragma unroll
                                for (int i = 0; i < 16; ++i) {
                                    const float lv = lvs[4 * (first + 4 * (i >> 2)) + (i & 1)];
                                    l[(i >> 1) & 1] += fast_exp2(__uint_as_float(x[i]) - m[(i >> 1) & 1] - (lv == lv ? lv : 0.f));
                                }
                            };
                            count(x0, 0);
                            count(x1, 16);
                        }
                        uint32_t hi[16], lo[16];
                        const float2* invs = reinterpret_cast<const float2*>(sh.inv[step & 3]) + half * 32 + l4;
                        const uint64_t m2[2] = {pack_f32x2(-m[0], -m[0]), pack_f32x2(-m[1], -m[1])};
                        uint64_t sum[2] = {0, 0};
                        auto weights = [&](const uint32_t (&x)[16], int first) {
#pragma unroll
                            for (int i = 0; i < 4; ++i) {
                                uint64_t n = 0;
                                if (S::kWidens) n = *reinterpret_cast<const uint64_t*>(invs + first + 4 * i);
#pragma unroll
                                for (int y = 0; y < 2; ++y) {
                                    float w0, w1;
                                    unpack_f32x2(add_f32x2(pack_f32x2(__uint_as_float(x[4 * i + 2 * y]), __uint_as_float(x[4 * i + 2 * y + 1])), m2[y]), w0, w1);
                                    w0 = fast_exp2(w0);
                                    w1 = fast_exp2(w1);
                                    sum[y] = S::kWidens ? fma_f32x2(pack_f32x2(w0, w1), n, sum[y]) : add_f32x2(sum[y], pack_f32x2(w0, w1));
                                    pack_weights<F>(w0, w1, hi[first / 2 + 2 * i + y], lo[first / 2 + 2 * i + y]);
                                }
                            }
                        };
                        weights(x0, 0);
                        weights(x1, 16);
                        tmem_st_16x128b_x8(s_addr + (uint32_t)(half * 64), hi);
                        if (!S::kWidens) tmem_st_16x128b_x8(s_addr + (uint32_t)(half * 64 + 32), lo);
#pragma unroll
                        for (int y = 0; y < 2; ++y) {
                            float a, b;
                            unpack_f32x2(sum[y], a, b);
                            if (!far) l[y] += a + b;
                        }
                    }
                    if (!ok) break;
                    tmem_st_wait();
                }
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(&sh.p_ready[place]);
            }
            steps_before += units;
            if (!ok) break;
            // ---- the piece is done: normalised to the output, or its sums to the CTA's slot
            if (mine_steps > 0) ok = wait(&sh.pv_done[place], (done - 1) & 1);
            if (!ok) break;
            if (F == AFLEX_CACHE_E4M3 && mine_steps > 0 && sh.odd[pc % kPieceRing] == pc + 1) {
                // some drafted token has a NaN in V: the lines that see it become NaN.  (A search of all of the piece's, a token per lane, for
                // something that seldom is; well inside a wait's limit for a million of them)
                const int end = min(d.sees, t0 + units * kBN);
#pragma unroll 1
                for (int j0 = max(t0, d.ctx); j0 < end; j0 += 32) {
                    bool odd = false;
                    if (j0 + lane < end) {
                        const int j = j0 + lane, id = fetch(p.page_table + (size_t)d.b * p.max_pages + j / kPageTokens);
                        const uint4* v = reinterpret_cast<const uint4*>(v_codes + (((size_t)(id >= 0 && id < p.num_pages ? id : 0) * p.Hkv + d.g) * kPageTokens + j % kPageTokens) * D);
#pragma unroll 1
                        for (int k = 0; k < D / 16; ++k) {
                            const uint4 x = fetch(v + k);
                            odd = odd || odd_e4m3(x.x) || odd_e4m3(x.y) || odd_e4m3(x.z) || odd_e4m3(x.w);
                        }
                    }
#pragma unroll 1
                    for (uint32_t left = __ballot_sync(0xffffffffu, odd); left != 0; left &= left - 1) {
                        const int j = j0 + __ffs(left) - 1 - d.ctx;
#pragma unroll
                        for (int y = 0; y < 2; ++y) {
                            const int line = line0 + hl + 8 * y, i = line >> p.g_shift;
                            if (line < d.lines && l[y] == l[y] && sees_drafted(p, d.row0 + i, d.i0 + i, j, d.m)) l[y] = __uint_as_float(0x7fc00000u);
                        }
                    }
                }
            }
#pragma unroll
            for (int y = 0; y < 2; ++y) {
                l[y] += __shfl_xor_sync(0xffffffffu, l[y], 1);
                l[y] += __shfl_xor_sync(0xffffffffu, l[y], 2);
            }
            float f[2][2] = {{1.f, 0.f}, {1.f, 0.f}};       // [line][this place's sums, the other's]: what they count
            const bool use[2] = {mine_steps > 0, !two && (place == 1 ? units > 0 : units > 1)};      // (an empty place's accumulator holds anything)
            int ch0 = 0, ch1 = D;
            tc_fence_after();
            if (!two) {
                // one tile in two places: both learn of the other's states, and store half of the channels each
                if (l4 == 0) {
                    sh.state[place][row0 + hl] = make_float2(m[0], l[0]);
                    sh.state[place][row0 + hl + 8] = make_float2(m[1], l[1]);
                }
                tc_fence_before();
                ok = meet();
                if (!ok) break;
                tc_fence_after();
#pragma unroll
                for (int y = 0; y < 2; ++y) {
                    const float2 other = sh.state[place ^ 1][row0 + hl + 8 * y];
                    const float M = fmaxf(m[y], other.x);
                    f[y][0] = fast_exp2(m[y] - M);
                    f[y][1] = fast_exp2(other.x - M);
                    l[y] = scale_sum(l[y], m[y] - M) + scale_sum(other.y, other.x - M);
                    m[y] = M;
                }
                ch0 = place * (D / 2);
                ch1 = ch0 + D / 2;
            }
            if (busy) {
                float* slot = p.parts + ((size_t)blockIdx.x * 2 + d.slot) * kWideSlot<D>;
                const bool whole = d.whole;
                float inv[2];
                size_t hq[2];
                bool there[2];
#pragma unroll
                for (int y = 0; y < 2; ++y) {
                    const int line = line0 + hl + 8 * y;
                    there[y] = line < d.lines;
                    hq[y] = (size_t)(d.row0 + (line >> p.g_shift)) * p.Hq + (size_t)d.g * p.G + (line & (p.G - 1));
                    inv[y] = l[y] == 0.f ? 0.f : __frcp_rn(l[y]) * p.unit;
                    if (there[y] && ch0 == 0 && l4 == 0) {
                        if (!whole) __stcg(reinterpret_cast<float2*>(slot) + line, make_float2(m[y], l[y]));
                        else if (p.lse != nullptr) p.lse[hq[y]] = l[y] == 0.f ? -INFINITY : (m[y] + __log2f(l[y])) * 0.6931471805599453f;
                    }
                }
#pragma unroll 1
                for (int c0 = ch0; c0 < ch1; c0 += 32) {
                    float x[16];
#pragma unroll
                    for (int i = 0; i < 16; ++i) x[i] = 0.f;
#pragma unroll
                    for (int o = 0; o < 2; ++o) {
                        if (use[o]) {
                            uint32_t r[16];
                            tmem_ld_16x256b_x4(o_addr + (uint32_t)((place ^ o) * D + c0), r);
                            tmem_ld_wait();
#pragma unroll
                            for (int i = 0; i < 16; ++i) x[i] = fmaf(__uint_as_float(r[i]), f[(i >> 1) & 1][o], x[i]);
                        }
                    }
#pragma unroll
                    for (int i = 0; i < 4; ++i)
#pragma unroll
                        for (int y = 0; y < 2; ++y) {
                            const int ch = c0 + 8 * i + 2 * l4;
                            if (!there[y]) continue;
                            if (whole) *reinterpret_cast<uint32_t*>(p.out + hq[y] * D + ch) = pack_bf16x2(x[4 * i + 2 * y] * inv[y], x[4 * i + 2 * y + 1] * inv[y]);
                            else __stcg(reinterpret_cast<float2*>(slot + kWideCarry + ((ch >> 2) * kWideLines + line0 + hl + 8 * y) * 4 + (ch & 2)), make_float2(x[4 * i + 2 * y], x[4 * i + 2 * y + 1]));
                        }
                }
            }
            tc_fence_before();
            // the next piece's products go where the other place still reads; a slot has to be complete
            if (!two || !d.whole) {
                ok = meet();
                if (!ok) break;
            }
            if (!d.whole && threadIdx.x == 0) {
                // the last of the item's CTAs to get here joins the pieces (offsets that decrease could name more items than there are counters)
                __threadfence();
                if (d.item >= kAttnCounterCap) atomicExch(p.status, AFLEX_ERR_BOUNDS);
                else if (atomicAdd(p.counters + d.item, 1) == sh.share.cta_of(d.last) - sh.share.cta_of(d.first)) {
                    p.counters[d.item] = 0;
                    sh.merge[sh.merges++] = d;
                }
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(&sh.left[pc % kPieceRing]);
        }
        // ---- join the pieces of the items that this CTA was the last one to work on, half of a line per thread
        ok = ok && meet();
        if (ok) {
            __threadfence();
            for (int j = 0; j < sh.merges; ++j) {
                const DraftPiece& d = sh.merge[j];
                const int c0 = sh.share.cta_of(d.first), n = sh.share.cta_of(d.last) - c0 + 1, line = threadIdx.x % kWideLines, part_of = threadIdx.x / kWideLines;
                if (line >= d.lines) continue;
                auto part = [&](int k) -> const float* { return p.parts + ((size_t)(c0 + k) * 2 + (k == 0 ? 1 : 0)) * kWideSlot<D>; };       // (the first CTA's second slot)
                float M = kLowest, L = 0.f;
                for (int k = 0; k < n; ++k) M = fmaxf(M, __ldcg(reinterpret_cast<const float2*>(part(k)) + line).x);
                for (int k = 0; k < n; ++k) {
                    const float2 ml = __ldcg(reinterpret_cast<const float2*>(part(k)) + line);
                    L += scale_sum(ml.y, ml.x - M);
                }
                constexpr int kAtOnce = 8;         // runs of four channels
#pragma unroll 1
                for (int r0 = part_of * (D / 8); r0 < (part_of + 1) * (D / 8); r0 += kAtOnce) {
                    float4 acc[kAtOnce];
#pragma unroll
                    for (int r = 0; r < kAtOnce; ++r) acc[r] = make_float4(0.f, 0.f, 0.f, 0.f);
                    for (int k = 0; k < n; ++k) {
                        const float g = fast_exp2(__ldcg(reinterpret_cast<const float2*>(part(k)) + line).x - M);
                        const float4* v = reinterpret_cast<const float4*>(part(k) + kWideCarry) + r0 * kWideLines + line;
#pragma unroll
                        for (int r = 0; r < kAtOnce; ++r) {
                            const float4 y = __ldcg(v + r * kWideLines);
                            acc[r].x = fmaf(y.x, g, acc[r].x); acc[r].y = fmaf(y.y, g, acc[r].y); acc[r].z = fmaf(y.z, g, acc[r].z); acc[r].w = fmaf(y.w, g, acc[r].w);
                        }
                    }
#pragma unroll
                    for (int r = 0; r < kAtOnce; ++r) store_run<D>(p, d, line, r0 + r, RunSum{M, L, acc[r]});
                }
            }
        }
        if (!ok) give_up();
    }
    tc_fence_before();
    __syncthreads();
    if (sh.abort) {                                // copies under way are waited for once more, since this memory will be another CTA's
        constexpr int kRing = S::kWidens ? 3 : S::kSlots;
        for (int i = max(0, sh.tiles - kRing); i < sh.tiles; ++i) mbar_wait(&sh.raw_full[i % kRing], (i / kRing) & 1);
        __syncthreads();
    }
    if (warp == kSoftmaxWarps + 1) { tc_fence_after(); tmem_dealloc(tmem, 512); }
}

template <int D, int F>
aflex_status launch_t(aflex_ctx* ctx, const aflex_cache* cache, int grid, const DraftParams& p, cudaStream_t st) {
    typedef WideForm<D, F> S;
    CUtensorMap tk = {}, tv = {};
    if (!S::kWidens) {
        const uint64_t rows = (uint64_t)cache->kv.num_pages * p.Hkv * kPageTokens;
        if (!encode_tmap_2d_bf16(&tk, cache->kv.k_cache, rows, D, (uint64_t)D * 2, kPageTokens, 64, true) ||
            !encode_tmap_2d_bf16(&tv, cache->kv.v_cache, rows, D, (uint64_t)D * 2, kPageTokens, 64, true))
            return set_error(ctx, AFLEX_ERR_CUDA, "draft attention: cuTensorMapEncodeTiled failed");
    }
    const size_t smem = (size_t)S::kSmem + sizeof(WideShared) + 1024;
    static_assert(S::kSmem + sizeof(WideShared) + 1024 <= kMaxDynamicSmem, "shared memory of one CTA");
    if (!ctx->draft_attr_set[D == 128][F][2]) {
        cudaError_t e = cudaFuncSetAttribute(attn_draft_wide_kernel<D, F>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
        if (e != cudaSuccess) return check_cuda(ctx, e, "cudaFuncSetAttribute(draft attention)");
        ctx->draft_attr_set[D == 128][F][2] = true;
    }
    KernelScope scope(ctx, kKAttnDraft, st);
    return check_cuda(ctx, launch_pdl(attn_draft_wide_kernel<D, F>, dim3((unsigned)grid), dim3(kWideThreads), smem, st, tk, tv, p,
                                      (const uint8_t*)cache->kv.k_cache, (const uint8_t*)cache->kv.v_cache),
                      "attn_draft_wide_kernel launch");
}

}  // namespace

// ------------------------------------------------------------------------------------------ host
size_t attn_draft_wide_workspace_bytes(int head_dim, int num_sms) {
    return align256((size_t)num_sms * 2 * (kWideCarry + kWideLines * head_dim) * sizeof(float));
}

aflex_status attn_draft_wide_launch(aflex_ctx* ctx, const aflex_cache* cache, int head_dim, const DraftParams& p, cudaStream_t st) {
    typedef aflex_status (*Launch)(aflex_ctx*, const aflex_cache*, int, const DraftParams&, cudaStream_t);
    const Launch launch[2][3] = {{launch_t<64, AFLEX_CACHE_BF16>, launch_t<64, AFLEX_CACHE_INT8>, launch_t<64, AFLEX_CACHE_E4M3>},
                                 {launch_t<128, AFLEX_CACHE_BF16>, launch_t<128, AFLEX_CACHE_INT8>, launch_t<128, AFLEX_CACHE_E4M3>}};
    return launch[head_dim == 128][cache->format](ctx, cache, ctx->num_sms, p, st);
}

}  // namespace aflex
