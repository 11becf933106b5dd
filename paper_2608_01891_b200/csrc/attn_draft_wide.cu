// Attention of drafted tokens over a paged cache in bf16 or in 8 bits, for sequences with more lines (rows x query heads of a KV head's
// group) than attn_draft.cu is for: a page's K and V serve up to 256 lines, the products bound it, and they run on the tcgen05 tensor cores.
//
//   work        as in attn_draft.cu: equal shares of the list of units, one CTA per SM, pieces joined by the CTA that is last
//   tiles       two S / P and two O accumulators in TMEM.  An item of more than 128 lines has two tiles of 128, both at every step of 128 cached
//               tokens; one of up to 128 has its one tile in both places, one for the even and one for the odd steps, so that one's softmax runs
//               under the other's products either way
//   data path   a producer warp brings pages; of an 8-bit cache they are widened to fp16 by a warp group of its own, exactly (the scales are the
//               softmax's business), into the swizzled layout that the tensor cores read; a bf16 cache's pages are copied into that layout by TMA
//               and the warp group only looks at the V of drafted tokens.  K is a K-major operand, V (as stored) an MN-major one
//   softmax     two warp groups, a line per thread; statistics, references and weights as in attn_draft.cu.  The weights of an 8-bit cache are
//               stored back over the scores they came from, in fp16; those of a bf16 cache as two bf16 parts, which fill the place of the
//               scores, and the second product is issued for each part
//
// Bound: of long trees the exponentials (16 per cycle and SM against 8192 multiply-adds) and the products about equally; of short ones with few lines
// the widening and the read of the cache.
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <math.h>

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
constexpr int kWideThreads = 512;                  // warp groups: softmax of places 0 and 1, producer + issuer, widening
constexpr int kRegsSoftmax = 184, kRegsIssue = 64, kRegsWiden = 80;
static_assert(256 * kRegsSoftmax + 128 * kRegsIssue + 128 * kRegsWiden <= 512 * 128, "the warp groups share what the block was launched with");
constexpr int kPieceRing = 4;

template <int D, int F> struct WideForm {
    static constexpr bool kWidens = F != AFLEX_CACHE_BF16;
    static constexpr int kHalves = D / 64;
    static constexpr int kHalf = kBN * 128;                           // 128 rows of 128 bytes: 64 channels of a tile of lines or of tokens
    static constexpr int kTile = kHalves * kHalf;                     // Q of a place, K or V of a step
    static constexpr int kSlots = kWidens ? 3 : 4;                    // ring of K and V: K(0) V(0) K(1) V(1) ..
    static constexpr int kRaws = kWidens ? 3 : 0;                     // ring of the same in 8 bits
    static constexpr int kRawTile = kBN * D;
    static constexpr int kRaw = kRawTile + kBN * 4;                   // and its scales
    static constexpr int kSmem = 2 * kTile + kSlots * kTile + kRaws * kRaw;
};

struct __align__(16) WideShared {
    float4 scale[2][kBN / 2];                      // by step: of two tokens, K's scales and log2 of V's
    float4 inv[2][kBN / 4];                        // 1 / V's, of four tokens
    float2 state[2][kBM];                          // of one tile in two places: references and sums
    uint32_t bad[4][kBN / 32];                     // by step: tokens whose V holds an infinity or NaN (bf16)
    uint64_t told[kPieceRing], left[kPieceRing];   // a piece's description is there, everybody has read it
    uint64_t raw_full[4], raw_empty[3];            // pages have landed (bf16: in their slot), have been widened
    uint64_t full[4], empty[4];                    // a slot can be read by the products, has been
    uint64_t q_ready[2], s_ready[2], p_ready[2], pv_done[2], meet;       // meet: the softmax warps
    DraftPiece piece[kPieceRing];
    DraftShare share;
    DraftPiece merge[2];
    int merges;
    uint32_t tmem_base;
    volatile int abort;
};

template <int F> __device__ __forceinline__ uint32_t wide_idesc(uint32_t n) {
    const uint32_t d = umma_idesc_bf16(kBM, n);
    return F == AFLEX_CACHE_BF16 ? d : d & ~((1u << 7) | (1u << 10));                     // fp16 operands
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
        for (int i = 0; i < kPieceRing; ++i) { mbar_init(&sh.told[i], 1); mbar_init(&sh.left[i], 13); }       // 8 softmax, 4 widening warps, the issuer
        for (int i = 0; i < 4; ++i) {
            mbar_init(&sh.raw_full[i], S::kWidens ? 33 : 1);
            mbar_init(&sh.full[i], 4);
            mbar_init(&sh.empty[i], 1);
        }
        for (int i = 0; i < 3; ++i) mbar_init(&sh.raw_empty[i], 4);
        for (int i = 0; i < 2; ++i) { mbar_init(&sh.q_ready[i], 4); mbar_init(&sh.s_ready[i], 1); mbar_init(&sh.p_ready[i], 4); mbar_init(&sh.pv_done[i], 1); }
        mbar_init(&sh.meet, 8);
        sh.abort = 0;
        sh.merges = 0;
        fence_mbar_init();
        if (!S::kWidens) { prefetch_tmap(&tmap_k); prefetch_tmap(&tmap_v); }
    }
    if (warp == 9) { tmem_alloc(&sh.tmem_base, 512); tmem_relinquish(); }
    pdl_launch_dependents();
    const DraftList<kBN> list(p);                  // (lengths, offsets and page table are no kernel's output: the plan need not wait)
    tc_fence_before();
    draft_plan<kBN, kWideThreads>(p, list, sh.share);
    tc_fence_after();
    const uint32_t tmem = sh.tmem_base;

    auto give_up = [&]() { if (lane == 0) { sh.abort = 1; atomicExch(p.status, AFLEX_ERR_TIMEOUT); } };
    // wait of a whole warp; false: it has run out, here or elsewhere
    auto wait = [&](uint64_t* bar, uint32_t parity) -> bool {
        const bool ok = mbar_wait(bar, parity);
        return __all_sync(0xffffffffu, ok);
    };

    if (group == 2) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kRegsIssue));
        if (warp == 8) {
            // -------------------------------------------------------------- producer: pieces and their pages
            const uint64_t policy = policy_evict_first();
            int pieces = 0, tile_no = 0;           // (tile_no: K and V tiles so far, two a step)
            bool ok = true;
            DraftWalk<kBN> w;
            const long long x1 = sh.share.x1, total = sh.share.total;
            if (sh.share.x0 < x1) w.start(p, list, sh.share.x0, sh.share.seq, sh.share.seq_first, sh.share.seq_tiles);
            else w.pos = x1;
            while (ok && w.pos < x1) {
                if (w.u == 0 && w.nu > 1) { w.advance(p, list, 1, total); continue; }
                ok = wait(&sh.left[pieces % kPieceRing], ((pieces / kPieceRing) & 1) ^ 1);
                if (!ok) break;
                const int units = draft_piece(p, list, w, x1).units;
                const int u0 = w.u, sees = list.sees(w.s, w.tile), g = w.g;
                if (lane == 0) {
                    sh.piece[pieces % kPieceRing] = draft_piece(p, list, w, x1);
                    mbar_arrive(&sh.told[pieces % kPieceRing]);
                }
                __syncwarp();
                ++pieces;
                const int32_t* table = p.page_table + (size_t)w.b * p.max_pages;
                const int page = lane & 7, part = lane >> 3;              // bf16: one box per (half, page)
                auto page_id = [&](int u) -> int {
                    const int i = (u - 1) * kUnitPages + page;
                    return u >= 1 && i * kPageTokens < sees ? fetch(table + i) : 0;
                };
                int id = page_id(u0);
                for (int u = u0; u < u0 + units && ok && u >= 1; ++u) {
                    const int id_next = u + 1 < u0 + units ? page_id(u + 1) : 0;
                    const int np = min(kUnitPages, (sees - (u - 1) * kBN + kPageTokens - 1) / kPageTokens);
                    if (page < np && (id < 0 || id >= p.num_pages)) { if (part == 0) atomicExch(p.status, AFLEX_ERR_BOUNDS); id = 0; }
                    if (tile_no == 0) pdl_wait();
                    for (int isv = 0; isv < 2 && ok; ++isv, ++tile_no) {
                        if (S::kWidens) {
                            const int r = tile_no % 3;
                            ok = wait(&sh.raw_empty[r], ((tile_no / 3) & 1) ^ 1);
                            if (!ok) break;
                            uint8_t* raw = sraw + r * S::kRaw;
                            if (lane == 0) mbar_expect_tx(&sh.raw_full[r], (uint32_t)(np * kPageTokens * D));
                            __syncwarp();
                            if (lane < np)
                                bulk_load_1d(raw + lane * (kPageTokens * D), (isv ? v_codes : k_codes) + ((size_t)id * p.Hkv + g) * (kPageTokens * D), kPageTokens * D, &sh.raw_full[r]);
                            const int from = __shfl_sync(0xffffffffu, id, lane >> 2);        // four lanes bring a page's scales
                            if ((lane >> 2) < np)
                                copy16(smem_u32(raw) + (uint32_t)(S::kRawTile + lane * 16), (isv ? p.v_scales : p.k_scales) + ((size_t)from * p.Hkv + g) * kPageTokens + (lane & 3) * 4);
                            copies_arrive(&sh.raw_full[r]);
                        } else {
                            const int s = tile_no % S::kSlots;
                            ok = wait(&sh.empty[s], ((tile_no / S::kSlots) & 1) ^ 1);
                            if (!ok) break;
                            if (lane == 0) mbar_expect_tx(&sh.raw_full[s], (uint32_t)(np * S::kHalves * kPageTokens * 128));
                            __syncwarp();
                            if (part < S::kHalves && page < np)
                                tma_load_2d_hint(skv + s * S::kTile + part * S::kHalf + page * (kPageTokens * 128), isv ? &tmap_v : &tmap_k, part * 64,
                                                 (id * p.Hkv + g) * kPageTokens, &sh.raw_full[s], policy);
                        }
                    }
                    id = id_next;
                }
                if (ok) w.advance(p, list, units, total);
            }
            if (ok) ok = wait(&sh.left[pieces % kPieceRing], ((pieces / kPieceRing) & 1) ^ 1);
            if (ok && lane == 0) {
                sh.piece[pieces % kPieceRing].units = 0;
                mbar_arrive(&sh.told[pieces % kPieceRing]);
            }
            if (!ok) give_up();
        } else if (warp == 9) {
            // -------------------------------------------------------------- issuer of the products (one thread)
            if (lane == 0) {
                const uint32_t idesc_s = wide_idesc<F>(kBN);
                const uint32_t idesc_pv = wide_idesc<F>(D) | (1u << 16);  // B operand (V) is MN-major
                int slot = 0, loaded = 0;          // K and V tiles so far; pieces with queries
                uint32_t done[2] = {0, 0};         // steps of either place so far
                bool ok = true;
                for (int pc = 0; ok; ++pc) {
                    ok = mbar_wait(&sh.told[pc % kPieceRing], (pc / kPieceRing) & 1);
                    if (!ok) break;
                    const DraftPiece& d = sh.piece[pc % kPieceRing];
                    const int units = d.t0 < 0 ? 0 : d.units;             // (an item without tokens has no step)
                    const bool end = d.units == 0, two = d.lines > kBM;
                    mbar_arrive(&sh.left[pc % kPieceRing]);
                    if (end) break;
                    if (units == 0) continue;
                    for (int i = 0; i < 2 && ok; ++i) ok = mbar_wait(&sh.q_ready[i], loaded & 1);
                    ++loaded;
                    if (!ok) break;
                    // S of step t in place i; the place's S / P columns are free once its previous P V has been issued: the pipe runs in order
                    auto issue_s = [&](int t, int i) {
                        const int j = slot + 2 * t, s = j % S::kSlots;
                        ok = ok && mbar_wait(&sh.full[s], (j / S::kSlots) & 1);
                        if (!ok) return;
                        tc_fence_after();
                        const uint32_t k_lo = desc_lo(smem_u32(skv + s * S::kTile), 16), q_lo = desc_lo(smem_u32(sq + i * S::kTile), 16);
#pragma unroll
                        for (int ks = 0; ks < D / 16; ++ks)
                            umma_ss(tmem + (uint32_t)(i * kBN), q_lo + (uint32_t)(((ks / 4) * S::kHalf + (ks % 4) * 32) >> 4),
                                    k_lo + (uint32_t)(((ks / 4) * S::kHalf + (ks % 4) * 32) >> 4), idesc_s, ks > 0 ? 1u : 0u);
                        umma_commit(&sh.s_ready[i]);
                    };
                    auto free_k = [&](int t) { umma_commit(&sh.empty[(slot + 2 * t) % S::kSlots]); };
                    // the first steps: of both places, 0; of one tile, 0 and 1
                    issue_s(0, 0);
                    if (two && ok) issue_s(0, 1);
                    if (ok) free_k(0);
                    if (!two && units > 1 && ok) { issue_s(1, 1); if (ok) free_k(1); }
                    for (int t = 0; t < units && ok; ++t) {
                        const int jv = slot + 2 * t + 1, sv = jv % S::kSlots;
                        for (int i = two ? 0 : t & 1; i < (two ? 2 : (t & 1) + 1) && ok; ++i) {
                            ok = mbar_wait(&sh.p_ready[i], done[i] & 1);
                            ok = ok && mbar_wait(&sh.full[sv], (jv / S::kSlots) & 1);
                            if (!ok) break;
                            tc_fence_after();
                            const bool first = two ? t == 0 : t < 2;
                            const uint32_t v_lo = desc_lo(smem_u32(skv + sv * S::kTile), S::kHalf);
#pragma unroll
                            for (int part = 0; part < (F == AFLEX_CACHE_BF16 ? 2 : 1); ++part)
#pragma unroll
                                for (int ks = 0; ks < kBN / 16; ++ks)
                                    umma_ts(tmem + kOCol + (uint32_t)(i * D), tmem + (uint32_t)(i * kBN + part * 64 + ks * 8), v_lo + (uint32_t)((ks * 2048) >> 4), idesc_pv,
                                            (!first || ks > 0 || part > 0) ? 1u : 0u);
                            umma_commit(&sh.pv_done[i]);
                            ++done[i];
                            // (the slot of V first: the widening of the step after next waits for it)
                            if (!two || i == 1) umma_commit(&sh.empty[sv]);
                            if (two && t + 1 < units) { issue_s(t + 1, i); if (i == 1 && ok) free_k(t + 1); }
                            if (!two && t + 2 < units) { issue_s(t + 2, i); if (ok) free_k(t + 2); }
                        }
                    }
                    slot += 2 * units;
                }
                if (!ok) { sh.abort = 1; atomicExch(p.status, AFLEX_ERR_TIMEOUT); }
            }
        }
    } else if (group == 3) {
        // ------------------------------------------------------------------ widening; bf16: a look at the V of drafted tokens
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kRegsWiden));
        const int tid = threadIdx.x - 384;
        int tile_no = 0, step = 0;
        bool ok = true;
        for (int pc = 0; ok; ++pc) {
            ok = wait(&sh.told[pc % kPieceRing], (pc / kPieceRing) & 1);
            if (!ok) break;
            const int units = sh.piece[pc % kPieceRing].units, t0 = sh.piece[pc % kPieceRing].t0, sees = sh.piece[pc % kPieceRing].sees, ctx = sh.piece[pc % kPieceRing].ctx;
            __syncwarp();
            if (lane == 0) mbar_arrive(&sh.left[pc % kPieceRing]);
            if (units == 0) break;
            if (t0 < 0) continue;
            for (int t = 0; t < units && ok; ++t, ++step) {
                const int here = sees - (t0 + t * kBN);                   // tokens of the step that count
                for (int isv = 0; isv < 2; ++isv, ++tile_no) {
                    const int s = tile_no % S::kSlots;
                    uint8_t* to = skv + s * S::kTile;
                    if (S::kWidens) {
                        const int r = tile_no % 3;
                        const uint8_t* raw = sraw + r * S::kRaw;
                        ok = wait(&sh.raw_full[r], (tile_no / 3) & 1);
                        ok = ok && wait(&sh.empty[s], ((tile_no / S::kSlots) & 1) ^ 1);
                        if (!ok) break;
                        {   // this thread's token's scale (the buffer of the step before last is free: its V's slot was waited for)
                            const float x = tid < here ? reinterpret_cast<const float*>(raw + S::kRawTile)[tid] : 0.f;
                            float* pair = reinterpret_cast<float*>(&sh.scale[step & 1][tid >> 1]) + (tid & 1);
                            if (isv == 0) pair[0] = x;
                            else {
                                float lv = tid < here ? __log2f(x) : 0.f;
                                if (lv < -64.f) lv = -64.f;               // (a scale of 0; NaN stays, and makes the scores of who sees it NaN)
                                pair[2] = lv;
                                const float n = fast_exp2(-lv);
                                reinterpret_cast<float*>(sh.inv[step & 1])[tid] = n == n ? n : 0.f;
                            }
                        }
                        // a chunk of 16 codes at a time: two chunks of 16 bytes of the tile, half c / 4
                        constexpr int kPer = D / 16, kRows = 128 / kPer;  // chunks per token, tokens per turn of the group
                        const int c = tid % kPer, row = tid / kPer;
                        uint8_t* half = to + (c >> 2) * S::kHalf;
                        const uint32_t at0 = (uint32_t)((((c & 3) * 2) ^ (row & 7)) << 4), at1 = at0 ^ 16;
#pragma unroll
                        for (int it = 0; it < kBN / kRows; ++it) {
                            const int token = it * kRows + row;           // (kRows is a multiple of 8: token & 7 == row & 7)
                            uint4 x = *reinterpret_cast<const uint4*>(raw + token * D + c * 16);
                            if (isv && token >= here) x = make_uint4(0, 0, 0, 0);          // slots behind the last token may hold anything
                            uint4 a, b;
                            if (token >= here && isv) a = b = make_uint4(0, 0, 0, 0);
                            else {
                                widen4<F>(x.x, a.x, a.y); widen4<F>(x.y, a.z, a.w);
                                widen4<F>(x.z, b.x, b.y); widen4<F>(x.w, b.z, b.w);
                            }
                            *reinterpret_cast<uint4*>(half + token * 128 + at0) = a;
                            *reinterpret_cast<uint4*>(half + token * 128 + at1) = b;
                        }
                        fence_proxy_async();
                        __syncwarp();
                        if (lane == 0) { mbar_arrive(&sh.full[s]); mbar_arrive(&sh.raw_empty[r]); }
                    } else {
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
                                    for (int i = 0; i < 4; ++i) odd = odd || (w[i] & 0x7f80u) == 0x7f80u || (w[i] & 0x7f800000u) == 0x7f800000u;
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
        // ------------------------------------------------------------------ softmax: a line per thread
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kRegsSoftmax));
        const int place = group, w4 = warp & 3, row = w4 * 32 + lane;
        const uint32_t lane_base = tmem + ((uint32_t)(w4 * 32) << 16);
        const uint32_t s_addr = lane_base + (uint32_t)(place * kBN), o_addr = lane_base + kOCol;
        int steps_before = 0;                      // of all pieces: the ring's position
        uint32_t done = 0;                         // steps of this place
        bool ok = true;
        uint32_t met = 0;
        auto meet = [&]() -> bool {                // both softmax groups (a bounded wait: a warp that has given up does not come)
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
            const DraftPiece d = sh.piece[pc % kPieceRing];
            __syncwarp();
            if (lane == 0) mbar_arrive(&sh.left[pc % kPieceRing]);
            if (d.units == 0) break;
            const int units = d.t0 < 0 ? 0 : d.units;
            const bool two = d.lines > kBM;
            const int line = two ? place * kBM + row : row;
            const bool there = line < d.lines;
            const bool busy = (two ? place * kBM : 0) + w4 * 32 < d.lines;                  // (a warp without lines only keeps step)
            const int mine = line >> p.g_shift, qrow = d.row0 + mine, qi = d.i0 + mine;
            float c = p.scale_log2;
            if (units > 0) {
                // ---- this line's queries into the place's tile, two halves of 128 bytes, swizzled
                uint8_t* tile = sq + place * S::kTile + row * 128;
                const uint4* src = reinterpret_cast<const uint4*>(p.q + ((size_t)(there ? qrow : d.row0) * p.Hq + (size_t)d.g * p.G + (line & (p.G - 1))) * D);
                if (busy) {
                    uint32_t big = 0;
                    if (S::kWidens) {
#pragma unroll 4
                        for (int k = 0; k < D / 8; ++k) {
                            const uint4 v = fetch(src + k);
                            big = __vmaxu2(big, __vmaxu2(__vmaxu2(v.x & 0x7fff7fffu, v.y & 0x7fff7fffu), __vmaxu2(v.z & 0x7fff7fffu, v.w & 0x7fff7fffu)));
                        }
                        big = max(big & 0xffffu, big >> 16);
                    }
                    // largest in [2^e, 2^(e + 1)): times 2^(14 - e); tiny lines by 2^126
                    const int e = max((int)(big >> 7) - 127, -112);
                    const float up = __uint_as_float((uint32_t)(127 + 14 - e) << 23);
                    if (S::kWidens) c = big >= 0x7f80u ? __uint_as_float(0x7fc00000u) : p.scale_log2 * __uint_as_float((uint32_t)(127 - 14 + e) << 23);
#pragma unroll 4
                    for (int k = 0; k < D / 8; ++k) {
                        uint4 v = fetch(src + k);
                        if (!there) v = make_uint4(0, 0, 0, 0);
                        if (S::kWidens) {
                            uint32_t* x = reinterpret_cast<uint32_t*>(&v);
#pragma unroll
                            for (int i = 0; i < 4; ++i) {
                                const __half2 h = __floats2half2_rn(__uint_as_float(x[i] << 16) * up, __uint_as_float(x[i] & 0xffff0000u) * up);
                                x[i] = *reinterpret_cast<const uint32_t*>(&h);
                            }
                        }
                        *reinterpret_cast<uint4*>(tile + (k >> 3) * S::kHalf + (((k & 7) ^ (row & 7)) << 4)) = v;
                    }
                }
                fence_proxy_async();
            }
            __syncwarp();
            if (units > 0 && lane == 0) mbar_arrive(&sh.q_ready[place]);
            float m = kLowest, l = 0.f;
            const int first = two ? 0 : place, by = two ? 1 : 2;
            int mine_steps = 0;
            for (int t = first; t < units && ok; t += by, ++done, ++mine_steps) {
                const int step = steps_before + t, jv = 2 * step + 1, sv = jv % S::kSlots, col0 = d.t0 + t * kBN;
                ok = wait(&sh.s_ready[place], done & 1);
                const bool masked = col0 + kBN > min(d.ctx, d.sees);
                if (S::kWidens || masked) ok = ok && wait(&sh.full[sv], (jv / S::kSlots) & 1);      // (the scales, and what is known of V)
                if (!ok) break;
                tc_fence_after();
                if (busy) {
                    float x[kBN];
#pragma unroll
                    for (int c0 = 0; c0 < kBN; c0 += 16) tmem_ld_32x32b_x16(s_addr + (uint32_t)c0, *reinterpret_cast<uint32_t(*)[16]>(&x[c0]));
                    tmem_ld_wait();
                    const uint64_t cc = pack_f32x2(c, c);
#pragma unroll
                    for (int j = 0; j < kBN; j += 2) {
                        uint64_t v = mul_f32x2(pack_f32x2(x[j], x[j + 1]), cc);
                        if (S::kWidens) {
                            const ulonglong2 sc = *reinterpret_cast<const ulonglong2*>(&sh.scale[step & 1][j >> 1]);
                            v = fma_f32x2(v, sc.x, sc.y);
                        }
                        unpack_f32x2(v, x[j], x[j + 1]);
                    }
                    bool poison = false;
                    if (masked) {
#pragma unroll
                        for (int q = 0; q < kBN / 32; ++q) {
                            // which of 32 tokens this line sees
                            const int j0 = col0 + 32 * q - d.ctx;         // drafted token of the first of them
                            uint32_t see = 0xffffffffu;
                            const int last = d.sees - (col0 + 32 * q);    // tokens behind the last do not count
                            if (last < 32) see = last <= 0 ? 0u : (1u << last) - 1u;
                            if (j0 + 31 >= 0 && see != 0) {
                                uint32_t drafted;                         // bits of tokens j0 .. j0 + 31, earlier ones set
                                const uint32_t early = j0 < 0 ? (1u << -j0) - 1u : 0u;
                                if (p.mask == nullptr) {
                                    const int upto = qi - j0 + 1;         // tokens 0 .. qi
                                    drafted = upto >= 32 ? 0xffffffffu : upto <= 0 ? 0u : (1u << upto) - 1u;
                                } else {
                                    auto word = [&](int i) -> uint32_t { return there && i >= 0 && i < p.mask_words ? fetch(p.mask + (size_t)qrow * p.mask_words + i) : 0u; };
                                    const int wi = j0 >> 5, sft = j0 & 31;                  // (arithmetic shift: -1 for tokens before the first)
                                    drafted = __funnelshift_r(word(wi), word(wi + 1), (uint32_t)sft);
                                    const int over = d.m - j0;            // bits of tokens that there are
                                    if (over < 32) drafted &= over <= 0 ? 0u : (1u << over) - 1u;
                                }
                                see &= drafted | early;
                            }
                            if (!there) see = 0;
                            if (!S::kWidens && (see & sh.bad[step & 3][q])) poison = true;
#pragma unroll
                            for (int j = 0; j < 32; ++j) if (!(see >> j & 1u)) x[32 * q + j] = -INFINITY;
                        }
                    }
                    float mx0 = -INFINITY, mx1 = -INFINITY, mx2 = -INFINITY, mx3 = -INFINITY;
#pragma unroll
                    for (int j = 0; j < kBN; j += 4) {
                        mx0 = fmaxf(mx0, x[j]); mx1 = fmaxf(mx1, x[j + 1]); mx2 = fmaxf(mx2, x[j + 2]); mx3 = fmaxf(mx3, x[j + 3]);
                    }
                    const float mx = fmaxf(fmaxf(mx0, mx1), fmaxf(mx2, mx3));
                    // weights are 2^(x - m), m the running maximum less 8: below 2^15 until a score outgrows it
                    if (__any_sync(0xffffffffu, mx > m + 15.f)) {
                        const float mn = fmaxf(m, mx - 8.f), corr = fast_exp2(m - mn);
                        m = mn;
                        l *= corr;
                        if (mine_steps > 0) {
                            ok = wait(&sh.pv_done[place], (done - 1) & 1);
                            if (!ok) break;                // (leaves the steps; noticed below)
                            tc_fence_after();
#pragma unroll
                            for (int c0 = 0; c0 < D; c0 += 16) {
                                uint32_t r[16];
                                tmem_ld_32x32b_x16(o_addr + (uint32_t)(place * D + c0), r);
                                tmem_ld_wait();
#pragma unroll
                                for (int j = 0; j < 16; ++j) r[j] = __float_as_uint(__uint_as_float(r[j]) * corr);
                                tmem_st_32x32b_x16(o_addr + (uint32_t)(place * D + c0), r);
                            }
                        }
                    }
                    const uint64_t m2 = pack_f32x2(-m, -m), one = pack_f32x2(1.f, 1.f);
                    uint64_t l0 = 0, l1 = 0;
#pragma unroll
                    for (int c0 = 0; c0 < kBN; c0 += 32) {
                        uint32_t hi[16], lo[16];
#pragma unroll
                        for (int j = 0; j < 32; j += 2) {
                            float w0, w1;
                            unpack_f32x2(fma_f32x2(pack_f32x2(x[c0 + j], x[c0 + j + 1]), one, m2), w0, w1);
                            w0 = fast_exp2(w0);
                            w1 = fast_exp2(w1);
                            uint64_t& sum = j & 2 ? l1 : l0;
                            if (S::kWidens) {
                                const float2 n = *reinterpret_cast<const float2*>(reinterpret_cast<const float*>(sh.inv[step & 1]) + c0 + j);
                                sum = fma_f32x2(pack_f32x2(w0, w1), pack_f32x2(n.x, n.y), sum);
                                const __half2 h = __floats2half2_rn(w0, w1);
                                hi[j >> 1] = *reinterpret_cast<const uint32_t*>(&h);
                            } else {
                                sum = fma_f32x2(pack_f32x2(w0, w1), one, sum);
                                hi[j >> 1] = pack_bf16x2(w0, w1);
                                lo[j >> 1] = pack_bf16x2(w0 - __uint_as_float(hi[j >> 1] << 16), w1 - __uint_as_float(hi[j >> 1] & 0xffff0000u));
                            }
                        }
                        tmem_st_32x32b_x16(s_addr + (uint32_t)(c0 / 2), hi);
                        if (!S::kWidens) tmem_st_32x32b_x16(s_addr + 64 + (uint32_t)(c0 / 2), lo);
                    }
                    tmem_st_wait();
                    float a, b, e, f;
                    unpack_f32x2(l0, a, b);
                    unpack_f32x2(l1, e, f);
                    l += (a + b) + (e + f);
                    if (poison) l = __uint_as_float(0x7fc00000u);
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
            float* slot = p.parts + ((size_t)blockIdx.x * 2 + d.slot) * kWideSlot<D>;
            float f[2] = {0.f, 0.f};               // what the places' sums count; 0: nothing is there
            int ch0 = 0, ch1 = D;                  // channels that this thread stores
            if (two || units == 0) f[place] = units > 0 ? 1.f : 0.f;
            if (!two) {
                // both groups learn of both states, and store half of the channels each
                sh.state[place][row] = make_float2(m, l);
                tc_fence_after();
                tc_fence_before();
                ok = meet();
                if (!ok) break;
                const float2 other = sh.state[place ^ 1][row];
                const float M = fmaxf(m, other.x), mine_f = fast_exp2(m - M), other_f = fast_exp2(other.x - M);
                l = l * mine_f + other.y * other_f;
                m = M;
                if (units > 0) {                   // (an empty place's accumulator holds anything)
                    f[place] = mine_steps > 0 ? mine_f : 0.f;
                    f[place ^ 1] = place == 1 || units > 1 ? other_f : 0.f;
                }
                ch0 = place * (D / 2);
                ch1 = ch0 + D / 2;
            }
            tc_fence_after();
            if (busy) {
                const bool use0 = two ? place == 0 && units > 0 : units > 0, use1 = two ? place == 1 && units > 0 : units > 1;
                const float inv = l == 0.f ? 0.f : __frcp_rn(l);
                const size_t hq = (size_t)(there ? qrow : d.row0) * p.Hq + (size_t)d.g * p.G + (line & (p.G - 1));
                uint4* out = reinterpret_cast<uint4*>(p.out + hq * D);
#pragma unroll 1
                for (int c0 = ch0; c0 < ch1; c0 += 16) {
                    float x[16];
#pragma unroll
                    for (int j = 0; j < 16; ++j) x[j] = 0.f;
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        if (i == 0 ? use0 : use1) {
                            uint32_t r[16];
                            tmem_ld_32x32b_x16(o_addr + (uint32_t)(i * D + c0), r);
                            tmem_ld_wait();
#pragma unroll
                            for (int j = 0; j < 16; ++j) x[j] = fmaf(__uint_as_float(r[j]), f[i], x[j]);
                        }
                    }
                    if (there && d.whole) {
                        uint32_t w[8];
#pragma unroll
                        for (int j = 0; j < 16; j += 2) w[j >> 1] = pack_bf16x2(x[j] * inv, x[j + 1] * inv);
                        out[c0 / 8] = make_uint4(w[0], w[1], w[2], w[3]);
                        out[c0 / 8 + 1] = make_uint4(w[4], w[5], w[6], w[7]);
                    } else if (there) {
#pragma unroll
                        for (int j = 0; j < 16; j += 4)
                            __stcg(reinterpret_cast<float4*>(slot + kWideCarry) + ((c0 + j) >> 2) * kWideLines + line, make_float4(x[j], x[j + 1], x[j + 2], x[j + 3]));
                    }
                }
                if (there && ch0 == 0) {
                    if (!d.whole) __stcg(reinterpret_cast<float2*>(slot) + line, make_float2(m, l));
                    else if (p.lse != nullptr) p.lse[hq] = l == 0.f ? -INFINITY : (m + __log2f(l)) * 0.6931471805599453f;
                }
            }
            tc_fence_before();
            if (!two || !d.whole) {                // the next piece's products go where the other group still reads; the slot has to be complete
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
        }
        // ---- join the pieces of the items that this CTA was the last one to work on, a line per thread
        ok = ok && meet();
        if (ok) {
            __threadfence();
            for (int j = 0; j < sh.merges; ++j) {
                const DraftPiece& d = sh.merge[j];
                const int c0 = sh.share.cta_of(d.first), n = sh.share.cta_of(d.last) - c0 + 1, line = threadIdx.x;
                if (line >= d.lines) continue;
                auto part = [&](int k) -> const float* { return p.parts + ((size_t)(c0 + k) * 2 + (k == 0 ? 1 : 0)) * kWideSlot<D>; };       // (the first CTA's second slot)
                float M = kLowest, L = 0.f;
                for (int k = 0; k < n; ++k) M = fmaxf(M, __ldcg(reinterpret_cast<const float2*>(part(k)) + line).x);
                for (int k = 0; k < n; ++k) {
                    const float2 ml = __ldcg(reinterpret_cast<const float2*>(part(k)) + line);
                    L = fmaf(ml.y, fast_exp2(ml.x - M), L);
                }
                constexpr int kAtOnce = 8;         // runs of four channels
#pragma unroll 1
                for (int r0 = 0; r0 < D / 4; r0 += kAtOnce) {
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
    if (warp == 9) { tc_fence_after(); tmem_dealloc(tmem, 512); }
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
