// What the kernels over rows of sequences share: where a row sits, loads that see a preceding kernel's stores, rotary lane layout and
// packed fp32 arithmetic.  A row is one query token: the one being decoded, or one of the last few of its sequence.
#pragma once
#include <cuda_bf16.h>
#include <stdint.h>

namespace aflex {

// A plain load, for what a preceding kernel may have written (projections, queries, lists, lengths, bounds): these kernels may have
// started before that one was done and wait for it, so the read-only path (ld.global.nc) would not be bound to see its stores.
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

// Lane layout of rotary kernels: D / 16 lanes hold one token's head, lane l the channels [8 l, 8 l + 8) and
// [D / 2 + 8 l, D / 2 + 8 l + 8) -- the two halves a rotary pair comes from; 32 / (D / 16) tokens per warp at a time.
template <int D> struct Lanes {
    static constexpr int kPer = D / 16;           // lanes per token
    static constexpr int kTok = 32 / kPer;        // tokens per warp at a time
    static constexpr int kIter = kPageTokens / kTok;
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
__device__ __forceinline__ uint64_t add_f32x2(uint64_t a, uint64_t b) {
    uint64_t d;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
    return d;
}
__device__ __forceinline__ uint64_t mul_f32x2(uint64_t a, uint64_t b) {
    uint64_t d;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
    return d;
}
}  // namespace aflex
