// Attention of a chunk of new tokens over a paged K/V cache: what its kernels share.
//
//   out[t, h] = sum_j p_j V_j,  p = softmax_j(scale q[t, h] . K_j),  j over the slots start[s] .. last(t)
//
// last(t) is the token's own slot (causal) or lens[s] - 1; a row that sees no slot is zero.  The G query heads of a KV head
// share its rows: the rows of a tile are (token, head of the group) pairs, TQ = BM / G tokens by G heads, so that K and V are read
// once per tile and not once per head.  A unit is one (sequence, KV head, row tile).
#pragma once
#include "paged.cuh"
#include "rope_rows.cuh"  // RowsView, PackRow

namespace lar {

// The softmax's reference m is the largest logit itself, and a weight 2^((s - m) scale_log2): s - m is exact where it matters, however large the logits
// are.  Scaled first, in one multiply-add per weight, the reference is off by half a step of its own, and from logits of 2^31 on that alone
// makes every weight of a row 0 or infinite.
__device__ __forceinline__ float softmax_ref(float m) { return m == -INFINITY ? 0.f : m; }  // (a row that has seen nothing yet)

struct PagedAttnArgs {
    PagedView kv;
    RowsView q, out;
    const int* start;  // [n_seqs] first slot that is seen, or null
    int group, causal;
    int tq;            // tokens of a row tile
    float scale_log2;  // softmax scale * log2(e)
    float* part_o;     // partial results of units whose slots are spread over several CTAs
    float* part_ml;
    int n_splits;
    int parts;         // fp32: 1: rows are left as parts (split); 2: as one of two passes that are joined
    float* row_o;      // kernels with PART: (O, m, l) of every (token, head) instead of its output row
    float* row_ml;
    int2* row_ref;     // where a row's unit is cut: first range + 65536 * last, place among a range's rows; else -1 (row_o, row_ml hold the row)
};

// two fp32 operations in one instruction
__device__ __forceinline__ uint64_t pack_f32x2(float a, float b) {
    uint64_t r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ void unpack_f32x2(uint64_t v, float& a, float& b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(v)); }
__device__ __forceinline__ uint64_t fma_f32x2(uint64_t a, uint64_t b, uint64_t c) {
    uint64_t r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}
__device__ __forceinline__ uint64_t mul_f32x2(uint64_t a, uint64_t b) {
    uint64_t r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ uint64_t add_f32x2(uint64_t a, uint64_t b) {
    uint64_t r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}

// Row tiles of a sequence.
__device__ __forceinline__ int tiles_of(const PagedAttnArgs& a, int s) {
    int t0, t1;
    chunk_of(a.kv, s, t0, t1);
    return (t1 - t0 + a.tq - 1) / a.tq;
}

}  // namespace lar
