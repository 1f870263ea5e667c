// Attention of sequences that have their first slots in common, in groups: the two small kernels around those of the chunk attention.
//
//   softmax over the slots 0 .. last(t) = the softmax over the L slots in common, once for all tokens of a group, joined with that over L .. last(t):
//       m = max(m1, m2),  out = (O1 e^(m1 - m) + O2 e^(m2 - m)) / (l1 e^(m1 - m) + l2 e^(m2 - m))       (O, l: sums without the division)
//
// The slots in common are one unit per (group, KV head), whose rows are all tokens of the group: they are read once per 256 rows and not once
// per sequence.  Every token of a group sees all of them (L is cut to what the shortest cache of the group held before its chunk), so that
// pass needs no mask.
//
// Bound by the slots' bytes and by what launches cost that wait for one another.  64 sequences of one token, 8192 slots in common and up to 577 of their own, 8 KV heads of 4
// x 128: 48 us, of which the groups take 3, each pass 30 to 36 beside the other and the join 5 (through the chunk attention alone, which
// reads the slots in common per sequence, from L2: 208 us).
#pragma once
#include "join_parts.cuh"
#include "paged_attn.cuh"
#include "part_range.h"

namespace lar {

struct SharedPrepArgs {
    PagedView kv;
    const int* groups;  // [n_groups + 1] sequences
    const int* shared;  // [n_groups] slots in common
    int n_groups;
    int* cu;      // [n_groups + 1] tokens
    int* len;     // [n_groups] slots in common of each
    int* row_of;  // [n_groups] the sequence whose pages are read
    int* start;   // [n_seqs] first slot of a sequence's own
};

constexpr int kSharedPrepThreads = 128;

// The groups as sequences, a CTA each.
static __global__ void __launch_bounds__(kSharedPrepThreads) shared_prep_kernel(const __grid_constant__ SharedPrepArgs a) {
    __shared__ int least[kSharedPrepThreads / 32], firsts[kSharedPrepThreads / 32];
    grid_dep_launch();
    const int tid = threadIdx.x, g = blockIdx.x, S = a.kv.n_seqs;
    const int s0 = min(max(a.groups[g], 0), S), s1 = min(max(a.groups[g + 1], s0), S);
    auto token_of = [&](int s) {  // the first token of sequence s; S: behind the last one's
        int t0, t1;
        chunk_of(a.kv, min(s, S - 1), t0, t1);
        return s < S ? t0 : t1;
    };
    int L = INT_MAX, first = INT_MAX;  // first: the first sequence with tokens; one without (an image that is done) may have given up its pages
    for (int s = s0 + tid; s < s1; s += kSharedPrepThreads) {
        int t0, t1;
        chunk_of(a.kv, s, t0, t1);
        if (t1 > t0) {
            L = min(L, max(live_len(a.kv, s, 0, false) - (t1 - t0), 0));
            first = min(first, s);
        }
    }
    L = __reduce_min_sync(0xffffffffu, L);
    first = __reduce_min_sync(0xffffffffu, first);
    if ((tid & 31) == 0) {
        least[tid >> 5] = L;
        firsts[tid >> 5] = first;
    }
    __syncthreads();
    for (int w = 0; w < kSharedPrepThreads / 32; ++w) {
        L = min(L, least[w]);
        first = min(first, firsts[w]);
    }
    L = L == INT_MAX ? 0 : min(L, max(a.shared[g], 0));  // (no tokens: nothing to do)
    for (int s = s0 + tid; s < s1; s += kSharedPrepThreads) a.start[s] = L;
    if (tid == 0) {
        a.cu[g] = token_of(s0);
        a.len[g] = L;
        a.row_of[g] = min(first, S - 1);
        if (g == a.n_groups - 1) a.cu[g + 1] = token_of(s1);
    }
    // sequences of no group have all slots for themselves
    if (g == 0)
        for (int s = tid; s < s0; s += kSharedPrepThreads) a.start[s] = 0;
    if (g == a.n_groups - 1)
        for (int s = s1 + tid; s < S; s += kSharedPrepThreads) a.start[s] = 0;
}

// What one of the two passes left: rows of whole units in row_o, row_ml ([n_tokens][hq][d]; parts of them behind one another where parts > 1); of the units
// that range boundaries cut the parts of every CTA, as join_parts_kernel finds them, and in row_ref which CTAs'.
struct SharedPass {
    const float* row_o;
    const float* row_ml;
    const int2* row_ref;  // null: nothing is cut
    const float* part_o;
    const float* part_ml;
    int parts, ranges, range_rows;  // ranges that units are cut into, rows that one leaves
};

struct SharedJoinArgs {
    PagedView kv;
    RowsView out;
    const int* cu;        // [n_groups + 1] tokens of the groups
    int n_groups, hq;
    float scale_log2;
    SharedPass pass[2];   // slots in common, own slots
};

constexpr int kSharedJoinThreads = 256;

// A row has 1, 2, 4 or 8 warps, as many as the grid has for it, and each of them every so many-th part.  Bound by latency: a few MB at most.
template <typename T, int D>
__global__ void __launch_bounds__(kSharedJoinThreads, 4) shared_join_kernel(const __grid_constant__ SharedJoinArgs a) {
    constexpr int LPR = D / 4, HALVES = 32 / LPR, WARPS = kSharedJoinThreads / 32;
    __shared__ PartSum sums[WARPS][LPR];
    grid_dep_wait();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, e = (lane % LPR) * 4;
    const long long n_rows = (long long)a.kv.n_tokens * a.hq;
    const int first = a.kv.cu ? a.kv.cu[0] : 0, end = a.kv.cu ? a.kv.cu[a.kv.n_seqs] : a.kv.n_tokens;  // (tokens of no sequence are left as they were)
    const int g0 = a.cu[0], g1 = a.cu[a.n_groups];
    int split = WARPS;  // warps of a row
    while (split > 1 && n_rows * split > (long long)gridDim.x * WARPS) split >>= 1;
    const int at_once = WARPS / split, part0 = (warp % split) * HALVES + lane / LPR, step = split * HALVES;
    for (long long row0 = (long long)blockIdx.x * at_once; row0 < n_rows; row0 += (long long)gridDim.x * at_once) {  // (the same trips for all warps)
        const long long row = row0 + warp / split;
        const int t = (int)(row / a.hq), h = (int)(row - (long long)t * a.hq);
        const bool mine = row < n_rows && t >= first && t < end;
        PartSum sum;
#pragma unroll
        for (int w = 0; w < 2; ++w) {  // the slots in common first
            const SharedPass& p = a.pass[w];
            if (!mine || (w == 0 && (t < g0 || t >= g1))) continue;  // (a sequence of no group)
            const int2 ref = p.row_ref ? p.row_ref[row] : make_int2(-1, 0);
            const PartRange r = part_range(ref.x, ref.y, p.ranges, p.range_rows);
            if (r.first >= 0) {
#pragma unroll 4
                for (int c = r.first + part0; c <= r.last; c += step) {
                    const size_t at = (size_t)(c * 2 + (c == r.first ? 1 : 0)) * p.range_rows + r.row;
                    sum.add(*reinterpret_cast<const float2*>(p.part_ml + at * 2), *reinterpret_cast<const float4*>(p.part_o + at * D + e), a.scale_log2);
                }
            } else {
#pragma unroll 4
                for (int s = part0; s < p.parts; s += step) {
                    const long long at = s * n_rows + row;
                    sum.add(*reinterpret_cast<const float2*>(p.row_ml + at * 2), *reinterpret_cast<const float4*>(p.row_o + at * D + e), a.scale_log2);
                }
            }
        }
        if (HALVES == 2) sum.add_lane(16, a.scale_log2);
        if (split > 1) {
            if (lane < LPR) sums[warp][lane] = sum;
            __syncthreads();
            if (warp % split == 0 && lane < LPR)
                for (int w = 1; w < split; ++w) {
                    const PartSum& s = sums[warp + w][lane];
                    sum.add(make_float2(s.M, s.L), s.o, a.scale_log2);
                }
        }
        if (mine && warp % split == 0 && lane < LPR) {
            const float inv = sum.L > 0.f ? 1.0f / sum.L : sum.L;  // nothing seen: 0; NaN stays NaN
            char* dst = a.out.p + ((long long)t * a.out.token_stride + (long long)h * a.out.head_stride + e) * (long long)sizeof(T);
            if (sizeof(T) == 4)
                *reinterpret_cast<float4*>(dst) = make_float4(sum.o.x * inv, sum.o.y * inv, sum.o.z * inv, sum.o.w * inv);
            else
                *reinterpret_cast<uint2*>(dst) = make_uint2(pack_bf16(sum.o.x * inv, sum.o.y * inv), pack_bf16(sum.o.z * inv, sum.o.w * inv));
        }
        if (split > 1) __syncthreads();
    }
}

}  // namespace lar
