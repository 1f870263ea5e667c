// Attention of sequences that have their first slots in common, in groups: the two small kernels around those of the chunk attention.
//
//   softmax over the slots 0 .. last(t) = the softmax over the L slots in common, once for all tokens of a group, joined with that over L .. last(t):
//       m = max(m1, m2),  out = (O1 e^(m1 - m) + O2 e^(m2 - m)) / (l1 e^(m1 - m) + l2 e^(m2 - m))       (O, l: sums without the division)
//
// The slots in common are one unit per (group, KV head), whose rows are all tokens of the group: they are read once per 256 rows and not once
// per sequence.  Every token of a group sees all of them (L is cut to what the shortest cache of the group held before its chunk), so that
// pass needs no mask.
#pragma once
#include "join_parts.cuh"
#include "paged_attn.cuh"

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
    __shared__ int least[kSharedPrepThreads / 32];
    grid_dep_launch();
    const int tid = threadIdx.x, g = blockIdx.x, S = a.kv.n_seqs;
    const int s0 = min(max(a.groups[g], 0), S), s1 = min(max(a.groups[g + 1], s0), S);
    auto token_of = [&](int s) {  // the first token of sequence s; S: behind the last one's
        int t0, t1;
        chunk_of(a.kv, min(s, S - 1), t0, t1);
        return s < S ? t0 : t1;
    };
    int L = INT_MAX;
    for (int s = s0 + tid; s < s1; s += kSharedPrepThreads) {
        int t0, t1;
        chunk_of(a.kv, s, t0, t1);
        if (t1 > t0) L = min(L, max(live_len(a.kv, s, 0, false) - (t1 - t0), 0));
    }
    L = __reduce_min_sync(0xffffffffu, L);
    if ((tid & 31) == 0) least[tid >> 5] = L;
    __syncthreads();
    for (int w = 0; w < kSharedPrepThreads / 32; ++w) L = min(L, least[w]);
    L = L == INT_MAX ? 0 : min(L, max(a.shared[g], 0));  // (no tokens: nothing to do)
    for (int s = s0 + tid; s < s1; s += kSharedPrepThreads) a.start[s] = L;
    if (tid == 0) {
        a.cu[g] = token_of(s0);
        a.len[g] = L;
        a.row_of[g] = min(s0, S - 1);
        if (g == a.n_groups - 1) a.cu[g + 1] = token_of(s1);
    }
    // sequences of no group have all slots for themselves
    if (g == 0)
        for (int s = tid; s < s0; s += kSharedPrepThreads) a.start[s] = 0;
    if (g == a.n_groups - 1)
        for (int s = s1 + tid; s < S; s += kSharedPrepThreads) a.start[s] = 0;
}

// What one of the two passes left: rows of whole units in row_o, row_ml ([n_tokens][hq][d]; parts of them behind one another where parts > 1); of the
// units that range boundaries cut the parts, as join_parts_kernel finds them.
struct SharedPass {
    const float* row_o;
    const float* row_ml;
    const int4* records;  // null: nothing is cut
    const float* part_o;
    const float* part_ml;
    int parts, ranges, nt, tq, rows_cap;
};

struct SharedJoinArgs {
    PagedView kv;
    RowsView out;
    const int* cu;        // [n_groups + 1] tokens of the groups
    int n_groups, hq, group;
    float scale_log2;
    SharedPass pass[2];   // slots in common, own slots
};

constexpr int kSharedJoinThreads = 256;

// A row per warp, the slots in common first.  Bound by latency: a few MB at most.
template <typename T, int D>
__global__ void __launch_bounds__(kSharedJoinThreads) shared_join_kernel(const __grid_constant__ SharedJoinArgs a) {
    constexpr int LPR = D / 4, HALVES = 32 / LPR;
    extern __shared__ int4 rec[];  // of both passes
    grid_dep_wait();
    for (int i = threadIdx.x; i < a.pass[0].ranges + a.pass[1].ranges; i += kSharedJoinThreads)
        rec[i] = i < a.pass[0].ranges ? a.pass[0].records[i] : a.pass[1].records[i - a.pass[0].ranges];
    const int lane = threadIdx.x & 31, e = (lane % LPR) * 4;
    const long long n_rows = (long long)a.kv.n_tokens * a.hq;
    const int first = a.kv.cu ? a.kv.cu[0] : 0, end = a.kv.cu ? a.kv.cu[a.kv.n_seqs] : a.kv.n_tokens;  // (tokens of no sequence are left as they were)
    const int g0 = a.cu[0], g1 = a.cu[a.n_groups];
    __syncthreads();
    for (long long row = (long long)blockIdx.x * (kSharedJoinThreads / 32) + (threadIdx.x >> 5); row < n_rows; row += (long long)gridDim.x * (kSharedJoinThreads / 32)) {
        const int t = (int)(row / a.hq), h = (int)(row - (long long)t * a.hq), kvh = h / a.group;
        if (t < first || t >= end) continue;
        PartSum sum;
#pragma unroll
        for (int w = 0; w < 2; ++w) {
            const SharedPass& p = a.pass[w];
            if (w == 0 && (t < g0 || t >= g1)) continue;  // a sequence of no group
            const int4* r = rec + (w ? a.pass[0].ranges : 0);
            int range = -1;  // the range that the row's unit begins in, if it is cut
            for (int c = lane; c < p.ranges; c += 32) {
                const int4 u = r[c];
                if (u.z == kvh && t >= u.x && t < u.x + u.y) range = c;
            }
            range = __reduce_max_sync(0xffffffffu, range);
            if (range >= 0) {
                const int4 u = r[range];
                const int tu = t - u.x, tile = p.nt == 2 && tu >= p.tq ? 1 : 0, last = min(u.w, p.ranges - 1);
                const int tile_row = (tu - tile * p.tq) * a.group + h - kvh * a.group;
#pragma unroll 8
                for (int c = range + lane / LPR; c <= last; c += HALVES) {
                    const size_t at = ((size_t)(c * 2 + (c == range ? 1 : 0)) * p.nt + tile) * p.rows_cap + tile_row;
                    sum.add(*reinterpret_cast<const float2*>(p.part_ml + at * 2), *reinterpret_cast<const float4*>(p.part_o + at * D + e), a.scale_log2);
                }
            } else {
#pragma unroll 8
                for (int s = lane / LPR; s < p.parts; s += HALVES) {
                    const long long at = s * n_rows + row;
                    sum.add(*reinterpret_cast<const float2*>(p.row_ml + at * 2), *reinterpret_cast<const float4*>(p.row_o + at * D + e), a.scale_log2);
                }
            }
        }
        if (HALVES == 2) sum.add_lane(16, a.scale_log2);
        if (lane >= LPR) continue;
        const float inv = sum.L > 0.f ? 1.0f / sum.L : sum.L;  // nothing seen: 0; NaN stays NaN
        char* dst = a.out.p + ((long long)t * a.out.token_stride + (long long)h * a.out.head_stride + e) * (long long)sizeof(T);
        if (sizeof(T) == 4)
            *reinterpret_cast<float4*>(dst) = make_float4(sum.o.x * inv, sum.o.y * inv, sum.o.z * inv, sum.o.w * inv);
        else
            *reinterpret_cast<uint2*>(dst) = make_uint2(pack_bf16(sum.o.x * inv, sum.o.y * inv), pack_bf16(sum.o.z * inv, sum.o.w * inv));
    }
}

}  // namespace lar
