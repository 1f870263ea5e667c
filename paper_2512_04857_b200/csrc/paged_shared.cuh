// Attention of sequences that have their first slots in common, in groups: the two small kernels around those of the chunk attention.
//
//   softmax over the slots 0 .. last(t) = the softmax over the L slots in common, once for all tokens of a group, joined with that over L .. last(t):
//       m = max(m1, m2),  out = (O1 e^(m1 - m) + O2 e^(m2 - m)) / (l1 e^(m1 - m) + l2 e^(m2 - m))       (O, l: sums without the division)
//
// The slots in common are one unit per (group, KV head), whose rows are all tokens of the group: they are read once per 256 rows and not once
// per sequence.  Every token of a group sees all of them (L is cut to what the shortest cache of the group held before its chunk), so that
// pass needs no mask.
#pragma once
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

struct SharedJoinArgs {
    PagedView kv;
    RowsView out;
    const int* cu;             // [n_groups + 1] tokens of the groups
    int n_groups, hq;
    float scale_log2;
    const float* o[2];         // slots in common, own slots: parts[i] times [n_tokens][hq][d]
    const float* ml[2];
    int parts[2];
};

// Four elements of a row per thread.
template <typename T, int D>
__global__ void __launch_bounds__(256) shared_join_kernel(const __grid_constant__ SharedJoinArgs a) {
    const long long i = (long long)blockIdx.x * 256 + threadIdx.x, n_rows = (long long)a.kv.n_tokens * a.hq, row = i / (D / 4);
    if (row >= n_rows) return;
    const int e = (int)(i % (D / 4)) * 4, t = (int)(row / a.hq), h = (int)(row - (long long)t * a.hq);
    if (a.kv.cu && (t < a.kv.cu[0] || t >= a.kv.cu[a.kv.n_seqs])) return;  // no sequence's token: left as it was
    const bool grouped = t >= a.cu[0] && t < a.cu[a.n_groups];
    float M = -INFINITY, L = 0.f;
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int w = 0; w < 2; ++w) {
        if (w == 0 && !grouped) continue;
#pragma unroll 4
        for (int s = 0; s < a.parts[w]; ++s) {
            const long long at = s * n_rows + row;
            const float2 ml = *reinterpret_cast<const float2*>(a.ml[w] + at * 2);
            const float4 p = *reinterpret_cast<const float4*>(a.o[w] + at * D + e);
            const float mn = fmaxf(M, ml.x), ref = softmax_ref(mn);
            const float f0 = exp2f((M - ref) * a.scale_log2), f = exp2f((ml.x - ref) * a.scale_log2);
            M = mn;
            L = fmaf(ml.y, f, L * f0);
            o.x = fmaf(p.x, f, o.x * f0);
            o.y = fmaf(p.y, f, o.y * f0);
            o.z = fmaf(p.z, f, o.z * f0);
            o.w = fmaf(p.w, f, o.w * f0);
        }
    }
    const float inv = L > 0.f ? 1.0f / L : L;  // nothing seen: 0; NaN stays NaN
    const float v[4] = {o.x * inv, o.y * inv, o.z * inv, o.w * inv};
    T* dst = reinterpret_cast<T*>(a.out.p) + (long long)t * a.out.token_stride + (long long)h * a.out.head_stride + e;
    if (sizeof(T) == 4)
        *reinterpret_cast<float4*>(dst) = make_float4(v[0], v[1], v[2], v[3]);
    else
        *reinterpret_cast<uint2*>(dst) = make_uint2(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]));
}

}  // namespace lar
