// The join behind kernels whose units are cut by the boundaries of equal ranges: a unit's parts (O, m, l) lie in the workspace, one for each CTA that
// had some of its slots, and the record of the CTA that began it says which.
//
// Latency is all there is to it (a few KB to a few MB), so every load is one of many under way: a CTA has some rows of the unit that its record names (none:
// nothing to do), each row is a group of 1, 2, 4 or 8 warps', as few as keep all of them busy, and each warp has every so many-th part.
#pragma once
#include "paged_attn_tc.cuh"

namespace lar {

constexpr int kJoinThreads = 256, kJoinWarps = 8;

// A sum of parts.
struct PartSum {
    float M = -INFINITY, L = 0.f;
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
    __device__ __forceinline__ void add(float2 ml, float4 p, float scale_log2) {
        const float mn = fmaxf(M, ml.x), ref = softmax_ref(mn);
        const float f0 = ex2_approx((M - ref) * scale_log2), f = ex2_approx((ml.x - ref) * scale_log2);
        M = mn;
        L = fmaf(ml.y, f, L * f0);
        o.x = fmaf(p.x, f, o.x * f0);
        o.y = fmaf(p.y, f, o.y * f0);
        o.z = fmaf(p.z, f, o.z * f0);
        o.w = fmaf(p.w, f, o.w * f0);
    }
    // with another lane's, the lower lane's first
    __device__ __forceinline__ void add_lane(int mask, float scale_log2) {
        float2 ml;
        float4 p;
        ml.x = __shfl_xor_sync(0xffffffffu, M, mask);
        ml.y = __shfl_xor_sync(0xffffffffu, L, mask);
        p.x = __shfl_xor_sync(0xffffffffu, o.x, mask);
        p.y = __shfl_xor_sync(0xffffffffu, o.y, mask);
        p.z = __shfl_xor_sync(0xffffffffu, o.z, mask);
        p.w = __shfl_xor_sync(0xffffffffu, o.w, mask);
        add(ml, p, scale_log2);
    }
};

// CTAs of a range's unit: few enough rows each that warps share them.
inline unsigned join_ctas(int unit_rows) { return unit_rows <= 2 ? 1u : unit_rows <= 64 ? (unsigned)(unit_rows + 1) / 2 : 32u; }

// A launch of (ranges, join_ctas) CTAs; rows of output type T; rows_cap and records as the kernel before left them (TcArgs).
// 3 us behind the attention of one token over 16 x 4288 slots.
template <typename T, int D>
__global__ void __launch_bounds__(kJoinThreads) join_parts_kernel(const __grid_constant__ TcArgs ta) {
    constexpr int LPR = D / 4, HALVES = 32 / LPR;  // lanes of a row of a part, parts that a warp reads at a time
    __shared__ PartSum sums[kJoinWarps][LPR];
    const PagedAttnArgs& a = ta.a;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, first = blockIdx.x;
    grid_dep_wait();
    const int4 u = ta.records[first];  // first token, tokens, head, last range
    const int unit_rows = u.y * a.group, per = (unit_rows + (int)gridDim.y - 1) / (int)gridDim.y;
    const int begin = blockIdx.y * per, end = min(begin + per, unit_rows), last = min(u.w, (int)gridDim.x - 1);
    int split = kJoinWarps;  // warps of a row
    while (split > 1 && per * split > kJoinWarps) split >>= 1;
    const int at_once = kJoinWarps / split, mine = warp / split, part0 = (warp % split) * HALVES + lane / LPR, e = (lane % LPR) * 4;
    for (int row0 = begin; row0 < end; row0 += at_once) {  // (the same trips for all warps)
        const int unit_row = row0 + mine;
        PartSum sum;
        if (unit_row < end) {
#pragma unroll 8
            for (int c = first + part0; c <= last; c += split * HALVES) {
                const size_t at = (size_t)(c * 2 + (c == first ? 1 : 0)) * ta.rows_cap + unit_row;
                sum.add(*reinterpret_cast<const float2*>(a.part_ml + at * 2), *reinterpret_cast<const float4*>(a.part_o + at * D + e), a.scale_log2);
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
        if (unit_row < end && warp % split == 0 && lane < LPR) {
            const float inv = sum.L > 0.f ? 1.0f / sum.L : sum.L;  // nothing seen: 0; NaN stays NaN
            const int t = unit_row / a.group, h = u.z * a.group + unit_row - t * a.group;
            char* dst = a.out.p + ((long long)(u.x + t) * a.out.token_stride + (long long)h * a.out.head_stride + e) * (long long)sizeof(T);
            if (sizeof(T) == 4)
                *reinterpret_cast<float4*>(dst) = make_float4(sum.o.x * inv, sum.o.y * inv, sum.o.z * inv, sum.o.w * inv);
            else
                *reinterpret_cast<uint2*>(dst) = make_uint2(pack_bf16(sum.o.x * inv, sum.o.y * inv), pack_bf16(sum.o.z * inv, sum.o.w * inv));
        }
        if (split > 1) __syncthreads();
    }
}

}  // namespace lar
