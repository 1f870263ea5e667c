// The 8-bit paged cache: what a row is, how it is written and read back.
//
// A row x of head_dim elements is held as e4m3 codes c and one byte b:  x = c 2^(b - 127),  b - 127 = k the smallest power for which no
// element exceeds 448 2^k (448 is e4m3's largest number), at least -117.  A power of two costs no accuracy (the codes have an exponent of
// their own: 4 significant bits down to 2^(k - 6), which is 2^-13.8 to 2^-14.8 of the row's largest element, absolute steps of 2^(k - 9) below), needs no
// division, and makes every value exact in bf16 and fp32, so that reading back loses nothing.  A row with an element that is not finite has
// b = 255 and codes of zero: it reads as NaN (0 times infinity), all of it.
#pragma once
#include <cuda_fp8.h>

#include "paged.cuh"
#include "rope_rows.cuh"  // RowsView, PackRow

namespace lar {

struct Q8View {
    unsigned char* k_scale;
    unsigned char* v_scale;
    long long page_stride, head_stride;  // bytes between pages and heads; the bytes of a page's slots lie side by side
};

constexpr int kQ8MinByte = 10, kQ8MaxByte = 247, kQ8NaN = 255;  // 2^-117 .. 2^120

// The scale byte of a row from the largest of its elements' magnitudes, as bits (NaN above infinity above all others).
__device__ __forceinline__ int q8_byte(unsigned largest) {
    if (largest >= 0x7f800000u) return kQ8NaN;
    const int e = (int)(largest >> 23) - ((largest & 0x7fffffu) <= 0x600000u ? 8 : 7);  // 1.75 * 2^8 = 448
    return largest == 0 ? 127 : max(e, kQ8MinByte);
}
__device__ __forceinline__ float q8_scale(int byte) { return __uint_as_float((unsigned)byte << 23); }             // 2^(byte - 127); 255: infinity
__device__ __forceinline__ float q8_inverse(int byte) { return __uint_as_float((unsigned)max(254 - byte, 0) << 23); }  // (255: zero)

// Four codes of scaled elements, the first in the lowest byte.
__device__ __forceinline__ unsigned q8_codes4(const float* x, int byte) {
    float y[4];
    const float f = q8_inverse(byte);
#pragma unroll
    for (int i = 0; i < 4; ++i) y[i] = x[i] * f;
    if (byte >= kQ8MaxByte) {  // 256 * 2^120 is beyond fp32; a row that is not finite has codes of zero
#pragma unroll
        for (int i = 0; i < 4; ++i) y[i] = byte == kQ8NaN ? 0.f : fminf(fmaxf(y[i], -240.f), 240.f);
    }
    const unsigned lo = __nv_cvt_float2_to_fp8x2(make_float2(y[0], y[1]), __NV_SATFINITE, __NV_E4M3);
    const unsigned hi = __nv_cvt_float2_to_fp8x2(make_float2(y[2], y[3]), __NV_SATFINITE, __NV_E4M3);
    return lo | (hi << 16);
}
// The values of four codes, exact.
__device__ __forceinline__ void q8_values4(unsigned codes, float scale, float* x) {
    const __half2 a(__half2_raw(__nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)(codes & 0xffffu), __NV_E4M3)));
    const __half2 b(__half2_raw(__nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)(codes >> 16), __NV_E4M3)));
    const float2 u = __half22float2(a), v = __half22float2(b);
    x[0] = u.x * scale;
    x[1] = u.y * scale;
    x[2] = v.x * scale;
    x[3] = v.y * scale;
}

// Slot and sequence of nt tokens from t0 on, by THREADS threads: seq_of -1 for a token that belongs to no sequence; slot_of -1 also
// for one whose slot the table does not hold (recorded).
template <int THREADS>
__device__ __forceinline__ void find_slots(const PagedView& kv, int t0, int nt, int* slot_of, int* seq_of) {
    const int tid = threadIdx.x;
    int s = 0;
    if (kv.cu) {  // sequence of a token: the number of sequences that end at or before it
        for (int tl = 0; tl < nt; ++tl) {
            int n = 0;
            for (int j = 0; j < kv.n_seqs; j += THREADS) n += __syncthreads_count(j + tid < kv.n_seqs && kv.cu[j + tid + 1] <= t0 + tl);
            if (tid == tl) s = n;
        }
    } else {
        s = (t0 + tid) / kv.chunk;
    }
    if (tid < nt) {
        const int t = t0 + tid;
        int slot = -1, b0 = 0, b1 = 0;
        if (s < kv.n_seqs) chunk_of(kv, s, b0, b1);
        if (t < b0 || t >= b1) {
            s = -1;
        } else {
            slot = kv.lens[s * kv.lens_stride] - (b1 - t);
            if (slot < 0 || slot >= (kv.table_cols << kv.page_shift)) {
                paged_report(kv, kStPage);
                slot = -1;
            }
        }
        slot_of[tid] = slot;
        seq_of[tid] = s;
    }
}

struct Q8ReadArgs {
    PagedView kv;
    Q8View q8;
    RowsView out[2];  // k, v rows [tokens][heads][d]
    int tokens_per_cta, rows;  // rows: 2 * heads
};

constexpr int kQ8ReadThreads = 128;

// The newest entries of every sequence as rows.  A thread takes 16 codes; bound by the bytes (1 in, 2 or 4 out for each element; 24 prompts of up to 2048
// tokens, 8 heads of 128, to bf16: 151 MB in 32 us).  A slot outside
// the table or a page outside the pool reads as zeros.
template <typename T, int D>
__global__ void __launch_bounds__(kQ8ReadThreads) q8_read_kernel(const __grid_constant__ Q8ReadArgs a) {
    constexpr int IPR = D / 16, E = Elt<T>::kPerChunk, BATCH = 4;
    __shared__ int slot_of[kQ8ReadThreads], seq_of[kQ8ReadThreads];
    const int tid = threadIdx.x, t0 = blockIdx.x * a.tokens_per_cta, nt = min(a.tokens_per_cta, a.kv.n_tokens - t0);
    find_slots<kQ8ReadThreads>(a.kv, t0, nt, slot_of, seq_of);
    __syncthreads();
    const int c = tid & (IPR - 1), heads = a.kv.n_kv_heads, n_items = nt * a.rows * IPR;
    for (int base = 0; base < n_items; base += kQ8ReadThreads * BATCH) {
        uint4 codes[BATCH];
        int byte[BATCH];
#pragma unroll
        for (int b = 0; b < BATCH; ++b) {
            const int r = (base + b * kQ8ReadThreads + tid) / IPR, tl = r / a.rows, row = r - tl * a.rows;
            codes[b] = make_uint4(0, 0, 0, 0);
            byte[b] = -1;
            if (tl >= nt || seq_of[tl] < 0) continue;
            const int is_v = row >= heads, head = row - (is_v ? heads : 0), slot = slot_of[tl];
            byte[b] = 127;
            if (slot < 0) continue;
            const int page = a.kv.table[seq_of[tl] * a.kv.table_seq_stride + head * a.kv.table_head_stride + (slot >> a.kv.page_shift)];
            if (page < 0 || page >= a.kv.n_pages) {
                if (c == 0) paged_report(a.kv, kStPage);
                continue;
            }
            const int in_page = slot & (a.kv.page_tokens - 1);
            const char* pool = is_v ? a.kv.v_pool : a.kv.k_pool;
            codes[b] = *reinterpret_cast<const uint4*>(pool + page * a.kv.page_stride + in_page * a.kv.row_stride + head * a.kv.head_stride + c * 16);
            byte[b] = (is_v ? a.q8.v_scale : a.q8.k_scale)[page * a.q8.page_stride + head * a.q8.head_stride + in_page];
        }
#pragma unroll
        for (int b = 0; b < BATCH; ++b) {
            if (byte[b] < 0) continue;
            const int r = (base + b * kQ8ReadThreads + tid) / IPR, tl = r / a.rows, row = r - tl * a.rows;
            const int is_v = row >= heads, head = row - (is_v ? heads : 0);
            const RowsView& o = a.out[is_v];
            T* dst = reinterpret_cast<T*>(o.p) + (long long)(t0 + tl) * o.token_stride + head * o.head_stride + c * 16;
            const float scale = q8_scale(byte[b]);
            float x[16];
            q8_values4(codes[b].x, scale, x);
            q8_values4(codes[b].y, scale, x + 4);
            q8_values4(codes[b].z, scale, x + 8);
            q8_values4(codes[b].w, scale, x + 12);
#pragma unroll
            for (int i = 0; i < 16; i += E) {
                float part[E];
#pragma unroll
                for (int e = 0; e < E; ++e) part[e] = x[i + e];
                *reinterpret_cast<uint4*>(dst + i) = PackRow<T>::pack(part);
            }
        }
    }
}

}  // namespace lar
