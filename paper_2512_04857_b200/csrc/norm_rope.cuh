// Norms of q and k per head with the rotary embedding in the same pass, on rows in memory and on the way into a paged cache (of the rows'
// type, or of 8 bits).
//
//   rms:    y = x / sqrt(mean(x^2) + eps) * w  (+ bias)        layer:  y = (x - mean(x)) / sqrt(mean((x - mean)^2) + eps) * w  (+ bias)
//   then the pairs of y are turned as in rope_rows.cuh, and the result is rounded once, to the storage type or to 8 bits.
//
// Bound: HBM bytes (each row once in, once out; about ten operations per element).  The work is dealt out as in rope_rows.cuh: a CTA has
// one or two tokens, a thread 16 bytes of each half of a row (or 32 bytes side by side where pairs interleave).  The D / 16 (bf16) or D / 8
// (fp32) threads of a row are neighbours in a warp, so that the row's sums are three or four shuffles, taken with the row in registers: the
// mean first and the squares of what is left after it, not the difference of two large sums.  Weights come through L1.
#pragma once
#include "paged_q8.cuh"
#include "rope_rows.cuh"

namespace lar {

struct HeadNormView {
    const char* weight;  // null: ones
    const char* bias;    // null: none
    long long head_stride;  // elements; 0: one row for all heads
    float eps;
    int on, layer, bf16;
};

struct NormRopeArgs {
    RopeRowsArgs r;
    HeadNormView norm[2];  // of q, of k
    Q8View q8;             // DEST 2 only
    int any_norm, any_layer;
};

// E parameters of a norm as fp32 (16 or 8 bytes)
template <int E>
__device__ __forceinline__ void norm_params(const char* p, long long at, int bf16, float (&w)[E]) {
    if (!bf16) {
#pragma unroll
        for (int i = 0; i < E; i += 4) {
            const float4 v = __ldg(reinterpret_cast<const float4*>(reinterpret_cast<const float*>(p) + at + i));
            w[i] = v.x; w[i + 1] = v.y; w[i + 2] = v.z; w[i + 3] = v.w;
        }
    } else if (E == 8) {
        const uint4 v = __ldg(reinterpret_cast<const uint4*>(p + at * 2));
        float f[8];
        Elt<__nv_bfloat16>::unpack(v, f);
#pragma unroll
        for (int i = 0; i < E; ++i) w[i] = f[i];
    } else {
        const uint2 v = __ldg(reinterpret_cast<const uint2*>(p + at * 2));
        w[0] = __uint_as_float(v.x << 16); w[1] = __uint_as_float(v.x & 0xffff0000u);
        w[2] = __uint_as_float(v.y << 16); w[3] = __uint_as_float(v.y & 0xffff0000u);
    }
}

// DEST: 0 rows, 1 pages of the rows' type, 2 pages of 8 bits
template <typename T, int D, bool INTER, int DEST>
__global__ void __launch_bounds__(kRopeThreads) norm_rope_kernel(const __grid_constant__ NormRopeArgs na) {
    constexpr int E = Elt<T>::kPerChunk;  // elements of a 16-byte chunk
    constexpr int IPR = D / (2 * E);      // threads of a row
    constexpr int HP = D / 2;
    const RopeRowsArgs& a = na.r;
    extern __shared__ __align__(16) float cs[];  // [tokens_per_cta][cos HP | sin HP], then the tokens' slots and sequences
    int* slot_of = reinterpret_cast<int*>(cs + a.tokens_per_cta * D);
    int* seq_of = slot_of + a.tokens_per_cta;

    const int tid = threadIdx.x;
    const int t0 = blockIdx.x * a.tokens_per_cta;
    const int nt = min(a.tokens_per_cta, a.n_tokens - t0);
    const int row0 = blockIdx.y * a.rows_per_slice;
    const int nr = min(a.rows_per_slice, a.n_rows - row0);
    const int n_items = nt * a.rows_per_slice * IPR;
    const int c = tid & (IPR - 1);
    const int o_lo = INTER ? 2 * c * E : c * E, o_hi = INTER ? (2 * c + 1) * E : HP + c * E;
    auto row_sum = [](float v) {
#pragma unroll
        for (int o = 1; o < IPR; o <<= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
        return v;
    };

    bool ready = false;
    for (int base = 0; base < n_items; base += kRopeThreads * kRopeBatch) {
        uint4 lo[kRopeBatch], hi[kRopeBatch];
        int tok[kRopeBatch], row[kRopeBatch];
#pragma unroll
        for (int b = 0; b < kRopeBatch; ++b) {
            const int item = base + b * kRopeThreads + tid;
            const int r = item / IPR;
            const int tl = a.rows_magic ? (int)__umulhi((unsigned)r, a.rows_magic) : r;
            const int rl = r - tl * a.rows_per_slice;
            tok[b] = item < n_items && rl < nr ? tl : -1;
            row[b] = row0 + rl;
            lo[b] = hi[b] = make_uint4(0, 0, 0, 0);
            if (tok[b] >= 0) {
                const int which = row[b] < a.heads[0] ? 0 : row[b] < a.heads[0] + a.heads[1] ? 1 : 2;
                const int head = row[b] - (which > 0 ? a.heads[0] : 0) - (which > 1 ? a.heads[1] : 0);
                const RowsView& s = a.src[which];
                const T* p = reinterpret_cast<const T*>(s.p) + (long long)(t0 + tl) * s.token_stride + head * s.head_stride;
                lo[b] = *reinterpret_cast<const uint4*>(p + o_lo);
                hi[b] = *reinterpret_cast<const uint4*>(p + o_hi);
            }
        }
        if (!ready) {  // sines, cosines and slots of the CTA's tokens, while the first rows are on the way
            ready = true;
            if (a.pos) {
                const int i = tid & (HP - 1);
                const double f = a.f.turns[i];
                const int* p = a.pos + a.f.axis[i] * a.pos_axis_stride + t0;
                for (int tl = tid / HP; tl < nt; tl += kRopeThreads / HP) {
                    const float2 v = cos_sin_of(f, p[tl]);
                    cs[tl * D + i] = v.x;
                    cs[tl * D + HP + i] = v.y;
                }
            }
            if (DEST) find_slots<kRopeThreads>(a.kv, a.state ? a.base_len : -1, t0, nt, slot_of, seq_of);
            __syncthreads();
        }
#pragma unroll
        for (int b = 0; b < kRopeBatch; ++b) {
            // (all lanes stay together to the stores: the row sums are warp-wide)
            const bool valid = tok[b] >= 0;
            const int which = row[b] < a.heads[0] ? 0 : row[b] < a.heads[0] + a.heads[1] ? 1 : 2;
            const int head = row[b] - (which > 0 ? a.heads[0] : 0) - (which > 1 ? a.heads[1] : 0);
            float x[2 * E];  // the low chunk, then the high one
            {
                float u[E], v[E];
                Elt<T>::unpack(lo[b], u);
                Elt<T>::unpack(hi[b], v);
#pragma unroll
                for (int i = 0; i < E; ++i) {
                    x[i] = u[i];
                    x[E + i] = v[i];
                }
            }
            if (na.any_norm) {
                const HeadNormView& h = na.norm[which == 0 ? 0 : 1];
                const bool on = valid && which < 2 && h.on;
                const bool layer = h.layer != 0;
                float mean = 0.f, up = 1.f, ss = 0.f;
                for (;;) {
                    float y = 0.f;
                    if (na.any_layer) {
#pragma unroll
                        for (int i = 0; i < 2 * E; ++i) y += x[i];
                        y = row_sum(y);
                        mean = layer ? y * (1.0f / D) : 0.f;
                    }
                    y = 0.f;
#pragma unroll
                    for (int i = 0; i < 2 * E; ++i) {
                        const float z = x[i] - mean;
                        y = fmaf(z, z, y);
                    }
                    ss = row_sum(y);
                    // squares beyond fp32: once more with the row scaled down (eps is nothing beside such a row)
                    const bool again = on && up == 1.f && !(ss <= 3.4e38f);
                    if (!__any_sync(0xffffffffu, again)) break;
                    if (again) {
                        up = 0x1p-80f;
#pragma unroll
                        for (int i = 0; i < 2 * E; ++i) x[i] *= up;
                    }
                }
                if (on) {
                    const float f = rsqrtf(fmaf(ss, 1.0f / D, h.eps * up * up));
#pragma unroll
                    for (int i = 0; i < 2 * E; ++i) x[i] = (x[i] - mean) * f;
                    const long long at = head * h.head_stride;
                    float w[E];
                    if (h.weight) {
                        norm_params<E>(h.weight, at + o_lo, h.bf16, w);
#pragma unroll
                        for (int i = 0; i < E; ++i) x[i] *= w[i];
                        norm_params<E>(h.weight, at + o_hi, h.bf16, w);
#pragma unroll
                        for (int i = 0; i < E; ++i) x[E + i] *= w[i];
                    }
                    if (h.bias) {
                        norm_params<E>(h.bias, at + o_lo, h.bf16, w);
#pragma unroll
                        for (int i = 0; i < E; ++i) x[i] += w[i];
                        norm_params<E>(h.bias, at + o_hi, h.bf16, w);
#pragma unroll
                        for (int i = 0; i < E; ++i) x[E + i] += w[i];
                    }
                }
            }
            if (a.pos && valid && which < 2) {
                const float* cosv = cs + tok[b] * D + c * E;
                const float* sinv = cosv + HP;
#pragma unroll
                for (int i = 0; i < E; ++i) {  // pair i of the thread: (2 i, 2 i + 1) where pairs interleave, else (i, E + i)
                    float& p = INTER ? x[2 * i] : x[i];
                    float& q = INTER ? x[2 * i + 1] : x[E + i];
                    const float2 u = turn_pair(p, q, cosv[i], sinv[i]);
                    p = u.x;
                    q = u.y;
                }
            }
            int byte = 0;
            if (DEST == 2) {
                unsigned largest = 0;
#pragma unroll
                for (int i = 0; i < 2 * E; ++i) largest = max(largest, __float_as_uint(x[i]) & 0x7fffffffu);
#pragma unroll
                for (int o = 1; o < IPR; o <<= 1) largest = max(largest, __shfl_xor_sync(0xffffffffu, largest, o));
                byte = q8_byte(largest);
            }
            if (!valid || (DEST && (which > 0 ? slot_of[tok[b]] : seq_of[tok[b]]) < 0)) continue;
            if (DEST && which > 0) {
                const int slot = slot_of[tok[b]], in_page = slot & (a.kv.page_tokens - 1);
                const int page = a.kv.table[seq_of[tok[b]] * a.kv.table_seq_stride + head * a.kv.table_head_stride + (slot >> a.kv.page_shift)];
                if (page < 0 || page >= a.kv.n_pages) {
                    if (c == 0) paged_report(a.kv, kStPage);
                    continue;
                }
                const long long at = page * a.kv.page_stride + in_page * a.kv.row_stride + head * a.kv.head_stride;
                char* pool = which == 1 ? a.kv.k_pool : a.kv.v_pool;
                if (DEST == 2) {
                    unsigned codes[E / 2];
#pragma unroll
                    for (int i = 0; i < E / 2; ++i) codes[i] = q8_codes4(x + 4 * i, byte);
                    char* p = pool + at;
                    if (INTER && E == 8) {
                        *reinterpret_cast<uint4*>(p + o_lo) = make_uint4(codes[0], codes[1], codes[E / 2 - 2], codes[E / 2 - 1]);
                    } else if (INTER) {
                        *reinterpret_cast<uint2*>(p + o_lo) = make_uint2(codes[0], codes[E / 2 - 1]);
                    } else if (E == 8) {
                        *reinterpret_cast<uint2*>(p + o_lo) = make_uint2(codes[0], codes[1]);
                        *reinterpret_cast<uint2*>(p + o_hi) = make_uint2(codes[E / 2 - 2], codes[E / 2 - 1]);
                    } else {
                        *reinterpret_cast<unsigned*>(p + o_lo) = codes[0];
                        *reinterpret_cast<unsigned*>(p + o_hi) = codes[E / 2 - 1];
                    }
                    if (c == 0) (which == 1 ? na.q8.k_scale : na.q8.v_scale)[page * na.q8.page_stride + head * na.q8.head_stride + in_page] = (unsigned char)byte;
                    continue;
                }
                float u[E], v[E];
#pragma unroll
                for (int i = 0; i < E; ++i) {
                    u[i] = x[i];
                    v[i] = x[E + i];
                }
                T* dst = reinterpret_cast<T*>(pool) + at;
                // (values are copied as they are: a pass through fp32 could touch the bits of a NaN)
                *reinterpret_cast<uint4*>(dst + o_lo) = which == 2 ? lo[b] : PackRow<T>::pack(u);
                *reinterpret_cast<uint4*>(dst + o_hi) = which == 2 ? hi[b] : PackRow<T>::pack(v);
                continue;
            }
            float u[E], v[E];
#pragma unroll
            for (int i = 0; i < E; ++i) {
                u[i] = x[i];
                v[i] = x[E + i];
            }
            const RowsView& d = a.dst[which];
            T* dst = reinterpret_cast<T*>(d.p) + (long long)(t0 + tok[b]) * d.token_stride + head * d.head_stride;
            *reinterpret_cast<uint4*>(dst + o_lo) = PackRow<T>::pack(u);
            *reinterpret_cast<uint4*>(dst + o_hi) = PackRow<T>::pack(v);
        }
    }
    if (DEST == 1 && a.state) {
        // the library's own cache: the index map's entries of the tokens; the last one sets the unit's length
        for (int i = tid; i < nt * a.kv.n_kv_heads && blockIdx.y == 0; i += kRopeThreads) {
            const int tl = i / a.kv.n_kv_heads, head = i - tl * a.kv.n_kv_heads;
            if (slot_of[tl] < 0) continue;
            const int unit = seq_of[tl] * a.kv.n_kv_heads + head;
            a.index_map[(size_t)unit * a.cap_pad + slot_of[tl]] = slot_of[tl];
            if (slot_of[tl] == a.base_len + a.kv.chunk - 1) {
                UnitState ns;
                ns.len = slot_of[tl] + 1;
                ns.n_tok = 0;
                a.state[unit] = ns;
            }
        }
    }
}

}  // namespace lar
