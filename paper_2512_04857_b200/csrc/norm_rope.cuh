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
#include "paged_attn.cuh"  // two fp32 operations in one instruction
#include "paged_q8.cuh"
#include "rope_rows.cuh"

namespace lar {

__device__ __forceinline__ uint64_t mul_f32x2(uint64_t a, uint64_t b) {
    uint64_t r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ float sum_of(uint64_t v) {
    float a, b;
    unpack_f32x2(v, a, b);
    return a + b;
}
__device__ __forceinline__ float max_nan(float a, float b) {  // NaN where one is
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}

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
    int shift;             // log2 of the tokens of a CTA
};

constexpr int kNormTokens = 8;  // tokens of a CTA at most

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
__global__ void __launch_bounds__(kRopeThreads, 5) norm_rope_kernel(const __grid_constant__ NormRopeArgs na) {
    constexpr int E = Elt<T>::kPerChunk;  // elements of a 16-byte chunk
    constexpr int IPR = D / (2 * E);      // threads of a row
    constexpr int HP = D / 2;
    constexpr int B = 16 / E;             // items (32 bytes each) that a thread has at a time: 32 registers once unpacked
    constexpr int GROUPS = kRopeThreads / IPR;  // rows that the CTA has at a time, once
    const RopeRowsArgs& a = na.r;
    __shared__ __align__(16) float cs[kNormTokens][D];  // cosines, sines
    __shared__ int slot_of[kNormTokens], seq_of[kNormTokens];

    const int tid = threadIdx.x;
    const int t0 = blockIdx.x * a.tokens_per_cta;  // (a power of two of tokens: 1 << na.shift)
    const int nt = min(a.tokens_per_cta, a.n_tokens - t0);
    const int row0 = blockIdx.y * a.rows_per_slice, row1 = min(row0 + a.rows_per_slice, a.n_rows);
    const int c = tid & (IPR - 1);
    const int o_lo = INTER ? 2 * c * E : c * E, o_hi = INTER ? (2 * c + 1) * E : HP + c * E;
    // a thread stays with its token and goes through heads
    const int tl = (tid / IPR) & (a.tokens_per_cta - 1), step = GROUPS >> na.shift, own = (tid / IPR) >> na.shift;
    const bool live = tl < nt;
    const long long t = t0 + tl;
    int slot = -1, seq = -1;

    // q, k and v rows one kind behind the other: what depends on the kind is the same for all threads
    auto heads_of = [&](int which, int& h0, int& h1) {  // heads h0 .. h1 - 1 of this CTA
        const int first = which > 1 ? a.heads[0] + a.heads[1] : which > 0 ? a.heads[0] : 0;
        h0 = max(row0 - first, 0);
        h1 = min(row1 - first, a.heads[which]);
    };
    auto fetch = [&](int which, int g, int h1, uint4 (&lo)[B], uint4 (&hi)[B]) {
        const T* from = reinterpret_cast<const T*>(a.src[which].p) + t * a.src[which].token_stride;
#pragma unroll
        for (int b = 0; b < B; ++b) {
            const int head = g + b * step + own;
            lo[b] = hi[b] = make_uint4(0, 0, 0, 0);
            if (live && head < h1) {
                const T* p = from + head * a.src[which].head_stride;
                lo[b] = *reinterpret_cast<const uint4*>(p + o_lo);
                hi[b] = *reinterpret_cast<const uint4*>(p + o_hi);
            }
        }
    };
    int which = 0, h0, h1;
    for (heads_of(which, h0, h1); h1 <= h0 && which < 2; heads_of(++which, h0, h1)) {}
    uint4 next_lo[B], next_hi[B];
    fetch(which, h0, h1, next_lo, next_hi);
    // sines, cosines and slots of the CTA's tokens, while the first rows are on the way
    if (a.pos) {
        const int i = tid & (HP - 1);
        const double f = a.f.turns[i];
        const int* p = a.pos + a.f.axis[i] * a.pos_axis_stride + t0;
        for (int l = tid / HP; l < nt; l += kRopeThreads / HP) {
            const float2 v = cos_sin_of(f, p[l]);
            cs[l][i] = v.x;
            cs[l][HP + i] = v.y;
        }
    }
    if (DEST) find_slots<kRopeThreads>(a.kv, a.state ? a.base_len : -1, t0, nt, slot_of, seq_of);
    __syncthreads();
    if (DEST && live) {
        slot = slot_of[tl];
        seq = seq_of[tl];
    }
    int g0 = h0;
#pragma unroll 1
    while (which < 3) {
        const HeadNormView& h = na.norm[which & 1];
        const bool on = which < 2 && h.on, layer = on && h.layer, turn = which < 2 && a.pos;
        char* pool = which == 1 ? a.kv.k_pool : a.kv.v_pool;
        {
            uint4 lo[B], hi[B];
            int head[B];
            bool has[B];
            long long at[B], scale_at[B];  // element of the pool (-1: the row is not written), its scale byte
#pragma unroll
            for (int b = 0; b < B; ++b) {
                head[b] = g0 + b * step + own;
                has[b] = live && head[b] < h1;
                lo[b] = next_lo[b];
                hi[b] = next_hi[b];
            }
            // the next rows are on the way while these are worked on
            int nwhich = which, ng = g0 + step * B, nh1 = h1;
            if (ng >= h1) {
                nh1 = ng = 0;
                while (nh1 <= ng && ++nwhich < 3) heads_of(nwhich, ng, nh1);
            }
            if (nwhich < 3) fetch(nwhich, ng, nh1, next_lo, next_hi);
#pragma unroll
            for (int b = 0; b < B; ++b) {
                at[b] = scale_at[b] = 0;
                if (!DEST || !has[b]) continue;
                if (which == 0) {
                    if (seq < 0) at[b] = -1;
                } else if (slot < 0) {
                    at[b] = -1;
                } else {
                    const int page = a.kv.table[seq * a.kv.table_seq_stride + head[b] * a.kv.table_head_stride + (slot >> a.kv.page_shift)];
                    const int in_page = slot & (a.kv.page_tokens - 1);
                    at[b] = page * a.kv.page_stride + in_page * a.kv.row_stride + head[b] * a.kv.head_stride;
                    if (DEST == 2) scale_at[b] = page * na.q8.page_stride + head[b] * na.q8.head_stride + in_page;
                    if (page < 0 || page >= a.kv.n_pages) {
                        at[b] = -1;
                        if (c == 0) paged_report(a.kv, kStPage);
                    }
                }
            }
            if (DEST == 1 && which == 2) {  // values as they are: a pass through fp32 could touch the bits of a NaN
#pragma unroll
                for (int b = 0; b < B; ++b)
                    if (has[b] && at[b] >= 0) {
                        *reinterpret_cast<uint4*>(reinterpret_cast<T*>(pool) + at[b] + o_lo) = lo[b];
                        *reinterpret_cast<uint4*>(reinterpret_cast<T*>(pool) + at[b] + o_hi) = hi[b];
                    }
                which = nwhich;
                g0 = ng;
                h1 = nh1;
                continue;
            }
            uint64_t x[B][E];  // two elements each: the low chunk, then the high one
#pragma unroll
            for (int b = 0; b < B; ++b) {
                float u[E], v[E];
                Elt<T>::unpack(lo[b], u);
                Elt<T>::unpack(hi[b], v);
#pragma unroll
                for (int i = 0; i < E / 2; ++i) {
                    x[b][i] = pack_f32x2(u[2 * i], u[2 * i + 1]);
                    x[b][E / 2 + i] = pack_f32x2(v[2 * i], v[2 * i + 1]);
                }
            }
            if (on) {
                // The row sums, one step for all rows of the batch at a time.  (Warp-wide: lanes without a row have zeros.)
                float mean[B], ss[B], up[B];
                auto sums = [&]() {
#pragma unroll
                    for (int b = 0; b < B; ++b) {
                        uint64_t y = x[b][0];
#pragma unroll
                        for (int i = 1; i < E; ++i) y = add_f32x2(y, x[b][i]);
                        mean[b] = sum_of(y);
                    }
#pragma unroll
                    for (int o = 1; o < IPR; o <<= 1)
#pragma unroll
                        for (int b = 0; b < B; ++b) mean[b] += __shfl_xor_sync(0xffffffffu, mean[b], o);
#pragma unroll
                    for (int b = 0; b < B; ++b) {
                        mean[b] *= -1.0f / D;
#pragma unroll
                        for (int i = 0; i < E; ++i) x[b][i] = add_f32x2(x[b][i], pack_f32x2(mean[b], mean[b]));
                    }
                };
                auto squares = [&]() {
#pragma unroll
                    for (int b = 0; b < B; ++b) {
                        uint64_t y = mul_f32x2(x[b][0], x[b][0]);
#pragma unroll
                        for (int i = 1; i < E; ++i) y = fma_f32x2(x[b][i], x[b][i], y);
                        ss[b] = sum_of(y);
                    }
#pragma unroll
                    for (int o = 1; o < IPR; o <<= 1)
#pragma unroll
                        for (int b = 0; b < B; ++b) ss[b] += __shfl_xor_sync(0xffffffffu, ss[b], o);
                };
                if (layer) sums();
                squares();
                bool beyond = false;
#pragma unroll
                for (int b = 0; b < B; ++b) {
                    up[b] = 1.f;
                    beyond |= !(ss[b] <= 3.4e38f);
                }
                if (__any_sync(0xffffffffu, beyond)) {
                    // squares (or the sum) beyond fp32: once more from the rows (not written yet) times 2^-80, beside which eps is nothing
                    fetch(which, g0, h1, lo, hi);
#pragma unroll
                    for (int b = 0; b < B; ++b) {
                        if (!(ss[b] <= 3.4e38f)) up[b] = 0x1p-80f;
                        float u[E], v[E];
                        Elt<T>::unpack(lo[b], u);
                        Elt<T>::unpack(hi[b], v);
#pragma unroll
                        for (int i = 0; i < E / 2; ++i) {
                            x[b][i] = pack_f32x2(u[2 * i] * up[b], u[2 * i + 1] * up[b]);
                            x[b][E / 2 + i] = pack_f32x2(v[2 * i] * up[b], v[2 * i + 1] * up[b]);
                        }
                    }
                    if (layer) sums();
                    squares();
                }
#pragma unroll
                for (int b = 0; b < B; ++b) {
                    if (!has[b]) continue;
                    const float f = rsqrtf(fmaf(ss[b], 1.0f / D, h.eps * up[b] * up[b]));
                    const uint64_t f2 = pack_f32x2(f, f);
                    const long long wat = head[b] * h.head_stride;
#pragma unroll
                    for (int half = 0; half < 2; ++half) {
                        uint64_t* y = x[b] + half * (E / 2);
                        const int o = half ? o_hi : o_lo;
                        float w[E];
#pragma unroll
                        for (int i = 0; i < E / 2; ++i) y[i] = mul_f32x2(y[i], f2);
                        if (h.weight && h.bias) {
                            float add[E];
                            norm_params<E>(h.weight, wat + o, h.bf16, w);
                            norm_params<E>(h.bias, wat + o, h.bf16, add);
#pragma unroll
                            for (int i = 0; i < E / 2; ++i) y[i] = fma_f32x2(y[i], pack_f32x2(w[2 * i], w[2 * i + 1]), pack_f32x2(add[2 * i], add[2 * i + 1]));
                        } else if (h.weight) {
                            norm_params<E>(h.weight, wat + o, h.bf16, w);
#pragma unroll
                            for (int i = 0; i < E / 2; ++i) y[i] = mul_f32x2(y[i], pack_f32x2(w[2 * i], w[2 * i + 1]));
                        } else if (h.bias) {
                            norm_params<E>(h.bias, wat + o, h.bf16, w);
#pragma unroll
                            for (int i = 0; i < E / 2; ++i) y[i] = add_f32x2(y[i], pack_f32x2(w[2 * i], w[2 * i + 1]));
                        }
                    }
                }
            }
            if (turn) {
                const uint64_t minus = pack_f32x2(-1.f, -1.f);
#pragma unroll
                for (int i = 0; i < E / 2; i += 2) {
                    const float4 u = *reinterpret_cast<const float4*>(&cs[tl][c * E + 2 * i]), v = *reinterpret_cast<const float4*>(&cs[tl][HP + c * E + 2 * i]);
                    const uint64_t co[2] = {pack_f32x2(u.x, u.y), pack_f32x2(u.z, u.w)}, si[2] = {pack_f32x2(v.x, v.y), pack_f32x2(v.z, v.w)};
#pragma unroll
                    for (int j = 0; j < 2; ++j)
#pragma unroll
                        for (int b = 0; b < B; ++b) {
                            // two pairs: side by side in the operands where pairs interleave, in the same place of both halves else
                            uint64_t& y0 = x[b][INTER ? 2 * (i + j) : i + j];
                            uint64_t& y1 = x[b][INTER ? 2 * (i + j) + 1 : E / 2 + i + j];
                            uint64_t p = y0, q = y1;
                            if (INTER) {
                                float p0, q0, p1, q1;
                                unpack_f32x2(y0, p0, q0);
                                unpack_f32x2(y1, p1, q1);
                                p = pack_f32x2(p0, p1);
                                q = pack_f32x2(q0, q1);
                            }
                            const uint64_t x2 = fma_f32x2(mul_f32x2(q, si[j]), minus, mul_f32x2(p, co[j])), z2 = fma_f32x2(q, co[j], mul_f32x2(p, si[j]));
                            if (INTER) {
                                float p0, q0, p1, q1;
                                unpack_f32x2(x2, p0, p1);
                                unpack_f32x2(z2, q0, q1);
                                y0 = pack_f32x2(p0, q0);
                                y1 = pack_f32x2(p1, q1);
                            } else {
                                y0 = x2;
                                y1 = z2;
                            }
                        }
                }
            }
            int byte[B];
            if (DEST == 2 && which > 0) {
                float largest[B];
#pragma unroll
                for (int b = 0; b < B; ++b) {
                    largest[b] = 0.f;
#pragma unroll
                    for (int i = 0; i < E; ++i) {
                        float p, q;
                        unpack_f32x2(x[b][i], p, q);
                        largest[b] = max_nan(max_nan(largest[b], fabsf(p)), fabsf(q));
                    }
                }
#pragma unroll
                for (int o = 1; o < IPR; o <<= 1)
#pragma unroll
                    for (int b = 0; b < B; ++b) largest[b] = max_nan(largest[b], __shfl_xor_sync(0xffffffffu, largest[b], o));
#pragma unroll
                for (int b = 0; b < B; ++b) byte[b] = q8_byte(__float_as_uint(largest[b]));
            }
#pragma unroll
            for (int b = 0; b < B; ++b) {
                if (!has[b] || at[b] < 0) continue;
                float y[2 * E];
#pragma unroll
                for (int i = 0; i < E; ++i) unpack_f32x2(x[b][i], y[2 * i], y[2 * i + 1]);
                if (DEST == 2 && which > 0) {
                    unsigned codes[E / 2];
#pragma unroll
                    for (int i = 0; i < E / 2; ++i) codes[i] = q8_codes4(y + 4 * i, byte[b]);
                    char* p = pool + at[b];
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
                    if (c == 0) {
                        (which == 1 ? na.q8.k_scale : na.q8.v_scale)[scale_at[b]] = (unsigned char)byte[b];
                    }
                    continue;
                }
                T* dst = DEST == 1 && which > 0 ? reinterpret_cast<T*>(pool) + at[b]
                                                : reinterpret_cast<T*>(a.dst[which].p) + t * a.dst[which].token_stride + head[b] * a.dst[which].head_stride;
                float u[E], v[E];
#pragma unroll
                for (int i = 0; i < E; ++i) {
                    u[i] = y[i];
                    v[i] = y[E + i];
                }
                *reinterpret_cast<uint4*>(dst + o_lo) = PackRow<T>::pack(u);
                *reinterpret_cast<uint4*>(dst + o_hi) = PackRow<T>::pack(v);
            }
            which = nwhich;
            g0 = ng;
            h1 = nh1;
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
