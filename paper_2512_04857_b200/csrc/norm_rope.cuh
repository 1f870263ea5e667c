// Norms of q and k per head with the rotary embedding in the same pass, on rows in memory and on the way into a paged cache (of the rows'
// type, or of 8 bits).
//
//   rms:    y = x / sqrt(mean(x^2) + eps) * w  (+ bias)        layer:  y = (x - mean(x)) / sqrt(mean((x - mean)^2) + eps) * w  (+ bias)
//   then the pairs of y are turned as in rope_rows.cuh, and the result is rounded once, to the storage type or to 8 bits.
//
// Bound: HBM bytes (each row once in, once out), as long as an element costs few instructions.  So a CTA has rows of one kind (q, k or v: what depends on the
// kind is the same for all its threads) and a thread stays with one head, of which it has 16 bytes of each half of a row (or 32 bytes side by side
// where pairs interleave), and goes through tokens: its pointers are in registers from the start, and weights, biases, sines, cosines and slots of the
// CTA in shared memory behind one barrier (weights in registers leave room for half the warps: 275 us where this takes 230, 5.9 TB/s, on 66560 tokens of 40 bf16 rows of 128, layer norm, in a graph; calls one by one take 244 to 256), in the
// order in which threads read them (sines and cosines in their own order cost bank conflicts: 247 us).  The D / 16 (bf16) or D / 8 (fp32) threads of a row are
// neighbours in a warp: the row's sums are a few shuffles, taken with the row in registers, the mean first and the squares of what is left after it, not the difference of two large sums.  fp32
// arithmetic goes two elements to an instruction.  While a token is worked on the next one is on the way.  16 tokens take 3.6 us, a launch; 24 prompts of up to 2048
// tokens into 8 bits 120 (4.9 TB/s: the rounding to codes comes on top).
#pragma once
#include "paged_attn.cuh"  // two fp32 operations in one instruction
#include "paged_q8.cuh"
#include "rope_rows.cuh"

namespace lar {

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
    int at_once[3];        // tokens of a pass of a CTA, of each kind of row
    int slices[3];         // CTAs that the heads of a kind take
    int heads[3];          // heads of a CTA
    int tokens;            // of a CTA
};

constexpr int kNormThreads = 256;  // of a CTA at most
constexpr int kNormTokens = 24;   // tokens of a CTA at most (with the weights of 256 threads just within 48 KB)

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

// Slot and sequence of token t, by a warp, as find_slots: the number of sequences that end at or before it.
__device__ __forceinline__ void find_slot(const PagedView& kv, int base_len, int t, int* slot_of, int* seq_of) {
    const int lane = threadIdx.x & 31;
    int s = 0;
    if (kv.cu) {
        for (int j = lane; j < kv.n_seqs; j += 32) s += kv.cu[j + 1] <= t;
        s = __reduce_add_sync(0xffffffffu, s);
    } else {
        s = t / kv.chunk;
    }
    if (lane == 0) {
        int slot = -1, b0 = 0, b1 = 0;
        if (s < kv.n_seqs) chunk_of(kv, s, b0, b1);
        if (t < b0 || t >= b1) {
            s = -1;
        } else {
            slot = base_len >= 0 ? base_len + (t - b0) : kv.lens[s * kv.lens_stride] - (b1 - t);
            if (slot < 0 || slot >= (kv.table_cols << kv.page_shift)) {
                paged_report(kv, kStPage);
                slot = -1;
            }
        }
        *slot_of = slot;
        *seq_of = s;
    }
}

// DEST: 0 rows, 1 pages of the rows' type, 2 pages of 8 bits
template <typename T, int D, bool INTER, int DEST>
struct NormRope {
    static constexpr int E = Elt<T>::kPerChunk;  // elements of a 16-byte chunk
    static constexpr int IPR = D / (2 * E);      // threads of a row
    static constexpr int HP = D / 2;

    static constexpr int NP = E;                 // pieces of four parameters that a thread has: weights and biases in turn

    struct Shared {
        float cs[kNormTokens][D];  // cosines, sines: a thread's four side by side with its neighbours'
        int slot_of[kNormTokens], seq_of[kNormTokens];
        float4 params[kNormThreads * NP];  // [head][piece][thread of the row]
    };

    static __device__ __forceinline__ float row_sum(float v) {
#pragma unroll
        for (int o = 1; o < IPR; o <<= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
        return v;
    }
    static __device__ __forceinline__ void unpack(const uint4& lo, const uint4& hi, float up, uint64_t (&x)[E]) {
        float u[E], v[E];
        Elt<T>::unpack(lo, u);
        Elt<T>::unpack(hi, v);
#pragma unroll
        for (int i = 0; i < E / 2; ++i) {
            x[i] = pack_f32x2(u[2 * i] * up, u[2 * i + 1] * up);
            x[E / 2 + i] = pack_f32x2(v[2 * i] * up, v[2 * i + 1] * up);
        }
    }

    // The rows of one kind of the CTA's tokens.
    template <int KIND>
    static __device__ __forceinline__ void rows(const NormRopeArgs& na, Shared& sh, int slice) {
        const RopeRowsArgs& a = na.r;
        const HeadNormView& h = na.norm[KIND & 1];
        const bool on = KIND < 2 && h.on, layer = on && h.layer, turn = KIND < 2 && a.pos;
        const int tid = threadIdx.x, c = tid & (IPR - 1), group = tid / IPR;
        const int sub = group / na.heads[KIND], head = slice * na.heads[KIND] + group - sub * na.heads[KIND];
        const bool has = sub < na.at_once[KIND] && head < a.heads[KIND];
        const int t0 = blockIdx.x * na.tokens, t1 = min(t0 + na.tokens, a.n_tokens), step = na.at_once[KIND];
        const int o_lo = INTER ? 2 * c * E : c * E, o_hi = INTER ? (2 * c + 1) * E : HP + c * E;
        int t = t0 + sub;
        const T* from = reinterpret_cast<const T*>(a.src[KIND].p) + head * a.src[KIND].head_stride + t * a.src[KIND].token_stride;
        const long long from_step = step * a.src[KIND].token_stride;
        auto fetch = [&](int t, uint4& lo, uint4& hi) {
            if (has && t < t1) {
                lo = __ldcg(reinterpret_cast<const uint4*>(from + o_lo));
                hi = __ldcg(reinterpret_cast<const uint4*>(from + o_hi));
            }
            from += from_step;
        };
        uint4 next_lo = make_uint4(0, 0, 0, 0), next_hi = next_lo;  // of the next token, on the way
        fetch(t, next_lo, next_hi);
        if (on && sub == 0) {
            // weights and biases, a thread's 16 bytes side by side with its neighbours'
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                float u[E], v[E];
#pragma unroll
                for (int i = 0; i < E; ++i) {
                    u[i] = 1.f;
                    v[i] = 0.f;
                }
                if (has) {
                    const long long at = head * h.head_stride + (half ? o_hi : o_lo);
                    if (h.weight) norm_params<E>(h.weight, at, h.bf16, u);
                    if (h.bias) norm_params<E>(h.bias, at, h.bf16, v);
                }
#pragma unroll
                for (int i = 0; i < E; i += 4) {
                    float4* p = sh.params + (group * NP + (half * E + i) / 2) * IPR + c;
                    p[0] = make_float4(u[i], u[i + 1], u[i + 2], u[i + 3]);
                    p[IPR] = make_float4(v[i], v[i + 1], v[i + 2], v[i + 3]);
                }
            }
        }
        const float4* params = sh.params + (group - sub * na.heads[KIND]) * NP * IPR + c;
        // sines, cosines and slots of the CTA's tokens
        if (turn) {
            const int i = tid & (HP - 1), at = ((i % E / 4) * IPR + i / E) * 4 + i % 4;
            const double f = a.f.turns[i];
            const int* p = a.pos + a.f.axis[i] * a.pos_axis_stride + t0;
            for (int l = tid / HP; l < t1 - t0; l += blockDim.x / HP) {
                const float2 v = cos_sin_of(f, p[l]);
                sh.cs[l][at] = v.x;
                sh.cs[l][HP + at] = v.y;
            }
        }
        if (DEST)
            for (int l = tid >> 5; l < t1 - t0; l += blockDim.x >> 5)
                find_slot(a.kv, a.state ? a.base_len : -1, t0 + l, &sh.slot_of[l], &sh.seq_of[l]);
        __syncthreads();

        const bool paged = DEST && KIND > 0;
        T* to = nullptr;
        long long to_step = 0;
        if (!paged) {
            to = reinterpret_cast<T*>(a.dst[KIND].p) + head * a.dst[KIND].head_stride + t * a.dst[KIND].token_stride;
            to_step = step * a.dst[KIND].token_stride;
        }
        const int* table = a.kv.table + head * a.kv.table_head_stride;
        char* pool = KIND == 1 ? a.kv.k_pool : a.kv.v_pool;
        auto work = [&](const uint4& lo, const uint4& hi) {
            uint64_t x[E];
            unpack(lo, hi, 1.f, x);
            if (on) {
                float ss, up = 1.f;
                auto sums = [&]() {
                    if (layer) {
                        uint64_t y[E / 2];  // (pairs of pairs: the sum of equal elements is exact, and so is their mean)
#pragma unroll
                        for (int i = 0; i < E / 2; ++i) y[i] = add_f32x2(x[i], x[E / 2 + i]);
#pragma unroll
                        for (int n = E / 4; n > 0; n >>= 1)
#pragma unroll
                            for (int i = 0; i < n; ++i) y[i] = add_f32x2(y[i], y[n + i]);
                        const float mean = row_sum(sum_of(y[0])) * (-1.0f / D);
                        const uint64_t m2 = pack_f32x2(mean, mean);
#pragma unroll
                        for (int i = 0; i < E; ++i) x[i] = add_f32x2(x[i], m2);
                    }
                    uint64_t y = mul_f32x2(x[0], x[0]);
#pragma unroll
                    for (int i = 1; i < E; ++i) y = fma_f32x2(x[i], x[i], y);
                    ss = row_sum(sum_of(y));
                };
                sums();
                if (__any_sync(0xffffffffu, !(ss <= 3.4e38f))) {
                    // squares (or the sum) beyond fp32: once more from the row times 2^-80.  What is left after the mean is then 2^96 of the row's units and more, beside which
                    // eps is nothing, or nothing at all
                    if (!(ss <= 3.4e38f)) up = 0x1p-80f;
                    unpack(lo, hi, up, x);
                    sums();
                }
                const float f = rsqrtf(max_nan(fmaf(ss, 1.0f / D, h.eps * up * up), 0x1p-126f));
                const uint64_t f2 = pack_f32x2(f, f);
#pragma unroll
                for (int i = 0; i < E; i += 2) {
                    const float4 w = params[i * IPR], v = params[(i + 1) * IPR];
                    x[i] = fma_f32x2(mul_f32x2(x[i], f2), pack_f32x2(w.x, w.y), pack_f32x2(v.x, v.y));
                    x[i + 1] = fma_f32x2(mul_f32x2(x[i + 1], f2), pack_f32x2(w.z, w.w), pack_f32x2(v.z, v.w));
                }
            }
            const int l = min(t - t0, kNormTokens - 1);
            if (turn) {
                const uint64_t minus = pack_f32x2(-1.f, -1.f);
                const float* cosv = &sh.cs[l][c * 4];
#pragma unroll
                for (int i = 0; i < E / 2; i += 2) {
                    const float4 u = *reinterpret_cast<const float4*>(cosv + i * 2 * IPR), v = *reinterpret_cast<const float4*>(cosv + HP + i * 2 * IPR);
                    const uint64_t co[2] = {pack_f32x2(u.x, u.y), pack_f32x2(u.z, u.w)}, si[2] = {pack_f32x2(v.x, v.y), pack_f32x2(v.z, v.w)};
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        // two pairs: side by side in the operands where pairs interleave, in the same place of both halves else
                        uint64_t& y0 = x[INTER ? 2 * (i + j) : i + j];
                        uint64_t& y1 = x[INTER ? 2 * (i + j) + 1 : E / 2 + i + j];
                        uint64_t p = y0, q = y1;
                        if (INTER) {
                            float p0, q0, p1, q1;
                            unpack_f32x2(y0, p0, q0);
                            unpack_f32x2(y1, p1, q1);
                            p = pack_f32x2(p0, p1);
                            q = pack_f32x2(q0, q1);
                        }
                        const uint64_t x2 = fma_f32x2(mul_f32x2(q, si[j]), minus, mul_f32x2(p, co[j])), z2 = fma_f32x2(q, co[j], mul_f32x2(p, si[j]));
                        y0 = x2;
                        y1 = z2;
                        if (INTER) {
                            float p0, q0, p1, q1;
                            unpack_f32x2(x2, p0, p1);
                            unpack_f32x2(z2, q0, q1);
                            y0 = pack_f32x2(p0, q0);
                            y1 = pack_f32x2(p1, q1);
                        }
                    }
                }
            }
            int byte = 0;
            if (DEST == 2 && paged) {
                float largest = 0.f;
#pragma unroll
                for (int i = 0; i < E; ++i) {
                    float p, q;
                    unpack_f32x2(x[i], p, q);
                    largest = max_nan(max_nan(largest, fabsf(p)), fabsf(q));
                }
#pragma unroll
                for (int o = 1; o < IPR; o <<= 1) largest = max_nan(largest, __shfl_xor_sync(0xffffffffu, largest, o));
                byte = q8_byte(__float_as_uint(largest));
            }
            if (!has || t >= t1) return;
            T* dst = to;
            if (DEST && !paged && sh.seq_of[l] < 0) return;
            if (paged) {
                const int slot = sh.slot_of[l];
                if (slot < 0) return;
                const int page = table[sh.seq_of[l] * a.kv.table_seq_stride + (slot >> a.kv.page_shift)];
                if (page < 0 || page >= a.kv.n_pages) {
                    if (c == 0) paged_report(a.kv, kStPage);
                    return;
                }
                const int in_page = slot & (a.kv.page_tokens - 1);
                const long long at = page * a.kv.page_stride + in_page * a.kv.row_stride + head * a.kv.head_stride;
                if (DEST == 2) {
                    float y[2 * E];
                    unsigned codes[E / 2];
#pragma unroll
                    for (int i = 0; i < E; ++i) unpack_f32x2(x[i], y[2 * i], y[2 * i + 1]);
#pragma unroll
                    for (int i = 0; i < E / 2; ++i) codes[i] = q8_codes4(y + 4 * i, byte);
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
                    if (c == 0) (KIND == 1 ? na.q8.k_scale : na.q8.v_scale)[page * na.q8.page_stride + head * na.q8.head_stride + in_page] = (unsigned char)byte;
                    return;
                }
                dst = reinterpret_cast<T*>(pool) + at;
                if (KIND == 2) {  // values as they are: a pass through fp32 could touch the bits of a NaN
                    *reinterpret_cast<uint4*>(dst + o_lo) = lo;
                    *reinterpret_cast<uint4*>(dst + o_hi) = hi;
                    return;
                }
            }
            float u[E], v[E];
#pragma unroll
            for (int i = 0; i < E / 2; ++i) {
                unpack_f32x2(x[i], u[2 * i], u[2 * i + 1]);
                unpack_f32x2(x[E / 2 + i], v[2 * i], v[2 * i + 1]);
            }
            __stcg(reinterpret_cast<uint4*>(dst + o_lo), PackRow<T>::pack(u));
            __stcg(reinterpret_cast<uint4*>(dst + o_hi), PackRow<T>::pack(v));
        };
        const int passes = (t1 - t0 + step - 1) / step;
#pragma unroll 1
        for (int p = 0; p < passes; ++p) {
            const uint4 lo = next_lo, hi = next_hi;
            fetch(t + step, next_lo, next_hi);
            work(lo, hi);
            t += step;
            to += to_step;
        }
    }
};

template <typename T, int D, bool INTER, int DEST>
__global__ void __launch_bounds__(kNormThreads, 4) norm_rope_kernel(const __grid_constant__ NormRopeArgs na) {
    using R = NormRope<T, D, INTER, DEST>;
    __shared__ __align__(16) typename R::Shared sh;
    const RopeRowsArgs& a = na.r;
    int y = blockIdx.y;
    if (y < na.slices[0]) {
        R::template rows<0>(na, sh, y);
    } else if ((y -= na.slices[0]) < na.slices[1]) {
        R::template rows<1>(na, sh, y);
    } else if (DEST) {
        R::template rows<2>(na, sh, y - na.slices[1]);
    }
    if (DEST == 1 && a.state && blockIdx.y == gridDim.y - 1) {
        // the library's own cache: the index map's entries of the tokens; the last one sets the unit's length
        const int t0 = blockIdx.x * na.tokens, nt = min(na.tokens, a.n_tokens - t0);
        for (int i = threadIdx.x; i < nt * a.kv.n_kv_heads; i += blockDim.x) {
            const int l = i / a.kv.n_kv_heads, head = i - l * a.kv.n_kv_heads, slot = sh.slot_of[l];
            if (slot < 0) continue;
            const int unit = sh.seq_of[l] * a.kv.n_kv_heads + head;
            a.index_map[(size_t)unit * a.cap_pad + slot] = slot;
            if (slot == a.base_len + a.kv.chunk - 1) {
                UnitState ns;
                ns.len = slot + 1;
                ns.n_tok = 0;
                a.state[unit] = ns;
            }
        }
    }
}

}  // namespace lar
