// Rotary position embedding with several position axes, on rows in memory (q, k) and on the way into a paged cache.
//
//   pair i of a token's row is turned by angle  pos[axis(i)][token] * theta^(-e_i):
//       x' = x cos - y sin,  y' = y cos + x sin        (fp32, every product and sum rounded, result rounded to the storage type)
//
// One kernel does both entry points: a token's rows are its q heads (rotated), k heads (rotated) and v heads (copied);
// k and v go either to dense rows or to the slot that the page table gives.
//
// Bound: HBM bytes (each row once in, once out; 3 flop per element).  The angles are formed in fp64, in turns: pos * f_i
// with f_i = theta^(-e_i) / 2 pi, minus its nearest integer, so a position of 10^6 loses nothing and the fp32 sine and
// cosine (sincospif) see [-1/2, 1/2] turns.  They are needed once per (token, pair) and shared by all heads of the token
// through shared memory: a CTA takes TB tokens, its threads first request their rows, then form TB * D / 2 sines while the
// rows are on the way, then rotate.  A thread owns 16 bytes of each half of a row (or 32 consecutive bytes where pairs
// interleave), so both members of a pair are in its registers and rotating in place is safe.
#pragma once
#include "paged.cuh"

namespace lar {

constexpr int kRopeThreads = 128;  // (256: 211 instead of 204 us on 66560 tokens of 40 rows, 120 instead of 102 us on 24 prompts into pages)
constexpr int kRopeMaxAxes = 4;
constexpr int kRopeBatch = 4;  // items (32 bytes each) a thread has in flight

struct RopeFreqs {
    double turns[64];        // turns per unit of position of each pair (negative: inverse rotation)
    unsigned char axis[64];  // position axis of each pair
};

struct RowsView {
    char* p;
    long long token_stride, head_stride;  // elements
};

struct RopeRowsArgs {
    RopeFreqs f;
    const int* pos;  // [axes][n_tokens], axes pos_axis_stride apart; null: rows are copied, not rotated
    long long pos_axis_stride;
    RowsView src[3], dst[3];  // q, k, v (dst[1], dst[2] unused when k and v go to pages)
    int heads[3];
    int n_rows;             // heads[0] + heads[1] + heads[2]
    int rows_per_slice;     // rows of a token that one CTA handles (grid.y slices)
    unsigned rows_magic;    // floor(2^32 / rows_per_slice) + 1, which 32 bits do not hold for one row: 0
    int n_tokens, tokens_per_cta;
    PagedView kv;           // PAGED only
    // the library's own cache (PAGED, may be null): every unit's length and index map advance with the append
    int* index_map;
    UnitState* state;
    int cap_pad, base_len;  // base_len: entries before the append, from the host (nobody reads a length that this kernel writes)
};

__device__ __forceinline__ float2 turn_pair(float x, float y, float c, float s) {
    return make_float2(__fsub_rn(__fmul_rn(x, c), __fmul_rn(y, s)), __fadd_rn(__fmul_rn(y, c), __fmul_rn(x, s)));
}
__device__ __forceinline__ float2 cos_sin_of(double turns_per_pos, int pos) {
    const double t = (double)pos * turns_per_pos;
    float s, c;
    sincospif(2.0f * (float)(t - rint(t)), &s, &c);
    return make_float2(c, s);
}

template <typename T>
struct PackRow;
template <>
struct PackRow<__nv_bfloat16> {
    static __device__ __forceinline__ uint4 pack(const float (&f)[8]) {
        uint4 r;
        __nv_bfloat162 a = __floats2bfloat162_rn(f[0], f[1]), b = __floats2bfloat162_rn(f[2], f[3]);
        __nv_bfloat162 c = __floats2bfloat162_rn(f[4], f[5]), d = __floats2bfloat162_rn(f[6], f[7]);
        r.x = *reinterpret_cast<uint32_t*>(&a); r.y = *reinterpret_cast<uint32_t*>(&b);
        r.z = *reinterpret_cast<uint32_t*>(&c); r.w = *reinterpret_cast<uint32_t*>(&d);
        return r;
    }
};
template <>
struct PackRow<float> {
    static __device__ __forceinline__ uint4 pack(const float (&f)[4]) {
        return make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3]));
    }
};

template <typename T, int D, bool INTER, bool PAGED>
__global__ void __launch_bounds__(kRopeThreads) rope_rows_kernel(const __grid_constant__ RopeRowsArgs a) {
    constexpr int E = Elt<T>::kPerChunk;   // elements of a 16-byte chunk
    constexpr int IPR = D / (2 * E);       // items (two chunks) of a row
    constexpr int HP = D / 2;              // pairs of a row
    extern __shared__ __align__(16) float cs[];  // [tokens_per_cta][cos HP | sin HP], then the tokens' slots (PAGED)
    int* slot_of = reinterpret_cast<int*>(cs + a.tokens_per_cta * D);  // slot of each token, -1: none
    int* seq_of = slot_of + a.tokens_per_cta;

    const int tid = threadIdx.x;
    const int t0 = blockIdx.x * a.tokens_per_cta;
    const int nt = min(a.tokens_per_cta, a.n_tokens - t0);
    const int row0 = blockIdx.y * a.rows_per_slice;
    const int nr = min(a.rows_per_slice, a.n_rows - row0);
    const int n_items = nt * a.rows_per_slice * IPR;  // (rows beyond nr are skipped: only the last slice has them)

    bool ready = false;
    for (int base = 0; base < n_items; base += kRopeThreads * kRopeBatch) {
        uint4 lo[kRopeBatch], hi[kRopeBatch];
        int tok[kRopeBatch], row[kRopeBatch];
        const int c = tid & (IPR - 1);
        const int o_lo = INTER ? 2 * c * E : c * E, o_hi = INTER ? (2 * c + 1) * E : HP + c * E;
#pragma unroll
        for (int b = 0; b < kRopeBatch; ++b) {
            const int item = base + b * kRopeThreads + tid;
            const int r = item / IPR;
            const int tl = a.rows_magic ? (int)__umulhi((unsigned)r, a.rows_magic) : r;
            const int rl = r - tl * a.rows_per_slice;
            tok[b] = item < n_items && rl < nr ? tl : -1;
            row[b] = row0 + rl;
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
            if (PAGED) {
                // sequence of a token: the number of sequences that end at or before it
                int s = 0;
                if (a.kv.cu) {
                    for (int tl = 0; tl < nt; ++tl) {
                        int n = 0;
                        for (int j = 0; j < a.kv.n_seqs; j += kRopeThreads)
                            n += __syncthreads_count(j + tid < a.kv.n_seqs && a.kv.cu[j + tid + 1] <= t0 + tl);
                        if (tid == tl) s = n;
                    }
                } else {
                    s = (t0 + tid) / a.kv.chunk;
                }
                if (tid < nt) {  // (tokens_per_cta <= threads)
                    const int t = t0 + tid;
                    int slot = -1, b0 = 0, b1 = 0;
                    if (s < a.kv.n_seqs) chunk_of(a.kv, s, b0, b1);
                    if (t < b0 || t >= b1) {
                        s = -1;  // a token before the first or behind the last sequence: nothing is written for it
                    } else {
                        slot = a.state ? a.base_len + (t - b0) : a.kv.lens[s * a.kv.lens_stride] - (b1 - t);
                        if (slot < 0 || slot >= (a.kv.table_cols << a.kv.page_shift)) {
                            paged_report(a.kv, kStPage);
                            slot = -1;
                        }
                    }
                    slot_of[tid] = slot;
                    seq_of[tid] = s;
                }
            }
            __syncthreads();
        }
#pragma unroll
        for (int b = 0; b < kRopeBatch; ++b) {
            if (tok[b] < 0) continue;
            const int which = row[b] < a.heads[0] ? 0 : row[b] < a.heads[0] + a.heads[1] ? 1 : 2;
            const int head = row[b] - (which > 0 ? a.heads[0] : 0) - (which > 1 ? a.heads[1] : 0);
            T* dst;
            if (PAGED && (which > 0 ? slot_of[tok[b]] : seq_of[tok[b]]) < 0) continue;
            if (PAGED && which > 0) {
                const int slot = slot_of[tok[b]];
                const int page = a.kv.table[seq_of[tok[b]] * a.kv.table_seq_stride + head * a.kv.table_head_stride + (slot >> a.kv.page_shift)];
                if (page < 0 || page >= a.kv.n_pages) {
                    paged_report(a.kv, kStPage);
                    continue;
                }
                char* pool = which == 1 ? a.kv.k_pool : a.kv.v_pool;
                dst = reinterpret_cast<T*>(pool) + page * a.kv.page_stride + (slot & (a.kv.page_tokens - 1)) * a.kv.row_stride + head * a.kv.head_stride;
            } else {
                const RowsView& d = a.dst[which];
                dst = reinterpret_cast<T*>(d.p) + (long long)(t0 + tok[b]) * d.token_stride + head * d.head_stride;
            }
            if (a.pos && which < 2) {
                float x[E], y[E];
                Elt<T>::unpack(lo[b], x);
                Elt<T>::unpack(hi[b], y);
                const float* cosv = cs + tok[b] * D + c * E;
                const float* sinv = cosv + HP;
                if (INTER) {  // x holds pairs 0 .. E/2 - 1 of the item, y the rest
#pragma unroll
                    for (int i = 0; i < E / 2; ++i) {
                        const float2 u = turn_pair(x[2 * i], x[2 * i + 1], cosv[i], sinv[i]);
                        const float2 v = turn_pair(y[2 * i], y[2 * i + 1], cosv[E / 2 + i], sinv[E / 2 + i]);
                        x[2 * i] = u.x; x[2 * i + 1] = u.y;
                        y[2 * i] = v.x; y[2 * i + 1] = v.y;
                    }
                } else {
#pragma unroll
                    for (int i = 0; i < E; ++i) {
                        const float2 u = turn_pair(x[i], y[i], cosv[i], sinv[i]);
                        x[i] = u.x;
                        y[i] = u.y;
                    }
                }
                lo[b] = PackRow<T>::pack(x);
                hi[b] = PackRow<T>::pack(y);
            }
            *reinterpret_cast<uint4*>(dst + o_lo) = lo[b];
            *reinterpret_cast<uint4*>(dst + o_hi) = hi[b];
        }
    }
    if (PAGED && a.state) {
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

// cos and sin of every pair for a list of positions: [n_rows][cos D/2 | sin D/2].  Bound by the fp64 products and the sines, not by the bytes: 66560 rows of
// 128 take 64 us (35 MB), 4160 rows 6.7 us; a step's 16 rows are one launch, 2.5 us.
static __global__ void __launch_bounds__(kRopeThreads) rope_table_kernel(const __grid_constant__ RopeFreqs f, const int* pos, long long pos_axis_stride,
                                                                  int n_rows, int half, float* out) {
    const long long n = (long long)n_rows * half;
    for (long long idx = (long long)blockIdx.x * kRopeThreads + threadIdx.x; idx < n; idx += (long long)gridDim.x * kRopeThreads) {
        const int row = (int)(idx / half), i = (int)(idx - (long long)row * half);
        const float2 v = cos_sin_of(f.turns[i], pos[f.axis[i] * pos_axis_stride + row]);
        out[(size_t)row * 2 * half + i] = v.x;
        out[(size_t)row * 2 * half + half + i] = v.y;
    }
}

}  // namespace lar
