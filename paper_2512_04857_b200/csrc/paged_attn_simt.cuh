// Chunk attention for fp32 storage, on the CUDA cores: the tensor cores take no fp32 operands, and rounding q, K and V
// to tf32 would lose what fp32 storage is chosen for.
//
// A CTA holds BM query rows and walks the unit's slots 64 at a time: S = Q K^T and O += P V as register tiles of 4 rows,
// operands in shared memory (Q and K transposed, so that a thread's 4 rows and its keys are vector loads), softmax with the
// running maximum and sum in fp32.  Bound: fp32 multiply-adds (64 rows), or, with BM = 16 for a few rows per
// sequence (a decode step), the cache bytes.  Slots of a unit may be split over gridDim.z CTAs (few rows, long cache): they
// leave (O, m, l) in the workspace and combine_splits_kernel joins them.
#pragma once
#include "paged_attn.cuh"

namespace lar {

constexpr int kSimtKeys = 64;

template <int D, int BM>
struct SimtShape {
    static constexpr int KG = BM == 64 ? 16 : 32;    // threads along the keys
    static constexpr int RG = BM / 4;                // threads along the rows, 4 rows each
    static constexpr int THREADS = KG * RG;
    static constexpr int KC = kSimtKeys / KG;        // keys of a thread
    static constexpr int OC = D / KG;                // output columns of a thread
    static constexpr int VC = OC < 4 ? OC : 4;       // ... in vectors of VC
    static constexpr int QS = BM + 4, KS = kSimtKeys + 4, PS = BM + 4;
    static constexpr int SMEM = (D * QS + D * KS + kSimtKeys * D + kSimtKeys * PS) * 4;
};

template <int N>
struct FVec;
template <> struct FVec<2> { using type = float2; };
template <> struct FVec<4> { using type = float4; };

template <int N>
__device__ __forceinline__ void load_vec(const float* p, float (&v)[N]) {
    *reinterpret_cast<typename FVec<N>::type*>(v) = *reinterpret_cast<const typename FVec<N>::type*>(p);
}

template <typename T, int D, int BM>
__global__ void __launch_bounds__(SimtShape<D, BM>::THREADS) paged_attn_simt_kernel(const PagedAttnArgs a) {
    using S = SimtShape<D, BM>;
    constexpr int E = Elt<T>::kPerChunk, CH = D / E;  // 16-byte chunks of a row
    extern __shared__ __align__(16) float sm[];
    float* qt = sm;                      // [D][QS]
    float* kt = qt + D * S::QS;          // [D][KS]
    float* vs = kt + D * S::KS;          // [64][D]
    float* pt = vs + kSimtKeys * D;      // [64][PS]

    const int tid = threadIdx.x, lane = tid & 31;
    const int kg = tid % S::KG, rg = tid / S::KG;
    const int head = blockIdx.y, G = a.group;

    // sequence and tile of this CTA: running sum of the sequences' row tiles
    int seq = -1, tile = 0;
    {
        int before = 0;
        for (int base = 0; base < a.kv.n_seqs; base += 32) {  // (every warp for itself)
            const int s = base + lane;
            const int n = s < a.kv.n_seqs ? tiles_of(a, s) : 0;
            int inc = n;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const int up = __shfl_up_sync(0xffffffffu, inc, o);
                if (lane >= o) inc += up;
            }
            const int x = (int)blockIdx.x - before;
            const unsigned hit = __ballot_sync(0xffffffffu, inc > x);
            if (hit) {
                const int l = __ffs(hit) - 1;
                seq = base + l;
                tile = x - __shfl_sync(0xffffffffu, inc - n, l);
                break;
            }
            before += __shfl_sync(0xffffffffu, inc, 31);
        }
    }
    if (seq < 0) return;
    int t0, t1;
    chunk_of(a.kv, seq, t0, t1);
    const int len = live_len(a.kv, seq);
    const int tok0 = t0 + tile * a.tq;                 // first token of the tile
    const int n_tok = min(a.tq, t1 - tok0);
    const int rows = n_tok * G;
    const int slot0 = len - (t1 - tok0);               // slot of the tile's first token
    const int lo = a.start ? max(a.start[seq], 0) : 0;
    const int hi = a.causal ? min(len, slot0 + n_tok) : len;
    // this CTA's share of the slots, in whole steps of 64
    const int b_lo = lo / kSimtKeys, b_hi = hi > lo ? (hi + kSimtKeys - 1) / kSimtKeys : b_lo;
    const int per = (b_hi - b_lo + a.n_splits - 1) / a.n_splits;
    const int b0 = min(b_hi, b_lo + (int)blockIdx.z * per), b1 = min(b_hi, b0 + per);

    // Q transposed; rows behind the tile's last are zero
    for (int i = tid; i < BM * CH; i += S::THREADS) {
        const int r = i % BM, c = i / BM;
        float f[E];
#pragma unroll
        for (int e = 0; e < E; ++e) f[e] = 0.f;
        if (r < rows) {
            const int t = r / G, g = r - t * G;
            const T* p = reinterpret_cast<const T*>(a.q.p) + (long long)(tok0 + t) * a.q.token_stride + (head * G + g) * a.q.head_stride;
            Elt<T>::unpack(*reinterpret_cast<const uint4*>(p + c * E), f);
        }
#pragma unroll
        for (int e = 0; e < E; ++e) qt[(c * E + e) * S::QS + r] = f[e];
    }

    float o[4][S::OC], m[4], l[4];
    int last[4];  // last slot each row sees
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        m[r] = -INFINITY;
        l[r] = 0.f;
        const int row = rg * 4 + r;
        last[r] = row >= rows ? -1 : a.causal ? min(slot0 + row / G, len - 1) : len - 1;
#pragma unroll
        for (int i = 0; i < S::OC; ++i) o[r][i] = 0.f;
    }

    for (int b = b0; b < b1; ++b) {
        const int j0 = b * kSimtKeys;
        __syncthreads();  // the previous step's tiles have been read
        // K and V rows of the step; slots outside [lo, hi) are zero whatever their memory holds
        for (int i = tid; i < kSimtKeys * CH; i += S::THREADS) {
            const int j = i % kSimtKeys, c = i / kSimtKeys, slot = j0 + j;
            float fk[E], fv[E];
#pragma unroll
            for (int e = 0; e < E; ++e) fk[e] = fv[e] = 0.f;
            if (slot >= lo && slot < hi) {
                const int page = a.kv.table[seq * a.kv.table_seq_stride + head * a.kv.table_head_stride + (slot >> a.kv.page_shift)];
                if (page >= 0 && page < a.kv.n_pages) {
                    const long long off = page * a.kv.page_stride + (slot & (a.kv.page_tokens - 1)) * a.kv.row_stride + head * a.kv.head_stride + c * E;
                    Elt<T>::unpack(*reinterpret_cast<const uint4*>(reinterpret_cast<const T*>(a.kv.k_pool) + off), fk);
                    Elt<T>::unpack(*reinterpret_cast<const uint4*>(reinterpret_cast<const T*>(a.kv.v_pool) + off), fv);
                } else if (c == 0) {
                    paged_report(a.kv, kStPage);
                }
            }
#pragma unroll
            for (int e = 0; e < E; ++e) {
                kt[(c * E + e) * S::KS + j] = fk[e];
                vs[j * D + c * E + e] = fv[e];
            }
        }
        __syncthreads();
        float s[4][S::KC];
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
            for (int k = 0; k < S::KC; ++k) s[r][k] = 0.f;
#pragma unroll 8
        for (int d = 0; d < D; ++d) {
            float qv[4], kv[S::KC];
            load_vec(qt + d * S::QS + rg * 4, qv);
            load_vec(kt + d * S::KS + kg * S::KC, kv);
#pragma unroll
            for (int r = 0; r < 4; ++r)
#pragma unroll
                for (int k = 0; k < S::KC; ++k) s[r][k] = fmaf(qv[r], kv[k], s[r][k]);
        }
        float p[S::KC][4];
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            float mx = -INFINITY;
#pragma unroll
            for (int k = 0; k < S::KC; ++k) {
                const int slot = j0 + kg * S::KC + k;
                s[r][k] = slot >= lo && slot <= last[r] ? s[r][k] * a.scale_log2 : -INFINITY;
                mx = fmaxf(mx, s[r][k]);
            }
#pragma unroll
            for (int w = S::KG / 2; w >= 1; w >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, w));
            const float mn = fmaxf(m[r], mx), ref = mn == -INFINITY ? 0.f : mn;  // (a row that has seen nothing yet)
            const float corr = exp2f(m[r] - ref);
            m[r] = mn;
            float sum = 0.f;
#pragma unroll
            for (int k = 0; k < S::KC; ++k) {
                p[k][r] = exp2f(s[r][k] - ref);
                sum += p[k][r];
            }
            l[r] = l[r] * corr + sum;  // (this thread's keys only: joined over the threads of the row at the end)
#pragma unroll
            for (int i = 0; i < S::OC; ++i) o[r][i] *= corr;
        }
#pragma unroll
        for (int k = 0; k < S::KC; ++k)
            *reinterpret_cast<float4*>(pt + (kg * S::KC + k) * S::PS + rg * 4) = make_float4(p[k][0], p[k][1], p[k][2], p[k][3]);
        // the threads that share these rows lie in one warp: their part of P is visible after a warp barrier
        __syncwarp();
#pragma unroll 4
        for (int j = 0; j < kSimtKeys; ++j) {
            float pv[4];
            load_vec(pt + j * S::PS + rg * 4, pv);
#pragma unroll
            for (int i = 0; i < S::OC / S::VC; ++i) {
                float vv[S::VC];
                load_vec(vs + j * D + i * (S::KG * S::VC) + kg * S::VC, vv);
#pragma unroll
                for (int r = 0; r < 4; ++r)
#pragma unroll
                    for (int e = 0; e < S::VC; ++e) o[r][i * S::VC + e] = fmaf(pv[r], vv[e], o[r][i * S::VC + e]);
            }
        }
    }
#pragma unroll
    for (int r = 0; r < 4; ++r) {
#pragma unroll
        for (int w = S::KG / 2; w >= 1; w >>= 1) l[r] += __shfl_xor_sync(0xffffffffu, l[r], w);
        const int row = rg * 4 + r;
        if (row >= rows) continue;
        const int t = row / G, g = row - t * G;
        if (a.n_splits > 1) {
            const size_t at = (size_t)blockIdx.z * a.kv.n_tokens * a.kv.n_kv_heads * G + (size_t)(tok0 + t) * a.kv.n_kv_heads * G + head * G + g;
#pragma unroll
            for (int i = 0; i < S::OC; ++i) a.part_o[at * D + (i / S::VC) * (S::KG * S::VC) + kg * S::VC + i % S::VC] = o[r][i];
            if (kg == 0) {
                a.part_ml[at * 2] = m[r];
                a.part_ml[at * 2 + 1] = l[r];
            }
        } else {
            const float inv = l[r] > 0.f ? 1.0f / l[r] : l[r];  // nothing seen: 0; NaN stays NaN
            T* dst = reinterpret_cast<T*>(a.out.p) + (long long)(tok0 + t) * a.out.token_stride + (head * G + g) * a.out.head_stride;
#pragma unroll
            for (int i = 0; i < S::OC; ++i) dst[(i / S::VC) * (S::KG * S::VC) + kg * S::VC + i % S::VC] = Elt<T>::from_float(o[r][i] * inv);
        }
    }
}

// Joins the splits of every row, in the order of the splits: one warp per (token, head).
template <typename T, int D>
__global__ void __launch_bounds__(128) combine_splits_kernel(const PagedAttnArgs a) {
    constexpr int PER = D / 32;
    const int hq = a.kv.n_kv_heads * a.group, lane = threadIdx.x & 31;
    const long long n_rows = (long long)a.kv.n_tokens * hq, row = (long long)blockIdx.x * 4 + (threadIdx.x >> 5);
    if (row >= n_rows) return;
    const int t = (int)(row / hq), h = (int)(row - (long long)t * hq);
    if (a.kv.cu && (t < a.kv.cu[0] || t >= a.kv.cu[a.kv.n_seqs])) return;  // no sequence's token: left as it was
    float M = -INFINITY;
    for (int s = 0; s < a.n_splits; ++s) M = fmaxf(M, a.part_ml[((size_t)s * n_rows + row) * 2]);
    const float ref = M == -INFINITY ? 0.f : M;
    float L = 0.f, o[PER];
#pragma unroll
    for (int i = 0; i < PER; ++i) o[i] = 0.f;
    for (int s = 0; s < a.n_splits; ++s) {
        const size_t at = (size_t)s * n_rows + row;
        const float f = exp2f(a.part_ml[at * 2] - ref);
        L = fmaf(a.part_ml[at * 2 + 1], f, L);
#pragma unroll
        for (int i = 0; i < PER; ++i) o[i] = fmaf(a.part_o[at * D + i * 32 + lane], f, o[i]);
    }
    const float inv = L > 0.f ? 1.0f / L : L;
    T* dst = reinterpret_cast<T*>(a.out.p) + (long long)t * a.out.token_stride + h * a.out.head_stride;
#pragma unroll
    for (int i = 0; i < PER; ++i) dst[i * 32 + lane] = Elt<T>::from_float(o[i] * inv);
}

}  // namespace lar
