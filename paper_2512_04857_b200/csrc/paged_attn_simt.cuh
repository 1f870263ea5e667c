// Chunk attention for fp32 storage, on the CUDA cores: the tensor cores take no fp32 operands, and rounding q, K and V
// to tf32 would lose what fp32 storage is chosen for.
//
// A CTA holds BM query rows and walks the unit's slots 64 at a time: S = Q K^T and O += P V as register tiles of RT rows by KC keys
// (columns), operands row by row in shared memory, softmax with the running maximum and sum in fp32.  Rows of Q and K are padded
// by 16 bytes, so that the 16-byte loads of the lanes of a quarter warp (8 keys) fall into different banks.  Bound: fp32 multiply-adds
// and the shared-memory loads that feed them (64 rows; 8 rows a thread where registers and shared memory allow three CTAs per SM), or, with BM = 16
// for a few rows per sequence (a decode step), the cache bytes.  K of the next step is copied (cp.async) while this step's P V
// runs, V while the next step's S is formed.  Slots of a unit may be split over gridDim.z CTAs (few rows, long cache): they leave
// (O, m, l) in the workspace and combine_splits_kernel joins them.
#pragma once
#include "paged_attn.cuh"

namespace lar {

constexpr int kSimtKeys = 64;

template <int D, int BM>
struct SimtShape {
    // rows of a thread: rg, rg + RG, ... (two neighbours in a warp, so that their loads fall into different banks)
    static constexpr int RT = BM == 64 && D == 64 ? 8 : 4;
    static constexpr int KG = BM == 64 ? 16 : 32;    // threads along the keys
    static constexpr int RG = BM / RT;               // threads along the rows
    static constexpr int THREADS = KG * RG;
    static constexpr int KC = kSimtKeys / KG;        // keys of a thread: kg, kg + KG, ...
    static constexpr int OC = D / KG;                // output columns of a thread
    static constexpr int VC = OC < 4 ? OC : 4;       // ... in vectors of VC
    static constexpr int QS = D + 4, KS = D + 4, PS = BM + 4;
    static constexpr int SMEM = (BM * QS + kSimtKeys * KS + kSimtKeys * D + kSimtKeys * PS) * 4;
};

template <int N>
struct FVec;
template <> struct FVec<2> { using type = float2; };
template <> struct FVec<4> { using type = float4; };

template <int N>
__device__ __forceinline__ void load_vec(const float* p, float* v) {
    *reinterpret_cast<typename FVec<N>::type*>(v) = *reinterpret_cast<const typename FVec<N>::type*>(p);
}
// 16 bytes to shared memory, or zeros
__device__ __forceinline__ void copy16_async(float* dst, const float* src, bool live) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(smem_u32(dst)), "l"(src), "r"(live ? 16 : 0) : "memory");
}
__device__ __forceinline__ void copy_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void copy_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

template <int D, int BM>
__global__ void __launch_bounds__(SimtShape<D, BM>::THREADS, SimtShape<D, BM>::RT == 8 ? 3 : 1) paged_attn_simt_kernel(const PagedAttnArgs a) {
    using S = SimtShape<D, BM>;
    constexpr int CH = D / 4, RT = S::RT;  // 16-byte chunks of a row
    extern __shared__ __align__(16) float sm[];
    float* qs = sm;                      // [BM][QS]
    float* ks = qs + BM * S::QS;         // [64][KS]
    float* vs = ks + kSimtKeys * S::KS;  // [64][D]
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
    tile = (t1 - t0 + a.tq - 1) / a.tq - 1 - tile;     // the tiles that see most first
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

    const int* table = a.kv.table + seq * a.kv.table_seq_stride + head * a.kv.table_head_stride;
    // the K or V rows of a step; slots outside [lo, hi) are zero whatever their memory holds
    auto fetch = [&](float* dst, int stride, const char* pool, int j0, bool report) {
        for (int i = tid; i < kSimtKeys * CH; i += S::THREADS) {
            const int j = i / CH, c = i % CH, slot = j0 + j;
            const float* src = reinterpret_cast<const float*>(pool);
            bool live = slot >= lo && slot < hi;
            if (live) {
                const int page = table[slot >> a.kv.page_shift];
                live = page >= 0 && page < a.kv.n_pages;
                if (live) src += page * a.kv.page_stride + (slot & (a.kv.page_tokens - 1)) * a.kv.row_stride + head * a.kv.head_stride + c * 4;
                else if (report && c == 0) paged_report(a.kv, kStPage);
            }
            copy16_async(dst + j * stride + c * 4, src, live);
        }
        copy_commit();
    };
    // Q; rows behind the tile's last are zero
    for (int i = tid; i < BM * CH; i += S::THREADS) {
        const int r = i / CH, c = i % CH, t = r / G, g = r - t * G;
        const float* p = reinterpret_cast<const float*>(a.q.p);
        const bool live = r < rows;
        if (live) p += (long long)(tok0 + t) * a.q.token_stride + (head * G + g) * a.q.head_stride + c * 4;
        copy16_async(qs + r * S::QS + c * 4, p, live);
    }
    if (b0 < b1) {
        fetch(ks, S::KS, a.kv.k_pool, b0 * kSimtKeys, true);   // (with Q: one group)
        fetch(vs, D, a.kv.v_pool, b0 * kSimtKeys, false);
    }

    uint64_t o[RT][S::OC / 2];  // pairs of columns
    float m[RT], l[RT];
    int last[RT];  // last slot each row sees
#pragma unroll
    for (int r = 0; r < RT; ++r) {
        m[r] = -INFINITY;
        l[r] = 0.f;
        const int row = rg + S::RG * r;
        last[r] = row >= rows ? -1 : a.causal ? min(slot0 + row / G, len - 1) : len - 1;
#pragma unroll
        for (int i = 0; i < S::OC / 2; ++i) o[r][i] = 0;
    }

    for (int b = b0; b < b1; ++b) {
        const int j0 = b * kSimtKeys;
        copy_wait<1>();   // K of this step (V may be on its way)
        __syncthreads();
        float s[RT][S::KC];
        {
            uint64_t acc[RT][S::KC];  // sums over the even and the odd elements of a row
#pragma unroll
            for (int r = 0; r < RT; ++r)
#pragma unroll
                for (int k = 0; k < S::KC; ++k) acc[r][k] = 0;
#pragma unroll 2
            for (int d = 0; d < D; d += 4) {
                ulonglong2 kv[S::KC];
#pragma unroll
                for (int k = 0; k < S::KC; ++k) kv[k] = *reinterpret_cast<const ulonglong2*>(ks + (kg + k * S::KG) * S::KS + d);
#pragma unroll
                for (int r = 0; r < RT; ++r) {
                    const ulonglong2 qv = *reinterpret_cast<const ulonglong2*>(qs + (rg + S::RG * r) * S::QS + d);
#pragma unroll
                    for (int k = 0; k < S::KC; ++k) acc[r][k] = fma_f32x2(qv.y, kv[k].y, fma_f32x2(qv.x, kv[k].x, acc[r][k]));
                }
            }
#pragma unroll
            for (int r = 0; r < RT; ++r)
#pragma unroll
                for (int k = 0; k < S::KC; ++k) {
                    float even, odd;
                    unpack_f32x2(acc[r][k], even, odd);
                    s[r][k] = even + odd;
                }
        }
        __syncthreads();  // K has been read
        if (b + 1 < b1) fetch(ks, S::KS, a.kv.k_pool, j0 + kSimtKeys, true);
        else copy_commit();
#pragma unroll
        for (int r = 0; r < RT; ++r) {
            float mx = -INFINITY;
#pragma unroll
            for (int k = 0; k < S::KC; ++k) {
                const int slot = j0 + kg + k * S::KG;
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
                s[r][k] = exp2f(s[r][k] - ref);
                sum += s[r][k];
            }
            l[r] = l[r] * corr + sum;  // (this thread's keys only: joined over the threads of the row at the end)
#pragma unroll
            for (int i = 0; i < S::OC / 2; ++i) o[r][i] = mul_f32x2(o[r][i], pack_f32x2(corr, corr));
        }
#pragma unroll
        for (int k = 0; k < S::KC; ++k)
#pragma unroll
            for (int r = 0; r < RT; r += 4)
                *reinterpret_cast<float4*>(pt + (kg + k * S::KG) * S::PS + rg * RT + r) = make_float4(s[r][k], s[r + 1][k], s[r + 2][k], s[r + 3][k]);
        copy_wait<1>();   // V of this step
        __syncthreads();
#pragma unroll 4
        for (int j = 0; j < kSimtKeys; ++j) {
            float pv[RT];
#pragma unroll
            for (int r = 0; r < RT; r += 4) load_vec<4>(pt + j * S::PS + rg * RT + r, pv + r);
#pragma unroll
            for (int i = 0; i < S::OC / S::VC; ++i) {
                uint64_t vv[S::VC / 2];
                load_vec<S::VC>(vs + j * D + i * (S::KG * S::VC) + kg * S::VC, reinterpret_cast<float*>(vv));
#pragma unroll
                for (int r = 0; r < RT; ++r)
#pragma unroll
                    for (int e = 0; e < S::VC / 2; ++e)
                        o[r][i * (S::VC / 2) + e] = fma_f32x2(pack_f32x2(pv[r], pv[r]), vv[e], o[r][i * (S::VC / 2) + e]);
            }
        }
        __syncthreads();  // V and P have been read
        if (b + 1 < b1) fetch(vs, D, a.kv.v_pool, j0 + kSimtKeys, false);
        else copy_commit();
    }
    copy_commit();
    copy_wait<0>();  // (nothing is in flight when the CTA ends)
#pragma unroll
    for (int r = 0; r < RT; ++r) {
#pragma unroll
        for (int w = S::KG / 2; w >= 1; w >>= 1) l[r] += __shfl_xor_sync(0xffffffffu, l[r], w);
        const int row = rg + S::RG * r;
        if (row >= rows) continue;
        const int t = row / G, g = row - t * G;
        const size_t at = (size_t)blockIdx.z * a.kv.n_tokens * a.kv.n_kv_heads * G + (size_t)(tok0 + t) * a.kv.n_kv_heads * G + head * G + g;
        float* dst = a.n_splits > 1 ? a.part_o + at * D
                                    : reinterpret_cast<float*>(a.out.p) + (long long)(tok0 + t) * a.out.token_stride + (head * G + g) * a.out.head_stride;
        const float inv = a.n_splits > 1 ? 1.f : l[r] > 0.f ? 1.0f / l[r] : l[r];  // nothing seen: 0; NaN stays NaN
#pragma unroll
        for (int i = 0; i < S::OC / S::VC; ++i) {
            typename FVec<S::VC>::type v;
#pragma unroll
            for (int e = 0; e < S::VC / 2; ++e) {
                float x, y;
                unpack_f32x2(o[r][i * (S::VC / 2) + e], x, y);
                reinterpret_cast<float*>(&v)[2 * e] = x * inv;
                reinterpret_cast<float*>(&v)[2 * e + 1] = y * inv;
            }
            *reinterpret_cast<typename FVec<S::VC>::type*>(dst + i * (S::KG * S::VC) + kg * S::VC) = v;
        }
        if (a.n_splits > 1 && kg == 0) {
            a.part_ml[at * 2] = m[r];
            a.part_ml[at * 2 + 1] = l[r];
        }
    }
}

// Joins the splits of every row, in the order of the splits: one warp per (token, head).
template <int D>
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
    float* dst = reinterpret_cast<float*>(a.out.p) + (long long)t * a.out.token_stride + h * a.out.head_stride;
#pragma unroll
    for (int i = 0; i < PER; ++i) dst[i * 32 + lane] = o[i] * inv;
}

}  // namespace lar
