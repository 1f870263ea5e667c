// Chunk attention for fp32 storage.
//
// A CTA holds its query rows and walks the unit's slots 64 at a time; K of the next step is copied (cp.async) while this step's P V
// runs, V while the next step's S is formed.  Slots of a unit may be split over gridDim.z CTAs: they leave (O, m, l) in the
// workspace and combine_splits_kernel joins them.
//
// The products run on the tensor cores with every operand split in two tf32 numbers (see Tf32Shape), so that what fp32 storage is chosen for is
// kept.
#pragma once
#include <type_traits>

#include "decode_stream.cuh"  // ldmatrix, ex2_approx
#include "paged_attn.cuh"

namespace lar {

constexpr int kFp32Keys = 64;  // slots of a step
constexpr int kFp32Threads = 128;

// 16 bytes to shared memory, or zeros
__device__ __forceinline__ void copy16_async(float* dst, const float* src, bool live) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(smem_u32(dst)), "l"(src), "r"(live ? 16 : 0) : "memory");
}
__device__ __forceinline__ void copy_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void copy_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

// A pass over slots in common or over sequences' own (parts = 2) is launched before its predecessor's end: the first waits at its start for the kernel that
// makes the groups; of the second, which runs beside the first, one CTA waits at its end, so that who waits for this kernel's end has waited for
// both.
__device__ __forceinline__ void pass_begin(const PagedAttnArgs& a) {
    if (a.parts != 2) return;
    if (a.kv.row_of) grid_dep_wait();
    grid_dep_launch();
}
__device__ __forceinline__ void pass_end(const PagedAttnArgs& a) {
    if (a.parts == 2 && !a.kv.row_of && blockIdx.x == gridDim.x - 1 && blockIdx.y == gridDim.y - 1 && blockIdx.z == gridDim.z - 1) grid_dep_wait();
}

// The unit of a CTA: blockIdx.x counts the row tiles of all sequences, blockIdx.y the KV heads, blockIdx.z the splits.
struct Fp32Unit {
    int seq, head, tok0, n_tok, rows;  // tokens of the tile, (token, head of the group) rows
    int slot0, len, lo, hi;            // slot of its first token; live slots; slots [lo, hi) that any row sees
    int b0, b1;                        // this CTA's share of the steps
    const int* table;

    // Every warp for itself: running sum of the sequences' row tiles.
    __device__ __forceinline__ bool find(const PagedAttnArgs& a) {
        const int lane = threadIdx.x & 31;
        int tile = 0, before = 0;
        seq = -1;
        for (int base = 0; base < a.kv.n_seqs; base += 32) {
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
        if (seq < 0) return false;
        int t0, t1;
        chunk_of(a.kv, seq, t0, t1);
        tile = (t1 - t0 + a.tq - 1) / a.tq - 1 - tile;  // the tiles that see most first
        head = blockIdx.y;
        len = live_len(a.kv, seq, t1 - t0, threadIdx.x == 0 && blockIdx.y == 0 && blockIdx.z == 0 && !a.kv.row_of);
        tok0 = t0 + tile * a.tq;
        n_tok = min(a.tq, t1 - tok0);
        rows = n_tok * a.group;
        slot0 = len - (t1 - tok0);
        lo = a.start ? max(__ldcg(a.start + seq), 0) : 0;  // (from L2: a pass's are written by a kernel before the last)
        hi = a.causal ? min(len, slot0 + n_tok) : len;
        const int first = lo / kFp32Keys, end = hi > lo ? (hi + kFp32Keys - 1) / kFp32Keys : first;
        const int per = (end - first + a.n_splits - 1) / a.n_splits;
        b0 = min(end, first + (int)blockIdx.z * per);
        b1 = min(end, b0 + per);
        table = a.kv.table + (a.kv.row_of ? a.kv.row_of[seq] : seq) * a.kv.table_seq_stride + head * a.kv.table_head_stride;
        return true;
    }
    // The K or V rows of a step; slots outside [lo, hi) are zero whatever their memory holds.  16 slots at a time: they lie in one page, so
    // the table is read and the address formed once for them (one look-up per 16-byte piece cost as many instructions as the products).
    template <int D>
    __device__ __forceinline__ void fetch(const PagedAttnArgs& a, float* dst, int stride, const char* pool, int j0, bool report) const {
        constexpr int PIECES = D / 4, ROWS = kFp32Threads / PIECES;  // of a row; rows that the CTA copies at once
        const int c = threadIdx.x % PIECES, r0 = threadIdx.x / PIECES;
        const float* from = reinterpret_cast<const float*>(pool);
#pragma unroll
        for (int g = 0; g < kFp32Keys; g += 16) {
            const int first = j0 + g;
            const float* p = from;
            bool page_ok = false;
            if (first < hi && first + 16 > lo) {
                const int page = table[first >> a.kv.page_shift];
                page_ok = page >= 0 && page < a.kv.n_pages;
                if (page_ok) p += page * a.kv.page_stride + (first & (a.kv.page_tokens - 1)) * a.kv.row_stride + head * a.kv.head_stride + c * 4;
                else if (report && threadIdx.x == 0) paged_report(a.kv, kStPage);
            }
#pragma unroll
            for (int r = 0; r < 16; r += ROWS) {
                const int slot = first + r + r0;
                const bool live = page_ok && slot >= lo && slot < hi;
                copy16_async(dst + (g + r + r0) * stride + c * 4, live ? p + (r + r0) * a.kv.row_stride : from, live);
            }
        }
        copy_commit();
    }
    // The query rows; rows behind the tile's last are zero.  (Not committed: one group with the first K rows.)
    template <int D>
    __device__ __forceinline__ void fetch_q(const PagedAttnArgs& a, float* dst, int stride, int n) const {
        for (int i = threadIdx.x; i < n * (D / 4); i += blockDim.x) {
            const int r = i / (D / 4), c = i % (D / 4), t = r / a.group, g = r - t * a.group;
            const float* p = reinterpret_cast<const float*>(a.q.p);
            const bool live = r < rows;
            if (live) p += (long long)(tok0 + t) * a.q.token_stride + (head * a.group + g) * a.q.head_stride + c * 4;
            copy16_async(dst + r * stride + c * 4, p, live);
        }
    }
    __device__ __forceinline__ int last_slot(const PagedAttnArgs& a, int row) const {
        return row >= rows ? -1 : a.causal ? min(slot0 + row / a.group, len - 1) : len - 1;
    }
    // Where a row's result goes: its output row, or its place among the partial results.
    __device__ __forceinline__ size_t part_row(const PagedAttnArgs& a, int row) const {
        const int t = row / a.group, g = row - t * a.group, hq = a.kv.n_kv_heads * a.group;
        return ((size_t)blockIdx.z * a.kv.n_tokens + tok0 + t) * hq + head * a.group + g;
    }
    __device__ __forceinline__ float* out_row(const PagedAttnArgs& a, int row, int d) const {
        if (a.parts) return a.part_o + part_row(a, row) * d;
        const int t = row / a.group, g = row - t * a.group;
        return reinterpret_cast<float*>(a.out.p) + (long long)(tok0 + t) * a.out.token_stride + (head * a.group + g) * a.out.head_stride;
    }
    // The warps' parts (O, m, l of every row, PS floats each) into the result.
    template <int D, int WARPS, int ROWS, int PS>
    __device__ __forceinline__ void merge_warps(const PagedAttnArgs& a, const float* parts) const {
        for (int i = threadIdx.x; i < rows * (D / 2); i += kFp32Threads) {
            const int row = i / (D / 2), e = i % (D / 2) * 2;
            const float* p = parts + row * PS;
            float M = -INFINITY, L = 0.f, x = 0.f, y = 0.f;
#pragma unroll
            for (int w = 0; w < WARPS; ++w) M = fmaxf(M, p[w * ROWS * PS + D]);
            const float ref = softmax_ref(M);
#pragma unroll
            for (int w = 0; w < WARPS; ++w) {
                const float2 ml = *reinterpret_cast<const float2*>(p + w * ROWS * PS + D), v = *reinterpret_cast<const float2*>(p + w * ROWS * PS + e);
                const float f = ex2_approx((ml.x - ref) * a.scale_log2);
                L = fmaf(ml.y, f, L);
                x = fmaf(v.x, f, x);
                y = fmaf(v.y, f, y);
            }
            const float inv = a.parts ? 1.f : L > 0.f ? 1.0f / L : L;  // nothing seen: 0; NaN stays NaN
            *reinterpret_cast<float2*>(out_row(a, row, D) + e) = make_float2(x * inv, y * inv);
            if (a.parts && e == 0) *reinterpret_cast<float2*>(a.part_ml + part_row(a, row) * 2) = make_float2(M, L);
        }
    }
};

// x = hi + lo with hi the nearest tf32 (11 significant bits, off by 2^-11 at most) and lo exact in fp32, of which the tensor core takes
// the first 11 bits: hi + lo is x to 2^-21 of it.  A product is hi hi + hi lo + lo hi (lo lo is below 2^-22; mma.sync m16n8k8): three
// products where CUDA cores need one, at 276 TFLOP/s (measured) against 72: a third of that is still more, and a warp's
// 16 rows cost it no shared-memory traffic per multiply-add.  tcgen05 has about three times that rate for tf32
// (half of its bf16 rate) but wants the split operands in shared memory, K and V twice for every step: not built, not measured.
//
// FEW = false: a tile of 64 rows, 16 for each warp: S (16 x 64), O (16 x D), running maximum and sum in registers.  FEW = true (at
// most 16 rows, a decode step): every warp has all of them and a quarter of the step's slots, with a running maximum of its own; the four
// results are merged at the end.  Bound by the products, and with few rows by the cache's bytes.
// P goes from the accumulators of S straight into the A operand of P V: the operand's columns q and q + 4 (q = lane % 4) are taken to be
// slots 2 q and 2 q + 1 of a block of 8, the accumulator's own pair, and V's rows are read in that order.  Rows are padded by 16 bytes:
// neither the 8 x 4 blocks of ldmatrix nor the single words of V (slots 2 q, columns lane / 4) meet in a bank.
template <int D, bool FEW>
struct Tf32Shape {
    static constexpr int BM = FEW ? 16 : 64, WARPS = 4, THREADS = kFp32Threads, RS = D + 4;
    static constexpr int NB = FEW ? 2 : 8;  // blocks of 8 slots of a warp in a step
    static constexpr int SMEM = (BM + 2 * kFp32Keys) * RS * 4;
    static constexpr int PER_SM = D == 128 ? 2 : FEW ? 4 : 3;
};

// (integer rounding, not cvt.rna.tf32: conversions run at an eighth of the rate and would take longer than the products)
// round = kRoundTf32 is the above.  A finite number within half a step of fp32's largest is infinite when it is rounded up, and what comes of it NaN.  A CTA
// that finds NaN in its result therefore walks its slots once more with round = 0: hi is cut off to 11 bits, lo has up to 13, and hi + lo is x to 2^-21
// of it still (lo lo, below 2^-20, is left out as before).  If the NaN was in the data it comes out again.  (One token over 16 x 4288 slots of 64- and
// 128-element rows, 5 chunks of 400 tokens over 800 slots of 64: without 67.7, 117 and 196 us; as it is 67.9, 117 and 199; with the addend in a
// register instead of a second copy of the loop 67.4, 117 and 203; with a test of every number before it is split 71, 127 and 214.)
constexpr uint32_t kRoundTf32 = 0x1000u;
__device__ __forceinline__ void split_tf32(uint32_t x, uint32_t round, uint32_t& hi, uint32_t& lo) {
    hi = (x + round) & 0xffffe000u;
    lo = __float_as_uint(__uint_as_float(x) - __uint_as_float(hi));
}
// Whether a row sum or an output element is NaN or infinite in any thread of the CTA.
template <int N>
__device__ __forceinline__ bool any_not_finite(const float (&l)[2], const float (&o)[N][4]) {
    float z = l[0] * 0.f + l[1] * 0.f;
#pragma unroll
    for (int i = 0; i < N; ++i) z += (o[i][0] * 0.f + o[i][1] * 0.f) + (o[i][2] * 0.f + o[i][3] * 0.f);
    return __syncthreads_or(!(z == 0.f));
}
__device__ __forceinline__ void mma_tf32(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm volatile(
        "mma.sync.aligned.m16n8k8.row.col.f32.tf32.tf32.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// N products by one row operand.  The tensor core's accumulation cuts its sum off instead of rounding it (an fp32 sum of many
// products drifts towards zero: 2.4e-6 of the result where all 432 products of a row went into one accumulator), so the large products
// and the small ones have accumulators of their own, of few products each, and are added up with rounded additions.
template <int N>
__device__ __forceinline__ void mma_split(float (*big)[4], float (*small)[4], const uint32_t (&ah)[4], const uint32_t (&al)[4], const uint32_t (&b)[2 * N], uint32_t round) {
    uint32_t h[2 * N], l[2 * N];
#pragma unroll
    for (int i = 0; i < 2 * N; ++i) split_tf32(b[i], round, h[i], l[i]);
#pragma unroll
    for (int i = 0; i < N; ++i) mma_tf32(small[i], al, h[2 * i], h[2 * i + 1]);
#pragma unroll
    for (int i = 0; i < N; ++i) mma_tf32(big[i], ah, h[2 * i], h[2 * i + 1]);
#pragma unroll
    for (int i = 0; i < N; ++i) mma_tf32(small[i], ah, l[2 * i], l[2 * i + 1]);
}
template <int N>
__device__ __forceinline__ void clear_tiles(float (*c)[4]) {
#pragma unroll
    for (int i = 0; i < N; ++i) c[i][0] = c[i][1] = c[i][2] = c[i][3] = 0.f;
}

template <int D, bool FEW>
__global__ void __launch_bounds__(Tf32Shape<D, FEW>::THREADS, Tf32Shape<D, FEW>::PER_SM) paged_attn_tf32_kernel(const PagedAttnArgs a) {
    using S = Tf32Shape<D, FEW>;
    constexpr int RS = S::RS, NB = S::NB, GB = NB < 4 ? NB : 4;
    extern __shared__ __align__(16) float sm[];
    float* qs = sm;
    float* ks = qs + S::BM * RS;
    float* vs = ks + kFp32Keys * RS;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, quad = lane & 3, qrow = lane >> 2;
    Fp32Unit u;
    pass_begin(a);
    if (!u.find(a)) {
        pass_end(a);
        return;
    }
    u.fetch_q<D>(a, qs, RS, S::BM);
    const int row_w = FEW ? 0 : warp * 16, slot_w = FEW ? warp * 16 : 0;  // the warp's first row, first slot of a step
    const int row0 = row_w + qrow;  // this thread's rows: row0, row0 + 8
    const bool active = row_w < u.rows;
    const int last[2] = {u.last_slot(a, row0), u.last_slot(a, row0 + 8)};
    const int min_last = u.last_slot(a, 0);
    float m[2], l[2], o[D / 8][4];
    const uint32_t q_at = smem_u32(qs + (row_w + (lane & 15)) * RS + (lane >> 4) * 4);
    const uint32_t k_at = smem_u32(ks + (slot_w + (lane & 7) + (lane >> 4) * 8) * RS + ((lane >> 3) & 1) * 4);

    auto walk = [&](auto rounding) {  // the CTA's slots from the first to the last
        constexpr uint32_t round = decltype(rounding)::value;
        m[0] = m[1] = -INFINITY;
        l[0] = l[1] = 0.f;
        clear_tiles<D / 8>(o);
        if (u.b0 < u.b1) {
            u.fetch<D>(a, ks, RS, a.kv.k_pool, u.b0 * kFp32Keys, true);
            u.fetch<D>(a, vs, RS, a.kv.v_pool, u.b0 * kFp32Keys, false);
        }
        for (int b = u.b0; b < u.b1; ++b) {
            const int j0 = b * kFp32Keys;
            copy_wait<1>();  // K of this step (V may be on its way)
            __syncthreads();
            float s[NB][4];
            if (active) {
                float small[NB][4];
                clear_tiles<NB>(s);
                clear_tiles<NB>(small);
#pragma unroll 2
                for (int k = 0; k < D / 8; ++k) {
                    uint32_t x[4], ah[4], al[4];
                    ldmatrix_x4(q_at + k * 32, x);  // rows 0-7 | rows 8-15, elements 8 k .. + 3, then the next four
#pragma unroll
                    for (int e = 0; e < 4; ++e) split_tf32(x[e], round, ah[e], al[e]);
#pragma unroll
                    for (int i = 0; i < NB; i += GB) {
                        uint32_t y[2 * GB];  // blocks of 8 slots, two 4-element halves each
#pragma unroll
                        for (int e = 0; e < GB; e += 2) ldmatrix_x4(k_at + ((i + e) * 8 * RS + k * 8) * 4, reinterpret_cast<uint32_t(&)[4]>(y[2 * e]));
                        mma_split<GB>(s + i, small + i, ah, al, y, round);
                    }
                }
#pragma unroll
                for (int i = 0; i < NB; ++i)
#pragma unroll
                    for (int e = 0; e < 4; ++e) s[i][e] += small[i][e];
            }
            __syncthreads();  // K has been read
            if (b + 1 < u.b1) u.fetch<D>(a, ks, RS, a.kv.k_pool, j0 + kFp32Keys, true);
            else copy_commit();
            if (active) {
                if (j0 < u.lo || j0 + kFp32Keys - 1 > min_last) {
#pragma unroll
                    for (int i = 0; i < NB; ++i)
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const int slot = j0 + slot_w + i * 8 + 2 * quad + (e & 1);
                            if (slot < u.lo || slot > last[e >> 1]) s[i][e] = -INFINITY;
                        }
                }
#pragma unroll
                for (int r = 0; r < 2; ++r) {
                    float mx = -INFINITY;
#pragma unroll
                    for (int i = 0; i < NB; ++i) mx = fmaxf(mx, fmaxf(s[i][2 * r], s[i][2 * r + 1]));
                    mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 1));
                    mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 2));
                    const float mn = fmaxf(m[r], mx), ref = softmax_ref(mn);
                    const float corr = ex2_approx((m[r] - ref) * a.scale_log2);
                    m[r] = mn;
                    float sum = 0.f;
#pragma unroll
                    for (int i = 0; i < NB; ++i)
#pragma unroll
                        for (int e = 0; e < 2; ++e) {
                            s[i][2 * r + e] = ex2_approx((s[i][2 * r + e] - ref) * a.scale_log2);
                            sum += s[i][2 * r + e];
                        }
                    l[r] = l[r] * corr + sum;  // (this thread's slots: joined over the row's four threads at the end)
#pragma unroll
                    for (int i = 0; i < D / 8; ++i) {
                        o[i][2 * r] *= corr;
                        o[i][2 * r + 1] *= corr;
                    }
                }
            }
            copy_wait<1>();  // V of this step
            __syncthreads();
            if (active) {
#pragma unroll
                for (int n = 0; n < D / 8; n += 4) {  // four blocks of 8 columns at a time, summed over the step's slots on their own
                    float big[4][4], small[4][4];
                    clear_tiles<4>(big);
                    clear_tiles<4>(small);
#pragma unroll
                    for (int i = 0; i < NB; ++i) {
                        uint32_t ah[4], al[4];
                        split_tf32(__float_as_uint(s[i][0]), kRoundTf32, ah[0], al[0]);
                        split_tf32(__float_as_uint(s[i][2]), kRoundTf32, ah[1], al[1]);
                        split_tf32(__float_as_uint(s[i][1]), kRoundTf32, ah[2], al[2]);
                        split_tf32(__float_as_uint(s[i][3]), kRoundTf32, ah[3], al[3]);
                        const float* v = vs + (slot_w + i * 8 + 2 * quad) * RS + qrow + n * 8;
                        uint32_t y[8];
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            y[2 * e] = __float_as_uint(v[e * 8]);
                            y[2 * e + 1] = __float_as_uint(v[RS + e * 8]);
                        }
                        mma_split<4>(big, FEW ? big : small, ah, al, y, round);  // (FEW: two blocks, six products in all)
                    }
#pragma unroll
                    for (int i = 0; i < 4; ++i)
#pragma unroll
                        for (int e = 0; e < 4; ++e) o[n + i][e] += FEW ? big[i][e] : big[i][e] + small[i][e];
                }
            }
            __syncthreads();  // V has been read
            if (b + 1 < u.b1) u.fetch<D>(a, vs, RS, a.kv.v_pool, j0 + kFp32Keys, false);
            else copy_commit();
        }
        copy_commit();
        copy_wait<0>();  // (nothing is in flight when the CTA ends)
    };
    walk(std::integral_constant<uint32_t, kRoundTf32>());
    if (any_not_finite(l, o)) walk(std::integral_constant<uint32_t, 0>());
#pragma unroll
    for (int r = 0; r < 2; ++r) {
        l[r] += __shfl_xor_sync(0xffffffffu, l[r], 1);
        l[r] += __shfl_xor_sync(0xffffffffu, l[r], 2);
    }
    if constexpr (FEW) {
        // the warps' parts side by side where K was (everybody is behind the last step's barrier, no copy is in flight)
        constexpr int PS = D + 2;
        static_assert(S::WARPS * S::BM * PS <= kFp32Keys * RS, "the parts fit where K was");
        __syncthreads();
#pragma unroll
        for (int r = 0; r < 2; ++r) {
            float* p = ks + (warp * S::BM + row0 + 8 * r) * PS;
#pragma unroll
            for (int n = 0; n < D / 8; ++n) *reinterpret_cast<float2*>(p + n * 8 + 2 * quad) = make_float2(o[n][2 * r], o[n][2 * r + 1]);
            if (quad == 0) *reinterpret_cast<float2*>(p + D) = make_float2(m[r], l[r]);
        }
        __syncthreads();
        u.merge_warps<D, S::WARPS, S::BM, PS>(a, ks);
        pass_end(a);
        return;
    }
#pragma unroll
    for (int r = 0; r < 2; ++r) {
        const int row = row0 + 8 * r;
        if (row >= u.rows) continue;
        const float inv = a.parts ? 1.f : l[r] > 0.f ? 1.0f / l[r] : l[r];
        float* dst = u.out_row(a, row, D) + 2 * quad;
#pragma unroll
        for (int n = 0; n < D / 8; ++n) *reinterpret_cast<float2*>(dst + n * 8) = make_float2(o[n][2 * r] * inv, o[n][2 * r + 1] * inv);
        if (a.parts && quad == 0) *reinterpret_cast<float2*>(a.part_ml + u.part_row(a, row) * 2) = make_float2(m[r], l[r]);
    }
    pass_end(a);
}

// At most 8 rows of a KV head (a decode step).  The slots are the 16 rows of a product and the query rows its 8 columns (S^T = K q^T,
// O^T = V^T P^T), so that few products are padding; as above every warp has all query rows and a quarter of a step's slots.  Bound by
// the instructions that split K and V into tf32 numbers and by the cache's bytes (16 x 4288 slots, 8 KV heads of 4: 64-element rows 68 us
// against 81 of the 16-row kernel above, 128-element rows 117 = 4.8 TB/s against 159; two such column blocks for 9 to 16 rows took
// 95 us against 83 and 171 against 168).
// P^T comes out of the accumulators transposed in 16-bit halves (movmatrix); its operand rows q and q + 4 (q = lane % 4) are taken to be
// slots 2 q and 2 q + 1 of a block of 8.  The rows of V^T are taken in the order in which a lane finds four of them in 16 bytes.
template <int D>
struct Tf32DecodeShape {
    static constexpr int ROWS = 8, WARPS = 4, RS = D + 4, KS = D / 8;
    static constexpr int Q_FLOATS = KS * 32 * 4;  // the query rows as operands, split
    static constexpr int SMEM = (Q_FLOATS + 2 * kFp32Keys * RS) * 4;
    static constexpr int PER_SM = D == 128 ? 3 : 4;
};

template <int D>
__global__ void __launch_bounds__(kFp32Threads, Tf32DecodeShape<D>::PER_SM) paged_attn_tf32_decode_kernel(const PagedAttnArgs a) {
    using S = Tf32DecodeShape<D>;
    constexpr int RS = S::RS, KS = S::KS, OT = D / 16;
    extern __shared__ __align__(16) float sm[];
    uint4* qf = reinterpret_cast<uint4*>(sm);
    float* ks = sm + S::Q_FLOATS;
    float* vs = ks + kFp32Keys * RS;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, quad = lane & 3, qrow = lane >> 2;
    Fp32Unit u;
    pass_begin(a);
    if (!u.find(a)) {
        pass_end(a);
        return;
    }
    const int slot_w = warp * 16;  // the warp's first slot of a step
    const int last[2] = {u.last_slot(a, 2 * quad), u.last_slot(a, 2 * quad + 1)};
    float m[2], l[2], o[OT][4];
    const int min_last = u.last_slot(a, 0);
    const uint32_t k_at = smem_u32(ks + (slot_w + (lane & 15)) * RS + (lane >> 4) * 4);
    const float* v_at = vs + (slot_w + 2 * quad) * RS + 4 * qrow;

    auto walk = [&](auto rounding) {  // the CTA's slots from the first to the last
        constexpr uint32_t round = decltype(rounding)::value;
        m[0] = m[1] = -INFINITY;
        l[0] = l[1] = 0.f;
        clear_tiles<OT>(o);
        if (u.b0 < u.b1) {
            u.fetch<D>(a, ks, RS, a.kv.k_pool, u.b0 * kFp32Keys, true);
            u.fetch<D>(a, vs, RS, a.kv.v_pool, u.b0 * kFp32Keys, false);
        }
        // elements 8 k + quad and 8 k + quad + 4 of row qrow, the high parts, then the low ones; rows behind the last are zero
        for (int i = threadIdx.x; i < KS * 32; i += kFp32Threads) {
            const int l = i & 31, k = i >> 5, row = l >> 2;
            uint32_t x0 = 0, x1 = 0;
            if (row < u.rows) {
                const int t = row / a.group, g = row - t * a.group;
                const uint32_t* p = reinterpret_cast<const uint32_t*>(a.q.p) + (long long)(u.tok0 + t) * a.q.token_stride + (u.head * a.group + g) * a.q.head_stride + k * 8 + (l & 3);
                x0 = p[0];
                x1 = p[4];
            }
            uint4 f;
            split_tf32(x0, round, f.x, f.z);
            split_tf32(x1, round, f.y, f.w);
            qf[i] = f;
        }
        for (int b = u.b0; b < u.b1; ++b) {
            const int j0 = b * kFp32Keys;
            copy_wait<1>();  // K of this step (V may be on its way)
            __syncthreads();
            float s[4];
            {
                float big[2][4], small[4][4];  // (accumulators of few products, and chains short enough)
                clear_tiles<2>(big);
                clear_tiles<4>(small);
#pragma unroll 8
                for (int k = 0; k < KS; ++k) {
                    uint32_t x[4], ah[4], al[4];
                    ldmatrix_x4(k_at + k * 32, x);  // slots 0-7 | 8-15, elements 8 k .. + 3, then the next four
#pragma unroll
                    for (int e = 0; e < 4; ++e) split_tf32(x[e], round, ah[e], al[e]);
                    const uint4 q = qf[k * 32 + lane];
                    mma_tf32(small[k & 1], al, q.x, q.y);
                    mma_tf32(big[k & 1], ah, q.x, q.y);
                    mma_tf32(small[2 + (k & 1)], ah, q.z, q.w);
                }
#pragma unroll
                for (int e = 0; e < 4; ++e) s[e] = big[0][e] + big[1][e] + ((small[0][e] + small[1][e]) + (small[2][e] + small[3][e]));
            }
            __syncthreads();  // K has been read
            if (b + 1 < u.b1) u.fetch<D>(a, ks, RS, a.kv.k_pool, j0 + kFp32Keys, true);
            else copy_commit();
            // this thread: slots qrow (+ 8), rows 2 quad (+ 1)
            if (j0 < u.lo || j0 + kFp32Keys - 1 > min_last) {
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int slot = j0 + slot_w + qrow + (e >> 1) * 8;
                    if (slot < u.lo || slot > last[e & 1]) s[e] = -INFINITY;
                }
            }
            float corr[2];
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                float mx = fmaxf(s[e], s[2 + e]);
#pragma unroll
                for (int w = 4; w <= 16; w <<= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, w));
                const float mn = fmaxf(m[e], mx), ref = softmax_ref(mn);
                corr[e] = ex2_approx((m[e] - ref) * a.scale_log2);
                m[e] = mn;
                s[e] = ex2_approx((s[e] - ref) * a.scale_log2);
                s[2 + e] = ex2_approx((s[2 + e] - ref) * a.scale_log2);
                l[e] = l[e] * corr[e] + (s[e] + s[2 + e]);  // (this thread's slots: joined over the row's threads at the end)
            }
            uint32_t ph[2][2], pl[2][2];  // P^T of slots 0-7 | 8-15: slots 2 quad and 2 quad + 1 of row qrow
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const uint32_t x = __float_as_uint(s[2 * h]), y = __float_as_uint(s[2 * h + 1]);
                const uint32_t hi = movmatrix_trans(__byte_perm(x, y, 0x7632)), lo = movmatrix_trans(__byte_perm(x, y, 0x5410));
                split_tf32(__byte_perm(lo, hi, 0x5410), kRoundTf32, ph[h][0], pl[h][0]);
                split_tf32(__byte_perm(lo, hi, 0x7632), kRoundTf32, ph[h][1], pl[h][1]);
            }
            if (__any_sync(0xffffffffu, corr[0] != 1.f || corr[1] != 1.f)) {
#pragma unroll
                for (int i = 0; i < OT; ++i) {
                    o[i][0] *= corr[0];
                    o[i][1] *= corr[1];
                    o[i][2] *= corr[0];
                    o[i][3] *= corr[1];
                }
            }
            copy_wait<1>();  // V of this step
            __syncthreads();
#pragma unroll
            for (int g = 0; g < D / 32; ++g) {  // elements 32 g + 4 qrow .. + 3: rows qrow and qrow + 8 of two products
                float part[2][4];
                clear_tiles<2>(part);
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const uint4 v0 = *reinterpret_cast<const uint4*>(v_at + h * 8 * RS + g * 32);
                    const uint4 v1 = *reinterpret_cast<const uint4*>(v_at + (h * 8 + 1) * RS + g * 32);
                    const uint32_t x[2][4] = {{v0.x, v0.y, v1.x, v1.y}, {v0.z, v0.w, v1.z, v1.w}};
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        uint32_t ah[4], al[4];
#pragma unroll
                        for (int e = 0; e < 4; ++e) split_tf32(x[i][e], round, ah[e], al[e]);
                        mma_tf32(part[i], al, ph[h][0], ph[h][1]);  // (six products in all)
                        mma_tf32(part[i], ah, pl[h][0], pl[h][1]);
                        mma_tf32(part[i], ah, ph[h][0], ph[h][1]);
                    }
                }
#pragma unroll
                for (int i = 0; i < 2; ++i)
#pragma unroll
                    for (int e = 0; e < 4; ++e) o[2 * g + i][e] += part[i][e];
            }
            __syncthreads();  // V has been read
            if (b + 1 < u.b1) u.fetch<D>(a, vs, RS, a.kv.v_pool, j0 + kFp32Keys, false);
            else copy_commit();
        }
        copy_commit();
        copy_wait<0>();  // (nothing is in flight when the CTA ends)
    };
    walk(std::integral_constant<uint32_t, kRoundTf32>());
    if (any_not_finite(l, o)) walk(std::integral_constant<uint32_t, 0>());
    // the warps' parts side by side where K was
    constexpr int PS = D + 4;
    static_assert(S::WARPS * S::ROWS * PS <= kFp32Keys * RS, "the parts fit where K was");
    __syncthreads();
#pragma unroll
    for (int e = 0; e < 2; ++e) {
#pragma unroll
        for (int w = 4; w <= 16; w <<= 1) l[e] += __shfl_xor_sync(0xffffffffu, l[e], w);
        float* p = ks + (warp * S::ROWS + 2 * quad + e) * PS;
#pragma unroll
        for (int g = 0; g < D / 32; ++g)
            *reinterpret_cast<float4*>(p + g * 32 + 4 * qrow) = make_float4(o[2 * g][e], o[2 * g][2 + e], o[2 * g + 1][e], o[2 * g + 1][2 + e]);
        if (qrow == 0) *reinterpret_cast<float2*>(p + D) = make_float2(m[e], l[e]);
    }
    __syncthreads();
    u.merge_warps<D, S::WARPS, S::ROWS, PS>(a, ks);
    pass_end(a);
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
    const float ref = softmax_ref(M);
    float L = 0.f, o[PER];
#pragma unroll
    for (int i = 0; i < PER; ++i) o[i] = 0.f;
    for (int s = 0; s < a.n_splits; ++s) {
        const size_t at = (size_t)s * n_rows + row;
        const float f = exp2f((a.part_ml[at * 2] - ref) * a.scale_log2);
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
