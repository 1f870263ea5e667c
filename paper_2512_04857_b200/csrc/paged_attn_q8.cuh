// Attention over an 8-bit paged cache (paged_q8.cuh) for at most 16 (token, head of the group) rows of a KV head per unit: single tokens and
// short candidate chunks.  Bound by the cache's bytes; one step below, by what turns codes into operands.
//
// The layout of work is that of paged_attn_few.cuh: every consumer warp takes a tile of 32 slots through S^T = K q^T and O^T += V^T P^T with
// mma.sync (the slots as the rows of the product), a producer warp keeps a ring of K/V tiles full, an epilogue warp merges the warps'
// partial results.  What 8 bits change:
//   * Codes go to fp16, which holds every e4m3 number: one conversion for two of them, no scale applied.  A row's scale is a power of two that belongs to a
//     slot, so K's multiplies the slot's logits and V's the slot's weights; no element is ever multiplied.
//   * The elements of a row may be contracted in any order, so a thread takes the four neighbouring codes that ldmatrix gives it as elements 2t,
//     2t + 1, 2t + 8, 2t + 9 of the product, and q's fragments are loaded to match.  V^T comes from ldmatrix.trans on pairs of codes: rows g and g + 8 of a
//     product are elements 2g and 2g + 1.
//   * q is scaled by a power of two to 2^8 .. 2^9 per row (exact in fp16 down to 2^-22 of the row's largest element, off by 2^-33 of it below).  fp32
//     rows take two fp16 numbers for q and for the weights (22 bits), and sums of a tile are added to the accumulator with rounding.
//   * A weight is p_j 2^(v_j), v_j the exponent of the slot's values.  fp16 has 5 bits of exponent, so each row keeps a reference vr of its own, the
//     largest (logit - m) log2(e) scale + v_j so far: weights are at most 2^14, and what fp16 cannot hold is below 2^-38 of the row's largest weight.
#pragma once
#include <cuda_fp16.h>

#include "paged_attn_tc.cuh"
#include "paged_q8.cuh"

namespace lar {

constexpr int kQ8Rows = 16;  // rows of a unit up to which the kernel below is taken

template <typename T, int D, int NR>
struct Q8Shape {
    static constexpr int KT = 32;                 // slots of a tile
    static constexpr int TERMS = sizeof(T) == 4 ? 2 : 1;
    static constexpr int MT = KT / 16, KS = D / 16;
    static constexpr int TILE_BYTES = KT * D, STAGE_BYTES = 2 * TILE_BYTES, SCALE_BYTES = 2 * KT;
    static constexpr int W = 4, THREADS = (W + 2) * 32;  // producer, consumers, epilogue
    static constexpr int NS = 8;                  // stages: a multiple of W, a stage is always read by the same consumer
    static constexpr int PER_SM = 2;
    static constexpr int ROWS = 8 * NR;
    static constexpr int Q_SLOT = ROWS * D * (int)sizeof(T);
    static constexpr int PS = D + 4;              // floats of a partial row: O, m, l, padding
    static constexpr int PBUFS = NR == 1 ? 2 : 1;
    static constexpr int PBUF_FLOATS = W * ROWS * PS;
    static constexpr int FIXED = 1024 + NS * (STAGE_BYTES + SCALE_BYTES) + 2 * Q_SLOT + PBUFS * PBUF_FLOATS * 4 + 32 * 8;
    static __host__ __device__ int bytes(int n_seqs) { return FIXED + n_seqs * 16 + 2 * (n_seqs + 1) * 4 + 16 * 4; }
};

struct Q8Maps {
    CUtensorMap q;     // {d, heads of a group, KV heads, tokens}, box d x group x 1 x tq, rows of T
    CUtensorMap k, v;  // {d, rows of a page, heads, pages} of bytes, box d x min(page, 32) x 1 x 1, swizzled by d bytes
};

// Two fp16 numbers from each half of four codes.
__device__ __forceinline__ void q8_halves(uint32_t codes, uint32_t& lo, uint32_t& hi) {
    asm("{\n .reg .b16 a, b;\n mov.b32 {a, b}, %2;\n cvt.rn.f16x2.e4m3x2 %0, a;\n cvt.rn.f16x2.e4m3x2 %1, b;\n}\n" : "=r"(lo), "=r"(hi) : "r"(codes));
}
__device__ __forceinline__ void mma_f16(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t pack_f16(float lo, float hi) {
    __half2 t = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<uint32_t*>(&t);
}
__device__ __forceinline__ float2 unpack_f16(uint32_t v) { return __half22float2(*reinterpret_cast<__half2*>(&v)); }

template <typename T>
struct OutRow;
template <>
struct OutRow<__nv_bfloat16> {
    static __device__ __forceinline__ void put(char* p, long long at, float4 o, float f) {
        *reinterpret_cast<uint2*>(p + at * 2) = make_uint2(pack_bf16(o.x * f, o.y * f), pack_bf16(o.z * f, o.w * f));
    }
    static __device__ __forceinline__ float4 get(const unsigned char* p) {  // four elements
        const uint2 v = *reinterpret_cast<const uint2*>(p);
        return make_float4(__uint_as_float(v.x << 16), __uint_as_float(v.x & 0xffff0000u), __uint_as_float(v.y << 16), __uint_as_float(v.y & 0xffff0000u));
    }
};
template <>
struct OutRow<float> {
    static __device__ __forceinline__ void put(char* p, long long at, float4 o, float f) {
        *reinterpret_cast<float4*>(p + at * 4) = make_float4(o.x * f, o.y * f, o.z * f, o.w * f);
    }
    static __device__ __forceinline__ float4 get(const unsigned char* p) { return *reinterpret_cast<const float4*>(p); }
};

template <typename T, int D, int NR>
__global__ void __launch_bounds__(Q8Shape<T, D, NR>::THREADS, Q8Shape<T, D, NR>::PER_SM)
paged_attn_q8_kernel(const __grid_constant__ TcArgs ta, const __grid_constant__ Q8View q8, const __grid_constant__ Q8Maps maps) {
    using S = Q8Shape<T, D, NR>;
    using Work = TcWork<1, S::KT, D>;
    constexpr int KT = S::KT, W = S::W, NS = S::NS, TERMS = S::TERMS, KS = S::KS, MT = S::MT;
    const PagedAttnArgs& a = ta.a;
    extern __shared__ unsigned char smem_raw[];
    const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    unsigned char* gbase = smem_raw + (base - smem_u32(smem_raw));
    const uint32_t ring = base, scales = base + NS * S::STAGE_BYTES;
    unsigned char* gscales = gbase + NS * S::STAGE_BYTES;   // per stage: KT bytes of K, KT of V
    unsigned char* gq = gscales + NS * S::SCALE_BYTES;
    const uint32_t qring = scales + NS * S::SCALE_BYTES;
    float* pbuf = reinterpret_cast<float*>(gq + 2 * S::Q_SLOT);
    uint64_t* bars = reinterpret_cast<uint64_t*>(pbuf + S::PBUFS * S::PBUF_FLOATS);
    const uint32_t bar0 = smem_u32(bars);
    auto full = [&](int st) { return bar0 + 8u * st; };
    auto empty = [&](int st) { return bar0 + 8u * (8 + st); };
    auto q_full = [&](int i) { return bar0 + 8u * (16 + i); };
    auto q_empty = [&](int i) { return bar0 + 8u * (18 + i); };
    auto p_full = [&](int i) { return bar0 + 8u * (20 + i); };
    auto p_empty = [&](int i) { return bar0 + 8u * (22 + i); };
    volatile int* abort_flag = reinterpret_cast<volatile int*>(bars + 24);
    SeqInfo* info = reinterpret_cast<SeqInfo*>(bars + 32);
    int* pre = reinterpret_cast<int*>(info + a.kv.n_seqs);
    int* wsum = pre + 2 * (a.kv.n_seqs + 1);

    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    if (tid == 0) {
        for (int i = 0; i < NS; ++i) {
            mbar_init(full(i), 1);
            mbar_init(empty(i), 1);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(q_full(i), 1);
            mbar_init(q_empty(i), W);
            mbar_init(p_full(i), W);
            mbar_init(p_empty(i), 1);
        }
        *abort_flag = 0;
        mbar_fence_init_smem();
    }
    if (ta.split) grid_dep_launch();  // (the joining kernel waits for this one's end)
    // units, or slot tiles where units may be cut, before each sequence
    {
        const int per = (a.kv.n_seqs + S::THREADS - 1) / S::THREADS, s0 = tid * per, s1 = min(s0 + per, a.kv.n_seqs);
        int sum = 0;
        for (int s = s0; s < s1; ++s) {
            SeqInfo v;
            int t1;
            chunk_of(a.kv, s, v.t0, t1);
            v.n = t1 - v.t0;
            v.len = live_len(a.kv, s, v.n, blockIdx.x == 0);
            v.lo = a.start ? max(a.start[s], 0) : 0;
            info[s] = v;
            sum += (v.n + a.tq - 1) / a.tq * a.kv.n_kv_heads * (ta.split ? Work::items_of_unit(v) : 1);
            pre[s + 1] = sum;
        }
        int inc = sum;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int up = __shfl_up_sync(0xffffffffu, inc, o);
            if (lane >= o) inc += up;
        }
        if (lane == 31) wsum[warp] = inc;
        __syncthreads();
        int before = inc - sum;
        for (int w = 0; w < warp; ++w) before += wsum[w];
        for (int s = s0; s < s1; ++s) pre[s + 1] += before;
        if (tid == 0) pre[0] = 0;
        __syncthreads();
    }
    Work work;
    work.info = info;
    work.pre = work.items = pre;
    work.n_seqs = a.kv.n_seqs;
    work.tq = a.tq;
    work.causal = a.causal;
    work.x = blockIdx.x;
    work.step = gridDim.x;
    work.end = ta.split ? 0 : pre[a.kv.n_seqs];
    work.first_cut = 0;
    work.y = work.y_end = 0;
    const int total = ta.split ? pre[a.kv.n_seqs] : 0;
    const int n_ranges = min((total + ta.min_items - 1) / ta.min_items, (int)gridDim.x);
    if ((int)blockIdx.x < n_ranges) {
        work.y = (int)((long long)total * blockIdx.x / n_ranges);
        work.y_end = (int)((long long)total * (blockIdx.x + 1) / n_ranges);
    }

    if (warp == 0) {
        // ------------------------------------------------------------------ producer: lanes 0, 1 K and 2, 3 V, a page (or part of one) each
        int issued = 0, segs = 0;
        RingPos kv;
        bool ok = true;
        const int nbox = KT / ta.box_rows;  // 1 or 2
        const int is_v = (lane >> 1) & 1, box = lane & 1;
        const bool boxes = lane < 4 && box < nbox;
        const int box_slot = box * ta.box_rows, row_mask = a.kv.page_tokens - 1;
        const int cap = a.kv.table_cols << a.kv.page_shift;
        const uint32_t dst0 = ring + is_v * S::TILE_BYTES + box_slot * D, sdst0 = scales + is_v * KT + box_slot;
        const CUtensorMap* map = is_v ? &maps.v : &maps.k;
        const unsigned char* scale_pool = is_v ? q8.v_scale : q8.k_scale;
        TcSeg g;
        while (ok && work.next(g)) {
            const int n = g.nb, len = min(g.len, cap), lo = g.lo;
            if (n == 0) continue;
            const int* table = a.kv.table + g.seq * a.kv.table_seq_stride + g.head * a.kv.table_head_stride;
            const int head_c = a.kv.head_stride > 0 ? g.head : 0;
            const unsigned char* sbase = scale_pool + g.head * q8.head_stride;
            int slot = g.jb * KT + box_slot;  // first slot of this lane's box
            auto page_of = [&](int slot) {
                int page = a.kv.n_pages;  // outside the tensor: the box is filled with zeros
                if (boxes && slot < len && slot + ta.box_rows > lo) {
                    const int p = table[slot >> a.kv.page_shift];
                    if (p >= 0 && p < a.kv.n_pages) page = p;
                    else paged_report(a.kv, kStPage);
                }
                return page;
            };
            int page = page_of(slot);
            const int qs = segs & 1;
            if (segs >= 2 && !(ok = warp_wait(q_empty(qs), ((segs >> 1) - 1) & 1, abort_flag))) break;
            ++segs;
            if (lane == 0) {
                mbar_expect_tx(q_full(qs), (uint32_t)(a.tq * a.group * D * (int)sizeof(T)));
                tma_load_4d(qring + qs * S::Q_SLOT, &maps.q, 0, 0, g.head, g.tok0, q_full(qs));
            }
            for (int j = 0; j < n; ++j) {
                const int page_next = j + 1 < n ? page_of(slot + KT) : 0;
                if (issued >= NS && !(ok = warp_wait(empty(kv.st), kv.ph ^ 1, abort_flag))) break;
                const bool there = boxes && page < a.kv.n_pages;
                const uint32_t sdst = sdst0 + kv.st * S::SCALE_BYTES;
                if (boxes && !there) {  // codes of zero: any finite scale
                    for (int i = 0; i < ta.box_rows; i += 16)
                        asm volatile("st.shared.v4.u32 [%0], {%1, %1, %1, %1};" ::"r"(sdst + i), "r"(0x7f7f7f7f) : "memory");
                    fence_proxy_async_smem();  // (before a later copy to the same place)
                }
                const int copies = __popc(__ballot_sync(0xffffffffu, there));
                if (lane == 0) mbar_expect_tx(full(kv.st), (uint32_t)(S::STAGE_BYTES + copies * ta.box_rows));
                __syncwarp();
                if (boxes) tma_load_4d(dst0 + kv.st * S::STAGE_BYTES, map, 0, slot & row_mask, head_c, page, full(kv.st));
                if (there) bulk_g2s(sdst, sbase + page * q8.page_stride + (slot & row_mask), (uint32_t)ta.box_rows, full(kv.st));
                ++issued;
                kv.next(NS);
                slot += KT;
                page = page_next;
            }
        }
        if (!ok && lane == 0) {
            // given up: the copies in flight land before the CTA's shared memory goes to somebody else
            for (int i = segs > 2 ? segs - 2 : 0; i < segs; ++i) mbar_wait_bounded(q_full(i & 1), (i >> 1) & 1);
            for (int i = issued > NS ? issued - NS : 0; i < issued; ++i) mbar_wait_bounded(full(i % NS), (i / NS) & 1);
        }
        __syncwarp();
    } else if (warp <= W) {
        // ------------------------------------------------------------------ consumers
        const int cw = warp - 1, quad = lane & 3, qrow = lane >> 2;  // fragment coordinates
        const int G = a.group;
        int t = cw, t_base = 0;   // next tile of this warp, first tile of the segment (in the CTA's list)
        int segs = 0, all_segs = 0;
        RingPos rp;
        rp.st = cw;
        bool ok = true;
        // byte offset of 16-byte chunk c of row r of a tile (128- or 64-byte swizzle)
        auto off = [](int r, int c) { return (uint32_t)(D == 128 ? r * 128 + ((c ^ (r & 7)) << 4) : r * 64 + ((c ^ ((r >> 1) & 3)) << 4)); };
        TcSeg g;
        while (ok && work.next(g)) {
            const int n = g.nb;
            // per row of this thread (8 r + 2 quad + e): largest logit, sum, reference of the weights, accumulator (element 16 k + 2 qrow: e, + 1: 2 + e)
            float m[NR][2], l[NR][2], vr[NR][2], o[NR][KS][4];
            float qs_row[NR][2], sc[NR][2];  // power of two that q was divided by, softmax scale of the divided logits
            int last[NR][2];
#pragma unroll
            for (int r = 0; r < NR; ++r) {
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const int row = 8 * r + 2 * quad + e;
                    m[r][e] = vr[r][e] = -INFINITY;
                    l[r][e] = 0.f;
                    qs_row[r][e] = sc[r][e] = 0.f;
                    last[r][e] = row >= g.n_tok * G ? -1 : a.causal ? min(g.slot0 + row / G, g.len - 1) : g.len - 1;
                }
#pragma unroll
                for (int k = 0; k < KS; ++k) o[r][k][0] = o[r][k][1] = o[r][k][2] = o[r][k][3] = 0.f;
            }
            const int min_last = a.causal ? min(g.slot0, g.len - 1) : g.len - 1;
            if (n > 0) {
                const int qs = segs & 1;
                if (!(ok = warp_wait(q_full(qs), (segs >> 1) & 1, abort_flag))) break;
                ++segs;
                uint32_t qf[TERMS][NR][KS][2];  // B operand: column = row of the unit, elements 4 quad .. + 3 of each 16
#pragma unroll
                for (int r = 0; r < NR; ++r) {
                    const unsigned char* src = gq + qs * S::Q_SLOT + (8 * r + qrow) * D * (int)sizeof(T);
                    float4 x[KS];
                    unsigned big = 0;
#pragma unroll
                    for (int k = 0; k < KS; ++k) {
                        x[k] = OutRow<T>::get(src + (16 * k + 4 * quad) * (int)sizeof(T));
                        big = max(big, max(max(__float_as_uint(x[k].x) & 0x7fffffffu, __float_as_uint(x[k].y) & 0x7fffffffu),
                                           max(__float_as_uint(x[k].z) & 0x7fffffffu, __float_as_uint(x[k].w) & 0x7fffffffu)));
                    }
                    big = max(big, __shfl_xor_sync(0xffffffffu, big, 1));
                    big = max(big, __shfl_xor_sync(0xffffffffu, big, 2));
                    const int ex = big == 0 ? 135 : max((int)(big >> 23), 9);
                    const float inv = __uint_as_float((unsigned)(262 - ex) << 23);          // 2^(8 - (ex - 127))
                    const float back = __uint_as_float((unsigned)(ex - 8) << 23);
#pragma unroll
                    for (int k = 0; k < KS; ++k) {
                        x[k].x *= inv; x[k].y *= inv; x[k].z *= inv; x[k].w *= inv;
                        qf[0][r][k][0] = pack_f16(x[k].x, x[k].y);
                        qf[0][r][k][1] = pack_f16(x[k].z, x[k].w);
                        if (TERMS == 2) {
                            const float2 h0 = unpack_f16(qf[0][r][k][0]), h1 = unpack_f16(qf[0][r][k][1]);
                            qf[TERMS - 1][r][k][0] = pack_f16(x[k].x - h0.x, x[k].y - h0.y);
                            qf[TERMS - 1][r][k][1] = pack_f16(x[k].z - h1.x, x[k].w - h1.y);
                        }
                    }
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        qs_row[r][e] = __shfl_sync(0xffffffffu, back, (2 * quad + e) * 4);
                        sc[r][e] = fmaxf(a.scale_log2 * qs_row[r][e], 1.17549435e-38f);  // (-inf times it is -inf)
                    }
                }
                __syncwarp();
                if (lane == 0) mbar_arrive(q_empty(qs));
                for (; t < t_base + n; t += W) {
                    const int st = rp.st;
                    if (!(ok = warp_wait(full(st), rp.ph, abort_flag))) break;
                    rp.skip(W, NS);
                    const int base_slot = (g.jb + t - t_base) * KT;
                    const uint32_t kt = ring + st * S::STAGE_BYTES, vt = kt + S::TILE_BYTES;
                    const bool ragged = base_slot < g.lo || base_slot + KT > g.len;
                    if (ragged) {
                        // values of slots that are not live: their weight is 0, but 0 * NaN is not
                        for (int i = lane; i < KT * (D / 16); i += 32) {
                            const int r = i / (D / 16);
                            if (base_slot + r < g.lo || base_slot + r >= g.len)
                                asm volatile("st.shared.v4.u32 [%0], {%1, %1, %1, %1};" ::"r"(vt + i * 16), "r"(0) : "memory");
                        }
                        __syncwarp();
                    }
                    // scales of this thread's slots 16 mt + qrow + 8 h
                    float kf[MT][2], ve[MT][2];
#pragma unroll
                    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            const int at = st * S::SCALE_BYTES + 16 * mt + qrow + 8 * h, vb = gscales[at + KT];
                            kf[mt][h] = q8_scale(gscales[at]);
                            ve[mt][h] = vb == kQ8NaN ? INFINITY : (float)(vb - 127);
                        }
                    // S^T[slot][row]
                    float s[MT][NR][4];
#pragma unroll
                    for (int mt = 0; mt < MT; ++mt) {
#pragma unroll
                        for (int r = 0; r < NR; ++r) s[mt][r][0] = s[mt][r][1] = s[mt][r][2] = s[mt][r][3] = 0.f;
#pragma unroll
                        for (int k = 0; k < KS; k += 2) {
                            uint32_t f[4], x[4], y[4];  // 8 slots x 16 codes each: slots 0-7, 8-15 of chunk k, then of chunk k + 1
                            ldmatrix_x4(kt + off(16 * mt + (lane & 15), k + (lane >> 4)), f);
#pragma unroll
                            for (int i = 0; i < 4; ++i) q8_halves(f[i], x[i], y[i]);
#pragma unroll
                            for (int r = 0; r < NR; ++r)
#pragma unroll
                                for (int u = 0; u < TERMS; ++u) {
                                    mma_f16(s[mt][r], x[0], x[1], y[0], y[1], qf[u][r][k][0], qf[u][r][k][1]);
                                    mma_f16(s[mt][r], x[2], x[3], y[2], y[3], qf[u][r][k + 1][0], qf[u][r][k + 1][1]);
                                }
                        }
#pragma unroll
                        for (int r = 0; r < NR; ++r)
#pragma unroll
                            for (int e = 0; e < 4; ++e) s[mt][r][e] *= kf[mt][e >> 1];
                    }
                    if (base_slot < g.lo || base_slot + KT - 1 > min_last) {
#pragma unroll
                        for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                            for (int h = 0; h < 2; ++h) {
                                const int slot = base_slot + 16 * mt + qrow + h * 8;
                                if (slot < g.lo || slot >= g.len) ve[mt][h] = 0.f;
#pragma unroll
                                for (int r = 0; r < NR; ++r)
#pragma unroll
                                    for (int e = 0; e < 2; ++e)
                                        if (slot < g.lo || slot > last[r][e]) s[mt][r][2 * h + e] = -INFINITY;
                            }
                    }
                    uint32_t pb[TERMS][MT][NR][2];  // weights^T as B operand
#pragma unroll
                    for (int r = 0; r < NR; ++r) {
                        float of[2];
#pragma unroll
                        for (int e = 0; e < 2; ++e) {
                            float mx = fmaxf(s[0][r][e], s[0][r][2 + e]);
#pragma unroll
                            for (int mt = 1; mt < MT; ++mt) mx = fmaxf(mx, fmaxf(s[mt][r][e], s[mt][r][2 + e]));
#pragma unroll
                            for (int w = 4; w <= 16; w <<= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, w));
                            const float mn = fmaxf(m[r][e], mx), ref = softmax_ref(mn);
                            const float shift = (m[r][e] - ref) * sc[r][e];
                            m[r][e] = mn;
                            float sum = 0.f, top = -INFINITY;
#pragma unroll
                            for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                                for (int h = 0; h < 2; ++h) {
                                    float& x = s[mt][r][2 * h + e];
                                    x = (x - ref) * sc[r][e];
                                    sum += ex2_approx(x);
                                    x += ve[mt][h];
                                    top = fmaxf(top, x);
                                }
                            l[r][e] = fmaf(l[r][e], ex2_approx(shift), sum);
#pragma unroll
                            for (int w = 4; w <= 16; w <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, w));
                            const float was = vr[r][e] + shift, vn = fmaxf(was, top), vref = softmax_ref(vn);
                            of[e] = ex2_approx(was - vref);
                            vr[r][e] = vn;
#pragma unroll
                            for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                                for (int h = 0; h < 2; ++h) s[mt][r][2 * h + e] = ex2_approx(s[mt][r][2 * h + e] - vref + 14.f);
                        }
#pragma unroll
                        for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                            for (int h = 0; h < 2; ++h) {
                                const float w0 = s[mt][r][2 * h], w1 = s[mt][r][2 * h + 1];
                                const uint32_t p = pack_f16(w0, w1);
                                pb[0][mt][r][h] = movmatrix_trans(p);
                                if (TERMS == 2) {
                                    const float2 hi = unpack_f16(p);
                                    pb[TERMS - 1][mt][r][h] = movmatrix_trans(pack_f16(w0 - hi.x, w1 - hi.y));
                                }
                            }
                        if (__any_sync(0xffffffffu, of[0] != 1.f || of[1] != 1.f)) {
#pragma unroll
                            for (int k = 0; k < KS; ++k) {
                                o[r][k][0] *= of[0];
                                o[r][k][1] *= of[1];
                                o[r][k][2] *= of[0];
                                o[r][k][3] *= of[1];
                            }
                        }
                    }
                    // O^T[element][row] += V^T w^T
#pragma unroll
                    for (int k = 0; k < KS; k += 2) {
                        float add[2][NR][4];
                        if (TERMS == 2) {
#pragma unroll
                            for (int r = 0; r < NR; ++r)
#pragma unroll
                                for (int i = 0; i < 8; ++i) add[i >> 2][r][i & 3] = 0.f;
                        }
#pragma unroll
                        for (int mt = 0; mt < MT; ++mt) {
                            uint32_t f[4];  // slots 0-7, 8-15 of chunk k, then of chunk k + 1
                            ldmatrix_x4_trans(vt + off(16 * mt + (lane & 15), k + (lane >> 4)), f);
#pragma unroll
                            for (int c = 0; c < 2; ++c) {
                                uint32_t a0, a1, a2, a3;
                                q8_halves(__byte_perm(f[2 * c], 0, 0x3120), a0, a1);
                                q8_halves(__byte_perm(f[2 * c + 1], 0, 0x3120), a2, a3);
#pragma unroll
                                for (int r = 0; r < NR; ++r)
#pragma unroll
                                    for (int u = 0; u < TERMS; ++u)
                                        mma_f16(TERMS == 2 ? add[c][r] : o[r][k + c], a0, a1, a2, a3, pb[u][mt][r][0], pb[u][mt][r][1]);
                            }
                        }
                        if (TERMS == 2) {
#pragma unroll
                            for (int r = 0; r < NR; ++r)
#pragma unroll
                                for (int i = 0; i < 8; ++i) o[r][k + (i >> 2)][i & 3] += add[i >> 2][r][i & 3];
                        }
                    }
                    if (ragged) fence_proxy_async_smem();  // the clearing before the next copy into the stage
                    __syncwarp();
                    if (lane == 0) mbar_arrive(empty(st));
                }
                if (!ok) break;
                t_base += n;
            }
            // this warp's part of the unit
            const int pb = all_segs % S::PBUFS, turn = all_segs / S::PBUFS;
            ++all_segs;
            if (turn > 0 && !(ok = warp_wait(p_empty(pb), (turn - 1) & 1, abort_flag))) break;
            float* part = pbuf + pb * S::PBUF_FLOATS + cw * S::ROWS * S::PS;
#pragma unroll
            for (int r = 0; r < NR; ++r)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
#pragma unroll
                    for (int w = 4; w <= 16; w <<= 1) l[r][e] += __shfl_xor_sync(0xffffffffu, l[r][e], w);
                    float* p = part + (8 * r + 2 * quad + e) * S::PS;
                    const float f = ex2_approx(vr[r][e] - 14.f);  // (nothing seen: 0)
#pragma unroll
                    for (int k = 0; k < KS; ++k) *reinterpret_cast<float2*>(p + 16 * k + 2 * qrow) = make_float2(o[r][k][e] * f, o[r][k][2 + e] * f);
                    if (qrow == 0) {
                        p[D] = m[r][e] == -INFINITY ? -INFINITY : m[r][e] * qs_row[r][e];
                        p[D + 1] = l[r][e];
                    }
                }
            __syncwarp();
            if (lane == 0) mbar_arrive(p_full(pb));
        }
    } else {
        // ------------------------------------------------------------------ epilogue
        constexpr int LPR = D / 4;  // lanes of a row, four elements each
        const int G = a.group;
        int all_segs = 0;
        bool ok = true, recorded = false;
        TcSeg g;
        while (ok && work.next(g)) {
            const int pb = all_segs % S::PBUFS, turn = all_segs / S::PBUFS;
            ++all_segs;
            if (!(ok = warp_wait(p_full(pb), turn & 1, abort_flag))) break;
            const int slotp = blockIdx.x * 2 + (g.b0 > 0 ? 0 : 1), e = (lane % LPR) * 4;
            for (int row = lane / LPR; row < g.n_tok * G; row += 32 / LPR) {
                const float* part = pbuf + pb * S::PBUF_FLOATS + row * S::PS;
                float mw[W], M = -INFINITY;
#pragma unroll
                for (int w = 0; w < W; ++w) {
                    mw[w] = part[w * S::ROWS * S::PS + D];
                    M = fmaxf(M, mw[w]);
                }
                const float ref = softmax_ref(M);
                float L = 0.f;
                float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
                for (int w = 0; w < W; ++w) {
                    const float f = ex2_approx((mw[w] - ref) * a.scale_log2);
                    const float4 p = *reinterpret_cast<const float4*>(part + w * S::ROWS * S::PS + e);
                    L = fmaf(part[w * S::ROWS * S::PS + D + 1], f, L);
                    o.x = fmaf(p.x, f, o.x);
                    o.y = fmaf(p.y, f, o.y);
                    o.z = fmaf(p.z, f, o.z);
                    o.w = fmaf(p.w, f, o.w);
                }
                if (g.whole) {
                    const float inv = L > 0.f ? 1.0f / L : L;  // nothing seen: 0; NaN stays NaN
                    const int t = row / G;
                    OutRow<T>::put(a.out.p, (long long)(g.tok0 + t) * a.out.token_stride + (long long)(g.head * G + row - t * G) * a.out.head_stride + e, o, inv);
                } else {
                    const size_t at = (size_t)slotp * ta.rows_cap + row;
                    *reinterpret_cast<float4*>(a.part_o + at * D + e) = o;
                    if (e == 0) *reinterpret_cast<float2*>(a.part_ml + at * 2) = make_float2(M, L);
                }
            }
            if (!g.whole && g.b0 == 0) {
                // the unit goes on in the next CTAs: up to the one that holds its last tile
                if (lane == 0) ta.records[blockIdx.x] = make_int4(g.tok0, g.n_tok, g.head, (int)(((long long)g.unit_end * n_ranges + total - 1) / total - 1));
                recorded = true;
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(p_empty(pb));
        }
        if (ta.split && !recorded && lane == 0) ta.records[blockIdx.x] = make_int4(0, 0, 0, 0);
    }
    __syncthreads();
    if (tid == 0 && *abort_flag) paged_report(a.kv, kStWaitLimit);
}

// Adds up the parts of the units that range boundaries cut, in the order of the CTAs that left them.
template <typename T, int D>
__global__ void __launch_bounds__(128) q8_join_kernel(const __grid_constant__ TcArgs ta) {
    grid_dep_wait();
    const PagedAttnArgs& a = ta.a;
    const int4 rec = ta.records[blockIdx.x];  // first token, tokens, head, last CTA
    const int c0 = blockIdx.x, c1 = min(rec.w, (int)gridDim.x - 1);
    for (int i = blockIdx.y * blockDim.x + threadIdx.x; i < rec.y * a.group * (D / 4); i += gridDim.y * blockDim.x) {
        const int row = i / (D / 4), e = (i - row * (D / 4)) * 4, t = row / a.group;
        auto at = [&](int c) { return (size_t)(c * 2 + (c == c0 ? 1 : 0)) * ta.rows_cap + row; };
        float M = -INFINITY, L = 0.f;
        float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
        for (int c = c0; c <= c1; ++c) {
            const float2 ml = *reinterpret_cast<const float2*>(a.part_ml + at(c) * 2);
            const float4 p = *reinterpret_cast<const float4*>(a.part_o + at(c) * D + e);
            const float mn = fmaxf(M, ml.x), ref = softmax_ref(mn);
            const float f0 = ex2_approx((M - ref) * a.scale_log2), f = ex2_approx((ml.x - ref) * a.scale_log2);
            M = mn;
            L = fmaf(ml.y, f, L * f0);
            o.x = fmaf(p.x, f, o.x * f0);
            o.y = fmaf(p.y, f, o.y * f0);
            o.z = fmaf(p.z, f, o.z * f0);
            o.w = fmaf(p.w, f, o.w * f0);
        }
        const int h = rec.z * a.group + row - t * a.group;
        OutRow<T>::put(a.out.p, (long long)(rec.x + t) * a.out.token_stride + (long long)h * a.out.head_stride + e, o, L > 0.f ? 1.0f / L : L);
    }
}

struct Q8UnpackArgs {
    PagedView kv;
    Q8View q8;
    const int* start;
    char* out[2];   // K, V: [sequences][cols * 128 slots][heads][d]
    int* table;     // [sequences][cols]: the pages in order
    int cols;
};

constexpr int kQ8UnpackSlots = 32;

// Live entries of every sequence as dense pages of 128 rows, for the kernels of longer chunks (each element is read by many row tiles there: turned once, not once for
// each).  A CTA has 32 slots of K or V; slots outside [start, len) are left alone: whoever reads the pages masks them.
template <typename T, int D>
__global__ void __launch_bounds__(kQ8ReadThreads) q8_unpack_kernel(const __grid_constant__ Q8UnpackArgs a) {
    constexpr int IPR = D / 16, E = Elt<T>::kPerChunk, BATCH = 4;
    const int tid = threadIdx.x, s = blockIdx.y, is_v = blockIdx.z, first = blockIdx.x * kQ8UnpackSlots;
    if (tid == 0 && is_v == 0 && (first & 127) == 0) a.table[s * a.cols + (first >> 7)] = s * a.cols + (first >> 7);
    const int len = min(live_len(a.kv, s, 0, false), a.cols * 128), lo = a.start ? max(a.start[s], 0) : 0;
    const int j0 = max(first, lo), j1 = min(first + kQ8UnpackSlots, len);
    if (j0 >= j1) return;
    const int c = tid & (IPR - 1), heads = a.kv.n_kv_heads, n_items = (j1 - j0) * heads * IPR;
    const char* pool = is_v ? a.kv.v_pool : a.kv.k_pool;
    const unsigned char* scale_pool = is_v ? a.q8.v_scale : a.q8.k_scale;
    T* out = reinterpret_cast<T*>(a.out[is_v]) + (long long)s * a.cols * 128 * heads * D;
    for (int base = 0; base < n_items; base += kQ8ReadThreads * BATCH) {
        uint4 codes[BATCH];
        int byte[BATCH];
#pragma unroll
        for (int b = 0; b < BATCH; ++b) {
            const int r = (base + b * kQ8ReadThreads + tid) / IPR, jl = r / heads, head = r - jl * heads, slot = j0 + jl;
            codes[b] = make_uint4(0, 0, 0, 0);
            byte[b] = 127;
            if (slot >= j1) continue;
            const int page = a.kv.table[s * a.kv.table_seq_stride + head * a.kv.table_head_stride + (slot >> a.kv.page_shift)];
            if (page < 0 || page >= a.kv.n_pages) {
                if (c == 0) paged_report(a.kv, kStPage);
                continue;
            }
            const int in_page = slot & (a.kv.page_tokens - 1);
            codes[b] = *reinterpret_cast<const uint4*>(pool + page * a.kv.page_stride + in_page * a.kv.row_stride + head * a.kv.head_stride + c * 16);
            byte[b] = scale_pool[page * a.q8.page_stride + head * a.q8.head_stride + in_page];
        }
#pragma unroll
        for (int b = 0; b < BATCH; ++b) {
            const int r = (base + b * kQ8ReadThreads + tid) / IPR, jl = r / heads;
            if (j0 + jl >= j1) continue;
            T* dst = out + ((long long)j0 * heads + r) * D + c * 16;
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
