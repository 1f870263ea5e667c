// Attention over an 8-bit paged cache (paged_q8.cuh) from its codes, at most 16 (token, head of the group) rows of a KV head per unit: single tokens and
// short candidate chunks, and whatever has fp32 rows.  Single tokens are bound by the cache's bytes (3 x 1 token over 23398 to 65537 slots, 8 KV heads
// of 128: 313 MB in 65 us; 16 x 129 to 4288 slots: 78 MB in 25 us, of which 9.6 are launch, lengths, page table and first tile, and 3 the join), short units by
// the chain of a tile, more rows by the warps that the registers leave room for (64 x 1 to 577 slots, 20 heads of 64, up to 16 fp32 rows: 38 us, tensor pipe
// 21 % busy, 11 warps on an SM).
//
// The layout of work is that of paged_attn_few.cuh: every consumer warp takes a tile of 64 slots (32 where registers are short) through S^T = K q^T and O^T += V^T P^T with
// mma.sync (the slots as the rows of the product), a producer warp keeps a ring of K/V tiles full, an epilogue warp merges the warps'
// partial results.  What 8 bits change:
//   * Codes go to fp16, which holds every e4m3 number: one conversion for two of them, no scale applied.  A row's scale is a power of two that belongs to a
//     slot, so K's multiplies the slot's logits and V's the slot's weights; no element is ever multiplied.
//   * The elements of a row may be contracted in any order, so a thread takes the four neighbouring codes that ldmatrix gives it as elements 2t,
//     2t + 1, 2t + 8, 2t + 9 of the product, and q's fragments are loaded to match.  V^T comes from ldmatrix.trans on pairs of codes: rows g and g + 8 of a
//     product are elements 2g and 2g + 1.
//   * q is scaled by a power of two to 2^4 .. 2^5 per row (bf16 exact in fp16 down to 2^-21 of the row's largest element, off by 2^-29 of it below), and K's powers by 2^-14,
//     so that the product of the two is at most 2^127; what both leave out of the logit comes back with the subtraction of the largest one.  So nothing on the way is beyond fp32
//     that the logit is not.  (Rows of q from 2^118 on are scaled to 2^14 at most, as the power that comes back ends at 2^127.)  fp32
//     rows take two fp16 numbers for q and for the weights (22 bits), and sums of a tile are added to the accumulator with rounding.
//   * A weight is p_j 2^(v_j), v_j the exponent of the slot's values.  fp16 has 5 bits of exponent, so each row keeps a reference vr of its own, the
//     largest (logit - m) log2(e) scale + v_j so far: weights are at most 2^14, and what fp16 cannot hold is below 2^-38 of the row's largest weight.  A row
//     of zeros, whose byte says nothing about it, has no weight.
#pragma once
#include <cuda_fp16.h>

#include "join_parts.cuh"
#include "paged_attn_tc.cuh"
#include "paged_q8.cuh"

namespace lar {

constexpr int kQ8Rows = 16;  // rows of a unit at most

// A step of a CTA's work, worked out by the producer: some slot tiles of one unit.
struct alignas(16) Q8Seg {
    int tok0, n_tok, head, slot0;  // tokens of the unit, slot of the first
    int lo, len, jb, nb;           // live slots of the sequence; first tile and tiles of this step (-1: no more work)
    int whole, b0, last_cta, pad;  // nothing of the unit lies in other CTAs; tiles before this step's; the CTA with its last one
};

template <typename T, int D, int NR>
struct Q8Shape {
    static constexpr int TERMS = sizeof(T) == 4 ? 2 : 1;
    // Slots of a tile (64 instead of 32, one token over 16 x 4288 slots: 25 instead of 27 us, 3 x 65537 slots 68 instead of 75; 16 rows of 64 fp32
    // elements 40 instead of 44).  With 16 rows of 128 elements tiles of 32 and two of them for each consumer (38.6 -> 33.6 us, 64 rows 96 -> 87; fp32 66 -> 57).
    // (These and the figures below were taken before logits of any size and rows of zeros were looked after, which costs 1 to 4 %.)
    static constexpr int KT = NR == 2 && D == 128 ? 32 : 64;
    static constexpr int MT = KT / 16, KS = D / 16;
    static constexpr int TILE_BYTES = KT * D, STAGE_BYTES = 2 * TILE_BYTES, SCALE_BYTES = 2 * KT;
    static constexpr int SCALE_PITCH = KT / 16 * 128;  // of a stage: a copy's destination is 128-byte aligned, and a page has 16 slots at least
    static constexpr int W = 4, THREADS = (W + 2) * 32;  // producer, consumers, epilogue
    // Stages: a multiple of W, a stage is always read by the same consumer.  Two for each where two CTAs still fit (16 rows of 64 elements over 16 x 4288 slots 30.1 -> 27.5 us
    // in fp32, 26.6 -> 25.4 in bf16): with one, a consumer that is done waits for the next tile.  One where rows are few: bandwidth then comes from many CTAs.
    static constexpr int NS = (D == 64 && NR == 2) || (TERMS == 1 && KT == 32) ? 8 : 4;
    static constexpr int PER_SM = D == 64 && NR == 1 ? 3 : 2;  // (64 x 577 slots, 20 heads of 64, 1 to 8 tokens: 27 us with three CTAs, 31 with two)
    static constexpr int ROWS = 8 * NR;
    // Units that the producer is ahead by at most.  (Two where rows are many, which lets two CTAs share an SM with 128 elements: 16 x 4288 slots, 16 rows 38.6 instead of 43.8
    // us, 32 rows 57 instead of 70; fp32 with 4 stages instead of 8, 51 instead of 55.  So with 8 rows of 128: four steps and two buffers of parts leave fp32 rows one CTA, and
    // bf16 rows from 192 sequences on, as the lengths take shared memory too: one fp32 row over 16 x 4288 slots 30.2 -> 23.7 us, 3 x 65537 81 -> 56, bf16 256 x 1153 102 -> 70, 1024 x
    // 577 251 -> 153; bf16 over few sequences is the same either way.)
    static constexpr int QS = NR == 2 || D == 128 ? 2 : 4;
    static constexpr int Q_SLOT = ROWS * D * (int)sizeof(T);
    static constexpr int PS = D + 4;              // floats of a partial row: O, m, l, padding
    static constexpr int PBUFS = NR == 1 && D == 64 ? 2 : 1;
    static constexpr int PBUF_FLOATS = W * ROWS * PS;
    static constexpr int FIXED = 1024 + NS * (STAGE_BYTES + SCALE_PITCH) + QS * (Q_SLOT + (int)sizeof(Q8Seg)) + PBUFS * PBUF_FLOATS * 4 + 32 * 8;
    static __host__ __device__ constexpr int bytes(int n_seqs) { return FIXED + n_seqs * 16 + 2 * (n_seqs + 1) * 4 + 16 * 4; }
};

struct Q8Maps {
    CUtensorMap q;     // {d, heads of a group, KV heads, tokens}, box d x group x 1 x tq, rows of T
    CUtensorMap kv;    // {d, rows of a page, heads, pages, 2} of bytes, box d x min(page, KT) x 1 x 1 x 2, swizzled by d bytes: K and V rows with one
                       // copy (issuing copies is what bounds a producer), the pool with the lower address first
    CUtensorMap scale; // {rows of a page, heads, pages, 2} of bytes, box min(page, KT) x 1 x 1 x 2
    int v_first, v_scale_first;
};

__device__ __forceinline__ void tma_load_5d(uint32_t dst, const CUtensorMap* map, int x, int y, int z, int w, int v, uint32_t bar) {
    asm volatile(
        "cp.async.bulk.tensor.5d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5, %6}], [%7];" ::"r"(dst),
        "l"(reinterpret_cast<uint64_t>(map)), "r"(x), "r"(y), "r"(z), "r"(w), "r"(v), "r"(bar)
        : "memory");
}

// Two fp16 numbers from each half of four codes.
__device__ __forceinline__ void q8_halves(uint32_t codes, uint32_t& lo, uint32_t& hi) {
    asm("{\n .reg .b16 a, b;\n mov.b32 {a, b}, %2;\n cvt.rn.f16x2.e4m3x2 %0, a;\n cvt.rn.f16x2.e4m3x2 %1, b;\n}\n" : "=r"(lo), "=r"(hi) : "r"(codes));
}
__device__ __forceinline__ void mma_f16(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm(
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
paged_attn_q8_kernel(const __grid_constant__ TcArgs ta, const __grid_constant__ Q8Maps maps) {
    using S = Q8Shape<T, D, NR>;
    using Work = TcWork<1, S::KT, D>;
    constexpr int KT = S::KT, W = S::W, NS = S::NS, TERMS = S::TERMS, KS = S::KS, MT = S::MT;
    static_assert(S::PER_SM * (S::bytes(128) + 1024) <= 233472, "shared memory of an SM");
    const PagedAttnArgs& a = ta.a;
    extern __shared__ unsigned char smem_raw[];
    const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    unsigned char* gbase = smem_raw + (base - smem_u32(smem_raw));
    const uint32_t ring = base, scales = base + NS * S::STAGE_BYTES;
    unsigned char* gscales = gbase + NS * S::STAGE_BYTES;
    unsigned char* gq = gscales + NS * S::SCALE_PITCH;
    const uint32_t qring = scales + NS * S::SCALE_PITCH;
    Q8Seg* segs_at = reinterpret_cast<Q8Seg*>(gq + S::QS * S::Q_SLOT);
    float* pbuf = reinterpret_cast<float*>(segs_at + S::QS);
    uint64_t* bars = reinterpret_cast<uint64_t*>(pbuf + S::PBUFS * S::PBUF_FLOATS);
    const uint32_t bar0 = smem_u32(bars);
    auto full = [&](int st) { return bar0 + 8u * st; };
    auto empty = [&](int st) { return bar0 + 8u * (8 + st); };
    auto q_full = [&](int i) { return bar0 + 8u * (16 + i); };
    auto q_empty = [&](int i) { return bar0 + 8u * (20 + i); };
    auto p_full = [&](int i) { return bar0 + 8u * (24 + i); };
    auto p_empty = [&](int i) { return bar0 + 8u * (26 + i); };
    volatile int* abort_flag = reinterpret_cast<volatile int*>(bars + 28);
    SeqInfo* info = reinterpret_cast<SeqInfo*>(bars + 32);
    int* pre = reinterpret_cast<int*>(info + a.kv.n_seqs);
    int* wsum = pre + 2 * (a.kv.n_seqs + 1);

    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    if (tid == 0) {
        for (int i = 0; i < NS; ++i) {
            mbar_init(full(i), 1);
            mbar_init(empty(i), 1);
        }
        for (int i = 0; i < S::QS; ++i) {
            mbar_init(q_full(i), 1);
            mbar_init(q_empty(i), W + 1);  // consumers and epilogue
        }
        for (int i = 0; i < 2; ++i) {
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
    if (warp == 0) {
        // ------------------------------------------------------------------ producer: a lane for every page (or part of one) of a tile
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
        int issued = 0, segs = 0;
        RingPos kv;
        bool ok = true;
        const int nbox = KT / ta.box_rows;  // at most 4
        const bool boxes = lane < nbox;
        const int box_slot = lane * ta.box_rows, row_mask = a.kv.page_tokens - 1;
        const int cap = a.kv.table_cols << a.kv.page_shift;
        const uint32_t dst0 = ring + box_slot * 2 * D, sdst0 = scales + lane * 128;
        TcSeg g = {};
        for (;;) {
            const bool more = work.next(g);
            const int n = more ? g.nb : 0, len = min(g.len, cap), lo = g.lo;
            const int* table = a.kv.table + g.seq * a.kv.table_seq_stride + g.head * a.kv.table_head_stride;
            const int head_c = a.kv.head_stride > 0 ? g.head : 0;
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
            int page = n > 0 ? page_of(slot) : 0;
            const int qs = segs % S::QS;
            if (segs >= S::QS && !(ok = warp_wait(q_empty(qs), (segs / S::QS - 1) & 1, abort_flag))) break;
            ++segs;
            if (lane == 0) {
                Q8Seg u;
                u.tok0 = g.tok0; u.n_tok = g.n_tok; u.head = g.head; u.slot0 = g.slot0;
                u.lo = g.lo; u.len = g.len; u.jb = g.jb; u.nb = more ? n : -1;
                u.whole = g.whole; u.b0 = g.b0; u.pad = 0;
                u.last_cta = more && !g.whole ? (int)(((long long)g.unit_end * n_ranges + total - 1) / total - 1) : 0;
                segs_at[qs] = u;
                if (n > 0) {
                    mbar_expect_tx(q_full(qs), (uint32_t)(a.tq * a.group * D * (int)sizeof(T)));
                    tma_load_4d(qring + qs * S::Q_SLOT, &maps.q, 0, 0, g.head, g.tok0, q_full(qs));
                } else {
                    mbar_arrive(q_full(qs));
                }
            }
            if (!more) break;
            for (int j = 0; j < n; ++j) {
                const int page_next = j + 1 < n ? page_of(slot + KT) : 0;
                if (issued >= NS && !(ok = warp_wait(empty(kv.st), kv.ph ^ 1, abort_flag))) break;
                if (lane == 0) mbar_expect_tx(full(kv.st), (uint32_t)(S::STAGE_BYTES + S::SCALE_BYTES));
                __syncwarp();
                if (boxes) {
                    tma_load_5d(dst0 + kv.st * S::STAGE_BYTES, &maps.kv, 0, slot & row_mask, head_c, page, 0, full(kv.st));
                    tma_load_4d(sdst0 + kv.st * S::SCALE_PITCH, &maps.scale, slot & row_mask, head_c, page, 0, full(kv.st));
                }
                ++issued;
                kv.next(NS);
                slot += KT;
                page = page_next;
            }
            if (!ok) break;
        }
        if (!ok && lane == 0) {
            // given up: the copies in flight land before the CTA's shared memory goes to somebody else
            for (int i = segs > S::QS ? segs - S::QS : 0; i < segs; ++i) mbar_wait_bounded(q_full(i % S::QS), (i / S::QS) & 1);
            for (int i = issued > NS ? issued - NS : 0; i < issued; ++i) mbar_wait_bounded(full(i % NS), (i / NS) & 1);
        }
        __syncwarp();
    } else if (warp <= W) {
        // ------------------------------------------------------------------ consumers
        const int cw = warp - 1, quad = lane & 3, qrow = lane >> 2;  // fragment coordinates
        const int G = a.group;
        const unsigned by_group = 65536u / G + 1u;  // (a row's token: row / G of at most 16 rows)
        int t = cw, t_base = 0;   // next tile of this warp, first tile of the step (in the CTA's list)
        RingPos rp;
        rp.st = cw;
        bool ok = true;
        // A stage holds one copy behind the other, each the rows of a page (or part of one) of one pool and then of the other: where 16 slots of a tile lie
        const uint32_t box_bytes = ta.box_rows * D, k_at = maps.v_first ? box_bytes : 0, v_at = maps.v_first ? 0 : box_bytes;
        const int ks_at = maps.v_scale_first ? ta.box_rows : 0, vs_at = maps.v_scale_first ? 0 : ta.box_rows;
        const int box_mask = ta.box_rows - 1, box_shift = __ffs(ta.box_rows) - 1;
        const int zero_slot = lane % (KT / 4) * 4, zero_at = (zero_slot >> box_shift) * 128 + (zero_slot & box_mask) + vs_at;  // four of V's bytes for each lane
        auto block = [&](int mt) { return (uint32_t)((16 * mt & ~box_mask) * 2 + (16 * mt & box_mask)); };  // rows before the block
        // byte offset of 16-byte chunk c of row r of a block (128- or 64-byte swizzle)
        auto off = [](int r, int c) { return (uint32_t)(D == 128 ? r * 128 + ((c ^ (r & 7)) << 4) : r * 64 + ((c ^ ((r >> 1) & 3)) << 4)); };
        for (int seg = 0;; ++seg) {
            const int qs = seg % S::QS;
            if (!(ok = warp_wait(q_full(qs), (seg / S::QS) & 1, abort_flag))) break;
            const Q8Seg g = segs_at[qs];
            const int n = g.nb;
            if (n < 0) break;
            // per row of this thread (8 r + 2 quad + e): largest logit, sum, reference of the weights, accumulator (element 16 k + 2 qrow: e, + 1: 2 + e)
            float m[NR][2], l[NR][2], vr[NR][2], o[NR][KS][4];
            float qs_row[NR][2];  // logit of a product of scaled q and K
            int last[NR][2];
#pragma unroll
            for (int r = 0; r < NR; ++r) {
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const int row = 8 * r + 2 * quad + e;
                    m[r][e] = vr[r][e] = -INFINITY;
                    l[r][e] = 0.f;
                    qs_row[r][e] = 0.f;
                    last[r][e] = row >= g.n_tok * G ? -1 : a.causal ? min(g.slot0 + (int)(row * by_group >> 16), g.len - 1) : g.len - 1;
                }
#pragma unroll
                for (int k = 0; k < KS; ++k) o[r][k][0] = o[r][k][1] = o[r][k][2] = o[r][k][3] = 0.f;
            }
            const int min_last = a.causal ? min(g.slot0, g.len - 1) : g.len - 1;
            if (n == 0) {
                __syncwarp();
                if (lane == 0) mbar_arrive(q_empty(qs));
            } else {
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
                    const float inv = __uint_as_float((unsigned)max(258 - ex, 14) << 23);    // 2^(4 - (ex - 127))
                    const float back = __uint_as_float((unsigned)min(ex + 10, 254) << 23);   // 2^14 / inv
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
                    for (int e = 0; e < 2; ++e) qs_row[r][e] = __shfl_sync(0xffffffffu, back, (2 * quad + e) * 4);
                }
                __syncwarp();
                if (lane == 0) mbar_arrive(q_empty(qs));
                for (; t < t_base + n; t += W) {
                    const int st = rp.st;
                    if (!(ok = warp_wait(full(st), rp.ph, abort_flag))) break;
                    rp.skip(W, NS);
                    const int base_slot = (g.jb + t - t_base) * KT;
                    const uint32_t tile = ring + st * S::STAGE_BYTES;
                    const bool ragged = base_slot < g.lo || base_slot + KT > g.len;
                    if (ragged) {
                        // values of slots that are not live: their weight is 0, but 0 * NaN is not
                        for (int i = lane; i < KT * (D / 16); i += 32) {
                            const int r = i / (D / 16);
                            if (base_slot + r < g.lo || base_slot + r >= g.len)
                                asm volatile("st.shared.v4.u32 [%0], {%1, %1, %1, %1};" ::"r"(tile + v_at + (block(r >> 4) + (r & 15)) * D + i % (D / 16) * 16), "r"(0) : "memory");
                        }
                        __syncwarp();
                    }
                    // S^T[slot][row]
                    float s[MT][NR][4];
#pragma unroll
                    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                        for (int r = 0; r < NR; ++r) s[mt][r][0] = s[mt][r][1] = s[mt][r][2] = s[mt][r][3] = 0.f;
#pragma unroll
                    for (int k = 0; k < KS; k += 2)
#pragma unroll
                        for (int mt = 0; mt < MT; ++mt) {
                            uint32_t f[4], x[4], y[4];  // 8 slots x 16 codes each: slots 0-7, 8-15 of chunk k, then of chunk k + 1
                            ldmatrix_x4(tile + k_at + block(mt) * D + off(lane & 15, k + (lane >> 4)), f);
#pragma unroll
                            for (int i = 0; i < 4; ++i) q8_halves(f[i], x[i], y[i]);
#pragma unroll
                            for (int u = 0; u < TERMS; ++u)
#pragma unroll
                                for (int r = 0; r < NR; ++r) mma_f16(s[mt][r], x[0], x[1], y[0], y[1], qf[u][r][k][0], qf[u][r][k][1]);
#pragma unroll
                            for (int u = 0; u < TERMS; ++u)
#pragma unroll
                                for (int r = 0; r < NR; ++r) mma_f16(s[mt][r], x[2], x[3], y[2], y[3], qf[u][r][k + 1][0], qf[u][r][k + 1][1]);
                        }
                    // scales of this thread's slots 16 mt + qrow + 8 h
                    float kf[MT][2], ve[MT][2];
#pragma unroll
                    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            const int at = st * S::SCALE_PITCH + (16 * mt >> box_shift) * 128 + (16 * mt & box_mask) + qrow + 8 * h, vb = gscales[at + vs_at], kb = gscales[at + ks_at];
                            kf[mt][h] = q8_scale(kb) * 0x1p-14f;
                            ve[mt][h] = vb == kQ8NaN ? INFINITY : (float)(vb - 127);
                        }
                    const uint32_t not127 = *reinterpret_cast<const uint32_t*>(gscales + st * S::SCALE_PITCH + zero_at) ^ 0x7f7f7f7fu;
                    if (__any_sync(0xffffffffu, ((not127 - 0x01010101u) & ~not127 & 0x80808080u) != 0)) {
                        // a row of zeros has a byte of 127: its weight is none, and must not be what the others' are measured by
#pragma unroll
                        for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                            for (int h = 0; h < 2; ++h) {
                                uint32_t any = 0;  // a quarter of the row's codes
#pragma unroll
                                for (int c = 0; c < D / 64; ++c) {
                                    uint32_t x[4];
                                    asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(x[0]), "=r"(x[1]), "=r"(x[2]), "=r"(x[3]) : "r"(tile + v_at + block(mt) * D + off(qrow + 8 * h, quad * (D / 64) + c)));
                                    any |= (x[0] | x[1] | x[2] | x[3]) & 0x7f7f7f7fu;
                                }
                                any |= __shfl_xor_sync(0xffffffffu, any, 1);
                                any |= __shfl_xor_sync(0xffffffffu, any, 2);
                                if (any == 0 && ve[mt][h] == 0.f) ve[mt][h] = -INFINITY;
                            }
                    }
#pragma unroll
                    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                        for (int r = 0; r < NR; ++r)
#pragma unroll
                            for (int e = 0; e < 4; ++e) s[mt][r][e] *= kf[mt][e >> 1];
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
                    // The softmax, one step for all columns at a time: a shuffle's latency is that of many instructions.
                    float mx[NR][2], top[NR][2], of[NR][2];
#pragma unroll
                    for (int r = 0; r < NR; ++r)
#pragma unroll
                        for (int e = 0; e < 2; ++e) {
                            mx[r][e] = fmaxf(s[0][r][e], s[0][r][2 + e]);
#pragma unroll
                            for (int mt = 1; mt < MT; ++mt) mx[r][e] = fmaxf(mx[r][e], fmaxf(s[mt][r][e], s[mt][r][2 + e]));
                        }
#pragma unroll
                    for (int w = 4; w <= 16; w <<= 1)
#pragma unroll
                        for (int r = 0; r < NR; ++r)
#pragma unroll
                            for (int e = 0; e < 2; ++e) mx[r][e] = fmaxf(mx[r][e], __shfl_xor_sync(0xffffffffu, mx[r][e], w));
#pragma unroll
                    for (int r = 0; r < NR; ++r)
#pragma unroll
                        for (int e = 0; e < 2; ++e) {
                            const float f = qs_row[r][e], mn = fmaxf(m[r][e], mx[r][e] * f);
                            const float ref = mn == INFINITY ? NAN : softmax_ref(mn), shift = (m[r][e] - ref) * a.scale_log2;  // (beyond fp32: NaN)
                            m[r][e] = mn;
                            vr[r][e] += shift;
                            float sum = 0.f, most = -INFINITY;
#pragma unroll
                            for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                                for (int h = 0; h < 2; ++h) {
                                    float& x = s[mt][r][2 * h + e];
                                    x = fmaf(x, f, -ref) * a.scale_log2;
                                    sum += ex2_approx(x);
                                    x += ve[mt][h];
                                    most = fmaxf(most, x);
                                }
                            l[r][e] = fmaf(l[r][e], ex2_approx(shift), sum);
                            top[r][e] = most;
                        }
#pragma unroll
                    for (int w = 4; w <= 16; w <<= 1)
#pragma unroll
                        for (int r = 0; r < NR; ++r)
#pragma unroll
                            for (int e = 0; e < 2; ++e) top[r][e] = fmaxf(top[r][e], __shfl_xor_sync(0xffffffffu, top[r][e], w));
                    uint32_t pb[TERMS][MT][NR][2];  // weights^T as B operand
                    bool moved = false;
#pragma unroll
                    for (int r = 0; r < NR; ++r) {
#pragma unroll
                        for (int e = 0; e < 2; ++e) {
                            const float vn = fmaxf(vr[r][e], top[r][e]), vref = softmax_ref(vn);
                            of[r][e] = ex2_approx(vr[r][e] - vref);
                            vr[r][e] = vn;
                            moved |= of[r][e] != 1.f;
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
                    }
                    if (__any_sync(0xffffffffu, moved)) {
#pragma unroll
                        for (int r = 0; r < NR; ++r)
#pragma unroll
                            for (int k = 0; k < KS; ++k) {
                                o[r][k][0] *= of[r][0];
                                o[r][k][1] *= of[r][1];
                                o[r][k][2] *= of[r][0];
                                o[r][k][3] *= of[r][1];
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
                            ldmatrix_x4_trans(tile + v_at + block(mt) * D + off(lane & 15, k + (lane >> 4)), f);
                            uint32_t v[2][4];
#pragma unroll
                            for (int c = 0; c < 2; ++c) {
                                q8_halves(__byte_perm(f[2 * c], 0, 0x3120), v[c][0], v[c][1]);
                                q8_halves(__byte_perm(f[2 * c + 1], 0, 0x3120), v[c][2], v[c][3]);
                            }
#pragma unroll
                            for (int u = 0; u < TERMS; ++u)
#pragma unroll
                                for (int c = 0; c < 2; ++c)
#pragma unroll
                                    for (int r = 0; r < NR; ++r)
                                        mma_f16(TERMS == 2 ? add[c][r] : o[r][k + c], v[c][0], v[c][1], v[c][2], v[c][3], pb[u][mt][r][0], pb[u][mt][r][1]);
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
            const int pb = seg % S::PBUFS, turn = seg / S::PBUFS;
            if (turn > 0 && !(ok = warp_wait(p_empty(pb), (turn - 1) & 1, abort_flag))) break;
            float* part = pbuf + pb * S::PBUF_FLOATS + cw * S::ROWS * S::PS;
#pragma unroll
            for (int r = 0; r < NR; ++r)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
#pragma unroll
                    for (int w = 4; w <= 16; w <<= 1) l[r][e] += __shfl_xor_sync(0xffffffffu, l[r][e], w);
                    float* p = part + (8 * r + 2 * quad + e) * S::PS;
                    const float f = ex2_approx(vr[r][e]);  // (nothing seen: 0; with the 2^-14 in it the smallest would be zero too)
#pragma unroll
                    for (int k = 0; k < KS; ++k) *reinterpret_cast<float2*>(p + 16 * k + 2 * qrow) = make_float2(o[r][k][e] * 0x1p-14f * f, o[r][k][2 + e] * 0x1p-14f * f);
                    if (qrow == 0) {
                        p[D] = m[r][e];
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
        const unsigned by_group = 65536u / G + 1u;
        bool ok = true, recorded = false;
        for (int seg = 0;; ++seg) {
            const int qs = seg % S::QS;
            if (!(ok = warp_wait(q_full(qs), (seg / S::QS) & 1, abort_flag))) break;
            const Q8Seg g = segs_at[qs];
            if (g.nb < 0) break;
            __syncwarp();
            if (lane == 0) mbar_arrive(q_empty(qs));
            const int pb = seg % S::PBUFS, turn = seg / S::PBUFS;
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
                    const int t = (int)(row * by_group >> 16);
                    OutRow<T>::put(a.out.p, (long long)(g.tok0 + t) * a.out.token_stride + (long long)(g.head * G + row - t * G) * a.out.head_stride + e, o, inv);
                } else {
                    const size_t at = (size_t)slotp * ta.rows_cap + row;
                    *reinterpret_cast<float4*>(a.part_o + at * D + e) = o;
                    if (e == 0) *reinterpret_cast<float2*>(a.part_ml + at * 2) = make_float2(M, L);
                }
            }
            if (!g.whole && g.b0 == 0) {
                // the unit goes on in the next CTAs: up to the one that holds its last tile
                if (lane == 0) ta.records[blockIdx.x] = make_int4(g.tok0, g.n_tok, g.head, g.last_cta);
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

struct Q8UnpackArgs {
    PagedView kv;
    Q8View q8;
    const int* start;
    char* out[2];   // K, V: [sequences][cols * 128 slots][heads][d]
    int* table;     // [sequences][cols]: the pages in order
    int cols;
};

constexpr int kQ8UnpackSlots = 32;

// Live entries of every sequence as dense pages of 128 bf16 rows (exact), for the kernels of longer chunks of bf16 rows (each element is read by many row tiles there: turned once, not once for
// each).  A CTA has 32 slots of K or V; slots outside [start, len) are left alone: whoever reads the pages masks them.  So are sequences without tokens: nobody reads theirs,
// and their own pages may be gone.
template <int D>
__global__ void __launch_bounds__(kQ8ReadThreads) q8_unpack_kernel(const __grid_constant__ Q8UnpackArgs a) {
    constexpr int IPR = D / 16, E = 8, BATCH = 4;
    const int tid = threadIdx.x, s = blockIdx.y, is_v = blockIdx.z, first = blockIdx.x * kQ8UnpackSlots;
    if (tid == 0 && is_v == 0 && (first & 127) == 0) a.table[s * a.cols + (first >> 7)] = s * a.cols + (first >> 7);
    int t0, t1;
    chunk_of(a.kv, s, t0, t1);
    if (t0 == t1) return;
    const int len = min(live_len(a.kv, s, 0, false), a.cols * 128), lo = a.start ? max(a.start[s], 0) : 0;
    const int j0 = max(first, lo), j1 = min(first + kQ8UnpackSlots, len);
    if (j0 >= j1) return;
    const int c = tid & (IPR - 1), heads = a.kv.n_kv_heads, n_items = (j1 - j0) * heads * IPR;
    const char* pool = is_v ? a.kv.v_pool : a.kv.k_pool;
    const unsigned char* scale_pool = is_v ? a.q8.v_scale : a.q8.k_scale;
    __nv_bfloat16* out = reinterpret_cast<__nv_bfloat16*>(a.out[is_v]) + (long long)s * a.cols * 128 * heads * D;
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
            __nv_bfloat16* dst = out + ((long long)j0 * heads + r) * D + c * 16;
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
                *reinterpret_cast<uint4*>(dst + i) = PackRow<__nv_bfloat16>::pack(part);
            }
        }
    }
}

}  // namespace lar
