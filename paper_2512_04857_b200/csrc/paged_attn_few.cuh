// Chunk attention for bf16 storage and few rows: at most 8 (128-element rows) or 16 (64) (token, head of the group) rows of a KV head per
// unit, i.e. single tokens and short candidate chunks.  Bound by the cache's bytes, and with many short units by what surrounds them.
//
// A 128-row tcgen05 tile would be nine tenths padding and, worse, one chain of product -> softmax -> product per slot tile.  Here each
// of W consumer warps takes a slot tile of its own (every W-th of the CTA's list) through the whole chain in registers: S^T = K q^T and
// O^T += V^T P^T with mma.sync, the slots as the M rows and the query rows as the 8 or 16 columns (NR column blocks), so that no
// row of a product is padding; running maximum and sum per warp in fp32.  A producer warp keeps a ring of K/V stages full (TMA boxes
// by page, as in paged_attn_tc.cuh, and the queries of the next unit), an epilogue warp merges the W partial results of a unit and writes
// its rows while the consumers are on the next one.  Two CTAs per SM with 128-element rows, four with 64.
//
// 620 MB of cache (3 x 1 token, 23398 to 65537 slots) take 98 us = 6.3 TB/s, 98 % of the measured copy rate.
//
// Work is dealt out as in paged_attn_tc.cuh with one row tile: equal ranges of slot tiles, cut units joined by join_ranges_kernel.
#pragma once
#include "paged_attn_tc.cuh"

namespace lar {

// Rows up to which this kernel is taken: 16 x 4288 slots, 8 KV heads of 32, here / the tcgen05 kernel with one row tile: 128-element rows, 4
// rows 51.4 / 54.5 us, 16 rows 60.3 / 58.0; 64-element rows, 4 rows 31.9 / 36.6, 16 rows 35.8 / 38.5.  64 x 577 slots: 33.7 / 38.4, 44.5 /
// 41.2; 16.3 / 28.2, 21.7 / 30.1.
constexpr int few_rows(int d) { return d == 64 ? 16 : 8; }

template <int D, int NR>
struct FewShape {
    static constexpr int KT = 32;                 // slots of a tile
    static constexpr int HALVES = D / 64;
    static constexpr int MT = KT / 16;            // 16-slot blocks
    static constexpr int KS = D / 16;
    static constexpr int TILE_BYTES = KT * D * 2, STAGE_BYTES = 2 * TILE_BYTES;
    static constexpr int W = 2, THREADS = (W + 2) * 32;  // producer, consumers, epilogue
    static constexpr int PER_SM = D == 64 ? 4 : 2;  // CTAs per SM: 64 KB of cache on the way in each
    static constexpr int NS = 4;                  // stages: a multiple of W, a stage is always read by the same consumer
    static constexpr int ROWS = 8 * NR;
    static constexpr int Q_HALF = ROWS * 128, Q_SLOT = Q_HALF * HALVES;
    static constexpr int PS = D + 4;              // floats of a partial row: O, m, l, padding
    static constexpr int PBUFS = 2;
    static constexpr int PBUF_FLOATS = W * ROWS * PS;
    static constexpr int FIXED = 1024 + NS * STAGE_BYTES + 2 * Q_SLOT + PBUFS * PBUF_FLOATS * 4 + 32 * 8;
    static __host__ __device__ int bytes(int n_seqs) { return FIXED + n_seqs * 16 + 2 * (n_seqs + 1) * 4 + 16 * 4; }
};

template <int D, int NR>
__global__ void __launch_bounds__(FewShape<D, NR>::THREADS, FewShape<D, NR>::PER_SM) paged_attn_few_kernel(const __grid_constant__ TcArgs ta, const __grid_constant__ TcMaps maps) {
    using S = FewShape<D, NR>;
    using Work = TcWork<1, S::KT, D>;
    constexpr int KT = S::KT, W = S::W, NS = S::NS, HALVES = S::HALVES;
    const PagedAttnArgs& a = ta.a;
    extern __shared__ unsigned char smem_raw[];
    const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    unsigned char* gbase = smem_raw + (base - smem_u32(smem_raw));
    const uint32_t ring = base, qring = base + NS * S::STAGE_BYTES;
    float* pbuf = reinterpret_cast<float*>(gbase + NS * S::STAGE_BYTES + 2 * S::Q_SLOT);
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
    if (ta.split) asm volatile("griddepcontrol.launch_dependents;" ::: "memory");  // (the joining kernel waits for this one's end)
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
        // ------------------------------------------------------------------ producer
        int issued = 0, segs = 0;
        RingPos kv;
        bool ok = true;
        const int nbox = KT / ta.box_rows;  // boxes of 64 columns of a tile (at most 4)
        const int is_v = lane >> 3, idx = lane & 7, box = idx & (nbox - 1), half = idx / nbox;
        const bool boxes = lane < 16 && half < HALVES;
        const int box_slot = box * ta.box_rows, row_mask = a.kv.page_tokens - 1;
        const int cap = a.kv.table_cols << a.kv.page_shift;
        const uint32_t dst0 = ring + is_v * S::TILE_BYTES + half * (KT * 128) + box_slot * 128;
        const CUtensorMap* map = is_v ? &maps.v : &maps.k;
        TcSeg g;
        while (ok && work.next(g)) {
            const int n = g.nb, len = min(g.len, cap), lo = g.lo;
            if (n == 0) continue;
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
            int page = page_of(slot);
            const int qs = segs & 1;
            if (segs >= 2 && !(ok = warp_wait(q_empty(qs), ((segs >> 1) - 1) & 1, abort_flag))) break;
            ++segs;
            if (lane == 0) {
                mbar_expect_tx(q_full(qs), (uint32_t)(a.tq * a.group * 128 * HALVES));
#pragma unroll
                for (int h = 0; h < HALVES; ++h) tma_load_4d(qring + qs * S::Q_SLOT + h * S::Q_HALF, &maps.q, h * 64, 0, g.head, g.tok0, q_full(qs));
            }
            for (int j = 0; j < n; ++j) {
                const int page_next = j + 1 < n ? page_of(slot + KT) : 0;
                if (issued >= NS && !(ok = warp_wait(empty(kv.st), kv.ph ^ 1, abort_flag))) break;
                if (lane == 0) mbar_expect_tx(full(kv.st), S::STAGE_BYTES);
                __syncwarp();
                if (boxes) tma_load_4d(dst0 + kv.st * S::STAGE_BYTES, map, half * 64, slot & row_mask, head_c, page, full(kv.st));
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
        const float sc = a.scale_log2;
        int t = cw, t_base = 0;   // next tile of this warp, first tile of the segment (in the CTA's list)
        int segs = 0, all_segs = 0;
        RingPos rp;
        rp.st = cw;
        bool ok = true;
        // byte offset of 16-byte chunk c of row r of a tile with `rows` rows (128-byte swizzle)
        auto off = [](int rows, int r, int c) { return (uint32_t)((c >> 3) * rows * 128 + r * 128 + (((c & 7) ^ (r & 7)) << 4)); };
        TcSeg g;
        while (ok && work.next(g)) {
            const int n = g.nb;
            float m[NR][2], l[NR][2], o[NR][S::KS][4];
            int last[NR][2];  // last slot of rows 8 nr + 2 quad, + 1
#pragma unroll
            for (int r = 0; r < NR; ++r) {
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const int row = 8 * r + 2 * quad + e;
                    m[r][e] = -INFINITY;
                    l[r][e] = 0.f;
                    last[r][e] = row >= g.n_tok * G ? -1 : a.causal ? min(g.slot0 + row / G, g.len - 1) : g.len - 1;
                }
#pragma unroll
                for (int k = 0; k < S::KS; ++k) o[r][k][0] = o[r][k][1] = o[r][k][2] = o[r][k][3] = 0.f;
            }
            const int min_last = a.causal ? min(g.slot0, g.len - 1) : g.len - 1;
            if (n > 0) {
                const int qs = segs & 1;
                if (!(ok = warp_wait(q_full(qs), (segs >> 1) & 1, abort_flag))) break;
                ++segs;
                uint32_t qf[NR][S::KS][2];  // B operand: column = row of the unit, 16 elements per k-step
                const uint32_t qa = qring + qs * S::Q_SLOT;
#pragma unroll
                for (int r = 0; r < NR; ++r)
#pragma unroll
                    for (int k = 0; k < S::KS; k += 2) {
                        uint32_t f[4];
                        ldmatrix_x4(qa + off(S::ROWS, 8 * r + (lane & 7), 2 * k + (lane >> 3)), f);
                        qf[r][k][0] = f[0];
                        qf[r][k][1] = f[1];
                        qf[r][k + 1][0] = f[2];
                        qf[r][k + 1][1] = f[3];
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
                        // value rows of slots that are not live: their weight is 0, but 0 * NaN is not
                        for (int i = lane; i < KT * HALVES * 8; i += 32) {
                            const int c = i & 7, r = (i >> 3) & (KT - 1), h = i / (KT * 8);
                            if (base_slot + r < g.lo || base_slot + r >= g.len)
                                asm volatile("st.shared.v4.u32 [%0], {%1, %1, %1, %1};" ::"r"(vt + h * KT * 128 + r * 128 + c * 16), "r"(0) : "memory");
                        }
                        __syncwarp();
                    }
                    // S^T[slot][row]
                    float s[S::MT][NR][4];
#pragma unroll
                    for (int mt = 0; mt < S::MT; ++mt) {
#pragma unroll
                        for (int r = 0; r < NR; ++r) s[mt][r][0] = s[mt][r][1] = s[mt][r][2] = s[mt][r][3] = 0.f;
#pragma unroll
                        for (int k = 0; k < S::KS; ++k) {
                            uint32_t f[4];
                            ldmatrix_x4(kt + off(KT, 16 * mt + (lane & 15), 2 * k + (lane >> 4)), f);
#pragma unroll
                            for (int r = 0; r < NR; ++r) mma_bf16(s[mt][r], f[0], f[1], f[2], f[3], qf[r][k][0], qf[r][k][1]);
                        }
                    }
                    // this thread: slots 16 mt + qrow (+ 8), rows 8 r + 2 quad (+ 1)
                    if (base_slot < g.lo || base_slot + KT - 1 > min_last) {
#pragma unroll
                        for (int mt = 0; mt < S::MT; ++mt)
#pragma unroll
                            for (int e = 0; e < 4; ++e) {
                                const int slot = base_slot + 16 * mt + qrow + (e >> 1) * 8;
#pragma unroll
                                for (int r = 0; r < NR; ++r)
                                    if (slot < g.lo || slot > last[r][e & 1]) s[mt][r][e] = -INFINITY;
                            }
                    }
                    uint32_t pb[S::MT][NR][2];  // P^T as B operand
#pragma unroll
                    for (int r = 0; r < NR; ++r) {
                        float corr[2], ref[2];
#pragma unroll
                        for (int e = 0; e < 2; ++e) {
                            float mx = fmaxf(s[0][r][e], s[0][r][2 + e]);
#pragma unroll
                            for (int mt = 1; mt < S::MT; ++mt) mx = fmaxf(mx, fmaxf(s[mt][r][e], s[mt][r][2 + e]));
#pragma unroll
                            for (int w = 4; w <= 16; w <<= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, w));
                            const float mn = fmaxf(m[r][e], mx);
                            ref[e] = softmax_ref(mn);
                            corr[e] = ex2_approx((m[r][e] - ref[e]) * sc);
                            m[r][e] = mn;
                            l[r][e] *= corr[e];
                        }
#pragma unroll
                        for (int mt = 0; mt < S::MT; ++mt) {
#pragma unroll
                            for (int e = 0; e < 4; ++e) s[mt][r][e] = ex2_approx((s[mt][r][e] - ref[e & 1]) * sc);
                            l[r][0] += s[mt][r][0] + s[mt][r][2];
                            l[r][1] += s[mt][r][1] + s[mt][r][3];
                            pb[mt][r][0] = movmatrix_trans(pack_bf16(s[mt][r][0], s[mt][r][1]));
                            pb[mt][r][1] = movmatrix_trans(pack_bf16(s[mt][r][2], s[mt][r][3]));
                        }
                        if (__any_sync(0xffffffffu, corr[0] != 1.f || corr[1] != 1.f)) {
#pragma unroll
                            for (int k = 0; k < S::KS; ++k) {
                                o[r][k][0] *= corr[0];
                                o[r][k][1] *= corr[1];
                                o[r][k][2] *= corr[0];
                                o[r][k][3] *= corr[1];
                            }
                        }
                    }
                    // O^T[element][row] += V^T P^T
#pragma unroll
                    for (int k = 0; k < S::KS; ++k)
#pragma unroll
                        for (int mt = 0; mt < S::MT; ++mt) {
                            uint32_t f[4];
                            ldmatrix_x4_trans(vt + off(KT, 16 * mt + (lane & 7) + 8 * (lane >> 4), 2 * k + ((lane >> 3) & 1)), f);
#pragma unroll
                            for (int r = 0; r < NR; ++r) mma_bf16(o[r][k], f[0], f[1], f[2], f[3], pb[mt][r][0], pb[mt][r][1]);
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
#pragma unroll
                    for (int k = 0; k < S::KS; ++k) {
                        p[16 * k + qrow] = o[r][k][e];
                        p[16 * k + 8 + qrow] = o[r][k][2 + e];
                    }
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
                    __nv_bfloat16* dst = reinterpret_cast<__nv_bfloat16*>(a.out.p) + (long long)(g.tok0 + t) * a.out.token_stride +
                                         (long long)(g.head * G + row - t * G) * a.out.head_stride + e;
                    *reinterpret_cast<uint2*>(dst) = make_uint2(pack_bf16(o.x * inv, o.y * inv), pack_bf16(o.z * inv, o.w * inv));
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

}  // namespace lar
