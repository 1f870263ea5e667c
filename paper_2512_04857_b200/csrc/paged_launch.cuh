// Launch shapes and launches of the chunk attention over bf16 and fp32 caches, shared by its entry points.
#pragma once
#include <math.h>
#include <string.h>

#include "host_util.h"
#include "paged_attn_few.cuh"
#include "paged_attn_fp32.cuh"
#include "paged_attn_tc.cuh"
#include "paged_host.h"
#include "tensor_map.h"

namespace lar {

// Where rows are joined with others anyway: slot tiles that a range has at least (bf16), slots that a CTA has (fp32).
constexpr int kPartItems = 3, kPartSlots = 64;
// Slots above which units of two row tiles that leave CTAs idle may be cut there (2 KV heads, 64 rows of 4 heads of 128, whole / cut: 512 slots 24.0 / 23.0 us, 768 27.4 / 24.4,
// 1024 30.3 / 24.0, 1536 37 / 23; 8 KV heads 23.8 / 24.4, 26.9 / 24.7, 30.1 / 24.2, 36 / 25.6).
constexpr int kJoinedLen = 640;

struct AttnPlan {
    int tq;        // tokens of a row tile
    int nt;        // bf16: row tiles of a CTA (0: the kernel for few rows)
    int nr;        // bf16, few rows: blocks of 8 rows (two with 64-element rows only)
    int stages, grid, rows_cap;  // bf16: K/V ring, persistent CTAs, rows of a row tile
    int splits;    // bf16: 1 units stay whole, 2 they may be cut, 3 they are handed out on demand; fp32: CTAs along a unit's slots
    int bm, tiles; // fp32: rows of a tile, bound on the row tiles of all sequences
    size_t bytes;  // workspace
    size_t smem;
};

template <int NT>
size_t tc_smem(int d, int rows_cap, int stages, int n_seqs) {
    return d == 64 ? TcSmem<64, NT>::bytes(rows_cap, stages, n_seqs) : TcSmem<128, NT>::bytes(rows_cap, stages, n_seqs);
}

// joined: the rows are joined with others behind the kernel anyway, so that cutting a unit costs no launch.
inline AttnPlan attn_plan(const lar_paged_kv_t& k, int group, int64_t n_tokens, int max_chunk, int max_len, bool split, bool joined = false) {
    AttnPlan p;
    memset(&p, 0, sizeof(p));
    const int64_t chunk = max_chunk > 0 ? max_chunk : (n_tokens + k.n_seqs - 1) / k.n_seqs;
    const int64_t cap = (int64_t)k.table_cols * k.page_tokens;
    const int64_t len = max_len > 0 && max_len < cap ? max_len : cap;
    const int64_t with_tokens = n_tokens < k.n_seqs ? n_tokens : k.n_seqs;
    const int d = k.head_dim;
    if (k.dtype == LAR_BF16) {
        // Two row tiles above 128 rows, and with 128-element rows and long caches above 32 (one row tile leaves its two CTAs per SM two
        // stages each; 16 x 4288 slots, one / two row tiles: 32 rows 62 / 65 us, 64 rows 75 / 66, 128 rows 78 / 69, 192 rows 120 / 74; 64 x 577
        // slots, 64 rows 55 / 59; 64-element rows 44 / 55, 48 / 56, 72 / 68).  All of it with 8 KV heads: how few units a call has is not looked at, here and in
        // what is cut below (one sequence of 300 tokens over 1500 slots: 40 units on 148 SMs).
        const int64_t rows = chunk * group;
        p.nt = rows > 128 || (d == 128 && rows > 32 && len >= 2048) ? 2 : rows > few_rows(d) ? 1 : 0;
        if (p.nt == 0) {
            p.tq = (int)chunk;
            p.rows_cap = p.tq * group;
            p.nr = p.rows_cap > 8 ? 2 : 1;
            p.smem = d == 64 ? (p.nr == 1 ? FewShape<64, 1>::bytes(k.n_seqs) : FewShape<64, 2>::bytes(k.n_seqs))
                             : FewShape<128, 1>::bytes(k.n_seqs);
            const int fit = (int)(233472 / (p.smem + 1024)), want = d == 64 ? FewShape<64, 1>::PER_SM : FewShape<128, 1>::PER_SM;
            p.grid = (fit < want ? fit : want) * kSms;
            // Units of few slots, or short ones that fill the SMs, stay whole: joining costs a launch (one token, 8 KV heads, cut / whole: 1 to
            // 64 sequences of up to 300 slots 8.3 / 7.7 to 12.1 / 9.0 us; up to 577 slots: 4 sequences 9.4 / 10.8, 64 14.6 / 12.0; up to 1153:
            // 37 15.2 / 17.9, 64 of unlike length 15.9 / 18.5).
            const bool cut = split && (joined ? len > 128 : len > 384 && (len > 640 || with_tokens * k.n_kv_heads < 2 * kSms));
            p.splits = cut ? 2 : 1;
            if (cut) p.bytes = (size_t)p.grid * (sizeof(int4) + 2 * (size_t)p.rows_cap * (d + 2) * sizeof(float));
            return p;
        }
        p.tq = 128 / group;
        if (p.nt == 1 && chunk < p.tq) p.tq = (int)chunk;
        p.rows_cap = (p.tq * group + 7) / 8 * 8;
        int per_sm = 1;
        if (p.nt == 2) {
            p.stages = kTcMaxStages;
            while (p.stages > 1 && tc_smem<2>(d, p.rows_cap, p.stages, k.n_seqs) > kMaxSmem) --p.stages;
            p.smem = tc_smem<2>(d, p.rows_cap, p.stages, k.n_seqs);
        } else {
            // two CTAs per SM, unless the lengths of very many sequences leave no room for two stages each
            constexpr size_t kHalf = 233472 / 2 - 1024;
            p.stages = kTcMaxStages;
            while (p.stages > 2 && tc_smem<1>(d, p.rows_cap, p.stages, k.n_seqs) > kHalf) --p.stages;
            per_sm = tc_smem<1>(d, p.rows_cap, p.stages, k.n_seqs) <= kHalf ? 2 : 1;
            p.smem = tc_smem<1>(d, p.rows_cap, p.stages, k.n_seqs);
        }
        p.grid = per_sm * kSms;
        // One row tile: cut above 1280 slots (8 tokens of 64-element rows, 8 KV heads, cut / whole: 37 sequences of up to 577 slots 22 / 14 us,
        // up to 1153 28 / 20, up to 2000 36 / 31, of unlike length 29 / 30, up to 4100 43 / 54; 16 sequences 18 / 14, 22 / 20, 25 / 29,
        // 34 / 52 at the same lengths).  Two: whole units on demand where there are many, or where their lengths differ much (chunks
        // that make up much of their cache); long units are cut where a few rounds of whole ones would leave CTAs idle (joined: shorter ones too).
        const int64_t units = (n_tokens / (p.tq * p.nt) + with_tokens) * k.n_kv_heads;
        p.splits = 1;
        if (split && (p.nt == 1 ? len > (joined ? 128 : 1280) : joined && units <= p.grid ? len > kJoinedLen : units < 4 * p.grid && len >= 2048 && (2 * chunk < len || units <= p.grid))) p.splits = 2;
        else if (split && p.nt == 2 && units > p.grid) p.splits = 3;
        if (p.splits == 2) p.bytes = (size_t)p.grid * (sizeof(int4) + 2 * p.nt * (size_t)p.rows_cap * (d + 2) * sizeof(float));
        if (p.splits == 3) p.bytes = sizeof(int4);
        return p;
    }
    p.bm = chunk * group <= 8 ? 8 : chunk * group <= 16 ? 16 : 64;
    p.tq = p.bm / group;
    const int64_t tiles = n_tokens / p.tq + with_tokens;
    p.tiles = (int)(tiles < n_tokens ? tiles : n_tokens);
    p.splits = 1;
    if (split) {
        const int64_t units = (int64_t)p.tiles * k.n_kv_heads;
        int64_t s = (12 * kSms + units - 1) / units;  // four rounds of three CTAs per SM: the last one costs little
        const int64_t least = joined ? kPartSlots : 256;  // slots that a CTA has at least
        if (s > (len + least - 1) / least) s = (len + least - 1) / least;
        if (s > 64) s = 64;
        // Few rows: short units that fill the SMs by themselves are not worth joining (one token, 8 KV heads, cut / whole: 37 sequences of up
        // to 577 slots 25.8 / 24.3 us, with 128-element rows 42.5 / 39.8, 16 of them 31.6 / 42.1; 64 sequences 37.4 / 32.0, of up to 1153
        // slots 60 / 58, with 128-element rows 103 / 112).
        if (!joined && p.bm < 64 && len <= 768 && units >= 2 * kSms) s = 1;
        p.splits = s < 1 ? 1 : (int)s;
    }
    p.bytes = p.splits > 1 ? (size_t)p.splits * n_tokens * k.n_kv_heads * group * (d + 2) * sizeof(float) : 0;
    return p;
}

// Workspace of a call and of every smaller one: the largest need over the launch shapes that attn_plan may choose for at most these
// sequences, tokens, tokens of a chunk (0: n_tokens) and entries (0: what the table holds).  A call's own need goes up and down with its
// sizes (fewer units are cut into more parts), and a program has one workspace for all of its calls.
inline size_t attn_workspace_bound(const lar_paged_kv_t& k, int group, int64_t n_tokens, int max_chunk, int max_len, bool joined = false) {
    const int64_t chunk = max_chunk > 0 ? max_chunk : n_tokens;
    const int64_t cap = (int64_t)k.table_cols * k.page_tokens;
    const int64_t len = max_len > 0 && max_len < cap ? max_len : cap;
    const int d = k.head_dim;
    if (k.dtype == LAR_BF16) {
        lar_paged_kv_t one = k;  // (few sequences leave shared memory for most CTAs)
        one.n_seqs = 1;
        const int few = few_rows(d);
        size_t most = 0;
        auto take = [&](size_t n) { most = n > most ? n : most; };
        // few rows: each chunk length is a launch shape; where any length up to len is cut, one near len is
        for (int64_t c = 1; c <= chunk && c * group <= few; ++c) {
            AttnPlan p = attn_plan(one, group, 1, (int)c, len > 640 ? 641 : (int)len, true, joined);
            take(p.bytes);
        }
        // one row tile (of two CTAs per SM at most), then two: their rows are bounded by the 128 of a tile
        const int64_t t1 = chunk < 128 / group ? chunk : 128 / group;
        const size_t part = (size_t)(d + 2) * sizeof(float), rows = (size_t)(t1 * group + 7) / 8 * 8, rows2 = (size_t)(128 / group * group + 7) / 8 * 8;
        if (chunk * group > few && len > (joined ? 128 : 1280)) take(2 * kSms * (sizeof(int4) + 2 * rows * part));
        if (chunk * group > 128 || (d == 128 && chunk * group > 32 && len >= 2048))
            take(len > (joined ? kJoinedLen : 2047) ? kSms * (sizeof(int4) + 4 * rows2 * part) : sizeof(int4));
        return most;
    }
    // fp32: s splits of n tokens, s <= 12 kSms / units + 1 with at least n / tq * KV heads units, so that s n <= 12 kSms tq / KV heads + n; and
    // two splits or more only where there are fewer than 12 kSms units
    const int bm = chunk * group <= 8 ? 8 : chunk * group <= 16 ? 16 : 64;
    const int64_t spread = 12ll * kSms * (bm / group) / k.n_kv_heads, n = n_tokens < spread ? n_tokens : spread;
    const int64_t least = joined ? kPartSlots : 256;
    int64_t s = (len + least - 1) / least;
    s = s > 64 ? 64 : s;
    if (s < 2) return 0;
    const int64_t rows = s * n < spread + n ? s * n : spread + n;
    return (size_t)rows * k.n_kv_heads * group * (d + 2) * sizeof(float);
}

// fp32 storage: row tiles of 64, 16 or 8.
template <int D>
lar_status_t launch_fp32(const PagedAttnArgs& a, const AttnPlan& p, cudaStream_t s, bool join = true) {
    void (*fn)(const PagedAttnArgs) = p.bm == 64   ? paged_attn_tf32_kernel<D, false>
                                           : p.bm == 16 ? paged_attn_tf32_kernel<D, true>
                                                        : paged_attn_tf32_decode_kernel<D>;
    const int smem = p.bm == 64   ? Tf32Shape<D, false>::SMEM
                     : p.bm == 16 ? Tf32Shape<D, true>::SMEM
                                  : Tf32DecodeShape<D>::SMEM;
    LAR_CUDA(cudaFuncSetAttribute((const void*)fn, cudaFuncAttributeMaxDynamicSharedMemorySize, smem));
    cudaLaunchConfig_t lc;
    memset(&lc, 0, sizeof(lc));
    lc.gridDim = dim3((unsigned)p.tiles, (unsigned)a.kv.n_kv_heads, (unsigned)p.splits);
    lc.blockDim = dim3(kFp32Threads, 1, 1);
    lc.dynamicSmemBytes = smem;
    lc.stream = s;
    cudaLaunchAttribute at;
    at.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at.val.programmaticStreamSerializationAllowed = 1;
    lc.attrs = &at;
    lc.numAttrs = a.parts == 2 ? 1 : 0;  // (waits by itself)
    LAR_CUDA(cudaLaunchKernelEx(&lc, fn, a));
    if (p.splits > 1 && join) {
        const int64_t rows = (int64_t)a.kv.n_tokens * a.kv.n_kv_heads * a.group;
        combine_splits_kernel<D><<<(unsigned)((rows + 3) / 4), 128, 0, s>>>(a);
        LAR_CUDA(cudaGetLastError());
    }
    return LAR_OK;
}

inline lar_status_t make_maps(const lar_paged_kv_t& k, const PagedAttnArgs& a, int box_rows, TcMaps& m) {
    const cuuint64_t d = (cuuint64_t)k.head_dim;
    const cuuint64_t qdim[4] = {d, (cuuint64_t)a.group, (cuuint64_t)k.n_kv_heads, (cuuint64_t)a.kv.n_tokens};
    const int64_t qst[3] = {a.q.head_stride, a.q.head_stride * a.group, a.q.token_stride};
    const cuuint32_t qbox[4] = {64, (cuuint32_t)a.group, 1, (cuuint32_t)a.tq};
    lar_status_t st = encode_map<4>(&m.q, kMapBf16, 128, a.q.p, qdim, qst, qbox);
    const int heads = k.head_stride > 0 ? k.n_kv_heads : 1;  // heads with pages of their own: every page is one head's
    const int64_t page_stride = k.n_pages > 1 ? k.page_stride : k.row_stride * k.page_tokens * heads;
    const cuuint64_t kdim[4] = {d, (cuuint64_t)k.page_tokens, (cuuint64_t)heads, (cuuint64_t)k.n_pages};
    const int64_t kst[3] = {k.row_stride, heads > 1 ? k.head_stride : page_stride, page_stride};
    const cuuint32_t kbox[4] = {64, (cuuint32_t)box_rows, 1, 1};
    if (st == LAR_OK) st = encode_map<4>(&m.k, kMapBf16, 128, k.k_pool, kdim, kst, kbox);
    if (st == LAR_OK) st = encode_map<4>(&m.v, kMapBf16, 128, k.v_pool, kdim, kst, kbox);
    return st;
}

// The bf16 kernels: NT row tiles of 128 rows, or (NT = 0) few rows in NR blocks of 8.
template <int D, int NT, int NR, bool PART>
struct TcKernel {
    static constexpr int BN = TcShape<D, NT>::BN, THREADS = TcShape<D, NT>::THREADS;
    static constexpr auto fn = paged_attn_tc_kernel<D, NT, PART>;
};
template <int D, int NR, bool PART>
struct TcKernel<D, 0, NR, PART> {
    static constexpr int BN = FewShape<D, NR>::KT, THREADS = FewShape<D, NR>::THREADS;
    static constexpr auto fn = paged_attn_few_kernel<D, NR, PART>;
};

template <int D, int NT_, int NR = 0, bool PART = false>
lar_status_t launch_tc(const lar_paged_kv_t& k, const PagedAttnArgs& a, const AttnPlan& p, cudaStream_t s) {
    using S = TcKernel<D, NT_, NR, PART>;
    constexpr int NT = NT_ == 0 ? 1 : NT_;
    TcArgs t;
    memset(&t, 0, sizeof(t));
    TcMaps m;
    t.a = a;
    t.stages = p.stages;
    t.rows_cap = p.rows_cap;
    t.box_rows = k.page_tokens < S::BN ? k.page_tokens : S::BN;
    t.split = p.splits == 2;
    t.min_items = PART ? kPartItems : 6;
    if (p.splits == 3) {
        t.counter = reinterpret_cast<int*>(a.part_o);
        LAR_CUDA(cudaMemsetAsync(t.counter, 0, sizeof(int), s));
    }
    if (t.split) {  // records, then (m, l), then O of every CTA's two parts
        t.records = reinterpret_cast<int4*>(a.part_o);
        t.a.part_ml = reinterpret_cast<float*>(t.records + p.grid);
        t.a.part_o = t.a.part_ml + (size_t)p.grid * 2 * NT * p.rows_cap * 2;
    }
    // First of all a call of the runtime, which makes the device's context current in a thread that has made none: encoding a tensor map is a
    // call of the driver and fails without one.
    constexpr auto fn = S::fn;
    // (The limit is the same whatever a call launches with: another thread's call may come between this one and the launch.)
    LAR_CUDA(cudaFuncSetAttribute((const void*)fn, cudaFuncAttributeMaxDynamicSharedMemorySize, kMaxSmem));
    lar_status_t st = make_maps(k, a, t.box_rows, m);
    if (st != LAR_OK) return st;
    if (NT_ == 2) {
        // the softmax warps take registers that the block has to have been launched with: a build that gives it fewer is refused
        static const int regs = [] {
            cudaFuncAttributes at;
            return cudaFuncGetAttributes(&at, (const void*)S::fn) == cudaSuccess ? at.numRegs : 0;
        }();
        if (regs * 3 < 2 * TcShape<D, 2>::SM_REGS + TcShape<D, 2>::OTHER_REGS) return LAR_ERR_CUDA;
    }
    // A kernel whose rows are joined elsewhere is launched before its predecessor's end: it waits for it by itself (the joining kernel likewise).
    cudaLaunchConfig_t lc;
    memset(&lc, 0, sizeof(lc));
    lc.gridDim = dim3((unsigned)p.grid, 1, 1);
    lc.blockDim = dim3(S::THREADS, 1, 1);
    lc.dynamicSmemBytes = p.smem;
    lc.stream = s;
    cudaLaunchAttribute at;
    at.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at.val.programmaticStreamSerializationAllowed = 1;
    lc.attrs = &at;
    lc.numAttrs = PART ? 1 : 0;
    LAR_CUDA(cudaLaunchKernelEx(&lc, fn, (const TcArgs)t, (const TcMaps)m));
    if (t.split && !PART) {
        lc.gridDim = dim3((unsigned)p.grid, (unsigned)((NT * p.rows_cap * (D / 4) + 511) / 512), 1);
        lc.blockDim = dim3(128, 1, 1);
        lc.dynamicSmemBytes = 0;
        lc.numAttrs = 1;
        LAR_CUDA(cudaLaunchKernelEx(&lc, join_ranges_kernel<D, NT>, (const TcArgs)t));
    }
    return LAR_OK;
}

// The bf16 kernel that a plan has chosen.
template <bool PART>
lar_status_t launch_bf16(const lar_paged_kv_t& k, const PagedAttnArgs& a, const AttnPlan& p, cudaStream_t s) {
    const int d = k.head_dim;
    if (p.nt == 2) return d == 64 ? launch_tc<64, 2, 0, PART>(k, a, p, s) : launch_tc<128, 2, 0, PART>(k, a, p, s);
    if (p.nt == 1) return d == 64 ? launch_tc<64, 1, 0, PART>(k, a, p, s) : launch_tc<128, 1, 0, PART>(k, a, p, s);
    if (p.nr == 2) return launch_tc<64, 0, 2, PART>(k, a, p, s);
    return d == 64 ? launch_tc<64, 0, 1, PART>(k, a, p, s) : launch_tc<128, 0, 1, PART>(k, a, p, s);
}

// The bf16 kernels count units and slot tiles in 31 bits.
inline bool countable(const lar_paged_kv_t& k, const AttnPlan& p, int64_t n_tokens) {
    const int64_t units = (n_tokens / p.tq + (n_tokens < k.n_seqs ? n_tokens : k.n_seqs)) * k.n_kv_heads;
    const int64_t tiles = ((int64_t)k.table_cols * k.page_tokens + 31) / 32 + 4;
    return units <= (1ll << 30) / tiles;
}

}  // namespace lar
