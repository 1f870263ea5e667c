// Host side of the entry points on caller-described paged caches and of the rotary embedding: argument checks, launch
// shapes, launches.  No allocation, no state between calls.
#include "../../include/lar.h"

#include <cuda_runtime.h>
#include <math.h>
#include <string.h>

#include "host_util.h"
#include "paged_attn_fp32.cuh"
#include "paged_attn_few.cuh"
#include "paged_attn_tc.cuh"
#include "paged_host.h"
#include "rope_rows.cuh"

namespace {

constexpr int kSms = 148;             // SMs of a B200 (launch shapes only)
constexpr int64_t kMaxTokens = 1 << 26;
constexpr int kMaxHeads = 4096;       // (the rotary kernel divides row numbers by multiplication: rows of two tokens x rows of one < 2^32)

int elt_of(int dtype) { return dtype == LAR_BF16 ? 2 : 4; }
bool is_dtype(int dtype) { return dtype == LAR_BF16 || dtype == LAR_FP32; }
bool aligned(const void* p, size_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }

bool rope_freqs(const lar_rope_t* r, int inverse, lar::RopeFreqs& f) {
    if (!r || r->struct_size != sizeof(lar_rope_t)) return false;
    if (!(r->head_dim == 64 || r->head_dim == 128) || r->n_axes < 1 || r->n_axes > lar::kRopeMaxAxes) return false;
    if (!(r->theta > 0.0) || !isfinite(r->theta)) return false;
    const int half = r->head_dim / 2;
    const double ln = log(r->theta);
    int first = 0;
    for (int a = 0; a < r->n_axes; ++a) {
        const int n = r->axis_pairs[a];
        if (n < 1 || n > half - first) return false;
        for (int i = 0; i < n; ++i) {
            const double e = r->restart ? (double)i / n : (double)(first + i) / half;
            const double t = exp(-e * ln) * 0.15915494309189533576888;  // 1 / (2 pi)
            f.turns[first + i] = inverse ? -t : t;
            f.axis[first + i] = (unsigned char)a;
        }
        first += n;
    }
    return first == half;
}

// Rows of [tokens][heads][d].  Strides of an extent of one do not matter; output rows may not overlap.
bool rows_view(const lar_rows_t* r, int64_t tokens, int heads, int d, int elt, bool output, lar::RowsView& v) {
    if (!r || !r->data || !aligned(r->data, 16)) return false;
    v.p = static_cast<char*>(r->data);
    v.token_stride = tokens > 1 ? r->token_stride : (int64_t)heads * d;
    v.head_stride = heads > 1 ? r->head_stride : d;
    if (v.token_stride < d || v.head_stride < d) return false;
    if (v.token_stride * elt % 16 || v.head_stride * elt % 16) return false;
    if (v.token_stride > (1ll << 36) || v.head_stride > (1ll << 36)) return false;
    if (output && tokens > 1 && heads > 1 && v.token_stride < (heads - 1) * v.head_stride + d && v.head_stride < (tokens - 1) * v.token_stride + d)
        return false;
    return true;
}

bool paged_view(const lar_paged_kv_t* k, int64_t n_tokens, const int32_t* cu, lar::PagedView& v) {
    if (!k || k->struct_size != sizeof(lar_paged_kv_t) || !is_dtype(k->dtype)) return false;
    if (k->n_seqs < 1 || k->n_kv_heads < 1 || !(k->head_dim == 64 || k->head_dim == 128)) return false;
    if (k->n_kv_heads > kMaxHeads) return false;
    int shift = 4;
    while (shift < 8 && (1 << shift) != k->page_tokens) ++shift;
    if (shift == 8 || k->n_pages < 1 || k->table_cols < 1) return false;
    if ((int64_t)k->table_cols * k->page_tokens > (1ll << 30)) return false;
    const int elt = elt_of(k->dtype);
    if (!k->k_pool || !k->v_pool || !aligned(k->k_pool, 16) || !aligned(k->v_pool, 16)) return false;
    const int64_t strides[3] = {k->page_stride, k->row_stride, k->head_stride};
    for (int64_t s : strides)
        if (s < 0 || s > (1ll << 36) || s * elt % 16) return false;
    if (k->row_stride < k->head_dim || (k->n_pages > 1 && k->page_stride < k->head_dim)) return false;
    // heads share a page's rows at a stride, or have pages of their own
    if (k->n_kv_heads > 1 && k->head_stride < k->head_dim && !(k->head_stride == 0 && k->table_head_stride > 0)) return false;
    if (!k->page_table || !k->lens || !aligned(k->page_table, 4) || !aligned(k->lens, 4) || !aligned(k->status, 4)) return false;
    if (k->table_seq_stride < 0 || k->table_head_stride < 0 || k->lens_stride < 0) return false;
    if (n_tokens < 0 || n_tokens > kMaxTokens || !aligned(cu, 4)) return false;
    if (!cu && n_tokens % k->n_seqs) return false;
    v.k_pool = static_cast<char*>(k->k_pool);
    v.v_pool = static_cast<char*>(k->v_pool);
    v.table = k->page_table;
    v.lens = k->lens;
    v.status = k->status;
    v.page_stride = k->page_stride;
    v.row_stride = k->row_stride;
    v.head_stride = k->head_stride;
    v.table_seq_stride = k->table_seq_stride;
    v.table_head_stride = k->table_head_stride;
    v.lens_stride = k->lens_stride;
    v.n_seqs = k->n_seqs;
    v.n_kv_heads = k->n_kv_heads;
    v.n_pages = k->n_pages;
    v.table_cols = k->table_cols;
    v.page_tokens = k->page_tokens;
    v.page_shift = shift;
    v.cu = cu;
    v.chunk = (int)(n_tokens / k->n_seqs);
    v.n_tokens = (int)n_tokens;
    return true;
}

// ------------------------------------------------------------------------------------------ rotary rows
using RopeFn = void (*)(const lar::RopeRowsArgs);
template <typename T, int D, bool PAGED>
RopeFn rope_fn_pairs(bool inter) { return inter ? lar::rope_rows_kernel<T, D, true, PAGED> : lar::rope_rows_kernel<T, D, false, PAGED>; }
template <bool PAGED>
RopeFn rope_fn(int dtype, int d, bool inter) {
    if (dtype == LAR_BF16) return d == 64 ? rope_fn_pairs<__nv_bfloat16, 64, PAGED>(inter) : rope_fn_pairs<__nv_bfloat16, 128, PAGED>(inter);
    return d == 64 ? rope_fn_pairs<float, 64, PAGED>(inter) : rope_fn_pairs<float, 128, PAGED>(inter);
}

lar_status_t launch_rope_rows(lar::RopeRowsArgs& a, RopeFn fn, int d, cudaStream_t s) {
    a.n_rows = a.heads[0] + a.heads[1] + a.heads[2];
    // One token per CTA while the batch is small, its rows dealt to enough CTAs that every SM has some; two tokens per CTA for
    // large batches (66560 tokens of 40 rows: 204 us, against 214 us with one and 203 us with four; 5193 tokens of fp32: 19.4,
    // 19.3 and 21.7 us).
    a.tokens_per_cta = a.n_tokens >= 16 * kSms ? 2 : 1;
    const int token_blocks = (a.n_tokens + a.tokens_per_cta - 1) / a.tokens_per_cta;
    int slices = token_blocks >= 2 * kSms ? 1 : (2 * kSms + token_blocks - 1) / token_blocks;
    const int most = (a.n_rows + 7) / 8;
    if (slices > most) slices = most;
    a.rows_per_slice = (a.n_rows + slices - 1) / slices;
    slices = (a.n_rows + a.rows_per_slice - 1) / a.rows_per_slice;
    a.rows_magic = a.rows_per_slice > 1 ? (unsigned)((1ull << 32) / (unsigned)a.rows_per_slice + 1ull) : 0u;
    const size_t smem = (size_t)a.tokens_per_cta * (d + 2) * 4;
    fn<<<dim3((unsigned)token_blocks, (unsigned)slices), lar::kRopeThreads, smem, s>>>(a);
    LAR_CUDA(cudaGetLastError());
    return LAR_OK;
}

// ------------------------------------------------------------------------------------------ chunk attention
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
    return d == 64 ? lar::TcSmem<64, NT>::bytes(rows_cap, stages, n_seqs) : lar::TcSmem<128, NT>::bytes(rows_cap, stages, n_seqs);
}

AttnPlan attn_plan(const lar_paged_kv_t& k, int group, int64_t n_tokens, int max_chunk, int max_len, bool split) {
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
        p.nt = rows > 128 || (d == 128 && rows > 32 && len >= 2048) ? 2 : rows > lar::few_rows(d) ? 1 : 0;
        if (p.nt == 0) {
            p.tq = (int)chunk;
            p.rows_cap = p.tq * group;
            p.nr = p.rows_cap > 8 ? 2 : 1;
            p.smem = d == 64 ? (p.nr == 1 ? lar::FewShape<64, 1>::bytes(k.n_seqs) : lar::FewShape<64, 2>::bytes(k.n_seqs))
                             : lar::FewShape<128, 1>::bytes(k.n_seqs);
            const int fit = (int)(233472 / (p.smem + 1024)), want = d == 64 ? lar::FewShape<64, 1>::PER_SM : lar::FewShape<128, 1>::PER_SM;
            p.grid = (fit < want ? fit : want) * kSms;
            // Units of few slots, or short ones that fill the SMs, stay whole: joining costs a launch (one token, 8 KV heads, cut / whole: 1 to
            // 64 sequences of up to 300 slots 8.3 / 7.7 to 12.1 / 9.0 us; up to 577 slots: 4 sequences 9.4 / 10.8, 64 14.6 / 12.0; up to 1153:
            // 37 15.2 / 17.9, 64 of unlike length 15.9 / 18.5).
            const bool cut = split && len > 384 && (len > 640 || with_tokens * k.n_kv_heads < 2 * kSms);
            p.splits = cut ? 2 : 1;
            if (cut) p.bytes = (size_t)p.grid * (sizeof(int4) + 2 * (size_t)p.rows_cap * (d + 2) * sizeof(float));
            return p;
        }
        p.tq = 128 / group;
        if (p.nt == 1 && chunk < p.tq) p.tq = (int)chunk;
        p.rows_cap = (p.tq * group + 7) / 8 * 8;
        int per_sm = 1;
        if (p.nt == 2) {
            p.stages = lar::kTcMaxStages;
            while (p.stages > 1 && tc_smem<2>(d, p.rows_cap, p.stages, k.n_seqs) > lar::kMaxSmem) --p.stages;
            p.smem = tc_smem<2>(d, p.rows_cap, p.stages, k.n_seqs);
        } else {
            // two CTAs per SM, unless the lengths of very many sequences leave no room for two stages each
            constexpr size_t kHalf = 233472 / 2 - 1024;
            p.stages = lar::kTcMaxStages;
            while (p.stages > 2 && tc_smem<1>(d, p.rows_cap, p.stages, k.n_seqs) > kHalf) --p.stages;
            per_sm = tc_smem<1>(d, p.rows_cap, p.stages, k.n_seqs) <= kHalf ? 2 : 1;
            p.smem = tc_smem<1>(d, p.rows_cap, p.stages, k.n_seqs);
        }
        p.grid = per_sm * kSms;
        // One row tile: cut above 1280 slots (8 tokens of 64-element rows, 8 KV heads, cut / whole: 37 sequences of up to 577 slots 22 / 14 us,
        // up to 1153 28 / 20, up to 2000 36 / 31, of unlike length 29 / 30, up to 4100 43 / 54; 16 sequences 18 / 14, 22 / 20, 25 / 29,
        // 34 / 52 at the same lengths).  Two: whole units on demand where there are many, or where their lengths differ much (chunks
        // that make up much of their cache); long units are cut where a few rounds of whole ones would leave CTAs idle.
        const int64_t units = (n_tokens / (p.tq * p.nt) + with_tokens) * k.n_kv_heads;
        p.splits = 1;
        if (split && (p.nt == 1 ? len > 1280 : units < 4 * p.grid && len >= 2048 && (2 * chunk < len || units <= p.grid))) p.splits = 2;
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
        if (s > (len + 255) / 256) s = (len + 255) / 256;  // at least 256 slots each
        if (s > 64) s = 64;
        // Few rows: short units that fill the SMs by themselves are not worth joining (one token, 8 KV heads, cut / whole: 37 sequences of up
        // to 577 slots 25.8 / 24.3 us, with 128-element rows 42.5 / 39.8, 16 of them 31.6 / 42.1; 64 sequences 37.4 / 32.0, of up to 1153
        // slots 60 / 58, with 128-element rows 103 / 112).
        if (p.bm < 64 && len <= 768 && units >= 2 * kSms) s = 1;
        p.splits = s < 1 ? 1 : (int)s;
    }
    p.bytes = p.splits > 1 ? (size_t)p.splits * n_tokens * k.n_kv_heads * group * (d + 2) * sizeof(float) : 0;
    return p;
}

// Workspace of a call and of every smaller one: the largest need over the launch shapes that attn_plan may choose for at most these
// sequences, tokens, tokens of a chunk (0: n_tokens) and entries (0: what the table holds).  A call's own need goes up and down with its
// sizes (fewer units are cut into more parts), and a program has one workspace for all of its calls.
size_t attn_workspace_bound(const lar_paged_kv_t& k, int group, int64_t n_tokens, int max_chunk, int max_len) {
    const int64_t chunk = max_chunk > 0 ? max_chunk : n_tokens;
    const int64_t cap = (int64_t)k.table_cols * k.page_tokens;
    const int64_t len = max_len > 0 && max_len < cap ? max_len : cap;
    const int d = k.head_dim;
    if (k.dtype == LAR_BF16) {
        lar_paged_kv_t one = k;  // (few sequences leave shared memory for most CTAs)
        one.n_seqs = 1;
        const int few = lar::few_rows(d);
        size_t most = 0;
        auto take = [&](size_t n) { most = n > most ? n : most; };
        // few rows: each chunk length is a launch shape; where any length up to len is cut, one near len is
        for (int64_t c = 1; c <= chunk && c * group <= few; ++c) {
            AttnPlan p = attn_plan(one, group, 1, (int)c, len > 640 ? 641 : (int)len, true);
            take(p.bytes);
        }
        // one row tile (of two CTAs per SM at most), then two: their rows are bounded by the 128 of a tile
        const int64_t t1 = chunk < 128 / group ? chunk : 128 / group;
        const size_t part = (size_t)(d + 2) * sizeof(float), rows = (size_t)(t1 * group + 7) / 8 * 8, rows2 = (size_t)(128 / group * group + 7) / 8 * 8;
        if (chunk * group > few && len > 1280) take(2 * kSms * (sizeof(int4) + 2 * rows * part));
        if (chunk * group > 128 || (d == 128 && chunk * group > 32 && len >= 2048))
            take(len >= 2048 ? kSms * (sizeof(int4) + 4 * rows2 * part) : sizeof(int4));
        return most;
    }
    // fp32: s splits of n tokens, s <= 12 kSms / units + 1 with at least n / tq * KV heads units, so that s n <= 12 kSms tq / KV heads + n; and
    // two splits or more only where there are fewer than 12 kSms units
    const int bm = chunk * group <= 8 ? 8 : chunk * group <= 16 ? 16 : 64;
    const int64_t spread = 12ll * kSms * (bm / group) / k.n_kv_heads, n = n_tokens < spread ? n_tokens : spread;
    int64_t s = (len + 255) / 256;
    s = s > 64 ? 64 : s;
    if (s < 2) return 0;
    const int64_t rows = s * n < spread + n ? s * n : spread + n;
    return (size_t)rows * k.n_kv_heads * group * (d + 2) * sizeof(float);
}

// fp32 storage: row tiles of 64, 16 or 8.
template <int D>
lar_status_t launch_fp32(const lar::PagedAttnArgs& a, const AttnPlan& p, cudaStream_t s) {
    void (*fn)(const lar::PagedAttnArgs) = p.bm == 64   ? lar::paged_attn_tf32_kernel<D, false>
                                           : p.bm == 16 ? lar::paged_attn_tf32_kernel<D, true>
                                                        : lar::paged_attn_tf32_decode_kernel<D>;
    const int smem = p.bm == 64   ? lar::Tf32Shape<D, false>::SMEM
                     : p.bm == 16 ? lar::Tf32Shape<D, true>::SMEM
                                  : lar::Tf32DecodeShape<D>::SMEM;
    LAR_CUDA(cudaFuncSetAttribute((const void*)fn, cudaFuncAttributeMaxDynamicSharedMemorySize, smem));
    fn<<<dim3((unsigned)p.tiles, (unsigned)a.kv.n_kv_heads, (unsigned)p.splits), lar::kFp32Threads, smem, s>>>(a);
    LAR_CUDA(cudaGetLastError());
    if (p.splits > 1) {
        const int64_t rows = (int64_t)a.kv.n_tokens * a.kv.n_kv_heads * a.group;
        lar::combine_splits_kernel<D><<<(unsigned)((rows + 3) / 4), 128, 0, s>>>(a);
        LAR_CUDA(cudaGetLastError());
    }
    return LAR_OK;
}

typedef CUresult (*EncodeTiledFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                                  const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                                  CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

lar_status_t encode_4d(EncodeTiledFn encode, CUtensorMap* m, void* p, const cuuint64_t (&dim)[4], const int64_t (&stride)[3],
                       const cuuint32_t (&box)[4]) {
    const cuuint32_t one[4] = {1, 1, 1, 1};
    const cuuint64_t st[3] = {(cuuint64_t)stride[0] * 2, (cuuint64_t)stride[1] * 2, (cuuint64_t)stride[2] * 2};
    if (encode(m, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, p, dim, st, box, one, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
               CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) != CUDA_SUCCESS) {
        lar::last_cuda_error() = (int)cudaErrorInvalidValue;
        return LAR_ERR_CUDA;
    }
    return LAR_OK;
}

lar_status_t make_maps(const lar_paged_kv_t& k, const lar::PagedAttnArgs& a, int box_rows, lar::TcMaps& m) {
    static const EncodeTiledFn encode = [] {
        void* fp = nullptr;
        cudaDriverEntryPointQueryResult res;
        if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &fp, cudaEnableDefault, &res) != cudaSuccess || res != cudaDriverEntryPointSuccess) {
            (void)cudaGetLastError();
            fp = nullptr;
        }
        return reinterpret_cast<EncodeTiledFn>(fp);
    }();
    if (!encode) {
        lar::last_cuda_error() = (int)cudaErrorNotSupported;
        return LAR_ERR_CUDA;
    }
    const cuuint64_t d = (cuuint64_t)k.head_dim;
    const cuuint64_t qdim[4] = {d, (cuuint64_t)a.group, (cuuint64_t)k.n_kv_heads, (cuuint64_t)a.kv.n_tokens};
    const int64_t qst[3] = {a.q.head_stride, a.q.head_stride * a.group, a.q.token_stride};
    const cuuint32_t qbox[4] = {64, (cuuint32_t)a.group, 1, (cuuint32_t)a.tq};
    lar_status_t st = encode_4d(encode, &m.q, a.q.p, qdim, qst, qbox);
    const int heads = k.head_stride > 0 ? k.n_kv_heads : 1;  // heads with pages of their own: every page is one head's
    const int64_t page_stride = k.n_pages > 1 ? k.page_stride : k.row_stride * k.page_tokens * heads;
    const cuuint64_t kdim[4] = {d, (cuuint64_t)k.page_tokens, (cuuint64_t)heads, (cuuint64_t)k.n_pages};
    const int64_t kst[3] = {k.row_stride, heads > 1 ? k.head_stride : page_stride, page_stride};
    const cuuint32_t kbox[4] = {64, (cuuint32_t)box_rows, 1, 1};
    if (st == LAR_OK) st = encode_4d(encode, &m.k, k.k_pool, kdim, kst, kbox);
    if (st == LAR_OK) st = encode_4d(encode, &m.v, k.v_pool, kdim, kst, kbox);
    return st;
}

// The bf16 kernels: NT row tiles of 128 rows, or (NT = 0) few rows in NR blocks of 8.
template <int D, int NT, int NR = 0>
struct TcKernel {
    static constexpr int BN = lar::TcShape<D, NT>::BN, THREADS = lar::TcShape<D, NT>::THREADS;
    static constexpr auto fn = lar::paged_attn_tc_kernel<D, NT>;
};
template <int D, int NR>
struct TcKernel<D, 0, NR> {
    static constexpr int BN = lar::FewShape<D, NR>::KT, THREADS = lar::FewShape<D, NR>::THREADS;
    static constexpr auto fn = lar::paged_attn_few_kernel<D, NR>;
};

template <int D, int NT_, int NR = 0>
lar_status_t launch_tc(const lar_paged_kv_t& k, const lar::PagedAttnArgs& a, const AttnPlan& p, cudaStream_t s) {
    using S = TcKernel<D, NT_, NR>;
    constexpr int NT = NT_ == 0 ? 1 : NT_;
    lar::TcArgs t;
    memset(&t, 0, sizeof(t));
    lar::TcMaps m;
    t.a = a;
    t.stages = p.stages;
    t.rows_cap = p.rows_cap;
    t.box_rows = k.page_tokens < S::BN ? k.page_tokens : S::BN;
    t.split = p.splits == 2;
    t.min_items = 6;
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
    LAR_CUDA(cudaFuncSetAttribute((const void*)fn, cudaFuncAttributeMaxDynamicSharedMemorySize, lar::kMaxSmem));
    lar_status_t st = make_maps(k, a, t.box_rows, m);
    if (st != LAR_OK) return st;
    if (NT_ == 2) {
        // the softmax warps take registers that the block has to have been launched with: a build that gives it fewer is refused
        static const int regs = [] {
            cudaFuncAttributes at;
            return cudaFuncGetAttributes(&at, (const void*)S::fn) == cudaSuccess ? at.numRegs : 0;
        }();
        if (regs * 3 < 2 * lar::TcShape<D, 2>::SM_REGS + lar::TcShape<D, 2>::OTHER_REGS) return LAR_ERR_CUDA;
    }
    fn<<<(unsigned)p.grid, S::THREADS, p.smem, s>>>(t, m);
    LAR_CUDA(cudaGetLastError());
    if (t.split) {
        cudaLaunchConfig_t lc;
        memset(&lc, 0, sizeof(lc));
        lc.gridDim = dim3((unsigned)p.grid, (unsigned)((NT * p.rows_cap * (D / 4) + 511) / 512), 1);
        lc.blockDim = dim3(128, 1, 1);
        lc.stream = s;
        cudaLaunchAttribute at;
        at.id = cudaLaunchAttributeProgrammaticStreamSerialization;
        at.val.programmaticStreamSerializationAllowed = 1;
        lc.attrs = &at;
        lc.numAttrs = 1;
        LAR_CUDA(cudaLaunchKernelEx(&lc, lar::join_ranges_kernel<D, NT>, (const lar::TcArgs)t));
    }
    return LAR_OK;
}

}  // namespace

namespace lar {

lar_status_t paged_append(const lar_paged_kv_t& kv, const lar_rope_t* rope, const int32_t* pos, int64_t pos_axis_stride,
                          const lar_rows_t* k, const lar_rows_t* v, const lar_rows_t* q, const lar_rows_t* q_out, int n_q_heads,
                          int64_t n_tokens, const int32_t* cu_tokens, const OwnCache* own, void* stream) {
    lar::RopeRowsArgs a;
    memset(&a, 0, sizeof(a));
    if (!paged_view(&kv, n_tokens, cu_tokens, a.kv)) return LAR_ERR_INVALID_ARG;
    if (rope && (!rope_freqs(rope, 0, a.f) || rope->head_dim != kv.head_dim)) return LAR_ERR_INVALID_ARG;
    if (n_tokens == 0) return LAR_OK;
    if ((rope != nullptr) != (pos != nullptr) || !aligned(pos, 4)) return LAR_ERR_INVALID_ARG;
    if (rope && rope->n_axes > 1 && pos_axis_stride < n_tokens) return LAR_ERR_INVALID_ARG;
    if (n_q_heads < 0 || n_q_heads > kMaxHeads || (n_q_heads > 0) != (q != nullptr) || (q != nullptr) != (q_out != nullptr)) return LAR_ERR_INVALID_ARG;
    const int elt = elt_of(kv.dtype);
    if (q && (!rows_view(q, n_tokens, n_q_heads, kv.head_dim, elt, false, a.src[0]) ||
              !rows_view(q_out, n_tokens, n_q_heads, kv.head_dim, elt, true, a.dst[0])))
        return LAR_ERR_INVALID_ARG;
    if (!rows_view(k, n_tokens, kv.n_kv_heads, kv.head_dim, elt, false, a.src[1]) ||
        !rows_view(v, n_tokens, kv.n_kv_heads, kv.head_dim, elt, false, a.src[2]))
        return LAR_ERR_INVALID_ARG;
    a.pos = pos;
    a.pos_axis_stride = pos_axis_stride;
    a.heads[0] = n_q_heads;
    a.heads[1] = a.heads[2] = kv.n_kv_heads;
    a.n_tokens = (int)n_tokens;
    if (own) {
        a.index_map = own->index_map;
        a.state = own->state;
        a.cap_pad = own->cap_pad;
        a.base_len = 0;
    }
    return launch_rope_rows(a, rope_fn<true>(kv.dtype, kv.head_dim, rope && rope->interleaved), kv.head_dim, (cudaStream_t)stream);
}

}  // namespace lar

extern "C" {

lar_status_t lar_rope_table(const lar_rope_t* rope, const int32_t* pos, int64_t pos_axis_stride, int n_rows, float* cos_sin,
                            void* stream) {
    lar::RopeFreqs f;
    memset(&f, 0, sizeof(f));
    if (!rope_freqs(rope, 0, f) || n_rows < 0 || n_rows > kMaxTokens) return LAR_ERR_INVALID_ARG;
    if (rope->n_axes > 1 && pos_axis_stride < n_rows) return LAR_ERR_INVALID_ARG;
    if (n_rows == 0) return LAR_OK;
    if (!pos || !cos_sin || !aligned(pos, 4) || !aligned(cos_sin, 4)) return LAR_ERR_INVALID_ARG;
    const int half = rope->head_dim / 2;
    long long blocks = ((long long)n_rows * half + lar::kRopeThreads - 1) / lar::kRopeThreads;
    if (blocks > 8 * kSms) blocks = 8 * kSms;
    lar::rope_table_kernel<<<(unsigned)blocks, lar::kRopeThreads, 0, (cudaStream_t)stream>>>(f, pos, pos_axis_stride, n_rows, half, cos_sin);
    LAR_CUDA(cudaGetLastError());
    return LAR_OK;
}

lar_status_t lar_rope_rotate(const lar_rope_t* rope, int dtype, const int32_t* pos, int64_t pos_axis_stride, int64_t n_tokens,
                             const lar_rows_t* q, const lar_rows_t* q_out, int n_q_heads, const lar_rows_t* k,
                             const lar_rows_t* k_out, int n_kv_heads, int inverse, void* stream) {
    lar::RopeRowsArgs a;
    memset(&a, 0, sizeof(a));
    if (!rope_freqs(rope, inverse, a.f) || !is_dtype(dtype) || n_tokens < 0 || n_tokens > kMaxTokens) return LAR_ERR_INVALID_ARG;
    if (rope->n_axes > 1 && pos_axis_stride < n_tokens) return LAR_ERR_INVALID_ARG;
    const int elt = elt_of(dtype), d = rope->head_dim;
    if (n_q_heads < 1 || n_q_heads > kMaxHeads || n_kv_heads < 0 || n_kv_heads > kMaxHeads) return LAR_ERR_INVALID_ARG;
    if ((n_kv_heads > 0) != (k != nullptr) || (k != nullptr) != (k_out != nullptr)) return LAR_ERR_INVALID_ARG;
    if (n_tokens == 0) return LAR_OK;
    if (!pos || !aligned(pos, 4)) return LAR_ERR_INVALID_ARG;
    if (!rows_view(q, n_tokens, n_q_heads, d, elt, false, a.src[0]) || !rows_view(q_out, n_tokens, n_q_heads, d, elt, true, a.dst[0]))
        return LAR_ERR_INVALID_ARG;
    if (k && (!rows_view(k, n_tokens, n_kv_heads, d, elt, false, a.src[1]) || !rows_view(k_out, n_tokens, n_kv_heads, d, elt, true, a.dst[1])))
        return LAR_ERR_INVALID_ARG;
    a.pos = pos;
    a.pos_axis_stride = pos_axis_stride;
    a.heads[0] = n_q_heads;
    a.heads[1] = n_kv_heads;
    a.n_tokens = (int)n_tokens;
    return launch_rope_rows(a, rope_fn<false>(dtype, d, rope->interleaved != 0), d, (cudaStream_t)stream);
}

lar_status_t lar_paged_append_rope(const lar_paged_kv_t* kv, const lar_rope_t* rope, const int32_t* pos, int64_t pos_axis_stride,
                                   const lar_rows_t* k, const lar_rows_t* v, const lar_rows_t* q, const lar_rows_t* q_out,
                                   int n_q_heads, int64_t n_tokens, const int32_t* cu_tokens, void* stream) {
    if (!kv) return LAR_ERR_INVALID_ARG;
    return lar::paged_append(*kv, rope, pos, pos_axis_stride, k, v, q, q_out, n_q_heads, n_tokens, cu_tokens, nullptr, stream);
}

size_t lar_paged_attn_workspace_bytes(const lar_paged_kv_t* kv, int n_q_heads, int64_t n_tokens, int max_chunk, int max_len) {
    lar::PagedView v;
    if (n_tokens < 1 || n_q_heads < 1 || !paged_view(kv, n_tokens, kv ? kv->lens : nullptr, v)) return 0;
    if (n_q_heads % kv->n_kv_heads || n_q_heads / kv->n_kv_heads > 16 || max_chunk < 0 || max_len < 0) return 0;
    return attn_workspace_bound(*kv, n_q_heads / kv->n_kv_heads, n_tokens, max_chunk, max_len);
}

lar_status_t lar_paged_attn(const lar_paged_kv_t* kv, const lar_rows_t* q, const lar_rows_t* out, int n_q_heads, int64_t n_tokens,
                            const int32_t* cu_tokens, const int32_t* kv_start, int causal, float softmax_scale, int max_chunk,
                            int max_len, void* workspace, size_t workspace_bytes, void* stream) {
    lar::PagedAttnArgs a;
    memset(&a, 0, sizeof(a));
    if (!paged_view(kv, n_tokens, cu_tokens, a.kv) || n_q_heads < 1 || n_q_heads % kv->n_kv_heads) return LAR_ERR_INVALID_ARG;
    const int group = n_q_heads / kv->n_kv_heads;
    if (group > 16) return LAR_ERR_INVALID_ARG;
    if (!(softmax_scale >= 0.f) || !isfinite(softmax_scale) || max_chunk < 0 || max_len < 0 || !aligned(kv_start, 4)) return LAR_ERR_INVALID_ARG;
    if (n_tokens == 0) return LAR_OK;
    const int elt = elt_of(kv->dtype), d = kv->head_dim;
    if (!rows_view(q, n_tokens, n_q_heads, d, elt, false, a.q) || !rows_view(out, n_tokens, n_q_heads, d, elt, true, a.out)) return LAR_ERR_INVALID_ARG;
    if (kv->dtype == LAR_BF16 && kv->n_seqs > lar::kTcMaxSeqs) return LAR_ERR_CAPACITY;
    const AttnPlan p = attn_plan(*kv, group, n_tokens, max_chunk, max_len, workspace != nullptr);
    if (workspace && !aligned(workspace, 16)) return LAR_ERR_INVALID_ARG;
    if (p.bytes > workspace_bytes) return LAR_ERR_NOMEM;
    if (kv->dtype == LAR_BF16) {  // the kernel counts units and slot tiles in 31 bits
        const int64_t units = (n_tokens / p.tq + (n_tokens < kv->n_seqs ? n_tokens : kv->n_seqs)) * kv->n_kv_heads;
        const int64_t tiles = ((int64_t)kv->table_cols * kv->page_tokens + 31) / 32 + 4;
        if (units > (1ll << 30) / tiles) return LAR_ERR_CAPACITY;
    }
    a.start = kv_start;
    a.group = group;
    a.causal = causal != 0;
    a.tq = p.tq;
    a.scale_log2 = (softmax_scale > 0.f ? softmax_scale : 1.0f / sqrtf((float)d)) * 1.4426950408889634f;
    a.n_splits = p.splits;
    a.part_o = static_cast<float*>(workspace);
    a.part_ml = p.splits > 1 ? a.part_o + (size_t)p.splits * n_tokens * n_q_heads * d : nullptr;  // (fp32; launch_tc lays its own out)
    cudaStream_t s = (cudaStream_t)stream;
    if (kv->dtype == LAR_BF16) {
        if (p.nt == 2) return d == 64 ? launch_tc<64, 2>(*kv, a, p, s) : launch_tc<128, 2>(*kv, a, p, s);
        if (p.nt == 1) return d == 64 ? launch_tc<64, 1>(*kv, a, p, s) : launch_tc<128, 1>(*kv, a, p, s);
        if (p.nr == 2) return launch_tc<64, 0, 2>(*kv, a, p, s);
        return d == 64 ? launch_tc<64, 0, 1>(*kv, a, p, s) : launch_tc<128, 0, 1>(*kv, a, p, s);
    }
    return d == 64 ? launch_fp32<64>(a, p, s) : launch_fp32<128>(a, p, s);
}

}  // extern "C"
