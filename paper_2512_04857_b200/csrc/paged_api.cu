// Host side of the entry points on caller-described paged caches and of the rotary embedding: argument checks, launch
// shapes, launches.  No allocation, no state between calls.
#include "../../include/lar.h"

#include <cuda_runtime.h>
#include <math.h>
#include <string.h>

#include "host_util.h"
#include "paged_host.h"
#include "paged_launch.cuh"
#include "rope_rows.cuh"

namespace lar {

bool rope_freqs(const lar_rope_t* r, int inverse, RopeFreqs& f) {
    if (!r || r->struct_size != sizeof(lar_rope_t)) return false;
    if (!(r->head_dim == 64 || r->head_dim == 128) || r->n_axes < 1 || r->n_axes > kRopeMaxAxes) return false;
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
bool rows_view(const lar_rows_t* r, int64_t tokens, int heads, int d, int elt, bool output, RowsView& v) {
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

bool paged_view(const lar_paged_kv_t* k, int64_t n_tokens, const int32_t* cu, PagedView& v, bool q8) {
    if (!k || k->struct_size != sizeof(lar_paged_kv_t) || !(q8 ? k->dtype == LAR_E4M3 : is_dtype(k->dtype))) return false;
    if (k->n_seqs < 1 || k->n_kv_heads < 1 || !(k->head_dim == 64 || k->head_dim == 128)) return false;
    if (k->n_kv_heads > kMaxHeads) return false;
    int shift = 4;
    while (shift < 8 && (1 << shift) != k->page_tokens) ++shift;
    if (shift == 8 || k->n_pages < 1 || k->table_cols < 1) return false;
    if ((int64_t)k->table_cols * k->page_tokens > (1ll << 30)) return false;
    const int elt = q8 ? 1 : elt_of(k->dtype);
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

lar_status_t paged_attn_fits(const lar_paged_kv_t& kv, int group, int64_t n_tokens, int max_chunk, int max_len, bool workspace, size_t workspace_bytes) {
    if (kv.dtype == LAR_BF16 && kv.n_seqs > kTcMaxSeqs) return LAR_ERR_CAPACITY;
    const AttnPlan p = attn_plan(kv, group, n_tokens, max_chunk, max_len, workspace);
    if (p.bytes > workspace_bytes) return LAR_ERR_NOMEM;
    return kv.dtype == LAR_BF16 && !countable(kv, p, n_tokens) ? LAR_ERR_CAPACITY : LAR_OK;
}

}  // namespace lar

namespace {

using namespace lar;

// ------------------------------------------------------------------------------------------ rotary rows
// Launch shape of the rotary kernels: token blocks x slices of a token's rows.
dim3 rope_grid(RopeRowsArgs& a) {
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
    return dim3((unsigned)token_blocks, (unsigned)slices);
}

using RopeFn = void (*)(const lar::RopeRowsArgs);
template <typename T, int D, bool PAGED>
RopeFn rope_fn_pairs(bool inter) { return inter ? lar::rope_rows_kernel<T, D, true, PAGED> : lar::rope_rows_kernel<T, D, false, PAGED>; }
template <bool PAGED>
RopeFn rope_fn(int dtype, int d, bool inter) {
    if (dtype == LAR_BF16) return d == 64 ? rope_fn_pairs<__nv_bfloat16, 64, PAGED>(inter) : rope_fn_pairs<__nv_bfloat16, 128, PAGED>(inter);
    return d == 64 ? rope_fn_pairs<float, 64, PAGED>(inter) : rope_fn_pairs<float, 128, PAGED>(inter);
}

lar_status_t launch_rope_rows(lar::RopeRowsArgs& a, RopeFn fn, int d, cudaStream_t s) {
    const dim3 grid = rope_grid(a);
    const size_t smem = (size_t)a.tokens_per_cta * (d + 2) * 4;
    fn<<<grid, lar::kRopeThreads, smem, s>>>(a);
    LAR_CUDA(cudaGetLastError());
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
    if (workspace && !aligned(workspace, 16)) return LAR_ERR_INVALID_ARG;
    const lar_status_t fits = lar::paged_attn_fits(*kv, group, n_tokens, max_chunk, max_len, workspace != nullptr, workspace_bytes);
    if (fits != LAR_OK) return fits;
    const AttnPlan p = attn_plan(*kv, group, n_tokens, max_chunk, max_len, workspace != nullptr);
    a.start = kv_start;
    a.group = group;
    a.causal = causal != 0;
    a.tq = p.tq;
    a.scale_log2 = (softmax_scale > 0.f ? softmax_scale : 1.0f / sqrtf((float)d)) * 1.4426950408889634f;
    a.n_splits = p.splits;
    a.parts = p.splits > 1;
    a.part_o = static_cast<float*>(workspace);
    a.part_ml = p.splits > 1 ? a.part_o + (size_t)p.splits * n_tokens * n_q_heads * d : nullptr;  // (fp32; launch_tc lays its own out)
    cudaStream_t s = (cudaStream_t)stream;
    if (kv->dtype == LAR_BF16) return launch_bf16<false>(*kv, a, p, s);
    return d == 64 ? launch_fp32<64>(a, p, s) : launch_fp32<128>(a, p, s);
}

}  // extern "C"
