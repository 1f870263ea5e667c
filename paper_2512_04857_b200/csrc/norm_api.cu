// Host side of the head norms and of the 8-bit cache's append and read-back: argument checks, launches.
#include "../../include/lar.h"

#include <cuda_runtime.h>
#include <math.h>
#include <string.h>

#include "host_util.h"
#include "norm_rope.cuh"
#include "paged_host.h"

namespace {

using namespace lar;

bool norm_view(const lar_head_norm_t* n, int heads, int d, HeadNormView& v) {
    memset(&v, 0, sizeof(v));
    if (!n) return true;
    if (n->struct_size != sizeof(lar_head_norm_t) || (n->kind != LAR_NORM_RMS && n->kind != LAR_NORM_LAYER) || !is_dtype(n->weight_dtype)) return false;
    if (!(n->eps >= 1e-12f) || !(n->eps <= 1.0f)) return false;
    if (!aligned(n->weight, 16) || !aligned(n->bias, 16) || n->head_stride < 0 || n->head_stride > (1ll << 36)) return false;
    const int64_t stride = heads > 1 ? n->head_stride : 0;
    if (stride * elt_of(n->weight_dtype) % 16 || (stride > 0 && stride < d)) return false;
    v.weight = static_cast<const char*>(n->weight);
    v.bias = static_cast<const char*>(n->bias);
    v.head_stride = stride;
    v.eps = n->eps;
    v.on = 1;
    v.layer = n->kind == LAR_NORM_LAYER;
    v.bf16 = n->weight_dtype == LAR_BF16;
    return true;
}

using NormFn = void (*)(const NormRopeArgs);
template <typename T, int D, int DEST>
NormFn norm_fn_pairs(bool inter) { return inter ? norm_rope_kernel<T, D, true, DEST> : norm_rope_kernel<T, D, false, DEST>; }
template <int DEST>
NormFn norm_fn(int dtype, int d, bool inter) {
    if (dtype == LAR_BF16) return d == 64 ? norm_fn_pairs<__nv_bfloat16, 64, DEST>(inter) : norm_fn_pairs<__nv_bfloat16, 128, DEST>(inter);
    return d == 64 ? norm_fn_pairs<float, 64, DEST>(inter) : norm_fn_pairs<float, 128, DEST>(inter);
}

lar_status_t launch_norm(NormRopeArgs& a, NormFn fn, int d, int elt, cudaStream_t s) {
    const int ipr = d * elt / 32;  // threads of a row
    // The number of threads that leaves fewest of them without a row.  A kind whose heads a CTA holds several times over has as many tokens in a pass; one
    // with more heads takes several CTAs.
    int threads = 0, best_rows = 0;
    double best = 0.0;
    for (int n = kNormThreads; n >= 128; n -= 32) {
        const int rows = n / ipr;
        double used = 0.0, all = 0.0;
        for (int i = 0; i < 3; ++i) {
            const int heads = a.r.heads[i];
            if (heads == 0) continue;
            const int slices = (heads + rows - 1) / rows, per = (heads + slices - 1) / slices;
            used += heads;
            all += (double)slices * rows / (rows / per);
        }
        if (used / all > best + 1e-9) {
            best = used / all;
            threads = n;
            best_rows = rows;
        }
    }
    int slices = 0;
    for (int i = 0; i < 3; ++i) {
        const int heads = a.r.heads[i];
        if (heads == 0) continue;
        a.slices[i] = (heads + best_rows - 1) / best_rows;
        a.heads[i] = (heads + a.slices[i] - 1) / a.slices[i];
        a.at_once[i] = best_rows / a.heads[i];
        slices += a.slices[i];
    }
    // Tokens of a CTA: what it sets up serves all of them, but there should be some rounds of CTAs.
    int64_t tokens = (int64_t)a.r.n_tokens * slices / (8 * kSms);
    tokens = tokens < 1 ? 1 : tokens > kNormTokens ? kNormTokens : tokens;
    a.tokens = (int)tokens;
    fn<<<dim3((unsigned)((a.r.n_tokens + tokens - 1) / tokens), (unsigned)slices), threads, 0, s>>>(a);
    LAR_CUDA(cudaGetLastError());
    return LAR_OK;
}

// What the appends have in common: everything but the cache.  rows_dtype: of q, k and v.
bool append_args(NormRopeArgs& a, int rows_dtype, int n_kv_heads, int d, const lar_head_norm_t* q_norm, const lar_head_norm_t* k_norm,
                 const lar_rope_t* rope, const int32_t* pos, int64_t pos_axis_stride, const lar_rows_t* k, const lar_rows_t* v,
                 const lar_rows_t* q, const lar_rows_t* q_out, int n_q_heads, int64_t n_tokens) {
    if (rope && (!rope_freqs(rope, 0, a.r.f) || rope->head_dim != d)) return false;
    if (!norm_view(q_norm, n_q_heads, d, a.norm[0]) || !norm_view(k_norm, n_kv_heads, d, a.norm[1])) return false;
    if (n_tokens == 0) return true;
    if ((rope != nullptr) != (pos != nullptr) || !aligned(pos, 4)) return false;
    if (rope && rope->n_axes > 1 && pos_axis_stride < n_tokens) return false;
    if (n_q_heads < 0 || n_q_heads > kMaxHeads || (n_q_heads > 0) != (q != nullptr) || (q != nullptr) != (q_out != nullptr)) return false;
    if (q_norm && !q) return false;
    const int elt = elt_of(rows_dtype);
    if (q && (!rows_view(q, n_tokens, n_q_heads, d, elt, false, a.r.src[0]) || !rows_view(q_out, n_tokens, n_q_heads, d, elt, true, a.r.dst[0])))
        return false;
    if (!rows_view(k, n_tokens, n_kv_heads, d, elt, false, a.r.src[1]) || !rows_view(v, n_tokens, n_kv_heads, d, elt, false, a.r.src[2])) return false;
    a.r.pos = pos;
    a.r.pos_axis_stride = pos_axis_stride;
    a.r.heads[0] = n_q_heads;
    a.r.heads[1] = a.r.heads[2] = n_kv_heads;
    a.r.n_tokens = (int)n_tokens;
    return true;
}

}  // namespace

namespace lar {

bool q8_view(const lar_paged_q8_t* c, int64_t n_tokens, const int32_t* cu, PagedView& v, Q8View& q) {
    if (!c || c->struct_size != sizeof(lar_paged_q8_t) || c->reserved || !paged_view(&c->kv, n_tokens, cu, v, true)) return false;
    if (c->kv.k_pool == c->kv.v_pool || c->k_scale == c->v_scale) return false;
    if (!c->k_scale || !c->v_scale || !aligned(c->k_scale, 16) || !aligned(c->v_scale, 16)) return false;
    // the attention's copies take K and V as one tensor with the distance as a stride, which a tensor map holds below 2^40 bytes
    auto far = [](const void* x, const void* y) {
        const uintptr_t p = reinterpret_cast<uintptr_t>(x), q = reinterpret_cast<uintptr_t>(y);
        return (p < q ? q - p : p - q) >= ((uintptr_t)1 << 40);
    };
    if (far(c->kv.k_pool, c->kv.v_pool) || far(c->k_scale, c->v_scale)) return false;
    const int64_t strides[2] = {c->scale_page_stride, c->scale_head_stride};
    for (int64_t s : strides)
        if (s < 0 || s > (1ll << 36) || s % 16) return false;
    if (c->kv.n_pages > 1 && c->scale_page_stride < c->kv.page_tokens) return false;
    // heads that share a page's rows have bytes of their own
    if (c->kv.n_kv_heads > 1 && c->kv.head_stride > 0 && c->scale_head_stride < c->kv.page_tokens) return false;
    if (c->kv.head_stride == 0 && c->kv.n_kv_heads > 1 && c->scale_head_stride != 0) return false;
    q.k_scale = c->k_scale;
    q.v_scale = c->v_scale;
    q.page_stride = c->scale_page_stride;
    q.head_stride = c->kv.n_kv_heads > 1 ? c->scale_head_stride : 0;
    return true;
}

lar_status_t paged_append_norm(const lar_paged_kv_t& kv, const lar_head_norm_t* q_norm, const lar_head_norm_t* k_norm, const lar_rope_t* rope,
                               const int32_t* pos, int64_t pos_axis_stride, const lar_rows_t* k, const lar_rows_t* v, const lar_rows_t* q,
                               const lar_rows_t* q_out, int n_q_heads, int64_t n_tokens, const int32_t* cu_tokens, const OwnCache* own,
                               void* stream) {
    if (!q_norm && !k_norm) return paged_append(kv, rope, pos, pos_axis_stride, k, v, q, q_out, n_q_heads, n_tokens, cu_tokens, own, stream);
    NormRopeArgs a;
    memset(&a, 0, sizeof(a));
    if (!paged_view(&kv, n_tokens, cu_tokens, a.r.kv)) return LAR_ERR_INVALID_ARG;
    if (!append_args(a, kv.dtype, kv.n_kv_heads, kv.head_dim, q_norm, k_norm, rope, pos, pos_axis_stride, k, v, q, q_out, n_q_heads, n_tokens))
        return LAR_ERR_INVALID_ARG;
    if (n_tokens == 0) return LAR_OK;
    if (own) {
        a.r.index_map = own->index_map;
        a.r.state = own->state;
        a.r.cap_pad = own->cap_pad;
    }
    return launch_norm(a, norm_fn<1>(kv.dtype, kv.head_dim, rope && rope->interleaved), kv.head_dim, elt_of(kv.dtype), (cudaStream_t)stream);
}

}  // namespace lar

extern "C" {

lar_status_t lar_norm_rope_rotate(const lar_head_norm_t* q_norm, const lar_head_norm_t* k_norm, const lar_rope_t* rope, int dtype, int head_dim,
                                  const int32_t* pos, int64_t pos_axis_stride, int64_t n_tokens, const lar_rows_t* q, const lar_rows_t* q_out,
                                  int n_q_heads, const lar_rows_t* k, const lar_rows_t* k_out, int n_kv_heads, void* stream) {
    NormRopeArgs a;
    memset(&a, 0, sizeof(a));
    if (!is_dtype(dtype) || !(head_dim == 64 || head_dim == 128) || n_tokens < 0 || n_tokens > kMaxTokens) return LAR_ERR_INVALID_ARG;
    if (rope && (!rope_freqs(rope, 0, a.r.f) || rope->head_dim != head_dim)) return LAR_ERR_INVALID_ARG;
    if (rope && rope->n_axes > 1 && pos_axis_stride < n_tokens) return LAR_ERR_INVALID_ARG;
    if (n_q_heads < 1 || n_q_heads > kMaxHeads || n_kv_heads < 0 || n_kv_heads > kMaxHeads) return LAR_ERR_INVALID_ARG;
    if ((n_kv_heads > 0) != (k != nullptr) || (k != nullptr) != (k_out != nullptr) || (k_norm && !k)) return LAR_ERR_INVALID_ARG;
    if (!norm_view(q_norm, n_q_heads, head_dim, a.norm[0]) || !norm_view(k_norm, n_kv_heads, head_dim, a.norm[1])) return LAR_ERR_INVALID_ARG;
    if (n_tokens == 0) return LAR_OK;
    if ((rope != nullptr) != (pos != nullptr) || !aligned(pos, 4)) return LAR_ERR_INVALID_ARG;
    const int elt = elt_of(dtype);
    if (!rows_view(q, n_tokens, n_q_heads, head_dim, elt, false, a.r.src[0]) || !rows_view(q_out, n_tokens, n_q_heads, head_dim, elt, true, a.r.dst[0]))
        return LAR_ERR_INVALID_ARG;
    if (k && (!rows_view(k, n_tokens, n_kv_heads, head_dim, elt, false, a.r.src[1]) || !rows_view(k_out, n_tokens, n_kv_heads, head_dim, elt, true, a.r.dst[1])))
        return LAR_ERR_INVALID_ARG;
    a.r.pos = pos;
    a.r.pos_axis_stride = pos_axis_stride;
    a.r.heads[0] = n_q_heads;
    a.r.heads[1] = n_kv_heads;
    a.r.n_tokens = (int)n_tokens;
    return launch_norm(a, norm_fn<0>(dtype, head_dim, rope && rope->interleaved), head_dim, elt, (cudaStream_t)stream);
}

lar_status_t lar_paged_append_norm_rope(const lar_paged_kv_t* kv, const lar_head_norm_t* q_norm, const lar_head_norm_t* k_norm, const lar_rope_t* rope,
                                        const int32_t* pos, int64_t pos_axis_stride, const lar_rows_t* k, const lar_rows_t* v,
                                        const lar_rows_t* q, const lar_rows_t* q_out, int n_q_heads, int64_t n_tokens, const int32_t* cu_tokens,
                                        void* stream) {
    if (!kv) return LAR_ERR_INVALID_ARG;
    return lar::paged_append_norm(*kv, q_norm, k_norm, rope, pos, pos_axis_stride, k, v, q, q_out, n_q_heads, n_tokens, cu_tokens, nullptr, stream);
}

lar_status_t lar_paged_q8_append(const lar_paged_q8_t* cache, int rows_dtype, const lar_head_norm_t* q_norm, const lar_head_norm_t* k_norm,
                                 const lar_rope_t* rope, const int32_t* pos, int64_t pos_axis_stride, const lar_rows_t* k, const lar_rows_t* v,
                                 const lar_rows_t* q, const lar_rows_t* q_out, int n_q_heads, int64_t n_tokens, const int32_t* cu_tokens,
                                 void* stream) {
    NormRopeArgs a;
    memset(&a, 0, sizeof(a));
    if (!is_dtype(rows_dtype) || !q8_view(cache, n_tokens, cu_tokens, a.r.kv, a.q8)) return LAR_ERR_INVALID_ARG;
    const int d = cache->kv.head_dim;
    if (!append_args(a, rows_dtype, cache->kv.n_kv_heads, d, q_norm, k_norm, rope, pos, pos_axis_stride, k, v, q, q_out, n_q_heads, n_tokens))
        return LAR_ERR_INVALID_ARG;
    if (n_tokens == 0) return LAR_OK;
    return launch_norm(a, norm_fn<2>(rows_dtype, d, rope && rope->interleaved), d, elt_of(rows_dtype), (cudaStream_t)stream);
}

lar_status_t lar_paged_q8_read(const lar_paged_q8_t* cache, int rows_dtype, const lar_rows_t* k_out, const lar_rows_t* v_out, int64_t n_rows,
                               const int32_t* cu_rows, void* stream) {
    Q8ReadArgs a;
    memset(&a, 0, sizeof(a));
    if (!is_dtype(rows_dtype) || !q8_view(cache, n_rows, cu_rows, a.kv, a.q8)) return LAR_ERR_INVALID_ARG;
    if (n_rows == 0) return LAR_OK;
    const int d = cache->kv.head_dim, heads = cache->kv.n_kv_heads, elt = elt_of(rows_dtype);
    if (!rows_view(k_out, n_rows, heads, d, elt, true, a.out[0]) || !rows_view(v_out, n_rows, heads, d, elt, true, a.out[1])) return LAR_ERR_INVALID_ARG;
    a.rows = 2 * heads;
    // As many tokens as the threads take in one go, while that leaves two CTAs to every SM.
    const int go = kQ8ReadThreads * 4 / (a.rows * (d / 16));
    int64_t tokens = n_rows / (2 * kSms);
    tokens = tokens > go ? go : tokens;
    a.tokens_per_cta = tokens < 1 ? 1 : (int)tokens;
    const unsigned grid = (unsigned)((n_rows + a.tokens_per_cta - 1) / a.tokens_per_cta);
    void (*fn)(const Q8ReadArgs) = rows_dtype == LAR_BF16 ? (d == 64 ? q8_read_kernel<__nv_bfloat16, 64> : q8_read_kernel<__nv_bfloat16, 128>)
                                                          : (d == 64 ? q8_read_kernel<float, 64> : q8_read_kernel<float, 128>);
    fn<<<grid, kQ8ReadThreads, 0, (cudaStream_t)stream>>>(a);
    LAR_CUDA(cudaGetLastError());
    return LAR_OK;
}

}  // extern "C"
