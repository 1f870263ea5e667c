// Host side of the attention over slots that sequences have in common: argument checks, launch shapes, launches.
#include "../../include/lar.h"

#include <cuda_runtime.h>
#include <limits.h>

#include "paged_launch.cuh"
#include "paged_shared.cuh"

namespace {

using namespace lar;

// Rows of a KV head per sequence above which the slots in common are read once per sequence as ever (the rows of one sequence fill the row tiles that
// share a read).
constexpr int kSharedRows = 128;

size_t up256(size_t n) { return (n + 255) / 256 * 256; }

struct SharedPlan {
    bool apart;            // the slots in common apart; else lar_paged_attn as it is
    AttnPlan pass[2];
    size_t ints, rows, ws0, ws1, bytes;
};

lar_paged_kv_t groups_of(const lar_paged_kv_t& k, int n_groups) {
    lar_paged_kv_t g = k;
    g.n_seqs = n_groups;
    return g;
}

int64_t own_len(int64_t cap, int max_len, int max_shared) {
    const int64_t len = max_len > 0 && max_len < cap ? max_len : cap;
    return max_shared > 0 && max_shared < len ? len - max_shared : len;
}

SharedPlan shared_plan(const lar_paged_kv_t& k, int group, int64_t n_tokens, int n_groups, int max_chunk, int max_len, int max_shared) {
    SharedPlan p;
    memset(&p, 0, sizeof(p));
    const int64_t cap = (int64_t)k.table_cols * k.page_tokens, chunk = max_chunk > 0 ? max_chunk : (n_tokens + k.n_seqs - 1) / k.n_seqs;
    const int hq = k.n_kv_heads * group, d = k.head_dim;
    p.apart = chunk * group <= kSharedRows && n_tokens * group <= (int64_t)k.n_seqs * kSharedRows;
    if (!p.apart) return p;
    const int64_t per_group = (n_tokens + n_groups - 1) / n_groups;
    p.pass[0] = attn_plan(groups_of(k, n_groups), group, n_tokens, (int)per_group, max_shared > 0 && max_shared < cap ? max_shared : (int)cap, true, true);
    p.pass[1] = attn_plan(k, group, n_tokens, (int)chunk, (int)own_len(cap, max_len, max_shared), true, true);
    if (k.dtype == LAR_BF16)
        for (AttnPlan& w : p.pass)
            if (w.splits == 3) {  // (whole units round-robin: the counter of units on demand is cleared by a copy between the kernels)
                w.splits = 1;
                w.bytes = 0;
            }
    if (k.dtype == LAR_BF16 && p.pass[0].nt == 2) {
        // Two row tiles have an SM to themselves: the passes run side by side, each on a share of the SMs as its work is (else one behind the other, the second's CTAs
        // taking the place of the first's): microseconds of an SM for a slot of a unit, where two row tiles keep
        // the tensor cores busy (2 us for 128 slots) or a slot's bytes pass (44 GB/s), and as many slots more as taking up a unit costs (TcWork).  Own
        // lengths are taken as half of what they may be, few rows' bytes pass faster.  (64 images of one prompt, 8192 slots in common: 45 us, 51 one behind the other.)
        auto work = [&](const AttnPlan& w, double units, double slots) {
            const double cost = w.nt == 2 ? 256 : w.nt == 1 ? (d == 64 ? 192 : 128) : (d == 64 ? 256 : 128);
            return units * k.n_kv_heads * (slots + cost) * (w.nt == 2 ? 2.0 / 128 : 4.0 * d / 44e3);
        };
        auto tiles = [](int64_t tokens, const AttnPlan& w) { return (tokens + w.tq * (w.nt == 2 ? 2 : 1) - 1) / (w.tq * (w.nt == 2 ? 2 : 1)); };
        const double work0 = (p.pass[1].nt == 0 ? 1.5 : 1.0) * work(p.pass[0], (double)n_groups * tiles(per_group, p.pass[0]), (double)(max_shared > 0 && max_shared < cap ? max_shared : cap));
        const double work1 = work(p.pass[1], (double)(n_tokens < k.n_seqs ? n_tokens : k.n_seqs) * tiles(chunk, p.pass[1]), own_len(cap, max_len, max_shared) / 2.0);
        int share = (int)(kSms * work0 / (work0 + work1) + 0.5);
        share = share < 8 ? 8 : share > kSms - 8 ? kSms - 8 : share;
        // Units that the kernel would leave whole are not looked at for cutting (3 us).
        const int64_t units = (n_tokens / (2 * p.pass[0].tq) + (n_tokens < n_groups ? n_tokens : n_groups)) * k.n_kv_heads;
        const int64_t common = max_shared > 0 && max_shared < cap ? max_shared : cap;
        if (p.pass[0].splits == 2 && common < 2048 && (units >= share || (common / 128 + 2) * (share - units) < kCutTilesJoined * share)) {
            p.pass[0].splits = 1;
            p.pass[0].bytes = 0;
        }
        p.pass[0].grid = p.pass[0].grid / kSms * share;
        p.pass[1].grid = p.pass[1].grid / kSms * (kSms - share);
    }
    p.ints = up256(((size_t)n_groups * 3 + 1 + k.n_seqs) * sizeof(int));
    const size_t row = (size_t)hq * (d + 2) * sizeof(float);
    if (k.dtype == LAR_BF16) {
        p.rows = up256((size_t)n_tokens * (row + hq * sizeof(int2)));
        p.ws0 = up256(p.pass[0].bytes);
        p.ws1 = up256(p.pass[1].bytes);
        p.bytes = p.ints + 2 * p.rows + p.ws0 + p.ws1;
    } else {  // the passes' parts are what is joined
        p.ws0 = up256(p.pass[0].splits * (size_t)n_tokens * row);
        p.ws1 = up256(p.pass[1].splits * (size_t)n_tokens * row);
        p.bytes = p.ints + p.ws0 + p.ws1;
    }
    return p;
}

bool shared_args(const lar_paged_kv_t* kv, int n_q_heads, int64_t n_tokens, int n_groups, int max_chunk, int max_len, int max_shared) {
    if (n_q_heads < 1 || n_q_heads % kv->n_kv_heads || n_q_heads / kv->n_kv_heads > 16) return false;
    return n_tokens >= 0 && n_groups >= 1 && max_chunk >= 0 && max_len >= 0 && max_shared >= 0;
}

}  // namespace

extern "C" {

size_t lar_paged_attn_shared_workspace_bytes(const lar_paged_kv_t* kv, int n_q_heads, int64_t n_tokens, int n_groups, int max_chunk, int max_len,
                                             int max_shared) {
    PagedView v;
    if (n_tokens < 1 || !paged_view(kv, n_tokens, kv ? kv->lens : nullptr, v) || !shared_args(kv, n_q_heads, n_tokens, n_groups, max_chunk, max_len, max_shared))
        return 0;
    const int group = n_q_heads / kv->n_kv_heads, d = kv->head_dim;
    const int64_t chunk = max_chunk > 0 ? max_chunk : n_tokens;
    const size_t whole = attn_workspace_bound(*kv, group, n_tokens, (int)(chunk > INT_MAX ? INT_MAX : chunk), max_len);
    // Apart: no more rows than the sequences have of the longest chunks that are taken apart; a pass is a call of its own with any lengths up to the bounds
    const int64_t most = (int64_t)kv->n_seqs * kSharedRows / group, n = n_tokens < most ? n_tokens : most;
    if (n < 1) return whole;
    const size_t row = (size_t)n_q_heads * ((d + 2) * sizeof(float) + (kv->dtype == LAR_BF16 ? sizeof(int2) : 0)), ints = up256(((size_t)n_groups * 3 + 1 + kv->n_seqs) * sizeof(int));
    const size_t a = attn_workspace_bound(groups_of(*kv, n_groups), group, n, (int)n, max_shared, true);
    const size_t b = attn_workspace_bound(*kv, group, n, (int)(chunk < kSharedRows / group ? chunk : kSharedRows / group), max_len, true);
    // (fp32: one part at least; the bounds hold from two parts on)
    const size_t rows = (size_t)n * row;
    const size_t apart = kv->dtype == LAR_BF16 ? ints + 2 * up256(rows) + up256(a) + up256(b) : ints + up256(a > rows ? a : rows) + up256(b > rows ? b : rows);
    return apart > whole ? apart : whole;
}

lar_status_t lar_paged_attn_shared(const lar_paged_kv_t* kv, const lar_rows_t* q, const lar_rows_t* out, int n_q_heads, int64_t n_tokens,
                                   const int32_t* cu_tokens, int n_groups, const int32_t* cu_groups, const int32_t* shared_lens, int causal,
                                   float softmax_scale, int max_chunk, int max_len, int max_shared, void* workspace, size_t workspace_bytes,
                                   void* stream) {
    PagedAttnArgs a;
    memset(&a, 0, sizeof(a));
    if (!paged_view(kv, n_tokens, cu_tokens, a.kv) || !shared_args(kv, n_q_heads, n_tokens, n_groups, max_chunk, max_len, max_shared)) return LAR_ERR_INVALID_ARG;
    if (!(softmax_scale >= 0.f) || !isfinite(softmax_scale)) return LAR_ERR_INVALID_ARG;
    if (!cu_groups || !shared_lens || !aligned(cu_groups, 4) || !aligned(shared_lens, 4)) return LAR_ERR_INVALID_ARG;
    if (n_tokens == 0) return LAR_OK;
    const int group = n_q_heads / kv->n_kv_heads, elt = elt_of(kv->dtype), d = kv->head_dim;
    if (!rows_view(q, n_tokens, n_q_heads, d, elt, false, a.q) || !rows_view(out, n_tokens, n_q_heads, d, elt, true, a.out)) return LAR_ERR_INVALID_ARG;
    if (workspace && !aligned(workspace, 16)) return LAR_ERR_INVALID_ARG;
    if (kv->n_seqs > kTcMaxSeqs || n_groups > kTcMaxSeqs) return LAR_ERR_CAPACITY;
    const SharedPlan p = shared_plan(*kv, group, n_tokens, n_groups, max_chunk, max_len, max_shared);
    if (!workspace || !p.apart)
        return lar_paged_attn(kv, q, out, n_q_heads, n_tokens, cu_tokens, nullptr, causal, softmax_scale, max_chunk, max_len, workspace, workspace_bytes, stream);
    if (p.bytes > workspace_bytes) return LAR_ERR_NOMEM;
    if (kv->dtype == LAR_BF16 && (!countable(groups_of(*kv, n_groups), p.pass[0], n_tokens) || !countable(*kv, p.pass[1], n_tokens))) return LAR_ERR_CAPACITY;
    cudaStream_t s = (cudaStream_t)stream;
    char* at = static_cast<char*>(workspace);
    SharedPrepArgs pr;
    memset(&pr, 0, sizeof(pr));
    pr.kv = a.kv;
    pr.groups = cu_groups;
    pr.shared = shared_lens;
    pr.n_groups = n_groups;
    pr.cu = reinterpret_cast<int*>(at);
    pr.len = pr.cu + n_groups + 1;
    pr.row_of = pr.len + n_groups;
    pr.start = pr.row_of + n_groups;
    at += p.ints;
    shared_prep_kernel<<<(unsigned)n_groups, kSharedPrepThreads, 0, s>>>(pr);
    LAR_CUDA(cudaGetLastError());

    a.group = group;
    a.scale_log2 = (softmax_scale > 0.f ? softmax_scale : 1.0f / sqrtf((float)d)) * 1.4426950408889634f;
    a.parts = 2;
    SharedJoinArgs j;
    memset(&j, 0, sizeof(j));
    j.kv = a.kv;
    j.out = a.out;
    j.cu = pr.cu;
    j.n_groups = n_groups;
    j.hq = n_q_heads;
    j.scale_log2 = a.scale_log2;
    const lar_paged_kv_t kg = groups_of(*kv, n_groups);
    for (int w = 0; w < 2; ++w) {
        const AttnPlan& plan = p.pass[w];
        SharedPass& left = j.pass[w];
        PagedAttnArgs b = a;
        b.tq = plan.tq;
        b.n_splits = plan.splits;
        if (w == 0) {
            b.kv.n_seqs = n_groups;
            b.kv.cu = pr.cu;
            b.kv.lens = pr.len;
            b.kv.lens_stride = 1;
            b.kv.row_of = pr.row_of;
            b.causal = 0;
        } else {
            b.start = pr.start;
            b.causal = causal != 0;
        }
        lar_status_t st;
        if (kv->dtype == LAR_BF16) {
            b.row_o = reinterpret_cast<float*>(at);
            b.row_ml = b.row_o + (size_t)n_tokens * n_q_heads * d;
            b.row_ref = reinterpret_cast<int2*>(b.row_ml + (size_t)n_tokens * n_q_heads * 2);
            at += p.rows;
            b.part_o = reinterpret_cast<float*>(at);
            left.row_o = b.row_o;
            left.row_ml = b.row_ml;
            left.parts = 1;
            left.ranges = plan.grid;
            left.range_rows = (plan.nt == 2 ? 2 : 1) * plan.rows_cap;
            if (plan.splits == 2) {  // as launch_tc lays it out
                left.row_ref = b.row_ref;
                left.part_ml = reinterpret_cast<const float*>(reinterpret_cast<int4*>(at) + plan.grid);
                left.part_o = left.part_ml + (size_t)plan.grid * 2 * left.range_rows * 2;
            }
            st = launch_bf16<true>(w == 0 ? kg : *kv, b, plan, s);
        } else {
            b.part_o = reinterpret_cast<float*>(at);
            b.part_ml = b.part_o + (size_t)plan.splits * n_tokens * n_q_heads * d;
            left.row_o = b.part_o;
            left.row_ml = b.part_ml;
            left.parts = plan.splits;
            st = d == 64 ? launch_fp32<64>(b, plan, s, false) : launch_fp32<128>(b, plan, s, false);
        }
        at += w == 0 ? p.ws0 : p.ws1;
        if (st != LAR_OK) return st;
    }
    const int64_t ctas = n_tokens * n_q_heads;
    cudaLaunchConfig_t lc;
    memset(&lc, 0, sizeof(lc));
    lc.gridDim = dim3((unsigned)(ctas < 4 * kSms ? ctas : 4 * kSms), 1, 1);
    lc.blockDim = dim3(kSharedJoinThreads, 1, 1);
    lc.stream = s;
    cudaLaunchAttribute attr;
    attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr.val.programmaticStreamSerializationAllowed = 1;
    lc.attrs = &attr;
    lc.numAttrs = 1;
    void (*fn)(const SharedJoinArgs) = kv->dtype == LAR_BF16 ? (d == 64 ? shared_join_kernel<__nv_bfloat16, 64> : shared_join_kernel<__nv_bfloat16, 128>)
                                                             : (d == 64 ? shared_join_kernel<float, 64> : shared_join_kernel<float, 128>);
    LAR_CUDA(cudaLaunchKernelEx(&lc, fn, (const SharedJoinArgs)j));
    return LAR_OK;
}

}  // extern "C"
