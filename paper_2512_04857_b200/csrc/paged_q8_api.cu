// Host side of the attention over 8-bit caches: argument checks, launch shapes, launches.
#include "../../include/lar.h"

#include <cuda_runtime.h>
#include <math.h>
#include <string.h>

#include "host_util.h"
#include "paged_attn_q8.cuh"
#include "paged_host.h"
#include "tensor_map.h"

namespace {

using namespace lar;

struct Q8Plan {
    int few;              // from the codes (else: unpacked first)
    int tq, rows_cap, nr, grid, split;
    size_t smem;
    int cols, batch;      // pages of 128 slots of a sequence, sequences at a time
    size_t table_bytes, dense_bytes;  // of a batch: its page table, its K (and its V)
    size_t bytes;         // workspace, without that of the attention over the unpacked pages
};

template <typename T>
size_t few_smem(int d, int nr, int n_seqs) {
    if (d == 64) return nr == 1 ? Q8Shape<T, 64, 1>::bytes(n_seqs) : Q8Shape<T, 64, 2>::bytes(n_seqs);
    return nr == 1 ? Q8Shape<T, 128, 1>::bytes(n_seqs) : Q8Shape<T, 128, 2>::bytes(n_seqs);
}

constexpr int kCodesRows = 64;  // bf16 rows of a KV head that are computed from the codes
constexpr size_t kUnpackBytes = (size_t)1 << 30;  // unpacked rows at a time

size_t round_up(size_t n, size_t to) { return (n + to - 1) / to * to; }

Q8Plan q8_plan(const lar_paged_kv_t& k, int rows_dtype, int group, int64_t n_tokens, int max_chunk, int max_len, bool split) {
    Q8Plan p;
    memset(&p, 0, sizeof(p));
    const int64_t chunk = max_chunk > 0 ? max_chunk : (n_tokens + k.n_seqs - 1) / k.n_seqs;
    const int64_t cap = (int64_t)k.table_cols * k.page_tokens;
    const int64_t len = max_len > 0 && max_len < cap ? max_len : cap;
    const int d = k.head_dim;
    // From the codes: fp32 rows, and up to 64 rows of bf16 (16 sequences of up to 4288 slots, 8 KV heads of 128, codes / unpacked: 48 bf16 rows 71 / 112 us,
    // 64 92 / 111, 96 about 125 / 110; elements of 64, 64 rows 59 / 62, 96 80 / 65; up to 600 slots, 64 rows 28 / 36; 4 sequences 27 / 42.  fp32, 12 sequences of
    // 2080 to 4160 slots: 64 rows 132 / 336, 2000 rows 3.1 / 5.2 ms, up to 8320 rows 5.4 / 7.2.
    // A bf16 cache takes 46, 62 and 62 us with 32, 64 and 96 rows of 128: from 32 rows on it is the faster one.)
    p.few = rows_dtype == LAR_FP32 || chunk * group <= kCodesRows;
    if (p.few) {
        p.tq = (int)(chunk < kQ8Rows / group ? chunk : kQ8Rows / group);
        p.rows_cap = p.tq * group;
        p.nr = p.rows_cap > 8 ? 2 : 1;
        p.smem = rows_dtype == LAR_BF16 ? few_smem<__nv_bfloat16>(d, p.nr, k.n_seqs) : few_smem<float>(d, p.nr, k.n_seqs);
        const int fit = (int)(233472 / (p.smem + 1024)), want = d == 64 && p.nr == 1 ? 3 : 2;  // Q8Shape::PER_SM
        p.grid = (fit < want ? fit : want) * kSms;
        // Units of few slots, or short ones in some number, stay whole: joining costs a launch (one token, 8 KV heads of 128, cut / whole: up to 300 slots 4
        // sequences 10.3 / 9.5 us, 64 20.5 / 17.3; up to 577: 4 sequences 10.3 / 12.3, 16 13.6 / 13.0, 64 27.4 / 24.7; up to 1153: 64 of unlike
        // length 25.4 / 28.7, with 20 heads 46.6 / 57.9).
        const int64_t seqs = n_tokens < k.n_seqs ? n_tokens : k.n_seqs, tiles = (n_tokens + p.tq - 1) / p.tq, units = (tiles > seqs ? tiles : seqs) * k.n_kv_heads;
        p.split = split && len > 384 && (len > 640 || units < kSms / 2);
        if (p.split) p.bytes = (size_t)p.grid * (sizeof(int4) + 2 * (size_t)p.rows_cap * (d + 2) * sizeof(float));
        return p;
    }
    p.cols = (int)((len + 127) / 128);
    const size_t page = (size_t)128 * k.n_kv_heads * d * 2, seq = 2 * page * p.cols;
    const size_t fit = seq > kUnpackBytes ? 1 : kUnpackBytes / seq;
    p.batch = fit < (size_t)k.n_seqs ? (int)fit : k.n_seqs;
    p.table_bytes = round_up((size_t)p.batch * p.cols * sizeof(int), 256);
    p.dense_bytes = page * p.cols * p.batch;
    p.bytes = p.table_bytes + 2 * p.dense_bytes;
    return p;
}

// The unpacked pages of a batch of sequences as a cache of their own.
lar_paged_kv_t unpacked(const lar_paged_kv_t& k, const Q8Plan& p, int n_seqs, void* workspace) {
    lar_paged_kv_t u = k;
    char* at = static_cast<char*>(workspace);
    u.dtype = LAR_BF16;
    u.n_seqs = n_seqs;
    u.page_tokens = 128;
    u.n_pages = n_seqs * p.cols;
    u.table_cols = p.cols;
    u.head_stride = k.head_dim;
    u.row_stride = (int64_t)k.n_kv_heads * k.head_dim;
    u.page_stride = 128 * u.row_stride;
    u.page_table = reinterpret_cast<const int32_t*>(at);
    u.table_seq_stride = p.cols;
    u.table_head_stride = 0;
    u.k_pool = at + p.table_bytes;
    u.v_pool = at + p.table_bytes + p.dense_bytes;
    return u;
}

template <typename T, int D, int NR>
lar_status_t launch_few(const lar_paged_q8_t& c, const PagedAttnArgs& a, const Q8Plan& p, cudaStream_t s) {
    using S = Q8Shape<T, D, NR>;
    const lar_paged_kv_t& k = c.kv;
    TcArgs t;
    memset(&t, 0, sizeof(t));
    t.a = a;
    t.rows_cap = p.rows_cap;
    t.box_rows = k.page_tokens < S::KT ? k.page_tokens : S::KT;
    t.split = p.split;
    t.min_items = 192 / S::KT;
    if (t.split) {  // records, then (m, l), then O of every CTA's two parts
        t.records = reinterpret_cast<int4*>(a.part_o);
        t.a.part_ml = reinterpret_cast<float*>(t.records + p.grid);
        t.a.part_o = t.a.part_ml + (size_t)p.grid * 2 * p.rows_cap * 2;
    }
    // (First a call of the runtime, then the tensor maps; the limit is the same whatever a call launches with, as other threads' calls may come between.)
    constexpr auto fn = paged_attn_q8_kernel<T, D, NR>;
    LAR_CUDA(cudaFuncSetAttribute((const void*)fn, cudaFuncAttributeMaxDynamicSharedMemorySize, kMaxSmem));
    Q8Maps m;
    const cuuint64_t qdim[4] = {(cuuint64_t)D, (cuuint64_t)a.group, (cuuint64_t)k.n_kv_heads, (cuuint64_t)a.kv.n_tokens};
    const int64_t qst[3] = {a.q.head_stride, a.q.head_stride * a.group, a.q.token_stride};
    const cuuint32_t qbox[4] = {(cuuint32_t)D, (cuuint32_t)a.group, 1, (cuuint32_t)a.tq};
    lar_status_t st = encode_map<4>(&m.q, sizeof(T) == 2 ? kMapBf16 : kMapFp32, 0, a.q.p, qdim, qst, qbox);
    const int heads = k.head_stride > 0 ? k.n_kv_heads : 1;  // heads with pages of their own: every page is one head's
    const int64_t page_stride = k.n_pages > 1 ? k.page_stride : k.row_stride * k.page_tokens * heads;
    const int64_t scale_stride = k.n_pages > 1 ? c.scale_page_stride : (int64_t)k.page_tokens * heads;
    char *kp = static_cast<char*>(k.k_pool), *vp = static_cast<char*>(k.v_pool);
    m.v_first = vp < kp;
    m.v_scale_first = c.v_scale < c.k_scale;
    const cuuint64_t dim[5] = {(cuuint64_t)D, (cuuint64_t)k.page_tokens, (cuuint64_t)heads, (cuuint64_t)k.n_pages, 2};
    const int64_t kst[4] = {k.row_stride, heads > 1 ? k.head_stride : page_stride, page_stride, m.v_first ? kp - vp : vp - kp};
    const cuuint32_t kbox[5] = {(cuuint32_t)D, (cuuint32_t)t.box_rows, 1, 1, 2};
    if (st == LAR_OK) st = encode_map<5>(&m.kv, kMapBytes, D, m.v_first ? vp : kp, dim, kst, kbox, k.row_stride == D ? 256 : D);  // (what lies beside a row is another head's)
    const cuuint64_t sdim[4] = {dim[1], dim[2], dim[3], 2};
    const int64_t sst[3] = {heads > 1 ? c.scale_head_stride : scale_stride, scale_stride, m.v_scale_first ? c.k_scale - c.v_scale : c.v_scale - c.k_scale};
    const cuuint32_t sbox[4] = {(cuuint32_t)t.box_rows, 1, 1, 2};
    if (st == LAR_OK) st = encode_map<4>(&m.scale, kMapBytes, 0, m.v_scale_first ? c.v_scale : c.k_scale, sdim, sst, sbox);
    if (st != LAR_OK) return st;
    fn<<<(unsigned)p.grid, S::THREADS, p.smem, s>>>(t, m);
    LAR_CUDA(cudaGetLastError());
    if (t.split) {
        cudaLaunchConfig_t lc;
        memset(&lc, 0, sizeof(lc));
        lc.gridDim = dim3((unsigned)p.grid, join_ctas(p.rows_cap), 1);
        lc.blockDim = dim3(kJoinThreads, 1, 1);
        lc.stream = s;
        cudaLaunchAttribute at;
        at.id = cudaLaunchAttributeProgrammaticStreamSerialization;
        at.val.programmaticStreamSerializationAllowed = 1;
        lc.attrs = &at;
        lc.numAttrs = 1;
        LAR_CUDA(cudaLaunchKernelEx(&lc, join_parts_kernel<T, D>, (const TcArgs)t));
    }
    return LAR_OK;
}

template <typename T>
lar_status_t launch_few_of(const lar_paged_q8_t& c, const PagedAttnArgs& a, const Q8Plan& p, cudaStream_t s) {
    if (c.kv.head_dim == 64) return p.nr == 1 ? launch_few<T, 64, 1>(c, a, p, s) : launch_few<T, 64, 2>(c, a, p, s);
    return p.nr == 1 ? launch_few<T, 128, 1>(c, a, p, s) : launch_few<T, 128, 2>(c, a, p, s);
}

}  // namespace

extern "C" {

size_t lar_paged_q8_attn_workspace_bytes(const lar_paged_q8_t* cache, int rows_dtype, int n_q_heads, int64_t n_tokens, int max_chunk, int max_len) {
    PagedView v;
    Q8View q8;
    if (n_tokens < 1 || n_q_heads < 1 || !is_dtype(rows_dtype) || !q8_view(cache, n_tokens, cache ? cache->kv.lens : nullptr, v, q8)) return 0;
    const lar_paged_kv_t& k = cache->kv;
    if (n_q_heads % k.n_kv_heads || n_q_heads / k.n_kv_heads > 16 || max_chunk < 0 || max_len < 0) return 0;
    const int group = n_q_heads / k.n_kv_heads;
    const int64_t chunk = max_chunk > 0 ? max_chunk : n_tokens;
    const int64_t cap = (int64_t)k.table_cols * k.page_tokens, len = max_len > 0 && max_len < cap ? max_len : cap;
    // few rows: each chunk length is a launch shape; few sequences leave shared memory for most CTAs
    lar_paged_kv_t one = k;
    one.n_seqs = 1;
    size_t most = 0;
    for (int64_t c = 1; c <= chunk && c * group <= kQ8Rows; ++c) {
        const size_t n = q8_plan(one, rows_dtype, group, 1, (int)c, len > 640 ? 641 : (int)len, true).bytes;
        most = n > most ? n : most;
    }
    if (rows_dtype == LAR_BF16 && chunk * group > kCodesRows) {
        // unpacked rows: at most what is unpacked at a time, or one sequence where that is more; a table of as many pages (at most one for every
        // 16 KB, the smallest page); and the workspace of the attention over them
        const size_t page = (size_t)128 * k.n_kv_heads * k.head_dim * 2, cols = (size_t)((len + 127) / 128);
        const size_t seq = 2 * page * cols, all = seq * k.n_seqs, dense = seq > kUnpackBytes ? seq : all < kUnpackBytes ? all : kUnpackBytes;
        const size_t table = round_up(dense / (2 * page) * sizeof(int), 256);
        const Q8Plan p = q8_plan(k, rows_dtype, group, n_tokens, (int)chunk, (int)len, true);
        lar_paged_kv_t u = unpacked(k, p, k.n_seqs, reinterpret_cast<void*>(256));
        const size_t n = table + dense + lar_paged_attn_workspace_bytes(&u, n_q_heads, n_tokens, (int)(chunk > INT32_MAX ? INT32_MAX : chunk), (int)len);
        most = n > most ? n : most;
    }
    return most;
}

lar_status_t lar_paged_q8_attn(const lar_paged_q8_t* cache, int rows_dtype, const lar_rows_t* q, const lar_rows_t* out, int n_q_heads,
                               int64_t n_tokens, const int32_t* cu_tokens, const int32_t* kv_start, int causal, float softmax_scale,
                               int max_chunk, int max_len, void* workspace, size_t workspace_bytes, void* stream) {
    PagedAttnArgs a;
    Q8View q8;
    memset(&a, 0, sizeof(a));
    if (!is_dtype(rows_dtype) || !q8_view(cache, n_tokens, cu_tokens, a.kv, q8) || n_q_heads < 1 || n_q_heads % cache->kv.n_kv_heads) return LAR_ERR_INVALID_ARG;
    const lar_paged_kv_t& k = cache->kv;
    const int group = n_q_heads / k.n_kv_heads, d = k.head_dim, elt = elt_of(rows_dtype);
    if (group > 16) return LAR_ERR_INVALID_ARG;
    if (!(softmax_scale >= 0.f) || !isfinite(softmax_scale) || max_chunk < 0 || max_len < 0 || !aligned(kv_start, 4)) return LAR_ERR_INVALID_ARG;
    if (n_tokens == 0) return LAR_OK;
    if (!rows_view(q, n_tokens, n_q_heads, d, elt, false, a.q) || !rows_view(out, n_tokens, n_q_heads, d, elt, true, a.out)) return LAR_ERR_INVALID_ARG;
    if (workspace && !aligned(workspace, 16)) return LAR_ERR_INVALID_ARG;
    if (k.n_seqs > kTcMaxSeqs) return LAR_ERR_CAPACITY;
    const Q8Plan p = q8_plan(k, rows_dtype, group, n_tokens, max_chunk, max_len, workspace != nullptr);
    if (p.bytes > workspace_bytes || (!p.few && !workspace)) return LAR_ERR_NOMEM;
    cudaStream_t s = (cudaStream_t)stream;
    if (p.few) {
        // the kernel counts units and slot tiles in 31 bits
        const int64_t units = (n_tokens / p.tq + (n_tokens < k.n_seqs ? n_tokens : k.n_seqs)) * k.n_kv_heads;
        const int64_t tiles = ((int64_t)k.table_cols * k.page_tokens + 31) / 32 + 8;
        if (units > (1ll << 30) / tiles) return LAR_ERR_CAPACITY;
        a.start = kv_start;
        a.group = group;
        a.causal = causal != 0;
        a.tq = p.tq;
        a.scale_log2 = (softmax_scale > 0.f ? softmax_scale : 1.0f / sqrtf((float)d)) * 1.4426950408889634f;
        a.n_splits = 1;
        a.part_o = static_cast<float*>(workspace);
        return rows_dtype == LAR_BF16 ? launch_few_of<__nv_bfloat16>(*cache, a, p, s) : launch_few_of<float>(*cache, a, p, s);
    }
    // Everything that may be refused is, before the first launch: a full batch, and the last one where it is smaller.
    for (int n : {p.batch, k.n_seqs % p.batch}) {
        if (n == 0) continue;
        const lar_status_t st = paged_attn_fits(unpacked(k, p, n, workspace), group, cu_tokens ? n_tokens : (int64_t)n * a.kv.chunk, max_chunk, max_len, true, workspace_bytes - p.bytes);
        if (st != LAR_OK) return st;
    }
    for (int s0 = 0; s0 < k.n_seqs; s0 += p.batch) {
        const int n = k.n_seqs - s0 < p.batch ? k.n_seqs - s0 : p.batch;
        lar_paged_kv_t u = unpacked(k, p, n, workspace);
        u.lens = k.lens + s0 * k.lens_stride;
        Q8UnpackArgs w;
        w.kv = a.kv;
        w.kv.table += s0 * k.table_seq_stride;
        w.kv.lens = u.lens;
        if (cu_tokens) w.kv.cu = cu_tokens + s0;
        w.kv.n_seqs = n;
        w.q8 = q8;
        w.start = kv_start ? kv_start + s0 : nullptr;
        w.out[0] = static_cast<char*>(u.k_pool);
        w.out[1] = static_cast<char*>(u.v_pool);
        w.table = const_cast<int*>(u.page_table);
        w.cols = p.cols;
        void (*fn)(const Q8UnpackArgs) = d == 64 ? q8_unpack_kernel<64> : q8_unpack_kernel<128>;
        fn<<<dim3((unsigned)(p.cols * (128 / kQ8UnpackSlots)), (unsigned)n, 2), kQ8ReadThreads, 0, s>>>(w);
        LAR_CUDA(cudaGetLastError());
        lar_rows_t qr = {q->data, a.q.token_stride, a.q.head_stride}, orow = {out->data, a.out.token_stride, a.out.head_stride};
        int64_t tokens = n_tokens;
        if (!cu_tokens) {  // equal chunks: these sequences' tokens
            tokens = (int64_t)n * a.kv.chunk;
            qr.data = static_cast<char*>(qr.data) + (int64_t)s0 * a.kv.chunk * a.q.token_stride * elt;
            orow.data = static_cast<char*>(orow.data) + (int64_t)s0 * a.kv.chunk * a.out.token_stride * elt;
        }
        const lar_status_t st = lar_paged_attn(&u, &qr, &orow, n_q_heads, tokens, cu_tokens ? cu_tokens + s0 : nullptr, w.start, causal, softmax_scale,
                                               max_chunk, max_len, static_cast<char*>(workspace) + p.bytes, workspace_bytes - p.bytes, stream);
        if (st != LAR_OK) return st;
    }
    return LAR_OK;
}

}  // extern "C"
