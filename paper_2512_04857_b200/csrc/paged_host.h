// Host side of the paged entry points, shared by their translation units and by the cache's own entry points.
#pragma once
#include "../../include/lar.h"
#include "common.cuh"
#include "paged.cuh"
#include "rope_rows.cuh"

namespace lar {

constexpr int kSms = 148;             // SMs of a B200 (launch shapes only)
constexpr int64_t kMaxTokens = 1 << 26;
constexpr int kMaxHeads = 4096;       // (the rotary kernels divide row numbers by multiplication: rows of two tokens x rows of one < 2^32)

inline int elt_of(int dtype) { return dtype == LAR_BF16 ? 2 : 4; }
inline bool is_dtype(int dtype) { return dtype == LAR_BF16 || dtype == LAR_FP32; }
inline bool aligned(const void* p, size_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }

// Argument checks: false for what the header does not allow.
bool rope_freqs(const lar_rope_t* r, int inverse, RopeFreqs& f);
bool rows_view(const lar_rows_t* r, int64_t tokens, int heads, int d, int elt, bool output, RowsView& v);
bool paged_view(const lar_paged_kv_t* k, int64_t n_tokens, const int32_t* cu, PagedView& v, bool q8 = false);
// What lar_paged_attn with these (checked) arguments would be refused for: LAR_ERR_CAPACITY, LAR_ERR_NOMEM, or LAR_OK.
lar_status_t paged_attn_fits(const lar_paged_kv_t& kv, int group, int64_t n_tokens, int max_chunk, int max_len, bool workspace, size_t workspace_bytes);
struct Q8View;
bool q8_view(const lar_paged_q8_t* c, int64_t n_tokens, const int32_t* cu, PagedView& v, Q8View& q);

// Bookkeeping of the library's own cache that an append advances along with the rows (empty caches only: the prefill).
struct OwnCache {
    int* index_map;
    UnitState* state;
    int cap_pad;
};

lar_status_t paged_append(const lar_paged_kv_t& kv, const lar_rope_t* rope, const int32_t* pos, int64_t pos_axis_stride,
                          const lar_rows_t* k, const lar_rows_t* v, const lar_rows_t* q, const lar_rows_t* q_out, int n_q_heads,
                          int64_t n_tokens, const int32_t* cu_tokens, const OwnCache* own, void* stream);
// The same with norms of q and k (null: none) on the way.
lar_status_t paged_append_norm(const lar_paged_kv_t& kv, const lar_head_norm_t* q_norm, const lar_head_norm_t* k_norm, const lar_rope_t* rope,
                               const int32_t* pos, int64_t pos_axis_stride, const lar_rows_t* k, const lar_rows_t* v, const lar_rows_t* q,
                               const lar_rows_t* q_out, int n_q_heads, int64_t n_tokens, const int32_t* cu_tokens, const OwnCache* own,
                               void* stream);

}  // namespace lar
