// Host side of the paged entry points, as the cache's own entry points use them.
#pragma once
#include "../../include/lar.h"
#include "common.cuh"

namespace lar {

// Bookkeeping of the library's own cache that an append advances along with the rows (empty caches only: the prefill).
struct OwnCache {
    int* index_map;
    UnitState* state;
    int cap_pad;
};

lar_status_t paged_append(const lar_paged_kv_t& kv, const lar_rope_t* rope, const int32_t* pos, int64_t pos_axis_stride,
                          const lar_rows_t* k, const lar_rows_t* v, const lar_rows_t* q, const lar_rows_t* q_out, int n_q_heads,
                          int64_t n_tokens, const int32_t* cu_tokens, const OwnCache* own, void* stream);

}  // namespace lar
