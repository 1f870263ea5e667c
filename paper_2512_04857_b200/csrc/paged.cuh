// Device view of a caller-described paged K/V cache (lar_paged_kv_t) and of a packed batch of token chunks, shared by the
// append and attention kernels: sequence s holds the tokens cu[s] .. cu[s + 1] - 1 (equal chunks without cu) and
// its cache lens[s] entries, the chunk's tokens being the newest.
#pragma once
#include "common.cuh"

namespace lar {

constexpr unsigned kStPage = 64u;  // a page number outside the pool, or a chunk that does not fit its sequence

struct PagedView {
    char* k_pool;
    char* v_pool;
    const int* table;
    const int* lens;
    unsigned* status;  // may be null
    long long page_stride, row_stride, head_stride;  // elements
    long long table_seq_stride, table_head_stride;   // table entries
    long long lens_stride;
    int n_seqs, n_kv_heads, n_pages, table_cols, page_tokens, page_shift;
    const int* cu;   // [n_seqs + 1], or null: every sequence has chunk tokens
    int chunk;
    int n_tokens;
    const int* row_of;  // row of the page table of each sequence, or null: its own number (groups of sequences with slots in common)
};

__device__ __forceinline__ void paged_report(const PagedView& v, unsigned bits) {
    if (v.status) atomicOr(v.status, bits);
}

// First and one-past-last token of a sequence, kept inside [0, n_tokens] whatever cu holds.
__device__ __forceinline__ void chunk_of(const PagedView& v, int s, int& t0, int& t1) {
    if (v.cu) {
        t0 = min(max(v.cu[s], 0), v.n_tokens);
        t1 = min(max(v.cu[s + 1], t0), v.n_tokens);
    } else {
        t0 = s * v.chunk;
        t1 = t0 + v.chunk;
    }
}

// Entries of the cache of a sequence with n tokens, kept inside what its table can address.  Tokens whose slots lie outside that (a length
// beyond the table, or of fewer entries than tokens) are recorded by the caller that says so.
__device__ __forceinline__ int live_len(const PagedView& v, int s, int n, bool report) {
    const int len = v.lens[s * v.lens_stride], cap = v.table_cols << v.page_shift;
    if (report && n > 0 && (len < n || len > cap)) paged_report(v, kStPage);
    return min(max(len, 0), cap);
}

}  // namespace lar
