// Internal interfaces between the C ABI of the language model's own step
// (lm_api.hip) and its kernels: cache append, attention of drafts, sampling.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "knnlm.h"

namespace knnlm {

// A paged cache: [n_pages, kv_heads, page_size, head_dim], and the table
// [S, table_width] that names each sequence's pages.
struct PagedCache {
    const int32_t *pages;
    int64_t n_pages;
    int64_t table_width;
    int page_log2;  // page_size = 1 << page_log2
};

struct AppendArgs {
    const void *q, *k, *v;  // q may be null
    const int64_t *row_offsets;
    const int32_t *cache_lens;
    const int32_t *positions;    // or null: the cache index
    const float *inv_freq;       // or null: nothing is rotated (rot_dim 0)
    const int32_t *source_rows;  // or null: row t itself
    int64_t rows, source_count, S;
    int q_heads, kv_heads, head_dim, rot_dim;
    bool interleaved;
    int64_t q_row, q_head, k_row, k_head, v_row, v_head;  // strides in elements
    PagedCache cache;
    void *q_out, *k_cache, *v_cache;
};

hipError_t launch_kv_append(const AppendArgs &args, knn_dtype dtype, hipStream_t stream);

}  // namespace knnlm
