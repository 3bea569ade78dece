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

struct AttendArgs {
    const void *q;  // [rows, q_heads, head_dim], rows q_row elements apart, heads q_head
    const void *k_cache, *v_cache;
    const int64_t *row_offsets;
    const int32_t *cache_lens;
    const uint32_t *tree_mask;  // [rows, mask_words] or null: a chain
    int64_t rows, S;
    int q_heads, kv_heads, head_dim;
    int64_t q_row, q_head;
    PagedCache cache;
    int64_t mask_words;
    int64_t max_rows, max_keys;
    float scale;
    void *out;   // [rows, q_heads, head_dim]
    float *lse;  // [rows, q_heads] or null
    int64_t first_tile;  // of this launch, where there are several
};

// How an attention call is cut: column tiles of `cols` (row, query head) pairs
// of one key head, and one run of keys for each of `teams` teams of workgroups,
// a workgroup a column tile.  The keys of all sequences and heads lie one
// behind the other for that, so that every team gets as many, whatever the
// sequences' lengths; what a team has of a head that others have parts of is
// joined by a second launch.  Where the parts of all column tiles would take
// more than kAttendParts bytes, the tiles are worked off `tiles` at a time.
struct AttendPlan {
    int cols;
    int step;    // keys of the steps that runs are counted in; a head of one step is not parted
    int stages;  // few columns: stages of a wave
    int64_t all_tiles, tiles, teams;
    size_t off_ml, total;  // workspace: the parts, then (maximum, sum); two parts a workgroup, or 0
};
constexpr size_t kAttendParts = size_t{512} << 20;

AttendPlan plan_attend(int64_t rows, int64_t S, int64_t q_heads, int64_t kv_heads, int64_t head_dim, int64_t max_rows,
                       int64_t max_keys);
hipError_t launch_attend(const AttendArgs &args, const AttendPlan &plan, knn_dtype dtype, void *workspace,
                         hipStream_t stream);

struct SampleArgs {
    const void *scores;  // [rows, V], rows `stride` elements apart
    const float *uniforms;
    const float *temperature;  // each [rows], or null: 1, 0, 1, 0
    const int32_t *top_k;
    const float *top_p, *min_p;
    int64_t rows;
    int V;
    int64_t stride;
    bool probabilities;
    int32_t *token;
    float *prob;    // or null
    int32_t *kept;  // or null
};

constexpr int64_t kSampleMaxV = int64_t{1} << 24;

hipError_t launch_sample(const SampleArgs &args, knn_dtype dtype, void *workspace, hipStream_t stream);

hipError_t launch_kv_append(const AppendArgs &args, knn_dtype dtype, hipStream_t stream);

}  // namespace knnlm
