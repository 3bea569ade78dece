// C ABI of the language model's own step around the mixture: cache append,
// attention of drafts, sampling.  Host-side validation and the launches on
// the caller's stream.
#include <math.h>
#include <stddef.h>
#include <stdint.h>

#include "knnlm.h"
#include "lm_internal.h"

namespace {

using namespace knnlm;

knn_status status_of(hipError_t e) { return e == hipSuccess ? KNN_OK : KNN_ERR_HIP; }

constexpr int64_t kMaxPage = 65536;

// The dtype and sizes of a paged cache; KNN_OK or the error.
knn_status check_cache(int64_t S, int64_t kv_heads, int64_t head_dim, int64_t n_pages, int64_t page_size,
                       int64_t table_width, knn_dtype dtype) {
    if (S < 1 || kv_heads < 1 || head_dim < 1 || n_pages < 1 || table_width < 1) return KNN_ERR_INVALID_ARG;
    if (dtype != KNN_F32 && dtype != KNN_BF16 && dtype != KNN_F16) return KNN_ERR_INVALID_ARG;
    if (page_size < 1 || (page_size & (page_size - 1)) != 0) return KNN_ERR_INVALID_ARG;
    if (dtype == KNN_F32 || page_size < 16 || page_size > kMaxPage || kv_heads > KNNLM_MAX_HEADS)
        return KNN_ERR_UNSUPPORTED;
    // every page starts at an element offset of fewer than 2^62
    if (n_pages > (int64_t{1} << 31) || S > 0x7fffffff || table_width > 0x7fffffff) return KNN_ERR_UNSUPPORTED;
    return KNN_OK;
}

PagedCache paged(const int32_t *pages, int64_t n_pages, int64_t page_size, int64_t table_width) {
    int log2 = 0;
    while ((int64_t{1} << log2) < page_size) ++log2;
    return PagedCache{pages, n_pages, table_width, log2};
}

}  // namespace

extern "C" {

knn_status knn_kv_append(const void *q, const void *k, const void *v, const int64_t *row_offsets,
                         const int32_t *cache_lens, const int32_t *pages, const int32_t *positions,
                         const float *inv_freq, const int32_t *source_rows, int64_t rows, int64_t source_count,
                         int64_t S, int64_t q_heads, int64_t kv_heads, int64_t head_dim, int64_t rot_dim,
                         int32_t interleaved, int64_t q_row_stride, int64_t q_head_stride, int64_t k_row_stride,
                         int64_t k_head_stride, int64_t v_row_stride, int64_t v_head_stride, int64_t n_pages,
                         int64_t page_size, int64_t table_width, knn_dtype dtype, void *q_out, void *k_cache,
                         void *v_cache, void *stream) {
    if (!k || !v || !row_offsets || !cache_lens || !pages || !k_cache || !v_cache) return KNN_ERR_INVALID_ARG;
    if ((q != nullptr) != (q_out != nullptr) || (q != nullptr) != (q_heads > 0) || q_heads < 0)
        return KNN_ERR_INVALID_ARG;
    if (rows < 1 || source_count < 1 || (source_rows == nullptr && source_count < rows)) return KNN_ERR_INVALID_ARG;
    const knn_status st = check_cache(S, kv_heads, head_dim, n_pages, page_size, table_width, dtype);
    if (st != KNN_OK) return st;
    if (rot_dim < 0 || rot_dim > head_dim || rot_dim % 2 != 0 || (inv_freq != nullptr) != (rot_dim > 0))
        return KNN_ERR_INVALID_ARG;
    if (q_row_stride < 0 || q_head_stride < 0 || k_row_stride < 0 || k_head_stride < 0 || v_row_stride < 0 ||
        v_head_stride < 0)
        return KNN_ERR_INVALID_ARG;
    if (head_dim > 1024 || q_heads > KNNLM_MAX_HEADS || rows > 0x7fffffff || source_count > 0x7fffffff)
        return KNN_ERR_UNSUPPORTED;
    AppendArgs a{};
    a.q = q, a.k = k, a.v = v;
    a.row_offsets = row_offsets, a.cache_lens = cache_lens, a.positions = positions;
    a.inv_freq = inv_freq, a.source_rows = source_rows;
    a.rows = rows, a.source_count = source_count, a.S = S;
    a.q_heads = static_cast<int>(q_heads), a.kv_heads = static_cast<int>(kv_heads);
    a.head_dim = static_cast<int>(head_dim), a.rot_dim = static_cast<int>(rot_dim);
    a.interleaved = interleaved != 0;
    a.q_row = q_row_stride, a.q_head = q_head_stride;
    a.k_row = k_row_stride, a.k_head = k_head_stride;
    a.v_row = v_row_stride, a.v_head = v_head_stride;
    a.cache = paged(pages, n_pages, page_size, table_width);
    a.q_out = q_out, a.k_cache = k_cache, a.v_cache = v_cache;
    return status_of(launch_kv_append(a, dtype, static_cast<hipStream_t>(stream)));
}

}  // extern "C"
