// C ABI of the language model's own step around the mixture: cache append,
// attention of drafts, weights of cached keys, eviction, adjusted scores,
// sampling.  Host-side validation and the launches on the caller's stream.
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
    // (every offset in bytes fits 64 bits)
    if (n_pages > (int64_t{1} << 31) || S > 0x7fffffff || table_width > 0x7fffffff ||
        static_cast<double>(n_pages) * kv_heads * page_size * head_dim > 4611686018427387904.0)  // 2^62
        return KNN_ERR_UNSUPPORTED;
    return KNN_OK;
}

PagedCache paged(const int32_t *pages, int64_t n_pages, int64_t page_size, int64_t table_width) {
    int log2 = 0;
    while ((int64_t{1} << log2) < page_size) ++log2;
    return PagedCache{pages, n_pages, table_width, log2};
}

// Whether an attention call's sizes are served; KNN_OK or the error.
knn_status check_attend(int64_t rows, int64_t S, int64_t q_heads, int64_t kv_heads, int64_t head_dim, int64_t max_rows,
                        int64_t max_keys) {
    if (rows < 1 || S < 1 || q_heads < 1 || kv_heads < 1 || q_heads % kv_heads != 0) return KNN_ERR_INVALID_ARG;
    if (max_rows < 1 || max_rows > rows || max_keys < 1) return KNN_ERR_INVALID_ARG;
    if (head_dim != 64 && head_dim != 128 && head_dim != 256) return KNN_ERR_UNSUPPORTED;
    // (the kernels count the steps of 64 keys of 64 sequences in 32 bits)
    if (rows > 0x7fffffff || max_rows > 65535 || max_keys > 0x7fffffff || q_heads > KNNLM_MAX_HEADS || S > 0x7fffffff)
        return KNN_ERR_UNSUPPORTED;
    return KNN_OK;
}

knn_status check_sample(int64_t rows, int64_t V, knn_dtype dtype) {
    if (rows < 1 || V < 1 || (dtype != KNN_F32 && dtype != KNN_BF16 && dtype != KNN_F16)) return KNN_ERR_INVALID_ARG;
    return rows > 0x7fffffff || V > kSampleMaxV ? KNN_ERR_UNSUPPORTED : KNN_OK;
}

knn_status check_evict(int64_t S, int64_t kv_heads, int64_t max_keys) {
    if (S < 1 || kv_heads < 1 || max_keys < 1) return KNN_ERR_INVALID_ARG;
    // (heads are counted in 31 bits, and a workspace of up to 12 bytes a token fits 64)
    if (kv_heads > KNNLM_MAX_HEADS || S > 0x7fffffff / kv_heads || max_keys > 0x7fffffff ||
        static_cast<double>(S) * kv_heads * max_keys > 72057594037927936.0)  // 2^56
        return KNN_ERR_UNSUPPORTED;
    return KNN_OK;
}

constexpr int64_t kAdjustMaxWidth = int64_t{1} << 28;  // (occurrences are counted in 30 bits)
constexpr int64_t kMaxMaskWords = int64_t{1} << 28;    // (weights find a mask's words in 32 bits)

// The bytes from the first to the last of a buffer (null: none), in doubles: no sum of strides can pass them.
struct Extent {
    const void *at;
    double bytes;
};

// Of [rows, heads, head_dim] 16-bit elements with these strides; of n elements of `size` bytes.
Extent strided(const void *at, int64_t rows, int64_t heads, int64_t head_dim, int64_t row, int64_t head) {
    return Extent{at, 2.0 * (static_cast<double>(rows - 1) * row + static_cast<double>(heads - 1) * head + head_dim)};
}
Extent dense(const void *at, double n, int size) { return Extent{at, n * size}; }

bool meet(const Extent &a, const Extent &b) {
    if (a.at == nullptr || b.at == nullptr) return false;
    const double apart = static_cast<double>(reinterpret_cast<uintptr_t>(b.at)) -
                         static_cast<double>(reinterpret_cast<uintptr_t>(a.at));
    return apart < a.bytes && -apart < b.bytes;
}

// Whether an output lies on an input or on another output.
template <size_t N, size_t M>
bool any_meet(const Extent (&outputs)[N], const Extent (&inputs)[M]) {
    for (size_t i = 0; i < N; ++i) {
        for (const Extent &in : inputs)
            if (meet(outputs[i], in)) return true;
        for (size_t j = 0; j < i; ++j)
            if (meet(outputs[i], outputs[j])) return true;
    }
    return false;
}

bool aligned(const void *p, size_t to) { return reinterpret_cast<uintptr_t>(p) % to == 0; }

}  // namespace

extern "C" {

size_t knn_tree_attention_workspace_size(int64_t rows, int64_t S, int64_t q_heads, int64_t kv_heads, int64_t head_dim,
                                         int64_t max_rows, int64_t max_keys) {
    if (check_attend(rows, S, q_heads, kv_heads, head_dim, max_rows, max_keys) != KNN_OK) return 0;
    const size_t need = plan_attend(rows, S, q_heads, kv_heads, head_dim, max_rows, max_keys).total;
    return need < 256 ? 256 : (need + 255) / 256 * 256;
}

knn_status knn_tree_attention(const void *q, const void *k_cache, const void *v_cache, const int32_t *pages,
                              const int64_t *row_offsets, const int32_t *cache_lens, const uint32_t *tree_mask,
                              int64_t rows, int64_t S, int64_t q_heads, int64_t kv_heads, int64_t head_dim,
                              int64_t q_row_stride, int64_t q_head_stride, int64_t n_pages, int64_t page_size,
                              int64_t table_width, int64_t mask_words, int64_t max_rows, int64_t max_keys,
                              knn_dtype dtype, float scale, void *out, float *lse, void *workspace,
                              size_t workspace_bytes, void *stream) {
    if (!q || !k_cache || !v_cache || !pages || !row_offsets || !cache_lens || !out) return KNN_ERR_INVALID_ARG;
    knn_status st = check_cache(S, kv_heads, head_dim, n_pages, page_size, table_width, dtype);
    if (st != KNN_OK) return st;
    st = check_attend(rows, S, q_heads, kv_heads, head_dim, max_rows, max_keys);
    if (st != KNN_OK) return st;
    if (max_keys > table_width * page_size || !isfinite(scale) || q_row_stride < 0 || q_head_stride < 0)
        return KNN_ERR_INVALID_ARG;
    if (tree_mask != nullptr && mask_words < (max_rows + 31) / 32) return KNN_ERR_INVALID_ARG;
    // (the stride of a single row or head says nothing)
    if (((rows > 1 ? q_row_stride : 0) | (q_heads > 1 ? q_head_stride : 0)) % 8 != 0 ||
        !aligned(q, 16) || !aligned(k_cache, 16) || !aligned(v_cache, 16) || !aligned(out, 16))
        return KNN_ERR_UNSUPPORTED;
    const size_t need =
        knn_tree_attention_workspace_size(rows, S, q_heads, kv_heads, head_dim, max_rows, max_keys);
    if (!workspace || !aligned(workspace, 256) || workspace_bytes < need) return KNN_ERR_WORKSPACE;
    const double cells = static_cast<double>(n_pages) * kv_heads * page_size * head_dim;
    const Extent outputs[] = {dense(out, static_cast<double>(rows) * q_heads * head_dim, 2),
                              dense(lse, static_cast<double>(rows) * q_heads, 4),
                              dense(workspace, static_cast<double>(need), 1)};
    const Extent inputs[] = {strided(q, rows, q_heads, head_dim, q_row_stride, q_head_stride),
                             dense(k_cache, cells, 2),
                             dense(v_cache, cells, 2),
                             dense(pages, static_cast<double>(S) * table_width, 4),
                             dense(row_offsets, static_cast<double>(S) + 1, 8),
                             dense(cache_lens, static_cast<double>(S), 4),
                             dense(tree_mask, static_cast<double>(rows) * mask_words, 4)};
    if (any_meet(outputs, inputs)) return KNN_ERR_INVALID_ARG;
    AttendArgs a{};
    a.q = q, a.k_cache = k_cache, a.v_cache = v_cache;
    a.row_offsets = row_offsets, a.cache_lens = cache_lens, a.tree_mask = tree_mask;
    a.rows = rows, a.S = S;
    a.q_heads = static_cast<int>(q_heads), a.kv_heads = static_cast<int>(kv_heads);
    a.head_dim = static_cast<int>(head_dim);
    a.q_row = q_row_stride, a.q_head = q_head_stride;
    a.cache = paged(pages, n_pages, page_size, table_width);
    a.mask_words = mask_words, a.max_rows = max_rows, a.max_keys = max_keys;
    a.scale = scale;
    a.out = out, a.lse = lse;
    return status_of(launch_attend(a, plan_attend(rows, S, q_heads, kv_heads, head_dim, max_rows, max_keys), dtype,
                                   workspace, static_cast<hipStream_t>(stream)));
}

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
    // (the stride of a single row or head says nothing)
    const bool in_place = q == q_out && source_rows == nullptr && (q_heads == 1 || q_head_stride == head_dim) &&
                          (rows == 1 || q_row_stride == q_heads * head_dim);
    // (The two caches may be one: what is written to them is the caller's.)
    const double cells = static_cast<double>(n_pages) * kv_heads * page_size * head_dim;
    const Extent caches[] = {dense(k_cache, cells, 2), dense(v_cache, cells, 2)};
    const Extent turned[] = {dense(q_out, static_cast<double>(rows) * q_heads * head_dim, 2)};
    const Extent queries = strided(q, source_count, q_heads, head_dim, q_row_stride, q_head_stride);
    const Extent inputs[] = {strided(k, source_count, kv_heads, head_dim, k_row_stride, k_head_stride),
                             strided(v, source_count, kv_heads, head_dim, v_row_stride, v_head_stride),
                             dense(pages, static_cast<double>(S) * table_width, 4),
                             dense(row_offsets, static_cast<double>(S) + 1, 8),
                             dense(cache_lens, static_cast<double>(S), 4),
                             dense(positions, static_cast<double>(rows), 4),
                             dense(inv_freq, static_cast<double>(rot_dim) / 2, 4),
                             dense(source_rows, static_cast<double>(rows), 4)};
    if ((!in_place && meet(turned[0], queries)) || any_meet(turned, inputs) || any_meet(turned, caches))
        return KNN_ERR_INVALID_ARG;
    for (const Extent &c : caches) {
        if (meet(c, queries)) return KNN_ERR_INVALID_ARG;
        for (const Extent &in : inputs)
            if (meet(c, in)) return KNN_ERR_INVALID_ARG;
    }
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

size_t knn_sample_workspace_size(int64_t rows, int64_t V, knn_dtype dtype) {
    return check_sample(rows, V, dtype) == KNN_OK ? 256 : 0;
}

knn_status knn_sample(const void *scores, const float *uniforms, const float *temperature, const int32_t *top_k,
                      const float *top_p, const float *min_p, int64_t rows, int64_t V, int64_t row_stride,
                      int32_t probabilities, knn_dtype dtype, int32_t *token, float *prob, int32_t *kept,
                      void *workspace, size_t workspace_bytes, void *stream) {
    if (!scores || !uniforms || !token) return KNN_ERR_INVALID_ARG;
    const knn_status st = check_sample(rows, V, dtype);
    if (st != KNN_OK) return st;
    if (row_stride < 0) return KNN_ERR_INVALID_ARG;
    if (!aligned(scores, dtype == KNN_F32 ? 4 : 2)) return KNN_ERR_UNSUPPORTED;
    if (!workspace || !aligned(workspace, 256) || workspace_bytes < knn_sample_workspace_size(rows, V, dtype))
        return KNN_ERR_WORKSPACE;
    const double elements = static_cast<double>(rows - 1) * row_stride + V;
    const Extent outputs[] = {dense(token, static_cast<double>(rows), 4), dense(prob, static_cast<double>(rows), 4),
                              dense(kept, static_cast<double>(rows), 4)};
    const Extent inputs[] = {dense(scores, elements, dtype == KNN_F32 ? 4 : 2)};
    if (any_meet(outputs, inputs)) return KNN_ERR_INVALID_ARG;
    SampleArgs a{};
    a.scores = scores, a.uniforms = uniforms;
    a.temperature = temperature, a.top_k = top_k, a.top_p = top_p, a.min_p = min_p;
    a.rows = rows, a.V = static_cast<int>(V), a.stride = row_stride;
    a.probabilities = probabilities != 0;
    a.token = token, a.prob = prob, a.kept = kept;
    return status_of(launch_sample(a, dtype, workspace, static_cast<hipStream_t>(stream)));
}

knn_status knn_key_weights(const void *q, const float *lse, const void *k_cache, const int32_t *pages,
                           const int64_t *row_offsets, const int32_t *cache_lens, const int32_t *positions,
                           const int32_t *source_rows, const uint32_t *tree_mask, int64_t rows, int64_t source_count,
                           int64_t S, int64_t q_heads, int64_t kv_heads, int64_t head_dim, int64_t q_row_stride,
                           int64_t q_head_stride, int64_t n_pages, int64_t page_size, int64_t table_width,
                           int64_t mask_words, int64_t max_rows, int64_t max_keys, knn_dtype dtype, float scale,
                           float decay, float *mass, int32_t *key_positions, void *stream) {
    if (!q || !lse || !k_cache || !pages || !row_offsets || !cache_lens || !mass) return KNN_ERR_INVALID_ARG;
    if (positions != nullptr && key_positions == nullptr) return KNN_ERR_INVALID_ARG;
    if (source_count < 1 || (source_rows == nullptr && source_count < rows)) return KNN_ERR_INVALID_ARG;
    knn_status st = check_cache(S, kv_heads, head_dim, n_pages, page_size, table_width, dtype);
    if (st != KNN_OK) return st;
    st = check_attend(rows, S, q_heads, kv_heads, head_dim, max_rows, max_keys);
    if (st != KNN_OK) return st;
    if (max_keys > table_width * page_size || !isfinite(scale) || !isfinite(decay) || decay < 0.0f ||
        q_row_stride < 0 || q_head_stride < 0)
        return KNN_ERR_INVALID_ARG;
    if (tree_mask != nullptr && mask_words < (max_rows + 31) / 32) return KNN_ERR_INVALID_ARG;
    // (the stride of a single row or head says nothing)
    if (((source_count > 1 ? q_row_stride : 0) | (q_heads > 1 ? q_head_stride : 0)) % 8 != 0 || !aligned(q, 16) ||
        !aligned(k_cache, 16) || source_count > 0x7fffffff || (tree_mask != nullptr && mask_words > kMaxMaskWords))
        return KNN_ERR_UNSUPPORTED;
    const double places = static_cast<double>(n_pages) * kv_heads * page_size;
    const Extent outputs[] = {dense(mass, places, 4), dense(key_positions, places, 4)};
    const Extent inputs[] = {strided(q, source_count, q_heads, head_dim, q_row_stride, q_head_stride),
                             dense(lse, static_cast<double>(source_count) * q_heads, 4),
                             dense(k_cache, places * head_dim, 2),
                             dense(pages, static_cast<double>(S) * table_width, 4),
                             dense(row_offsets, static_cast<double>(S) + 1, 8),
                             dense(cache_lens, static_cast<double>(S), 4),
                             dense(positions, static_cast<double>(rows), 4),
                             dense(source_rows, static_cast<double>(rows), 4),
                             dense(tree_mask, static_cast<double>(rows) * mask_words, 4)};
    if (any_meet(outputs, inputs)) return KNN_ERR_INVALID_ARG;
    WeighArgs a{};
    a.q = q, a.lse = lse, a.k_cache = k_cache;
    a.row_offsets = row_offsets, a.cache_lens = cache_lens, a.positions = positions;
    a.source_rows = source_rows, a.tree_mask = tree_mask;
    a.rows = rows, a.source_count = source_count, a.S = S;
    a.q_heads = static_cast<int>(q_heads), a.kv_heads = static_cast<int>(kv_heads);
    a.head_dim = static_cast<int>(head_dim);
    a.q_row = q_row_stride, a.q_head = q_head_stride;
    a.cache = paged(pages, n_pages, page_size, table_width);
    a.mask_words = mask_words, a.max_rows = max_rows, a.max_keys = max_keys;
    a.scale = scale, a.decay = decay;
    a.mass = mass, a.key_positions = key_positions;
    return status_of(launch_key_weights(a, dtype, static_cast<hipStream_t>(stream)));
}

size_t knn_cache_evict_workspace_size(int64_t S, int64_t kv_heads, int64_t max_keys) {
    if (check_evict(S, kv_heads, max_keys) != KNN_OK) return 0;
    const size_t need = evict_workspace(S, kv_heads, max_keys);
    return need < 256 ? 256 : (need + 255) / 256 * 256;
}

knn_status knn_cache_evict(void *k_cache, void *v_cache, float *mass, int32_t *key_positions, const int32_t *pages,
                           const int32_t *cache_lens, const int32_t *budgets, const int32_t *next_positions, int64_t S,
                           int64_t kv_heads, int64_t head_dim, int64_t n_pages, int64_t page_size, int64_t table_width,
                           int64_t max_keys, int32_t sinks, int32_t recent, knn_dtype dtype, float *mass_out,
                           int32_t *positions_out, int32_t *new_lens, void *workspace, size_t workspace_bytes,
                           void *stream) {
    if (!k_cache || !v_cache || !mass || !pages || !cache_lens || !budgets || !mass_out || !new_lens ||
        (key_positions != nullptr) != (positions_out != nullptr))
        return KNN_ERR_INVALID_ARG;
    knn_status st = check_cache(S, kv_heads, head_dim, n_pages, page_size, table_width, dtype);
    if (st != KNN_OK) return st;
    st = check_evict(S, kv_heads, max_keys);
    if (st != KNN_OK) return st;
    if (max_keys > table_width * page_size || sinks < 0 || recent < 0) return KNN_ERR_INVALID_ARG;
    if (head_dim > 1024) return KNN_ERR_UNSUPPORTED;
    const size_t need = knn_cache_evict_workspace_size(S, kv_heads, max_keys);
    if (!workspace || !aligned(workspace, 256) || workspace_bytes < need) return KNN_ERR_WORKSPACE;
    const double places = static_cast<double>(n_pages) * kv_heads * page_size;
    // (A ledger that is written in place is no input beside itself.)
    const bool same_mass = mass_out == mass, same_positions = positions_out == key_positions;
    const Extent outputs[] = {dense(k_cache, places * head_dim, 2),
                              dense(v_cache, places * head_dim, 2),
                              dense(mass_out, places, 4),
                              dense(positions_out, places, 4),
                              dense(new_lens, static_cast<double>(S), 4),
                              dense(workspace, static_cast<double>(need), 1)};
    const Extent inputs[] = {dense(same_mass ? nullptr : mass, places, 4),
                             dense(same_positions ? nullptr : key_positions, places, 4),
                             dense(pages, static_cast<double>(S) * table_width, 4),
                             dense(cache_lens, static_cast<double>(S), 4),
                             dense(budgets, static_cast<double>(S), 4),
                             dense(next_positions, static_cast<double>(S), 4)};
    if (any_meet(outputs, inputs)) return KNN_ERR_INVALID_ARG;
    EvictArgs a{};
    a.k_cache = k_cache, a.v_cache = v_cache;
    a.mass = mass, a.key_positions = key_positions;
    a.cache_lens = cache_lens, a.budgets = budgets, a.next_positions = next_positions;
    a.S = S, a.kv_heads = static_cast<int>(kv_heads), a.head_dim = static_cast<int>(head_dim);
    a.cache = paged(pages, n_pages, page_size, table_width);
    a.max_keys = max_keys;
    a.sinks = sinks, a.recent = recent;
    a.mass_out = mass_out, a.positions_out = positions_out, a.new_lens = new_lens;
    return status_of(launch_cache_evict(a, workspace, static_cast<hipStream_t>(stream)));
}

knn_status knn_adjust_scores(const void *scores, const int32_t *history, const int32_t *history_lens,
                             const int32_t *prompt_lens, const int64_t *row_offsets, const int32_t *row_tokens,
                             const uint32_t *tree_mask, const float *repetition, const float *presence,
                             const float *frequency, const int32_t *bias_tokens, const float *bias_values,
                             const uint32_t *allowed, int64_t rows, int64_t V, int64_t S, int64_t row_stride,
                             int64_t history_width, int64_t mask_words, int64_t bias_width, int64_t out_stride,
                             int32_t probabilities, knn_dtype dtype, void *out, void *stream) {
    if (!scores || !out) return KNN_ERR_INVALID_ARG;
    const knn_status st = check_sample(rows, V, dtype);
    if (st != KNN_OK) return st;
    if (S < 1 || (row_offsets == nullptr && S != rows) || row_stride < 0 || (rows > 1 && out_stride < V))
        return KNN_ERR_INVALID_ARG;
    if ((history != nullptr) != (history_lens != nullptr) || (history != nullptr && history_width < 1) ||
        (prompt_lens != nullptr && history == nullptr))
        return KNN_ERR_INVALID_ARG;
    if (tree_mask != nullptr && (row_tokens == nullptr || mask_words < 1)) return KNN_ERR_INVALID_ARG;
    if ((repetition != nullptr || presence != nullptr || frequency != nullptr) && history == nullptr &&
        row_tokens == nullptr)
        return KNN_ERR_INVALID_ARG;
    if ((bias_tokens != nullptr) != (bias_values != nullptr) || (bias_tokens != nullptr && bias_width < 1))
        return KNN_ERR_INVALID_ARG;
    const int size = dtype == KNN_F32 ? 4 : 2;
    const int64_t most = kAdjustMaxWidth;
    if (S > 0x7fffffff || (history != nullptr && history_width > most) || (bias_tokens != nullptr && bias_width > most) ||
        (row_tokens != nullptr && rows > most) || (tree_mask != nullptr && mask_words > kMaxMaskWords) ||
        !aligned(scores, size) || !aligned(out, size))
        return KNN_ERR_UNSUPPORTED;
    const bool in_place = out == scores && (rows == 1 || out_stride == row_stride);
    const Extent outputs[] = {dense(out, static_cast<double>(rows - 1) * out_stride + V, size)};
    const double words = static_cast<double>((V + 31) / 32);
    const Extent inputs[] = {
        dense(in_place ? nullptr : scores, static_cast<double>(rows - 1) * row_stride + V, size),
        dense(history, static_cast<double>(S) * history_width, 4),
        dense(history_lens, static_cast<double>(S), 4),
        dense(prompt_lens, static_cast<double>(S), 4),
        dense(row_offsets, static_cast<double>(S) + 1, 8),
        dense(row_tokens, static_cast<double>(rows), 4),
        dense(tree_mask, static_cast<double>(rows) * mask_words, 4),
        dense(repetition, static_cast<double>(rows), 4),
        dense(presence, static_cast<double>(rows), 4),
        dense(frequency, static_cast<double>(rows), 4),
        dense(bias_tokens, static_cast<double>(S) * bias_width, 4),
        dense(bias_values, static_cast<double>(S) * bias_width, 4),
        dense(allowed, static_cast<double>(rows) * words, 4)};
    if (any_meet(outputs, inputs)) return KNN_ERR_INVALID_ARG;
    AdjustArgs a{};
    a.scores = scores, a.out = out;
    a.history = history, a.history_lens = history_lens, a.prompt_lens = prompt_lens;
    a.row_offsets = row_offsets, a.row_tokens = row_tokens, a.tree_mask = tree_mask;
    a.repetition = repetition, a.presence = presence, a.frequency = frequency;
    a.bias_tokens = bias_tokens, a.bias_values = bias_values, a.allowed = allowed;
    a.rows = rows, a.S = S, a.V = static_cast<int>(V);
    a.stride = row_stride, a.out_stride = out_stride;
    a.history_width = history_width, a.mask_words = mask_words, a.bias_width = bias_width;
    a.probabilities = probabilities != 0;
    return status_of(launch_adjust_scores(a, dtype, static_cast<hipStream_t>(stream)));
}

}  // extern "C"
