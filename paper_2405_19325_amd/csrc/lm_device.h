// Device helpers of the calls over rows and a paged cache.
#pragma once

#include "knnlm_device.h"
#include "lm_internal.h"

namespace knnlm {

// A sequence's rows and keys.
struct Tile {
    int64_t r0;      // first row of the sequence
    int n;           // its rows
    int64_t length;  // cached tokens
    int64_t total;   // keys
};

// Of AttendArgs or WeighArgs; rows and keys past the hints are left out.
template <class Args>
__device__ __forceinline__ Tile tile_of(const Args &a, int64_t s) {
    Tile t;
    t.r0 = a.row_offsets[s];
    int64_t r1 = a.row_offsets[s + 1];
    if (r1 > a.rows) r1 = a.rows;
    const int64_t n = r1 - t.r0;
    t.n = static_cast<int>(n < 0 ? 0 : n > a.max_rows ? a.max_rows : n);
    const int64_t len = a.cache_lens[s];
    t.length = len < 0 ? 0 : len;
    t.total = t.length + t.n;
    if (t.total > a.max_keys) t.total = a.max_keys;
    const int64_t room = a.cache.table_width << a.cache.page_log2;
    if (t.total > room) t.total = room;
    return t;
}

// 16-byte chunk c of row r of a tile in LDS lies at chunk c ^ spread(r).  LDS
// has 64 banks, 16 chunks wide: the 16 rows x 1 chunk that 16 lanes of a
// product's operand read take at once, and the 8 rows x 2 neighbouring chunks
// of 32 lanes of a transposing read, then fall on 16 different ones.  (Rows of
// 8 chunks lie two in 16.)
template <int D>
__device__ __forceinline__ int spread(int r) {
    if constexpr (D == 64) return (((r >> 1) & 3) << 1) | ((r >> 3) & 1);
    return ((r & 7) << 1) | ((r >> 3) & 1);
}

// Where cache index c of sequence s and key head h lies: its place in [n_pages,
// kv_heads, page_size], or -1 where its page is none.  c is within the table.
__device__ __forceinline__ int64_t place_of(const PagedCache &cache, int kv_heads, int64_t s, int h, int64_t c) {
    const int64_t page = cache.pages[s * cache.table_width + (c >> cache.page_log2)];
    if (page < 0 || page >= cache.n_pages) return -1;
    return ((page * kv_heads + h) << cache.page_log2) + (c & ((int64_t{1} << cache.page_log2) - 1));
}

}  // namespace knnlm
