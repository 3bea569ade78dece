// Attention of the rows of drafts over a paged cache.
//
// Row i of a sequence with L cached tokens sees the keys j < L and, of the
// drafts' keys L + j, those that its mask names (a chain: j <= i).  Per query
// head, with x_j = scale q.k_j over the keys seen,
//   out = sum_j exp(x_j - m) v_j / sum_j exp(x_j - m),   lse = m + log(sum).
// One pass over the keys: a running reference m, and sums relative to it that
// are scaled when it moves.  m need not be the maximum: it follows the maximum
// only when that rises by more than 2^kSlack over it, so the weights stay
// under 2^kSlack, far inside the range of either type, and most tiles neither
// reduce a maximum over lanes nor scale anything.
//
// All query heads of a key head and all rows of a sequence read the same keys,
// so they are the columns of one matrix product: S^T = K Q^T with 16 keys x 16
// columns per matrix instruction.  A lane then holds 4 consecutive keys of one
// column, which is what the second product O^T = V^T P^T wants of its right
// operand, in an order of the keys that the left operand follows: the weights
// never leave the registers.  V^T comes out of LDS by the transposing read.
// The matrix instruction takes both operands in one type, so the weights are
// rounded to 16 bits for it: errors of 0.0023 of the largest output in bf16 and
// 0.00029 in f16, 0.0017 and 0.00021 of these the output's own rounding.  (A product
// of what the rounding leaves would be half as many matrix instructions again.)
// The row of ones in front of V sums the weights as they were rounded, in 32 bits,
// so that they sum to one.
//
// What bounds it.  Up to 16 columns a key head (decoding, spans without shared
// heads): the bytes of the keys, each of which is read once.  64 ragged
// sequences of 2,000 to 16,000 tokens, 8 key heads: 408 us for 2.36 GB, 5.8 TB/s
// with the join (a plain read: 7.0).  64 and more columns: the issue of a
// weight's vector instructions beside its two matrix products, at 128 columns
// of head_dim 128 with nearly a full register file (239 of 256).  Trees
// of 64 rows on 4 x 131,072 tokens, 64 query heads on 8: 1.28 ms, 857 TFLOP/s
// (a large library product: 1,166).  One token on 1,000 keys: 13.9 us, of which
// 5.2 are the join's launch, and 8.7 two waits for memory, the barriers and the
// launch of the first.
#include "lm_internal.h"
#include "mfma_device.h"

namespace knnlm {

namespace {

constexpr float kFloor = -3.0e38f;  // reference before the first key
constexpr float kSlack = 8.0f;
constexpr float kBelow = 7.0f;
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;
constexpr int64_t kWhole = 256;   // keys of a head that is not parted
constexpr int64_t kWide = 16384;  // workgroups of a wide call

typedef uint32_t u32x2_t __attribute__((ext_vector_type(2)));
typedef short s16x4_t __attribute__((ext_vector_type(4)));

// What a workgroup works on.
struct Tile {
    int64_t r0;      // first row of the sequence
    int n;           // its rows
    int64_t length;  // cached tokens
    int64_t total;   // keys
};

__device__ __forceinline__ Tile tile_of(const AttendArgs &a, int64_t s) {
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

template <knn_dtype DT>
__device__ __forceinline__ uint32_t pack2(float a, float b) {  // to nearest, ties to even
    if constexpr (DT == KNN_BF16) {
        const bf16x2_t v = {static_cast<__bf16>(a), static_cast<__bf16>(b)};
        return __builtin_bit_cast(uint32_t, v);
    } else {
        const f16x2_t v = {static_cast<_Float16>(a), static_cast<_Float16>(b)};
        return __builtin_bit_cast(uint32_t, v);
    }
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

// Four 16-bit elements of one column: lane l of each 16 gets column l of the 4
// rows whose 8-byte pieces the 16 lanes point at.
__device__ __forceinline__ u32x2_t read_transposed(uint32_t lds) {
    const s16x4_t v = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
        reinterpret_cast<__attribute__((address_space(3))) s16x4_t *>(static_cast<uintptr_t>(lds)));
    return __builtin_bit_cast(u32x2_t, v);
}

// The 16-bit elements of w that are infinite or NaN: as a word with 0xffff there.
template <knn_dtype DT>
__device__ __forceinline__ uint32_t not_finite(uint32_t w) {
    constexpr uint32_t kExp = DT == KNN_BF16 ? 0x7f80u : 0x7c00u;
    return ((w & kExp) == kExp ? 0xffffu : 0u) | (((w >> 16) & kExp) == kExp ? 0xffff0000u : 0u);
}

// Which of the four keys from `at` on a row sees, as bits, whether or not they
// have pages: those before `limit`, of these the cached ones and the drafts.
__device__ __forceinline__ uint32_t first_bits(int64_t n) { return n <= 0 ? 0u : n >= 4 ? 15u : (1u << n) - 1u; }
__device__ __forceinline__ uint32_t seen(const AttendArgs &a, const Tile &t, int row, int64_t at, int64_t limit) {
    const int64_t draft = at - t.length;  // of the first key
    if (a.tree_mask == nullptr) {
        const int64_t own = t.length + row + 1;
        return first_bits((own < limit ? own : limit) - at);
    }
    // Four bits of the row's mask from `draft` on (or from draft 0 on, moved up by the cached keys before it); they may
    // lie in two words.  Words past the last are read as the last and count as none.
    const uint32_t *words = a.tree_mask + (t.r0 + row) * a.mask_words;
    const int64_t from = draft < 0 ? 0 : draft, w0 = from >> 5, w1 = (from + 3) >> 5, last = a.mask_words - 1;
    const uint32_t lo = words[w0 < last ? w0 : last], hi = words[w1 < last ? w1 : last];
    const uint64_t both = (w0 <= last ? lo : 0u) | static_cast<uint64_t>(w1 <= last ? hi : 0u) << 32;
    uint32_t bits = w0 == w1 ? static_cast<uint32_t>(both) >> (from & 31) : static_cast<uint32_t>(both >> (from & 31));
    bits = draft <= -4 ? 0u : bits << (from - draft);
    return (first_bits(-draft) | bits) & first_bits(limit - at);
}

// From q.k (with the scale's sign) to the exponent of two.
__device__ __forceinline__ float c2_of(const AttendArgs &a) { return a.scale == 0.0f ? 1.0f : fabsf(a.scale) * kLog2e; }

// The keys of a span, counted from its first one, k0 (a multiple
// of 64): where they lie, and how many rows there are to read.
template <int D>
struct Keys {
    const int32_t *table;  // of k0's page
    int page_log2, slot0;  // slot0: k0's in its page
    int64_t n_pages, head_bytes, page_bytes;
    int last;  // the last key

    __device__ __forceinline__ Keys(const AttendArgs &a, int64_t s, int h, int64_t k0, int64_t end)
        : table(a.cache.pages + s * a.cache.table_width + (k0 >> a.cache.page_log2)), page_log2(a.cache.page_log2),
          slot0(static_cast<int>(k0 & ((int64_t{1} << a.cache.page_log2) - 1))), n_pages(a.cache.n_pages),
          head_bytes(static_cast<int64_t>(h) * 2 * D << a.cache.page_log2),
          page_bytes(static_cast<int64_t>(a.kv_heads) * 2 * D << a.cache.page_log2), last(static_cast<int>(end - 1 - k0)) {}
    // The page of a key (keys past the last one are read as the last one; 32 tiles ahead they may pass 2^31).
    __device__ __forceinline__ int32_t entry(int64_t key) const {
        return table[(slot0 + (key < last ? static_cast<int>(key) : last)) >> page_log2];
    }
    __device__ __forceinline__ bool real(int32_t page) const { return page >= 0 && page < n_pages; }
    // Byte offset of 16 keys from `key` on in either cache; `rows`: the last of them that there is.
    __device__ __forceinline__ int64_t at(int key, int32_t page, int &rows) const {
        if (!real(page)) page = 0;
        key = key > last ? last & ~15 : key;
        rows = min(last - key, 15);
        return page * page_bytes + head_bytes + ((slot0 + key) & ((1 << page_log2) - 1)) * (2 * D);
    }
};

// The columns of a wave: NT x 16 (row, query head) pairs of one key head.
template <knn_dtype DT, int D, int NT>
struct Columns {
    static constexpr int KK = D / 32, DB = D / 16, ROW = 2 * D;
    u32x4_t q[NT][KK];  // right operand of the scores: lane = (column, 8 elements a quad)
    f32x4_t o[NT][DB];  // lane = (column, 4 elements a quad)
    f32x4_t sum[NT];    // the same sum four times
    float m[NT];        // reference: of q.k, whatever the scale, so that keys of one score weigh the same however large it is
    int row_of[NT];     // row within the sequence
    float c2;           // scale log2(e), positive: its sign is in q
    float slack, below; // how far a score may lie over the reference, and the reference under the score that sets it

    __device__ __forceinline__ void load(const AttendArgs &a, const Tile &t, int h, int g, int c0, int cols, int col,
                                         int quad) {
        c2 = c2_of(a);
        below = DT == KNN_F16 ? kBelow / c2 : 0.0f;
        slack = (DT == KNN_F16 ? kSlack + kBelow : kSlack) / c2;
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            const int c = c0 + 16 * n + col;
            const bool live = c < cols;
            row_of[n] = live ? c / g : 0;
            const uint16_t *at = static_cast<const uint16_t *>(a.q) + (t.r0 + row_of[n]) * a.q_row +
                                 (h * g + (live ? c - row_of[n] * g : 0)) * a.q_head;
#pragma unroll
            for (int k = 0; k < KK; ++k) {
                u32x4_t v = *reinterpret_cast<const u32x4_t *>(at + 32 * k + 8 * quad);
                if (a.scale == 0.0f) v = u32x4_t{0, 0, 0, 0};
                if (a.scale < 0.0f) v ^= u32x4_t{0x80008000u, 0x80008000u, 0x80008000u, 0x80008000u};
                q[n][k] = v;
            }
            m[n] = kFloor;
            sum[n] = f32x4_t{0, 0, 0, 0};
#pragma unroll
            for (int d = 0; d < DB; ++d) o[n][d] = f32x4_t{0, 0, 0, 0};
        }
    }

    // U x 32 keys from `key` on, 32 each in LDS at kt[u] and their values behind them.  `all`: every column sees every
    // one of them; else a key is seen if it is before `end`, its half's page is one (bit 2 u + half of `real`), and it
    // is cached or named by the row's mask.
    template <int U>
    __device__ __forceinline__ void tile(const AttendArgs &a, const Tile &t, const uint32_t (&kt)[U], int64_t key, bool all,
                                         int64_t end, uint32_t real, int col, int quad, bool &left_out) {
        f32x4_t x[2 * U][NT];
#pragma unroll
        for (int u = 0; u < 2 * U; ++u) {
#pragma unroll
            for (int n = 0; n < NT; ++n) x[u][n] = f32x4_t{0, 0, 0, 0};
#pragma unroll
            for (int k = 0; k < KK; ++k) {
                const u32x4_t kr = *reinterpret_cast<const __attribute__((address_space(3))) u32x4_t *>(
                    static_cast<uintptr_t>(kt[u / 2] + (16 * (u & 1) + col) * ROW + 16 * ((4 * k + quad) ^ spread<D>(col))));
#pragma unroll
                for (int n = 0; n < NT; ++n) x[u][n] = mfma16<DT>(kr, q[n][k], x[u][n]);
            }
        }
        if (!all) {
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int u = 0; u < 2 * U; ++u) {
                    const uint32_t bits = (real >> u & 1u) != 0u ? seen(a, t, row_of[n], key + 16 * u + 4 * quad, end) : 0u;
#pragma unroll
                    for (int j = 0; j < 4; ++j) x[u][n][j] = (bits >> j & 1u) != 0u ? x[u][n][j] : -INFINITY;
                }
        }
        u32x4_t p[U][NT];
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            float top = -INFINITY;  // (the median with +inf is the larger one, in one instruction; fmaxf takes two)
#pragma unroll
            for (int u = 0; u < 2 * U; ++u)
#pragma unroll
                for (int j = 0; j < 4; ++j) top = __builtin_amdgcn_fmed3f(top, x[u][n][j], INFINITY);
            if (__any(top - m[n] > slack)) {  // (their difference is right where m + slack may round to twice the slack)
                top = fmaxf(top, __shfl_xor(top, 16));
                top = fmaxf(top, __shfl_xor(top, 32));
                const float to = fmaxf(m[n], DT == KNN_F16 ? top - below : top);
                const float by = exp2f((m[n] - to) * c2);
                m[n] = to;
#pragma unroll
                for (int j = 0; j < 4; ++j) sum[n][j] *= by;
#pragma unroll
                for (int d = 0; d < DB; ++d)
#pragma unroll
                    for (int j = 0; j < 4; ++j) o[n][d][j] *= by;
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                float e[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) e[j] = __builtin_amdgcn_exp2f((x[2 * u + (j >> 2)][n][j & 3] - m[n]) * c2);
                p[u][n] = u32x4_t{pack2<DT>(e[0], e[1]), pack2<DT>(e[2], e[3]), pack2<DT>(e[4], e[5]), pack2<DT>(e[6], e[7])};
            }
        }
        constexpr uint32_t kOne = DT == KNN_BF16 ? 0x3f803f80u : 0x3c003c00u;
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int n = 0; n < NT; ++n) sum[n] = mfma16<DT>(u32x4_t{kOne, kOne, kOne, kOne}, p[u][n], sum[n]);
        const int vrow = 4 * quad + (col >> 2);
        auto values = [&](int u, int d) {
            const uint32_t at =
                kt[u] + 32 * ROW + vrow * ROW + 16 * ((2 * d + ((col >> 1) & 1)) ^ spread<D>(vrow)) + 8 * (col & 1);
            const u32x2_t va = read_transposed(at), vb = read_transposed(at + 16 * ROW);
            return u32x4_t{va.x, va.y, vb.x, vb.y};
        };
        if (all) {
#pragma unroll
            for (int u = 0; u < U; ++u)
#pragma unroll
                for (int d = 0; d < DB; ++d) {
                    const u32x4_t v = values(u, d);
#pragma unroll
                    for (int n = 0; n < NT; ++n) o[n][d] = mfma16<DT>(v, p[u][n], o[n][d]);
                }
            return;
        }
        // A column must not take an infinity or NaN from a key that it does not see (0 * NaN is NaN): such elements are left
        // out of the product, and poison() gives them to those who see them.
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int d = 0; d < DB; ++d) {
                u32x4_t v = values(u, d);
                const u32x4_t bad = {not_finite<DT>(v.x), not_finite<DT>(v.y), not_finite<DT>(v.z), not_finite<DT>(v.w)};
                if (__any((bad.x | bad.y | bad.z | bad.w) != 0u)) {
                    v &= ~bad;
                    left_out = left_out || key + 32 * u < end;  // (a tile behind the end was not filled: it holds anything)
                }
#pragma unroll
                for (int n = 0; n < NT; ++n) o[n][d] = mfma16<DT>(v, p[u][n], o[n][d]);
            }
    }

    // Where a tile left values out: makes infinite, whatever the key's weight, the sums of the columns that see them (for
    // mean() to make NaN), by a product of 2^127 and 2^127 in bf16 for either type.  32-key tiles first, first + step, ...
    // of a span of n; the values come from memory once more, since their stage is long filled anew.  Behind the loop over the
    // tiles and not in it, where the masks that it needs would hold registers (2% of the time of trees, 7% of a prompt's).
    __device__ __forceinline__ void poison(const AttendArgs &a, const Tile &t, const Keys<D> &keys, int64_t k0, int64_t end,
                                           int first, int step, int n_tiles, int col, int quad) {
        constexpr uint32_t kFar = 0x7f00u;
#pragma unroll 1
        for (int i = first; i < n_tiles; i += step) {
            u32x4_t far[NT];
            const uint16_t *from[8];  // the values of element `col` of this lane's keys
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                const int key = 32 * i + 16 * half;
                const int32_t page = keys.entry(key);
                int rows;
                const char *at = static_cast<const char *>(a.v_cache) + keys.at(key, page, rows);
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    from[4 * half + j] = reinterpret_cast<const uint16_t *>(at) + min(4 * quad + j, rows) * D + col;
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                    const uint32_t bits = keys.real(page) ? seen(a, t, row_of[n], k0 + key + 4 * quad, end) : 0u;
                    far[n][2 * half] = ((bits & 1u) | (bits & 2u) << 15) * kFar;
                    far[n][2 * half + 1] = ((bits >> 2 & 1u) | (bits >> 2 & 2u) << 15) * kFar;
                }
            }
#pragma unroll
            for (int d = 0; d < DB; ++d) {
                u32x4_t bad;
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    bad[j] = not_finite<DT>(from[2 * j][16 * d] | static_cast<uint32_t>(from[2 * j + 1][16 * d]) << 16) &
                             (kFar | kFar << 16);
#pragma unroll
                for (int n = 0; n < NT; ++n) o[n][d] = mfma16<KNN_BF16>(bad, far[n], o[n][d]);
            }
        }
    }
};

// An element of the result: NaN where a value that is not finite was seen.  A tile that all columns see has them in its
// product, which leaves an infinity or (of a weight of 0, or two signs) NaN.
__device__ __forceinline__ float mean(float sum, float by) {
    const float v = sum * by;
    return fabsf(v) < INFINITY ? v : __builtin_nanf("");
}

// Four elements of a finished column, or of a part of one (`part` not null: its
// columns [cols][D]), and with d == 0 its reference and sum.
template <knn_dtype DT, int D>
__device__ __forceinline__ void store(const AttendArgs &a, int64_t at, int col, int d, f32x4_t r, float top, float l,
                                      float *part, float *part_ml) {
    if (part != nullptr) {
        if (d == 0) *reinterpret_cast<float2 *>(part_ml + 2 * col) = make_float2(top, l);
        *reinterpret_cast<f32x4_t *>(part + static_cast<int64_t>(col) * D + d) = r;
    } else {
        const float by = l > 0.0f ? 1.0f / l : l == 0.0f ? 0.0f : l;  // no key: 0; NaN stays
        *reinterpret_cast<u32x2_t *>(static_cast<uint16_t *>(a.out) + at * D + d) =
            u32x2_t{pack2<DT>(mean(r[0], by), mean(r[1], by)), pack2<DT>(mean(r[2], by), mean(r[3], by))};
        if (d == 0 && a.lse != nullptr) a.lse[at] = l == 0.0f ? -INFINITY : (top * c2_of(a) + log2f(l)) * kLn2;
    }
}

template <int D>
struct Shape {
    static constexpr int ROW = 2 * D;           // bytes of a key
    static constexpr int HALF = 32 * ROW;       // of 32 keys: one stage's K, then its V
    static constexpr int LOADS = HALF / 1024;   // wave loads of one half
    static constexpr int LANES = ROW / 16;      // lanes of a load on one key
    static constexpr int PER = 64 / LANES;      // keys of one load
    // Few columns: each wave on keys of its own.
    static constexpr int W = D == 256 ? 2 : 4;
    static constexpr size_t few_lds(int stages) { return static_cast<size_t>(W) * static_cast<size_t>(stages) * 2 * HALF; }
    // Many columns: four waves on the same keys.
    static constexpr int U = D == 256 ? 1 : 2;  // 32-key tiles between two barriers
    static constexpr int RING = D == 64 ? 8 : D == 128 ? 5 : 2;
    static constexpr size_t RING_LDS = static_cast<size_t>(RING) * 2 * HALF;
};

// Unsigned quotient, in 32 bits where that is enough (a fifth of the instructions).
__device__ __forceinline__ uint64_t quotient(uint64_t a, uint64_t b) {
    if (((a | b) >> 32) == 0) return static_cast<uint32_t>(a) / static_cast<uint32_t>(b);
    return a / b;
}

// Steps of `step` keys that a head of a sequence has.
__device__ __forceinline__ int steps_of(const Tile &t, int step) {
    return t.n > 0 ? static_cast<int>(quotient(static_cast<uint64_t>(t.total + step - 1), static_cast<uint64_t>(step))) : 0;
}

__device__ __forceinline__ int64_t uniform(int64_t v) {
    return static_cast<int64_t>(static_cast<uint64_t>(static_cast<uint32_t>(__builtin_amdgcn_readfirstlane(
                                    static_cast<int>(static_cast<uint64_t>(v) >> 32)))) << 32 |
                                static_cast<uint32_t>(__builtin_amdgcn_readfirstlane(static_cast<int>(v))));
}
__device__ __forceinline__ int64_t readlane64(int64_t v, int lane) {
    return static_cast<int64_t>(static_cast<uint64_t>(readlane_u32(static_cast<uint32_t>(static_cast<uint64_t>(v) >> 32), lane)) << 32 |
                                readlane_u32(static_cast<uint32_t>(v), lane));
}

// The steps of all sequences and key heads one behind the other (sequences in
// order, each one's heads in order), cut into one run a team; they differ by one
// step at most, and with fewer steps than teams only as many teams have one.
// Found by a wave, 64 sequences at a time, which its lanes keep.
struct Runs {
    uint64_t total, teams, each, more;  // steps; the teams that have any; the first `more` runs have each + 1 steps
    int64_t base;                       // first sequence of those the lanes hold
    int64_t behind;                     // steps of a head of the sequences before them
    Tile mine;
    uint32_t incl, own;  // steps of a head up to this lane's sequence, and its own
    int step;            // keys of one

    __device__ __forceinline__ void hold(const AttendArgs &a, int64_t s) {
        const int lane = threadIdx.x & 63;
        base = s;
        mine = tile_of(a, s + lane < a.S ? s + lane : a.S - 1);
        own = s + lane < a.S ? static_cast<uint32_t>(steps_of(mine, step)) : 0u;
        incl = wave_incl_scan_u32(own, lane);
    }
    __device__ __forceinline__ Runs(const AttendArgs &a, int64_t most, int step_keys) : step(step_keys) {
        behind = 0;
        hold(a, 0);
        uint64_t sum = readlane_u32(incl, 63);
        for (int64_t s = 64; s < a.S; s += 64) {
            behind = static_cast<int64_t>(sum);
            hold(a, s);
            sum += readlane_u32(incl, 63);
        }
        total = sum * static_cast<uint64_t>(a.kv_heads);
        teams = total < static_cast<uint64_t>(most) ? total : static_cast<uint64_t>(most);
        each = teams > 0 ? quotient(total, teams) : 0;
        more = total - each * teams;
    }
    __device__ __forceinline__ uint64_t begin(uint64_t team) const { return team * each + (team < more ? team : more); }
    // The team whose run holds step `at`.
    __device__ __forceinline__ int64_t team_of(uint64_t at) const {
        const uint64_t longer = more * (each + 1);
        return static_cast<int64_t>(at < longer ? quotient(at, each + 1) : more + quotient(at - longer, each));
    }
    // The sequence for which of(lane's steps before it, its steps) is true first, held and its lane returned.
    template <typename F>
    __device__ __forceinline__ int find(const AttendArgs &a, F of) {
        if (a.S > 64) {
            behind = 0;
            hold(a, 0);
        }
        while (true) {
            const uint64_t hit = __ballot(of(static_cast<uint64_t>(behind) + incl - own, static_cast<uint64_t>(own)));
            if (hit != 0) return __ffsll(static_cast<unsigned long long>(hit)) - 1;
            if (base + 64 >= a.S) return 0;  // not reached
            behind += readlane_u32(incl, 63);
            hold(a, base + 64);
        }
    }
    __device__ __forceinline__ Tile tile(int lane) const {
        return Tile{readlane64(mine.r0, lane), __builtin_amdgcn_readlane(mine.n, lane), readlane64(mine.length, lane),
                    readlane64(mine.total, lane)};
    }
    // Steps of a head before the sequence of a lane.
    __device__ __forceinline__ uint64_t before(int lane) const {
        return static_cast<uint64_t>(behind) + readlane_u32(incl, lane) - readlane_u32(own, lane);
    }
};

// A workgroup is column tile `ct` of a team.  Neighbours in the grid go to the 8
// XCDs in turn: a team's workgroups, which read the same keys, go to one.
struct Place {
    int64_t team, ct;
};
__device__ __forceinline__ Place place_of(int64_t tiles) {
    const int64_t id = blockIdx.x, in = id % (8 * tiles);
    return Place{id / (8 * tiles) * 8 + in % 8, in / 8};
}

// The keys k0 .. end - 1 of head h of sequence s, as far as column tile `ct`
// sees them, into the output or, where the head has keys in other runs too,
// into a part: f(tile, s, h, k0, end, part, part_ml) for one after the other of a
// team's run.  `cols` columns a tile.
template <int D, typename F>
__device__ __forceinline__ void each_span(const AttendArgs &a, int64_t tiles, int64_t teams, int step_keys, int cols, float *part,
                                          float *part_ml, F f) {
    const Place at = place_of(tiles);
    Runs runs(a, teams, step_keys);
    if (static_cast<uint64_t>(at.team) >= runs.teams) return;
    int64_t pos = static_cast<int64_t>(runs.begin(at.team));
    const int64_t stop = static_cast<int64_t>(runs.begin(at.team + 1));
    const uint64_t heads = static_cast<uint64_t>(a.kv_heads);
    const int l = runs.find(a, [&](uint64_t before, uint64_t own) { return (before + own) * heads > static_cast<uint64_t>(pos); });
    int64_t s = runs.base + l;
    const uint64_t off = static_cast<uint64_t>(pos) - runs.before(l) * heads;
    Tile t = runs.tile(l);
    int steps = steps_of(t, step_keys);
    int h = static_cast<int>(quotient(off, static_cast<uint64_t>(steps)));
    int step = static_cast<int>(off - static_cast<uint64_t>(h) * static_cast<uint64_t>(steps));
    const int g = a.q_heads / a.kv_heads;
    while (true) {
        const int n = static_cast<int>(steps - step < stop - pos ? steps - step : stop - pos);
        const int c0 = static_cast<int>(a.first_tile + at.ct) * cols, all = t.n * g;
        if (c0 < all) {
            int64_t end = static_cast<int64_t>(step + n) * step_keys;
            if (end > t.total) end = t.total;
            if (a.tree_mask == nullptr) {  // a chain: nothing sees what lies behind the tile's last row
                const int last = (c0 + cols < all ? c0 + cols - 1 : all - 1) / g;
                if (t.length + last + 1 < end) end = t.length + last + 1;
            }
            const bool whole = n == steps;
            const int64_t slot = (at.team * tiles + at.ct) * 2 + (step == 0 ? 1 : 0);
            f(t, s, h, static_cast<int64_t>(step) * step_keys, end, whole ? nullptr : part + slot * cols * D,
              whole ? nullptr : part_ml + slot * cols * 2);
        }
        pos += n;
        if (pos >= stop) return;
        step = 0;
        if (++h == a.kv_heads) {
            h = 0;
            do {
                t = tile_of(a, ++s);
                t.r0 = uniform(t.r0), t.length = uniform(t.length), t.total = uniform(t.total);
                t.n = __builtin_amdgcn_readfirstlane(t.n);
                steps = steps_of(t, step_keys);
            } while (steps == 0);
        }
        __syncthreads();  // the stages are read: the next keys may overwrite them
    }
}

// Few columns (NT x 16): the W waves share them and wave w takes the 32-key
// tiles w, w + W, ... of a span with a reference and sums of its own, joined at
// the end.  Each wave fills its own two stages by loads straight to LDS, one
// tile ahead, and waits only for its own loads: no barrier in the loop.  Where
// no wave gets a second tile it has one stage (NT = 1), and a CU two workgroups.
template <knn_dtype DT, int D, int NT>
__device__ __forceinline__ void span_few(const AttendArgs &a, const Tile &t, int64_t s, int h, int c0, int64_t k0,
                                         int64_t end, int stages, u32x4_t *lds, float *part, float *part_ml) {
    using Sh = Shape<D>;
    constexpr int W = Sh::W, DB = D / 16, COLS = 16 * NT;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int col = lane & 15, quad = lane >> 4;
    const int g = a.q_heads / a.kv_heads;
    const int cols = t.n * g;
    Columns<DT, D, NT> c;
    c.load(a, t, h, g, c0, cols, col, quad);
    const uint32_t mine =
        __builtin_amdgcn_readfirstlane(lds_offset(lds)) + wave * static_cast<uint32_t>(stages * 2 * Sh::HALF);
    const int n_tiles = end > k0 ? static_cast<int>((end - k0 + 31) / 32) : 0;
    const int own = n_tiles > wave ? (n_tiles - wave + W - 1) / W : 0;  // this wave's tiles
    const int whole = static_cast<int>((t.length < end ? t.length : end) - k0);  // keys that every column sees
    const Keys<D> keys(a, s, h, k0, end);
    // Lane l keeps the page of half l & 1 of this wave's tile l / 2 from tile `held` on.
    int32_t page_reg = 0;
    auto hold_pages = [&](int held) {
        page_reg = keys.entry(int64_t{32} * (wave + W * (held + (lane >> 1))) + 16 * (lane & 1));
    };
    auto page_of = [&](int tile, int half) { return __builtin_amdgcn_readlane(page_reg, 2 * (tile & 31) + half); };
    auto fill = [&](int i) {  // tile i of this wave into stage i & 1
        const uint32_t to = mine + static_cast<uint32_t>(i & 1) * (2 * Sh::HALF);
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            int rows;
            const int64_t at = keys.at(32 * (wave + W * i) + 16 * half, page_of(i, half), rows);
            const char *kp = static_cast<const char *>(a.k_cache) + at;
            const char *vp = static_cast<const char *>(a.v_cache) + at;
#pragma unroll
            for (int j = 0; j < Sh::LOADS / 2; ++j) {
                const int r = j * Sh::PER + lane / Sh::LANES;
                const int from = r < rows ? r : rows;
                const uint32_t off = from * Sh::ROW + 16 * ((lane % Sh::LANES) ^ spread<D>(r));
                load_to_lds_16(kp, off, to + half * (Sh::HALF / 2) + j * 1024);
                load_to_lds_16(vp, off, to + Sh::HALF + half * (Sh::HALF / 2) + j * 1024);
            }
        }
    };

    bool left_out = false;
    if (own > 0) {
        hold_pages(0);
        fill(0);
    }
    for (int i = 0; i < own; ++i) {
        const bool real_a = keys.real(page_of(i, 0)), real_b = keys.real(page_of(i, 1));
        if (i + 1 < own) {
            if (((i + 1) & 31) == 0) hold_pages(i + 1);
            fill(i + 1);
            __builtin_amdgcn_s_waitcnt(vmcnt_encoding<2 * Sh::LOADS>());
        } else {
            __builtin_amdgcn_s_waitcnt(kVmcntZero);
        }
        asm volatile("" ::: "memory");
        const uint32_t kt[1] = {mine + static_cast<uint32_t>(i & 1) * (2 * Sh::HALF)};
        const int key = 32 * (wave + W * i);
        const bool all = key <= whole - 32 && real_a && real_b;
        c.template tile<1>(a, t, kt, k0 + key, all, end, (real_a ? 1u : 0u) | (real_b ? 2u : 0u), col, quad, left_out);
        // the stage is read: the next round's loads may overwrite it
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    }

    if (left_out) c.poison(a, t, keys, k0, end, wave, W, n_tiles, col, quad);

    // Join the waves: references first, then each one's sums relative to the common reference.
    __syncthreads();  // every wave is done with its stages (its loads have landed)
    constexpr int PITCH = D + 4;
    float *stat = reinterpret_cast<float *>(lds);    // [2][W][COLS]: reference, sum
    float *acc = stat + 2 * W * COLS;                // [W][COLS][PITCH]
    static_assert((2 * W * COLS + W * COLS * PITCH) * sizeof(float) <= Sh::few_lds(NT == 1 ? 1 : 2), "the join fits the stages");
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        if (quad == 0) {
            stat[wave * COLS + 16 * n + col] = c.m[n];
            stat[W * COLS + wave * COLS + 16 * n + col] = c.sum[n][0];
        }
#pragma unroll
        for (int d = 0; d < DB; ++d)
            *reinterpret_cast<f32x4_t *>(acc + (wave * COLS + 16 * n + col) * PITCH + 16 * d + 4 * quad) = c.o[n][d];
    }
    __syncthreads();
    for (int i = threadIdx.x; i < COLS * (D / 4); i += W * 64) {
        const int cc = i / (D / 4), d = i % (D / 4) * 4;
        if (c0 + cc >= cols) continue;
        float top = kFloor;
#pragma unroll
        for (int w = 0; w < W; ++w) top = fmaxf(top, stat[w * COLS + cc]);
        float l = 0.0f;
        f32x4_t r{0, 0, 0, 0};
#pragma unroll
        for (int w = 0; w < W; ++w) {
            const float by = exp2f((stat[w * COLS + cc] - top) * c.c2);
            l += by * stat[W * COLS + w * COLS + cc];
            r += by * *reinterpret_cast<const f32x4_t *>(acc + (w * COLS + cc) * PITCH + d);
        }
        const int row = (c0 + cc) / g;
        const int64_t at = (t.r0 + row) * a.q_heads + h * g + (c0 + cc - row * g);  // (row, query head)
        store<DT, D>(a, at, cc, d, r, top, l, part, part_ml);
    }
}

template <knn_dtype DT, int D, int NT>
__global__ __launch_bounds__(Shape<D>::W * 64, NT == 1 && D < 256 ? 2 : 1) void k_attend(AttendArgs a, int64_t tiles, int64_t teams, int step,
                                                                int stages, float *part, float *part_ml) {
    extern __shared__ __align__(16) u32x4_t lds[];
    const int c0 = static_cast<int>(a.first_tile + place_of(tiles).ct) * (16 * NT);
    each_span<D>(a, tiles, teams, step, 16 * NT, part, part_ml,
                 [&](const Tile &t, int64_t s, int h, int64_t k0, int64_t end, float *to, float *to_ml) {
                     span_few<DT, D, NT>(a, t, s, h, c0, k0, end, stages, lds, to, to_ml);
                 });
}

// Many columns: four waves of NT x 16 each on the same keys, 64 at a time (32 at
// head_dim 256), which all of them read out of a ring of 32-key stages.  Each
// wave fetches a quarter of a tile.  One barrier every U tiles: behind it every
// wave's loads of them have landed and every wave has read the U before, whose
// stages are filled next.
template <knn_dtype DT, int D, int NT>
__device__ __forceinline__ void span_many(const AttendArgs &a, const Tile &t, int64_t s, int h, int c0, int64_t k0,
                                          int64_t end, u32x4_t *lds, float *part, float *part_ml) {
    using Sh = Shape<D>;
    constexpr int DB = D / 16, U = Sh::U, RING = Sh::RING, MINE = Sh::LOADS / 2;  // loads of a wave and tile
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int col = lane & 15, quad = lane >> 4;
    const int g = a.q_heads / a.kv_heads;
    const int cols = t.n * g;
    Columns<DT, D, NT> c;
    c.load(a, t, h, g, c0 + 16 * NT * wave, cols, col, quad);
    const uint32_t base = __builtin_amdgcn_readfirstlane(lds_offset(lds));
    const int n = end > k0 ? static_cast<int>((end - k0 + 31) / 32) : 0;
    const int whole = static_cast<int>((t.length < end ? t.length : end) - k0);  // keys that every column sees
    const Keys<D> keys(a, s, h, k0, end);
    // Lane l keeps the page of half l & 1 of tile l / 2 from tile `held` on, and of the 32 tiles before.
    int32_t page_reg = 0, page_old = 0;
    auto hold_pages = [&](int held) {
        page_old = page_reg;
        page_reg = keys.entry(int64_t{32} * (held + (lane >> 1)) + 16 * (lane & 1));
    };
    const int half = wave >> 1;  // of a tile's 32 keys: which 16 this wave fetches half of
    auto fill = [&](int i) {     // this wave's quarter of tile i into its stage
        if ((i & 31) == 0) hold_pages(i);
        const uint32_t to = base + static_cast<uint32_t>(i % RING) * (2 * Sh::HALF);
        int rows;
        const int64_t at = keys.at(32 * i + 16 * half, __builtin_amdgcn_readlane(page_reg, 2 * (i & 31) + half), rows);
        const char *kp = static_cast<const char *>(a.k_cache) + at, *vp = static_cast<const char *>(a.v_cache) + at;
#pragma unroll
        for (int j = 0; j < MINE / 2; ++j) {
            const int r = ((wave & 1) * (MINE / 2) + j) * Sh::PER + lane / Sh::LANES;  // row of the half
            const uint32_t off = min(r, rows) * Sh::ROW + 16 * ((lane % Sh::LANES) ^ spread<D>(r));
            load_to_lds_16(kp, off, to + (wave * (MINE / 2) + j) * 1024);
            load_to_lds_16(vp, off, to + Sh::HALF + (wave * (MINE / 2) + j) * 1024);
        }
    };

#pragma unroll
    for (int i = 0; i < RING - U; ++i)
        if (i < n) fill(i);
    uint32_t stage = base, real = 0, kt[U];
    bool left_out = false;
    // Makes ready the tiles i .. i + U - 1; whether every column sees all of their keys.
    auto ready = [&](int i) {
        // This wave's loads of them have landed when only the later tiles' are on their way.
        if (i + RING - U - 1 < n) __builtin_amdgcn_s_waitcnt(vmcnt_encoding<(RING - 2 * U) * MINE>());
        else __builtin_amdgcn_s_waitcnt(kVmcntZero);
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (i + RING - U + u < n) fill(i + RING - U + u);
        // the pages of tiles i .. i + U - 1 (of one 32): held since they were filled
        const int filled = i + RING - 1 < n ? i + RING - 1 : n - 1;
        const int32_t pages = (filled >> 5) != (i >> 5) ? page_old : page_reg;
        real = 0;
#pragma unroll
        for (int u = 0; u < 2 * U; ++u) real |= keys.real(__builtin_amdgcn_readlane(pages, 2 * (i & 31) + u)) ? 1u << u : 0u;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            kt[u] = stage;
            stage += 2 * Sh::HALF;
            if (stage == base + RING * 2 * Sh::HALF) stage = base;
        }
        return 32 * i <= whole - 32 * U && real == (1u << 2 * U) - 1u;
    };
    // (Two loops in one another: one for both kinds of tile moves half of the sums from register to register every time.)
    for (int i = 0; i < n; i += U) {
        bool all = ready(i);
        while (all) {
            c.template tile<U>(a, t, kt, k0 + 32 * i, true, end, real, col, quad, left_out);
            i += U;
            if (i >= n) break;
            all = ready(i);
        }
        if (!all) c.template tile<U>(a, t, kt, k0 + 32 * i, false, end, real, col, quad, left_out);
    }
    if (left_out) c.poison(a, t, keys, k0, end, 0, 1, n, col, quad);
#pragma unroll
    for (int i = 0; i < NT; ++i) {
        const int cc = 16 * NT * wave + 16 * i + col;
        if (c0 + cc >= cols) continue;
        const int row = (c0 + cc) / g;
        const int64_t at = (t.r0 + row) * a.q_heads + h * g + (c0 + cc - row * g);
#pragma unroll
        for (int d = 0; d < DB; ++d)
            store<DT, D>(a, at, cc, 16 * d + 4 * quad, c.o[i][d], c.m[i], c.sum[i][0], part, part_ml);
    }
}

template <knn_dtype DT, int D, int NT>
__global__ __launch_bounds__(256, 2) void k_attend_many(AttendArgs a, int64_t tiles, int64_t teams, int step,
                                                                      float *part, float *part_ml) {
    extern __shared__ __align__(16) u32x4_t lds[];
    const int c0 = static_cast<int>(a.first_tile + place_of(tiles).ct) * (64 * NT);
    each_span<D>(a, tiles, teams, step, 64 * NT, part, part_ml,
                 [&](const Tile &t, int64_t s, int h, int64_t k0, int64_t end, float *to, float *to_ml) {
                     span_many<DT, D, NT>(a, t, s, h, c0, k0, end, lds, to, to_ml);
                 });
}

// Joins the parts of a (row, query head) whose keys lie in several runs, one
// wave each: the references of up to 64 parts at once, a lane each, then the
// parts' outputs.
template <knn_dtype DT, int D>
__global__ __launch_bounds__(256) void k_attend_join(AttendArgs a, int64_t tiles, bool by_sequence, int64_t teams, int step,
                                                     int cols, const float *part, const float *part_ml) {
    constexpr int PER = D / 64;  // elements of a lane
    const int lane = threadIdx.x & 63;
    const int64_t heads = a.q_heads;
    int64_t at = static_cast<int64_t>(blockIdx.x) * 4 + (threadIdx.x >> 6);  // (row, query head)
    if (by_sequence) {  // of sequence blockIdx.y, from the first row that has columns in these tiles
        at += (a.row_offsets[blockIdx.y] + a.first_tile * cols / (heads / a.kv_heads)) * heads;
        if (at >= a.row_offsets[blockIdx.y + 1] * heads) return;
    }
    const int64_t row = static_cast<int64_t>(quotient(static_cast<uint64_t>(at), static_cast<uint64_t>(heads)));
    if (row >= a.rows || row >= a.row_offsets[a.S]) return;  // the whole wave
    Runs runs(a, teams, step);
    int64_t s = 0;
    if (a.S > 64) s = set_of_query_wave(a.row_offsets, a.S, row);
    const int lane_of = a.S > 64 ? runs.find(a, [&](uint64_t, uint64_t) { return runs.base + lane == s; })
                                 : __ffsll(static_cast<unsigned long long>(__ballot(
                                       lane < a.S && runs.mine.r0 <= row && row < runs.mine.r0 + runs.mine.n))) - 1;
    if (lane_of < 0) return;  // a row past the most that the caller said
    const Tile t = runs.tile(lane_of);
    if (row - t.r0 >= t.n) return;
    const int g = a.q_heads / a.kv_heads, head = static_cast<int>(at - row * heads), h = head / g;
    const int col = static_cast<int>(row - t.r0) * g + head - h * g, c = col % cols;
    const int64_t ct = col / cols - a.first_tile;
    if (ct < 0 || ct >= tiles) return;  // of another launch
    const uint64_t steps = static_cast<uint64_t>(steps_of(t, step));
    const uint64_t first = runs.before(lane_of) * static_cast<uint64_t>(a.kv_heads) + static_cast<uint64_t>(h) * steps;
    const int64_t w0 = runs.team_of(first), w1 = runs.team_of(first + steps - 1);
    if (w0 == w1) return;  // one team had all of it
    auto slot = [&](int64_t w) { return ((w * tiles + ct) * 2 + (w == w0 ? 1 : 0)) * cols + c; };
    const float c2 = c2_of(a);
    float top = kFloor, l = 0.0f, r[PER] = {};
    for (int64_t base = w0; base <= w1; base += 64) {
        const int n = static_cast<int>(w1 - base + 1 < 64 ? w1 - base + 1 : 64);
        const float2 ml = lane < n ? *reinterpret_cast<const float2 *>(part_ml + 2 * slot(base + lane)) : make_float2(kFloor, 0.0f);
        const float to = fmaxf(top, wave_allmax(ml.x));
        const float old = exp2f((top - to) * c2), mine = exp2f((ml.x - to) * c2);
        top = to;
        l *= old;
#pragma unroll
        for (int j = 0; j < PER; ++j) r[j] *= old;
        l += wave_allsum(mine * ml.y);
        for (int i = 0; i < n; i += 4) {  // four parts on their way at once
            float v[4][PER];
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const float *from = part + slot(base + min(i + u, n - 1)) * D + lane * PER;
#pragma unroll
                for (int j = 0; j < PER; ++j) v[u][j] = from[j];
            }
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                if (i + u >= n) break;
                const float by = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(mine), i + u));
#pragma unroll
                for (int j = 0; j < PER; ++j) r[j] += by * v[u][j];
            }
        }
    }
    const float by = l > 0.0f ? 1.0f / l : l == 0.0f ? 0.0f : l;
    uint16_t *out = static_cast<uint16_t *>(a.out) + at * D + lane * PER;
    if constexpr (PER == 1) {
        out[0] = static_cast<uint16_t>(pack2<DT>(mean(r[0], by), 0.0f));
    } else {
#pragma unroll
        for (int j = 0; j < PER; j += 2) *reinterpret_cast<uint32_t *>(out + j) = pack2<DT>(mean(r[j], by), mean(r[j + 1], by));
    }
    if (lane == 0 && a.lse != nullptr) a.lse[at] = l == 0.0f ? -INFINITY : (top * c2_of(a) + log2f(l)) * kLn2;
}

template <knn_dtype DT, int D>
hipError_t launch(AttendArgs a, const AttendPlan &p, float *part, float *part_ml, hipStream_t stream) {
    if (p.teams * p.tiles > 0x7fffffffLL || (a.rows * a.q_heads + 3) / 4 > 0x7fffffffLL) return hipErrorInvalidConfiguration;
    const dim3 few(Shape<D>::W * 64);
    constexpr int N = D < 256 ? D : 64;  // (the wider kinds are not taken at 256)
    const int64_t g = a.q_heads / a.kv_heads;
    for (int64_t first = 0; first < p.all_tiles; first += p.tiles) {
        const int64_t tiles = p.all_tiles - first < p.tiles ? p.all_tiles - first : p.tiles;
        const dim3 grid(static_cast<unsigned>(p.teams * tiles));
        a.first_tile = first;
        if (p.cols == 16) k_attend<DT, D, 1><<<grid, few, Shape<D>::few_lds(p.stages), stream>>>(a, tiles, p.teams, p.step, p.stages, part, part_ml);
        else if (p.cols == 32) k_attend<DT, N, 2><<<grid, few, Shape<D>::few_lds(p.stages), stream>>>(a, tiles, p.teams, p.step, p.stages, part, part_ml);
        else if (p.cols == 64) k_attend_many<DT, D, 1><<<grid, 256, Shape<D>::RING_LDS, stream>>>(a, tiles, p.teams, p.step, part, part_ml);
        else k_attend_many<DT, N, 2><<<grid, 256, Shape<D>::RING_LDS, stream>>>(a, tiles, p.teams, p.step, part, part_ml);
        if (p.total == 0) continue;
        // All rows, or where those are fewer as many of each sequence as may have columns in these tiles.
        const int64_t some = (tiles * p.cols + g - 1) / g + 1;
        const bool by_sequence = tiles < p.all_tiles && a.S <= 65535 && a.S * some < a.rows;
        const dim3 joins(static_cast<unsigned>(((by_sequence ? some : a.rows) * a.q_heads + 3) / 4),
                         by_sequence ? static_cast<unsigned>(a.S) : 1u);
        k_attend_join<DT, D><<<joins, 256, 0, stream>>>(a, tiles, by_sequence, p.teams, p.step, p.cols, part, part_ml);
    }
    return hipGetLastError();
}

template <knn_dtype DT>
hipError_t launch(const AttendArgs &a, const AttendPlan &p, float *part, float *part_ml, hipStream_t stream) {
    switch (a.head_dim) {
    case 64: return launch<DT, 64>(a, p, part, part_ml, stream);
    case 128: return launch<DT, 128>(a, p, part, part_ml, stream);
    default: return launch<DT, 256>(a, p, part, part_ml, stream);
    }
}

}  // namespace

AttendPlan plan_attend(int64_t rows, int64_t S, int64_t q_heads, int64_t kv_heads, int64_t head_dim, int64_t max_rows,
                       int64_t max_keys) {
    AttendPlan p{};
    const int64_t cols = max_rows * (q_heads / kv_heads);
    // As few columns a workgroup as hold a sequence's, so that its keys are read once a head; measured on 32 sequences of
    // 2,000 to 8,000 tokens, 8 heads of 128: 16 columns 133 us, 137 in the kind of 32; 20 columns 138 in that of 32, 143
    // in two tiles of 16; 64 columns 158, 163 in the kind of 128 and 186 in two tiles of 32; 68 columns 166 in that of
    // 128, 193 in two tiles of 64.  (Heads of 64 on 4 sequences of 16,000 to 32,000 tokens would be the faster in two
    // narrow tiles up to 64 columns: 41 us for 48 at 20, 50 for 53 at 64.)  At head_dim 256 the wider kind of either
    // kernel does not fit the registers.
    p.cols = cols <= 16 ? 16 : cols <= 32 && head_dim < 256 ? 32 : cols <= 64 || head_dim == 256 ? 64 : 128;
    p.all_tiles = p.tiles = (cols + p.cols - 1) / p.cols;
    // As many workgroups as the CUs hold at once, each with 256 keys or more (many columns: 128); teams a multiple of 8
    // (the XCDs).  Heads of up to kWhole keys are not parted: nothing to join (of 1,001 keys, one token and 32 heads:
    // 15.8 us, in four parts 14.5).  Nor are those of wide calls, whose column tiles leave room for fewer than 8 teams
    // where there are 8 heads or more: a workgroup each for a head and a tile (up to kWide of them) fill the CUs as they
    // get free, whatever a chain's tiles see.  (A sequence of fewer than 8 key heads would have fewer workgroups a tile than
    // 8 teams: it is parted where it may be over 8 times as long as the rows.)  Four prompts of 4,000 to 8,000 rows with 64
    // heads on 8 take 6.05 ms, 9.5 in 8 teams, and a prompt's 1,040 rows beside 63 decoding sequences of 100 to 8,000 tokens
    // 0.97 ms, 7.95.  As wide are those whose rows cannot fill half of the tiles that max_rows asks for (a sequence has
    // rows g / cols / S + 1 of them at most, on average), with four and more heads for each team that there would be room
    // for: 512 rows of as many sequences with 64 heads on 8, of which max_rows says nothing, take 1.29 ms, 6.97 in 16 teams
    // (0.31 where it is 1).
    const int64_t g = q_heads / kv_heads, heads = S * kv_heads, room = 512 / p.tiles / 8 * 8;
    const bool loose = p.tiles * p.cols * S >= 2 * (rows * g + p.cols * S) && heads >= 4 * room;
    const bool many = p.cols > 32, short_ones = heads >= 8 && max_keys <= 8 * max_rows;
    const bool wide = max_keys <= (int64_t{1} << 30) && (room < 8 ? kv_heads >= 8 || short_ones : loose);
    const bool whole = max_keys <= kWhole || wide;
    p.step = whole ? static_cast<int>((max_keys + 63) / 64 * 64) : 64;
    p.stages = p.cols == 16 && max_keys <= 32 * (head_dim == 256 ? 2 : 4) ? 1 : 2;
    int64_t slots = wide ? kWide : 512;
    if (!many && head_dim >= 128 && p.stages == 2) slots = 256;
    const int64_t least = many ? 128 : 256, most = heads * (whole ? 1 : (max_keys + least - 1) / least);
    p.teams = (most + 7) / 8 * 8;
    if (p.teams * p.tiles > slots) p.teams = slots / p.tiles / 8 * 8;  // one workgroup too many takes a second round
    if (p.teams < 8) p.teams = 8;
    // (The heads of one sequence in as many runs, or in a divisor of their number, are not parted either.)
    if (whole || (S == 1 && kv_heads % p.teams == 0)) return p;
    // Under 8 heads and over 64 column tiles there are 8 teams all the same, and parts of 16 times a head's queries in
    // fp32: 4 GiB for 8,000 rows with 64 heads on one.  In eight launches that share 512 MiB these take 5.75 ms, in one
    // 5.57.
    const size_t tile = static_cast<size_t>(p.teams) * 2 * static_cast<size_t>(p.cols) * (static_cast<size_t>(head_dim) + 2) * sizeof(float);
    const int64_t at_once = static_cast<int64_t>(kAttendParts / tile), launches = (p.tiles + at_once - 1) / at_once;
    p.tiles = (p.tiles + launches - 1) / launches;
    const size_t cells = static_cast<size_t>(p.teams * p.tiles) * 2 * static_cast<size_t>(p.cols);
    p.off_ml = cells * static_cast<size_t>(head_dim) * sizeof(float);
    p.total = p.off_ml + cells * 2 * sizeof(float);
    return p;
}

hipError_t launch_attend(const AttendArgs &a, const AttendPlan &p, knn_dtype dtype, void *workspace,
                         hipStream_t stream) {
    float *part = static_cast<float *>(workspace);
    float *part_ml = reinterpret_cast<float *>(static_cast<char *>(workspace) + p.off_ml);
    return dtype == KNN_BF16 ? launch<KNN_BF16>(a, p, part, part_ml, stream)
                             : launch<KNN_F16>(a, p, part, part_ml, stream);
}

}  // namespace knnlm
