// The weight that a sequence's rows put on each of its cached keys.
//
// With the logarithms of the rows' sums in hand (attention's lse), a key's
// weight of row i and query head a is exp(scale q_ia.k_j - lse_ia); a key's
// mass is what all rows that see it and all heads of its key head put on it,
// and a share of what it was before.
//
// The rows and query heads of a key head are the columns of S = Q K^T on the
// matrix cores: 16 columns x 16 keys an instruction, with the keys as its right
// operand, so that a lane holds 4 columns of one key and the sum over columns
// stays within it until the end of a tile.  A wave holds 64 keys (32 of
// head_dim 256) in the registers that the instructions read, straight from
// memory; the queries of the sequence's rows lie in LDS, read by all waves of
// the workgroup.  So keys are read once, by a wave each, and waves wait for
// each other only where a workgroup goes on to another head.
#include "lm_device.h"
#include "mfma_device.h"

namespace knnlm {

namespace {

constexpr float kLog2e = 1.4426950408889634f;
constexpr int kCus = 256;
constexpr int kNobody = -0x7fffffff - 1;

template <int D>
struct Shape {
    static constexpr int KK = D / 32;       // matrix instructions over a head
    static constexpr int ROW = 2 * D;       // bytes
    static constexpr int B = D == 256 ? 2 : 4;  // 16-key blocks of a tile
    static constexpr int KEYS = 16 * B;
    static constexpr int MOST = 65536 / D;  // columns in LDS at once: 128 KiB
};

__host__ __device__ constexpr int64_t tiles_of(int64_t keys, int tile) { return (keys + tile - 1) / tile; }

// What a tile of a sequence costs: the time that its keys take from memory, or
// that of its columns on the cores, whichever is more (16 column tiles of 64
// keys take as long as 16 KiB).
__device__ __forceinline__ int64_t cost_of(int n, int g, int keys) {
    const int64_t work = ((static_cast<int64_t>(n) * g + 15) / 16 * keys + 63) / 64;
    return work > 16 ? work : 16;
}

// The columns that are staged in LDS.
struct Staged {
    u32x4_t *q;      // [columns][D / 8], chunk c of column r at c ^ spread(r)
    float *lse2;     // [columns] lse log2(e), +inf of a column that adds nothing
    int32_t *row;    // [columns] row within the sequence, kNobody of such a column
};

// Columns c0 .. c0 + n - 1 of key head h into LDS, and zeros up to `padded`.
template <int D, int THREADS>
__device__ __forceinline__ void stage(const WeighArgs &a, const Tile &t, const Staged &st, int h, int g, int c0, int n,
                                      int padded) {
    constexpr int CHUNKS = D / 8;
    auto source_of = [&](int i) -> int64_t {
        const int64_t source = a.source_rows != nullptr ? a.source_rows[t.r0 + i] : t.r0 + i;
        return source < a.source_count ? source : -1;
    };
    for (int c = static_cast<int>(threadIdx.x); c < padded; c += THREADS) {
        const int i = (c0 + c) / g;
        const int64_t source = c < n ? source_of(i) : -1;
        const float lse = source >= 0 ? a.lse[source * a.q_heads + h * g + (c0 + c - i * g)] : INFINITY;
        st.lse2[c] = isfinite(lse) ? lse * kLog2e : INFINITY;
        st.row[c] = isfinite(lse) ? i : kNobody;
    }
    for (int e = static_cast<int>(threadIdx.x); e < padded * CHUNKS; e += THREADS) {
        const int c = e / CHUNKS, chunk = e % CHUNKS, i = (c0 + c) / g;
        const int64_t source = c < n ? source_of(i) : -1;
        u32x4_t v{0, 0, 0, 0};
        if (source >= 0)
            v = *reinterpret_cast<const u32x4_t *>(static_cast<const uint16_t *>(a.q) + source * a.q_row +
                                                   (h * g + (c0 + c - i * g)) * a.q_head + chunk * 8);
        st.q[c * CHUNKS + (chunk ^ spread<D>(c))] = v;
    }
}

// Whether a column of this row sees a key: all see the cached ones (draft < 0).
__device__ __forceinline__ bool sees(const WeighArgs &a, const Tile &t, int row, int draft) {
    if (a.tree_mask == nullptr || draft < 0 || row == kNobody) return draft <= row;
    return draft < 32 * a.mask_words && (a.tree_mask[(t.r0 + row) * a.mask_words + (draft >> 5)] >> (draft & 31) & 1u) != 0u;
}

template <knn_dtype DT, int D, int WAVES>
__global__ __launch_bounds__(WAVES * kWave, 4) void k_key_weights(WeighArgs a, int most) {
    using Sh = Shape<D>;
    constexpr int KK = Sh::KK, B = Sh::B, THREADS = WAVES * kWave;
    extern __shared__ __align__(16) u32x4_t lds[];
    __shared__ int64_t sums[WAVES];
    __shared__ int64_t found[2];
    const Staged st{lds, reinterpret_cast<float *>(lds + static_cast<size_t>(most) * (D / 8)),
                    reinterpret_cast<int32_t *>(lds + static_cast<size_t>(most) * (D / 8)) + most};
    const int tid = static_cast<int>(threadIdx.x), lane = tid & (kWave - 1);
    const int wave = __builtin_amdgcn_readfirstlane(tid / kWave);
    const int col = lane & 15, quad = lane >> 4;
    const int g = a.q_heads / a.kv_heads;
    const float c2 = a.scale * kLog2e;

    // The tiles of all sequences and heads lie one behind the other, and this
    // workgroup takes those that begin in its share of their cost.
    const int64_t per = (a.S + THREADS - 1) / THREADS, s_lo = tid * per < a.S ? tid * per : a.S;
    const int64_t s_hi = s_lo + per < a.S ? s_lo + per : a.S;
    auto whole_cost = [&](int64_t s) {
        const Tile t = tile_of(a, s);
        return t.n == 0 ? 0 : tiles_of(t.total, Sh::KEYS) * a.kv_heads * cost_of(t.n, g, Sh::KEYS);
    };
    int64_t mine = 0;
    for (int64_t s = s_lo; s < s_hi; ++s) mine += whole_cost(s);
    int64_t before = mine;  // inclusive over the wave, then exclusive over the workgroup
#pragma unroll
    for (int off = 1; off < kWave; off *= 2) {
        const int64_t o = __shfl_up(before, off);
        if (lane >= off) before += o;
    }
    if (lane == kWave - 1) sums[wave] = before;
    if (tid == 0) found[0] = a.S, found[1] = 0;
    __syncthreads();
    int64_t all = 0;
    before -= mine;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) {
        if (w == wave) before += all;
        all += sums[w];
    }
    const int64_t from = all / gridDim.x * blockIdx.x + all % gridDim.x * blockIdx.x / gridDim.x;
    const int64_t to = all / gridDim.x * (blockIdx.x + 1) + all % gridDim.x * (blockIdx.x + 1) / gridDim.x;
    if (from >= before && from < before + mine) {  // (one thread)
        int64_t s = s_lo, base = before;
        while (s < s_hi) {
            const int64_t c = whole_cost(s);
            if (from < base + c) break;
            base += c, ++s;
        }
        found[0] = s, found[1] = base;
    }
    __syncthreads();
    int64_t s = found[0], base = found[1];
    for (; s < a.S && base < to; ++s) {
        const Tile t = tile_of(a, s);
        if (t.n == 0) continue;
        const int64_t tiles = tiles_of(t.total, Sh::KEYS), cost = cost_of(t.n, g, Sh::KEYS), each = tiles * a.kv_heads;
        const int64_t first = from > base ? (from - base + cost - 1) / cost : 0;
        const int64_t end = (to - base + cost - 1) / cost;
        const int64_t last = end < each ? end : each;
        base += each * cost;
        const int cols = t.n * g;
        for (int64_t at = first; at < last;) {
            const int h = static_cast<int>(at / tiles);
            const int tile0 = static_cast<int>(at - h * tiles);
            const int tile1 = static_cast<int>(last - h * tiles < tiles ? last - h * tiles : tiles);
            at = (h + 1) * tiles;
            const int32_t *table = a.cache.pages + s * a.cache.table_width;
            const int total_keys = static_cast<int>(t.total), last_block = (total_keys - 1) >> 4;
            const int length = static_cast<int>(t.length < t.total ? t.length : t.total);
            const int in_page = (1 << a.cache.page_log2) - 1;
            // Rounds of one tile a wave, with the columns once more each; one round of all tiles where they fit LDS.
            const int step = cols > most ? WAVES : tile1 - tile0;
            for (int round = tile0; round < tile1; round += step) {
                const int stop = step < tile1 - round ? round + step : tile1;
                float sum[B] = {};
                for (int c0 = 0; c0 < cols; c0 += most) {
                    const int n = cols - c0 < most ? cols - c0 : most, padded = (n + 15) & ~15;
                    __syncthreads();
                    stage<D, THREADS>(a, t, st, h, g, c0, n, padded);
                    __syncthreads();
                    // The pages of this wave's next tiles: block b of the i-th in lane i B + b, or -1.
                    constexpr int AHEAD = kWave / B;
                    int32_t pages = 0;
                    for (int tile = round + wave, i = 0; tile < stop; tile += WAVES, ++i) {
                        const int block0 = tile * B, first = i % AHEAD * B;
                        if (first == 0) {
                            const int block = (tile + lane / B * WAVES) * B + lane % B;
                            pages = table[min(block, last_block) << 4 >> a.cache.page_log2];
                            pages = pages >= 0 && pages < a.cache.n_pages ? pages : -1;
                        }
                        // Each quarter of the wave has a block's masses.
                        const int j0 = tile * Sh::KEYS, j = j0 + 16 * (quad & (B - 1)) + col;
                        const int32_t p = __shfl(pages, first + (quad & (B - 1)));
                        const bool mine = quad < B && j < total_keys && p >= 0;
                        const int64_t place = ((static_cast<int64_t>(p) * a.kv_heads + h) << a.cache.page_log2) + (j & in_page);
                        float mass = 0.0f;
                        if (mine && j < length && a.decay != 0.0f && c0 + most >= cols) mass = a.mass[place];
                        u32x4_t k[B][KK];
#pragma unroll
                        for (int b = 0; b < B; ++b) {
                            const int32_t page = __builtin_amdgcn_readlane(pages, first + b);
                            const int64_t at_page = static_cast<int64_t>(page < 0 ? 0 : page) * a.kv_heads + h;
                            const int slot = (min(block0 + b, last_block) << 4) & in_page;
                            // (of the last block, the places behind the last key are read as well, whatever they hold)
                            const u32x4_t *kp = reinterpret_cast<const u32x4_t *>(static_cast<const uint16_t *>(a.k_cache) +
                                                                                  ((at_page << a.cache.page_log2) + slot) * D);
#pragma unroll
                            for (int kk = 0; kk < KK; ++kk) k[b][kk] = kp[col * (D / 8) + quad + 4 * kk];
                        }
                        auto scores = [&](int c, f32x4_t (&x)[B]) {
                            u32x4_t q[KK];
#pragma unroll
                            for (int kk = 0; kk < KK; ++kk)
                                q[kk] = st.q[(c + col) * (D / 8) + ((4 * kk + quad) ^ spread<D>(col))];
#pragma unroll
                            for (int b = 0; b < B; ++b) x[b] = f32x4_t{0, 0, 0, 0};
#pragma unroll
                            for (int kk = 0; kk < KK; ++kk)
#pragma unroll
                                for (int b = 0; b < B; ++b) x[b] = mfma16<DT>(q[kk], k[b][kk], x[b]);
                        };
                        float w[B] = {};
                        bool plain = j0 + Sh::KEYS <= length;
                        if (plain) {
#pragma unroll 1
                            for (int c = 0; c < padded; c += 16) {
                                f32x4_t x[B];
                                scores(c, x);
                                const f32x4_t l = *reinterpret_cast<const f32x4_t *>(st.lse2 + c + 4 * quad);
#pragma unroll
                                for (int b = 0; b < B; ++b)
#pragma unroll
                                    for (int r = 0; r < 4; ++r) w[b] += __builtin_amdgcn_exp2f(fmaf(x[b][r], c2, -l[r]));
                            }
                            // Keys that are not finite: whose they are is looked at column by column.
                            bool odd = false;
#pragma unroll
                            for (int b = 0; b < B; ++b) odd = odd || w[b] != w[b];
                            plain = !__any(odd);
                        }
                        if (!plain) {
                            const int draft0 = j0 + col - length;  // of block 0's key
#pragma unroll
                            for (int b = 0; b < B; ++b) {  // (a block at a time, to spare registers)
                                w[b] = 0.0f;
#pragma unroll 1
                                for (int c = 0; c < padded; c += 16) {
                                    f32x4_t x{0, 0, 0, 0};
#pragma unroll
                                    for (int kk = 0; kk < KK; ++kk)
                                        x = mfma16<DT>(st.q[(c + col) * (D / 8) + ((4 * kk + quad) ^ spread<D>(col))], k[b][kk], x);
#pragma unroll
                                    for (int r = 0; r < 4; ++r) {
                                        const int row = st.row[c + 4 * quad + r];
                                        const float e = __builtin_amdgcn_exp2f(fmaf(x[r], c2, -st.lse2[c + 4 * quad + r]));
                                        w[b] += sees(a, t, row, draft0 + 16 * b) ? e : 0.0f;
                                    }
                                }
                            }
                        }
#pragma unroll
                        for (int b = 0; b < B; ++b) sum[b] = w[b] + (c0 > 0 ? sum[b] : 0.0f);
                        if (c0 + most < cols) continue;
#pragma unroll
                        for (int b = 0; b < B; ++b) {
                            sum[b] += __shfl_xor(sum[b], 16);
                            sum[b] += __shfl_xor(sum[b], 32);
                        }
                        float drawn = sum[0];
#pragma unroll
                        for (int b = 1; b < B; ++b) drawn = quad == b ? sum[b] : drawn;
                        if (!mine) continue;
                        a.mass[place] = drawn + a.decay * mass;
                        if (j >= length && a.key_positions != nullptr)
                            a.key_positions[place] = a.positions != nullptr ? a.positions[t.r0 + (j - length)] : j;
                    }
                }
            }
        }
    }
}

template <knn_dtype DT, int D, int WAVES>
void launch(const WeighArgs &a, int most, hipStream_t stream) {
    using Sh = Shape<D>;
    const size_t lds = static_cast<size_t>(most) * (Sh::ROW + 8);
    const size_t fit = (size_t{156} << 10) / (lds + 1024);
    const int64_t room = fit * WAVES > 16 ? 16 / WAVES : fit < 1 ? 1 : static_cast<int64_t>(fit);  // workgroups of a CU
    // (a sequence has max_rows rows at most, and there are `rows`)
    const int64_t tiles = a.S * a.kv_heads * tiles_of(a.max_keys, Sh::KEYS);
    int64_t blocks = (tiles + WAVES - 1) / WAVES;
    if (blocks > kCus * room) blocks = kCus * room;
    k_key_weights<DT, D, WAVES><<<dim3(static_cast<unsigned>(blocks)), WAVES * kWave, lds, stream>>>(a, most);
}

template <knn_dtype DT, int D>
hipError_t launch(const WeighArgs &a, hipStream_t stream) {
    const int64_t cols = (a.max_rows * (a.q_heads / a.kv_heads) + 15) / 16 * 16;
    const int most = static_cast<int>(cols < Shape<D>::MOST ? cols : Shape<D>::MOST);
    if (most * 4 <= Shape<D>::MOST) launch<DT, D, 4>(a, most, stream);
    else if (most * 2 <= Shape<D>::MOST) launch<DT, D, 8>(a, most, stream);
    else launch<DT, D, 16>(a, most, stream);
    return hipGetLastError();
}

template <knn_dtype DT>
hipError_t launch(const WeighArgs &a, hipStream_t stream) {
    switch (a.head_dim) {
    case 64: return launch<DT, 64>(a, stream);
    case 128: return launch<DT, 128>(a, stream);
    default: return launch<DT, 256>(a, stream);
    }
}

}  // namespace

hipError_t launch_key_weights(const WeighArgs &a, knn_dtype dtype, hipStream_t stream) {
    return dtype == KNN_BF16 ? launch<KNN_BF16>(a, stream) : launch<KNN_F16>(a, stream);
}

}  // namespace knnlm
