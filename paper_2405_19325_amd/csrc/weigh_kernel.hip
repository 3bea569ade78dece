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
// stays within it until the end of a tile.  Weights are worked out as 2^(x c -
// lse c'), whose rounding is that of lse itself, and summed in 32 bits.
//
// What bounds it.  Up to 96 columns a key head (decoding, accepted paths): the
// bytes of the keys.  Each wave has a run of keys of its own, which come through
// LDS; 64 ragged sequences of 2,000 to 16,000 tokens, 8 key heads: 228 us for 1.22
// GB, 5.3 TB/s (189 without the masses, whose scattered writes of 64 bytes cost
// more than their share).  More columns: the exponential's 16 clocks and the 8 of
// a multiplication and a sum for 64 weights, beside 16 of the matrix cores.  A
// wave holds 64 keys in the registers that the instructions read, straight from
// memory, and the queries lie in LDS, read by all waves of the workgroup; 64 rows
// of 64 heads on 8 on 4 x 131,008 tokens: 564 us, 970 TFLOP/s (a large library
// product: 1,190); the matrix cores are busy half of the time.  Where a call has
// few tiles, waits are what it takes, and waves share a tile's columns: 40 rows of
// 64 heads on 8 over 30 tokens 15 us (28 where a tile is one wave's).
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
    constexpr int AHEAD = 4;  // loads of a thread on their way
    for (int e0 = static_cast<int>(threadIdx.x); e0 < padded * CHUNKS; e0 += AHEAD * THREADS) {
        u32x4_t v[AHEAD];
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) {
            const int e = e0 + u * THREADS, c = e / CHUNKS, chunk = e % CHUNKS, i = (c0 + c) / g;
            const int64_t source = c < n ? source_of(i) : -1;
            v[u] = u32x4_t{0, 0, 0, 0};
            if (source >= 0)
                v[u] = *reinterpret_cast<const u32x4_t *>(static_cast<const uint16_t *>(a.q) + source * a.q_row +
                                                          (h * g + (c0 + c - i * g)) * a.q_head + chunk * 8);
        }
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) {
            const int e = e0 + u * THREADS, c = e / CHUNKS;
            if (c < padded) st.q[c * CHUNKS + (e % CHUNKS ^ spread<D>(c))] = v[u];
        }
    }
}

// Which of 64 keys a column of this row sees, as bits: the first of them is the
// sequence's draft d0 (a cached one where negative, and no less than -64).
__device__ __forceinline__ uint64_t seen_of(const WeighArgs &a, const Tile &t, int row, int d0) {
    auto first_bits = [](int n) { return n <= 0 ? uint64_t{0} : n >= 64 ? ~uint64_t{0} : (uint64_t{1} << n) - 1; };
    if (row == kNobody) return 0;
    if (a.tree_mask == nullptr) return first_bits(row - d0 + 1);
    const uint32_t *words = a.tree_mask + (t.r0 + row) * a.mask_words;
    const int from = d0 < 0 ? 0 : d0, last = static_cast<int>(a.mask_words) - 1;  // (at most 2^28)
    uint32_t w[3];
#pragma unroll
    for (int i = 0; i < 3; ++i) {
        const int at = (from >> 5) + i;
        w[i] = words[at < last ? at : last];
        w[i] = at <= last ? w[i] : 0u;
    }
    const int off = from & 31;
    uint64_t bits = (w[0] | static_cast<uint64_t>(w[1]) << 32) >> off;
    if (off != 0) bits |= static_cast<uint64_t>(w[2]) << (64 - off);
    if (d0 >= 0) return bits;
    return d0 <= -64 ? ~uint64_t{0} : bits << -d0 | first_bits(-d0);
}

// SHARED: where a workgroup has fewer tiles than waves, several of these share a
// tile's columns; half as many waves, with the registers of two.
template <knn_dtype DT, int D, int WAVES, bool SHARED>
__global__ __launch_bounds__(WAVES * kWave, SHARED ? WAVES / 4 : 4) void k_key_weights(WeighArgs a, int most) {
    using Sh = Shape<D>;
    constexpr int KK = Sh::KK, B = Sh::B, THREADS = WAVES * kWave;
    extern __shared__ __align__(16) u32x4_t lds[];
    __shared__ int64_t sums[WAVES];
    __shared__ int64_t found[2];
    __shared__ float parts_of[SHARED ? WAVES : 1][kWave];
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
            auto put = [&](int64_t place, int j, float drawn, float mass) {
                a.mass[place] = drawn + a.decay * mass;
                if (j >= length && a.key_positions != nullptr)
                    a.key_positions[place] = a.positions != nullptr ? a.positions[t.r0 + (j - length)] : j;
            };
            // Rounds of one tile a wave, with the columns once more each; one round of all tiles where they fit LDS.
            const int step = cols > most ? WAVES : tile1 - tile0;
            for (int round = tile0; round < tile1; round += step) {
                const int stop = step < tile1 - round ? round + step : tile1;
                int share_log2 = 0;
                if constexpr (SHARED)
                    while (2 * (stop - round) << share_log2 <= WAVES) ++share_log2;
                const int pace = WAVES >> share_log2, share = wave & ((1 << share_log2) - 1);
                float sum[B] = {};
                for (int c0 = 0; c0 < cols; c0 += most) {
                    const int n = cols - c0 < most ? cols - c0 : most, padded = (n + 15) & ~15;
                    __syncthreads();
                    stage<D, THREADS>(a, t, st, h, g, c0, n, padded);
                    __syncthreads();
                    // The pages of this wave's next tiles: block b of the i-th in lane i B + b, or -1.
                    constexpr int AHEAD = kWave / B;
                    int32_t pages = 0;
                    for (int tile = round + (wave >> share_log2), i = 0; tile < stop; tile += pace, ++i) {
                        const int block0 = tile * B, first = i % AHEAD * B;
                        if (first == 0) {
                            const int block = (tile + lane / B * pace) * B + lane % B;
                            pages = table[min(block, last_block) << 4 >> a.cache.page_log2];
                            pages = pages >= 0 && pages < a.cache.n_pages ? pages : -1;
                        }
                        // Each quarter of the wave has a block's masses.
                        const int j0 = tile * Sh::KEYS, part = 16 * (quad & (B - 1)) + col;
                        const int j = static_cast<int>(static_cast<uint32_t>(j0) + part);
                        const int32_t p = __shfl(pages, first + (quad & (B - 1)));
                        const bool mine = quad < B && part < total_keys - j0 && p >= 0;
                        const int64_t place = ((static_cast<int64_t>(p) * a.kv_heads + h) << a.cache.page_log2) + (j & in_page);
                        float mass = 0.0f;
                        if (mine && j < length && a.decay != 0.0f && c0 + most >= cols && (!SHARED || share_log2 == 0)) mass = a.mass[place];
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
                        bool plain = length - j0 >= Sh::KEYS;  // (a length may be all that 31 bits hold)
                        if (plain) {
#pragma unroll 1
                            for (int c = 16 * share; c < padded; c += 16 << share_log2) {
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
#pragma unroll
                            for (int b = 0; b < B; ++b) w[b] = 0.0f;
#pragma unroll 1
                            for (int c = 16 * share; c < padded; c += 16 << share_log2) {
                                uint64_t seen[4];
                                u32x4_t q[KK];
#pragma unroll
                                for (int r = 0; r < 4; ++r) seen[r] = seen_of(a, t, st.row[c + 4 * quad + r], max(j0 - length, -64)) >> col;
#pragma unroll
                                for (int kk = 0; kk < KK; ++kk)
                                    q[kk] = st.q[(c + col) * (D / 8) + ((4 * kk + quad) ^ spread<D>(col))];
#pragma unroll
                                for (int b = 0; b < B; ++b) {  // (a block at a time, to spare registers)
                                    f32x4_t x{0, 0, 0, 0};
#pragma unroll
                                    for (int kk = 0; kk < KK; ++kk) x = mfma16<DT>(q[kk], k[b][kk], x);
#pragma unroll
                                    for (int r = 0; r < 4; ++r) {
                                        const float e = __builtin_amdgcn_exp2f(fmaf(x[r], c2, -st.lse2[c + 4 * quad + r]));
                                        w[b] += (seen[r] >> 16 * b & 1u) != 0u ? e : 0.0f;
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
                        if (SHARED && share_log2 > 0) {  // (one tile a wave: the parts are joined in a fixed order)
                            parts_of[wave][lane] = drawn;
                            continue;
                        }
                        if (mine) put(place, j, drawn, mass);
                    }
                    if (!SHARED || share_log2 == 0 || c0 + most < cols) continue;
                    __syncthreads();
                    const int tile = round + (wave >> share_log2), j0 = tile * Sh::KEYS, part = 16 * quad + col;
                    if (share > 0 || tile >= stop || quad >= B || part >= total_keys - j0) continue;
                    const int j = static_cast<int>(static_cast<uint32_t>(j0) + part);
                    const int64_t place = place_of(a.cache, a.kv_heads, s, h, j);
                    if (place < 0) continue;
                    float drawn = parts_of[wave][lane];
                    for (int w = 1; w < 1 << share_log2; ++w) drawn += parts_of[wave + w][lane];
                    put(place, j, drawn, j < length && a.decay != 0.0f ? a.mass[place] : 0.0f);
                }
            }
        }
    }
}

// Four bytes a lane into LDS, lane l's at lds + 4 l (as load_to_lds_16).
__device__ __forceinline__ void load_to_lds_4(const void *src, uint32_t lds) {
    asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dword %0, off" ::"v"(src), "s"(lds));
}

constexpr int kRing = 4;          // stages of a wave
constexpr int kStageBytes = 8192;  // of keys
constexpr int kStageOps = 9;       // loads of a stage: 8 of keys, 1 of masses

// Few columns, NT x 16 at most: the bytes of the keys are the bound.  Each wave
// has a run of stages of its own, and their keys on the way to its ring in LDS
// up to three stages ahead, a row's bytes by lanes side by side and past the
// caches (a plain read of 4 KiB pieces in that order: 6.8 TB/s; in the order of
// the instructions' registers 5.9).  The columns' queries stay in registers.
template <knn_dtype DT, int D, int NT>
__global__ __launch_bounds__(4 * kWave, 1) void k_key_weights_few(WeighArgs a) {
    constexpr int KK = D / 32, ROW = 2 * D, KEYS = kStageBytes / ROW, B = KEYS / 16;
    constexpr int LANES = D / 8, PER = kWave / LANES;  // lanes of a row, rows of a load
    __shared__ __align__(16) u32x4_t ring[4][kRing][kStageBytes / 16];
    __shared__ float masses[4][kRing][kWave];
    const int tid = static_cast<int>(threadIdx.x), lane = tid & (kWave - 1);
    const int wave = __builtin_amdgcn_readfirstlane(tid / kWave);
    const int col = lane & 15, quad = lane >> 4;
    const int g = a.q_heads / a.kv_heads;
    const float c2 = a.scale * kLog2e;
    const uint32_t ring_at = __builtin_amdgcn_readfirstlane(lds_offset(ring[wave][0]));
    const uint32_t masses_at = __builtin_amdgcn_readfirstlane(
        static_cast<uint32_t>(reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) float *)masses[wave][0])));

    // The stages of all sequences and heads lie one behind the other; this wave
    // takes those that begin in its share.
    const int64_t per = (a.S + kWave - 1) / kWave, s_lo = lane * per < a.S ? lane * per : a.S;
    const int64_t s_hi = s_lo + per < a.S ? s_lo + per : a.S;
    auto stages_of = [&](int64_t s) {
        const Tile t = tile_of(a, s);
        return t.n == 0 ? 0 : tiles_of(t.total, KEYS) * a.kv_heads;
    };
    int64_t mine = 0;
    for (int64_t s = s_lo; s < s_hi; ++s) mine += stages_of(s);
    int64_t upto = mine;
#pragma unroll
    for (int off = 1; off < kWave; off *= 2) {
        const int64_t o = __shfl_up(upto, off);
        if (lane >= off) upto += o;
    }
    // (the same in all lanes: kept in scalar registers)
    auto uniform = [](int64_t x) {
        return static_cast<int64_t>(static_cast<uint32_t>(__builtin_amdgcn_readfirstlane(static_cast<int>(x)))) |
               static_cast<int64_t>(__builtin_amdgcn_readfirstlane(static_cast<int>(x >> 32))) << 32;
    };
    const int64_t all = uniform(__shfl(upto, kWave - 1));
    const int64_t waves = static_cast<int64_t>(gridDim.x) * 4, self = static_cast<int64_t>(blockIdx.x) * 4 + wave;
    const int64_t from = all / waves * self + all % waves * self / waves;
    const int64_t to = all / waves * (self + 1) + all % waves * (self + 1) / waves;
    if (from >= to) return;
    int64_t s = s_lo, base = upto - mine;
    const bool has = from >= base && from < upto;  // (one lane)
    if (has)
        for (; s < s_hi; ++s) {
            const int64_t n = stages_of(s);
            if (from < base + n) break;
            base += n;
        }
    const int owner = __ffsll(static_cast<unsigned long long>(__ballot(has))) - 1;
    s = uniform(__shfl(s, owner)), base = uniform(__shfl(base, owner));

    for (; s < a.S && base < to; ++s) {
        const Tile t = tile_of(a, s);
        if (t.n == 0) continue;
        const int64_t stages = uniform(tiles_of(t.total, KEYS)), each = stages * a.kv_heads;
        const int64_t first = from > base ? from - base : 0, last = to - base < each ? to - base : each;
        base += each;
        const int cols = t.n * g, total_keys = static_cast<int>(t.total), last_block = (total_keys - 1) >> 4;
        const int length = static_cast<int>(t.length < t.total ? t.length : t.total);
        const int in_page = (1 << a.cache.page_log2) - 1;
        const int32_t *table = a.cache.pages + s * a.cache.table_width;
        for (int64_t at = first; at < last;) {
            const int h = static_cast<int>(uniform(at / stages));
            const int st0 = static_cast<int>(at - h * stages);
            const int n = static_cast<int>((last - h * stages < stages ? last - h * stages : stages) - st0);
            at += n;
            auto page_of = [&](int block) {
                const int32_t page = load_scalar_i32(table + ((min(block, last_block) << 4) >> a.cache.page_log2));
                return page >= 0 && page < a.cache.n_pages ? page : -1;
            };
            // Stage i of the run into its place of the ring.
            auto fill = [&](int i) {
                const uint32_t lds = ring_at + static_cast<uint32_t>(i % kRing) * kStageBytes;
                int64_t mass_at = 0;
#pragma unroll
                for (int b = 0; b < B; ++b) {
                    const int block = (st0 + i) * B + b, page = page_of(block);
                    const int64_t at_page = static_cast<int64_t>(page < 0 ? 0 : page) * a.kv_heads + h;
                    // (of the last block, the places behind the last key are read as well, whatever they hold)
                    const int64_t place = (at_page << a.cache.page_log2) + ((min(block, last_block) << 4) & in_page);
                    const char *from_block = static_cast<const char *>(a.k_cache) + place * ROW;
#pragma unroll
                    for (int j = 0; j < 16 / PER; ++j) {
                        const int r = j * PER + lane / LANES;
                        load_to_lds_16_nt(from_block, r * ROW + 16 * ((lane % LANES) ^ spread<D>(r)),
                                          lds + b * 16 * ROW + j * 1024);
                    }
                    if (b == 0 || quad == b) mass_at = place;
                }
                load_to_lds_4(a.mass + mass_at + col, masses_at + static_cast<uint32_t>(i % kRing) * (4 * kWave));
            };
#pragma unroll
            for (int i = 0; i < kRing - 1; ++i)
                if (i < n) fill(i);
            // The columns: lane = (column, 8 elements a quad) of the queries, four columns of the sums.
            u32x4_t q[NT][KK];
            f32x4_t lse2[NT];
            auto source_of = [&](int c) -> int64_t {
                if (c >= cols) return -1;
                const int64_t row = t.r0 + c / g, source = a.source_rows != nullptr ? a.source_rows[row] : row;
                return source < a.source_count ? source : -1;
            };
#pragma unroll
            for (int m = 0; m < NT; ++m) {
                if (NT > 1 && 32 * (m / 2) >= cols) break;  // (in pairs: zeros where the second one has no column)
                const int c = 16 * m + col;
                const int64_t source = source_of(c);
                const uint16_t *from_q = static_cast<const uint16_t *>(a.q) + (source < 0 ? 0 : source) * a.q_row +
                                         (h * g + (c < cols ? c % g : 0)) * a.q_head;
#pragma unroll
                for (int kk = 0; kk < KK; ++kk) {
                    q[m][kk] = *reinterpret_cast<const u32x4_t *>(from_q + 32 * kk + 8 * quad);
                    if (source < 0) q[m][kk] = u32x4_t{0, 0, 0, 0};
                }
                const float l = source < 0 ? INFINITY : a.lse[source * a.q_heads + h * g + c % g];
                const float l2 = isfinite(l) ? l * kLog2e : INFINITY;
#pragma unroll
                for (int r = 0; r < 4; ++r) lse2[m][r] = __shfl(l2, 4 * quad + r);
            }

            for (int i = 0; i < n; ++i) {
                asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // the stage that is filled next has been read
                if (i + kRing - 1 < n) {
                    fill(i + kRing - 1);
                    // This stage's loads are done when no more are under way than those of the later ones.
                    asm volatile("s_waitcnt vmcnt(%0)" ::"n"((kRing - 1) * kStageOps) : "memory");
                } else {
                    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
                }
                const uint32_t lds = ring_at + static_cast<uint32_t>(i % kRing) * kStageBytes;
                const int j0 = (st0 + i) * KEYS;
                float w[B];
                auto key = [&](int b, int kk) {
                    return *reinterpret_cast<const __attribute__((address_space(3))) u32x4_t *>(
                        static_cast<uintptr_t>(lds + (16 * b + col) * ROW + 16 * ((4 * kk + quad) ^ spread<D>(col))));
                };
                bool plain = length - j0 >= KEYS;  // (a length may be all that 31 bits hold)
                if (plain) {
                    // Two column tiles and all blocks at a time: as many chains of matrix instructions beside each other.
                    constexpr int M = NT > 1 ? 2 : 1;
                    u32x4_t k[B][KK];
                    bool odd = false;
#pragma unroll
                    for (int b = 0; b < B; ++b) {
                        w[b] = 0.0f;
#pragma unroll
                        for (int kk = 0; kk < KK; ++kk) k[b][kk] = key(b, kk);
                    }
#pragma unroll
                    for (int m0 = 0; m0 < NT; m0 += M) {
                        if (16 * m0 >= cols) break;
                        f32x4_t x[M][B];
#pragma unroll
                        for (int m = 0; m < M; ++m)
#pragma unroll
                            for (int b = 0; b < B; ++b) x[m][b] = f32x4_t{0, 0, 0, 0};
#pragma unroll
                        for (int kk = 0; kk < KK; ++kk)
#pragma unroll
                            for (int m = 0; m < M; ++m)
#pragma unroll
                                for (int b = 0; b < B; ++b) x[m][b] = mfma16<DT>(q[m0 + m][kk], k[b][kk], x[m][b]);
#pragma unroll
                        for (int m = 0; m < M; ++m)
#pragma unroll
                            for (int b = 0; b < B; ++b) {
                                float e[4];
#pragma unroll
                                for (int r = 0; r < 4; ++r) e[r] = __builtin_amdgcn_exp2f(fmaf(x[m][b][r], c2, -lse2[m0 + m][r]));
                                w[b] += (e[0] + e[1]) + (e[2] + e[3]);
                            }
                    }
#pragma unroll
                    for (int b = 0; b < B; ++b) odd = odd || w[b] != w[b];
                    // Keys that are not finite: whose they are is looked at column by column.
                    plain = !__any(odd);
                }
                if (!plain) {
#pragma unroll
                    for (int b = 0; b < B; ++b) w[b] = 0.0f;
#pragma unroll
                    for (int m = 0; m < NT; ++m) {
                        if (16 * m >= cols) break;
                        uint64_t seen[4];
#pragma unroll
                        for (int r = 0; r < 4; ++r) {
                            const int row = lse2[m][r] < INFINITY ? (16 * m + 4 * quad + r) / g : kNobody;
                            seen[r] = seen_of(a, t, row, max(j0 - length, -64)) >> col;
                        }
#pragma unroll
                        for (int b = 0; b < B; ++b) {
                            f32x4_t x{0, 0, 0, 0};
#pragma unroll
                            for (int kk = 0; kk < KK; ++kk) x = mfma16<DT>(q[m][kk], key(b, kk), x);
#pragma unroll
                            for (int r = 0; r < 4; ++r) {
                                const float e = __builtin_amdgcn_exp2f(fmaf(x[r], c2, -lse2[m][r]));
                                w[b] += (seen[r] >> 16 * b & 1u) != 0u ? e : 0.0f;
                            }
                        }
                    }
                }
#pragma unroll
                for (int b = 0; b < B; ++b) {
                    w[b] += __shfl_xor(w[b], 16);
                    w[b] += __shfl_xor(w[b], 32);
                }
                // Each quarter of the wave writes a block.
                float drawn = w[0];
                int page = page_of((st0 + i) * B);
#pragma unroll
                for (int b = 1; b < B; ++b) {
                    const int other = page_of((st0 + i) * B + b);
                    drawn = quad == b ? w[b] : drawn, page = quad == b ? other : page;
                }
                const float mass = masses[wave][i % kRing][lane];
                const int part = 16 * quad + col, j = static_cast<int>(static_cast<uint32_t>(j0) + part);
                if (quad < B && part < total_keys - j0 && page >= 0) {
                    const int64_t place = ((static_cast<int64_t>(page) * a.kv_heads + h) << a.cache.page_log2) + (j & in_page);
                    // (written through, as an agent's: paths over 8 x 100,000 tokens 334 us, 346 by way of the caches' write-back)
                    __hip_atomic_store(a.mass + place, drawn + (j < length && a.decay != 0.0f ? a.decay * mass : 0.0f),
                                       __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
                    if (j >= length && a.key_positions != nullptr)
                        a.key_positions[place] = a.positions != nullptr ? a.positions[t.r0 + (j - length)] : j;
                }
            }
        }
    }
}

template <knn_dtype DT, int D, int NT>
void launch_few(const WeighArgs &a, hipStream_t stream) {
    const double stages = static_cast<double>(a.S) * a.kv_heads * static_cast<double>(tiles_of(a.max_keys, kStageBytes / (2 * D)));
    const int64_t blocks = stages < 4 * kCus ? (static_cast<int64_t>(stages) + 3) / 4 : kCus;
    k_key_weights_few<DT, D, NT><<<dim3(static_cast<unsigned>(blocks)), 4 * kWave, 0, stream>>>(a);
}

template <knn_dtype DT, int D, int WAVES, bool SHARED>
void launch(const WeighArgs &a, int most, double tiles, hipStream_t stream) {
    const size_t lds = static_cast<size_t>(most) * (Shape<D>::ROW + 8);
    const size_t fit = (size_t{156} << 10) / (lds + 1024);
    const int64_t room = fit * WAVES > 16 ? 16 / WAVES : fit < 1 ? 1 : static_cast<int64_t>(fit);  // workgroups of a CU
    // (A workgroup a tile where there are so few: another head's queries are another wait.)
    const int64_t most_blocks = kCus * room, blocks = tiles < most_blocks ? static_cast<int64_t>(tiles) : most_blocks;
    k_key_weights<DT, D, WAVES, SHARED><<<dim3(static_cast<unsigned>(blocks)), WAVES * kWave, lds, stream>>>(a, most);
}

template <knn_dtype DT, int D>
hipError_t launch(const WeighArgs &a, hipStream_t stream) {
    const int64_t cols = (a.max_rows * (a.q_heads / a.kv_heads) + 15) / 16 * 16;
    const int most = static_cast<int>(cols < Shape<D>::MOST ? cols : Shape<D>::MOST);
    // Waves of their own while the columns' queries fit the registers; measured on 4 x 65,536 tokens, 64 heads on 8: 8
    // columns 96 us, 117 the other way; 96 columns 117 and 128; at head_dim 256 183 and 210, 195 and 221; at 64, where a
    // column tile does half the work for the same exponentials, 55 and 62, but 75 and 65 at 48 columns.
    if (most <= 16) launch_few<DT, D, 1>(a, stream);
    else if (most <= 32) launch_few<DT, D, 2>(a, stream);
    else if (D > 64 && most <= 96) launch_few<DT, (D > 64 ? D : 128), 6>(a, stream);
    else {
        const double tiles =
            static_cast<double>(a.S) * a.kv_heads * static_cast<double>(tiles_of(a.max_keys, Shape<D>::KEYS));
        // Eight waves that share a tile's columns while there is at most a tile a CU, or so many that their columns' queries
        // take over 40 KiB and each has several of its own: the waits of one tile behind the other weigh more than half as
        // many waves.  Measured in turn, us, this way and the other: 64 rows of 64 heads on 8 over 2 x 300 tokens 18 and 38, as
        // trees 22 and 59; 8 x 400 27 and 46; 8 x 900 34 and 48; 8 x 7,000 82 and 93, 4 x 130,000 556 and 548; at head_dim 64
        // 8 x 900 35 and 40, 8 x 2,000 46 and 41; at 256 8 x 900 54 and 65, 8 x 2,000 99 and 89.  Of 160 columns, 8 x 1,500
        // tokens on 2 key heads: 24 and 21.  1,024 columns on 2 x 30,000: 215 and 203.
        const int several = most * Shape<D>::ROW <= 40960 ? 1 : D == 64 ? 6 : D == 256 || cols > Shape<D>::MOST ? 8 : 32;
        if (tiles <= several * kCus) launch<DT, D, 8, true>(a, most, tiles, stream);
        // Four waves a workgroup while four of these fit a CU's LDS with their queries; else eight, or all sixteen.
        else if (most * 4 <= Shape<D>::MOST) launch<DT, D, 4, false>(a, most, tiles, stream);
        else if (most * 2 <= Shape<D>::MOST) launch<DT, D, 8, false>(a, most, tiles, stream);
        else launch<DT, D, 16, false>(a, most, tiles, stream);
    }
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
