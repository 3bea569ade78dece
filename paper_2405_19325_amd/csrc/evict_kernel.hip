// Eviction of the tokens of little weight from a paged cache.
//
// Each key head of a sequence keeps its own tokens: the first `budget` of an
// order by (protected, mass, lower index).  The kept ones that lie behind the
// budget go, in order, to the places before it that are given up, so nothing
// else moves: sources and targets are apart, and no move waits for another.
//
// The order as one number: the bits of a float, with the sign turned so that
// they order like the values, lie in 1 .. 0xff800000 (0x007fffff is -infinity, 1
// NaN).  With no more protected tokens than the budget these are 0xffffffff,
// and all stay; with more, all others are 0 and none does.  The border is the
// budget-th largest number; of those equal to it the first ones stay.
//
// Heads of up to 8,192 tokens: a workgroup has them in registers and finds the
// border two bits a round, by counting.  Longer ones are cut into segments,
// a workgroup each, which ends at the budget so that a segment holds sources or
// targets only.  All of a head's workgroups look at the same 4,096 tokens,
// whose order gives two numbers that the border lies between but for one head
// in thousands; each counts its segment's numbers above, at and below these and
// lists those between.  A second launch finds the border in the few that are
// listed (or, where it lies elsewhere, in all), and with it each segment's
// share of the moves, which a last one makes.
#include "lm_device.h"

namespace knnlm {

namespace {

constexpr int kThreads = 1024;
constexpr int kWaves = kThreads / kWave;
constexpr int kHeld = 8;                    // tokens of a thread
constexpr int kChunk = kHeld * kThreads;
constexpr int kSegments = 64;               // of a head, about
constexpr int kSamples = 4;                 // of a thread
constexpr int64_t kGrid = int64_t{1} << 20;  // heads at once

// A number that orders like x, NaN first.
__device__ __forceinline__ uint32_t order_of(float x) {
    if (x != x) return 1u;
    const uint32_t b = __float_as_uint(x + 0.0f);  // one zero
    return b ^ ((b >> 31) != 0 ? 0xffffffffu : 0x80000000u);
}

// LDS of the collective steps.  Their words alternate, so that a step may be
// called again without a barrier.
struct Shared {
    uint32_t part[2][4 * kWaves];
};

// The sums over the workgroup of N numbers that each wave has (the same in all
// of its lanes).
template <int N>
__device__ __forceinline__ void block_sums(uint32_t (&v)[N], Shared &sh, int &turn) {
    static_assert(N <= 4, "a row of 16 lanes each");
    const int lane = static_cast<int>(threadIdx.x) & (kWave - 1), wave = static_cast<int>(threadIdx.x) / kWave;
    turn ^= 1;
    uint32_t mine = v[0];
#pragma unroll
    for (int i = 1; i < N; ++i) mine = lane == i ? v[i] : mine;
    if (lane < N) sh.part[turn][lane * kWaves + wave] = mine;
    __syncthreads();
    uint32_t x = lane < N * kWaves ? sh.part[turn][lane] : 0u;  // 16 waves: a row of lanes a number
    x += dpp_u32<0xB1>(0u, x);
    x += dpp_u32<0x4E>(0u, x);
    x += dpp_u32<0x141>(0u, x);
    x += dpp_u32<0x140>(0u, x);
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = readlane_u32(x, 16 * i);
}

__device__ __forceinline__ uint32_t votes(bool flag) { return static_cast<uint32_t>(__popcll(__ballot(flag))); }

// The rank-th largest (from 1) of what `count` counts: count(a, b, c, v) sets v
// to how many numbers of this wave are at least a, b and c (a < b < c).  Where
// a count is the rank itself, its bound serves as well as the number.
template <class Count>
__device__ __forceinline__ uint32_t border_of(uint32_t rank, Count count, Shared &sh, int &turn, bool exact) {
    uint32_t border = 0;
    for (int bit = 30; bit >= 0; bit -= 2) {
        uint32_t v[3];
        count(border | 1u << bit, border | 2u << bit, border | 3u << bit, v);
        block_sums(v, sh, turn);
        const uint32_t digit = v[2] >= rank ? 3u : v[1] >= rank ? 2u : v[0] >= rank ? 1u : 0u;
        border |= digit << bit;
        if (!exact && (v[0] == rank || v[1] == rank || v[2] == rank)) break;
    }
    return border;
}

// What comes before this wave's counts of each row of threads, rows first and
// waves within them, and all of them.  `ranks`: kHeld x kWaves words.
__device__ __forceinline__ void before(uint32_t *ranks, const uint32_t (&mine)[kHeld], uint32_t (&sum)[kHeld], uint32_t &total) {
    static_assert(kHeld * kWaves == 2 * kWave, "two a lane");
    const int lane = static_cast<int>(threadIdx.x) & (kWave - 1);
    const int wave = __builtin_amdgcn_readfirstlane(static_cast<int>(threadIdx.x) / kWave);
    __syncthreads();
    uint32_t v = mine[0];
#pragma unroll
    for (int r = 1; r < kHeld; ++r) v = lane == r ? mine[r] : v;
    if (lane < kHeld) ranks[lane * kWaves + wave] = v;
    __syncthreads();
    const uint32_t lo = ranks[2 * lane], hi = ranks[2 * lane + 1];
    const uint32_t upto = wave_incl_scan_u32(lo + hi, lane);
    const uint32_t mine_first = upto - lo - hi + ((wave & 1) != 0 ? lo : 0u);
#pragma unroll
    for (int r = 0; r < kHeld; ++r) sum[r] = readlane_u32(mine_first, (r * kWaves + wave) >> 1);
    total = readlane_u32(upto, kWave - 1);
}

// A head of a sequence and what becomes of it.
struct Head {
    int64_t s;
    int h;
    int64_t n, keep;  // tokens; those that stay
    int64_t recent_from;
    bool leave;       // left as it is

    __device__ __forceinline__ int64_t place(const EvictArgs &a, int64_t j) const {
        return place_of(a.cache, a.kv_heads, s, h, j);
    }
    // Tokens j[0], j[1], ... (all of them there): their numbers by mass alone, and as bits which are protected.  The
    // loads of all are on their way together.
    template <int N>
    __device__ __forceinline__ void orders(const EvictArgs &a, const int (&j)[N], uint32_t (&o)[N], uint32_t &fixed) const {
        const int32_t *table = a.cache.pages + s * a.cache.table_width;
        const int in_page = (1 << a.cache.page_log2) - 1;
        int64_t at[N];
        float m[N];
        int32_t p[N];
#pragma unroll
        for (int i = 0; i < N; ++i)
            at[i] = ((static_cast<int64_t>(table[j[i] >> a.cache.page_log2]) * a.kv_heads + h) << a.cache.page_log2) + (j[i] & in_page);
#pragma unroll
        for (int i = 0; i < N; ++i) {
            m[i] = a.mass[at[i]];
            p[i] = a.key_positions != nullptr ? a.key_positions[at[i]] : j[i];
        }
        fixed = 0;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            o[i] = order_of(m[i]);
            fixed |= p[i] < a.sinks || p[i] >= recent_from ? 1u << i : 0u;
        }
    }
    // The numbers themselves, where there are no more protected ones than the budget (few), or more.
    template <int N>
    __device__ __forceinline__ void numbers(const EvictArgs &a, const int (&j)[N], bool few, uint32_t (&o)[N]) const {
        uint32_t fixed;
        orders(a, j, o, fixed);
#pragma unroll
        for (int i = 0; i < N; ++i) o[i] = number(o[i], (fixed >> i & 1u) != 0u, few);
    }
    __device__ static __forceinline__ uint32_t number(uint32_t order, bool fixed, bool few) {
        return few ? (fixed ? 0xffffffffu : order) : (fixed ? order : 0u);
    }
};

// For all threads of a workgroup together.
__device__ __forceinline__ Head head_of(const EvictArgs &a, int64_t pair) {
    Head x;
    x.s = pair / a.kv_heads;
    x.h = static_cast<int>(pair - x.s * a.kv_heads);
    const int64_t len = a.cache_lens[x.s], budget = a.budgets[x.s];
    const int64_t room = a.cache.table_width << a.cache.page_log2, limit = a.max_keys < room ? a.max_keys : room;
    const int64_t n = len < 0 ? 0 : len;
    x.recent_from = (a.next_positions != nullptr ? a.next_positions[x.s] : len) - a.recent;
    x.leave = budget < 0 || budget >= n || n > limit;
    if (!x.leave) {
        bool whole = true;
        const int64_t entries = (n + (int64_t{1} << a.cache.page_log2) - 1) >> a.cache.page_log2;
        const int32_t *table = a.cache.pages + x.s * a.cache.table_width;
        for (int64_t e = threadIdx.x; e < entries; e += 4 * kThreads) {
            int32_t page[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) page[u] = table[e + u * kThreads < entries ? e + u * kThreads : e];
#pragma unroll
            for (int u = 0; u < 4; ++u) whole = whole && page[u] >= 0 && page[u] < a.cache.n_pages;
        }
        x.leave = __syncthreads_or(!whole) != 0;
    }
    x.n = n < limit ? n : limit;
    x.keep = x.leave ? x.n : budget;
    return x;
}

__device__ __forceinline__ void put_len(const EvictArgs &a, const Head &x) {
    a.new_lens[x.s] = x.leave ? a.cache_lens[x.s] : static_cast<int32_t>(x.keep);
}

// The ledger's entry of a token that stays where it is, where the ledger of
// afterwards is another.
__device__ __forceinline__ void carry(const EvictArgs &a, int64_t at) {
    if (a.mass_out != a.mass) a.mass_out[at] = a.mass[at];
    if (a.positions_out != a.key_positions) a.positions_out[at] = a.key_positions[at];
}

__device__ __forceinline__ void carry_all(const EvictArgs &a, const Head &x, int64_t from, int64_t to) {
    if (a.mass_out == a.mass && a.positions_out == a.key_positions) return;
    for (int64_t j = from + threadIdx.x; j < to; j += kThreads) {
        const int64_t at = x.place(a, j);
        if (at >= 0) carry(a, at);
    }
}

// Moves that a wave makes at once: four loads of 16 bytes a lane of either cache.
constexpr int batch_of(int chunks) { return chunks > 0 ? 4 * kWave / chunks : 16; }

// Up to 64 moves by a wave, one a lane: keys, values and the ledger's entries.
template <int CHUNKS>  // of 16 bytes in a head; 0: any number of elements
__device__ __forceinline__ void move(const EvictArgs &a, int64_t from, int64_t to, int count) {
    const int lane = static_cast<int>(threadIdx.x) & (kWave - 1);
    if (lane < count) {
        a.mass_out[to] = a.mass[from];
        if (a.key_positions != nullptr) a.positions_out[to] = a.key_positions[from];
    }
    const int from_lo = static_cast<int>(from), from_hi = static_cast<int>(from >> 32);
    const int to_lo = static_cast<int>(to), to_hi = static_cast<int>(to >> 32);
    auto of = [](int lo, int hi, int m) {
        return static_cast<int64_t>(static_cast<uint32_t>(__shfl(lo, m))) | static_cast<int64_t>(__shfl(hi, m)) << 32;
    };
    if constexpr (CHUNKS > 0) {
        constexpr int AT_ONCE = kWave / CHUNKS, UNROLL = 4;
        const int mine = lane / CHUNKS, chunk = lane % CHUNKS;
        u32x4_t *k = static_cast<u32x4_t *>(a.k_cache), *v = static_cast<u32x4_t *>(a.v_cache);
        for (int m = 0; m < count; m += AT_ONCE * UNROLL) {
            u32x4_t kr[UNROLL], vr[UNROLL];
#pragma unroll
            for (int u = 0; u < UNROLL; ++u) {
                const int i = m + u * AT_ONCE + mine;
                const int64_t src = of(from_lo, from_hi, i < count ? i : 0) * CHUNKS + chunk;
                kr[u] = k[src], vr[u] = v[src];
            }
#pragma unroll
            for (int u = 0; u < UNROLL; ++u) {
                const int i = m + u * AT_ONCE + mine;
                const int64_t dst = of(to_lo, to_hi, i < count ? i : 0) * CHUNKS + chunk;
                if (i < count) k[dst] = kr[u], v[dst] = vr[u];
            }
        }
    } else {
        uint16_t *k = static_cast<uint16_t *>(a.k_cache), *v = static_cast<uint16_t *>(a.v_cache);
        for (int m = 0; m < count; ++m) {
            const int64_t src = of(from_lo, from_hi, m) * a.head_dim, dst = of(to_lo, to_hi, m) * a.head_dim;
            for (int e = lane; e < a.head_dim; e += kWave) k[dst + e] = k[src + e], v[dst + e] = v[src + e];
        }
    }
}

// The moves that a head's workgroups found.
struct Moves {
    int32_t *count;  // [heads]
    int32_t *from;   // [heads][most] cache indices, then where to
    int64_t most;
};

// A head in a workgroup's registers.  `CHUNKS` as in move; MOVE: made here,
// else left to another launch.
template <bool MOVE, int CHUNKS>
__global__ __launch_bounds__(kThreads) void k_evict_held(EvictArgs a, Moves moves) {
    __shared__ Shared sh;
    __shared__ uint32_t ranks[kHeld * kWaves];
    __shared__ uint16_t lists[MOVE ? 2 : 1][MOVE ? kChunk / 2 : 1];  // sources, targets
    const int tid = static_cast<int>(threadIdx.x), lane = tid & (kWave - 1), wave = tid / kWave;
    const uint64_t under = (uint64_t{1} << lane) - 1;
    int turn = 0;
    for (int64_t pair = blockIdx.x; pair < a.S * a.kv_heads; pair += gridDim.x) {
        const Head x = head_of(a, pair);
        if (x.h == 0 && tid == 0) put_len(a, x);
        if (x.leave) {
            carry_all(a, x, 0, x.n);
            if (!MOVE && tid == 0) moves.count[pair] = 0;
            continue;
        }
        const int n = static_cast<int>(x.n), keep = static_cast<int>(x.keep);
        uint32_t order[kHeld], fixed, protects[1] = {0};
        int j[kHeld];
#pragma unroll
        for (int r = 0; r < kHeld; ++r) j[r] = r * kThreads + tid < n ? r * kThreads + tid : n - 1;
        x.orders(a, j, order, fixed);
#pragma unroll
        for (int r = 0; r < kHeld; ++r) protects[0] += votes(r * kThreads + tid < n && (fixed >> r & 1u) != 0u);
        block_sums(protects, sh, turn);
        const bool few = protects[0] <= static_cast<uint32_t>(keep);
#pragma unroll
        for (int r = 0; r < kHeld; ++r)  // 0 behind the last token
            order[r] = r * kThreads + tid < n ? Head::number(order[r], (fixed >> r & 1u) != 0u, few) : 0u;
        uint32_t border = 0xffffffffu, all[2] = {0, 0};  // at the border and above, above
        if (keep > 0) {
            border = border_of(
                keep,
                [&](uint32_t b0, uint32_t b1, uint32_t b2, uint32_t(&v)[3]) {
                    v[0] = v[1] = v[2] = 0;
#pragma unroll
                    for (int r = 0; r < kHeld; ++r) {
                        if (r * kThreads >= n) break;
                        v[0] += votes(order[r] >= b0);
                        v[1] += votes(order[r] >= b1);
                        v[2] += votes(order[r] >= b2);
                    }
                },
                sh, turn, false);
#pragma unroll
            for (int r = 0; r < kHeld; ++r) {
                all[0] += votes(order[r] >= border);
                all[1] += votes(order[r] > border);
            }
            block_sums(all, sh, turn);
        }
        uint32_t kept = 0;  // as bits
        if (keep > 0 && all[0] != static_cast<uint32_t>(keep)) {
            const uint32_t even = keep - all[1];  // of those at the border
            uint32_t mine[kHeld], sum[kHeld], total;
#pragma unroll
            for (int r = 0; r < kHeld; ++r) mine[r] = votes(order[r] == border);
            before(ranks, mine, sum, total);
#pragma unroll
            for (int r = 0; r < kHeld; ++r) {
                const uint32_t rank = sum[r] + static_cast<uint32_t>(__popcll(__ballot(order[r] == border) & under));
                kept |= order[r] > border || (order[r] == border && rank < even) ? 1u << r : 0u;
            }
        } else if (keep > 0) {
#pragma unroll
            for (int r = 0; r < kHeld; ++r) kept |= order[r] >= border ? 1u << r : 0u;
        }
        uint32_t mine[kHeld], sum[kHeld], total;
        uint64_t sources[kHeld], targets[kHeld];
#pragma unroll
        for (int r = 0; r < kHeld; ++r) {
            const int j = r * kThreads + tid;
            const bool k = (kept >> r & 1u) != 0u;
            sources[r] = __ballot(k && j >= keep);
            targets[r] = __ballot(!k && j < keep);
            mine[r] = static_cast<uint32_t>(__popcll(sources[r])) | static_cast<uint32_t>(__popcll(targets[r])) << 16;
            if (k && j < keep && (a.mass_out != a.mass || a.positions_out != a.key_positions)) carry(a, x.place(a, j));
        }
        before(ranks, mine, sum, total);
        total &= 0xffffu;
#pragma unroll
        for (int r = 0; r < kHeld; ++r) {
            const int j = r * kThreads + tid;
            const bool source = (sources[r] >> lane & 1u) != 0u, target = (targets[r] >> lane & 1u) != 0u;
            const uint32_t rs = (sum[r] & 0xffffu) + static_cast<uint32_t>(__popcll(sources[r] & under));
            const uint32_t rt = (sum[r] >> 16) + static_cast<uint32_t>(__popcll(targets[r] & under));
            if constexpr (MOVE) {
                if (source) lists[0][rs] = static_cast<uint16_t>(j);
                if (target) lists[1][rt] = static_cast<uint16_t>(j);
            } else {
                if (source) moves.from[pair * 2 * moves.most + rs] = j;
                if (target) moves.from[(pair * 2 + 1) * moves.most + rt] = j;
            }
        }
        if constexpr (MOVE) __syncthreads();
        if constexpr (MOVE) {
            constexpr int BATCH = batch_of(CHUNKS);
            for (uint32_t m = wave * BATCH; m < total; m += kWaves * BATCH) {
                const uint32_t i = lane < BATCH && m + lane < total ? m + lane : m;
                move<CHUNKS>(a, x.place(a, lists[0][i]), x.place(a, lists[1][i]),
                             static_cast<int>(total - m < BATCH ? total - m : BATCH));
            }
            __syncthreads();
        } else if (tid == 0) {
            moves.count[pair] = static_cast<int32_t>(total);
        }
    }
}

template <int CHUNKS>
__global__ __launch_bounds__(256) void k_evict_move(EvictArgs a, Moves moves) {
    const int lane = static_cast<int>(threadIdx.x) & (kWave - 1);
    for (int64_t pair = blockIdx.y; pair < a.S * a.kv_heads; pair += gridDim.y) {
        const int64_t s = pair / a.kv_heads;
        const int h = static_cast<int>(pair - s * a.kv_heads);
        const int64_t count = moves.count[pair];
        const int32_t *from = moves.from + pair * 2 * moves.most, *to = from + moves.most;
        constexpr int BATCH = batch_of(CHUNKS);
        for (int64_t m = (static_cast<int64_t>(blockIdx.x) * 4 + threadIdx.x / kWave) * BATCH; m < count;
             m += static_cast<int64_t>(gridDim.x) * 4 * BATCH) {
            const int64_t i = lane < BATCH && m + lane < count ? m + lane : m;
            move<CHUNKS>(a, place_of(a.cache, a.kv_heads, s, h, from[i]), place_of(a.cache, a.kv_heads, s, h, to[i]),
                         static_cast<int>(count - m < BATCH ? count - m : BATCH));
        }
    }
}

// What a segment's workgroup counted in the first launch.
struct Counts {
    uint32_t low, high;               // the two numbers, the same for all segments of a head
    uint32_t above, at_high, between, at_low;  // how many of the segment's are over `high`, at it, ...
    uint32_t fixed;
    uint32_t pad;
};

// The segments of a head: [0, keep) and [keep, n) in pieces of `size`.
struct Segments {
    int64_t size;
    int below, all;  // how many lie below the budget; all

    __device__ __forceinline__ Segments(const Head &x, int64_t size_) : size(size_) {
        below = static_cast<int>((x.keep + size - 1) / size);
        all = below + static_cast<int>((x.n - x.keep + size - 1) / size);
    }
    __device__ __forceinline__ int64_t begin(const Head &x, int w) const {
        return w < below ? w * size : x.keep + (w - below) * size;
    }
    __device__ __forceinline__ int64_t end(const Head &x, int w) const {
        const int64_t e = begin(x, w) + size, most = w < below ? x.keep : x.n;
        return e < most ? e : most;
    }
    __device__ __forceinline__ int of(const Head &x, int64_t j) const {
        return j < x.keep ? static_cast<int>(j / size) : below + static_cast<int>((j - x.keep) / size);
    }
};

constexpr int kMostSegments = kSegments + 2;

// The first launch over long heads: counts, and the numbers between, listed in
// the segment's part of `lists` [heads][max_keys].
__global__ __launch_bounds__(kThreads) void k_evict_count(EvictArgs a, Counts *counts, uint32_t *lists, int64_t size) {
    __shared__ Shared sh;
    __shared__ uint32_t listed;
    const int tid = static_cast<int>(threadIdx.x), lane = tid & (kWave - 1);
    int turn = 0;
    for (int64_t pair = blockIdx.x; pair < a.S * a.kv_heads; pair += gridDim.x) {
        const Head x = head_of(a, pair);
        const Segments seg(x, size);
        const int w = static_cast<int>(blockIdx.y);
        if (x.leave || w >= seg.all || x.keep == 0) continue;
        // One token of each of 4,096 equal pieces, at no regular distance.
        uint32_t sample[kSamples];
        constexpr int kAll = kSamples * kThreads;
        const int64_t some = x.n < kAll ? x.n : kAll;
        int which[kSamples];
#pragma unroll
        for (int r = 0; r < kSamples; ++r) {
            const int64_t i = r * kThreads + tid < some ? r * kThreads + tid : some - 1;
            const int64_t j0 = i * x.n / some, j1 = (i + 1) * x.n / some;
            uint32_t mix = static_cast<uint32_t>(i) * 2654435761u;
            mix ^= mix >> 15;
            which[r] = static_cast<int>(j0 + mix % static_cast<uint32_t>(j1 - j0));
        }
        x.numbers(a, which, true, sample);
#pragma unroll
        for (int r = 0; r < kSamples; ++r) sample[r] = r * kThreads + tid < some ? sample[r] : 0u;
        auto count = [&](uint32_t b0, uint32_t b1, uint32_t b2, uint32_t(&v)[3]) {
            v[0] = v[1] = v[2] = 0;
#pragma unroll
            for (int r = 0; r < kSamples; ++r) {
                v[0] += votes(sample[r] >= b0);
                v[1] += votes(sample[r] >= b1);
                v[2] += votes(sample[r] >= b2);
            }
        };
        // Four standard deviations of the sample's count to either side.
        const float share = static_cast<float>(x.keep) / static_cast<float>(x.n), rank = share * static_cast<float>(some);
        const float off = some < kAll ? 1.0f : 4.0f * sqrtf(rank * (1.0f - share)) + 2.0f;
        const int first = static_cast<int>(rank - off), last = static_cast<int>(rank + off) + 1;
        const uint32_t high = first < 1 ? 0xffffffffu : border_of(first, count, sh, turn, true);
        const uint32_t low = last > some ? 0u : border_of(last, count, sh, turn, true);
        if (tid == 0) listed = 0;
        __syncthreads();
        uint32_t v[4] = {0, 0, 0, 0}, fixed[1] = {0};
        const int64_t begin = seg.begin(x, w), end = seg.end(x, w);
        uint32_t *list = lists + pair * a.max_keys + begin;
        for (int64_t j0 = begin; j0 < end; j0 += kChunk) {
            int j[kHeld];
            uint32_t o[kHeld], protects;
#pragma unroll
            for (int r = 0; r < kHeld; ++r) j[r] = static_cast<int>(j0 + r * kThreads + tid < end ? j0 + r * kThreads + tid : end - 1);
            x.orders(a, j, o, protects);
            // How many this thread lists, and where.
            uint32_t set = 0;
#pragma unroll
            for (int r = 0; r < kHeld; ++r) {
                const bool in = j0 + r * kThreads + tid < end, f = in && (protects >> r & 1u) != 0u;
                o[r] = f ? 0xffffffffu : o[r];
                v[0] += votes(in && o[r] > high);
                v[1] += votes(in && o[r] == high);
                v[3] += votes(in && o[r] == low && o[r] != high);
                fixed[0] += votes(f);
                set |= in && o[r] > low && o[r] < high ? 1u << r : 0u;
            }
            const uint32_t mine = __popc(set), upto = wave_incl_scan_u32(mine, lane), sum = readlane_u32(upto, kWave - 1);
            v[2] += sum;
            uint32_t at = 0;
            if (lane == 0 && sum != 0) at = atomicAdd(&listed, sum);
            at = readlane_u32(at, 0) + upto - mine;
#pragma unroll
            for (int r = 0; r < kHeld; ++r)
                if (set >> r & 1u) list[at++] = o[r];
        }
        block_sums(v, sh, turn);
        block_sums(fixed, sh, turn);
        if (tid == 0)
            counts[pair * kMostSegments + w] = Counts{low, high, v[0], v[1], v[2], v[3], fixed[0], 0};
        __syncthreads();
    }
}

// The second one: the border, and each segment's sources or targets.
__global__ __launch_bounds__(kThreads) void k_evict_list(EvictArgs a, const Counts *counts, const uint32_t *lists, int64_t size,
                                                         Moves moves) {
    __shared__ Shared sh;
    __shared__ Counts held[kMostSegments];
    __shared__ uint32_t over[kMostSegments], even[kMostSegments];  // over and at the border, of each segment
    __shared__ uint32_t starts[kMostSegments + 1];                 // of the listed numbers
    __shared__ uint32_t ranks[kHeld * kWaves];
    const int tid = static_cast<int>(threadIdx.x), lane = tid & (kWave - 1);
    const uint64_t under = (uint64_t{1} << lane) - 1;
    int turn = 0;
    for (int64_t pair = blockIdx.x; pair < a.S * a.kv_heads; pair += gridDim.x) {
        const Head x = head_of(a, pair);
        const Segments seg(x, size);
        const int w = static_cast<int>(blockIdx.y);
        if (x.h == 0 && w == 0 && tid == 0) put_len(a, x);
        if (w == 0 && tid == 0 && (x.leave || x.keep == 0)) moves.count[pair] = 0;
        if (w >= seg.all) continue;
        const int64_t begin = seg.begin(x, w), end = seg.end(x, w);
        if (x.leave || x.keep == 0) {
            if (x.leave) carry_all(a, x, begin, end);
            continue;
        }
        __syncthreads();
        if (tid < seg.all) held[tid] = counts[pair * kMostSegments + tid], over[tid] = even[tid] = 0;
        __syncthreads();
        uint32_t above = 0, at_high = 0, between = 0, at_low = 0, fixed = 0;
        for (int i = 0; i < seg.all; ++i) {
            if (tid == 0) starts[i] = between;
            above += held[i].above, at_high += held[i].at_high, between += held[i].between, at_low += held[i].at_low;
            fixed += held[i].fixed;
        }
        if (tid == 0) starts[seg.all] = between;
        __syncthreads();
        const uint32_t keep = static_cast<uint32_t>(x.keep), low = held[0].low, high = held[0].high;
        const bool few = fixed <= keep;
        uint32_t border;  // (1 and more)
        // The numbers of tokens j0 .. j0 + kChunk - 1 before `stop`, 0 of the others.
        auto some = [&](int64_t j0, int64_t stop, uint32_t(&o)[kHeld]) {
            int j[kHeld];
#pragma unroll
            for (int r = 0; r < kHeld; ++r) j[r] = static_cast<int>(j0 + r * kThreads + tid < stop ? j0 + r * kThreads + tid : stop - 1);
            x.numbers(a, j, few, o);
#pragma unroll
            for (int r = 0; r < kHeld; ++r) o[r] = j0 + r * kThreads + tid < stop ? o[r] : 0u;
        };
        auto listed = [&](uint32_t e, int &of) {  // the e-th listed number, and its segment
            int lo = 0, hi = seg.all;
            while (hi - lo > 1) {
                const int mid = (lo + hi) >> 1;
                if (starts[mid] <= e) lo = mid; else hi = mid;
            }
            of = lo;
            return lists[pair * a.max_keys + seg.begin(x, lo) + (e - starts[lo])];
        };
        if (few && keep > above && keep <= above + at_high) {
            border = high;
            if (tid < seg.all) over[tid] = held[tid].above, even[tid] = held[tid].at_high;
        } else if (few && keep > above + at_high && keep <= above + at_high + between) {
            const uint32_t rank = keep - above - at_high;
            uint32_t o[kHeld];
            const bool fits = between <= static_cast<uint32_t>(kChunk);
#pragma unroll
            for (int r = 0; r < kHeld; ++r) {
                const uint32_t e = r * kThreads + tid;
                int of;
                o[r] = fits && e < between ? listed(e, of) : 0u;
            }
            border = border_of(
                rank,
                [&](uint32_t b0, uint32_t b1, uint32_t b2, uint32_t(&v)[3]) {
                    v[0] = v[1] = v[2] = 0;
                    if (fits) {
#pragma unroll
                        for (int r = 0; r < kHeld; ++r) {
                            if (static_cast<uint32_t>(r * kThreads) >= between) break;
                            v[0] += votes(o[r] >= b0);
                            v[1] += votes(o[r] >= b1);
                            v[2] += votes(o[r] >= b2);
                        }
                    } else {
                        for (uint32_t e0 = 0; e0 < between; e0 += kThreads) {
                            int of;
                            const uint32_t n = e0 + tid < between ? listed(e0 + tid, of) : 0u;
                            v[0] += votes(n >= b0);
                            v[1] += votes(n >= b1);
                            v[2] += votes(n >= b2);
                        }
                    }
                },
                sh, turn, true);
            if (tid < seg.all) over[tid] = held[tid].above + held[tid].at_high;
            __syncthreads();
            for (uint32_t e = tid; e < between; e += kThreads) {
                int of;
                const uint32_t n = listed(e, of);
                if (n > border) atomicAdd(&over[of], 1u);
                if (n == border) atomicAdd(&even[of], 1u);
            }
        } else if (few && keep > above + at_high + between && keep <= above + at_high + between + at_low) {
            border = low;
            if (tid < seg.all) {
                over[tid] = held[tid].above + held[tid].at_high + held[tid].between;
                even[tid] = held[tid].at_low;
            }
        } else {  // the two numbers do not hold it, or more tokens are protected than stay
            border = border_of(
                keep,
                [&](uint32_t b0, uint32_t b1, uint32_t b2, uint32_t(&v)[3]) {
                    v[0] = v[1] = v[2] = 0;
                    for (int64_t j0 = 0; j0 < x.n; j0 += kChunk) {
                        uint32_t o[kHeld];
                        some(j0, x.n, o);
#pragma unroll
                        for (int r = 0; r < kHeld; ++r) {
                            v[0] += votes(o[r] >= b0);
                            v[1] += votes(o[r] >= b1);
                            v[2] += votes(o[r] >= b2);
                        }
                    }
                },
                sh, turn, true);
            for (int64_t j0 = 0; j0 < x.n; j0 += kChunk) {
                uint32_t o[kHeld];
                some(j0, x.n, o);
#pragma unroll
                for (int r = 0; r < kHeld; ++r) {
                    const int64_t j = j0 + r * kThreads + tid;
                    if (o[r] > border) atomicAdd(&over[seg.of(x, j)], 1u);
                    if (o[r] == border) atomicAdd(&even[seg.of(x, j)], 1u);
                }
            }
        }
        __syncthreads();
        // Of those at the border the first ones stay; and what comes before this segment.
        uint32_t left = keep, first_even = 0, stays = 0, first = 0, all = 0;
        for (int i = 0; i < seg.all; ++i) left -= over[i];
        for (int i = 0; i < seg.all; ++i) {
            const uint32_t take = even[i] < left ? even[i] : left;
            const uint32_t kept = over[i] + take;
            left -= take;
            const uint32_t mine = i < seg.below ? static_cast<uint32_t>(seg.end(x, i) - seg.begin(x, i)) - kept : kept;
            if (i == w) stays = take;
            if (i < w && (i < seg.below) == (w < seg.below)) first += mine;
            if (i >= seg.below) all += mine;
        }
        if (w == 0 && tid == 0) moves.count[pair] = static_cast<int32_t>(all);
        int32_t *out = moves.from + (pair * 2 + (w < seg.below ? 1 : 0)) * moves.most;
        const bool below = w < seg.below, carries = below && (a.mass_out != a.mass || a.positions_out != a.key_positions);
        for (int64_t j0 = begin; j0 < end; j0 += kChunk) {
            uint32_t o[kHeld], mine[kHeld], sum[kHeld], kept = 0, total;
            some(j0, end, o);
#pragma unroll
            for (int r = 0; r < kHeld; ++r) {
                kept |= o[r] > border ? 1u << r : 0u;
                mine[r] = votes(o[r] == border);
            }
            before(ranks, mine, sum, total);
#pragma unroll
            for (int r = 0; r < kHeld; ++r) {
                const uint32_t rank = first_even + sum[r] + static_cast<uint32_t>(__popcll(__ballot(o[r] == border) & under));
                kept |= o[r] == border && rank < stays ? 1u << r : 0u;
            }
            first_even += total;
            uint64_t set[kHeld];
#pragma unroll
            for (int r = 0; r < kHeld; ++r) {
                const bool in = j0 + r * kThreads + tid < end, k = (kept >> r & 1u) != 0u;
                set[r] = __ballot(in && k != below);
                mine[r] = static_cast<uint32_t>(__popcll(set[r]));
                if (carries && in && k) carry(a, x.place(a, j0 + r * kThreads + tid));
            }
            before(ranks, mine, sum, total);
#pragma unroll
            for (int r = 0; r < kHeld; ++r)
                if (set[r] >> lane & 1u)
                    out[first + sum[r] + static_cast<uint32_t>(__popcll(set[r] & under))] = static_cast<int32_t>(j0 + r * kThreads + tid);
            first += total;
        }
        __syncthreads();
    }
}

struct Plan {
    int64_t size, segments;  // of long heads
    size_t off_counts, off_lists, off_from, total;
    int64_t most;
};

Plan plan_evict(int64_t heads, int64_t max_keys) {
    Plan p{};
    const size_t n = static_cast<size_t>(heads), keys = static_cast<size_t>(max_keys);
    auto take = [&](size_t bytes) {
        const size_t at = p.total;
        p.total += (bytes + 255) / 256 * 256;
        return at;
    };
    take(n * sizeof(int32_t));  // how many moves
    p.most = max_keys / 2 + 1;  // no more than half of a head's tokens move
    p.off_from = take(n * 2 * static_cast<size_t>(p.most) * sizeof(int32_t));
    if (max_keys > kChunk) {
        p.size = ((max_keys + kSegments - 1) / kSegments + kChunk - 1) / kChunk * kChunk;
        p.segments = (max_keys + p.size - 1) / p.size + 1;
        p.off_counts = take(n * kMostSegments * sizeof(Counts));
        p.off_lists = take(n * keys * sizeof(uint32_t));
    }
    return p;
}

template <int CHUNKS>
hipError_t launch(const EvictArgs &a, char *workspace, hipStream_t stream) {
    const int64_t heads = a.S * a.kv_heads;
    const Plan p = plan_evict(heads, a.max_keys);
    const Moves moves{reinterpret_cast<int32_t *>(workspace), reinterpret_cast<int32_t *>(workspace + p.off_from), p.most};
    const unsigned grid = static_cast<unsigned>(heads < kGrid ? heads : kGrid);
    if (a.max_keys <= kChunk) {
        if (heads >= 256 || a.max_keys <= 2048) {
            k_evict_held<true, CHUNKS><<<dim3(grid), kThreads, 0, stream>>>(a, moves);
            return hipGetLastError();
        }
        k_evict_held<false, CHUNKS><<<dim3(grid), kThreads, 0, stream>>>(a, moves);
    } else {
        Counts *counts = reinterpret_cast<Counts *>(workspace + p.off_counts);
        uint32_t *lists = reinterpret_cast<uint32_t *>(workspace + p.off_lists);
        const dim3 segments(grid, static_cast<unsigned>(p.segments));
        k_evict_count<<<segments, kThreads, 0, stream>>>(a, counts, lists, p.size);
        k_evict_list<<<segments, kThreads, 0, stream>>>(a, counts, lists, p.size, moves);
    }
    // Enough workgroups for 256 CUs; no more than a head can have moves for.
    constexpr int64_t BATCH = batch_of(CHUNKS);
    const int64_t batches = (p.most + 4 * BATCH - 1) / (4 * BATCH), wanted = (8192 + heads - 1) / heads;
    const dim3 movers(static_cast<unsigned>(batches < wanted ? batches : wanted),
                      static_cast<unsigned>(heads < 65535 ? heads : 65535));
    k_evict_move<CHUNKS><<<movers, 256, 0, stream>>>(a, moves);
    return hipGetLastError();
}

}  // namespace

size_t evict_workspace(int64_t S, int64_t kv_heads, int64_t max_keys) { return plan_evict(S * kv_heads, max_keys).total; }

hipError_t launch_cache_evict(const EvictArgs &a, void *workspace, hipStream_t stream) {
    char *ws = static_cast<char *>(workspace);
    const bool aligned = reinterpret_cast<uintptr_t>(a.k_cache) % 16 == 0 && reinterpret_cast<uintptr_t>(a.v_cache) % 16 == 0;
    switch (aligned ? a.head_dim : 0) {
    case 64: return launch<8>(a, ws, stream);
    case 128: return launch<16>(a, ws, stream);
    case 256: return launch<32>(a, ws, stream);
    default: return launch<0>(a, ws, stream);
    }
}

}  // namespace knnlm
