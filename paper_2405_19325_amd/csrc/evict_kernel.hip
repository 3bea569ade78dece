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
// Heads of up to 8,192 tokens: a workgroup has them in registers, 16 places a
// thread, and finds the border eleven bits at a time by counting into bins.
// Longer ones are cut into segments,
// a workgroup each, which ends at the budget so that a segment holds sources or
// targets only.  All of a head's workgroups look at the same 4,096 tokens,
// whose order gives two numbers that the border lies between but for one head
// in thousands; each counts its segment's numbers above, at and below these and
// lists those between.  A second launch finds the border in the few that are
// listed, and with it each segment's share of the moves, which a last one makes.
// Where the border lies elsewhere, or as many tokens are protected as stay or
// more, each of the workgroups goes through the whole head for it: 16 heads of
// 131,072 tokens to 16,384 in 201 us where 16,384 are protected, 281 where more
// are, 89 where fewer.
//
// What bounds it.  A step's few moves: waits, one behind the other; 512 heads of
// 4,100 tokens in 19 us, 7 until their loads are on the way, 5 for these and the
// ledger of afterwards, 2 for the border, 3 for the lists, 2 for the moves.  A
// prompt's cut: the moves, at 5.2 to 5.6 TB/s read and written (keys of 128
// heads 31 us of 58; two prompts of 131,072 tokens to an eighth 46 of 101, behind
// 19 for the counts and 24 for the border and the lists).  The order is found
// by counting, not by sorting: it reads each mass once, or twice where heads are
// long.
#include "lm_device.h"

namespace knnlm {

namespace {

constexpr int kThreads = 512;
constexpr int kWaves = kThreads / kWave;
constexpr int kGroups = 4;                   // of four tokens of a thread, which lie within a page
constexpr int kHeld = 4 * kGroups;
constexpr int kRow = 4 * kThreads;           // tokens from a thread's group to its next one
constexpr int kChunk = kHeld * kThreads;
constexpr int kSegments = 64;                // of a head, about
constexpr int kBits = 11, kBins = 1 << kBits;
constexpr int64_t kGrid = int64_t{1} << 20;  // heads of a row of the grid

// A number that orders like x, NaN first.
__device__ __forceinline__ uint32_t order_of(float x) {
    if (x != x) return 1u;
    const uint32_t b = __float_as_uint(x + 0.0f);  // one zero
    return b ^ ((b >> 31) != 0 ? 0xffffffffu : 0x80000000u);
}

// LDS of the collective steps.
struct Shared {
    uint32_t bins[kBins];      // all 0 between them
    uint32_t part[2][3][kWaves]; // these alternate, so that a sum may follow another without a barrier between
    uint32_t bin[2], rank[2], count[2];
    uint32_t n, few[kWave];    // the numbers of a bin with few
};

__device__ __forceinline__ void clear(Shared &sh) {
    static_assert(kBins == 4 * kThreads, "four bins a thread");
    reinterpret_cast<uint4 *>(sh.bins)[threadIdx.x] = make_uint4(0, 0, 0, 0);
    if (threadIdx.x == 0) sh.n = 0;
}

__device__ __forceinline__ uint32_t votes(bool flag) { return static_cast<uint32_t>(__popcll(__ballot(flag))); }

// What the threads before this one have of v together, and all (up to 2^32).
__device__ __forceinline__ uint32_t before(uint32_t v, uint32_t &all, Shared &sh, int &turn) {
    const int lane = static_cast<int>(threadIdx.x) & (kWave - 1), wave = static_cast<int>(threadIdx.x) / kWave;
    const uint32_t upto = wave_incl_scan_u32(v, lane);
    turn ^= 1;
    if (lane == kWave - 1) sh.part[turn][0][wave] = upto;
    __syncthreads();
    uint32_t first = upto - v;
    all = 0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
        const uint32_t x = sh.part[turn][0][w];
        first += w < wave ? x : 0u;
        all += x;
    }
    return first;
}

// The workgroup's sums of three.
__device__ __forceinline__ void sums(uint32_t &a, uint32_t &b, uint32_t &c, Shared &sh, int &turn) {
    const int lane = static_cast<int>(threadIdx.x) & (kWave - 1), wave = static_cast<int>(threadIdx.x) / kWave;
    a = wave_incl_scan_u32(a, lane), b = wave_incl_scan_u32(b, lane), c = wave_incl_scan_u32(c, lane);
    turn ^= 1;
    if (lane == kWave - 1) sh.part[turn][0][wave] = a, sh.part[turn][1][wave] = b, sh.part[turn][2][wave] = c;
    __syncthreads();
    a = b = c = 0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) a += sh.part[turn][0][w], b += sh.part[turn][1][w], c += sh.part[turn][2][w];
}

// For tokens held as Held has them: how many of `set` (bits) come before each of
// this thread's groups, and all; the workgroup's sum of `more`.
__device__ __forceinline__ void before_groups(uint32_t set, uint32_t (&first)[kGroups], uint32_t &all, uint32_t &more, Shared &sh,
                                              int &turn) {
    static_assert(kGroups == 4 && kRow < 1 << 16, "two rows' counts in a word");
    const int lane = static_cast<int>(threadIdx.x) & (kWave - 1), wave = static_cast<int>(threadIdx.x) / kWave;
    uint32_t v[2], upto[2], rows[2] = {0, 0};
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        v[i] = __popc(set >> (8 * i) & 15u) | __popc(set >> (8 * i + 4) & 15u) << 16;
        upto[i] = wave_incl_scan_u32(v[i], lane);
    }
    const uint32_t sum = wave_incl_scan_u32(more, lane);
    turn ^= 1;
    if (lane == kWave - 1) sh.part[turn][0][wave] = upto[0], sh.part[turn][1][wave] = upto[1], sh.part[turn][2][wave] = sum;
    __syncthreads();
    more = 0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) more += sh.part[turn][2][w];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        upto[i] -= v[i];
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
            const uint32_t x = sh.part[turn][i][w];
            upto[i] += w < wave ? x : 0u;
            rows[i] += x;
        }
    }
    all = 0;
#pragma unroll
    for (int g = 0; g < kGroups; ++g) {
        const int at = 16 * (g & 1);
        first[g] = all + (upto[g / 2] >> at & 0xffffu);
        all += rows[g / 2] >> at & 0xffffu;
    }
}

// f(bit) for each bit that is set: the few of each thread one behind the other
// (a step's move or two), or all of them looked at (13 us for the four prompts'
// heads, 16 the other way).
template <bool FEW, class F>
__device__ __forceinline__ void each_bit(uint32_t set, F f) {
    if constexpr (FEW) {
        while (set != 0u) {
            f(__ffs(static_cast<int>(set)) - 1);
            set &= set - 1u;
        }
    } else {
#pragma unroll
        for (int i = 0; i < kHeld; ++i)
            if (set >> i & 1u) f(i);
    }
}

// The workgroup's sum, least and largest.
__device__ __forceinline__ void reduce(uint32_t &sum, uint32_t &least, uint32_t &largest, Shared &sh, int &turn) {
    const int lane = static_cast<int>(threadIdx.x) & (kWave - 1), wave = static_cast<int>(threadIdx.x) / kWave;
    turn ^= 1;
    const uint32_t s = readlane_u32(wave_incl_scan_u32(sum, lane), kWave - 1);
    const uint32_t lo = wave_allmin_u32(least), hi = wave_allmax_u32(largest);
    if (lane == 0) sh.part[turn][0][wave] = s, sh.part[turn][1][wave] = lo, sh.part[turn][2][wave] = hi;
    __syncthreads();
    sum = 0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
        sum += sh.part[turn][0][w];
        least = min(least, sh.part[turn][1][w]);
        largest = max(largest, sh.part[turn][2][w]);
    }
}

// The border of the `rank` largest numbers: those over `over` are among them,
// and of those equal to it the first `even`.
struct Border {
    uint32_t over, even;
};

// Numbers base .. base + 2^bits - 1, the rank-th largest of which is looked for.
struct Range {
    uint32_t base;
    int bits;
    uint32_t rank, count;
    __device__ __forceinline__ bool has(uint32_t o) const { return bits >= 32 || (o >= base && (o - base) >> bits == 0u); }
};

__device__ __forceinline__ Range range_of(uint32_t least, uint32_t largest, uint32_t rank) {
    return Range{least, 32 - __clz(static_cast<int>(largest - least)), rank, 0xffffffffu};
}

// Cuts a range down to one of its 2,048 bins (several, for as many ranks in it).
// each(f) calls f with all of this thread's numbers (0: none), the same ones
// every time; a rank is at least 1 and at most as many as the range has.
template <int N, class Each>
__device__ __forceinline__ void narrow(Range (&r)[N], Each each, Shared &sh, int &turn) {
    const uint32_t base = r[0].base;
    const int shift = r[0].bits > kBits ? r[0].bits - kBits : 0;
    const Range in = r[0];
    each([&](uint32_t o) {
        if (o != 0u && in.has(o)) atomicAdd(&sh.bins[(o - base) >> shift], 1u);
    });
    __syncthreads();
    // Four bins a thread, the highest ones first.
    uint4 *mine = reinterpret_cast<uint4 *>(sh.bins) + (kThreads - 1 - threadIdx.x);
    const uint4 c = *mine;
    *mine = make_uint4(0, 0, 0, 0);
    uint32_t all;
    const uint32_t first = before(c.x + c.y + c.z + c.w, all, sh, turn);
#pragma unroll
    for (int i = 0; i < N; ++i)
        if (r[i].rank > first && r[i].rank <= first + c.x + c.y + c.z + c.w) {
            uint32_t left = r[i].rank - first, bin = 4 * (kThreads - 1 - threadIdx.x) + 3, count = c.w;
            if (left > count) left -= count, --bin, count = c.z;
            if (left > count) left -= count, --bin, count = c.y;
            if (left > count) left -= count, --bin, count = c.x;
            sh.bin[i] = bin, sh.rank[i] = left, sh.count[i] = count;
        }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; ++i) r[i] = Range{base + (sh.bin[i] << shift), shift, sh.rank[i], sh.count[i]};
}

// The border, all numbers being in [least, largest].
template <class Each>
__device__ __forceinline__ Border border_of(uint32_t rank, uint32_t least, uint32_t largest, Each each, Shared &sh, int &turn) {
    Range r[1] = {range_of(least, largest, rank)};
    do {
        narrow(r, each, sh, turn);
        if (r[0].count == r[0].rank) return Border{r[0].base - 1u, 0u};  // all of the bin (no number is 0)
    } while (r[0].bits > 0 && r[0].count > kWave);
    if (r[0].bits == 0) return Border{r[0].base, r[0].rank};
    // The few that are left, a lane each in every wave.
    each([&](uint32_t o) {
        if (o != 0u && r[0].has(o)) sh.few[atomicAdd(&sh.n, 1u)] = o;
    });
    __syncthreads();
    const int lane = static_cast<int>(threadIdx.x) & (kWave - 1), n = static_cast<int>(r[0].count);
    const uint32_t x = lane < n ? sh.few[lane] : 0u;
    uint32_t over = 0, upto = 0;
    for (int i = 0; i < n; ++i) {
        const uint32_t y = readlane_u32(x, i);
        over += y > x ? 1u : 0u;
        upto += y >= x ? 1u : 0u;
    }
    const uint64_t at = __ballot(lane < n && over < r[0].rank && r[0].rank <= upto);
    const int which = __ffsll(static_cast<unsigned long long>(at)) - 1;
    return Border{readlane_u32(x, which), r[0].rank - readlane_u32(over, which)};
}

// A head of a sequence and what becomes of it.
struct Head {
    int64_t s;
    int h;
    int64_t n, keep;  // tokens, and those that stay; of a head that is left as it is, those that its table has room for
    int32_t recent_from;
    bool leave;       // left as it is
    bool vec;         // the ledgers lie on 16 bytes

    __device__ __forceinline__ int64_t place(const EvictArgs &a, int64_t j) const {
        return place_of(a.cache, a.kv_heads, s, h, j);
    }
    // The number of a token, where there are no more protected ones than the budget (few), or more.
    __device__ static __forceinline__ uint32_t number(uint32_t order, bool fixed, bool few) {
        return few ? (fixed ? 0xffffffffu : order) : (fixed ? order : 0u);
    }
    __device__ __forceinline__ bool fixed(const EvictArgs &a, int32_t p) const { return p < a.sinks || p >= recent_from; }
};

__device__ __forceinline__ int64_t pair_of() { return static_cast<int64_t>(blockIdx.z) * kGrid + blockIdx.x; }

// (Without a look at its pages.)
__device__ __forceinline__ Head head_of(const EvictArgs &a, int64_t pair) {
    Head x;
    x.s = pair / a.kv_heads;
    x.h = static_cast<int>(pair - x.s * a.kv_heads);
    const int64_t len = a.cache_lens[x.s], budget = a.budgets[x.s];
    const int64_t room = a.cache.table_width << a.cache.page_log2, limit = a.max_keys < room ? a.max_keys : room;
    const int64_t n = len < 0 ? 0 : len;
    const int64_t recent_from = (a.next_positions != nullptr ? a.next_positions[x.s] : len) - a.recent;
    x.recent_from = static_cast<int32_t>(recent_from > -0x80000000LL ? recent_from : -0x80000000LL);
    x.leave = budget < 0 || budget >= n || n > limit;
    x.n = n < room ? n : room;
    x.keep = x.leave ? x.n : budget;
    x.vec = ((reinterpret_cast<uintptr_t>(a.mass) | reinterpret_cast<uintptr_t>(a.key_positions) |
              reinterpret_cast<uintptr_t>(a.mass_out) | reinterpret_cast<uintptr_t>(a.positions_out)) % 16) == 0;
    return x;
}

__device__ __forceinline__ void put_len(const EvictArgs &a, const Head &x) {
    a.new_lens[x.s] = x.leave ? a.cache_lens[x.s] : static_cast<int32_t>(x.keep);
}

// Groups of four tokens, from j[0], j[1], ... on (multiples of four): what the ledger has of those in [from, to).
template <int G = kGroups>
struct Held {
    int64_t at[G];   // place of a group's first
    uint32_t in;     // as bits: those in the range
    uint32_t fixed;  // and of these the protected ones
    bool missing;    // there are some whose page is none
    union {
        float m[4 * G];
        float4 m4[G];
    };
    union {
        int32_t p[4 * G];
        int4 p4[G];
    };

    __device__ __forceinline__ void load(const EvictArgs &a, const Head &x, const int64_t (&j)[G], int64_t from, int64_t to) {
        in = 0;
        missing = false;
        bool some[G];
#pragma unroll
        for (int g = 0; g < G; ++g) {
            some[g] = j[g] < to && j[g] + 4 > from;
            at[g] = some[g] ? x.place(a, j[g]) : 0;
            if (at[g] < 0) missing = true, some[g] = false;
        }
#pragma unroll
        for (int g = 0; g < G; ++g) {
            if (!some[g]) continue;
            uint32_t bits = 15u;
            if (j[g] < from) bits &= 15u << (from - j[g]);
            if (j[g] + 4 > to) bits &= (1u << (to - j[g])) - 1u;
            in |= bits << 4 * g;
            if (x.vec) {
                m4[g] = *reinterpret_cast<const float4 *>(a.mass + at[g]);
                if (a.key_positions != nullptr) p4[g] = *reinterpret_cast<const int4 *>(a.key_positions + at[g]);
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    m[4 * g + e] = a.mass[at[g] + e];
                    if (a.key_positions != nullptr) p[4 * g + e] = a.key_positions[at[g] + e];
                }
            }
        }
        if (a.key_positions != nullptr) return;
#pragma unroll
        for (int i = 0; i < 4 * G; ++i) p[i] = static_cast<int32_t>(j[i / 4]) + i % 4;
    }
    // What was loaded is looked at: apart, so that other loads may follow before it has come.
    __device__ __forceinline__ void look(const EvictArgs &a, const Head &x) {
        fixed = 0;
#pragma unroll
        for (int i = 0; i < 4 * G; ++i) fixed |= x.fixed(a, p[i]) ? 1u << i : 0u;
        fixed &= in;
    }
    // This thread's part of kChunk tokens from j0 on.
    __device__ __forceinline__ void load_chunk(const EvictArgs &a, const Head &x, int64_t j0, int64_t from, int64_t to) {
        int64_t j[G];
#pragma unroll
        for (int g = 0; g < G; ++g) j[g] = token(j0, 4 * g);
        load(a, x, j, from, to);
    }
    __device__ static __forceinline__ int64_t token(int64_t j0, int bit) {
        return j0 + static_cast<int64_t>(bit / 4) * kRow + 4 * static_cast<int>(threadIdx.x) + bit % 4;
    }
    // 0 of those out of the range.
    __device__ __forceinline__ void numbers(bool few, uint32_t (&o)[4 * G]) const {
#pragma unroll
        for (int i = 0; i < 4 * G; ++i)
            o[i] = (in >> i & 1u) != 0u ? Head::number(order_of(m[i]), (fixed >> i & 1u) != 0u, few) : 0u;
    }
    // The entries of `some` go into a ledger of afterwards that is another.  (Those of places that are given up are written
    // over by what moves there, later.)
    __device__ __forceinline__ void carry(const EvictArgs &a, const Head &x, uint32_t some) const {
        const bool masses = a.mass_out != a.mass, positions = a.positions_out != a.key_positions;
#pragma unroll
        for (int g = 0; g < G; ++g) {
            const uint32_t bits = some >> 4 * g & 15u;
            if (bits == 15u && x.vec) {
                if (masses) *reinterpret_cast<float4 *>(a.mass_out + at[g]) = m4[g];
                if (positions) *reinterpret_cast<int4 *>(a.positions_out + at[g]) = p4[g];
                continue;
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                if ((bits >> e & 1u) == 0u) continue;
                if (masses) a.mass_out[at[g] + e] = m[4 * g + e];
                if (positions) a.positions_out[at[g] + e] = p[4 * g + e];
            }
        }
    }
};

__device__ __forceinline__ bool carries(const EvictArgs &a) {
    return a.mass_out != a.mass || a.positions_out != a.key_positions;
}

// The ledger's entries [from, to) of a head that is left as it is, as far as it has pages.
__device__ __forceinline__ void carry_all(const EvictArgs &a, const Head &x, int64_t from, int64_t to) {
    if (!carries(a)) return;
    for (int64_t j = from + threadIdx.x; j < to; j += kThreads) {
        const int64_t at = x.place(a, j);
        if (at < 0) continue;
        if (a.mass_out != a.mass) a.mass_out[at] = a.mass[at];
        if (a.positions_out != a.key_positions) a.positions_out[at] = a.key_positions[at];
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

// Of the tokens that a thread holds of kChunk from j0 on, those below `keep`, as bits.
__device__ __forceinline__ uint32_t below_of(int64_t j0, int64_t keep) {
    uint32_t bits = 0;
#pragma unroll
    for (int g = 0; g < kGroups; ++g) {
        const int64_t left = keep - Held<>::token(j0, 4 * g);
        bits |= (left <= 0 ? 0u : left >= 4 ? 15u : (1u << left) - 1u) << 4 * g;
    }
    return bits;
}

// How many are kept before the token of bit i, `first` those before its group.
__device__ __forceinline__ uint32_t kept_before(uint32_t kept, const uint32_t (&first)[kGroups], int i) {
    const int g = i / 4;
    const uint32_t at = g == 0 ? first[0] : g == 1 ? first[1] : g == 2 ? first[2] : first[3];
    return at + __popc((kept >> 4 * g & 15u) & ((1u << (i & 3)) - 1u));
}

// A head in a workgroup's registers.  `CHUNKS` as in move; MOVE: the moves are
// made here, else left to another launch.
template <bool MOVE, int CHUNKS>
__global__ __launch_bounds__(kThreads, 4) void k_evict_held(EvictArgs a, Moves moves) {
    __shared__ Shared sh;
    __shared__ uint16_t lists[MOVE ? 2 : 1][MOVE ? kChunk / 2 : 1];  // sources, targets
    const int tid = static_cast<int>(threadIdx.x), lane = tid & (kWave - 1), wave = tid / kWave;
    int turn = 0;
    clear(sh);
    const int64_t pair = pair_of();
    if (pair >= a.S * a.kv_heads) return;
    Head x = head_of(a, pair);
    const int n = static_cast<int>(x.n), keep = static_cast<int>(x.keep);
    Held<> t;
    t.load_chunk(a, x, 0, 0, x.leave ? 0 : n);  // every page is some thread's
    t.look(a, x);
    const uint32_t low = below_of(0, keep);
    if (carries(a) && (t.in & low) != 0u) t.carry(a, x, t.in & low);
    uint32_t o[kHeld], least = 0xffffffffu, largest = 0u;
    t.numbers(true, o);
#pragma unroll
    for (int i = 0; i < kHeld; ++i) {
        if (o[i] == 0u || o[i] == 0xffffffffu) continue;
        least = min(least, o[i]), largest = max(largest, o[i]);
    }
    uint32_t protects = t.missing ? 1u << 16 : __popc(t.fixed);  // 8,192 at most are protected
    if (!x.leave) {
        reduce(protects, least, largest, sh, turn);
        x.leave = protects >> 16 != 0u;
    }
    if (x.h == 0 && tid == 0) put_len(a, x);
    if (x.leave) {
        carry_all(a, x, 0, x.n);
        if (!MOVE && tid == 0) moves.count[pair] = 0;
        return;
    }
    const bool few = protects <= static_cast<uint32_t>(keep);
    if (!few) t.numbers(false, o), least = 1u, largest = 0xff800000u;
    const uint32_t rank = few ? keep - protects : keep;  // among those that are not protected, or among these alone
    Border border{few ? 0xfffffffeu : 0xffffffffu, 0u};
    if (rank > 0)
        border = border_of(
            rank, least, largest,
            [&](auto count) {
#pragma unroll
                for (int i = 0; i < kHeld; ++i)
                    if (o[i] != 0xffffffffu) count(o[i]);
            },
            sh, turn);
    uint32_t kept = 0, at_it = 0;  // as bits
#pragma unroll
    for (int i = 0; i < kHeld; ++i) {
        kept |= o[i] > border.over ? 1u << i : 0u;
        at_it |= o[i] == border.over ? 1u << i : 0u;
    }
    uint32_t first[kGroups], all, kept_low = 0;
    if (border.even != 0) {
        before_groups(at_it, first, all, kept_low, sh, turn);
#pragma unroll
        for (int i = 0; i < kHeld; ++i)
            if (at_it >> i & 1u) kept |= first[i / 4]++ < border.even ? 1u << i : 0u;
    }
    // With as many kept before it, a target is what lies before it less these, and a source these less those below the budget.
    kept_low = __popc(kept & low);
    before_groups(kept, first, all, kept_low, sh, turn);
    const uint32_t total = keep - kept_low;
    int32_t *out = MOVE ? nullptr : moves.from + pair * 2 * moves.most;
    each_bit<MOVE>((kept & ~low) | (t.in & low & ~kept), [&](int i) {
        const uint32_t j = static_cast<uint32_t>(Held<>::token(0, i)), before_it = kept_before(kept, first, i);
        const bool target = (low >> i & 1u) != 0u;
        const uint32_t to = target ? j - before_it : before_it - kept_low;
        if constexpr (MOVE) lists[target ? 1 : 0][to] = static_cast<uint16_t>(j);
        else out[(target ? moves.most : 0) + to] = static_cast<int32_t>(j);
    });
    if constexpr (MOVE) {
        __syncthreads();
        constexpr int BATCH = batch_of(CHUNKS);
        for (uint32_t m = wave * BATCH; m < total; m += kWaves * BATCH) {
            const uint32_t i = lane < BATCH && m + lane < total ? m + lane : m;
            move<CHUNKS>(a, x.place(a, lists[0][i]), x.place(a, lists[1][i]),
                         static_cast<int>(total - m < BATCH ? total - m : BATCH));
        }
    } else if (tid == 0) {
        moves.count[pair] = static_cast<int32_t>(total);
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
    uint32_t low, high;                        // the two numbers, the same for all segments of a head
    uint32_t above, at_high, between, at_low;  // how many of the segment's are over `high`, at it, ...
    uint32_t fixed;
    uint32_t missing;                          // threads that met a page that is none
};

// The segments of a head: [0, keep) and [keep, n) in pieces of `size`, a
// multiple of kChunk; those behind the budget count from its multiple of kHeld.
struct Segments {
    int64_t size, behind;
    int below, all;  // how many lie below the budget; all

    __device__ __forceinline__ Segments(const Head &x, int64_t size_) : size(size_), behind(x.keep / kHeld * kHeld) {
        below = static_cast<int>((x.keep + size - 1) / size);
        all = below + static_cast<int>((x.n - (x.keep < x.n ? behind : x.n) + size - 1) / size);
    }
    __device__ __forceinline__ int64_t start(int w) const { return w < below ? w * size : behind + (w - below) * size; }
    __device__ __forceinline__ int64_t begin(const Head &x, int w) const {
        const int64_t b = start(w);
        return w < below || b > x.keep ? b : x.keep;
    }
    __device__ __forceinline__ int64_t end(const Head &x, int w) const {
        const int64_t e = start(w) + size, most = w < below ? x.keep : x.n;
        return e < most ? e : most;
    }
    __device__ __forceinline__ int of(const Head &x, int64_t j) const {
        return j < x.keep ? static_cast<int>(j / size) : below + static_cast<int>((j - behind) / size);
    }
};

constexpr int kMostSegments = kSegments + 2;

// The first launch over long heads: counts, and the numbers between, listed in
// the segment's part of `lists` [heads][max_keys].
__global__ __launch_bounds__(kThreads, 4) void k_evict_count(EvictArgs a, Counts *counts, uint32_t *lists, int64_t size) {
    __shared__ Shared sh;
    const int tid = static_cast<int>(threadIdx.x);
    int turn = 0;
    clear(sh);
    const int64_t pair = pair_of();
    if (pair >= a.S * a.kv_heads) return;
    const Head x = head_of(a, pair);
    const Segments seg(x, size);
    const int w = static_cast<int>(blockIdx.y);
    if (x.leave || w >= seg.all) return;
    // Four tokens of each of 2,048 equal pieces, at no regular distance; all of as many.  (Neighbours may be alike: what
    // they say is worth that of 2,048 tokens at least.)
    constexpr int kLog2 = 11;
    static_assert(kGroups * kThreads == 1 << kLog2, "pieces by shifts");
    const bool whole = x.n <= kChunk;
    int64_t which[kGroups];
#pragma unroll
    for (int g = 0; g < kGroups; ++g) {
        const uint32_t i = g * kThreads + tid, mix = i * 2654435761u;
        const int64_t j0 = i * x.n >> kLog2, j1 = (i + 1) * x.n >> kLog2;
        const int64_t j = j0 + __umulhi(mix ^ mix >> 15, static_cast<uint32_t>(j1 - j0));
        which[g] = whole ? Held<>::token(0, 4 * g) : j & ~int64_t{3};
    }
    const int64_t begin = seg.begin(x, w), end = seg.end(x, w);
    Held<> t;  // the segment's own tokens, on their way together with the sample
    t.load_chunk(a, x, seg.start(w), begin, end);
    uint32_t sample[kHeld], least = 0xffffffffu, largest = 0u, held = 0;  // held: with those protected ones << 16
    {
        Held<> some;
        some.load(a, x, which, 0, x.n);
        some.look(a, x);
        some.numbers(true, sample);
        held = __popc(some.in & ~some.fixed) | __popc(some.fixed) << 16;
    }
#pragma unroll
    for (int i = 0; i < kHeld; ++i) {
        if (sample[i] == 0u || sample[i] == 0xffffffffu) continue;
        least = min(least, sample[i]), largest = max(largest, sample[i]);
    }
    reduce(held, least, largest, sh, turn);
    const int others = static_cast<int>(held & 0xffffu), fixed_ones = static_cast<int>(held >> 16);
    // Six standard deviations of the sample's count to either side: three where neighbours are alike.
    const float share = static_cast<float>(x.keep) / static_cast<float>(x.n);
    const float rank = share * static_cast<float>(others + fixed_ones);
    const float off = whole ? 1.0f : 6.0f * sqrtf(rank * (1.0f - share)) + 2.0f;
    const int first = static_cast<int>(rank - off) - fixed_ones, last = static_cast<int>(rank + off) + 1 - fixed_ones;
    uint32_t high = 0xfffffffeu, low = 0u;  // protected tokens are above, and no number is 0
    if (others > 0) {
        auto each = [&](auto count) {
#pragma unroll
            for (int i = 0; i < kHeld; ++i)
                if (sample[i] != 0xffffffffu) count(sample[i]);
        };
        // The bins of both ranks; one that holds many is cut further (they may all be equal).
        auto clamp = [&](int i) { return static_cast<uint32_t>(i < 1 ? 1 : i > others ? others : i); };
        Range r[2] = {range_of(least, largest, clamp(first)), range_of(least, largest, clamp(last))};
        narrow(r, each, sh, turn);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            Range one[1] = {r[i]};
            while (one[0].bits > 0 && one[0].count > kWave) narrow(one, each, sh, turn);
            r[i] = one[0];
        }
        // A bin's numbers lie between; one number is a border itself.
        if (first >= 1) high = r[0].bits > 0 ? r[0].base + (1u << r[0].bits) : r[0].base;
        if (last <= others) low = r[1].bits > 0 ? r[1].base - 1u : r[1].base;
    }
    uint32_t above = 0, at_high = 0, at_low = 0, fixed = 0, missing = 0, listed = 0;
    uint32_t *list = lists + pair * a.max_keys + begin;
    for (int64_t at = seg.start(w); at < end; at += kChunk) {
        if (at != seg.start(w)) t.load_chunk(a, x, at, begin, end);
        t.look(a, x);
        uint32_t o[kHeld], set = 0, all;
        t.numbers(true, o);
        fixed += __popc(t.fixed);
        missing |= t.missing ? 1u : 0u;
#pragma unroll
        for (int i = 0; i < kHeld; ++i) {  // (0 is none)
            above += o[i] > high ? 1u : 0u;
            at_high += o[i] == high ? 1u : 0u;
            at_low += o[i] == low && o[i] != high && o[i] != 0u ? 1u : 0u;
            set |= o[i] > low && o[i] < high ? 1u << i : 0u;
        }
        uint32_t to = listed + before(__popc(set), all, sh, turn);
        listed += all;
#pragma unroll
        for (int i = 0; i < kHeld; ++i)
            if (set >> i & 1u) list[to++] = o[i];
    }
    Counts c{low, high, 0, 0, listed, 0, 0, 0};  // (all threads have the same `listed`)
    sums(above, at_high, at_low, sh, turn);
    sums(fixed, missing, listed, sh, turn);
    c.above = above, c.at_high = at_high, c.at_low = at_low, c.fixed = fixed, c.missing = missing;
    if (tid == 0) counts[pair * kMostSegments + w] = c;
}

// How many of the ascending starts[0 .. n - 1] are at most e, for a wave together.
__device__ __forceinline__ int votes_upto(const uint32_t *starts, int n, uint32_t e, int lane) {
    static_assert(kMostSegments <= 2 * kWave, "two a lane");
    return static_cast<int>(votes(lane < n && starts[lane < n ? lane : 0] <= e) +
                            votes(lane + kWave < n && starts[lane + kWave < n ? lane + kWave : 0] <= e));
}

// The second one: the border, and each segment's sources or targets.
__global__ __launch_bounds__(kThreads, 4) void k_evict_list(EvictArgs a, const Counts *counts, const uint32_t *lists, int64_t size,
                                                         Moves moves) {
    __shared__ Shared sh;
    __shared__ Counts held[kMostSegments];
    __shared__ uint32_t over[kMostSegments], even[kMostSegments];  // over and at the border, of each segment
    __shared__ uint32_t starts[kMostSegments + 1];                 // of the listed numbers
    const int tid = static_cast<int>(threadIdx.x), lane = tid & (kWave - 1);
    const int wave = __builtin_amdgcn_readfirstlane(tid / kWave);
    int turn = 0;
    clear(sh);
    const int64_t pair = pair_of();
    if (pair >= a.S * a.kv_heads) return;
    Head x = head_of(a, pair);
    const Segments seg(x, size);
    const int w = static_cast<int>(blockIdx.y);
    const int64_t begin = seg.begin(x, w), end = seg.end(x, w);
    uint32_t above = 0, at_high = 0, between = 0, at_low = 0, fixed = 0, missing = 0;
    if (!x.leave) {
        if (tid < seg.all) held[tid] = counts[pair * kMostSegments + tid], over[tid] = even[tid] = 0;
        __syncthreads();
        for (int i = 0; i < seg.all; ++i) {
            if (tid == 0) starts[i] = between;
            above += held[i].above, at_high += held[i].at_high, between += held[i].between, at_low += held[i].at_low;
            fixed += held[i].fixed, missing += held[i].missing;
        }
        x.leave = missing != 0u;
    }
    if (w == 0 && tid == 0) {
        if (x.h == 0) put_len(a, x);
        if (x.leave || x.keep == 0) moves.count[pair] = 0;
    }
    if (x.leave) {  // (its length may be more than max_keys, which the grid is for)
        for (int64_t from = w * size; from < x.n; from += gridDim.y * size)
            carry_all(a, x, from, from + size < x.n ? from + size : x.n);
        return;
    }
    if (w >= seg.all || x.keep == 0) return;
    if (tid == 0) starts[seg.all] = between;
    Held<> t;  // the segment's own tokens, on their way while the border is looked for
    t.load_chunk(a, x, seg.start(w), begin, end);
    __syncthreads();
    const uint32_t keep = static_cast<uint32_t>(x.keep), low = held[0].low, high = held[0].high;
    const bool few = fixed <= keep;
    Border border;
    // The segments of the 64 listed numbers from e0 on, a lane each (all lanes of the wave together).
    auto segment_of = [&](uint32_t e0) {
        const uint32_t end = e0 + kWave - 1 < between ? e0 + kWave - 1 : between - 1;
        int of = votes_upto(starts, seg.all, e0, lane) - 1, next = of + 1;
        for (; next < seg.all && starts[next] <= end; ++next) of = starts[next] <= e0 + lane ? next : of;
        return of;
    };
    auto listed = [&](uint32_t e0, int of) {
        const uint32_t e = e0 + lane < between ? e0 + lane : between - 1;
        return lists[pair * a.max_keys + seg.begin(x, of) + (e - starts[of])];
    };
    if (few && keep > above && keep <= above + at_high) {
        border = Border{high, keep - above};
        if (tid < seg.all) over[tid] = held[tid].above, even[tid] = held[tid].at_high;
    } else if (few && keep > above + at_high && keep <= above + at_high + between) {
        // As many as the registers hold are read once, the others again and again.
        uint32_t o[kHeld];
        int segment[kHeld];
        auto at = [&](int r) { return static_cast<uint32_t>((r * kWaves + wave) * kWave); };
#pragma unroll
        for (int r = 0; r < kHeld; ++r) segment[r] = at(r) < between ? segment_of(at(r)) : 0;
#pragma unroll
        for (int r = 0; r < kHeld; ++r) {
            o[r] = 0u;
            if (at(r) < between) o[r] = listed(at(r), segment[r]);
        }
        uint32_t least = 0xffffffffu, largest = 0u, sum = 0;
#pragma unroll
        for (int r = 0; r < kHeld; ++r) {
            if (at(r) + lane >= between) o[r] = 0u;
            if (o[r] != 0u) least = min(least, o[r]), largest = max(largest, o[r]);
        }
        auto rest = [&](auto f) {
            for (uint32_t e = at(kHeld); e < between; e += kThreads) {
                const int of = segment_of(e);
                const uint32_t n = listed(e, of);
                f(e + lane < between ? n : 0u, of);
            }
        };
        if (between > static_cast<uint32_t>(kChunk)) least = low + 1u, largest = high;
        reduce(sum, least, largest, sh, turn);
        border = border_of(
            keep - above - at_high, least, largest,
            [&](auto count) {
#pragma unroll
                for (int r = 0; r < kHeld; ++r) count(o[r]);
                rest([&](uint32_t n, int) { count(n); });
            },
            sh, turn);
        if (tid < seg.all) over[tid] = held[tid].above + held[tid].at_high;
        __syncthreads();
        auto sort = [&](uint32_t n, int of) {  // by segments: most often the wave's are all of one
            const int one = __builtin_amdgcn_readfirstlane(of);
            if (__all(of == one)) {
                const uint32_t more = votes(n > border.over), same = votes(n == border.over && n != 0u);
                if (lane == 0 && more != 0u) atomicAdd(&over[one], more);
                if (lane == 0 && same != 0u) atomicAdd(&even[one], same);
            } else {
                if (n > border.over) atomicAdd(&over[of], 1u);
                if (n == border.over && n != 0u) atomicAdd(&even[of], 1u);
            }
        };
#pragma unroll
        for (int r = 0; r < kHeld; ++r)
            if (at(r) < between) sort(o[r], segment[r]);
        rest(sort);
    } else if (few && keep > above + at_high + between && keep <= above + at_high + between + at_low) {
        border = Border{low, keep - above - at_high - between};
        if (tid < seg.all) {
            over[tid] = held[tid].above + held[tid].at_high + held[tid].between;
            even[tid] = held[tid].at_low;
        }
    } else {  // the two numbers do not hold it, or as many tokens are protected as stay, or more
        auto all_of_them = [&](auto f) {
            for (int64_t at = 4 * tid; at < x.n; at += kRow) {
                Held<1> four;
                const int64_t j[1] = {at};
                four.load(a, x, j, 0, x.n);
                four.look(a, x);
                uint32_t o[4];
                four.numbers(few, o);
#pragma unroll
                for (int i = 0; i < 4; ++i) f(o[i], at + i);
            }
        };
        border = border_of(keep, 1u, 0xffffffffu, [&](auto count) { all_of_them([&](uint32_t o, int64_t) { count(o); }); }, sh, turn);
        all_of_them([&](uint32_t o, int64_t j) {
            if (o > border.over) atomicAdd(&over[seg.of(x, j)], 1u);
            if (o == border.over && o != 0u) atomicAdd(&even[seg.of(x, j)], 1u);
        });
    }
    __syncthreads();
    // Of those at the border the first ones stay; and what comes before this segment.
    uint32_t left = border.even, stays = 0, first = 0, all = 0;
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
    const bool below = w < seg.below;
    int32_t *out = moves.from + (pair * 2 + (below ? 1 : 0)) * moves.most;
    uint32_t first_even = 0;
    for (int64_t at = seg.start(w); at < end; at += kChunk) {
        if (at != seg.start(w)) t.load_chunk(a, x, at, begin, end);
        t.look(a, x);
        if (below && carries(a) && t.in != 0u) t.carry(a, x, t.in);
        uint32_t o[kHeld], kept = 0, at_it = 0, before_it[kGroups], total, none = 0;
        t.numbers(few, o);
#pragma unroll
        for (int i = 0; i < kHeld; ++i) {
            kept |= o[i] > border.over ? 1u << i : 0u;
            at_it |= o[i] == border.over ? 1u << i : 0u;
        }
        at_it &= t.in;
        if (border.even != 0) {
            before_groups(at_it, before_it, total, none, sh, turn);
#pragma unroll
            for (int i = 0; i < kHeld; ++i)
                if (at_it >> i & 1u) kept |= first_even + before_it[i / 4]++ < stays ? 1u << i : 0u;
            first_even += total;
        }
        before_groups(kept, before_it, total, none, sh, turn);
        // Below the budget, whose segments begin with a token of theirs, a target has before it what is not kept.
        each_bit<false>(below ? t.in & ~kept : kept, [&](int i) {
            const int64_t j = Held<>::token(at, i);
            const uint32_t k = kept_before(kept, before_it, i);
            out[first + (below ? static_cast<uint32_t>(j - at) - k : k)] = static_cast<int32_t>(j);
        });
        first += below ? static_cast<uint32_t>((end - at < kChunk ? end - at : kChunk)) - total : total;
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
    const dim3 grid(static_cast<unsigned>(heads < kGrid ? heads : kGrid), 1, static_cast<unsigned>((heads + kGrid - 1) / kGrid));
    if (a.max_keys <= kChunk) {
        // Moves by the head's own workgroup where there are heads enough to fill the CUs with them, or few tokens. (8 heads, a
        // step over 4,000 tokens 9.8 us, 12.3 in two launches; to half of them 25.0 and 15.1; of 2,000 16.0 and 13.2, a step of
        // 1,025 7.4 and 9.8.  128 heads of 4,000 48.7 and 51.0, of 8,000 to a quarter 72.8 and 64.5; 256 104 and 108.)
        if (a.max_keys <= 2048 || a.max_keys <= 32 * heads) {
            k_evict_held<true, CHUNKS><<<grid, kThreads, 0, stream>>>(a, moves);
            return hipGetLastError();
        }
        k_evict_held<false, CHUNKS><<<grid, kThreads, 0, stream>>>(a, moves);
    } else {
        Counts *counts = reinterpret_cast<Counts *>(workspace + p.off_counts);
        uint32_t *lists = reinterpret_cast<uint32_t *>(workspace + p.off_lists);
        const dim3 segments(grid.x, static_cast<unsigned>(p.segments), grid.z);
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
