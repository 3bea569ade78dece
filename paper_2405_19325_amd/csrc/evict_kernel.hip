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
// and all stay; with more, all others are 0 and none does.  The budget-th
// largest number is found bit by bit.
//
// A workgroup takes a head of a sequence.
#include "lm_device.h"

namespace knnlm {

namespace {

constexpr int kThreads = 1024;
constexpr int kWaves = kThreads / kWave;

// A number that orders like x, NaN first.
__device__ __forceinline__ uint32_t order_of(float x) {
    if (x != x) return 1u;
    const uint32_t b = __float_as_uint(x + 0.0f);  // one zero
    return b ^ ((b >> 31) != 0 ? 0xffffffffu : 0x80000000u);
}

// The sum over the workgroup, for every thread.  `part`: kWaves words.
__device__ __forceinline__ uint32_t block_sum(uint32_t v, uint32_t *part) {
    const int lane = static_cast<int>(threadIdx.x) & (kWave - 1);
    v = wave_incl_scan_u32(v, lane);
    __syncthreads();
    if (lane == kWave - 1) part[threadIdx.x / kWave] = v;
    __syncthreads();
    uint32_t sum = 0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) sum += part[w];
    return sum;
}

// How many threads before this one have `flag`, and how many there are.
__device__ __forceinline__ uint32_t block_rank(bool flag, uint32_t &total, uint32_t *part) {
    const int lane = static_cast<int>(threadIdx.x) & (kWave - 1), wave = static_cast<int>(threadIdx.x) / kWave;
    const uint64_t set = __ballot(flag);
    __syncthreads();
    if (lane == 0) part[wave] = static_cast<uint32_t>(__popcll(set));
    __syncthreads();
    uint32_t before = 0;
    total = 0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
        if (w == wave) before = total;
        total += part[w];
    }
    return before + static_cast<uint32_t>(__popcll(set & ((uint64_t{1} << lane) - 1)));
}

struct Ledger {
    const EvictArgs &a;
    int64_t s;
    int h;
    int64_t recent_from;
    int mode;  // 0: protected ones are above all; 1: others are below all

    __device__ __forceinline__ int64_t place(int64_t j) const { return place_of(a.cache, a.kv_heads, s, h, j); }
    __device__ __forceinline__ bool fixed(int64_t j, int64_t at) const {
        const int64_t p = a.key_positions != nullptr ? a.key_positions[at] : j;
        return p < a.sinks || p >= recent_from;
    }
    __device__ __forceinline__ uint32_t order(int64_t j) const {
        const int64_t at = place(j);
        const bool f = fixed(j, at);
        if (mode == 0) return f ? 0xffffffffu : order_of(a.mass[at]);
        return f ? order_of(a.mass[at]) : 0u;
    }
};

__global__ __launch_bounds__(kThreads) void k_cache_evict(EvictArgs a, int32_t *lists, int64_t most) {
    __shared__ uint32_t part[kWaves];
    const int64_t pair = blockIdx.x;
    const int64_t s = pair / a.kv_heads;
    const int h = static_cast<int>(pair % a.kv_heads);
    const int64_t len = a.cache_lens[s], budget = a.budgets[s];
    const int64_t room = a.cache.table_width << a.cache.page_log2;
    const int64_t limit = a.max_keys < room ? a.max_keys : room;
    const int64_t n = len < 0 ? 0 : len;
    // Left as it is: within the budget, too long, or with a page that is none.
    bool whole = n <= limit;
    const int64_t entries = ((n < limit ? n : limit) + (int64_t{1} << a.cache.page_log2) - 1) >> a.cache.page_log2;
    for (int64_t e = threadIdx.x; e < entries; e += kThreads) {
        const int64_t page = a.cache.pages[s * a.cache.table_width + e];
        if (page < 0 || page >= a.cache.n_pages) whole = false;
    }
    const bool leave = __syncthreads_or(!whole) != 0 || budget < 0 || budget >= n;
    const int64_t K = leave ? n : budget;
    if (h == 0 && threadIdx.x == 0) a.new_lens[s] = static_cast<int32_t>(leave ? len : budget);
    const bool copies = a.mass_out != a.mass, turns = a.positions_out != a.key_positions;
    if (copies || turns) {
        const int64_t upto = K < limit ? K : limit;
        for (int64_t j = threadIdx.x; j < upto; j += kThreads) {
            const int64_t at = place_of(a.cache, a.kv_heads, s, h, j);
            if (at < 0) continue;
            if (copies) a.mass_out[at] = a.mass[at];
            if (turns) a.positions_out[at] = a.key_positions[at];
        }
    }
    if (leave) return;

    const int64_t next = a.next_positions != nullptr ? a.next_positions[s] : len;
    Ledger ledger{a, s, h, next - a.recent, 0};
    uint32_t count = 0;
    for (int64_t j = threadIdx.x; j < n; j += kThreads) count += ledger.fixed(j, ledger.place(j)) ? 1u : 0u;
    ledger.mode = block_sum(count, part) > static_cast<uint64_t>(K) ? 1 : 0;
    uint32_t border = 0;  // the K-th largest number, the largest of which K are as large
    uint32_t above = 0;   // how many are larger
    if (K > 0) {
        for (int bit = 31; bit >= 0; --bit) {
            const uint32_t to = border | 1u << bit;
            count = 0;
            for (int64_t j = threadIdx.x; j < n; j += kThreads) count += ledger.order(j) >= to ? 1u : 0u;
            count = block_sum(count, part);
            if (count >= static_cast<uint64_t>(K)) border = to;
        }
    } else {
        border = 0xffffffffu;
    }
    count = 0;
    for (int64_t j = threadIdx.x; j < n; j += kThreads) count += ledger.order(j) > border ? 1u : 0u;
    above = block_sum(count, part);
    // Of those at the border the first ones stay.
    const int64_t even = K - above;
    int32_t *from = lists + pair * 2 * most, *to = from + most;
    int64_t evens = 0, froms = 0, tos = 0;
    for (int64_t j0 = 0; j0 < n; j0 += kThreads) {
        const int64_t j = j0 + threadIdx.x;
        const uint32_t o = j < n ? ledger.order(j) : 0u;
        uint32_t total;
        const bool at_border = j < n && o == border && K > 0;
        const int64_t rank = evens + block_rank(at_border, total, part);
        evens += total;
        const bool kept = j < n && K > 0 && (o > border || (at_border && rank < even));
        const bool source = kept && j >= K, target = j < K && !kept;
        int64_t r = froms + block_rank(source, total, part);
        froms += total;
        if (source) from[r] = static_cast<int32_t>(j);
        r = tos + block_rank(target, total, part);
        tos += total;
        if (target) to[r] = static_cast<int32_t>(j);
    }
    __syncthreads();
    for (int64_t m = threadIdx.x / kWave; m < froms; m += kWaves) {
        const int lane = static_cast<int>(threadIdx.x) & (kWave - 1);
        const int64_t src = ledger.place(from[m]), dst = ledger.place(to[m]);
        for (int e = lane; e < a.head_dim; e += kWave) {
            uint16_t *k = static_cast<uint16_t *>(a.k_cache), *v = static_cast<uint16_t *>(a.v_cache);
            k[dst * a.head_dim + e] = k[src * a.head_dim + e];
            v[dst * a.head_dim + e] = v[src * a.head_dim + e];
        }
        if (lane == 0) {
            a.mass_out[dst] = a.mass[src];
            if (a.key_positions != nullptr) a.positions_out[dst] = a.key_positions[src];
        }
    }
    if (a.key_positions == nullptr) return;
}

}  // namespace

// The indices that move and where to: no more than half of a head's tokens do.
size_t evict_workspace(int64_t S, int64_t kv_heads, int64_t max_keys) {
    return sizeof(int32_t) * 2 * static_cast<size_t>(S * kv_heads) * static_cast<size_t>(max_keys / 2 + 1);
}

hipError_t launch_cache_evict(const EvictArgs &a, void *workspace, hipStream_t stream) {
    k_cache_evict<<<dim3(static_cast<unsigned>(a.S * a.kv_heads)), kThreads, 0, stream>>>(
        a, static_cast<int32_t *>(workspace), a.max_keys / 2 + 1);
    return hipGetLastError();
}

}  // namespace knnlm
