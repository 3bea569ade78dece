// Drawing a token of a row: temperature, top-k, top-p, min-p, and the inverse
// of the running weight at a given uniform number.
//
// Weights are w_i = exp((x_i - max) / T) of logits or (x_i / max)^(1 / T) of
// probabilities, in 64 bits, and are summed as whole numbers of 2^-s of the
// largest one (2^s <= 2^62 / V, so no sum overflows).  Whole numbers add up to
// the same sum in any order, so the outcome depends neither on how a row is
// cut nor on the order of atomics; what a weight loses is under 2^-(s+1) of
// the largest, 2^-46 for 131,072 tokens, which moves the drawn token for one
// row in 10^7.  (In 32 bits it would for one row in 50.)
//
// Every filter keeps a first part of one order: larger x first, the lower
// index first among equals.  A cut in it is a value and how many of the
// elements equal to it stay (the ones with the lowest indexes).  A cut is
// found on the 32-bit keys that order like the values, eleven bits a pass,
// from the largest down: a histogram of counts (top-k) or of weights (top-p).
#include "knnlm_device.h"
#include "lm_internal.h"

namespace knnlm {

namespace {

constexpr int kThreads = 1024;
constexpr int kWaves = kThreads / kWave;
constexpr int kBins = 2048;

template <knn_dtype DT>
__device__ __forceinline__ float element(const void *row, int i) {
    if constexpr (DT == KNN_F32) return static_cast<const float *>(row)[i];
    if constexpr (DT == KNN_BF16)
        return __uint_as_float(static_cast<uint32_t>(static_cast<const uint16_t *>(row)[i]) << 16);
    return static_cast<float>(static_cast<const _Float16 *>(row)[i]);
}

// A key that orders like x; 0 where x is absent (NaN, -inf; of probabilities
// also what is not above 0).
__device__ __forceinline__ uint32_t key_of(float x, bool probabilities) {
    if (!(x > (probabilities ? 0.0f : -INFINITY))) return 0;
    const uint32_t b = __float_as_uint(x == 0.0f ? 0.0f : x);
    return b ^ ((b >> 31) != 0 ? 0xffffffffu : 0x80000000u);
}

__device__ __forceinline__ float value_of(uint32_t key) {
    return __uint_as_float(key ^ ((key >> 31) != 0 ? 0x80000000u : 0xffffffffu));
}

// The weights of a row, as a function of the key.
struct Weights {
    double top;      // the largest value
    double inv_t;
    double scale;    // 2^s, or 2^s over the largest value's power of two where the values are the weights
    double least;    // min-p
    bool probabilities, plain, flat;  // plain: probabilities at T = 1; flat: the largest is infinite

    __device__ __forceinline__ double of(uint32_t key) const {  // the largest one's is 2^s (plain: at most)
        const double x = value_of(key);
        if (flat) return scale;
        if (plain) return x * scale;
        return exp((probabilities ? log(x / top) : x - top) * inv_t) * scale;
    }
    __device__ __forceinline__ uint64_t whole(double w) const { return static_cast<uint64_t>(w + 0.5); }
    __device__ __forceinline__ bool heavy(double w) const { return w >= least * (plain ? top * scale : scale); }
};

struct Shared {
    uint64_t mass[kBins];
    uint32_t count[kBins];
    uint64_t part[kWaves];
    uint32_t part32[kWaves];
    uint64_t answer64;
    uint32_t answer, answer2;
};

__device__ __forceinline__ uint64_t wave_sum64(uint64_t v) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o);
    return v;
}
__device__ __forceinline__ uint32_t wave_sum32(uint32_t v) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o);
    return v;
}

__device__ __forceinline__ uint64_t block_sum64(uint64_t v, Shared &sh) {
    v = wave_sum64(v);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) sh.part[threadIdx.x >> 6] = v;
    __syncthreads();
    uint64_t r = 0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) r += sh.part[w];
    return r;
}

// The key at which the running count (or weight) from the largest key down
// first reaches `goal`, given that it does: {key, what lies above it}.  Keys
// under `floor_key` do not count.
template <bool MASS, typename Each>
__device__ uint32_t descend(double goal, uint32_t floor_key, const Weights &w, Shared &sh, Each each, uint64_t &above) {
    uint32_t prefix = 0;
    above = 0;
    for (int level = 0; level < 3; ++level) {
        const int shift = level == 0 ? 21 : level == 1 ? 10 : 0, bits = level == 2 ? 10 : 11;
        const uint32_t mask = (1u << bits) - 1;
        __syncthreads();
        for (int i = threadIdx.x; i < kBins; i += kThreads) {
            if constexpr (MASS) sh.mass[i] = 0; else sh.count[i] = 0;
        }
        __syncthreads();
        each([&](uint32_t key) {
            if (key == 0 || key < floor_key) return;
            if (level > 0 && (key >> (shift + bits)) != prefix) return;
            const uint32_t bin = (key >> shift) & mask;
            if constexpr (MASS)
                atomicAdd(reinterpret_cast<unsigned long long *>(&sh.mass[bin]), static_cast<unsigned long long>(w.whole(w.of(key))));
            else
                atomicAdd(&sh.count[bin], 1u);
        });
        __syncthreads();
        // One wave walks the bins down, 64 at a time.
        if (threadIdx.x < kWave) {
            const int lane = threadIdx.x;
            uint64_t run = above;
            uint32_t found = 0;
            uint64_t before = above;
            bool done = false;
            for (int b = static_cast<int>(mask); b >= 0 && !done; b -= kWave) {
                const int bin = b - lane;
                const uint64_t v = MASS ? sh.mass[bin] : static_cast<uint64_t>(sh.count[bin]);
                uint64_t incl = v;
#pragma unroll
                for (int o = 1; o < kWave; o <<= 1) {
                    const uint64_t up = __shfl_up(incl, o);
                    if (lane >= o) incl += up;
                }
                const uint64_t hit = __ballot(v != 0 && static_cast<double>(run + incl) >= goal);
                const uint64_t some = __ballot(v != 0);
                if (some != 0) {  // where the goal is never reached (by a rounding), the last bin with anything
                    const int lane_at = hit != 0 ? __ffsll(static_cast<unsigned long long>(hit)) - 1
                                                 : 63 - __clzll(static_cast<long long>(some));
                    found = static_cast<uint32_t>(b - lane_at);
                    before = run + __shfl(incl - v, lane_at);
                    done = hit != 0;
                }
                run += __shfl(incl, 63);
            }
            if (lane == 0) {
                sh.answer = found;
                sh.answer64 = before;
            }
        }
        __syncthreads();
        prefix = (prefix << bits) | sh.answer;
        above = sh.answer64;
    }
    return prefix;
}

template <knn_dtype DT>
__global__ __launch_bounds__(kThreads) void k_sample(SampleArgs a, int log2_scale) {
    __shared__ Shared sh;
    const int64_t r = blockIdx.x;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const char *row = static_cast<const char *>(a.scores) + r * a.stride * (DT == KNN_F32 ? 4 : 2);
    const int V = a.V;
    // The waves take consecutive pieces of the row, so that what lies before an element is known by wave.
    const int piece = (V + kWaves - 1) / kWaves;
    const int i0 = min(V, wave * piece), i1 = min(V, i0 + piece);
    auto each = [&](auto f) {
        for (int i = i0 + lane; i < i1; i += kWave) f(key_of(element<DT>(row, i), a.probabilities));
    };

    uint32_t top = 0;
    each([&](uint32_t key) { top = max(top, key); });
    top = wave_allmax_u32(top);
    if (lane == 0) sh.part32[wave] = top;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kWaves; ++w) top = max(top, sh.part32[w]);
    if (top == 0) {
        if (threadIdx.x == 0) {
            a.token[r] = -1;
            if (a.prob != nullptr) a.prob[r] = 0.0f;
            if (a.kept != nullptr) a.kept[r] = 0;
        }
        return;
    }
    const float t = a.temperature != nullptr ? a.temperature[r] : 1.0f;
    const bool greedy = !(t > 0.0f);
    Weights w{};
    w.top = value_of(top);
    w.inv_t = 1.0 / static_cast<double>(t);
    w.probabilities = a.probabilities;
    w.flat = value_of(top) == INFINITY;
    w.plain = !w.flat && a.probabilities && t == 1.0f;
    w.scale = ldexp(1.0, log2_scale - (w.plain ? ilogb(w.top) + 1 : 0));
    const float least = a.min_p != nullptr ? a.min_p[r] : 0.0f;
    w.least = least > 0.0f ? fmin(static_cast<double>(least), 1.0) : 0.0;

    // The cut: keys above `cut` stay, and the first `rest` of those equal to it.
    uint32_t cut = w.flat ? top - 1 : 0;
    uint64_t rest = 0;
    if (greedy) {
        cut = top;
        rest = 1;
    }
    const uint32_t floor_key = cut + 1;  // what counts at all
    const int k = a.top_k != nullptr ? a.top_k[r] : 0;
    if (!greedy && k > 0 && k < V) {
        uint32_t n = 0;
        each([&](uint32_t key) { n += key >= floor_key ? 1u : 0u; });
        if (static_cast<uint64_t>(k) < block_sum64(n, sh)) {
            uint64_t above;
            cut = descend<false>(static_cast<double>(k), floor_key, w, sh, each, above);
            rest = static_cast<uint64_t>(k) - above;
        }
    }
    const float p = a.top_p != nullptr ? a.top_p[r] : 1.0f;
    if (!greedy && p < 1.0f) {
        if (!(p > 0.0f)) {
            cut = top;
            rest = 1;
        } else {
            uint64_t sum = 0;
            each([&](uint32_t key) { sum += key > cut ? w.whole(w.of(key)) : 0; });
            sum = block_sum64(sum, sh);
            if (rest > 0) sum += rest * w.whole(w.of(cut));
            const double goal = static_cast<double>(p) * static_cast<double>(sum);
            uint64_t above;
            const uint32_t at = descend<true>(goal, rest > 0 ? cut : cut + 1, w, sh, each, above);
            const uint64_t one = w.whole(w.of(at));
            uint64_t n = 1;
            if (one > 0 && goal > static_cast<double>(above)) {
                n = static_cast<uint64_t>((goal - static_cast<double>(above)) / static_cast<double>(one));
                while (static_cast<double>(above + n * one) < goal) ++n;
                while (n > 1 && static_cast<double>(above + (n - 1) * one) >= goal) --n;
            }
            rest = at == cut && n > rest ? rest : n;
            cut = at;
        }
    }

    // Elements equal to the cut before each wave's piece, then in index order: what stays, and its weight.
    uint32_t ties = 0;
    if (rest > 0) {
        each([&](uint32_t key) { ties += key == cut ? 1u : 0u; });
        ties = wave_sum32(ties);
        __syncthreads();
        if (lane == 0) sh.part32[wave] = ties;
        __syncthreads();
        ties = 0;
        for (int v = 0; v < wave; ++v) ties += sh.part32[v];
    }
    auto ordered = [&](auto f) {  // f(index, weight or 0) for the wave's piece, 64 consecutive elements at a time
        uint64_t run = ties;
        for (int base = i0; base < i1; base += kWave) {
            const int i = base + lane;
            const uint32_t key = i < i1 ? key_of(element<DT>(row, i), a.probabilities) : 0;
            bool stays = key > cut;
            if (rest > 0) {
                const uint64_t eq = __ballot(i < i1 && key == cut);
                stays |= i < i1 && key == cut && run + __popcll(eq & ((1ull << lane) - 1)) < rest;
                run += __popcll(eq);
            }
            double x = 0.0;
            if (stays) {
                x = greedy ? w.scale : w.of(key);
                stays = w.heavy(x) || greedy;
            }
            if (f(i, stays, stays ? w.whole(x) : 0, x)) break;
        }
    };
    uint64_t sum = 0;
    uint32_t n = 0;
    ordered([&](int, bool stays, uint64_t q, double) {
        sum += q;
        n += stays ? 1u : 0u;
        return false;
    });
    sum = wave_sum64(sum);
    n = wave_sum32(n);
    __syncthreads();
    if (lane == 0) {
        sh.part[wave] = sum;
        sh.part32[wave] = n;
    }
    __syncthreads();
    uint64_t total = 0, mine = 0;
    uint32_t kept = 0;
    for (int v = 0; v < kWaves; ++v) {
        if (v == wave) mine = total;
        total += sh.part[v];
        kept += sh.part32[v];
    }
    if (threadIdx.x == 0 && a.kept != nullptr) a.kept[r] = static_cast<int32_t>(kept);
    const float u = a.uniforms[r];
    const double aim = (u > 0.0f ? fmin(static_cast<double>(u), 1.0) : 0.0) * static_cast<double>(total);
    uint64_t goal = static_cast<uint64_t>(aim);  // the token is the first whose running weight exceeds it
    if (goal >= total) goal = total - 1;
    if (goal < mine || goal >= mine + sum) return;
    ordered([&](int i, bool, uint64_t q, double x) {
        uint64_t incl = q;
#pragma unroll
        for (int o = 1; o < kWave; o <<= 1) {
            const uint64_t up = __shfl_up(incl, o);
            if (lane >= o) incl += up;
        }
        const uint64_t hit = __ballot(mine + incl > goal);
        if (hit != 0) {
            if (lane == __ffsll(static_cast<unsigned long long>(hit)) - 1) {
                a.token[r] = i;
                if (a.prob != nullptr) a.prob[r] = static_cast<float>(x / static_cast<double>(total));
            }
            return true;
        }
        mine += __shfl(incl, 63);
        return false;
    });
}

}  // namespace

hipError_t launch_sample(const SampleArgs &a, knn_dtype dtype, void *, hipStream_t stream) {
    int bits = 0;
    while ((int64_t{1} << bits) < a.V) ++bits;
    const dim3 grid(static_cast<unsigned>(a.rows));
    switch (dtype) {
    case KNN_F32: k_sample<KNN_F32><<<grid, kThreads, 0, stream>>>(a, 62 - bits); break;
    case KNN_BF16: k_sample<KNN_BF16><<<grid, kThreads, 0, stream>>>(a, 62 - bits); break;
    default: k_sample<KNN_F16><<<grid, kThreads, 0, stream>>>(a, 62 - bits); break;
    }
    return hipGetLastError();
}

}  // namespace knnlm
