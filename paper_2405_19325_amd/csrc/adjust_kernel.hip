// Penalties for repeated tokens, biases and the tokens that a grammar allows,
// on rows of logits or probabilities.
//
// A workgroup takes a slice of a row's tokens, 8 of them a thread, whose scores
// are on their way from memory while it counts in LDS how often each token is
// in the row's history and in the drafts that the row sees (integer atomics: the
// same counts in any order), and finds the last bias of each (the largest
// entry).
//
// Logits are worked out in 32 bits where they are held.  Probabilities are
// worked out as logarithms in 64 bits, since the logarithm of a small one times
// a penalty, in 32 bits, would be off by 2^-18 of the outcome; the few tokens
// that are touched are listed first, so that all lanes have one.
#include "knnlm_device.h"
#include "lm_internal.h"

namespace knnlm {

namespace {

constexpr int64_t kGrid = 1 << 20;      // rows of a row of the grid
constexpr int kPer = 8;                 // tokens of a thread
constexpr uint32_t kPrompt = 1u << 31;  // beside a token's count: it is in the prompt

template <knn_dtype DT>
struct Type {
    static constexpr int SIZE = DT == KNN_F32 ? 4 : 2;
    static constexpr int VEC = 16 / SIZE;          // of 16 bytes
    static constexpr int GROUPS = kPer / VEC;      // of a thread
    __device__ static __forceinline__ float widen(const u32x4_t &v, int e) {
        if constexpr (DT == KNN_F32) return __uint_as_float(v[e]);
        const uint32_t h = e % 2 != 0 ? v[e / 2] >> 16 : v[e / 2] & 0xffffu;
        if constexpr (DT == KNN_BF16) return __uint_as_float(h << 16);
        return static_cast<float>(__builtin_bit_cast(_Float16, static_cast<uint16_t>(h)));
    }
    __device__ static __forceinline__ uint32_t narrow(float x) {  // to nearest, ties to even
        if constexpr (DT == KNN_F32) return __float_as_uint(x);
        if constexpr (DT == KNN_BF16) return __builtin_bit_cast(uint16_t, static_cast<__bf16>(x));
        return __builtin_bit_cast(uint16_t, static_cast<_Float16>(x));
    }
    __device__ static __forceinline__ void put(u32x4_t &v, int e, float x) {
        if constexpr (DT == KNN_F32) v[e] = narrow(x);
        else v[e / 2] = e % 2 != 0 ? (v[e / 2] & 0xffffu) | narrow(x) << 16 : (v[e / 2] & 0xffff0000u) | narrow(x);
    }
    __device__ static __forceinline__ uint32_t raw(const void *p, int64_t i) {
        if constexpr (DT == KNN_F32) return static_cast<const uint32_t *>(p)[i];
        return static_cast<const uint16_t *>(p)[i];
    }
    __device__ static __forceinline__ void set(void *p, int64_t i, uint32_t x) {
        if constexpr (DT == KNN_F32) static_cast<uint32_t *>(p)[i] = x;
        else static_cast<uint16_t *>(p)[i] = static_cast<uint16_t>(x);
    }
};

// What a row's parameters make of a score.
struct Rule {
    float repetition, presence, frequency;  // 1, 0, 0: off

    template <class T>
    __device__ __forceinline__ T of(T x, uint32_t seen, bool biased, float bias) const {
        const uint32_t c = seen & ~kPrompt;
        if (seen != 0u) x = x > T(0) ? x / T(repetition) : x * T(repetition);
        if (c != 0u) x = x - T(presence) - T(c) * T(frequency);
        if (biased) x += T(bias);
        return x;
    }
};

__device__ __forceinline__ float parameter(const float *p, int64_t t, float off) {
    const float x = p != nullptr ? p[t] : off;
    return isfinite(x) ? x : off;
}

// LAZY: in place and without a mask, where only touched scores are read.
template <knn_dtype DT, bool PROBS, bool LAZY, int THREADS>
__global__ __launch_bounds__(THREADS) void k_adjust(AdjustArgs a) {
    using Ty = Type<DT>;
    constexpr int SLICE = kPer * THREADS, VEC = Ty::VEC, GROUPS = Ty::GROUPS;
    extern __shared__ __align__(16) uint32_t lds[];  // counts [slice], then where there are biases the last of each [slice]
    __shared__ uint16_t touched[PROBS ? SLICE : 1];
    __shared__ uint32_t n_touched;
    uint32_t *seen = lds;
    int32_t *last = reinterpret_cast<int32_t *>(lds + SLICE);
    const int tid = static_cast<int>(threadIdx.x);
    const bool counts = a.history != nullptr || a.row_tokens != nullptr, biased = a.bias_tokens != nullptr;
    const uint32_t off = PROBS ? 0u : Ty::narrow(-INFINITY);
    const int64_t t = static_cast<int64_t>(blockIdx.z) * kGrid + blockIdx.x;
    if (t >= a.rows) return;
    int64_t s = t, first = t;
    if (a.row_offsets != nullptr) {
        if (t >= a.row_offsets[a.S]) return;
        s = set_of_query(a.row_offsets, a.S, t);
        first = a.row_offsets[s];
    }
    const char *in = static_cast<const char *>(a.scores) + t * a.stride * Ty::SIZE;
    char *out = static_cast<char *>(a.out) + t * a.out_stride * Ty::SIZE;
    // Places are counted from the 16 bytes that hold the first score; place p is token p - lead.
    const int lead = static_cast<int>(reinterpret_cast<uintptr_t>(in) % 16) / Ty::SIZE;
    const int p0 = static_cast<int>(blockIdx.y) * SLICE, v0 = p0 - lead;
    if (v0 >= a.V) return;
    const bool even = (reinterpret_cast<uintptr_t>(out) - reinterpret_cast<uintptr_t>(in)) % 16 == 0;
    u32x4_t x[GROUPS];
    uint32_t may[GROUPS];  // a bit a token: it is allowed
    auto group = [&](int g) { return (g * THREADS + tid) * VEC; };  // place in the slice
    auto fetch = [&](int g) {
        const int v = v0 + group(g);
        if (v >= 0 && v + VEC <= a.V) {
            x[g] = *reinterpret_cast<const u32x4_t *>(in + static_cast<int64_t>(v) * Ty::SIZE);
        } else {
            x[g] = u32x4_t{0, 0, 0, 0};
#pragma unroll
            for (int e = 0; e < VEC; ++e)
                if (v + e >= 0 && v + e < a.V) {
                    if constexpr (DT == KNN_F32) x[g][e] = Ty::raw(in, v + e);
                    else x[g][e / 2] |= Ty::raw(in, v + e) << (e % 2 * 16);
                }
        }
    };
#pragma unroll
    for (int g = 0; g < GROUPS; ++g) {
        if constexpr (!LAZY) fetch(g);
        may[g] = ~0u;
        if (!LAZY && a.allowed != nullptr) {
            const int words = (a.V + 31) / 32, v = v0 + group(g);
            const uint32_t *row = a.allowed + t * words;
            const int w = v < 0 ? 0 : v >> 5, lo = w < words ? w : words - 1, hi = w + 1 < words ? w + 1 : words - 1;
            const uint64_t both = static_cast<uint64_t>(row[lo]) | static_cast<uint64_t>(row[hi]) << 32;
            may[g] = static_cast<uint32_t>(v < 0 ? both << -v : both >> (v & 31));
        }
    }
    for (int i = tid; i < SLICE; i += THREADS) {
        if (counts) seen[i] = 0u;
        if (biased) last[i] = -1;
    }
    if (tid == 0) n_touched = 0;
    __syncthreads();
    auto at = [&](int64_t v) {  // the place of a token in this slice; -1: in another, or none
        const int64_t p = v - v0;
        return v >= 0 && v < a.V && p >= 0 && p < SLICE ? static_cast<int>(p) : -1;
    };
    if (a.history != nullptr) {
        const int64_t len = a.history_lens[s] < a.history_width ? a.history_lens[s] : a.history_width;
        const int64_t prompt = a.prompt_lens != nullptr ? a.prompt_lens[s] : 0;
        const int32_t *history = a.history + s * a.history_width;
        for (int64_t i0 = tid; i0 < len; i0 += kPer * THREADS) {
            int32_t v[kPer];
#pragma unroll
            for (int u = 0; u < kPer; ++u) v[u] = history[i0 + u * THREADS < len ? i0 + u * THREADS : i0];
#pragma unroll
            for (int u = 0; u < kPer; ++u) {
                const int64_t i = i0 + u * THREADS;
                const int p = i < len ? at(v[u]) : -1;
                if (p >= 0 && i < prompt) atomicOr(&seen[p], kPrompt);
                if (p >= 0 && i >= prompt) atomicAdd(&seen[p], 1u);
            }
        }
    }
    if (a.row_tokens != nullptr) {
        int64_t rows = a.row_offsets != nullptr ? a.row_offsets[s + 1] : t + 1;
        rows = (rows < a.rows ? rows : a.rows) - first;
        if (a.tree_mask == nullptr) rows = t - first + 1;
        else if (rows > 32 * a.mask_words) rows = 32 * a.mask_words;
        for (int64_t i = tid; i < rows; i += THREADS) {
            const bool sees = a.tree_mask == nullptr || (a.tree_mask[t * a.mask_words + (i >> 5)] >> (i & 31) & 1u) != 0u;
            const int p = at(a.row_tokens[first + i]);
            if (sees && p >= 0) atomicAdd(&seen[p], 1u);
        }
    }
    if (biased)
        for (int64_t i = tid; i < a.bias_width; i += THREADS) {
            const int p = at(a.bias_tokens[s * a.bias_width + i]);
            if (p >= 0) atomicMax(&last[p], static_cast<int32_t>(i));
        }
    Rule rule{parameter(a.repetition, t, 1.0f), parameter(a.presence, t, 0.0f), parameter(a.frequency, t, 0.0f)};
    if (!(rule.repetition > 0.0f)) rule.repetition = 1.0f;
    __syncthreads();
    const float *biases = a.bias_values + s * a.bias_width;
#pragma unroll
    for (int g = 0; g < GROUPS; ++g) {
        const int v = v0 + group(g);
        uint32_t c[VEC];
        int32_t b[VEC];
        uint32_t any = 0;
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
            c[e] = counts ? seen[group(g) + e] : 0u;
            b[e] = biased ? last[group(g) + e] : -1;
            any |= c[e] != 0u || b[e] >= 0 ? 1u << e : 0u;
        }
        if constexpr (LAZY) {
            if (any == 0u) continue;
            if constexpr (!PROBS) fetch(g);
        }
        uint32_t change = ~may[g] & ((1u << VEC) - 1u);
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
            if (change >> e & 1u) {
                if constexpr (DT == KNN_F32) x[g][e] = off;
                else x[g][e / 2] = e % 2 != 0 ? (x[g][e / 2] & 0xffffu) | off << 16 : (x[g][e / 2] & 0xffff0000u) | off;
            } else if (any >> e & 1u) {
                if constexpr (PROBS) {
                    touched[atomicAdd(&n_touched, 1u)] = static_cast<uint16_t>(group(g) + e);
                } else {
                    Ty::put(x[g], e, rule.of(Ty::widen(x[g], e), c[e], b[e] >= 0, b[e] >= 0 ? biases[b[e]] : 0.0f));
                    change |= 1u << e;
                }
            }
        }
        if (a.out == a.scores && change == 0u) continue;
        if (even && v >= 0 && v + VEC <= a.V) {
            *reinterpret_cast<u32x4_t *>(out + static_cast<int64_t>(v) * Ty::SIZE) = x[g];
        } else {
#pragma unroll
            for (int e = 0; e < VEC; ++e)
                if (v + e >= 0 && v + e < a.V) {
                    if constexpr (DT == KNN_F32) Ty::set(out, v + e, x[g][e]);
                    else Ty::set(out, v + e, x[g][e / 2] >> (e % 2 * 16) & 0xffffu);
                }
        }
    }
    if constexpr (PROBS) {
        __syncthreads();
        for (uint32_t i = tid; i < n_touched; i += THREADS) {
            const int p = touched[i], v = v0 + p;
            const uint32_t raw = Ty::raw(in, v);
            const float from = Ty::widen(u32x4_t{raw, 0, 0, 0}, 0);
            if (!(from > 0.0f)) continue;  // (it was written as it is)
            const int32_t b = biased ? last[p] : -1;
            const double y = rule.of(log(static_cast<double>(from)), counts ? seen[p] : 0u, b >= 0, b >= 0 ? biases[b] : 0.0f);
            Ty::set(out, v, Ty::narrow(static_cast<float>(exp(y))));
        }
    }
}

template <knn_dtype DT, bool PROBS, bool LAZY, int THREADS>
hipError_t launch(const AdjustArgs &a, hipStream_t stream) {
    constexpr int SLICE = kPer * THREADS;
    const int64_t slices = (a.V + Type<DT>::VEC - 1 + SLICE - 1) / SLICE;
    const dim3 grid(static_cast<unsigned>(a.rows < kGrid ? a.rows : kGrid), static_cast<unsigned>(slices),
                    static_cast<unsigned>((a.rows + kGrid - 1) / kGrid));
    k_adjust<DT, PROBS, LAZY, THREADS><<<grid, THREADS, sizeof(uint32_t) * SLICE * (a.bias_tokens != nullptr ? 2 : 1), stream>>>(a);
    return hipGetLastError();
}

template <knn_dtype DT, bool PROBS, bool LAZY>
hipError_t launch(const AdjustArgs &a, hipStream_t stream) {
    if (a.rows * ((a.V + 2047) / 2048) <= 1024) return launch<DT, PROBS, LAZY, 256>(a, stream);
    return launch<DT, PROBS, LAZY, 1024>(a, stream);
}

template <knn_dtype DT>
hipError_t launch(const AdjustArgs &a, hipStream_t stream) {
    const bool lazy = a.out == a.scores && a.allowed == nullptr;
    if (a.probabilities) return lazy ? launch<DT, true, true>(a, stream) : launch<DT, true, false>(a, stream);
    return lazy ? launch<DT, false, true>(a, stream) : launch<DT, false, false>(a, stream);
}

}  // namespace

hipError_t launch_adjust_scores(const AdjustArgs &a, knn_dtype dtype, hipStream_t stream) {
    switch (dtype) {
    case KNN_F32: return launch<KNN_F32>(a, stream);
    case KNN_BF16: return launch<KNN_BF16>(a, stream);
    default: return launch<KNN_F16>(a, stream);
    }
}

}  // namespace knnlm
