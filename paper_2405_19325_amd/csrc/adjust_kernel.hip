// Penalties for repeated tokens, biases and the tokens that a grammar allows,
// on rows of logits or probabilities.
//
// A workgroup takes a slice of a row's tokens.  It counts in LDS how often each
// of them is in the row's history and in the drafts that the row sees (integer
// atomics: the same counts in any order), and finds the last bias of each (the
// largest entry), then goes over the slice once.  Logits are worked out in 32
// bits; probabilities as logarithms in 64, since a small one's logarithm times
// a penalty, in 32 bits, would be off by 2^-18 of the outcome.
#include "knnlm_device.h"
#include "lm_internal.h"

namespace knnlm {

namespace {

constexpr int kThreads = 1024;
constexpr int kSlice = 8192;             // tokens of a workgroup
constexpr uint32_t kPrompt = 1u << 31;   // beside a token's count: it is in the prompt

template <knn_dtype DT>
__device__ __forceinline__ float element(const void *row, int64_t i) {
    if constexpr (DT == KNN_F32) return static_cast<const float *>(row)[i];
    if constexpr (DT == KNN_BF16)
        return __uint_as_float(static_cast<uint32_t>(static_cast<const uint16_t *>(row)[i]) << 16);
    return static_cast<float>(static_cast<const _Float16 *>(row)[i]);
}

// To nearest, ties to even.
template <knn_dtype DT>
__device__ __forceinline__ void put(void *row, int64_t i, float x) {
    if constexpr (DT == KNN_F32) static_cast<float *>(row)[i] = x;
    if constexpr (DT == KNN_BF16) static_cast<__bf16 *>(row)[i] = static_cast<__bf16>(x);
    if constexpr (DT == KNN_F16) static_cast<_Float16 *>(row)[i] = static_cast<_Float16>(x);
}

// What a row's parameters make of a score.
struct Rule {
    float repetition, presence, frequency;  // 1, 0, 0: off

    template <class T>
    __device__ __forceinline__ T steps(T x, uint32_t seen, bool biased, float bias) const {
        const uint32_t c = seen & ~kPrompt;
        if (seen != 0u) x = x > T(0) ? x / T(repetition) : x * T(repetition);
        if (c != 0u) x = x - T(presence) - T(c) * T(frequency);
        if (biased) x += T(bias);
        return x;
    }
    __device__ __forceinline__ float of(float x, bool probabilities, uint32_t seen, bool biased, float bias) const {
        if (!probabilities) return steps(x, seen, biased, bias);
        if (!(x > 0.0f)) return x;
        return static_cast<float>(exp(steps(log(static_cast<double>(x)), seen, biased, bias)));
    }
};

__device__ __forceinline__ float parameter(const float *p, int64_t t, float off) {
    const float x = p != nullptr ? p[t] : off;
    return isfinite(x) ? x : off;
}

template <knn_dtype DT>
__global__ __launch_bounds__(kThreads) void k_adjust(AdjustArgs a) {
    extern __shared__ uint32_t lds[];  // counts [slice], then the last bias of each [slice]
    uint32_t *seen = lds;
    int32_t *last = reinterpret_cast<int32_t *>(lds + kSlice);
    const int64_t t = blockIdx.x;
    const int v0 = static_cast<int>(blockIdx.y) * kSlice;
    const int n = a.V - v0 < kSlice ? a.V - v0 : kSlice;
    int64_t s = t, first = t;
    if (a.row_offsets != nullptr) {
        if (t >= a.row_offsets[a.S]) return;
        s = set_of_query(a.row_offsets, a.S, t);
        first = a.row_offsets[s];
    }
    const bool counts = a.history != nullptr || a.row_tokens != nullptr;
    for (int i = threadIdx.x; i < n; i += kThreads) {
        seen[i] = 0u;
        if (a.bias_tokens != nullptr) last[i] = -1;
    }
    __syncthreads();
    if (a.history != nullptr) {
        const int64_t len = a.history_lens[s] < a.history_width ? a.history_lens[s] : a.history_width;
        const int64_t prompt = a.prompt_lens != nullptr ? a.prompt_lens[s] : 0;
        for (int64_t i = threadIdx.x; i < len; i += kThreads) {
            const int64_t v = static_cast<int64_t>(a.history[s * a.history_width + i]) - v0;
            if (v < 0 || v >= n) continue;
            if (i < prompt) atomicOr(&seen[v], kPrompt);
            else atomicAdd(&seen[v], 1u);
        }
    }
    if (a.row_tokens != nullptr) {
        int64_t rows = a.row_offsets != nullptr ? a.row_offsets[s + 1] : t + 1;
        rows = (rows < a.rows ? rows : a.rows) - first;
        if (a.tree_mask == nullptr) rows = t - first + 1;
        else if (rows > 32 * a.mask_words) rows = 32 * a.mask_words;
        for (int64_t i = threadIdx.x; i < rows; i += kThreads) {
            if (a.tree_mask != nullptr && (a.tree_mask[t * a.mask_words + (i >> 5)] >> (i & 31) & 1u) == 0u) continue;
            const int64_t v = static_cast<int64_t>(a.row_tokens[first + i]) - v0;
            if (v >= 0 && v < n) atomicAdd(&seen[v], 1u);
        }
    }
    if (a.bias_tokens != nullptr)
        for (int64_t i = threadIdx.x; i < a.bias_width; i += kThreads) {
            const int64_t v = static_cast<int64_t>(a.bias_tokens[s * a.bias_width + i]) - v0;
            if (v >= 0 && v < n) atomicMax(&last[v], static_cast<int32_t>(i));
        }
    __syncthreads();
    Rule rule{parameter(a.repetition, t, 1.0f), parameter(a.presence, t, 0.0f), parameter(a.frequency, t, 0.0f)};
    if (!(rule.repetition > 0.0f)) rule.repetition = 1.0f;
    constexpr int SIZE = DT == KNN_F32 ? 4 : 2;
    const char *in = static_cast<const char *>(a.scores) + (t * a.stride + v0) * SIZE;
    char *out = static_cast<char *>(a.out) + (t * a.out_stride + v0) * SIZE;
    const uint32_t *allowed = a.allowed != nullptr ? a.allowed + t * ((a.V + 31) / 32) + v0 / 32 : nullptr;
    for (int i = threadIdx.x; i < n; i += kThreads) {
        const float x = element<DT>(in, i);
        const uint32_t c = counts ? seen[i] : 0u;
        const int32_t b = a.bias_tokens != nullptr ? last[i] : -1;
        float y = x;
        bool touched = c != 0u || b >= 0;
        if (touched) y = rule.of(x, a.probabilities, c, b >= 0, b >= 0 ? a.bias_values[s * a.bias_width + b] : 0.0f);
        if (allowed != nullptr && (allowed[i >> 5] >> (i & 31) & 1u) == 0u) {
            y = a.probabilities ? 0.0f : -INFINITY;
            touched = true;
        }
        if (touched) put<DT>(out, i, y);
        else if constexpr (SIZE == 4) reinterpret_cast<uint32_t *>(out)[i] = reinterpret_cast<const uint32_t *>(in)[i];
        else reinterpret_cast<uint16_t *>(out)[i] = reinterpret_cast<const uint16_t *>(in)[i];
    }
}

}  // namespace

hipError_t launch_adjust_scores(const AdjustArgs &a, knn_dtype dtype, hipStream_t stream) {
    const int64_t slices = (a.V + kSlice - 1) / kSlice;
    const dim3 grid(static_cast<unsigned>(a.rows), static_cast<unsigned>(slices));
    const size_t lds = sizeof(uint32_t) * kSlice * (a.bias_tokens != nullptr ? 2 : 1);
    if (dtype == KNN_F32) k_adjust<KNN_F32><<<grid, kThreads, lds, stream>>>(a);
    else if (dtype == KNN_BF16) k_adjust<KNN_BF16><<<grid, kThreads, lds, stream>>>(a);
    else k_adjust<KNN_F16><<<grid, kThreads, lds, stream>>>(a);
    return hipGetLastError();
}

}  // namespace knnlm
