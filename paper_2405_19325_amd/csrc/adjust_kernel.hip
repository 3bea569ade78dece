// Penalties for repeated tokens, biases and the tokens that a grammar allows,
// on rows of logits or probabilities.
//
// A workgroup takes a slice of 8,192 of a row's tokens, 8 a thread, copies its
// scores but for those that are not allowed, and meanwhile counts in LDS how
// often each token is in the row's history and in the drafts that the row sees
// (integer atomics: the same counts in any order), and finds the last bias of
// each (the largest entry).  A history has far fewer tokens than the vocabulary:
// those that are touched are listed by the first thread that comes to each, and
// the list is worked off by all.  Of logits the outcome is put among the copied
// scores on their way (256 rows of 131,072: 3 us less than where it is written
// over them); of probabilities it is written over them, since the scores would be
// held beside the 64-bit functions' registers (4 to 15 us more for 128 rows of
// 50,257).
//
// What bounds it.  256 rows of 131,072 fp32 logits with all steps take 81 us:
// the copy and its mask 55 (4.9 TB/s), the histories 17, biases and the touched
// tokens the rest, waits during which little is on its way; of 128 rows of
// 50,257 probabilities, 18 us, the 64-bit functions take 3 and the histories 5.
//
// Logits are worked out in 32 bits; probabilities as logarithms in 64, since the
// logarithm of a small one times a penalty, in 32 bits, would be off by 2^-18 of
// the outcome.
#include "knnlm_device.h"
#include "lm_internal.h"

namespace knnlm {

namespace {

constexpr int64_t kGrid = 1 << 15;      // groups of rows of a row of the grid
constexpr int kThreads = 1024;
constexpr int kPer = 8;                 // tokens of a thread
constexpr int kSlice = kPer * kThreads;
// Beside a token's count: it is in the prompt; it has a bias.
constexpr uint32_t kPrompt = 1u << 31, kBiased = 1u << 30;

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
    __device__ static __forceinline__ uint32_t raw(const void *p, int64_t i) {
        if constexpr (DT == KNN_F32) return static_cast<const uint32_t *>(p)[i];
        return static_cast<const uint16_t *>(p)[i];
    }
    __device__ static __forceinline__ void set(void *p, int64_t i, uint32_t x) {
        if constexpr (DT == KNN_F32) static_cast<uint32_t *>(p)[i] = x;
        else static_cast<uint16_t *>(p)[i] = static_cast<uint16_t>(x);
    }
};

typedef uint32_t u32x4_at4_t __attribute__((ext_vector_type(4), aligned(4)));

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

// A slice of a row's scores; the grid's x goes through 2^log2 rows and their
// slices.  LDS: words [slice], where there are biases the last of each [slice], and the list.
template <knn_dtype DT, bool PROBS>
__global__ __launch_bounds__(kThreads, 8) void k_adjust(AdjustArgs a, int log2) {
    using Ty = Type<DT>;
    constexpr int VEC = Ty::VEC, GROUPS = Ty::GROUPS;
    extern __shared__ __align__(16) uint32_t lds[];
    const bool biased = a.bias_tokens != nullptr;
    uint32_t *seen = lds;  // a touched token's count, later its score
    int32_t *last = reinterpret_cast<int32_t *>(lds + kSlice);
    // A bit a token: it is touched.  Then those that are, by first come.  Two workgroups just fit a CU, so
    // the list is that much shorter than a slice, and a slice that is touched nearly whole is gone through without it.
    uint32_t *bits = lds + (biased ? 2 : 1) * kSlice, *listed = bits + kSlice / 32;
    uint16_t *list = reinterpret_cast<uint16_t *>(listed + 1);
    constexpr uint32_t LIST = kSlice - kSlice / 16 - 2;
    const int tid = static_cast<int>(threadIdx.x);
    const uint32_t off = PROBS ? 0u : Ty::narrow(-INFINITY);
    const int64_t t = ((static_cast<int64_t>(blockIdx.z) * kGrid + blockIdx.y) << log2) + (blockIdx.x & ((1u << log2) - 1u));
    if (t >= a.rows) return;
    int64_t s = t, first = t;
    if (a.row_offsets != nullptr) {
        if (t >= a.row_offsets[a.S]) return;
        s = set_of_query_wave(a.row_offsets, a.S, t);
        first = a.row_offsets[s];
    }
    const char *in = static_cast<const char *>(a.scores) + t * a.stride * Ty::SIZE;
    char *out = static_cast<char *>(a.out) + t * a.out_stride * Ty::SIZE;
    // Places are counted from the 16 bytes that hold the first score; place p is token p - lead.
    const int lead = static_cast<int>(reinterpret_cast<uintptr_t>(in) % 16) / Ty::SIZE;
    const int v0 = static_cast<int>(blockIdx.x >> log2) * kSlice - lead;
    if (v0 >= a.V) return;
    const bool even = (reinterpret_cast<uintptr_t>(out) - reinterpret_cast<uintptr_t>(in)) % 16 == 0;
    const bool in_place = a.out == a.scores, copies = !in_place || a.allowed != nullptr;
    const int words = (a.V + 31) / 32;
    const uint32_t *allowed = a.allowed != nullptr ? a.allowed + t * words : nullptr;

    // The slice's scores, and a bit a token: it is allowed.
    u32x4_t x[GROUPS];
    uint32_t may[GROUPS];
    auto group = [&](int g) { return (g * kThreads + tid) * VEC; };  // place in the slice
    if (copies) {
#pragma unroll
        for (int g = 0; g < GROUPS; ++g) {
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
            may[g] = ~0u;
            if (allowed != nullptr) {
                const int w = v < 0 ? 0 : v >> 5, lo = w < words ? w : words - 1, hi = w + 1 < words ? w + 1 : words - 1;
                const uint64_t both = static_cast<uint64_t>(allowed[lo]) | static_cast<uint64_t>(allowed[hi]) << 32;
                may[g] = static_cast<uint32_t>(v < 0 ? both << -v : both >> (v & 31));
            }
        }
    }

    uint4 *words4 = reinterpret_cast<uint4 *>(lds);
#pragma unroll
    for (int i = 0; i < kPer / 4; ++i) {
        words4[i * kThreads + tid] = make_uint4(0, 0, 0, 0);
        if (biased) words4[(kPer / 4 + i) * kThreads + tid] = make_uint4(~0u, ~0u, ~0u, ~0u);
    }
    if (tid <= kSlice / 32) bits[tid] = 0;  // and the count of the list
    __syncthreads();

    // Tokens are counted from the slice's first one; q is none of its where it is not under `count`.
    const int vmin = v0 < 0 ? 0 : v0;
    const uint32_t count = static_cast<uint32_t>((v0 + kSlice < a.V ? v0 + kSlice : a.V) - vmin);
    auto place = [&](int32_t v) { return static_cast<uint32_t>(v) - static_cast<uint32_t>(vmin); };
    const int shift = vmin - v0;  // from there to the place in the slice
    auto touch = [&](uint32_t p, uint32_t old) {
        if (old != 0u) return;  // another thread was the first
        if (!PROBS && copies) atomicOr(&bits[p >> 5], 1u << (p & 31));
        const uint32_t i = atomicAdd(listed, 1u);
        if (i < LIST) list[i] = static_cast<uint16_t>(p);
    };
    if (a.history != nullptr) {
        const int64_t all = a.history_lens[s];
        const int len = static_cast<int>(all < a.history_width ? all : a.history_width);
        const int64_t all_prompt = a.prompt_lens != nullptr ? a.prompt_lens[s] : 0;
        const int prompt = static_cast<int>(all_prompt < len ? all_prompt : len);
        const int32_t *history = a.history + s * a.history_width;
        auto note = [&](uint32_t q, bool before) {
            if (q >= count) return;
            const uint32_t p = q + shift;
            touch(p, before ? atomicOr(&seen[p], kPrompt) : atomicAdd(&seen[p], 1u));
        };
        // Four tokens a load, two loads a thread; what is left at the end one by one.
        constexpr int STEP = kPer * kThreads;
        int i0 = 0;
        for (; i0 + STEP <= len; i0 += STEP) {
            u32x4_at4_t v[kPer / 4];
#pragma unroll
            for (int u = 0; u < kPer / 4; ++u)
                v[u] = *reinterpret_cast<const u32x4_at4_t *>(history + i0 + (u * kThreads + tid) * 4);
#pragma unroll
            for (int u = 0; u < kPer / 4; ++u)
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    note(place(static_cast<int32_t>(v[u][e])), i0 + (u * kThreads + tid) * 4 + e < prompt);
        }
        if (i0 < len) {
            int32_t v[kPer];
#pragma unroll
            for (int u = 0; u < kPer; ++u) v[u] = history[i0 + u * kThreads + tid < len ? i0 + u * kThreads + tid : i0];
#pragma unroll
            for (int u = 0; u < kPer; ++u) {
                if (i0 + u * kThreads >= len) break;
                if (i0 + u * kThreads + tid < len) note(place(v[u]), i0 + u * kThreads + tid < prompt);
            }
        }
    }
    if (a.row_tokens != nullptr) {
        int64_t rows = a.row_offsets != nullptr ? a.row_offsets[s + 1] : t + 1;
        rows = (rows < a.rows ? rows : a.rows) - first;
        const int64_t drafts = a.tree_mask == nullptr ? t - first + 1 : rows < 32 * a.mask_words ? rows : 32 * a.mask_words;
        for (int64_t i = tid; i < drafts; i += kThreads) {
            const bool sees = a.tree_mask == nullptr || (a.tree_mask[t * a.mask_words + (i >> 5)] >> (i & 31) & 1u) != 0u;
            const uint32_t q = place(a.row_tokens[first + i]);
            if (sees && q < count) touch(q + shift, atomicAdd(&seen[q + shift], 1u));
        }
    }
    if (biased) {
        for (int64_t i = tid; i < a.bias_width; i += kThreads) {
            const uint32_t q = place(a.bias_tokens[s * a.bias_width + i]);
            if (q >= count) continue;
            atomicMax(&last[q + shift], static_cast<int32_t>(i));
            touch(q + shift, atomicOr(&seen[q + shift], kBiased));
        }
    }
    // The scores as they are, but for those that are not allowed and (of logits) those that are touched.
    auto copy = [&]() {
#pragma unroll
        for (int g = 0; g < GROUPS; ++g) {
            const int v = v0 + group(g);
            constexpr uint32_t ALL = (1u << VEC) - 1u;
            const uint32_t never = ~may[g] & ALL, other = PROBS ? 0u : bits[group(g) >> 5] >> (group(g) & 31) & ALL;
            if (in_place && (never | other) == 0u) continue;
            if ((never | other) != 0u) {
#pragma unroll
                for (int e = 0; e < VEC; ++e) {
                    if (((never | other) >> e & 1u) == 0u) continue;
                    const uint32_t to = (never >> e & 1u) != 0u ? off : seen[group(g) + e];
                    if constexpr (DT == KNN_F32) x[g][e] = to;
                    else x[g][e / 2] = e % 2 != 0 ? (x[g][e / 2] & 0xffffu) | to << 16 : (x[g][e / 2] & 0xffff0000u) | to;
                }
            }
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
    };
    if (PROBS && copies) copy();
    __syncthreads();

    Rule rule{parameter(a.repetition, t, 1.0f), parameter(a.presence, t, 0.0f), parameter(a.frequency, t, 0.0f)};
    if (!(rule.repetition > 0.0f)) rule.repetition = 1.0f;
    auto adjust = [&](uint32_t p) {
        const int v = v0 + static_cast<int>(p);
        const uint32_t raw = Ty::raw(in, v);
        const float from = Ty::widen(u32x4_t{raw, 0, 0, 0}, 0);
        const uint32_t c = seen[p] & ~kBiased;
        const int32_t b = biased ? last[p] : -1;
        const float bias = b >= 0 ? a.bias_values[s * a.bias_width + b] : 0.0f;
        uint32_t to = raw;
        if constexpr (PROBS) {
            if (from > 0.0f)
                to = Ty::narrow(static_cast<float>(exp(rule.of(log(static_cast<double>(from)), c, b >= 0, bias))));
        } else {
            to = Ty::narrow(rule.of(from, c, b >= 0, bias));
        }
        if (!PROBS && copies) seen[p] = to;
        else if (allowed == nullptr || (allowed[v >> 5] >> (v & 31) & 1u) != 0u) Ty::set(out, v, to);
    };
    const uint32_t n = *listed;
    if (n <= LIST) {
        for (uint32_t i = tid; i < n; i += kThreads) adjust(list[i]);
    } else {
        for (uint32_t p = shift + tid; p < shift + count; p += kThreads)
            if (seen[p] != 0u) adjust(p);
    }
    if (PROBS || !copies) return;
    __syncthreads();
    copy();
}

template <knn_dtype DT, bool PROBS>
hipError_t launch(const AdjustArgs &a, hipStream_t stream) {
    const int64_t slices = (a.V + Type<DT>::VEC - 1 + kSlice - 1) / kSlice;
    // Workgroups go to the eight dies in turn: with rows by eights the slices of one lie behind each other on one die, whose
    // cache has the row's history after the first (256 rows of 131,072 logits: 158 MB read and 81 us, 253 and 84 with all
    // rows' first slices before their second ones).  Probabilities, whose slices differ more in what they take: by 32 (128
    // rows of 50,257 17.9 us, 18.6 that way, 19.7 by eights).
    const int log2 = a.rows < 8 ? 0 : PROBS ? 5 : 3;
    const int64_t groups = (a.rows + (1 << log2) - 1) >> log2;
    const dim3 grid(static_cast<unsigned>(slices << log2), static_cast<unsigned>(groups < kGrid ? groups : kGrid),
                    static_cast<unsigned>((groups + kGrid - 1) / kGrid));
    const size_t words = kSlice * (a.bias_tokens != nullptr ? 2 : 1) + kSlice / 2;
    k_adjust<DT, PROBS><<<grid, kThreads, sizeof(uint32_t) * words, stream>>>(a, log2);
    return hipGetLastError();
}

template <knn_dtype DT>
hipError_t launch(const AdjustArgs &a, hipStream_t stream) {
    return a.probabilities ? launch<DT, true>(a, stream) : launch<DT, false>(a, stream);
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
