// The weight that a sequence's rows put on each of its cached keys.
//
// With the logarithms of the rows' sums in hand (attention's lse), a key's
// weight of row i and query head a is exp(scale q_ia.k_j - lse_ia); a key's
// mass is what all rows that see it and all heads of its key head put on it,
// and a share of what it was before.
//
// A thread takes a key: its elements in registers, the rows' queries one after
// the other.
#include "lm_device.h"

namespace knnlm {

namespace {

constexpr int kThreads = 256;
constexpr float kLog2e = 1.4426950408889634f;

template <knn_dtype DT, int D>
__global__ __launch_bounds__(kThreads) void k_key_weights(WeighArgs a) {
    const int h = static_cast<int>(blockIdx.y), g = a.q_heads / a.kv_heads;
    for (int64_t s = blockIdx.z; s < a.S; s += gridDim.z) {
        const Tile t = tile_of(a, s);
        const int64_t j = static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x;
        if (t.n == 0 || j >= t.total) continue;
        const int64_t at = place_of(a.cache, a.kv_heads, s, h, j);
        if (at < 0) continue;
        uint4 k[D / 8];
        const uint4 *key = reinterpret_cast<const uint4 *>(static_cast<const uint16_t *>(a.k_cache) + at * D);
#pragma unroll
        for (int c = 0; c < D / 8; ++c) k[c] = key[c];
        const int64_t draft = j - t.length;
        float w = 0.0f;
        for (int i = 0; i < t.n; ++i) {
            const int64_t row = t.r0 + i;
            const int64_t source = a.source_rows != nullptr ? a.source_rows[row] : row;
            if (source < 0 || source >= a.source_count) continue;
            bool sees = draft <= i;
            if (a.tree_mask != nullptr && draft >= 0)
                sees = draft < 32 * a.mask_words && (a.tree_mask[row * a.mask_words + (draft >> 5)] >> (draft & 31) & 1u) != 0u;
            for (int e = 0; e < g; ++e) {
                const float lse = a.lse[source * a.q_heads + h * g + e];
                const uint4 *q = reinterpret_cast<const uint4 *>(static_cast<const uint16_t *>(a.q) + source * a.q_row +
                                                                 (h * g + e) * a.q_head);
                float x = 0.0f;
#pragma unroll
                for (int c = 0; c < D / 8; ++c) x = dot_chunk<DT>(q[c], k[c], x);
                if (sees && isfinite(lse)) w += exp2f(fmaf(x, a.scale, -lse) * kLog2e);
            }
        }
        const bool own = draft >= 0;
        if (!own && a.decay != 0.0f) w += a.decay * a.mass[at];
        a.mass[at] = w;
        if (own && a.key_positions != nullptr)
            a.key_positions[at] = a.positions != nullptr ? a.positions[t.r0 + draft] : static_cast<int32_t>(j);
    }
}

template <knn_dtype DT>
hipError_t launch(const WeighArgs &a, hipStream_t stream) {
    const int64_t tiles = (a.max_keys + kThreads - 1) / kThreads;
    const dim3 grid(static_cast<unsigned>(tiles), static_cast<unsigned>(a.kv_heads),
                    static_cast<unsigned>(a.S < 65535 ? a.S : 65535));
    if (a.head_dim == 64) k_key_weights<DT, 64><<<grid, kThreads, 0, stream>>>(a);
    else if (a.head_dim == 128) k_key_weights<DT, 128><<<grid, kThreads, 0, stream>>>(a);
    else k_key_weights<DT, 256><<<grid, kThreads, 0, stream>>>(a);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_key_weights(const WeighArgs &a, knn_dtype dtype, hipStream_t stream) {
    return dtype == KNN_BF16 ? launch<KNN_BF16>(a, stream) : launch<KNN_F16>(a, stream);
}

}  // namespace knnlm
