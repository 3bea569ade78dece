// New rows of keys and values into a paged cache, with the rotation that
// carries a token's position, and the rows' queries rotated in the same pass.
//
// Row t of sequence s goes to cache index c = cache_lens[s] + t -
// row_offsets[s]: page pages[s, c / page_size], slot c % page_size.  With
// position p (c unless given) each pair (a, b) of rotated elements becomes
//   (a cos x - b sin x, b cos x + a sin x),   x = p inv_freq[i],
// in 32 bits, rounded once to the element type.  x is taken in turns,
// p inv_freq / 2 pi, whose whole part is dropped in 64 bits: at position 10^6
// a 32-bit product is off by up to 0.06 radians, this one by 2e-7.
//
// Bound by the bytes: every element is read and written once.  The sines and
// cosines are those of the token, so a workgroup takes whole tokens, works
// them out once into LDS (one pair a lane) and uses them for all of its heads.
// An item is two 16-byte chunks of one head, i and its partner half a rotation
// further (or two neighbouring chunks where pairs lie side by side or nothing
// is rotated), so that a lane holds both elements of each pair.  Measured: the
// rows of four prompts of 4,000 to 8,000 tokens, 32 heads of 128: 1.23 GB in
// 236 us, 5.2 TB/s (a copy of 2 GiB: 4.96); one row 3.2 us.
#include "knnlm_device.h"
#include "lm_internal.h"

namespace knnlm {

namespace {

constexpr int kThreads = 256;
constexpr int kMaxTokens = 8;  // tokens of a workgroup

template <knn_dtype DT>
__device__ __forceinline__ float widen(uint16_t h) {
    if constexpr (DT == KNN_BF16) return __uint_as_float(static_cast<uint32_t>(h) << 16);
    return static_cast<float>(__builtin_bit_cast(_Float16, h));
}

template <knn_dtype DT>
__device__ __forceinline__ uint16_t narrow(float x) {  // to nearest, ties to even
    if constexpr (DT == KNN_BF16) return __builtin_bit_cast(uint16_t, static_cast<__bf16>(x));
    return __builtin_bit_cast(uint16_t, static_cast<_Float16>(x));
}

template <knn_dtype DT>
__device__ __forceinline__ void rotate(uint16_t &a, uint16_t &b, float2 cs) {
    const float x = widen<DT>(a), y = widen<DT>(b);
    a = narrow<DT>(x * cs.x - y * cs.y);
    b = narrow<DT>(y * cs.x + x * cs.y);
}

// Where one head of one token is read and written; null dst: nowhere.
struct Head {
    const uint16_t *src;
    uint16_t *dst;
    bool turn;  // rotated (queries and keys)
};

struct Token {
    int64_t source;  // row of q, k and v, or -1: the token is left out
    int64_t slot;    // page * kv_heads * page_size + slot in the page, or -1: no page
    int64_t position;
};

__device__ __forceinline__ Head head_of(const AppendArgs &a, const Token &tok, int64_t t, int h) {
    Head r{nullptr, nullptr, true};
    if (tok.source < 0) return r;
    if (h < a.q_heads) {
        r.src = static_cast<const uint16_t *>(a.q) + tok.source * a.q_row + h * a.q_head;
        r.dst = static_cast<uint16_t *>(a.q_out) + (t * a.q_heads + h) * a.head_dim;
        return r;
    }
    h -= a.q_heads;
    const bool key = h < a.kv_heads;
    if (!key) h -= a.kv_heads;
    r.turn = key;
    r.src = key ? static_cast<const uint16_t *>(a.k) + tok.source * a.k_row + h * a.k_head
                : static_cast<const uint16_t *>(a.v) + tok.source * a.v_row + h * a.v_head;
    if (tok.slot >= 0)
        r.dst = static_cast<uint16_t *>(key ? a.k_cache : a.v_cache) +
                (tok.slot + (static_cast<int64_t>(h) << a.cache.page_log2)) * a.head_dim;
    return r;
}

// VEC: 16-byte chunks (aligned rows, head_dim a multiple of 16, each half of
// the rotated part a multiple of 8, or all of it of 16 where pairs lie side by
// side); else one pair of elements an item.  `tokens` per workgroup in x, the
// items of a workgroup's tokens cut into gridDim.y shares.
template <knn_dtype DT, bool VEC>
__global__ __launch_bounds__(kThreads) void k_kv_append(AppendArgs a, int tokens) {
    extern __shared__ float2 turns[];  // [tokens][rot_dim / 2]: cosine, sine
    __shared__ Token token_of[kMaxTokens];
    const int64_t t0 = static_cast<int64_t>(blockIdx.x) * tokens;
    const int half = a.rot_dim / 2;
    const int64_t last = a.row_offsets[a.S];
    if (threadIdx.x < static_cast<unsigned>(tokens)) {
        const int64_t t = t0 + threadIdx.x;
        Token tok{-1, -1, 0};
        if (t < a.rows && t < last) {
            const int64_t source = a.source_rows != nullptr ? a.source_rows[t] : t;
            if (source >= 0 && source < a.source_count) {
                tok.source = source;
                const int64_t s = set_of_query(a.row_offsets, a.S, t);
                const int64_t c = a.cache_lens[s] + (t - a.row_offsets[s]);
                const int64_t entry = c >> a.cache.page_log2;
                tok.position = a.positions != nullptr ? a.positions[t] : c;
                if (c >= 0 && entry < a.cache.table_width) {
                    const int64_t page = a.cache.pages[s * a.cache.table_width + entry];
                    if (page >= 0 && page < a.cache.n_pages)
                        tok.slot = ((page * a.kv_heads) << a.cache.page_log2) + (c & ((1 << a.cache.page_log2) - 1));
                }
            }
        }
        token_of[threadIdx.x] = tok;
    }
    __syncthreads();
    for (int i = threadIdx.x; i < tokens * half; i += kThreads) {
        const double p = static_cast<double>(token_of[i / half].position);
        const double x = p * static_cast<double>(a.inv_freq[i % half]) * 0.15915494309189533577;  // 1 / (2 pi)
        float sn, cs;
        sincospif(2.0f * static_cast<float>(x - rint(x)), &sn, &cs);
        turns[i] = make_float2(cs, sn);
    }
    __syncthreads();

    const int heads = a.q_heads + 2 * a.kv_heads;
    constexpr int PER = VEC ? 16 : 2;  // elements of an item
    const int head_items = (a.head_dim + PER - 1) / PER;
    const int items = tokens * heads * head_items;
    for (int i = blockIdx.y * kThreads + threadIdx.x; i < items; i += gridDim.y * kThreads) {
        const int e = i % head_items, th = i / head_items;
        const int tok = th / heads;
        const Head hd = head_of(a, token_of[tok], t0 + tok, th % heads);
        if (hd.dst == nullptr) continue;
        const float2 *cs = turns + tok * half;
        if constexpr (VEC) {
            const bool spread = !a.interleaved && hd.turn && e * 8 < half;  // chunk e and its partner, half further
            // past the rotated part (or without one): neighbours of 16 elements
            const int c0 = spread ? e * 8 : e * 16;
            const int c1 = spread ? c0 + half : c0 + 8;
            const bool turn = hd.turn && (spread || (a.interleaved && c0 < a.rot_dim));
            union Chunk {
                u32x4_t v;
                uint16_t h[8];
            } x, y;
            x.v = *reinterpret_cast<const u32x4_t *>(hd.src + c0);
            y.v = *reinterpret_cast<const u32x4_t *>(hd.src + c1);
            if (turn) {
                if (spread) {
#pragma unroll
                    for (int j = 0; j < 8; ++j) rotate<DT>(x.h[j], y.h[j], cs[c0 + j]);
                } else {
#pragma unroll
                    for (int j = 0; j < 8; j += 2) {
                        rotate<DT>(x.h[j], x.h[j + 1], cs[(c0 + j) / 2]);
                        rotate<DT>(y.h[j], y.h[j + 1], cs[(c1 + j) / 2]);
                    }
                }
            }
            *reinterpret_cast<u32x4_t *>(hd.dst + c0) = x.v;
            *reinterpret_cast<u32x4_t *>(hd.dst + c1) = y.v;
        } else {
            const bool spread = !a.interleaved && hd.turn && e < half;
            const int i0 = spread ? e : 2 * e;
            const int i1 = spread ? e + half : 2 * e + 1;
            uint16_t x = hd.src[i0], y = i1 < a.head_dim ? hd.src[i1] : uint16_t{0};
            if (spread || (a.interleaved && hd.turn && i0 < a.rot_dim)) rotate<DT>(x, y, cs[e]);
            hd.dst[i0] = x;
            if (i1 < a.head_dim) hd.dst[i1] = y;
        }
    }
}

bool aligned16(const void *p) { return reinterpret_cast<uintptr_t>(p) % 16 == 0; }

}  // namespace

hipError_t launch_kv_append(const AppendArgs &a, knn_dtype dtype, hipStream_t stream) {
    const int half = a.rot_dim / 2;
    const int64_t odd = (a.q != nullptr ? a.q_row | a.q_head : 0) | a.k_row | a.k_head | a.v_row | a.v_head;
    const bool vec = a.head_dim % 16 == 0 && (a.interleaved ? a.rot_dim % 16 == 0 : half % 8 == 0) && odd % 8 == 0 &&
                     aligned16(a.q) && aligned16(a.k) && aligned16(a.v) && aligned16(a.q_out) &&
                     aligned16(a.k_cache) && aligned16(a.v_cache);
    // Items of a token; several tokens a workgroup where one has too few to
    // fill it, or several workgroups a token where there are few tokens.
    const int per = vec ? 16 : 2;
    const int64_t items = static_cast<int64_t>(a.q_heads + 2 * a.kv_heads) * ((a.head_dim + per - 1) / per);
    int tokens = 1;
    while (tokens < kMaxTokens && tokens * 2 * items <= 2 * kThreads && a.rows >= 1024 * tokens) tokens *= 2;
    const int64_t blocks = (a.rows + tokens - 1) / tokens;
    int64_t shares = (items * tokens + kThreads - 1) / kThreads;
    if (shares * blocks > 1024) shares = blocks >= 1024 ? 1 : 1024 / blocks;
    if (blocks > 0x7fffffffLL || shares > 65535) return hipErrorInvalidConfiguration;
    const dim3 grid(static_cast<unsigned>(blocks), static_cast<unsigned>(shares));
    const size_t lds = sizeof(float2) * static_cast<size_t>(tokens) * static_cast<size_t>(half);
    if (dtype == KNN_BF16) {
        if (vec) k_kv_append<KNN_BF16, true><<<grid, kThreads, lds, stream>>>(a, tokens);
        else k_kv_append<KNN_BF16, false><<<grid, kThreads, lds, stream>>>(a, tokens);
    } else {
        if (vec) k_kv_append<KNN_F16, true><<<grid, kThreads, lds, stream>>>(a, tokens);
        else k_kv_append<KNN_F16, false><<<grid, kThreads, lds, stream>>>(a, tokens);
    }
    return hipGetLastError();
}

}  // namespace knnlm
