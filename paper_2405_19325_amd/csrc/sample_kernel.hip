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
// index first among equals.  A cut in it is its last element.  To find one,
// the elements go into 2048 bins that follow the order, of about a 64th of a
// factor e (of an octave, for probabilities) each: counts for top-k, weights
// for top-p.  A scan finds the bin of the cut; its elements, a few dozen as a
// rule, are listed, and each one's place and what lies before it come from
// comparing it with all others.  Where they are more than the list holds (a
// value that hundreds of tokens share, a row far from any logarithmic
// spread), the cut is found on the keys that order like the values, eleven
// bits a pass.
//
// One workgroup takes a row.  A row of up to 128 KiB stays in LDS from the first
// pass on; a longer one is read three times, from the caches after the first.
#include "knnlm_device.h"
#include "lm_internal.h"

namespace knnlm {

namespace {

constexpr int kThreads = 1024;
constexpr int kWaves = kThreads / kWave;
constexpr int kBins = 2048;

constexpr size_t kHeldBytes = 128 * 1024;
constexpr int kList = 512;  // elements of a cut's bin that are compared with each other

template <knn_dtype DT>
__device__ __forceinline__ float element(const void *row, int i) {
    if constexpr (DT == KNN_F32) return static_cast<const float *>(row)[i];
    if constexpr (DT == KNN_BF16)
        return __uint_as_float(static_cast<uint32_t>(static_cast<const uint16_t *>(row)[i]) << 16);
    return static_cast<float>(static_cast<const _Float16 *>(row)[i]);
}

// -inf for what is absent (NaN; of probabilities also what is not above 0); one zero.
__device__ __forceinline__ float present(float x, bool probabilities) {
    return x > (probabilities ? 0.0f : -INFINITY) ? x + 0.0f : -INFINITY;
}

// A key that orders like a present x; 0 for an absent one.
__device__ __forceinline__ uint32_t key_of(float x) {
    if (!(x > -INFINITY)) return 0;
    const uint32_t b = __float_as_uint(x);
    return b ^ ((b >> 31) != 0 ? 0xffffffffu : 0x80000000u);
}

__device__ __forceinline__ float value_of(uint32_t key) {
    return __uint_as_float(key ^ ((key >> 31) != 0 ? 0x80000000u : 0xffffffffu));
}

// 2^(y / 64) 2^e for y <= 0, to 2^-51 relative: a table of the 64th roots of
// two, and the power series of exp(f ln(2) / 64), |f| <= 1/2, whose 6th term is
// 4e-17.  What is under 2^-200 counts as that.
__device__ __forceinline__ double power2(double y, int e, const double *roots) {
    y = fmax(y, -12800.0);
    const double moved = y + 6755399441055744.0;  // 1.5 2^52: the nearest whole number in the low bits
    const double f = y - (moved - 6755399441055744.0);
    const int n = static_cast<int>(__double_as_longlong(moved));
    const double root = roots[n & 63];
    double r = 1.2417843701716923e-12;           // c^5 / 5!, c = ln(2) / 64
    r = fma(r, f, 5.732851688640402e-10);       // c^4 / 4!
    r = fma(r, f, 2.1173137155464774e-07);       // c^3 / 3!
    r = fma(r, f, 5.864904955056169e-05);       // c^2 / 2
    r = fma(r, f, 0.010830424696249145);       // c
    return ldexp(fma(root, r * f, root), (n >> 6) + e);
}

// log2 of a positive finite x, to 2^-50: x = 2^e m, and with c one of 64 values
// near 1 / m, log2 m = -log2 c + log2(1 + r), r = m c - 1, |r| < 2^-6.9, by
// the series of the logarithm, whose 8th term is 2^-58.
__device__ __forceinline__ double log2_of(float x, const double2 *logs) {
    const uint64_t bits = static_cast<uint64_t>(__double_as_longlong(static_cast<double>(x)));
    const double m = __longlong_as_double(static_cast<long long>((bits & 0x000fffffffffffffull) | 0x3ff0000000000000ull));
    const double2 at = logs[(bits >> 46) & 63];
    const double r = fma(m, at.x, -1.0);
    double q = 1.0 / 7.0;
    q = fma(q, r, -1.0 / 6.0);
    q = fma(q, r, 1.0 / 5.0);
    q = fma(q, r, -1.0 / 4.0);
    q = fma(q, r, 1.0 / 3.0);
    q = fma(q, r, -1.0 / 2.0);
    q = fma(q, r, 1.0);
    return fma(r * q, 1.4426950408889634074, at.y) + static_cast<double>(static_cast<int>(bits >> 52) - 1023);
}

// The weights of a row, as a function of the value; the largest one's is 2^s.
// Probabilities at T = 1 are their own weights (`plain`), brought under 2^s by
// a power of two.
template <bool PROBS>
struct Weights {
    double top;    // the largest value, or its log2 where the values are probabilities
    double rate;   // 64 log2(e) / T, or 64 / T of probabilities
    double unit;   // 2^s
    double least;  // min-p, as a weight
    int log2_unit;
    bool plain;
    const double *roots;
    const double2 *logs;

    // An infinite value is as far from the largest as that from itself.
    __device__ __forceinline__ static float finite(float x) { return fminf(x, 3.402823466e38f); }
    template <int N>
    __device__ __forceinline__ void of(const float (&x)[N], double (&v)[N]) const {
        if (PROBS && plain) {
#pragma unroll
            for (int c = 0; c < N; ++c) v[c] = static_cast<double>(x[c]) * unit;
        } else {
#pragma unroll
            for (int c = 0; c < N; ++c) {
                const double far = (PROBS ? log2_of(finite(x[c]), logs) : static_cast<double>(finite(x[c]))) - top;
                v[c] = power2(far * rate, log2_unit, roots);
            }
        }
    }
    __device__ __forceinline__ double of(float x) const {
        const float y[1] = {x};
        double v[1];
        of(y, v);
        return v[0];
    }
    // To the nearest whole number: w < 2^52, so the sum's low bits are it.
    __device__ __forceinline__ static uint64_t whole(double w) {
        return static_cast<uint64_t>(__double_as_longlong(w + 4503599627370496.0) - 0x4330000000000000ll);
    }
};

struct Shared {
    double roots[64];  // 2^(i / 64)
    double2 logs[64];  // of the 64ths of [1, 2): c = 1 / its middle, -log2(c)
    uint64_t mass[kBins];  // bins, then the weights of the row's pieces
    uint64_t list[kList];  // key << 32 | ~index: larger is earlier in the order
    uint64_t weight[kList];
    uint64_t part[kWaves];
    uint32_t part32[kWaves];
    uint64_t before, cut;
    uint32_t bin, listed, kept;
    int index;
};

template <int CTRL>
__device__ __forceinline__ uint64_t dpp_u64(uint64_t v) {
    return static_cast<uint64_t>(dpp_u32<CTRL>(0u, static_cast<uint32_t>(v >> 32))) << 32 |
           dpp_u32<CTRL>(0u, static_cast<uint32_t>(v));
}
__device__ __forceinline__ uint64_t readlane_u64(uint64_t v, int lane) {
    return static_cast<uint64_t>(readlane_u32(static_cast<uint32_t>(v >> 32), lane)) << 32 |
           readlane_u32(static_cast<uint32_t>(v), lane);
}
// Sum over the wave, in scalar registers: exchanges within the 16 lanes of a row, then the four rows.
__device__ __forceinline__ uint64_t wave_sum64(uint64_t v) {
    v += dpp_u64<0xB1>(v);   // quad_perm [1,0,3,2]
    v += dpp_u64<0x4E>(v);   // quad_perm [2,3,0,1]
    v += dpp_u64<0x141>(v);  // row_half_mirror
    v += dpp_u64<0x140>(v);  // row_mirror
    return (readlane_u64(v, 0) + readlane_u64(v, 16)) + (readlane_u64(v, 32) + readlane_u64(v, 48));
}
__device__ __forceinline__ uint32_t wave_sum32(uint32_t v) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o);
    return v;
}
// What the lanes up to this one hold: shifts within the 16 lanes of a row, then the rows before.
__device__ __forceinline__ uint64_t wave_scan64(uint64_t v, int lane) {
    v += dpp_u64<0x111>(v);  // row_shr:1
    v += dpp_u64<0x112>(v);  // row_shr:2
    v += dpp_u64<0x114>(v);  // row_shr:4
    v += dpp_u64<0x118>(v);  // row_shr:8
    const uint64_t r0 = readlane_u64(v, 15), r1 = r0 + readlane_u64(v, 31), r2 = r1 + readlane_u64(v, 47);
    const int row = lane >> 4;
    return v + (row == 0 ? 0 : row == 1 ? r0 : row == 2 ? r1 : r2);
}

// The sum of sh.mass; with hit(before, own) true for one entry, its number and
// what lies before it in sh.bin and sh.before.
template <typename Goal, typename Hit>
__device__ __forceinline__ uint64_t scan_bins(Shared &sh, Goal goal_of, Hit hit) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const uint64_t a = sh.mass[2 * threadIdx.x], b = sh.mass[2 * threadIdx.x + 1];
    const uint64_t incl = wave_scan64(a + b, lane);
    if (lane == 63) sh.part[wave] = incl;
    __syncthreads();
    uint64_t before = 0, total = 0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
        const uint64_t v = sh.part[w];
        before += w < wave ? v : 0;
        total += v;
    }
    before += incl - a - b;
    const auto goal = goal_of(total);
    if (hit(before, a, goal)) sh.bin = 2 * threadIdx.x, sh.before = before;
    if (hit(before + a, b, goal)) sh.bin = 2 * threadIdx.x + 1, sh.before = before + a;
    __syncthreads();
    return total;
}

constexpr int kPieceLog2 = 9;  // elements of a row's pieces (more where a row would have over kBins of them)

// A row of scores: in LDS from the first reading on (HELD), or in memory.  Its
// places start at the 4-element boundary in memory at or before the first
// element: element i is at place i + lead, places outside the row are absent.
template <knn_dtype DT, bool HELD, bool PROBS>
struct Row {
    static constexpr int SIZE = DT == KNN_F32 ? 4 : 2;
    const char *row;  // place 0
    char *held;
    int lead, end;  // the elements' places
    int pieces, piece_log2;

    __device__ __forceinline__ static void widen4(const void *p, float (&x)[4]) {
        if constexpr (DT == KNN_F32) {
            const float4 v = *static_cast<const float4 *>(p);
            x[0] = v.x, x[1] = v.y, x[2] = v.z, x[3] = v.w;
        } else {
            const uint2 v = *static_cast<const uint2 *>(p);
            const uint16_t h[4] = {static_cast<uint16_t>(v.x), static_cast<uint16_t>(v.x >> 16),
                                   static_cast<uint16_t>(v.y), static_cast<uint16_t>(v.y >> 16)};
#pragma unroll
            for (int c = 0; c < 4; ++c) x[c] = element<DT>(h, c);
        }
    }
    __device__ __forceinline__ float at(int i) const {
        return i >= lead && i < end ? present(element<DT>(row, i), PROBS) : -INFINITY;
    }
    // Places i .. i + 3 (i a multiple of four).
    __device__ __forceinline__ void read4(int i, float (&x)[4]) const {
        if (i >= lead && i + 3 < end) {
            widen4(row + static_cast<int64_t>(i) * SIZE, x);
#pragma unroll
            for (int c = 0; c < 4; ++c) x[c] = present(x[c], PROBS);
        } else {
#pragma unroll
            for (int c = 0; c < 4; ++c) x[c] = at(i + c);
        }
    }
    __device__ __forceinline__ void load4(int i, float (&x)[4]) const {
        if constexpr (HELD) widen4(held + i * SIZE, x); else read4(i, x);
    }
    __device__ __forceinline__ void load8(int i, float (&x)[8]) const {
        float u[4], v[4];
        load4(i, u);
        load4(i + 256, v);
#pragma unroll
        for (int c = 0; c < 4; ++c) x[c] = u[c], x[c + 4] = v[c];
    }
    // f(place, value) over this wave's pieces, one place a lane: where there is little code to spare.
    template <typename F, typename Done>
    __device__ __forceinline__ void slow_pass(int wave, int lane, F f, Done done) const {
        const int each = (pieces + kWaves - 1) / kWaves;
        const int last = min(pieces, (wave + 1) * each);
        for (int piece = wave * each; piece < last; ++piece) {
#pragma unroll 1
            for (int i = piece << piece_log2; i < (piece + 1) << piece_log2; i += kWave) f(i + lane, at(i + lane));
            done(piece);
        }
    }
    __device__ __forceinline__ void keep4(int i, const float (&x)[4]) const {
        if constexpr (DT == KNN_F32) {
            *reinterpret_cast<float4 *>(held + i * 4) = make_float4(x[0], x[1], x[2], x[3]);
        } else {  // the values came from the type, so they go back exactly
            uint32_t h[4];
#pragma unroll
            for (int c = 0; c < 4; ++c)
                h[c] = DT == KNN_BF16 ? __float_as_uint(x[c]) >> 16
                                      : __builtin_bit_cast(uint16_t, static_cast<_Float16>(x[c]));
            *reinterpret_cast<uint2 *>(held + i * 2) = make_uint2(h[0] | h[1] << 16, h[2] | h[3] << 16);
        }
    }
    // f(place of x[0], x) for this wave's pieces, which are consecutive, four
    // places a lane; done(piece) after each piece.  FIRST: the first reading.
    template <bool FIRST = false, typename F, typename Done>
    __device__ __forceinline__ void pass(int wave, int lane, F f, Done done) const {
        const int each = (pieces + kWaves - 1) / kWaves;
        const int last = min(pieces, (wave + 1) * each);
        if constexpr (FIRST) {  // eight loads a lane in flight
            const int stop = last << piece_log2;
            for (int i = (wave * each) << piece_log2; i < stop; i += 2048) {
                float x[8][4];
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    if (i + 256 * j < stop) read4(i + 256 * j + 4 * lane, x[j]);
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    if (i + 256 * j < stop) {
                        if constexpr (HELD) keep4(i + 256 * j + 4 * lane, x[j]);
                        f(i + 256 * j + 4 * lane, x[j]);
                    }
                }
            }
        } else {
            // x[c] is at place i + 4 lane + c + (c < 4 ? 0 : 252); the next eight are on their way meanwhile
            const int stop = last << piece_log2, mask = (1 << piece_log2) - 1;
            int i = (wave * each) << piece_log2;
            if (i >= stop) return;
            float x[8], next[8];
            load8(i + 4 * lane, x);
            for (; i < stop; i += 512) {
                if (i + 512 < stop) load8(i + 512 + 4 * lane, next);
                f(i + 4 * lane, x);
                if (((i + 512) & mask) == 0) done(i >> piece_log2);
#pragma unroll
                for (int c = 0; c < 8; ++c) x[c] = next[c];
            }
        }
    }
};

__device__ __forceinline__ int place(int i, int c) { return i + c + (c < 4 ? 0 : 252); }

// The filters and the draw of a row whose largest present value is `top` and
// smallest `low`, at a temperature t > 0 and top-p p > 0.
template <bool PROBS, typename R>
__device__ __forceinline__ void draw(const SampleArgs &a, const R &rw, Shared &sh, int64_t r, float top, float low, float t,
                                     float p, int log2_unit) {
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int V = rw.end - rw.lead, pieces = rw.pieces, piece_log2 = rw.piece_log2;
    auto pass = [&](auto f, auto done) { rw.pass(wave, lane, f, done); };
    auto nothing = [](int) {};
    Weights<PROBS> w;
    w.plain = PROBS && t == 1.0f && top < INFINITY;
    w.roots = sh.roots;
    w.logs = sh.logs;
    w.top = PROBS ? log2_of(w.finite(top), sh.logs) : static_cast<double>(w.finite(top));
    w.rate = (PROBS ? 64.0 : 92.332482616893656874) / static_cast<double>(t);
    w.log2_unit = log2_unit - (w.plain ? ilogb(static_cast<double>(top)) + 1 : 0);
    w.unit = ldexp(1.0, w.log2_unit);
    const float min_p = a.min_p != nullptr ? a.min_p[r] : 0.0f;
    w.least = (min_p > 0.0f ? fmin(static_cast<double>(min_p), 1.0) : 0.0) *
              (w.plain ? static_cast<double>(top) * w.unit : w.unit);

    // Bins that follow the order; what is past the last one's start is in it.
    // Logits: steps of the distance from the largest, over 32 T or the row's
    // range.  Probabilities: steps of the bits, which grow like a logarithm.
    const float span = fminf(top - low, 32.0f * t);
    const float step = span > 0.0f ? kBins / span : 0.0f;
    const uint32_t top_bits = __float_as_uint(top);
    int shift = 0;
    if (PROBS) {
        const float octaves = fminf(46.0f * t, 255.0f);  // 2^-46 = e^-32
        uint32_t bits = min(top_bits - __float_as_uint(fminf(low, top)), static_cast<uint32_t>(octaves * 8388608.0f));
        while (bits >> shift >= kBins) ++shift;
    }
    auto bin_of = [&](float x) -> uint32_t {
        if (PROBS) return min((top_bits - __float_as_uint(x)) >> shift, static_cast<uint32_t>(kBins - 1));
        return static_cast<uint32_t>(fminf((top - x) * step, static_cast<float>(kBins - 1)));
    };

    // What stays: x above `cut_x`, or equal to it with an index up to `cut_i`.
    float cut_x = top == INFINITY ? 3.402823466e38f : -INFINITY;
    int cut_i = -1;
    auto stays = [&](int i, float x) { return x > cut_x || (x == cut_x && i <= cut_i); };
    auto clear = [&]() {
        __syncthreads();
        sh.mass[2 * threadIdx.x] = 0;
        sh.mass[2 * threadIdx.x + 1] = 0;
        if (threadIdx.x == 0) sh.listed = 0, sh.cut = ~0ull;
        __syncthreads();
    };
    uint32_t kept = 0;
    bool summed = false;
    uint64_t run = 0;  // this wave's weights of the piece at hand
    auto end_piece = [&](int piece) {
        const uint64_t s = wave_sum64(run);
        if (lane == 0) sh.mass[piece] = s;
        run = 0;
    };
    // The weights of eight places at once, where any lane needs one.
    auto weigh = [&](const float (&x)[8], const bool (&in)[8], auto f) {
        bool any = false;
#pragma unroll
        for (int c = 0; c < 8; ++c) any |= in[c];
        if (!__any(any)) return;
        double v[8];
        w.of(x, v);
#pragma unroll
        for (int c = 0; c < 8; ++c) f(c, v[c]);
    };
    auto add = [&](const float (&x)[8], const bool (&in)[8]) {
        weigh(x, in, [&](int c, double v) {
            const bool keep = in[c] && v >= w.least;
            run += keep ? Weights<PROBS>::whole(v) : 0;
            kept += keep ? 1u : 0u;
        });
    };
    auto count = [&](uint64_t v, uint32_t bin) {
        atomicAdd(reinterpret_cast<unsigned long long *>(&sh.mass[bin]), static_cast<unsigned long long>(v));
    };
    // The cuts: by count (top-k), then by weight (top-p).
    const int k = a.top_k != nullptr ? a.top_k[r] : 0;
    const bool stages[2] = {k > 0 && k < V, p < 1.0f};
#pragma unroll 1
    for (int stage = 0; stage < 2; ++stage) {
        if (stage == 0 ? !stages[0] : !stages[1]) continue;
        const bool by_weight = stage == 1, last = by_weight || !stages[1];  // last: sums the row's pieces too
        clear();
        pass(
            [&](int i, const float (&x)[8]) {
                bool in[8];
#pragma unroll
                for (int c = 0; c < 8; ++c) in[c] = stays(place(i, c), x[c]);
                if (by_weight) {
                    weigh(x, in, [&](int c, double v) {
                        if (in[c]) count(Weights<PROBS>::whole(v), bin_of(x[c]));
                    });
                } else {
#pragma unroll
                    for (int c = 0; c < 8; ++c)
                        if (in[c]) count(1, bin_of(x[c]));
                }
            },
            nothing);
        __syncthreads();
        const double share = p;
        auto goal_of = [&](uint64_t all) { return by_weight ? share * static_cast<double>(all) : static_cast<double>(k); };
        auto crosses = [](uint64_t at, uint64_t v, double to) {
            return static_cast<double>(at) < to && static_cast<double>(at + v) >= to;
        };
        const uint64_t all = scan_bins(sh, goal_of, crosses);
        if (!by_weight && static_cast<uint64_t>(k) >= all) continue;  // all that is present stays
        const double goal = goal_of(all);
        const uint32_t bin = sh.bin;
        const uint64_t before = sh.before;
        pass(
            [&](int i, const float (&x)[8]) {
                bool under[8];
#pragma unroll
                for (int c = 0; c < 8; ++c) {
                    const bool in = stays(place(i, c), x[c]);
                    const uint32_t b = bin_of(x[c]);
                    if (in && b == bin) {
                        const uint32_t at = atomicAdd(&sh.listed, 1u);
                        if (at < kList)
                            sh.list[at] = static_cast<uint64_t>(key_of(x[c])) << 32 | ~static_cast<uint32_t>(place(i, c));
                    }
                    under[c] = in && b < bin;
                }
                if (last) add(x, under);
            },
            [&](int piece) {
                if (last) end_piece(piece);
            });
        __syncthreads();
        const int n = static_cast<int>(sh.listed);
        if (n <= kList) {
            if (static_cast<int>(threadIdx.x) < n) {
                const double v = w.of(value_of(static_cast<uint32_t>(sh.list[threadIdx.x] >> 32)));
                sh.weight[threadIdx.x] = Weights<PROBS>::whole(v);
            }
            __syncthreads();
            // What lies before each entry: eight lanes an entry, each over an eighth of the others.
            for (int first = 0; first < n; first += kThreads / 8) {
                const int me = first + static_cast<int>(threadIdx.x >> 3);
                const uint64_t mine = me < n ? sh.list[me] : ~0ull;
                uint64_t ahead = 0;
                for (int j = threadIdx.x & 7; j < n; j += 8)
                    ahead += sh.list[j] > mine ? (by_weight ? sh.weight[j] : 1) : 0;
                ahead += dpp_u64<0xB1>(ahead);
                ahead += dpp_u64<0x4E>(ahead);
                ahead += dpp_u64<0x141>(ahead);
                if (me < n && (threadIdx.x & 7) == 0 && static_cast<double>(before + ahead) < goal) {
                    atomicMin(reinterpret_cast<unsigned long long *>(&sh.cut), static_cast<unsigned long long>(mine));
                    const double v = w.of(value_of(static_cast<uint32_t>(mine >> 32)));
                    if (last && v >= w.least) {
                        count(sh.weight[me], ~static_cast<uint32_t>(mine) >> piece_log2);
                        ++kept;
                    }
                }
            }
            __syncthreads();
            cut_x = value_of(static_cast<uint32_t>(sh.cut >> 32));
            cut_i = static_cast<int>(~static_cast<uint32_t>(sh.cut));
            summed = last;
            continue;
        }
        kept = 0;
        run = 0;
        // By keys, eleven bits a pass: the key of the cut, and how much of the goal is left for the elements equal to it.
        uint32_t prefix = 0;
        uint64_t above = 0;
#pragma unroll 1
        for (int level = 0; level < 3; ++level) {
            const int low_bit = level == 0 ? 21 : level == 1 ? 10 : 0, bits = level == 2 ? 10 : 11;
            clear();
            rw.slow_pass(
                wave, lane,
                [&](int i, float x) {
                    const uint32_t key = key_of(x);
                    if (!stays(i, x) || (level > 0 && key >> (low_bit + bits) != prefix)) return;
                    count(by_weight ? Weights<PROBS>::whole(w.of(x)) : 1,
                          kBins - 1 - ((key >> low_bit) & ((1u << bits) - 1)));
                },
                nothing);
            __syncthreads();
            const uint64_t base = above;
            scan_bins(sh, [&](uint64_t) { return goal; },
                      [&](uint64_t at, uint64_t v, double to) { return crosses(base + at, v, to); });
            prefix = prefix << bits | ((kBins - 1 - sh.bin) & ((1u << bits) - 1));
            above = base + sh.before;
        }
        const float x_at = value_of(prefix);
        const uint64_t one = by_weight ? Weights<PROBS>::whole(w.of(x_at)) : 1;
        // The n-th element equal to it is the last before which less than the goal lies.
        uint64_t left = static_cast<uint64_t>((goal - static_cast<double>(above)) / static_cast<double>(one));
        while (static_cast<double>(above + left * one) < goal) ++left;
        while (left > 1 && static_cast<double>(above + (left - 1) * one) >= goal) --left;
        clear();
        uint32_t equal = 0;
        rw.slow_pass(
            wave, lane, [&](int i, float x) { equal += x == x_at && stays(i, x) ? 1u : 0u; },
            [&](int piece) {
                const uint32_t s = wave_sum32(equal);
                if (lane == 0) sh.mass[piece] = s;
                equal = 0;
            });
        __syncthreads();
        scan_bins(sh, [&](uint64_t) { return static_cast<double>(left); }, crosses);
        if (wave == 0) {
            uint64_t seen = sh.before;
            bool found = false;
            for (int i = static_cast<int>(sh.bin) << piece_log2; !found; i += kWave) {
                const int at = i + lane;
                const float x = rw.at(at);
                const uint64_t eq = __ballot(x == x_at && stays(at, x));
                const int here = __popcll(eq & ((2ull << lane) - 1));
                if (((eq >> lane) & 1) != 0 && seen + here == left) sh.index = at;
                seen += __popcll(eq);
                found = seen >= left || i + kWave >= rw.end;
            }
        }
        __syncthreads();
        cut_i = sh.index;
        cut_x = x_at;
    }
    if (!summed) {
        clear();
        pass(
            [&](int i, const float (&x)[8]) {
                bool in[8];
#pragma unroll
                for (int c = 0; c < 8; ++c) in[c] = stays(place(i, c), x[c]);
                add(x, in);
            },
            end_piece);
    } else {
        __syncthreads();
    }
    kept = wave_sum32(kept);
    if (lane == 0) atomicAdd(&sh.kept, kept);
    // Entries past the last piece hold no weight.
    for (int i = pieces + threadIdx.x; i < kBins; i += kThreads) sh.mass[i] = 0;
    __syncthreads();
    const float u = a.uniforms[r];
    const double at = u > 0.0f ? fmin(static_cast<double>(u), 1.0) : 0.0;
    auto aim = [&](uint64_t all) {  // the token is the first whose running weight exceeds it
        const uint64_t goal = static_cast<uint64_t>(at * static_cast<double>(all));
        return goal < all ? goal : all - 1;
    };
    const uint64_t total =
        scan_bins(sh, aim, [](uint64_t before, uint64_t v, uint64_t to) { return before <= to && to < before + v; });
    if (wave != 0) return;
    const uint64_t goal = aim(total);
    uint64_t before = sh.before;
    for (int i = static_cast<int>(sh.bin) << piece_log2;; i += 256) {
        float x[4];
        rw.load4(i + 4 * lane, x);
        uint64_t q[4], sum = 0;
#pragma unroll
        for (int c = 0; c < 4; ++c) {
            const double v = stays(i + 4 * lane + c, x[c]) ? w.of(x[c]) : 0.0;
            q[c] = v >= w.least ? Weights<PROBS>::whole(v) : 0;
            sum += q[c];
        }
        const uint64_t incl = wave_scan64(sum, lane);
        const uint64_t hit = __ballot(before + incl > goal);
        if (hit != 0) {
            if (lane == __ffsll(static_cast<unsigned long long>(hit)) - 1) {
                uint64_t here = before + incl - sum;
                int c = 0;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    here += q[j];
                    c += here <= goal ? 1 : 0;
                }
                const float v = c == 0 ? x[0] : c == 1 ? x[1] : c == 2 ? x[2] : x[3];
                a.token[r] = i + 4 * lane + c - rw.lead;
                if (a.prob != nullptr) a.prob[r] = static_cast<float>(w.of(v) / static_cast<double>(total));
                if (a.kept != nullptr) a.kept[r] = static_cast<int32_t>(sh.kept);
            }
            return;
        }
        before += __shfl(incl, 63);
        if (i + 256 >= rw.end) return;  // not reached: the piece holds the goal
    }
}

template <knn_dtype DT, bool HELD, bool PROBS>
__global__ __launch_bounds__(kThreads) void k_sample(SampleArgs a, int log2_unit, int piece_log2) {
    __shared__ Shared sh;
    extern __shared__ __align__(16) char held[];
    const int64_t r = blockIdx.x;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    using R = Row<DT, HELD, PROBS>;
    const char *first_of_row = static_cast<const char *>(a.scores) + r * a.stride * R::SIZE;
    const int lead = static_cast<int>(reinterpret_cast<uintptr_t>(first_of_row) % (4 * R::SIZE)) / R::SIZE;
    const R rw{first_of_row - lead * R::SIZE, held, lead, lead + a.V, (lead + a.V + (1 << piece_log2) - 1) >> piece_log2,
               piece_log2};

    if (threadIdx.x < 64) {
        sh.roots[threadIdx.x] = exp2(threadIdx.x * (1.0 / 64.0));
        if constexpr (PROBS) {
            const double c = 1.0 / (1.0 + (threadIdx.x + 0.5) * (1.0 / 64.0));
            sh.logs[threadIdx.x] = make_double2(c, -log2(c));
        }
    }
    float top = -INFINITY, low = INFINITY;  // the largest and the smallest present value
    rw.template pass<true>(
        wave, lane,
        [&](int, const float (&x)[4]) {
#pragma unroll
            for (int c = 0; c < 4; ++c) top = fmaxf(top, x[c]), low = fminf(low, x[c] > -INFINITY ? x[c] : INFINITY);
        },
        [](int) {});
    top = wave_allmax(top);
    low = wave_allmin(low);
    if (lane == 0) sh.part32[wave] = __float_as_uint(top), sh.part[wave] = __float_as_uint(low);
    if (threadIdx.x == 0) sh.kept = 0, sh.index = 0x7fffffff;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
        top = fmaxf(top, __uint_as_float(sh.part32[w]));
        low = fminf(low, __uint_as_float(static_cast<uint32_t>(sh.part[w])));
    }
    if (!(top > -INFINITY)) {
        if (threadIdx.x == 0) {
            a.token[r] = -1;
            if (a.prob != nullptr) a.prob[r] = 0.0f;
            if (a.kept != nullptr) a.kept[r] = 0;
        }
        return;
    }
    const float t = a.temperature != nullptr ? a.temperature[r] : 1.0f;
    const float p = a.top_p != nullptr ? a.top_p[r] : 1.0f;
    if (!(t > 0.0f) || p <= 0.0f) {  // the first element of the order
        int first = 0x7fffffff;
        rw.pass(
            wave, lane,
            [&](int i, const float (&x)[8]) {
#pragma unroll
                for (int c = 0; c < 8; ++c) first = x[c] == top && place(i, c) < first ? place(i, c) : first;
            },
            [](int) {});
        first = static_cast<int>(wave_allmin_u32(static_cast<uint32_t>(first)));
        if (lane == 0) atomicMin(&sh.index, first);
        __syncthreads();
        if (threadIdx.x == 0) {
            a.token[r] = sh.index - lead;
            if (a.prob != nullptr) a.prob[r] = 1.0f;
            if (a.kept != nullptr) a.kept[r] = 1;
        }
        return;
    }
    draw<PROBS>(a, rw, sh, r, top, low, t, p, log2_unit);
}

template <knn_dtype DT, bool PROBS>
void launch(const SampleArgs &a, int log2_unit, int piece_log2, hipStream_t stream) {
    const dim3 grid(static_cast<unsigned>(a.rows));
    // Whole pieces, with up to three places before the first element.
    const size_t bytes = ((static_cast<size_t>(a.V) + 3 + 511) & ~size_t{511}) * (DT == KNN_F32 ? 4 : 2);
    if (bytes <= kHeldBytes) k_sample<DT, true, PROBS><<<grid, kThreads, bytes, stream>>>(a, log2_unit, piece_log2);
    else k_sample<DT, false, PROBS><<<grid, kThreads, 0, stream>>>(a, log2_unit, piece_log2);
}

template <knn_dtype DT>
hipError_t launch(const SampleArgs &a, hipStream_t stream) {
    int bits = 0;
    while ((int64_t{1} << bits) < a.V + 3) ++bits;
    const int unit = bits < 11 ? 51 : 62 - bits;  // 2^51 is what a sum with 2^52 can round to a whole number
    const int piece = bits - 11 > kPieceLog2 ? bits - 11 : kPieceLog2;  // at most kBins pieces
    if (a.probabilities) launch<DT, true>(a, unit, piece, stream);
    else launch<DT, false>(a, unit, piece, stream);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_sample(const SampleArgs &a, knn_dtype dtype, void *, hipStream_t stream) {
    switch (dtype) {
    case KNN_F32: return launch<KNN_F32>(a, stream);
    case KNN_BF16: return launch<KNN_BF16>(a, stream);
    default: return launch<KNN_F16>(a, stream);
    }
}

}  // namespace knnlm
