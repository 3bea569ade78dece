// Drawing a token of a row: temperature, top-k, top-p, min-p, and the inverse
// of the running weight at a given uniform number.
//
// Weights are w_i = exp((x_i - max) / T) of logits or (x_i / max)^(1 / T) of
// probabilities, in 64 bits, and are summed as whole numbers of 2^-s of the
// largest one (2^s <= 2^62 / V, so no sum overflows).  Whole numbers add up to
// the same sum in any order, so the outcome depends neither on how a row is
// cut nor on the order of atomics; what a weight loses is under 2^-(s+1) of
// the largest, 2^-45 for 131,072 tokens, which moves the drawn token for one
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
// bits a pass.  A small k needs neither bins nor a weight for each element:
// the k-th largest of the threads' own largest values bounds it from below,
// and what is not under that bound is listed at once (32,000 logits, k = 50,
// p = 0.9: 17 us, 32 by bins).  Min-p alone lists what is above its value
// likewise (12 us, 18 by a pass that weighs).
//
// One workgroup takes a row.  A row of up to 128 KiB stays in LDS from the first
// pass on; a longer one is read three times, from the caches after the first.
//
// Measured, with the call: 32,000 bfloat16 logits, one row: largest element
// alone 6.7 us, drawn from all 18, top-p 24; 256 rows of 131,072 float logits
// with top-p 122 us, of which 19 would read them once.  The time is that of the
// issue of 64-bit operations: 13 of a weight's 20 instructions are such, a weight
// of 64 elements takes a SIMD about 160 clocks.  (Weights in 32 bits would draw
// another token in one row of 50.)  The pass after a cut weighs all 512 places of a
// wave where one of them stays; of a nucleus of one element in 25 that is next to
// all.  An atomic of 64 lanes on the bins takes 40 clocks of the CU.
#include "knnlm_device.h"
#include "lm_internal.h"

namespace knnlm {

namespace {

constexpr int kThreads = 1024;
constexpr int kWaves = kThreads / kWave;
constexpr int kBins = 2048;

constexpr size_t kHeldBytes = 128 * 1024;
constexpr int kList = 512;  // elements that are compared with each other
constexpr int kFew = 256;   // the largest k whose elements are listed at once

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
// 4e-17.  What is under 2^-200 counts as that; what is not `in` is under 2^-500.
__device__ __forceinline__ double power2(double y, bool in, int e, const double *roots) {
    y = fmax(y, -12800.0);
    // Not `in`: about -32768, by the high word alone.
    y = __hiloint2double(in ? __double2hiint(y) : static_cast<int>(0xc0e00000), __double2loint(y));
    const double moved = y + 6755399441055744.0;  // 1.5 2^52: the nearest whole number in the low bits
    const double f = y - (moved - 6755399441055744.0);
    const int n = static_cast<int>(__double_as_longlong(moved));
    const double root = roots[n & 63];
    double r = 1.2417843701716923e-12;           // c^5 / 5!, c = ln(2) / 64
    r = fma(r, f, 5.732851688640402e-10);       // c^4 / 4!
    r = fma(r, f, 2.1173137155464774e-07);       // c^3 / 3!
    r = fma(r, f, 5.864904955056169e-05);       // c^2 / 2
    r = fma(r, f, 0.010830424696249145);       // c
    const double v = fma(root, r * f, root);  // its exponent and the others' sum stay within those of normal numbers
    return __hiloint2double(__double2hiint(v) + ((n >> 6) + e) * (1 << 20), __double2loint(v));
}

// log2 of a positive finite x, its whole part apart from the rest, which is in
// [0, 1) and right to 2^-52: in one number the rest of a small probability
// would lose up to 7 bits to the whole part, and 1 / T as much more.  x = 2^e m,
// and with c one of 64 values near 1 / m, log2 m = -log2 c + log2(1 + r),
// r = m c - 1, |r| < 2^-6.9, by the series of the logarithm, whose 8th term is
// 2^-58.
struct Log2 {
    double rest;
    int whole;
};
__device__ __forceinline__ Log2 log2_of(float x, const double2 *logs) {
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
    return Log2{fma(r * q, 1.4426950408889634074, at.y), static_cast<int>(bits >> 52) - 1023};
}

// The weights of a row, as a function of the value; the largest one's is 2^s.
// Probabilities at T = 1 are their own weights (`plain`), brought under 2^s by
// a power of two.
template <bool PROBS>
struct Weights {
    double top;    // the largest value, or where the values are probabilities its log2: the rest, and
    int top_whole; // the whole part
    double rate;   // 64 log2(e) / T, or 64 / T of probabilities
    double unit;   // 2^s
    int log2_unit;
    bool plain;
    bool even;     // the largest value is infinite, and only such values stay
    const double *roots;
    const double2 *logs;

    // Of those `in`; of the others something that no whole number is left of.
    template <int N>
    __device__ __forceinline__ void of(const float (&x)[N], const bool (&in)[N], double (&v)[N]) const {
        if (even) {
#pragma unroll
            for (int c = 0; c < N; ++c) v[c] = in[c] ? unit : 0.0;
        } else if (PROBS && plain) {
#pragma unroll
            for (int c = 0; c < N; ++c) v[c] = static_cast<double>(in[c] ? x[c] : 0.0f) * unit;
        } else {
#pragma unroll
            for (int c = 0; c < N; ++c) {
                double far;
                if constexpr (PROBS) {
                    const Log2 l = log2_of(x[c], logs);
                    far = (l.rest - top) + static_cast<double>(l.whole - top_whole);
                } else {
                    far = static_cast<double>(x[c]) - top;
                }
                v[c] = power2(far * rate, in[c], log2_unit, roots);
            }
        }
    }
    __device__ __forceinline__ double of(float x) const {
        const float y[1] = {x};
        const bool in[1] = {true};
        double v[1];
        of(y, in, v);
        return v[0];
    }
    // To the nearest whole number: w < 2^52, so the sum's low bits are it.
    __device__ __forceinline__ static uint64_t whole(double w) {
        return static_cast<uint64_t>(__double_as_longlong(w + 4503599627370496.0) - 0x4330000000000000ll);
    }
};

// What a row asks for; read before the row, since each is a wait for memory of its own.
struct Wish {
    float u, t, p, min_p;
    int k;
};

struct Shared {
    double roots[64];  // 2^(i / 64)
    double2 logs[64];  // of the 64ths of [1, 2): c = 1 / its middle, -log2(c)
    uint64_t mass[kBins];  // bins, then the weights of the row's pieces
    uint64_t list[kList];  // key << 32 | ~index: larger is earlier in the order
    uint64_t weight[kList];
    uint64_t part[kWaves];
    uint32_t part32[kWaves];
    uint64_t before, cut, total;
    uint32_t bin, listed, kept, key;
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

// What the waves before this one have in sh.part, and what all have.
__device__ __forceinline__ uint64_t before_wave(const Shared &sh, int wave, int lane, uint64_t &all) {
    static_assert(kWaves == 16, "one row of 16 lanes scans them");
    uint64_t v = sh.part[lane & 15];
    v += dpp_u64<0x111>(v);  // row_shr:1
    v += dpp_u64<0x112>(v);  // row_shr:2
    v += dpp_u64<0x114>(v);  // row_shr:4
    v += dpp_u64<0x118>(v);  // row_shr:8
    all = readlane_u64(v, 15);
    return wave == 0 ? 0 : readlane_u64(v, wave - 1);
}

// The sum of sh.mass; with hit(before, own) true for one entry, its number and
// what lies before it in sh.bin and sh.before.
template <typename Goal, typename Hit>
__device__ __forceinline__ uint64_t scan_bins(Shared &sh, Goal goal_of, Hit hit) {
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint64_t a = sh.mass[2 * threadIdx.x], b = sh.mass[2 * threadIdx.x + 1];
    const uint64_t incl = wave_scan64(a + b, lane);
    if (lane == 63) sh.part[wave] = incl;
    __syncthreads();
    uint64_t total;
    const uint64_t before = before_wave(sh, wave, lane, total) + incl - a - b;
    const auto goal = goal_of(total);
    if (hit(before, a, goal)) sh.bin = 2 * threadIdx.x, sh.before = before;
    if (hit(before + a, b, goal)) sh.bin = 2 * threadIdx.x + 1, sh.before = before + a;
    __syncthreads();
    return total;
}

constexpr int kUnit = 512;  // places that a wave reads at a time

// A row of scores: in LDS from the first reading on (HELD), or in memory.  Its
// places start at the 4-element boundary in memory at or before the first
// element: element i is at place i + lead, places outside the row are absent.
template <knn_dtype DT, bool HELD, bool PROBS>
struct Row {
    static constexpr int SIZE = DT == KNN_F32 ? 4 : 2;
    const char *row;  // place 0
    char *held;
    int lead, end;  // the elements' places
    // Units of kUnit places; a wave has `each` of them, one after another, in `per` pieces of 2^group units (the last one
    // may be shorter): what the row's weights are summed by.
    int each, per, group;

    __device__ __forceinline__ int pieces() const { return kWaves * per; }
    __device__ __forceinline__ int units() const { return (end + kUnit - 1) / kUnit; }
    __device__ __forceinline__ int piece_of(int place) const {
        const int unit = place / kUnit, of = unit / each;
        return of * per + ((unit - of * each) >> group);
    }
    __device__ __forceinline__ int first_unit(int piece) const {
        return piece / per * each + ((piece % per) << group);
    }

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
    // Places i + 4 lane .. i + 4 lane + 3 (i the wave's, a multiple of 256).  Whether all of the wave's are in the row is
    // one scalar branch, so that no load is waited for before it is used.
    __device__ __forceinline__ void read4(int i, int lane, float (&x)[4]) const {
        if (i >= lead && i + 255 < end) {
            widen4(row + static_cast<int64_t>(i + 4 * lane) * SIZE, x);
        } else {
#pragma unroll
            for (int c = 0; c < 4; ++c) x[c] = at(i + 4 * lane + c);
        }
    }
    __device__ __forceinline__ void load4(int i, int lane, float (&x)[4]) const {
        if constexpr (HELD) widen4(held + (i + 4 * lane) * SIZE, x); else read4(i, lane, x);
    }
    __device__ __forceinline__ void load8(int i, int lane, float (&x)[8]) const {
        float u[4], v[4];
        load4(i, lane, u);
        load4(i + 256, lane, v);
#pragma unroll
        for (int c = 0; c < 4; ++c) x[c] = u[c], x[c + 4] = v[c];
    }
    // f(place, value) over this wave's pieces, one place a lane: where there is little code to spare.
    template <typename F, typename Done>
    __device__ __forceinline__ void slow_pass(int wave, int lane, F f, Done done) const {
        const int stop = min(units(), (wave + 1) * each);
        for (int unit = wave * each; unit < stop; ++unit) {
#pragma unroll 1
            for (int i = unit * kUnit; i < (unit + 1) * kUnit; i += kWave) f(i + lane, at(i + lane));
            ended(wave, unit, stop, done);
        }
    }
    template <typename Done>
    __device__ __forceinline__ void ended(int wave, int unit, int stop, Done done) const {
        const int n = unit - wave * each;
        if (((n + 1) & ((1 << group) - 1)) == 0 || unit + 1 == stop) done(wave * per + (n >> group));
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
        const int first = wave * each, last = min(units(), first + each);
        if constexpr (FIRST) {  // eight loads a lane in flight
            const int stop = last * kUnit;
            for (int i = first * kUnit; i < stop; i += 2048) {
                float x[8][4];
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    if (i + 256 * j < stop) read4(i + 256 * j, lane, x[j]);
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    if (i + 256 * j < stop) {
#pragma unroll
                        for (int c = 0; c < 4; ++c) x[j][c] = present(x[j][c], PROBS);
                        if constexpr (HELD) keep4(i + 256 * j + 4 * lane, x[j]);
                        f(i + 256 * j + 4 * lane, x[j]);
                    }
                }
            }
        } else {
            // x[c] is at place i + 4 lane + c + (c < 4 ? 0 : 252); the next eight are on their way meanwhile
            if (first >= last) return;
            float x[8], next[8];
            load8(first * kUnit, lane, x);
            for (int unit = first; unit < last; ++unit) {
                if (unit + 1 < last) load8((unit + 1) * kUnit, lane, next);
                if constexpr (!HELD) {
#pragma unroll
                    for (int c = 0; c < 8; ++c) x[c] = present(x[c], PROBS);
                }
                f(unit * kUnit + 4 * lane, x);
                ended(wave, unit, last, done);
#pragma unroll
                for (int c = 0; c < 8; ++c) x[c] = next[c];
            }
        }
    }
};

__device__ __forceinline__ int place(int i, int c) { return i + c + (c < 4 ? 0 : 252); }

// The filters and the draw of a row whose largest present value is `top` and
// smallest `low`, `mine` the largest that this thread read, at a temperature
// and a top-p above 0 and a min-p of up to 1.
template <bool PROBS, typename R>
__device__ __forceinline__ void draw(const SampleArgs &a, const R &rw, Shared &sh, int64_t r, float top, float low, float mine,
                                     const Wish &wish, int log2_unit) {
    const float t = wish.t, p = wish.p, min_p = wish.min_p;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int V = rw.end - rw.lead;
    auto pass = [&](auto f, auto done) { rw.pass(wave, lane, f, done); };
    auto nothing = [](int) {};
    Weights<PROBS> w;
    w.plain = PROBS && t == 1.0f;
    w.even = top == INFINITY;
    w.roots = sh.roots;
    w.logs = sh.logs;
    const Log2 top_log = PROBS ? log2_of(top, sh.logs) : Log2{static_cast<double>(top), 0};
    w.top = top_log.rest;
    w.top_whole = top_log.whole;
    w.rate = (PROBS ? 64.0 : 92.332482616893656874) / static_cast<double>(t);
    w.log2_unit = log2_unit - (w.plain && !w.even ? ilogb(static_cast<double>(top)) + 1 : 0);
    w.unit = ldexp(1.0, w.log2_unit);
    // What min-p leaves is not below `least`, the first value of enough weight: between one a thousandth of an octave
    // under it (log2f is right to 2^-20) and the largest, in 64ths.
    float least = -INFINITY;
    if (min_p > 0.0f && !w.even) {
        const double enough = w.of(top) * static_cast<double>(min_p);
        const float far = t * (log2f(min_p) - 0.001f);
        const float under = PROBS ? top * exp2f(far) * 0.999f
                                  : __double2float_rd(static_cast<double>(top) + 0.69314718 * static_cast<double>(far));
        uint32_t lo = key_of(under), hi = key_of(top);
        while (hi - lo > 1) {
            const uint32_t each = (hi - lo) / 64 + 1, key = min(lo + (lane + 1) * each, hi);
            const uint64_t above = __ballot(key == hi || w.of(value_of(key)) >= enough);
            const uint32_t n = __ffsll(static_cast<unsigned long long>(above)) - 1;
            hi = min(hi, lo + (n + 1) * each);
            lo += n * each;
        }
        least = value_of(hi);
    }

    // Bins that follow the order; what is past the last one's start is in it.
    // Logits: steps of the distance from the largest, over 32 T or the row's
    // range.  Probabilities: steps of the bits, which grow like a logarithm.
    // (Places do not depend on T: for them it is at least 1.)
    const uint32_t top_bits = __float_as_uint(top);
    float step = 0.0f;
    int shift = 0;
    auto bins_for = [&](float warm) {
        const float span = fminf(top - low, 32.0f * warm);
        step = span > 0.0f ? kBins / span : 0.0f;
        shift = 0;
        if (PROBS) {
            const float octaves = fminf(46.0f * warm, 255.0f);  // 2^-46 = e^-32
            uint32_t bits = min(top_bits - __float_as_uint(fminf(low, top)), static_cast<uint32_t>(octaves * 8388608.0f));
            while (bits >> shift >= kBins) ++shift;
        }
    };
    auto spot = [&](float x) {  // the bin, and of logits where in it
        if constexpr (PROBS) return min((top_bits - __float_as_uint(x)) >> shift, static_cast<uint32_t>(kBins - 1));
        else return fminf((top - x) * step, static_cast<float>(kBins - 1));
    };
    auto bin_of = [&](float x) { return static_cast<uint32_t>(spot(x)); };

    // What stays: x above `cut_x`, or equal to it with an index up to `cut_i`.
    float cut_x = top == INFINITY ? 3.402823466e38f : -INFINITY;
    int cut_i = -1;
    auto stays = [&](int i, float x) { return x > cut_x || (x == cut_x && i <= cut_i); };
    auto stay8 = [&](int i, const float (&x)[8], bool (&in)[8]) {
        bool equal = false;
#pragma unroll
        for (int c = 0; c < 8; ++c) in[c] = x[c] > cut_x, equal |= x[c] == cut_x;
        if (__any(equal)) {
#pragma unroll
            for (int c = 0; c < 8; ++c) in[c] = stays(place(i, c), x[c]);
        }
    };
    auto clear = [&]() {
        __syncthreads();
        sh.mass[2 * threadIdx.x] = 0;
        sh.mass[2 * threadIdx.x + 1] = 0;
        if (threadIdx.x == 0) sh.listed = 0, sh.cut = ~0ull, sh.total = 0, sh.key = ~0u;
        __syncthreads();
    };
    uint32_t kept = 0;  // by this wave
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
        w.of(x, in, v);
#pragma unroll
        for (int c = 0; c < 8; ++c) f(c, Weights<PROBS>::whole(v[c]));
    };
    auto add = [&](const float (&x)[8], const bool (&in)[8]) {
        bool keep[8];
#pragma unroll
        for (int c = 0; c < 8; ++c) {
            keep[c] = in[c] && x[c] >= least;
            kept += static_cast<uint32_t>(__popcll(__ballot(keep[c])));
        }
        weigh(x, keep, [&](int, uint64_t v) { run += v; });
    };
    auto count = [&](uint64_t v, uint32_t bin) {
        atomicAdd(reinterpret_cast<unsigned long long *>(&sh.mass[bin]), static_cast<unsigned long long>(v));
    };
    auto crosses = [](uint64_t at, uint64_t v, double to) {
        return static_cast<double>(at) < to && static_cast<double>(at + v) >= to;
    };
    auto list = [&](int i, float x) {
        const uint32_t at = atomicAdd(&sh.listed, 1u);
        if (at < kList) sh.list[at] = static_cast<uint64_t>(key_of(x)) << 32 | ~static_cast<uint32_t>(i);
    };
    auto weigh_list = [&](int n) {
        if (static_cast<int>(threadIdx.x) < n)
            sh.weight[threadIdx.x] =
                Weights<PROBS>::whole(w.of(value_of(static_cast<uint32_t>(sh.list[threadIdx.x] >> 32))));
        __syncthreads();
    };
    // The last of the n listed, `from` and earlier in the order, before which less than the goal lies, in sh.cut: eight
    // lanes an entry, each over an eighth of the others.  `take`: their weights are the row's.
    auto cut_list = [&](int n, uint64_t from, uint64_t before, double goal, bool by_weight, bool take) {
        for (int first = 0; first < n; first += kThreads / 8) {
            const int me = first + static_cast<int>(threadIdx.x >> 3);
            const uint64_t own = me < n ? sh.list[me] : ~0ull;
            uint64_t ahead = 0;
            for (int j = threadIdx.x & 7; j < n; j += 8) ahead += sh.list[j] > own ? (by_weight ? sh.weight[j] : 1) : 0;
            ahead += dpp_u64<0xB1>(ahead);
            ahead += dpp_u64<0x4E>(ahead);
            ahead += dpp_u64<0x141>(ahead);
            const bool ours = me < n && (threadIdx.x & 7) == 0 && own >= from && static_cast<double>(before + ahead) < goal;
            if (ours) atomicMin(reinterpret_cast<unsigned long long *>(&sh.cut), static_cast<unsigned long long>(own));
            const bool keep = ours && take && value_of(static_cast<uint32_t>(own >> 32)) >= least;
            if (keep) count(sh.weight[me], rw.piece_of(static_cast<int>(~static_cast<uint32_t>(own))));
            kept += static_cast<uint32_t>(__popcll(__ballot(keep)));
        }
        __syncthreads();
    };
    // Lists what is not below `from`; returns how many they are.
    auto list_from = [&](float from) {
        pass(
            [&](int i, const float (&x)[8]) {
                bool in[8], any = false;
#pragma unroll
                for (int c = 0; c < 8; ++c) any |= in[c] = x[c] >= from;
                if (!__any(any)) return;
#pragma unroll
                for (int c = 0; c < 8; ++c)
                    if (in[c]) list(place(i, c), x[c]);
            },
            nothing);
        __syncthreads();
        return static_cast<int>(sh.listed);
    };
    // The cuts: by count (top-k), then by weight (top-p).
    const int k = wish.k;
    bool stages[2] = {k > 0 && k < V, p < 1.0f};

    // Min-p alone: where few are left, only they are weighed.  (A pass that lists too many is lost: 6 us of 50,000 float
    // elements.  400 threads out of 1024 have an element of 512 that lie anywhere.)
    if (least > -INFINITY && !stages[0] && !stages[1] && __syncthreads_count(mine >= least) <= 384) {
        clear();
        const int n = list_from(least);
        if (n <= kList) {
            weigh_list(n);
            cut_list(n, 0, 0, INFINITY, false, true);
            cut_x = value_of(static_cast<uint32_t>(sh.cut >> 32));
            cut_i = static_cast<int>(~static_cast<uint32_t>(sh.cut));
            summed = true;
        }
    }

    // A small k: what is not below the k-th largest of the threads' own largest
    // values is k elements or more, and in an order that is not of the row's
    // making few more.  All of them listed, both cuts are among them, and
    // nothing else of the row is weighed.
    if (stages[0] && k <= kFew) {
        bins_for(fmaxf(t, 1.0f));
        clear();
        const bool in = mine > cut_x;
        if (in) count(1, bin_of(mine));
        __syncthreads();
        auto goal_of = [&](uint64_t) { return static_cast<double>(k); };
        if (scan_bins(sh, goal_of, crosses) >= static_cast<uint64_t>(k)) {
            const uint32_t bin = sh.bin;
            clear();
            if (in && bin_of(mine) <= bin) atomicMin(&sh.key, key_of(mine));
            __syncthreads();
            const int n = list_from(value_of(sh.key));
            if (n <= kList) {
                weigh_list(n);
                cut_list(n, 0, 0, k, false, !stages[1]);
                if (stages[1]) {
                    const uint64_t from = sh.cut;
                    const bool stay = static_cast<int>(threadIdx.x) < n && sh.list[threadIdx.x] >= from;
                    const uint64_t sum = wave_sum64(stay ? sh.weight[threadIdx.x] : 0);
                    if (lane == 0 && sum != 0)
                        atomicAdd(reinterpret_cast<unsigned long long *>(&sh.total), static_cast<unsigned long long>(sum));
                    __syncthreads();
                    if (threadIdx.x == 0) sh.cut = ~0ull;
                    __syncthreads();
                    cut_list(n, from, 0, p * static_cast<double>(sh.total), true, true);
                }
                cut_x = value_of(static_cast<uint32_t>(sh.cut >> 32));
                cut_i = static_cast<int>(~static_cast<uint32_t>(sh.cut));
                summed = true;
                stages[0] = stages[1] = false;
            }
        }
    }
#pragma unroll 1
    for (int stage = 0; stage < 2; ++stage) {
        if (stage == 0 ? !stages[0] : !stages[1]) continue;
        const bool by_weight = stage == 1, last = by_weight || !stages[1];  // last: sums the row's pieces too
        bins_for(by_weight ? t : fmaxf(t, 1.0f));
        clear();
        pass(
            [&](int i, const float (&x)[8]) {
                bool in[8];
                stay8(i, x, in);
                if (by_weight) {
                    weigh(x, in, [&](int c, uint64_t v) {
                        if (v != 0) count(v, bin_of(x[c]));
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
        const uint64_t all = scan_bins(sh, goal_of, crosses);
        if (!by_weight && static_cast<uint64_t>(k) >= all) continue;  // all that is present stays
        const double goal = goal_of(all);
        const uint32_t bin = sh.bin;
        const uint64_t before = sh.before;
        const auto bin_first = static_cast<decltype(spot(0.0f))>(bin), bin_end = bin_first + 1;
        clear();  // for the pieces' weights
        pass(
            [&](int i, const float (&x)[8]) {
                bool in[8], under[8], at[8], any = false;
                stay8(i, x, in);
#pragma unroll
                for (int c = 0; c < 8; ++c) {
                    const auto b = spot(x[c]);
                    under[c] = in[c] && b < bin_first;
                    at[c] = in[c] && b >= bin_first && b < bin_end;
                    any |= at[c];
                }
                if (__any(any)) {
#pragma unroll
                    for (int c = 0; c < 8; ++c)
                        if (at[c]) list(place(i, c), x[c]);
                }
                if (last) add(x, under);
            },
            [&](int piece) {
                if (last) end_piece(piece);
            });
        __syncthreads();
        const int n = static_cast<int>(sh.listed);
        if (n <= kList) {
            weigh_list(n);
            cut_list(n, 0, before, goal, by_weight, last);
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
            for (int i = rw.first_unit(static_cast<int>(sh.bin)) * kUnit; !found; i += kWave) {
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
                stay8(i, x, in);
                add(x, in);
            },
            end_piece);
    } else {
        __syncthreads();
    }
    if (lane == 0) atomicAdd(&sh.kept, kept);
    __syncthreads();
    const double at = wish.u > 0.0f ? fmin(static_cast<double>(wish.u), 1.0) : 0.0;
    auto aim = [&](uint64_t all) {  // the token is the first whose running weight exceeds it
        const uint64_t goal = static_cast<uint64_t>(at * static_cast<double>(all));
        return goal < all ? goal : all - 1;
    };
    const uint64_t total =
        scan_bins(sh, aim, [](uint64_t before, uint64_t v, uint64_t to) { return before <= to && to < before + v; });
    const uint64_t goal = aim(total);
    uint64_t before = sh.before;
    for (int i = rw.first_unit(static_cast<int>(sh.bin)) * kUnit; i < rw.end; i += kWaves * 256) {  // 256 places a wave
        const int own = i + 256 * wave;
        float x[4];
        uint64_t q[4], sum = 0;
        if (own < rw.end) {
            rw.load4(own, lane, x);
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                x[c] = present(x[c], PROBS);
                const bool in = x[c] >= least && stays(own + 4 * lane + c, x[c]);
                q[c] = in ? Weights<PROBS>::whole(w.of(x[c])) : 0;
                sum += q[c];
            }
        }
        const uint64_t incl = wave_scan64(sum, lane);
        __syncthreads();
        if (lane == 63) sh.part[wave] = incl;
        __syncthreads();
        uint64_t all;
        uint64_t here = before + before_wave(sh, wave, lane, all) + incl - sum;
        if (here <= goal && goal < here + sum) {
            int c = 0;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                here += q[j];
                c += here <= goal ? 1 : 0;
            }
            const float v = c == 0 ? x[0] : c == 1 ? x[1] : c == 2 ? x[2] : x[3];
            a.token[r] = own + 4 * lane + c - rw.lead;
            if (a.prob != nullptr) a.prob[r] = static_cast<float>(w.of(v) / static_cast<double>(total));
            if (a.kept != nullptr) a.kept[r] = static_cast<int32_t>(sh.kept);
        }
        before += all;
        if (before > goal) return;
    }
}

template <knn_dtype DT, bool HELD, bool PROBS>
__global__ __launch_bounds__(kThreads) void k_sample(SampleArgs a, int log2_unit, int group) {
    __shared__ Shared sh;
    extern __shared__ __align__(16) char held[];
    const int64_t r = blockIdx.x;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    using R = Row<DT, HELD, PROBS>;
    const char *first_of_row = static_cast<const char *>(a.scores) + r * a.stride * R::SIZE;
    const int lead = static_cast<int>(reinterpret_cast<uintptr_t>(first_of_row) % (4 * R::SIZE)) / R::SIZE;
    const int each = ((lead + a.V + kUnit - 1) / kUnit + kWaves - 1) / kWaves;
    const R rw{first_of_row - lead * R::SIZE, held, lead, lead + a.V, each, ((each - 1) >> group) + 1, group};

    Wish wish;
    wish.u = a.uniforms[r];
    wish.t = a.temperature != nullptr ? a.temperature[r] : 1.0f;
    wish.p = a.top_p != nullptr ? a.top_p[r] : 1.0f;
    wish.min_p = a.min_p != nullptr ? a.min_p[r] : 0.0f;
    wish.k = a.top_k != nullptr ? a.top_k[r] : 0;
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
    const float mine = top;
    top = wave_allmax(top);
    low = wave_allmin(low);
    if (lane == 0) sh.part32[wave] = __float_as_uint(top), sh.part[wave] = __float_as_uint(low);
    if (threadIdx.x == 0) sh.kept = 0, sh.index = 0x7fffffff;
    __syncthreads();
    top = wave_allmax(__uint_as_float(sh.part32[lane & 15]));
    low = wave_allmin(__uint_as_float(static_cast<uint32_t>(sh.part[lane & 15])));
    if (!(top > -INFINITY)) {
        if (threadIdx.x == 0) {
            a.token[r] = -1;
            if (a.prob != nullptr) a.prob[r] = 0.0f;
            if (a.kept != nullptr) a.kept[r] = 0;
        }
        return;
    }
    // The first element of the order.  A min-p above 1 leaves only that one too: no weight reaches it, not even an equal one's.
    if (!(wish.t > 0.0f) || wish.p <= 0.0f || wish.min_p > 1.0f) {
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
    draw<PROBS>(a, rw, sh, r, top, low, mine, wish, log2_unit);
}

template <knn_dtype DT, bool PROBS>
void launch(const SampleArgs &a, int log2_unit, int group, hipStream_t stream) {
    const dim3 grid(static_cast<unsigned>(a.rows));
    // Whole pieces, with up to three places before the first element.
    const size_t bytes = ((static_cast<size_t>(a.V) + 3 + 511) & ~size_t{511}) * (DT == KNN_F32 ? 4 : 2);
    if (bytes <= kHeldBytes) k_sample<DT, true, PROBS><<<grid, kThreads, bytes, stream>>>(a, log2_unit, group);
    else k_sample<DT, false, PROBS><<<grid, kThreads, 0, stream>>>(a, log2_unit, group);
}

template <knn_dtype DT>
hipError_t launch(const SampleArgs &a, hipStream_t stream) {
    int bits = 0;
    while ((int64_t{1} << bits) < a.V + 3) ++bits;
    const int unit = bits < 11 ? 51 : 62 - bits;  // 2^51 is what a sum with 2^52 can round to a whole number
    const int group = bits > 22 ? bits - 20 : 2;  // at most kBins pieces
    if (a.probabilities) launch<DT, true>(a, unit, group, stream);
    else launch<DT, false>(a, unit, group, stream);
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
