// Tokens from logits: temperature, top-k, top-p, min-p and a draw by one random number per row.
//
// The order of the tokens is never written out: what is kept ends at a logit and, among tokens with that logit, at a token number, and both are
// found by histograms of counts or weights that narrow an interval 2048-fold.  Weights are computed in binary64 and rounded to 64-bit fixed point: integer sums
// are the same in any order, so atomics on LDS leave no trace, and borders lie where exact sums put them (off by 2^-42 of the greatest
// weight per token), not where a rounding of a long binary32 sum would.
//
// A workgroup has a row, whose first tokens it keeps in LDS: no second launch, no sums in memory, and rows of different settings side by side.  HBM bounds none of this.
// Rows of greedy tokens are bound by what a CU reads (64 x 131071 binary16 15 us), top-k of up to 128 by that and a chain of some ten barriers (64 x 131071 17.5 us, one
// row of 32000 9), all others by their passes over the row with a weight in binary64, some 130 cycles for the 64 tokens of a wave: one row of 32000 with temperature alone 16
// us, with top-p 0.9 28 to 30; 300 rows of 32003 28 and 53 to 57.  Few rows leave CUs idle: to divide a row among several, all would have to wait for each other
// between passes, three times at least.
#include <cfloat>
#include <cstddef>
#include <type_traits>

#include "decode_device.h"

namespace apgemv {

namespace {

struct SampleArgs {
    const void *logits;
    int64_t stride, rows;
    const float *uniform, *temperature, *top_p, *min_p;
    const int32_t *top_k;
    int64_t *tokens;
    void *probabilities;
    int vocabulary;
    int unit; // a weight of 1 is 2^unit
};

constexpr int kEach = 8;          // adjacent tokens of a lane and tile
constexpr int kTile = 64 * kEach; // tokens of a wave and step: up to 2^20 / kTile = kBins sums of tiles take the bins' place
constexpr int kBins = 2048;
constexpr int kList = 2048;       // tokens that are listed
// Top-k up to which a row's candidates are listed, found by groups of 8 tokens where there are four for each of the k (with fewer they give a limit that lists too many), or, up
// to kFew and a quarter of the lanes, by the tokens of each lane.  us, binary16, top-p too, one row of 131071 by lanes / by groups: top-k 20 11.6 / 18.5, 100 18.1 / 21.9, 128
// 22.0 / 24.6, 200 30.2 / 29.7, 256 45.4 / 29.6; by groups / without: 129 24.6 / 80, 500 31.7 / 100, 1000 35.7 / 108, 1500 39 / 111, 2000 140 / 117, as the list overflows.  300 rows
// of 32000 by lanes / by groups: 100 21.4 / 21.8, 128 30.4 / 28.3.  Four groups for each are on the safe side, by groups / without: 8000 tokens 256 16.4 / 18.4, 400 16.9 / 20.1,
// 1000 23.5 / 20.7; 32000 tokens 1024 22.6 / 39.1.
constexpr int kMostListed = 1024;
constexpr int kFew = 128;
constexpr int kRanked = 256; // tokens that are ranked among each other, at most
constexpr int kWaves = 16;        // of a workgroup, at most
constexpr int kFinders = 4;       // waves that look for a place in the bins: all 16 take turns on the four SIMDs, and twice as long
constexpr double kLog2e = 1.4426950408889634, kLn2 = 0.6931471805599453;

// Greater logits have smaller keys; -0 and 0 the same one
__device__ __forceinline__ uint32_t key_of(float x)
{
    const uint32_t b = __float_as_uint(x + 0.0f);
    return b >> 31 ? b : ~(b | 0x80000000u);
}
__device__ __forceinline__ float logit_of(uint32_t key) { return __uint_as_float(key >> 31 ? key : ~key & 0x7fffffffu); }

// Sums over the lanes up to each, by data-parallel moves: of rows of 16 (ROWS), or of all 64
template <int CTRL, int ROWS> __device__ __forceinline__ uint64_t moved(uint64_t x)
{
    const uint32_t low = __builtin_amdgcn_update_dpp(0, (int)(uint32_t)x, CTRL, ROWS, 0xf, false), high = __builtin_amdgcn_update_dpp(0, (int)(uint32_t)(x >> 32), CTRL, ROWS, 0xf, false);
    return (uint64_t)high << 32 | low;
}
__device__ __forceinline__ uint64_t row_scan(uint64_t x)
{
    x += moved<0x111, 0xf>(x); // row_shr:1, 2, 4, 8
    x += moved<0x112, 0xf>(x);
    x += moved<0x114, 0xf>(x);
    return x + moved<0x118, 0xf>(x);
}
__device__ __forceinline__ uint64_t wave_scan(uint64_t x)
{
    x = row_scan(x);
    x += moved<0x142, 0xa>(x); // row_bcast:15 into rows 1 and 3
    return x + moved<0x143, 0xc>(x); // row_bcast:31 into rows 2 and 3
}
__device__ __forceinline__ uint64_t lane_of(uint64_t x, int lane)
{
    return (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(x >> 32), lane) << 32 | (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)x, lane);
}

// 2^(j / kSteps), by the power series of exp
constexpr int kSteps = 512;
struct Powers {
    double x[kSteps];
    constexpr Powers() : x()
    {
        for (int j = 0; j < kSteps; ++j) {
            double sum = 1.0;
            for (int i = 20; i > 0; --i) sum = 1.0 + sum * (j * (kLn2 / kSteps)) / i;
            x[j] = sum;
        }
    }
};
__device__ constexpr Powers kPowers;

constexpr uint64_t kFixedBase = 0x4330000000000000ull; // the bits of 2^52

// What the tokens of a row weigh: 2^(d / kSteps) with d = kSteps log2 e (x - most) / temperature <= 0, as 2^n times a table's 2^(j / kSteps) times the power series
// of exp on half a step either way, off by 1e-14 (with a table of 64 one more term).  Adding 1.5 2^52 leaves the whole part of d in the low bits of the sum.
struct Weights {
    double most, rate;
    const double *table; // LDS
    int unit;
    float floor, far; // logits that weigh less than 2^-3 in fixed point, and less than 2^-160; not infinite
    // 2^scale times the weight of x
    __device__ __forceinline__ double of(float x, int scale) const
    {
        const double magic = 0x1.8p52 + (double)kSteps * scale, y = (double)x - most, t = __builtin_fma(y, rate, magic), f = __builtin_fma(y, rate, magic - t);
        const int k = (int)(uint32_t)__double_as_longlong(t);
        constexpr double c = kLn2 / kSteps;
        double p = __builtin_fma(c * c * c / 6, f, c * c / 2);
        p = __builtin_fma(p, f, c);
        p = __builtin_fma(p, f, 1.0);
        return __longlong_as_double(__double_as_longlong(table[k & (kSteps - 1)] * p) + ((long long)(k >> 9) << 52));
    }
    // In fixed point: a number below 2^52 added to 2^52 has its integer part in the low bits, kFixedBase above them.  Not for logits below floor.
    __device__ uint64_t fixed_up(float x) const { return (uint64_t)__double_as_longlong(of(x, unit) + 0x1p52); }
    __device__ uint64_t fixed(float x) const { return fixed_up(fmaxf(x, floor)) - kFixedBase; }
    // a number below 2^-159 instead of any less
    __device__ double exact(float x) const { return of(fmaxf(x, far), 0); }
};
static_assert(kSteps == 1 << 9, "the shift of Weights::of");

// The beginning of the order that is kept: logits above x, and of those equal to it the tokens up to `last`
struct Cut {
    float x;
    int last;
    __device__ __forceinline__ bool keeps(float y, int v) const { return y > x || (y == x && v <= last); }
    // of n adjacent tokens; mostly all that are equal to x are kept
    template <int n> __device__ __forceinline__ void keeps(const float (&y)[n], int v, bool (&out)[n]) const
    {
#pragma unroll
        for (int i = 0; i < n; ++i) out[i] = y[i] >= x && y[i] > -INFINITY;
        if (last < 0x7fffffff) {
#pragma unroll
            for (int i = 0; i < n; ++i) out[i] = keeps(y[i], v + i);
        }
    }
};

// 8 adjacent values of rows that start at any element: 16-byte accesses that ask for the element's alignment only
template <class T> struct Eight {
    typedef T values_t __attribute__((ext_vector_type(kEach)));
    struct __attribute__((packed, aligned(sizeof(T)))) Place {
        values_t x;
    };
    __device__ static values_t load(const T *row, int v, int count)
    {
        if (v + kEach <= count) return reinterpret_cast<const Place *>(row + v)->x;
        values_t e;
#pragma unroll
        for (int i = 0; i < kEach; ++i) e[i] = v + i < count ? row[v + i] : (T)-INFINITY;
        return e;
    }
    __device__ static void store(T *row, int v, int count, values_t e)
    {
        if (v + kEach <= count) {
            reinterpret_cast<Place *>(row + v)->x = e;
            return;
        }
        for (int i = 0; i < kEach - 1; ++i)
            if (v + i < count) row[v + i] = e[i];
    }
};

// The wave's number as a scalar, so that branches on its tiles are
__device__ __forceinline__ int wave_of_block() { return __builtin_amdgcn_readfirstlane(threadIdx.x >> 6); }

// A row of logits.  Its first `staged` tokens (a multiple of kTile) are in LDS, -inf behind the last one; the others are read again in every pass.
template <class T> struct Row {
    const T *x;
    const T *stage;
    int staged, vocabulary;
    bool infinite; // +inf is the greatest: such logits are 0, all others -inf

    // NaN stays: no comparison holds for it
    __device__ float value(T t) const
    {
        const float x = (float)t;
        if (infinite) return x == INFINITY ? 0.0f : -INFINITY;
        return x;
    }
    // the lane's logits of tile t, a scalar; returns the first one's token
    __device__ __forceinline__ int tile(int t, float (&out)[kEach]) const
    {
        const int v = t * kTile + (threadIdx.x & 63) * kEach;
        typename Eight<T>::values_t e;
        if (t * kTile < staged) e = *reinterpret_cast<const typename Eight<T>::values_t *>(stage + v);
        else e = Eight<T>::load(x, v, vocabulary);
#pragma unroll
        for (int i = 0; i < kEach; ++i) out[i] = (float)e[i];
        if (infinite) {
#pragma unroll
            for (int i = 0; i < kEach; ++i) out[i] = out[i] == INFINITY ? 0.0f : -INFINITY;
        }
        return v;
    }
    // f(logits, first token) for the wave's tiles
    template <class F> __device__ __forceinline__ void tiles(const F &f) const
    {
        const int waves = blockDim.x >> 6;
        for (int t = wave_of_block(); t * kTile < vocabulary; t += waves) {
            float e[kEach];
            const int v = tile(t, e);
            f(e, v);
        }
    }
    // f(logit, token), in little code for what is seldom run
    template <class F> __device__ __forceinline__ void each(const F &f) const
    {
#pragma unroll 1
        for (int v = threadIdx.x; v < vocabulary; v += blockDim.x) f(value(v < staged ? stage[v] : x[v]), v);
    }
};

// The tokens that s.list holds, as few as may be kept
struct List {
    const uint2 *list;
    int count, vocabulary;
    template <class F> __device__ __forceinline__ void tiles(const F &f) const
    {
        for (int i = threadIdx.x; i < count; i += blockDim.x) {
            const uint2 x = list[i];
            const float e[1] = {logit_of(x.y)};
            f(e, (int)x.x);
        }
    }
};

struct Shared {
    alignas(16) uint64_t bins[kBins]; // or the sums of tiles; read and cleared by 16 bytes
    uint2 list[kList];           // (token, key)
    double table[kSteps];
    uint64_t wave_sum[kFinders];
    uint64_t before, amount, all, wanted;
    float wave_most[kWaves];
    uint32_t low, high;
    int count, place, kept, zeroed;
};
static_assert(offsetof(Shared, bins) % 16 == 0 && alignof(Shared) % 16 == 0, "16-byte accesses of the bins");

// Where in the sum of kept weights a uniform number draws: the first token up to which they reach it.  At least 1, at most the sum.
__device__ __forceinline__ uint64_t wanted_of(float u, uint64_t sum)
{
    const double x = __builtin_floor((double)u * (double)sum);
    return !(u < 1) || x >= (double)sum ? sum : x > 0 ? (uint64_t)x + 1 : 1;
}
// The weight that a share of the sum asks for
__device__ __forceinline__ uint64_t share_of(float p, uint64_t sum)
{
    const double x = __builtin_ceil((double)p * (double)sum);
    return x >= 1 ? (uint64_t)x : 1;
}

// The first of `count` numbers in LDS at which the sum up to it reaches the target that target(sum of all) gives: s.place, s.before (the sum before it), s.amount
// (it), s.all and s.wanted, the target.  count <= kBins.  A target is 1 at least; one beyond the sum leaves s.place at -1.
template <class F> __device__ __forceinline__ void find(Shared &s, int count, const F &target)
{
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, finders = blockDim.x >> 6 < kFinders ? blockDim.x >> 6 : kFinders;
    const int per = (count + 64 * finders - 1) / (64 * finders), first = threadIdx.x * per;
    constexpr int kMost = kBins / (64 * kFinders);
    const bool all_bins = count == kBins && finders == kFinders;
    uint64_t x[kMost], mine = 0, upto = 0;
    if (wave < finders) {
        if (all_bins) {
            typedef uint64_t pair_t __attribute__((ext_vector_type(2)));
#pragma unroll
            for (int i = 0; i < kMost; i += 2) {
                const pair_t y = *reinterpret_cast<const pair_t *>(&s.bins[first + i]);
                x[i] = y[0], x[i + 1] = y[1];
                mine += y[0] + y[1];
            }
        } else {
            for (int i = 0; i < per; ++i)
                if (first + i < count) mine += s.bins[first + i];
        }
        upto = wave_scan(mine);
        if (lane == 63) s.wave_sum[wave] = upto;
        if (threadIdx.x == 0) s.place = -1;
    }
    __syncthreads();
    if (wave < finders) {
        uint64_t before = upto - mine, all = 0;
#pragma unroll
        for (int w = 0; w < kFinders; ++w) {
            const uint64_t y = w < finders ? s.wave_sum[w] : 0;
            before += w < wave ? y : 0;
            all += y;
        }
        const uint64_t wanted = target(all);
        if (threadIdx.x == 0) s.all = all, s.wanted = wanted;
        if (before < wanted && wanted <= before + mine) {
            if (all_bins) {
#pragma unroll
                for (int i = 0; i < kMost; ++i) {
                    if (before < wanted && wanted <= before + x[i]) s.place = first + i, s.before = before, s.amount = x[i];
                    before += x[i];
                }
            } else {
                for (int i = 0; i < per; ++i) {
                    const uint64_t y = s.bins[first + i];
                    if (wanted <= before + y) {
                        s.place = first + i, s.before = before, s.amount = y;
                        break;
                    }
                    before += y;
                }
            }
        }
    }
    __syncthreads();
}

__device__ __forceinline__ void clear_bins(Shared &s)
{
    for (int i = threadIdx.x; i < kBins / 2; i += blockDim.x) reinterpret_cast<uint4_t *>(s.bins)[i] = uint4_t{0, 0, 0, 0};
    __syncthreads();
}
__device__ __forceinline__ void add(Shared &s, int bin, uint64_t x) { atomicAdd((unsigned long long *)&s.bins[bin], (unsigned long long)x); }

// The place of a logit among the first bins, which are even in it, 40 to a factor of two in the weight: tokens spread over many, and few are in the one
// that matters.  The last bin holds all the rest, whose weights are 0 in fixed point.
constexpr int kBinsPerOctave = 40;
static_assert(kBins / kBinsPerOctave >= 51, "the smallest weight in fixed point");
struct Even {
    float most, rate;
    __device__ float place(float x) const { return (most - x) * rate; }
    __device__ int bin(float x) const { return (int)fminf(place(x), (float)(kBins - 1)); }
};

// Where the tokens that `cut` keeps, in order, reach `count` (weigh = false), or their weights the share p of their sum.
//
// The tokens of the even bin that reaches it are listed.  Few are ranked among each other; else their interval of keys is divided into bins until one key is left; where it has more tokens than
// are wanted, an interval of token numbers is, for the first ones.  A bin that holds more than the list is looked for in the row.
template <class S> __device__ __forceinline__ Cut select(Shared &s, const S &source, const Weights &w, const Cut cut, const Even even, bool weigh, int count, float p)
{
    constexpr bool kListed = std::is_same_v<S, List>;
    clear_bins(s);
    source.tiles([&](const auto &e, int v) {
        constexpr int n = sizeof(e) / sizeof(e[0]);
        bool keep[n];
        cut.keeps(e, v, keep);
        if (weigh) { // (weights of 0 stay away: they are many where one token has nearly all)
            uint64_t x[n];
#pragma unroll
            for (int i = 0; i < n; ++i) x[i] = w.fixed(e[i]);
#pragma unroll
            for (int i = 0; i < n; ++i)
                if (keep[i] && e[i] >= w.floor) add(s, even.bin(e[i]), x[i]);
        } else {
#pragma unroll
            for (int i = 0; i < n; ++i)
                if (keep[i]) add(s, even.bin(e[i]), 1);
        }
    });
    if (threadIdx.x == 0) s.count = 0, s.low = 0xffffffffu, s.high = 0;
    __syncthreads();
    find(s, kBins, [&](uint64_t all) { return weigh ? share_of(p, all) : (uint64_t)count; });
    const int bin = s.place;
    if (bin < 0) return cut; // fewer tokens than wanted
    uint64_t wanted = s.wanted - s.before, amount = s.amount;
    const float from = bin, to = bin == kBins - 1 ? __builtin_nanf("") : (float)(bin + 1); // not at or beyond NaN: everything
    const auto inside = [&](float x, int v) {
        const float at = even.place(x);
        return at >= from && !(at >= to) && cut.keeps(x, v);
    };
    uint64_t *const orders = s.bins; // of the bin's tokens
    source.tiles([&](const auto &e, int v) {
        constexpr int n = sizeof(e) / sizeof(e[0]);
#pragma unroll
        for (int i = 0; i < n; ++i)
            if (inside(e[i], v + i)) {
                const uint32_t key = key_of(e[i]);
                const int at = atomicAdd(&s.count, 1);
                if (at < kRanked) orders[at] = (uint64_t)key << 32 | (uint32_t)(v + i);
                if (!kListed && at < kList) s.list[at] = make_uint2(v + i, key);
                atomicMin(&s.low, key);
                atomicMax(&s.high, key);
            }
    });
    __syncthreads();
    int listed = s.count;
    if (const int columns = (listed + 63) & ~63; listed <= kRanked && columns <= (int)blockDim.x) {
        // few: each one's sum of those ahead of it, in parts of the others
        uint64_t *const weights = s.bins + kRanked, *const aheads = s.bins + 2 * kRanked;
        const int i = threadIdx.x, column = i % columns, part = i / columns, parts = blockDim.x / columns;
        if (i < columns) weights[i] = i >= listed ? 0 : weigh ? w.fixed(logit_of((uint32_t)(orders[i] >> 32))) : 1, aheads[i] = 0;
        if (threadIdx.x == 0) s.place = 0;
        __syncthreads();
        const uint64_t order = orders[column < listed ? column : 0];
        if (column < listed && part < parts) {
            uint64_t ahead = 0;
            for (int j = part; j < listed; j += parts) ahead += orders[j] < order ? weights[j] : 0;
            atomicAdd((unsigned long long *)&aheads[column], (unsigned long long)ahead);
        }
        __syncthreads();
        if (i < listed && aheads[i] < wanted && wanted <= aheads[i] + weights[i]) s.low = (uint32_t)(order >> 32), s.high = (uint32_t)order;
        __syncthreads();
        if (i < listed && (uint32_t)(order >> 32) == s.low && (uint32_t)order > s.high) s.place = 1; // one with the same logit is not kept
        __syncthreads();
        const float x = logit_of(s.low);
        return Cut{x, s.place ? (int)s.high : x == cut.x ? cut.last : 0x7fffffff};
    }
    if constexpr (kListed) listed = source.count;
    uint32_t low = s.low, high = s.high, key = 0;
    bool numbers = false; // of the tokens with `key`
    while (low <= high) {
        if (low == high) {
            if (numbers) return Cut{logit_of(key), (int)low};
            key = low;
            const float x = logit_of(key);
            const uint64_t one = weigh ? w.fixed(x) : 1;
            wanted = (wanted + one - 1) / one;
            if (wanted >= amount / one) return Cut{x, x == cut.x ? cut.last : 0x7fffffff};
            numbers = true;
            low = 0, high = source.vocabulary - 1;
        }
        const int bits = 32 - __builtin_clz(high - low), shift = bits > 11 ? bits - 11 : 0;
        clear_bins(s);
        const auto consider = [&](int v, uint32_t k) {
            const uint32_t number = numbers ? (uint32_t)v : k;
            if (number >= low && number <= high && (!numbers || k == key)) add(s, (number - low) >> shift, weigh && !numbers ? w.fixed(logit_of(k)) : 1);
        };
        if (listed <= kList) {
            for (int i = threadIdx.x; i < listed; i += blockDim.x) {
                const uint2 x = s.list[i];
                if (!kListed || cut.keeps(logit_of(x.y), (int)x.x)) consider((int)x.x, x.y);
            }
        } else if constexpr (!kListed) {
            source.each([&](float x, int v) {
                if (inside(x, v)) consider(v, key_of(x));
            });
        }
        __syncthreads();
        find(s, kBins, [&](uint64_t) { return wanted; });
        const int at = s.place < 0 ? 0 : s.place; // always found
        wanted -= s.before;
        amount = s.amount;
        low += (uint32_t)at << shift;
        const uint32_t end = low + ((1u << shift) - 1);
        high = end < high ? end : high;
        __syncthreads();
    }
    return cut; // not reached: the bin holds tokens
}

// Candidates of a small top-k.  The k-th best of the greatest logits of groups of tokens leaves k tokens before it at least, and few more where k is small beside the
// groups: those are listed.  Groups are the tokens of a lane (groups = false: of 1024) or 8 adjacent ones.  Returns their number, -1 where the place is not to be had.
template <class T> __device__ __forceinline__ int candidates(Shared &s, const Row<T> &row, const Even even, float lane_most, int k, bool groups)
{
    const auto top_of = [](const float(&e)[kEach]) {
        float top = e[0];
#pragma unroll
        for (int i = 1; i < kEach; ++i) top = fmaxf(top, e[i]);
        return top;
    };
    clear_bins(s);
    if (groups) {
        row.tiles([&](const float(&e)[kEach], int) {
            const float top = top_of(e);
            if (top > -INFINITY) add(s, even.bin(top), 1);
        });
    } else if (lane_most != -INFINITY) {
        add(s, even.bin(lane_most), 1);
    }
    if (threadIdx.x == 0) s.count = 0, s.kept = 0;
    __syncthreads();
    find(s, kBins, [&](uint64_t) { return (uint64_t)k; });
    const int bin = s.place;
    if (bin < 0 || bin == kBins - 1) return -1;
    const float limit = bin + 1;
    const auto put = [&](float x, int v) {
        if (!(even.place(x) < limit)) return;
        const int at = atomicAdd(&s.count, 1);
        if (at < kList) s.list[at] = make_uint2(v, key_of(x));
    };
    if (groups) {
        row.tiles([&](const float(&e)[kEach], int v) {
            if (!(even.place(top_of(e)) < limit)) return;
#pragma unroll
            for (int i = 0; i < kEach; ++i) put(e[i], v + i);
        });
    } else {
        // the lanes that have one, then a thread for each token of theirs
        int *const lanes = reinterpret_cast<int *>(s.bins);
        if (even.place(lane_most) < limit) lanes[atomicAdd(&s.kept, 1)] = threadIdx.x;
        __syncthreads();
        const int waves = blockDim.x >> 6, each = (row.vocabulary + kTile * waves - 1) / (kTile * waves) * kEach, items = s.kept * each;
        for (int i = threadIdx.x; i < items; i += blockDim.x) {
            const int l = i / each, j = i - l * each, of = lanes[l], v = ((of >> 6) + j / kEach * waves) * kTile + (of & 63) * kEach + j % kEach;
            if (v < row.vocabulary) put(row.value(v < row.staged ? row.stage[v] : row.x[v]), v);
        }
    }
    __syncthreads();
    return s.count;
}

// Ranks the n listed tokens among each other.  *token, and the kept ones' *cut and the sum of their weights.
//
// The sum of the weights ahead of a token is that over all others: their number is divided among the waves, whose parts meet in LDS.
__device__ __forceinline__ void rank(Shared &s, const Weights &w, int n, int k, float p, float least, float u, int64_t *token, Cut *cut, uint64_t *all)
{
    const uint64_t *const orders = reinterpret_cast<const uint64_t *>(s.list); // (token, key): the key is the high half
    uint64_t *const weights = s.bins, *const aheads = s.bins + kRanked;
    int *const ranks = reinterpret_cast<int *>(s.bins + 2 * kRanked);
    const int i = threadIdx.x, columns = (n + 63) & ~63, parts = blockDim.x / columns, column = i % columns, part = i / columns; // parts of the others
    const bool mine = i < n, work = column < n && part < parts;
    uint64_t weight = 0;
    float x = 0;
    if (i < columns) {
        x = mine ? logit_of(s.list[i].y) : 0.0f;
        weight = mine ? w.fixed(x) : 0;
        weights[i] = weight, aheads[i] = 0, ranks[i] = 0;
    }
    if (threadIdx.x == 0) s.kept = 0;
    __syncthreads();
    // f(other's place) for the part
    const auto others = [&](const auto &f) {
        if (work)
            for (int j = part; j < n; j += parts) f(j);
    };
    uint64_t ahead = 0;
    int before = 0;
    const uint64_t order = orders[column < n ? column : 0];
    others([&](int j) {
        const bool first = orders[j] < order;
        before += first;
        ahead += first ? weights[j] : 0;
    });
    if (work) {
        atomicAdd(&ranks[column], before);
        atomicAdd((unsigned long long *)&aheads[column], (unsigned long long)ahead);
    }
    __syncthreads();
    if (mine) {
        before = ranks[i];
        ahead = aheads[i];
        if (before == (k < n ? k : n) - 1) s.amount = ahead + weight;
    }
    __syncthreads();
    const bool kept = mine && before < k && (!(p < 1) || ahead < share_of(p, s.amount)) && (before == 0 || x >= least);
    const uint64_t wave_kept = __ballot(kept);
    if ((threadIdx.x & 63) == 0 && wave_kept) atomicAdd(&s.kept, __builtin_popcountll(wave_kept));
    if (i < columns) weights[i] = kept ? weight : 0, aheads[i] = 0;
    __syncthreads();
    // the kept ones are the first in the order
    if (kept && before == s.kept - 1) s.low = s.list[i].y, s.high = s.list[i].x, s.all = ahead + weight;
    ahead = 0;
    others([&](int j) { ahead += (uint32_t)orders[j] < (uint32_t)order ? weights[j] : 0; });
    if (work) atomicAdd((unsigned long long *)&aheads[column], (unsigned long long)ahead);
    __syncthreads();
    if (kept) {
        const uint64_t wanted = wanted_of(u, s.all), from = aheads[i];
        if (from < wanted && wanted <= from + weight) *token = s.list[i].x;
    }
    *cut = Cut{logit_of(s.low), (int)s.high};
    *all = s.all;
}

// The least logit whose weight is `share` at least: 64 keys at a time (64 lanes call together)
__device__ float least_logit(const Weights &w, float most, double share)
{
    uint32_t low = key_of(most), high = 0xff7fffffu; // the greatest key that is still enough lies in low .. high; low is
    while (low < high) {
        const uint32_t step = (high - low) / 64 + 1, at = low + step * ((threadIdx.x & 63) + 1);
        const bool enough = at > low && at <= high && w.exact(logit_of(at)) >= share;
        const int n = __builtin_popcountll(__ballot(enough));
        const uint32_t next = low + step * n, end = next + (step - 1);
        high = end >= next && end < high ? end : high;
        low = next;
    }
    return logit_of(low);
}

// STAGE: bytes of LDS for the row
template <class T, class P, int STAGE> __global__ __launch_bounds__(64 * kWaves) void sample_kernel(const SampleArgs a)
{
    __shared__ Shared s;
    __shared__ __attribute__((aligned(16))) T stage[STAGE / sizeof(T)];
    const int lane = threadIdx.x & 63, wave = wave_of_block(), waves = blockDim.x >> 6, V = a.vocabulary, tiles = (V + kTile - 1) / kTile;
    constexpr int kStaged = STAGE / (int)sizeof(T) / kTile * kTile;
    const int64_t r = blockIdx.x;
    Row<T> row{static_cast<const T *>(a.logits) + r * a.stride, stage, tiles * kTile < kStaged ? tiles * kTile : kStaged, V, false};
    const float t = a.temperature ? a.temperature[r] : 1.0f, u = a.uniform[r], p = a.top_p ? a.top_p[r] : 1.0f, min_p = a.min_p ? a.min_p[r] : 0.0f;
    const int k = a.top_k ? a.top_k[r] : 0;

    float lane_most = -INFINITY;
#pragma unroll 4
    for (int tile = wave; tile < tiles; tile += waves) {
        const int v = tile * kTile + lane * kEach;
        const auto e = Eight<T>::load(row.x, v, V);
#pragma unroll
        for (int i = 0; i < kEach; ++i) lane_most = fmaxf(lane_most, (float)e[i]);
        if (v < row.staged) *reinterpret_cast<typename Eight<T>::values_t *>(stage + v) = e;
    }
    for (int i = threadIdx.x; i < kSteps; i += blockDim.x) s.table[i] = kPowers.x[i];
    float most = lane_most;
    for (int m = 1; m < 64; m <<= 1) most = fmaxf(most, __shfl_xor(most, m));
    if (lane == 0) s.wave_most[wave] = most;
    if (threadIdx.x == 0) s.place = 0x7fffffff;
    __syncthreads();
    most = (lane & 15) < waves ? s.wave_most[lane & 15] : -INFINITY;
    for (int m = 1; m < 16; m <<= 1) most = fmaxf(most, __shfl_xor(most, m));

    P *const kept = a.probabilities ? static_cast<P *>(a.probabilities) + r * V : nullptr;
    typedef typename Eight<P>::values_t out_t;
    const auto write = [&](const auto &probability) {
        if (!kept) return;
#pragma unroll 1
        for (int tile = wave; tile < tiles; tile += waves) {
            const int v = tile * kTile + lane * kEach;
            Eight<P>::store(kept, v, V, probability(tile, v));
        }
    };
    // Where few tokens can be kept all probabilities are 0 first, while the search goes on, and those of the kept ones follow at the end
    const bool few = !(t > 0) || most == -INFINITY || (k > 0 && k < V && k <= kMostListed && ((4 * k <= (int)blockDim.x && k <= kFew) || 32 * k <= V));
    // zeros in whole 16 bytes, adjacent lanes side by side
    const auto clear = [&] {
        if (!kept) return;
        constexpr int kWide = 16 / sizeof(P);
        const int ahead = (int)(-reinterpret_cast<uintptr_t>(kept) / sizeof(P) & (kWide - 1)), head = ahead < V ? ahead : V, wide = (V - head) / kWide, tail = head + wide * kWide;
        if ((int)threadIdx.x < head) kept[threadIdx.x] = (P)0.0f;
        if ((int)threadIdx.x < V - tail) kept[tail + threadIdx.x] = (P)0.0f;
        for (int i = threadIdx.x; i < wide; i += blockDim.x) reinterpret_cast<uint4_t *>(kept + head)[i] = uint4_t{0, 0, 0, 0};
    };
    if (few) clear();
    if (threadIdx.x == 0) s.zeroed = few;
    const auto zeros_are_there = [&] {
        if (!kept) return;
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();
    };
    if (!(t > 0) || most == -INFINITY) { // the first token alone, or none
        if (most != -INFINITY && lane_most == most) {
            row.tiles([&](const float(&e)[kEach], int v) {
#pragma unroll
                for (int i = 0; i < kEach; ++i)
                    if (e[i] == most) atomicMin(&s.place, v + i);
            });
        }
        __syncthreads();
        const int first = most == -INFINITY ? -1 : s.place;
        if (threadIdx.x == 0) a.tokens[r] = first;
        zeros_are_there();
        if (kept && threadIdx.x == 0 && first >= 0) kept[first] = (P)1.0f;
        return;
    }
    if (most == INFINITY) {
        row.infinite = true;
        lane_most = lane_most == INFINITY ? 0.0f : -INFINITY;
        most = 0;
    }
    Weights w;
    w.most = most;
    w.rate = kSteps * kLog2e / (double)t;
    w.table = s.table;
    w.unit = a.unit;
    // From a rate on the next logit below the greatest weighs 2^-512, nothing by any measure: a greater one would only take exponents out of their range
    const double next = (double)most - (double)logit_of(key_of(most) + 1);
    if (w.rate * next > 0x1p18 && next < (double)FLT_MAX) w.rate = 0x1p18 / next;
    const double octave = kSteps / w.rate; // in logits
    const double floor = (double)most - (a.unit + 4) * octave;
    w.floor = floor >= -(double)FLT_MAX ? (float)floor : -FLT_MAX;
    if ((double)w.floor > floor) w.floor = w.floor > -FLT_MAX ? logit_of(key_of(w.floor) + 1) : -FLT_MAX;
    const double far = (double)most - 161 * octave;
    w.far = far >= -(double)FLT_MAX ? (float)far : -FLT_MAX;
    if ((double)w.far > far) w.far = w.far > -FLT_MAX ? logit_of(key_of(w.far) + 1) : -FLT_MAX;
    const Even even{most, fmaxf(fminf((float)(w.rate * ((double)kBinsPerOctave / kSteps)), 1e30f), 1e-30f)};
    const float least = min_p > 0 ? least_logit(w, most, min_p < 1 ? (double)min_p : 1.0) : -INFINITY;

    Cut cut{-INFINITY, -1};
    uint64_t all = 0; // weights kept
    int listed = -1;
    if (k > 0 && k < V && k <= kMostListed) {
        if (4 * k <= (int)blockDim.x && k <= kFew) {
            listed = candidates(s, row, even, lane_most, k, false);
            if (listed > kRanked || listed > (int)blockDim.x) listed = -1;
        }
        if (listed < 0 && 32 * k <= V) {
            __syncthreads();
            listed = candidates(s, row, even, lane_most, k, true);
            if (listed > kList) listed = -1;
        }
    }
    __syncthreads();
    const auto cuts = [&](const auto &source) {
#pragma unroll 1
        for (int weigh = 0; weigh < 2; ++weigh)
            if (weigh ? p < 1 : k > 0 && k < V) cut = select(s, source, w, cut, even, weigh, k, p);
        if (least > cut.x) cut = Cut{least, 0x7fffffff};
        __syncthreads();
    };
    // The kept logits of a tile one behind the other, in the list's memory: weights are evaluated for these alone.  at: the lane's places, -1 for others; returns their
    // number, of which kGathered are there.
    constexpr int kGathered = kList * sizeof(uint2) / sizeof(float) / kWaves;
    float *const gathered = reinterpret_cast<float *>(s.list) + wave * kGathered;
    const auto gather = [&](const float(&e)[kEach], int v, int (&at)[kEach]) {
        bool keep[kEach];
        cut.keeps(e, v, keep);
        int n = 0;
#pragma unroll
        for (int j = 0; j < kEach; ++j) {
            const uint64_t lanes = __ballot(keep[j]);
            const int mine = n + (int)__builtin_amdgcn_mbcnt_hi((uint32_t)(lanes >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)lanes, 0));
            if (keep[j] && mine < kGathered) gathered[mine] = e[j];
            at[j] = keep[j] ? mine : -1;
            n += __builtin_popcountll(lanes);
        }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); // other lanes of the wave read them
        return n;
    };
    const bool sorted = listed >= 0 && listed <= kRanked && listed <= (int)blockDim.x;
    if (sorted) {
        rank(s, w, listed, k, p, least, u, a.tokens + r, &cut, &all);
    } else if (listed >= 0) {
        cuts(List{s.list, listed, V});
    } else {
        cuts(row);
        // The kept tokens are listed where they are few, until a tile has many: the passes that are left evaluate no others then
        if (cut.x > -INFINITY) {
            if (threadIdx.x == 0) s.count = 0;
            __syncthreads();
            for (int tile = wave; tile < tiles && s.count <= kList; tile += waves) {
                float e[kEach];
                const int v = row.tile(tile, e);
                bool keep[kEach];
                cut.keeps(e, v, keep);
                uint64_t lanes[kEach];
                int total = 0;
#pragma unroll
                for (int j = 0; j < kEach; ++j) {
                    lanes[j] = __ballot(keep[j]);
                    total += __builtin_popcountll(lanes[j]);
                }
                if (total == 0) continue;
                int at = 0;
                if (lane == 0) at = atomicAdd(&s.count, total > kTile / 16 ? kList + 1 : total);
                at = __builtin_amdgcn_readfirstlane(at);
#pragma unroll
                for (int j = 0; j < kEach; ++j) {
                    const int mine = at + (int)__builtin_amdgcn_mbcnt_hi((uint32_t)(lanes[j] >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)lanes[j], 0));
                    if (keep[j] && mine < kList) s.list[mine] = make_uint2(v + j, key_of(e[j]));
                    at += __builtin_popcountll(lanes[j]);
                }
            }
            __syncthreads();
            if (s.count <= kList) listed = s.count;
            __syncthreads();
            if (listed >= 0 && !s.zeroed) clear();
        }
    }
    if (sorted) {
    } else if (listed >= 0) {
        const List list{s.list, listed, V};
        clear_bins(s);
        list.tiles([&](const auto &e, int v) {
            if (cut.keeps(e[0], v)) add(s, v / kTile, w.fixed(e[0]));
        });
        if (threadIdx.x == 0) s.count = 0;
        __syncthreads();
        find(s, tiles, [&](uint64_t sum) { return wanted_of(u, sum); });
        const int tile = s.place;
        const uint64_t wanted = s.wanted - s.before;
        all = s.all;
        // the kept tokens of the tile, each with the sum of those before it
        uint64_t *const weights = s.bins, *const numbers = s.bins + kTile;
        list.tiles([&](const auto &e, int v) {
            if (v / kTile != tile || !cut.keeps(e[0], v)) return;
            const int at = atomicAdd(&s.count, 1);
            weights[at] = w.fixed(e[0]), numbers[at] = v;
        });
        __syncthreads();
        for (int i = threadIdx.x; i < s.count; i += blockDim.x) {
            uint64_t before = 0;
            for (int j = 0; j < s.count; ++j) before += numbers[j] < numbers[i] ? weights[j] : 0;
            if (before < wanted && wanted <= before + weights[i]) a.tokens[r] = numbers[i];
        }
    } else {
        // Sums of groups of up to 4 tiles, a wave each; then a wave for each tile of the group that the random number meets
        const int group = tiles >= 4 * waves ? 4 : tiles >= 2 * waves ? 2 : 1, groups = (tiles + group - 1) / group;
        // a logit that is not kept is taken as one that weighs nothing
        const auto weigh = [&](const float(&e)[kEach], int v, uint64_t (&x)[kEach]) {
            bool keep[kEach];
            cut.keeps(e, v, keep);
#pragma unroll
            for (int j = 0; j < kEach; ++j) x[j] = w.fixed_up(keep[j] && e[j] >= w.floor ? e[j] : w.floor);
            if (w.floor == -FLT_MAX) { // at the greatest temperatures every logit weighs something
#pragma unroll
                for (int j = 0; j < kEach; ++j) x[j] = keep[j] ? x[j] : kFixedBase;
            }
        };
        for (int i = wave; i < groups; i += waves) {
            uint64_t sum = 0;
#pragma unroll 1
            for (int t = 0; t < group; ++t) {
                float e[kEach];
                uint64_t x[kEach];
                const int v = row.tile(i * group + t, e);
                if (cut.x > -INFINITY) {
                    int at[kEach];
                    const int n = gather(e, v, at);
                    if (n <= kGathered) {
                        for (int q = lane; q < n; q += 64) sum += w.fixed(gathered[q]);
                        continue;
                    }
                }
                weigh(e, v, x);
#pragma unroll
                for (int j = 0; j < kEach; ++j) sum += x[j];
                sum -= kEach * kFixedBase;
            }
            sum = wave_scan(sum);
            if (lane == 63) s.bins[i] = sum;
        }
        __syncthreads();
        find(s, groups, [&](uint64_t sum) { return wanted_of(u, sum); });
        all = s.all;
        const uint64_t wanted = s.wanted;
        uint64_t x[kEach], sum = 0, upto = 0;
        int v = 0;
        if (wave < group) {
            float e[kEach];
            v = row.tile(__builtin_amdgcn_readfirstlane(s.place) * group + wave, e);
            weigh(e, v, x);
#pragma unroll
            for (int j = 0; j < kEach; ++j) sum += x[j] -= kFixedBase;
            upto = wave_scan(sum);
            if (lane == 63) s.wave_sum[wave] = upto;
        }
        __syncthreads();
        if (wave < group) {
            uint64_t before = s.before + upto - sum;
#pragma unroll
            for (int i = 0; i < 4; ++i) before += i < wave ? s.wave_sum[i] : 0;
            if (before < wanted && wanted <= before + sum) {
#pragma unroll
                for (int j = 0; j < kEach; ++j) {
                    if (before < wanted && wanted <= before + x[j]) a.tokens[r] = v + j;
                    before += x[j];
                }
            }
        }
    }
    const double share = __builtin_ldexp(1.0, a.unit) / (double)all;
    if (listed >= 0 || s.zeroed) zeros_are_there();
    if (listed >= 0) {
        if (kept) {
            for (int i = threadIdx.x; i < listed; i += blockDim.x) {
                const float x = logit_of(s.list[i].y);
                const int v = (int)s.list[i].x;
                if (cut.keeps(x, v)) kept[v] = (P)(float)(w.exact(x) * share);
            }
        }
        return;
    }
    write([&](int tile, int) {
        float e[kEach];
        const int v = row.tile(tile, e);
        out_t y;
        if (cut.x > -INFINITY) {
            int at[kEach];
            const int n = gather(e, v, at);
            if (n <= kGathered) {
                for (int q = lane; q < n; q += 64) gathered[q] = (float)(w.exact(gathered[q]) * share);
                asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
#pragma unroll
                for (int i = 0; i < kEach; ++i) {
                    const float x = gathered[at[i] < 0 ? 0 : at[i]];
                    y[i] = (P)(at[i] < 0 ? 0.0f : x);
                }
                asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
                return y;
            }
        }
        bool keep[kEach], some = false;
        cut.keeps(e, v, keep);
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            y[i] = (P)0.0f;
            some = some || keep[i];
        }
        if (some) {
#pragma unroll
            for (int i = 0; i < kEach; ++i) {
                const float x = (float)(w.exact(e[i]) * share);
                y[i] = (P)(keep[i] ? x : 0.0f);
            }
        }
        return y;
    });
}

template <class T, class P> void launch(const SampleArgs &k, hipStream_t stream)
{
    // Of more rows than CUs two workgroups share one: 8 waves and 43 KB of the row each, instead of 16 and 120 KB.  us with one / two, 300 x 32003 binary32: greedy
    // 12.2 / 10.1, top-k 50 21.1 / 16.1, temperature alone 34.9 / 27.9, top-p 0.9 60.8 / 55.4
    const int tiles = (k.vocabulary + kTile - 1) / kTile, most = k.rows > 256 ? kWaves / 2 : kWaves, threads = 64 * (tiles < most ? tiles : most);
    const dim3 grid((unsigned)k.rows);
    if (k.rows > 256 || tiles * kTile * sizeof(T) <= 43 << 10) sample_kernel<T, P, 43 << 10><<<grid, threads, 0, stream>>>(k);
    else sample_kernel<T, P, 120 << 10><<<grid, threads, 0, stream>>>(k);
}

} // namespace

hipError_t launch_sample(const ap_sampling &a, hipStream_t stream)
{
    SampleArgs k;
    k.logits = a.logits;
    k.stride = a.stride, k.rows = a.rows;
    k.uniform = a.uniform, k.temperature = a.temperature, k.top_p = a.top_p, k.min_p = a.min_p, k.top_k = a.top_k;
    k.tokens = a.tokens, k.probabilities = a.probabilities;
    k.vocabulary = (int)a.vocabulary;
    int bits = 0;
    while ((int64_t)1 << bits < a.vocabulary) ++bits;
    k.unit = 62 - bits < 51 ? 62 - bits : 51;
    if (a.half) {
        if (a.half_probabilities) launch<_Float16, _Float16>(k, stream);
        else launch<_Float16, float>(k, stream);
    } else {
        if (a.half_probabilities) launch<float, _Float16>(k, stream);
        else launch<float, float>(k, stream);
    }
    return hipGetLastError();
}

} // namespace apgemv
