// Tokens from logits: temperature, top-k, top-p, min-p and a draw by one random number per row.
//
// The order of the tokens is never written out: what is kept ends at a logit and, among tokens with that logit, at a token number, and both are
// found by histograms of counts or weights that narrow an interval 2048-fold.  Weights are computed in binary64 and rounded to 64-bit fixed point: integer sums
// are the same in any order, so atomics on LDS leave no trace, and borders lie where exact sums put them (off by 2^-42 of the greatest
// weight per token), not where a rounding of a long binary32 sum would.
//
// A workgroup has a row, whose first tokens it keeps in LDS.
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
constexpr int kTile = 64 * kEach; // tokens of a wave and step: up to 2^20 / kTile sums of tiles take the histogram's place
constexpr int kBins = 2048;
constexpr int kList = 1024;       // tokens of one bin that are listed
constexpr int kFew = 128;         // top-k up to which the tokens are ranked among each other,
constexpr int kRanked = 256;      // so many at most
constexpr int kWaves = 16;        // of a workgroup, at most
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

// 2^(j / 64), by the power series of exp
constexpr int kSteps = 64;
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

// What the tokens of a row weigh: 2^(d / 64) with d = 64 log2 e (x - most) / temperature <= 0, as 2^n times a table's 2^(j / 64) times the power series of exp on
// half a step either way, off by 4e-14.  Adding 1.5 2^52 leaves the whole part of d in the low bits of the sum.
struct Weights {
    double most, rate;
    const double *table; // LDS
    int unit;
    // 2^scale times the weight, d not below `least`
    __device__ double of(float x, int scale, double least) const
    {
        const double magic = 0x1.8p52 + 64.0 * scale, d = fmax(((double)x - most) * rate, least), t = d + magic, f = d - (t - magic);
        const int k = (int)(uint32_t)__double_as_longlong(t);
        constexpr double c = kLn2 / 64;
        double p = __builtin_fma(c * c * c * c / 24, f, c * c * c / 6);
        p = __builtin_fma(p, f, c * c / 2);
        p = __builtin_fma(p, f, c);
        p = __builtin_fma(p, f, 1.0);
        return __longlong_as_double(__double_as_longlong(table[k & 63] * p) + ((long long)(k >> 6) << 52));
    }
    // In fixed point: a number below 2^52 added to 2^52 has its integer part in the low bits.  2^-3 and less are 0, as is the weight of -inf.
    __device__ uint64_t fixed(float x) const { return (uint64_t)__double_as_longlong(of(x, unit, -64.0 * (unit + 3)) + 0x1p52) & 0xfffffffffffffull; }
    __device__ double exact(float x) const { return of(x, 0, -64.0 * 1000); }
};

// The beginning of the order that is kept: logits above x, and of those equal to it the tokens up to `last`
struct Cut {
    float x;
    int last;
    __device__ bool keeps(float y, int v) const { return y > x || (y == x && v <= last); }
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

// A row of logits.  Its first `staged` tokens (a multiple of kTile) are in LDS, -inf behind the last one; the others are read again in every pass.
template <class T> struct Row {
    const T *x;
    const T *stage;
    int staged, vocabulary;
    bool infinite; // +inf is the greatest: such logits are 0, all others -inf

    __device__ float value(T t) const
    {
        const float x = fmaxf((float)t, -INFINITY); // NaN counts as -inf
        if (infinite) return x == INFINITY ? 0.0f : -INFINITY;
        return x;
    }
    __device__ typename Eight<T>::values_t raw(int v) const
    {
        return v < staged ? *reinterpret_cast<const typename Eight<T>::values_t *>(stage + v) : Eight<T>::load(x, v, vocabulary);
    }
    // the lane's logits of tile t; returns the first one's token
    __device__ int tile(int t, float (&out)[kEach]) const
    {
        const int v = t * kTile + (threadIdx.x & 63) * kEach;
        const auto e = raw(v);
#pragma unroll
        for (int i = 0; i < kEach; ++i) out[i] = value(e[i]);
        return v;
    }
    // f(first token, logits) for the wave's tiles
    template <class F> __device__ void tiles(const F &f) const
    {
        const int waves = blockDim.x >> 6;
        for (int t = threadIdx.x >> 6; t * kTile < vocabulary; t += waves) {
            float e[kEach];
            const int v = tile(t, e);
            f(v, e);
        }
    }
    // f(logit, token), in little code for what is seldom run
    template <class F> __device__ void each(const F &f) const
    {
#pragma unroll 1
        for (int v = threadIdx.x; v < vocabulary; v += blockDim.x) f(value(v < staged ? stage[v] : x[v]), v);
    }
};

struct Shared {
    uint64_t bins[kBins];        // or the sums of tiles
    uint2 list[kList];           // (token, key)
    uint64_t wave_sum[kWaves];
    double table[kSteps];
    uint64_t before, amount;
    float wave_most[kWaves];
    uint32_t low, high;
    int count, place, kept;
};

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

// The first of `count` numbers in LDS at which the sum up to it reaches the target that target(sum of all) gives: s.place, s.before (the sum
// before it) and s.amount (it).  count <= kBins.  A target is 1 at least; one beyond the sum leaves s.place at -1.
template <class F> __device__ uint64_t find(Shared &s, int count, const F &target)
{
    const int wave = threadIdx.x >> 6, waves = blockDim.x >> 6, lane = threadIdx.x & 63;
    const int per = blockDim.x == 1024 ? kBins / 1024 : (count + blockDim.x - 1) / blockDim.x, first = threadIdx.x * per;
    uint64_t mine = 0;
    for (int i = 0; i < per; ++i)
        if (first + i < count) mine += s.bins[first + i];
    const uint64_t upto = wave_scan(mine);
    if (lane == 63) s.wave_sum[wave] = upto;
    if (threadIdx.x == 0) s.place = -1;
    __syncthreads();
    const uint64_t sums = row_scan((lane & 15) < waves ? s.wave_sum[lane & 15] : 0), all = lane_of(sums, 15);
    uint64_t before = upto - mine + (wave > 0 ? lane_of(sums, wave - 1) : 0);
    const uint64_t wanted = target(all);
    if (before < wanted && wanted <= before + mine) {
        for (int i = 0; i < per; ++i) {
            const uint64_t x = s.bins[first + i];
            if (wanted <= before + x) {
                s.place = first + i;
                s.before = before;
                s.amount = x;
                break;
            }
            before += x;
        }
    }
    __syncthreads();
    return all;
}

__device__ __forceinline__ void clear_bins(Shared &s)
{
    for (int i = threadIdx.x; i < kBins / 2; i += blockDim.x) reinterpret_cast<uint4_t *>(s.bins)[i] = uint4_t{0, 0, 0, 0};
    __syncthreads();
}
__device__ __forceinline__ void add(Shared &s, int bin, uint64_t x) { atomicAdd((unsigned long long *)&s.bins[bin], (unsigned long long)x); }

// The place of a logit among the first bins, which are even in it, 64 to a factor of two in the weight: tokens spread over many, and few are in the one
// that matters.  The last bin holds all the rest.
struct Even {
    float most, rate;
    __device__ float place(float x) const { return (most - x) * rate; }
    __device__ int bin(float x) const { return (int)fminf(place(x), (float)(kBins - 1)); }
};

// Where the tokens that `cut` keeps, in order, reach `count` (weigh = false), or their weights the share p of their sum.
//
// The tokens of the even bin that reaches it are listed.  Their interval of keys is divided into bins until one key is left; where it has more tokens than
// are wanted, an interval of token numbers is, for the first ones.  A bin that holds more than the list is looked for in the row.
template <class T> __device__ Cut select(Shared &s, const Row<T> &row, const Weights &w, const Cut cut, const Even even, bool weigh, int count, float p)
{
    clear_bins(s);
    row.tiles([&](int v, const float(&e)[kEach]) {
        uint64_t x[kEach];
#pragma unroll
        for (int i = 0; i < kEach; ++i) x[i] = 1;
        if (weigh) {
#pragma unroll
            for (int i = 0; i < kEach; ++i) x[i] = w.fixed(e[i]);
        }
#pragma unroll
        for (int i = 0; i < kEach; ++i)
            if (cut.keeps(e[i], v + i)) add(s, even.bin(e[i]), x[i]);
    });
    if (threadIdx.x == 0) s.count = 0, s.low = 0xffffffffu, s.high = 0;
    __syncthreads();
    uint64_t wanted = 0;
    find(s, kBins, [&](uint64_t all) { return wanted = weigh ? share_of(p, all) : (uint64_t)count; });
    const int bin = s.place;
    if (bin < 0) return cut; // fewer tokens than wanted
    wanted -= s.before;
    uint64_t amount = s.amount;
    const float from = bin, to = bin == kBins - 1 ? __builtin_nanf("") : (float)(bin + 1); // not at or beyond NaN: everything
    const auto inside = [&](float x, int v) {
        const float at = even.place(x);
        return at >= from && !(at >= to) && cut.keeps(x, v);
    };
    row.tiles([&](int v, const float(&e)[kEach]) {
#pragma unroll
        for (int i = 0; i < kEach; ++i)
            if (inside(e[i], v + i)) {
                const uint32_t key = key_of(e[i]);
                const int at = atomicAdd(&s.count, 1);
                if (at < kList) s.list[at] = make_uint2(v + i, key);
                atomicMin(&s.low, key);
                atomicMax(&s.high, key);
            }
    });
    __syncthreads();
    const int listed = s.count;
    uint32_t low = s.low, high = s.high, key = 0;
    bool numbers = false; // of the tokens with `key`
    for (;;) {
        if (low == high) {
            if (numbers) return Cut{logit_of(key), (int)low};
            key = low;
            const float x = logit_of(key);
            const uint64_t one = weigh ? w.fixed(x) : 1;
            wanted = (wanted + one - 1) / one;
            if (wanted >= amount / one) return Cut{x, x == cut.x ? cut.last : 0x7fffffff};
            numbers = true;
            low = 0, high = row.vocabulary - 1;
        }
        const int bits = 32 - __builtin_clz(high - low), shift = bits > 11 ? bits - 11 : 0;
        clear_bins(s);
        const auto consider = [&](int v, uint32_t k) {
            const uint32_t number = numbers ? (uint32_t)v : k;
            if (number >= low && number <= high && (!numbers || k == key)) add(s, (number - low) >> shift, weigh && !numbers ? w.fixed(logit_of(k)) : 1);
        };
        if (listed <= kList) {
            for (int i = threadIdx.x; i < listed; i += blockDim.x) consider((int)s.list[i].x, s.list[i].y);
        } else {
            row.each([&](float x, int v) {
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
}

// Few tokens that a row keeps at most, ranked among each other.  The k-th best of the lanes' own best tokens leaves k tokens before it at least, and few more
// where k is small beside the lanes: those are listed, a thread each.  False where that does not hold; the kept ones' *cut and the sum of their weights otherwise.
template <class T> __device__ bool few(Shared &s, const Row<T> &row, const Weights &w, const Even even, float lane_most, int k, float p, float least, float u, int64_t *token, Cut *cut, uint64_t *all)
{
    clear_bins(s);
    if (lane_most != -INFINITY) add(s, even.bin(lane_most), 1);
    if (threadIdx.x == 0) s.count = 0, s.kept = 0;
    __syncthreads();
    find(s, kBins, [&](uint64_t) { return (uint64_t)k; });
    const int bin = s.place;
    if (bin < 0 || bin == kBins - 1) return false;
    const float limit = bin + 1;
    row.tiles([&](int v, const float(&e)[kEach]) {
        float top = e[0];
#pragma unroll
        for (int i = 1; i < kEach; ++i) top = fmaxf(top, e[i]);
        if (!(even.place(top) < limit)) return;
#pragma unroll
        for (int i = 0; i < kEach; ++i)
            if (even.place(e[i]) < limit) {
                const int at = atomicAdd(&s.count, 1);
                if (at < kRanked) s.list[at] = make_uint2(v + i, key_of(e[i]));
            }
    });
    __syncthreads();
    const int n = s.count, i = threadIdx.x;
    if (n > kRanked || n > (int)blockDim.x) {
        __syncthreads();
        return false;
    }
    // Loops over the n tokens take eight at a time, all waves that have one together; behind the last one are tokens that come after all and weigh nothing.
    constexpr int kStep = 8;
    uint64_t *const orders = reinterpret_cast<uint64_t *>(s.list), *const weights = s.bins;
    const bool mine = i < n;
    const uint2 me = mine ? s.list[i] : make_uint2(0xffffffffu, 0xffffffffu);
    const uint64_t order = (uint64_t)me.y << 32 | me.x;
    const uint64_t weight = mine ? w.fixed(logit_of(me.y)) : 0;
    for (int j = i; j < n + kStep; j += blockDim.x) weights[j] = j == i ? weight : 0;
    if (i < kStep) s.list[n + i] = make_uint2(0xffffffffu, 0xffffffffu);
    __syncthreads();
    int rank = 0;
    uint64_t before = 0;
    if (i < (n + 63 & ~63))
        for (int j = 0; j < n; j += kStep)
#pragma unroll
            for (int l = 0; l < kStep; ++l) {
                const uint64_t other = orders[j + l], x = weights[j + l]; // (token, key): the key is the high half
                const bool ahead = other < order;
                rank += ahead;
                before += ahead ? x : 0;
            }
    if (mine && rank == (k < n ? k : n) - 1) s.amount = before + weight;
    __syncthreads();
    const bool kept = mine && rank < k && (!(p < 1) || before < share_of(p, s.amount)) && (rank == 0 || logit_of(me.y) >= least);
    const uint64_t wave_kept = __ballot(kept);
    if ((threadIdx.x & 63) == 0 && wave_kept) atomicAdd(&s.kept, __builtin_popcountll(wave_kept));
    if (mine) weights[i] = kept ? weight : 0;
    __syncthreads();
    if (kept && rank == s.kept - 1) s.low = me.y, s.high = me.x; // the kept ones are the first in the order
    uint64_t sum = 0;
    before = 0;
    if (i < (n + 63 & ~63))
        for (int j = 0; j < n; j += kStep)
#pragma unroll
            for (int l = 0; l < kStep; ++l) {
                const uint64_t x = weights[j + l];
                sum += x;
                before += (uint32_t)orders[j + l] < me.x ? x : 0;
            }
    const uint64_t wanted = wanted_of(u, sum);
    if (kept && before < wanted && wanted <= before + weight) *token = (int)me.x;
    if (i == 0) s.before = sum;
    __syncthreads();
    *cut = Cut{logit_of(s.low), (int)s.high};
    *all = s.before;
    return true;
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
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = blockDim.x >> 6, V = a.vocabulary, tiles = (V + kTile - 1) / kTile;
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
    if (threadIdx.x < kSteps) s.table[lane] = kPowers.x[lane];
    float most = lane_most;
    for (int m = 1; m < 64; m <<= 1) most = fmaxf(most, __shfl_xor(most, m));
    if (lane == 0) s.wave_most[wave] = most;
    if (threadIdx.x == 0) s.place = 0x7fffffff;
    __syncthreads();
    most = (lane & 15) < waves ? s.wave_most[lane & 15] : -INFINITY;
    for (int m = 1; m < 16; m <<= 1) most = fmaxf(most, __shfl_xor(most, m));

    P *const kept = a.probabilities ? static_cast<P *>(a.probabilities) + r * V : nullptr;
    const auto write = [&](const auto &probability) {
        if (!kept) return;
#pragma unroll 1
        for (int tile = wave; tile < tiles; tile += waves) {
            const int v = tile * kTile + lane * kEach;
            Eight<P>::store(kept, v, V, probability(tile, v));
        }
    };
    typedef typename Eight<P>::values_t out_t;
    if (!(t > 0) || most == -INFINITY) { // the first token alone, or none
        if (most != -INFINITY && lane_most == most) {
            row.tiles([&](int v, const float(&e)[kEach]) {
#pragma unroll
                for (int i = 0; i < kEach; ++i)
                    if (e[i] == most) atomicMin(&s.place, v + i);
            });
        }
        __syncthreads();
        const int first = most == -INFINITY ? -1 : s.place;
        if (threadIdx.x == 0) a.tokens[r] = first;
        write([&](int, int v) {
            out_t y;
#pragma unroll
            for (int i = 0; i < kEach; ++i) y[i] = (P)(v + i == first ? 1.0f : 0.0f);
            return y;
        });
        return;
    }
    if (most == INFINITY) {
        row.infinite = true;
        lane_most = lane_most == INFINITY ? 0.0f : -INFINITY;
        most = 0;
    }
    Weights w;
    w.most = most;
    w.rate = 64 * kLog2e / (double)t;
    w.table = s.table;
    w.unit = a.unit;
    const Even even{most, fmaxf(fminf((float)w.rate, 1e30f), 1e-30f)};
    const float least = min_p > 0 ? least_logit(w, most, min_p < 1 ? (double)min_p : 1.0) : -INFINITY;

    Cut cut{-INFINITY, -1};
    uint64_t all = 0; // weights kept
    if (!(k > 0 && k < V && k <= kFew && few(s, row, w, even, lane_most, k, p, least, u, a.tokens + r, &cut, &all))) {
#pragma unroll 1
        for (int weigh = 0; weigh < 2; ++weigh)
            if (weigh ? p < 1 : k > 0 && k < V) cut = select(s, row, w, cut, even, weigh, k, p);
        if (least > cut.x) cut = Cut{least, 0x7fffffff};
        __syncthreads();
        for (int i = wave; i < tiles; i += waves) {
            float e[kEach];
            const int v = row.tile(i, e);
            uint64_t sum = 0;
#pragma unroll
            for (int j = 0; j < kEach; ++j) {
                const uint64_t x = w.fixed(e[j]);
                sum += cut.keeps(e[j], v + j) ? x : 0;
            }
            sum = wave_scan(sum);
            if (lane == 63) s.bins[i] = sum;
        }
        __syncthreads();
        uint64_t wanted = 0;
        all = find(s, tiles, [&](uint64_t sum) { return wanted = wanted_of(u, sum); });
        if (wave == 0) {
            float e[kEach];
            const int v = row.tile(s.place, e);
            uint64_t x[kEach], sum = 0;
#pragma unroll
            for (int j = 0; j < kEach; ++j) {
                x[j] = w.fixed(e[j]);
                x[j] = cut.keeps(e[j], v + j) ? x[j] : 0;
                sum += x[j];
            }
            uint64_t before = s.before + wave_scan(sum) - sum;
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
    write([&](int tile, int) {
        float e[kEach];
        const int v = row.tile(tile, e);
        out_t y;
        bool some = false;
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            y[i] = (P)0.0f;
            some = some || cut.keeps(e[i], v + i);
        }
        if (some) {
#pragma unroll
            for (int i = 0; i < kEach; ++i) {
                const float x = (float)(w.exact(e[i]) * share);
                y[i] = (P)(cut.keeps(e[i], v + i) ? x : 0.0f);
            }
        }
        return y;
    });
}

template <class T, class P> void launch(const SampleArgs &k, hipStream_t stream)
{
    const int tiles = (k.vocabulary + kTile - 1) / kTile, threads = 64 * (tiles < kWaves ? tiles : kWaves);
    const dim3 grid((unsigned)k.rows);
    if (k.rows > 256 || tiles * kTile * sizeof(T) <= 52 << 10) sample_kernel<T, P, 52 << 10><<<grid, threads, 0, stream>>>(k);
    else sample_kernel<T, P, 128 << 10><<<grid, threads, 0, stream>>>(k);
}

} // namespace

size_t sample_work(const ap_sampling &) { return 0; }

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
