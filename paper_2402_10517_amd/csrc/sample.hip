// Tokens from logits: temperature, top-k, top-p, min-p and a draw by one random number per row.
//
// The order of the tokens is never written out: what is kept ends at a key (the logit's bits) and, among equal logits, at a number of tokens, and both are
// found by histograms of counts or weights that narrow an interval of keys 2048-fold.  Weights are exp2 in binary64, each rounded to 64-bit fixed point:
// integer sums are the same in any order, so atomics on LDS leave no trace, and borders lie where exact sums put them (off by 2^-42 of the greatest
// weight per token), not where a rounding of a long binary32 sum would.
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

constexpr int kEach = 8;          // adjacent tokens of a lane
constexpr int kTile = 64 * kEach; // tokens of a wave and step: up to 2^20 / kTile sums of tiles take the histogram's place
constexpr int kBins = 2048;
constexpr int kList = 2048;       // tokens of one bin that are listed
constexpr double kLog2e = 1.4426950408889634;

template <class T> struct __attribute__((packed, aligned(sizeof(T)))) Eight {
    T x[kEach];
};

// Greater logits have smaller keys; -0 and 0 the same one
__device__ __forceinline__ uint32_t key_of(float x)
{
    const uint32_t b = __float_as_uint(x + 0.0f);
    return b >> 31 ? b : ~(b | 0x80000000u);
}
__device__ __forceinline__ float logit_of(uint32_t key) { return __uint_as_float(key >> 31 ? key : ~key & 0x7fffffffu); }

// 2^x for x <= 0: the power series of exp on half an octave either way, off by 1e-14
__device__ __forceinline__ double exp2_of(double x)
{
    x = fmax(x, -1000.0);
    const double n = __builtin_rint(x), r = (x - n) * 0.6931471805599453;
    double p = 1.0 / 39916800;
    p = __builtin_fma(p, r, 1.0 / 3628800);
    p = __builtin_fma(p, r, 1.0 / 362880);
    p = __builtin_fma(p, r, 1.0 / 40320);
    p = __builtin_fma(p, r, 1.0 / 5040);
    p = __builtin_fma(p, r, 1.0 / 720);
    p = __builtin_fma(p, r, 1.0 / 120);
    p = __builtin_fma(p, r, 1.0 / 24);
    p = __builtin_fma(p, r, 1.0 / 6);
    p = __builtin_fma(p, r, 0.5);
    p = __builtin_fma(p, r, 1.0);
    p = __builtin_fma(p, r, 1.0);
    return __builtin_ldexp(p, (int)n);
}

// What the tokens of a row weigh
struct Weights {
    double most, rate; // greatest logit; log2 e / temperature
    double least;      // of the weights that count
    int unit;
    __device__ double of(float x) const { return exp2_of(((double)x - most) * rate); }
    // in fixed point: a number below 2^52 added to 2^52 has its integer part in the low bits
    __device__ uint64_t fixed(double w) const { return (uint64_t)(__double_as_longlong(__builtin_ldexp(w, unit) + 0x1p52) & 0xfffffffffffffll); }
};

// The beginning of the order that is kept: keys before `key`, and of those with it the tokens up to `last`
struct Cut {
    uint32_t key;
    int last;
    __device__ bool keeps(uint32_t k, int v) const { return k < key || (k == key && v <= last); }
};

template <class T> struct Row {
    const T *x;
    int vocabulary;
    bool infinite; // +inf is the greatest: such logits are 0, all others -inf

    __device__ float value(float x) const
    {
        x = fmaxf(x, -INFINITY); // NaN counts as -inf
        return infinite ? x == INFINITY ? 0.0f : -INFINITY : x;
    }
    // the 8 logits of a lane from token v on; -inf where there are none
    __device__ void load(int v, float (&out)[kEach]) const
    {
        if (v + kEach <= vocabulary) {
            const Eight<T> e = *reinterpret_cast<const Eight<T> *>(x + v);
#pragma unroll
            for (int i = 0; i < kEach; ++i) out[i] = value((float)e.x[i]);
        } else {
#pragma unroll
            for (int i = 0; i < kEach; ++i) out[i] = v + i < vocabulary ? value((float)x[v + i]) : -INFINITY;
        }
    }
    // f(tile, first token of the lane, its logits) for the wave's tiles
    template <class F> __device__ void tiles(const F &f) const
    {
        const int waves = blockDim.x >> 6, wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
        for (int tile = wave; tile * kTile < vocabulary; tile += waves) {
            float e[kEach];
            const int v = tile * kTile + lane * kEach;
            load(v, e);
            f(tile, v, e);
        }
    }
    template <class F> __device__ void each(const F &f) const
    {
        tiles([&](int, int v, const float(&e)[kEach]) {
#pragma unroll
            for (int i = 0; i < kEach; ++i) f(e[i], v + i);
        });
    }
};

struct Shared {
    uint64_t bins[kBins]; // or the sums of tiles
    uint2 list[kList];    // (key, token)
    uint64_t wave_sum[16];
    uint64_t before, amount;
    uint32_t low, high;
    int count, place;
};

__device__ __forceinline__ uint64_t wave_scan(uint64_t x)
{
    const int lane = threadIdx.x & 63;
    for (int d = 1; d < 64; d <<= 1) {
        const uint64_t y = __shfl_up((unsigned long long)x, d);
        if (lane >= d) x += y;
    }
    return x;
}

// The first of `count` numbers in LDS at which the sum up to it reaches the target that target(sum of all) gives: s.place, s.before (the sum
// before it) and s.amount (it).  count <= kBins.  A target is 1 at least; one beyond the sum leaves s.place at -1.
template <class F> __device__ uint64_t find(Shared &s, int count, const F &target)
{
    const int per = (count + blockDim.x - 1) / blockDim.x, first = threadIdx.x * per, wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
    uint64_t mine = 0;
    for (int i = 0; i < per; ++i)
        if (first + i < count) mine += s.bins[first + i];
    const uint64_t upto = wave_scan(mine);
    if ((threadIdx.x & 63) == 63) s.wave_sum[wave] = upto;
    if (threadIdx.x == 0) s.place = -1;
    __syncthreads();
    uint64_t before = upto - mine, all = 0;
    for (int w = 0; w < waves; ++w) {
        if (w < wave) before += s.wave_sum[w];
        all += s.wave_sum[w];
    }
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
    for (int i = threadIdx.x; i < kBins; i += blockDim.x) s.bins[i] = 0;
    __syncthreads();
}

// Narrows [low, high] to the number at which the amounts of the numbers up to it reach `target`, `before` those before low: source(add) calls
// add(number, amount) for all numbers.  Returns it, *before the sum before it and *amount its own.
template <class F> __device__ uint32_t narrow(Shared &s, uint32_t low, uint32_t high, uint64_t target, uint64_t *before, uint64_t *amount, const F &source)
{
    while (low < high) {
        const int bits = 32 - __builtin_clz(high - low), shift = bits > 11 ? bits - 11 : 0;
        clear_bins(s);
        source([&](uint32_t r, uint64_t x) {
            if (r >= low && r <= high) atomicAdd((unsigned long long *)&s.bins[(r - low) >> shift], (unsigned long long)x);
        });
        __syncthreads();
        const uint64_t wanted = target - *before;
        find(s, kBins, [&](uint64_t) { return wanted; });
        const uint32_t place = s.place < 0 ? 0 : s.place; // always found
        *before += s.before;
        *amount = s.amount;
        low += place << shift;
        const uint32_t end = low + ((1u << shift) - 1);
        high = end < high ? end : high;
        __syncthreads();
    }
    return low;
}

// Where the amounts of the tokens that `cut` keeps, in order, reach target(their sum).  amount(logit) is a token's: 1, or its weight.
template <class T, class A, class F> __device__ Cut select(Shared &s, const Row<T> &row, Cut cut, float most, float rate, const A &amount, const F &target)
{
    // First bins are even in the logit, 64 to a factor of two in the weight: tokens spread over many, and few are in the one that matters
    const auto bin_of = [&](float x) { return (int)fminf((most - x) * rate, (float)(kBins - 1)); };
    clear_bins(s);
    row.each([&](float x, int v) {
        if (x != -INFINITY && cut.keeps(key_of(x), v)) atomicAdd((unsigned long long *)&s.bins[bin_of(x)], (unsigned long long)amount(x));
    });
    __syncthreads();
    if (threadIdx.x == 0) s.count = 0, s.low = 0xffffffffu, s.high = 0;
    uint64_t wanted = 0;
    find(s, kBins, [&](uint64_t all) { return wanted = target(all); });
    const int bin = s.place;
    uint64_t before = s.before, sum = s.amount;
    if (bin < 0) return cut; // fewer tokens than wanted
    row.each([&](float x, int v) {
        if (x == -INFINITY || bin_of(x) != bin) return;
        const uint32_t key = key_of(x);
        if (!cut.keeps(key, v)) return;
        const int at = atomicAdd(&s.count, 1);
        if (at < kList) s.list[at] = make_uint2(key, v);
        atomicMin(&s.low, key);
        atomicMax(&s.high, key);
    });
    __syncthreads();
    const int listed = s.count;
    const uint32_t low = s.low, high = s.high;
    __syncthreads();
    // the bin's tokens: from the list, or from the row where it holds too many
    const auto tokens = [&](const auto &f) {
        if (listed <= kList) {
            for (int i = threadIdx.x; i < listed; i += blockDim.x) f(s.list[i].x, (int)s.list[i].y);
        } else {
            row.each([&](float x, int v) {
                if (x != -INFINITY && bin_of(x) == bin && cut.keeps(key_of(x), v)) f(key_of(x), v);
            });
        }
    };
    Cut out;
    out.key = narrow(s, low, high, wanted, &before, &sum, [&](const auto &add) { tokens([&](uint32_t key, int) { add(key, amount(logit_of(key))); }); });
    const uint64_t one = amount(logit_of(out.key)), enough = (wanted - before + one - 1) / one, there = sum / one;
    out.last = 0x7fffffff;
    if (enough < there) {
        uint64_t ahead = 0, unused;
        out.last = (int)narrow(s, 0, row.vocabulary - 1, enough, &ahead, &unused, [&](const auto &add) {
            tokens([&](uint32_t key, int v) {
                if (key == out.key) add((uint32_t)v, 1);
            });
        });
    } else if (out.key == cut.key) {
        out.last = cut.last;
    }
    return out;
}

template <class T, class P> __global__ __launch_bounds__(1024) void sample_kernel(const SampleArgs a)
{
    __shared__ Shared s;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = blockDim.x >> 6, V = a.vocabulary;
    const int64_t r = blockIdx.x;
    Row<T> row{static_cast<const T *>(a.logits) + r * a.stride, V, false};

    uint64_t best = 0; // (key, token), inverted: the least of both is the greatest
    row.each([&](float x, int v) {
        const uint64_t y = x == -INFINITY ? 0 : (uint64_t)~key_of(x) << 32 | (uint32_t)~(uint32_t)v;
        best = y > best ? y : best;
    });
    for (int m = 1; m < 64; m <<= 1) {
        const uint64_t y = __shfl_xor((unsigned long long)best, m);
        best = y > best ? y : best;
    }
    if (lane == 0) s.wave_sum[wave] = best;
    __syncthreads();
    for (int w = 0; w < waves; ++w) best = s.wave_sum[w] > best ? s.wave_sum[w] : best;
    __syncthreads();
    P *const kept = a.probabilities ? static_cast<P *>(a.probabilities) + r * V : nullptr;
    const auto write = [&](const auto &probability) {
        if (!kept) return;
        row.tiles([&](int, int v, const float(&e)[kEach]) {
            Eight<P> p;
#pragma unroll
            for (int i = 0; i < kEach; ++i) p.x[i] = (P)probability(e[i], v + i);
            if (v + kEach <= V) *reinterpret_cast<Eight<P> *>(kept + v) = p;
            else
                for (int i = 0; i < kEach; ++i)
                    if (v + i < V) kept[v + i] = p.x[i];
        });
    };
    const float t = a.temperature ? a.temperature[r] : 1.0f;
    const int first = best ? (int)~(uint32_t)best : -1;
    if (!(t > 0) || first < 0) { // the first token alone, or none
        if (threadIdx.x == 0) a.tokens[r] = first;
        write([&](float, int v) { return v == first ? 1.0f : 0.0f; });
        return;
    }
    float most = logit_of(~(uint32_t)(best >> 32));
    if (most == INFINITY) {
        row.infinite = true;
        most = 0;
    }
    Weights w;
    w.most = most;
    w.rate = kLog2e / (double)t;
    w.unit = a.unit;
    const float least = a.min_p ? a.min_p[r] : 0.0f;
    w.least = least > 0 ? least < 1 ? (double)least : 1.0 : 0.0;
    const float rate = fmaxf(fminf(64 * (float)w.rate, 1e30f), 1e-30f);

    Cut cut{0xffffffffu, 0x7fffffff};
    const int k = a.top_k ? a.top_k[r] : 0;
    const float p = a.top_p ? a.top_p[r] : 1.0f;
    if (k > 0 && k < V) cut = select(s, row, cut, most, rate, [](float) { return (uint64_t)1; }, [&](uint64_t) { return (uint64_t)k; });
    if (p < 1)
        cut = select(s, row, cut, most, rate, [&](float x) { return w.fixed(w.of(x)); }, [&](uint64_t all) {
            const double x = __builtin_ceil((double)p * (double)all);
            return x >= 1 ? (uint64_t)x : (uint64_t)1;
        });

    const auto weight = [&](float x, int v) {
        if (x == -INFINITY || !cut.keeps(key_of(x), v)) return 0.0;
        const double y = w.of(x);
        return y >= w.least ? y : 0.0;
    };
    __syncthreads();
    row.tiles([&](int tile, int v, const float(&e)[kEach]) {
        uint64_t sum = 0;
#pragma unroll
        for (int i = 0; i < kEach; ++i) sum += w.fixed(weight(e[i], v + i));
        for (int m = 1; m < 64; m <<= 1) sum += __shfl_xor((unsigned long long)sum, m);
        if (lane == 0) s.bins[tile] = sum;
    });
    __syncthreads();
    const float u = a.uniform[r];
    uint64_t wanted = 0;
    const uint64_t all = find(s, (V + kTile - 1) / kTile, [&](uint64_t sum) {
        const double x = __builtin_floor((double)u * (double)sum);
        wanted = !(u < 1) || x >= (double)sum ? sum : x > 0 ? (uint64_t)x + 1 : 1;
        return wanted;
    });
    if (wave == 0) {
        float e[kEach];
        const int v = s.place * kTile + lane * kEach;
        row.load(v, e);
        uint64_t each[kEach], sum = 0;
#pragma unroll
        for (int i = 0; i < kEach; ++i) sum += each[i] = w.fixed(weight(e[i], v + i));
        uint64_t before = wave_scan(sum) - sum + s.before;
        if (before < wanted && wanted <= before + sum) {
#pragma unroll
            for (int i = 0; i < kEach; ++i) {
                if (before < wanted && wanted <= before + each[i]) a.tokens[r] = v + i;
                before += each[i];
            }
        }
    }
    const double share = __builtin_ldexp(1.0, a.unit) / (double)all;
    write([&](float x, int v) { return (float)(weight(x, v) * share); });
}

template <class T, class P> void launch(const SampleArgs &k, hipStream_t stream)
{
    const int tiles = (k.vocabulary + kTile - 1) / kTile;
    sample_kernel<T, P><<<(unsigned)k.rows, 64 * (tiles < 16 ? tiles : 16), 0, stream>>>(k);
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
