// Verification of drafted tokens: accepted prefix, and the token after it by an exponential race.
//
// The token is the argmax of w / noise with lowest index first: no sum is taken, so any division of the vocabulary gives the same token, bit for bit.
// Bound by HBM: one row of target and draft probabilities and the noise per sequence.  Few sequences leave most of the card idle, so a vocabulary is
// divided among workgroups (2048 tokens at least each) and joined by a second launch, small ones aside. 64 sequences over 131071 binary16 probabilities take 16.3 to
// 17.3 us (67 MB, 3.9 to 4.1 TB/s), 4 drafts over 32000 tokens 8.1 to 9.1, two launches.
#include "decode_device.h"

namespace apgemv {

namespace {

constexpr int kThreads = 256; // of a workgroup that shares a vocabulary, or has one among many
constexpr int kWide = 1024;   // of one that has a small vocabulary for itself
constexpr int kEach = 8;      // consecutive tokens of a thread
constexpr int kStep = kThreads * kEach;

struct VerifyArgs {
    const void *target, *draft;
    const int64_t *drafted;
    const float *uniform, *noise;
    const int32_t *counts;
    int64_t *tokens;
    int32_t *accepted;
    uint64_t *best; // sequences x parts
    int64_t vocabulary, slice;
    int sequences, drafts, parts;
};

// A candidate as one number whose order is that of (ratio, lower index): ratios are not negative, so their bits order like they do, and indexes are
// below 2^31, so that every candidate is greater than kNoNoise: tokens with a weight, none with noise that counts.  0 = no token with a weight
constexpr uint64_t kNoNoise = 1;
__device__ __forceinline__ uint64_t candidate(float ratio, int64_t v, bool weight)
{
    return ratio >= 0.0f ? (uint64_t)__float_as_uint(ratio) << 32 | (uint32_t)~(uint32_t)v : weight ? kNoNoise : 0;
}

template <int THREADS> __device__ __forceinline__ uint64_t block_max(uint64_t x)
{
    __shared__ uint64_t best[THREADS / 64];
    for (int m = 1; m < 64; m <<= 1) {
        const uint64_t y = __shfl_xor((unsigned long long)x, m);
        x = y > x ? y : x;
    }
    __syncthreads();
    if ((threadIdx.x & 63) == 0) best[threadIdx.x >> 6] = x;
    __syncthreads();
    for (int w = 0; w < THREADS / 64; ++w) x = best[w] > x ? best[w] : x;
    return x;
}

// Rows of an odd vocabulary start at any element: 16-byte loads that ask for the element's alignment only
template <class T> struct __attribute__((packed, aligned(sizeof(T)))) Eight {
    T x[kEach];
};

// The best of tokens [from, to): w = p - q, or p where there is no q
template <class T, int THREADS> __device__ __forceinline__ uint64_t race(const T *p, const T *q, const float *noise, int64_t from, int64_t to)
{
    float best = -1.0f;
    int64_t at = 0;
    bool weight = false;
    const auto consider = [&](float pv, float qv, float e, int64_t v) {
        const float w = pv - qv, ratio = w / e;
        weight = weight || w > 0.0f;
        if (w > 0.0f && e >= 0.0f && ratio > best) { // in ascending order: the lowest of equals stays
            best = ratio;
            at = v;
        }
    };
    int64_t v = from + (int64_t)threadIdx.x * kEach;
    for (; v + kEach <= to; v += THREADS * kEach) {
        const Eight<T> a = *reinterpret_cast<const Eight<T> *>(p + v);
        const Eight<float> e = *reinterpret_cast<const Eight<float> *>(noise + v);
        Eight<T> b;
        if (q) b = *reinterpret_cast<const Eight<T> *>(q + v);
#pragma unroll
        for (int i = 0; i < kEach; ++i) consider((float)a.x[i], q ? (float)b.x[i] : 0.0f, e.x[i], v + i);
    }
    for (int i = 0; i < kEach && v + i < to; ++i) consider((float)p[v + i], q ? (float)q[v + i] : 0.0f, noise[v + i], v + i);
    return block_max<THREADS>(candidate(best, at, weight));
}

struct Sequence {
    int count, accepted;
};

template <class T> __device__ __forceinline__ Sequence accept(const VerifyArgs &a, int64_t s)
{
    const int lane = threadIdx.x & 63;
    const int64_t V = a.vocabulary;
    Sequence r;
    r.count = a.counts ? a.counts[s] : a.drafts;
    r.count = r.count < 0 ? 0 : r.count > a.drafts ? a.drafts : r.count;
    r.accepted = r.count;
    for (int first = 0; first < r.count; first += 64) {
        const int i = first + lane;
        bool refused = false;
        if (i < r.count) {
            const int64_t x = a.drafted[s * a.drafts + i];
            refused = true;
            if (x >= 0 && x < V) {
                const float p = (float)static_cast<const T *>(a.target)[(s * (a.drafts + 1) + i) * V + x];
                const float q = (float)static_cast<const T *>(a.draft)[(s * a.drafts + i) * V + x];
                refused = !(a.uniform[s * a.drafts + i] * q < p);
            }
        }
        const uint64_t out = __ballot(refused);
        if (out) {
            r.accepted = first + __builtin_ctzll(out);
            break;
        }
    }
    return r;
}

// The end of a sequence, once the best of the whole vocabulary is known (0 after a refusal: no token has more than its draft)
template <class T, int THREADS> __device__ __forceinline__ void finish(const VerifyArgs &a, int64_t s, int accepted, bool refused, uint64_t won)
{
    if (!won && refused)
        won = race<T, THREADS>(static_cast<const T *>(a.target) + (s * (a.drafts + 1) + accepted) * a.vocabulary, nullptr, a.noise + s * a.vocabulary, 0, a.vocabulary);
    const int64_t token = won > kNoNoise ? (int64_t)(uint32_t)~(uint32_t)won : -1;
    for (int i = threadIdx.x; i <= a.drafts; i += THREADS)
        a.tokens[s * (a.drafts + 1) + i] = i < accepted ? a.drafted[s * a.drafts + i] : i == accepted ? token : -1;
}

template <class T, int THREADS> __global__ __launch_bounds__(THREADS) void verify_kernel(const VerifyArgs a)
{
    const int64_t s = blockIdx.x / a.parts, V = a.vocabulary;
    const int part = blockIdx.x - (int)s * a.parts;
    const Sequence r = accept<T>(a, s);
    const bool refused = r.accepted < r.count;
    const T *p = static_cast<const T *>(a.target) + (s * (a.drafts + 1) + r.accepted) * V;
    const T *q = refused ? static_cast<const T *>(a.draft) + (s * a.drafts + r.accepted) * V : nullptr;
    const int64_t from = part * a.slice, to = from + a.slice < V ? from + a.slice : V;
    const uint64_t won = race<T, THREADS>(p, q, a.noise + s * V, from, to);
    if (a.parts == 1) finish<T, THREADS>(a, s, r.accepted, refused, won);
    else if (threadIdx.x == 0) a.best[blockIdx.x] = won;
    if (part == 0 && threadIdx.x == 0) a.accepted[s] = r.accepted;
}

template <class T> __global__ __launch_bounds__(kThreads) void verify_join_kernel(const VerifyArgs a)
{
    const int64_t s = blockIdx.x;
    uint64_t won = 0;
    for (int i = threadIdx.x; i < a.parts; i += kThreads) {
        const uint64_t x = a.best[s * a.parts + i];
        won = x > won ? x : won;
    }
    won = block_max<kThreads>(won);
    int count = a.counts ? a.counts[s] : a.drafts;
    count = count > a.drafts ? a.drafts : count;
    const int accepted = a.accepted[s];
    finish<T, kThreads>(a, s, accepted, accepted < count, won);
}

struct Plan {
    int parts, threads;
};

// Parts of a vocabulary: as many as give the card four workgroups per CU, of one step at least.  A vocabulary of up to two steps of a wide workgroup is
// not divided, which saves the second launch.  us divided / not, 4 drafts: 1 sequence of 8000 tokens 8.7 / 5.4, 16000 9.2 / 6.7, 32000 8.8 / 8.6; 64
// sequences of 32000 8.4 / 9.7, 300 of 20000 in binary16 14.0 / 16.2.
Plan plan_of(const ap_verification &a)
{
    const int64_t steps = (a.vocabulary + kStep - 1) / kStep, wanted = (1024 + a.sequences - 1) / a.sequences;
    const int parts = (int)(wanted < steps ? wanted : steps);
    if (parts > 1 && a.vocabulary <= 2 * kWide * kEach) return Plan{1, kWide};
    return Plan{parts, kThreads};
}

template <class T> void launch(const VerifyArgs &k, const Plan &p, hipStream_t stream)
{
    const dim3 grid((unsigned)k.sequences * (unsigned)p.parts);
    if (p.threads == kWide) verify_kernel<T, kWide><<<grid, kWide, 0, stream>>>(k);
    else verify_kernel<T, kThreads><<<grid, kThreads, 0, stream>>>(k);
    if (p.parts > 1) verify_join_kernel<T><<<k.sequences, kThreads, 0, stream>>>(k);
}

} // namespace

size_t verify_work(const ap_verification &a)
{
    const int parts = plan_of(a).parts;
    return parts == 1 ? 0 : (size_t)parts * a.sequences * sizeof(uint64_t);
}

hipError_t launch_verify(const ap_verification &a, hipStream_t stream)
{
    const Plan p = plan_of(a);
    const int64_t steps = (a.vocabulary + kStep - 1) / kStep, slice = (steps + p.parts - 1) / p.parts * kStep;
    const VerifyArgs k{a.target,   a.draft,    a.drafted,                      a.uniform,    a.noise, a.counts,    a.tokens,
                       a.accepted, static_cast<uint64_t *>(a.work), a.vocabulary, slice,   a.sequences, a.drafts, p.parts};
    if (a.half) launch<_Float16>(k, p, stream);
    else launch<float>(k, p, stream);
    return hipGetLastError();
}

} // namespace apgemv
