// Verification of drafted tokens: accepted prefix, and the token after it by an exponential race.
#include "decode_device.h"

namespace apgemv {

namespace {

constexpr int kThreads = 256;

struct VerifyArgs {
    const void *target, *draft;
    const int64_t *drafted;
    const float *uniform, *noise;
    const int32_t *counts;
    int64_t *tokens;
    int32_t *accepted;
    int64_t vocabulary;
    int sequences, drafts;
};

// A candidate as one number whose order is that of (ratio, lower index): ratios are not negative, so their bits order like they do.
__device__ __forceinline__ uint64_t candidate(float w, float noise, int64_t v)
{
    const float ratio = w / noise;
    if (!(w > 0.0f) || !(ratio >= 0.0f)) return 0;
    return (uint64_t)__float_as_uint(ratio) << 32 | (uint32_t)~(uint32_t)v;
}

__device__ __forceinline__ uint64_t wave_max(uint64_t x)
{
    for (int m = 1; m < 64; m <<= 1) {
        const uint64_t y = __shfl_xor((unsigned long long)x, m);
        x = y > x ? y : x;
    }
    return x;
}

template <class T> __global__ __launch_bounds__(kThreads) void verify_kernel(const VerifyArgs a)
{
    const int64_t s = blockIdx.x, V = a.vocabulary;
    const T *target = static_cast<const T *>(a.target) + s * (a.drafts + 1) * V;
    const T *draft = static_cast<const T *>(a.draft) + s * a.drafts * V;
    const int64_t *drafted = a.drafted + s * a.drafts;
    const float *uniform = a.uniform + s * a.drafts, *noise = a.noise + s * V;
    int count = a.counts ? a.counts[s] : a.drafts;
    count = count < 0 ? 0 : count > a.drafts ? a.drafts : count;
    int n = 0;
    while (n < count) {
        const int64_t x = drafted[n];
        if (x < 0 || x >= V || !(uniform[n] * (float)draft[n * V + x] < (float)target[n * V + x])) break;
        ++n;
    }
    const bool refused = n < count;
    uint64_t rest = 0, full = 0;
    for (int64_t v = threadIdx.x; v < V; v += kThreads) {
        const float p = (float)target[n * V + v], e = noise[v];
        const uint64_t f = candidate(p, e, v);
        full = f > full ? f : full;
        if (refused) {
            const uint64_t r = candidate(p - (float)draft[n * V + v], e, v);
            rest = r > rest ? r : rest;
        }
    }
    __shared__ uint64_t best[2][kThreads / 64];
    rest = wave_max(rest);
    full = wave_max(full);
    if ((threadIdx.x & 63) == 0) best[0][threadIdx.x >> 6] = rest, best[1][threadIdx.x >> 6] = full;
    __syncthreads();
    for (int w = 0; w < kThreads / 64; ++w) {
        rest = best[0][w] > rest ? best[0][w] : rest;
        full = best[1][w] > full ? best[1][w] : full;
    }
    const uint64_t won = rest ? rest : full;
    const int64_t token = won ? (int64_t)(uint32_t)~(uint32_t)won : -1;
    for (int i = threadIdx.x; i <= a.drafts; i += kThreads) a.tokens[s * (a.drafts + 1) + i] = i < n ? drafted[i] : i == n ? token : -1;
    if (threadIdx.x == 0) a.accepted[s] = n;
}

} // namespace

size_t verify_work(const ap_verification &) { return 0; }

hipError_t launch_verify(const ap_verification &a, hipStream_t stream)
{
    const VerifyArgs k{a.target, a.draft, a.drafted, a.uniform, a.noise, a.counts, a.tokens, a.accepted, a.vocabulary, a.sequences, a.drafts};
    if (a.half) verify_kernel<_Float16><<<a.sequences, kThreads, 0, stream>>>(k);
    else verify_kernel<float><<<a.sequences, kThreads, 0, stream>>>(k);
    return hipGetLastError();
}

} // namespace apgemv
