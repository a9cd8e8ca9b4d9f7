// Attention of one query row by one wave, for any source of keys and values: the online softmax
//   m' = max(m, max s_j),  l' = l e^(m - m') + sum e^(s_j - m'),  o' = o e^(m - m') + sum e^(s_j - m') v_j
// over 64 keys at a time: a lane takes a key for the scores, then D / 64 channels for the values.
#ifndef APGEMV_ATTENTION_ROWS_H
#define APGEMV_ATTENTION_ROWS_H

#include "decode_device.h"

namespace apgemv {

// The sequence of token i (all 64 lanes call together); -1 for a token of none
__device__ __forceinline__ int sequence_of(const int32_t *starts, int64_t i, int64_t tokens, int sequences)
{
    if (!starts) return (int)(i / (tokens / sequences));
    const int lane = threadIdx.x & 63;
    for (int first = 0; first < sequences; first += 64) {
        bool mine = false;
        if (first + lane < sequences) {
            int64_t a, b;
            token_range(starts, first + lane, tokens, sequences, &a, &b);
            mine = i >= a && i < b;
        }
        const uint64_t found = __ballot(mine);
        if (found) return first + __builtin_ctzll(found);
    }
    return -1;
}

// keys 0 .. seen - 1 of `source`; q: the row; out: D values
template <int D, class Source>
__device__ __forceinline__ void attend_row(const Source &source, int64_t seen, const _Float16 *q, float scale, _Float16 *out)
{
    constexpr int C = D / 64;
    __shared__ float weight[64];
    __shared__ float query[D];
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int c = 0; c < C; ++c) query[c * 64 + lane] = (float)q[c * 64 + lane];
    __syncthreads();
    float m = -INFINITY, l = 0, o[C] = {};
    for (int64_t first = 0; first < seen; first += 64) {
        const bool valid = first + lane < seen;
        const float s = valid ? source.score(first + lane, query) * scale : -INFINITY;
        float top = s;
        for (int x = 1; x < 64; x <<= 1) top = fmaxf(top, __shfl_xor(top, x));
        const float next = fmaxf(m, top), base = next == -INFINITY ? 0.0f : next;
        const float keep = expf(m - base), p = valid ? expf(s - base) : 0.0f;
        float sum = p;
        for (int x = 1; x < 64; x <<= 1) sum += __shfl_xor(sum, x);
        l = l * keep + sum;
        m = next;
        weight[lane] = p;
        __syncthreads();
        const int n = (int)(seen - first < 64 ? seen - first : 64);
#pragma unroll
        for (int c = 0; c < C; ++c) {
            o[c] *= keep;
            for (int j = 0; j < n; ++j) o[c] += weight[j] * source.value(first + j, c * 64 + lane);
        }
        __syncthreads();
    }
#pragma unroll
    for (int c = 0; c < C; ++c) out[c * 64 + lane] = (_Float16)(l == 0.0f ? 0.0f : o[c] / l);
}

} // namespace apgemv
#endif
