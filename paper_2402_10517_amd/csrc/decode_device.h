// Device helpers of the decoder operators: addresses in the 4-bit cache, rows of the sequences of a packed batch.
#ifndef APGEMV_DECODE_DEVICE_H
#define APGEMV_DECODE_DEVICE_H

#include <hip/hip_runtime.h>

#include "decode.h"

namespace apgemv {

typedef _Float16 half8_t __attribute__((ext_vector_type(8)));
typedef _Float16 half4_t __attribute__((ext_vector_type(4)));
typedef float float4_t __attribute__((ext_vector_type(4)));
typedef uint32_t uint4_t __attribute__((ext_vector_type(4)));
typedef uint32_t uint2_t __attribute__((ext_vector_type(2)));

// Byte offsets inside one (page, key head)
template <int D> struct CacheLayout {
    static constexpr int kRow = D / 2;   // code bytes of a token
    static constexpr int kHalves = D / 64; // words per chunk and pair of tokens of the value codes
    __device__ static int64_t block_bytes(int log_page) { return (int64_t)(D + 8) << log_page; }
    __device__ static int key(int t) { return t * kRow; }
    // the 16 bits that hold channels c * D/16 + 4 h .. + 3 of token t
    __device__ static int value(int log_page, int t, int c, int h)
    {
        return (kRow << log_page) + (t >> 2) * 4 * kRow + c * 8 * kHalves + ((t >> 1) & 1) * 4 * kHalves + h * 4 + (t & 1) * 2;
    }
    __device__ static int key_scale(int log_page, int t) { return (D << log_page) + t * 4; }
    __device__ static int value_scale(int log_page, int t) { return ((D + 4) << log_page) + t * 4; }
    __device__ static uint8_t *block(const CacheShape &c, int64_t page, int head)
    {
        return c.data + (page * c.kv_heads + head) * block_bytes(c.log_page);
    }
};

// Tokens [begin, end) of sequence s; none, and false, where the two starts descend or leave [0, tokens]
__device__ __forceinline__ bool token_range(const int32_t *starts, int s, int64_t tokens, int sequences, int64_t *begin, int64_t *end)
{
    if (!starts) {
        const int64_t each = tokens / sequences;
        *begin = s * each;
        *end = *begin + each;
        return true;
    }
    const int64_t a = starts[s], b = starts[s + 1];
    const bool ok = a >= 0 && a <= b && b <= tokens;
    *begin = ok ? a : 0;
    *end = ok ? b : 0;
    return ok;
}

// Ranges of rows that begin before the end of an earlier one are none: no row has two owners, and all row tiles together are as many as the host has counted.  64 lanes call
// together, each with its range, for the first 64 ranges, the next 64 and so on.  ok: the range is as its starts say, or the lane has none.  Starts that do not descend have no
// such ranges, and cost a vote of the wave.
struct Apart {
    int upto = 0; // the greatest end so far
    bool ordered = true;
    __device__ __forceinline__ void cut(bool ok, int64_t *begin, int64_t *end)
    {
        ordered = ordered && __all(ok);
        const bool filled = *begin < *end;
        if (ordered) {
            const uint64_t lanes = __ballot(filled);
            if (lanes) upto = __builtin_amdgcn_readlane((int)*end, 63 - __builtin_clzll(lanes));
            return;
        }
        const int lane = threadIdx.x & 63;
#pragma unroll 1
        for (int i = 0; i < 64; ++i) {
            const int from = __builtin_amdgcn_readlane((int)*begin, i), to = __builtin_amdgcn_readlane((int)*end, i);
            if (from < upto && lane == i) *begin = *end = 0;
            if (from < to && to > upto) upto = to;
        }
    }
};

// The sequence of token i (all 64 lanes call together); -1 for a token of none, as those of a sequence that begins in an earlier one are
__device__ __forceinline__ int sequence_of(const int32_t *starts, int64_t i, int64_t tokens, int sequences)
{
    if (!starts) return (int)(i / (tokens / sequences));
    const int lane = threadIdx.x & 63;
    Apart apart;
    for (int first = 0; first < sequences; first += 64) {
        int64_t a = 0, b = 0;
        const bool ok = first + lane >= sequences || token_range(starts, first + lane, tokens, sequences, &a, &b);
        apart.cut(ok, &a, &b);
        const uint64_t found = __ballot(i >= a && i < b);
        if (found) return first + __builtin_ctzll(found);
    }
    return -1;
}

} // namespace apgemv
#endif
