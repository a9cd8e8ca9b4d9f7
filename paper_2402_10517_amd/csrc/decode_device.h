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

// Tokens [begin, end) of sequence s; none where the two starts descend or leave [0, tokens]
__device__ __forceinline__ void token_range(const int32_t *starts, int s, int64_t tokens, int sequences, int64_t *begin, int64_t *end)
{
    if (!starts) {
        const int64_t each = tokens / sequences;
        *begin = s * each;
        *end = *begin + each;
        return;
    }
    const int64_t a = starts[s], b = starts[s + 1];
    const bool ok = a >= 0 && a <= b && b <= tokens;
    *begin = ok ? a : 0;
    *end = ok ? b : 0;
}

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

} // namespace apgemv
#endif
