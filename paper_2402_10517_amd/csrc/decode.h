// Internal interface between the decoder operators' entry points (decode_api.cpp) and their HIP kernels, and the device layout
// of the 4-bit cache.
#ifndef APGEMV_DECODE_H
#define APGEMV_DECODE_H

#include <hip/hip_runtime_api.h>
#include <stddef.h>
#include <stdint.h>

#include "../../include/apdecode.h"

namespace apgemv {

// One (page, key head) of the cache is contiguous, P = page_tokens, D = head_dim:
//   key codes     P rows of D / 2 bytes, code of channel d in nibble d & 1 of byte d / 2
//   value codes   per quad of 4 tokens 2 * D bytes: 16 chunks c (channels c * D/16 ..), each with the pairs of tokens (0, 1), (2, 3),
//                 each with D / 64 words: bits 0-15 four channels of the even token, bits 16-31 of the odd one
//   (low, scale)  binary16 pairs: of the keys by token, then of the values
// The matrix instructions want consecutive tokens of one channel in a lane for the values: (word >> 4 n) & 0x000f000f is channel n
// of two adjacent tokens in the halves of a register, without an exchange between lanes.
struct CacheShape {
    uint8_t *data;
    int64_t pages;
    int log_page; // page_tokens = 1 << log_page
    int kv_heads;
};
inline int cache_log_page(int page_tokens)
{
    for (int l = 4; l <= 8; ++l)
        if (page_tokens == 1 << l) return l;
    return -1;
}

// Workgroups of a launch: a grid has fewer than 2^32 threads, and a workgroup 256.  An attention has one per row tile (16 rows of the cached one at
// least, 128 of the prompts', one more per sequence) and key head; several per tile only where these are too few for the card.
constexpr int64_t kMostGroups = ((int64_t)1 << 24) - 1;
inline bool groups_ok(int64_t rows, int rows_per_tile, int64_t sequences, int kv_heads) { return rows / rows_per_tile + sequences * kv_heads <= kMostGroups; }

hipError_t launch_cache_append(const ap_cache &c, const ap_append &a, hipStream_t stream);
hipError_t launch_cache_read(const ap_cache &c, const int64_t *slots, int64_t tokens, void *k, void *v, hipStream_t stream);
size_t attention_cached_work(const ap_cache &c, const ap_cached &a);
hipError_t launch_attention_cached(const ap_cache &c, const ap_cached &a, hipStream_t stream);
size_t attention_prompt_work(const ap_prompt &a);
hipError_t launch_attention_prompt(const ap_prompt &a, hipStream_t stream);
size_t verify_work(const ap_verification &a);
hipError_t launch_verify(const ap_verification &a, hipStream_t stream);
size_t attention_shared_work(const ap_cache &c, const ap_shared &a);
hipError_t launch_attention_shared(const ap_cache &c, const ap_shared &a, hipStream_t stream);
hipError_t launch_norm(const ap_normed &a, hipStream_t stream);
hipError_t launch_sample(const ap_sampling &a, hipStream_t stream);

inline CacheShape cache_shape(const ap_cache &c)
{
    return CacheShape{static_cast<uint8_t *>(c.data), c.pages, cache_log_page(c.page_tokens), c.kv_heads};
}

// The scale that a kernel works with.  One of 0 makes all weights equal, as 1e-30 does, and leaves scores of -inf (keys that are not seen) what they are;
// from 1e30 on, short of where products with log2 e and 2^24 overflow, the greatest score has all the weight either way (others are 2^-48 below it at least).
inline float scale_in_range(float scale)
{
    const float size = scale < 0 ? -scale : scale;
    return size < 1e-30f ? 1e-30f : size <= 1e30f ? scale : scale < 0 ? -1e30f : 1e30f;
}

} // namespace apgemv
#endif
