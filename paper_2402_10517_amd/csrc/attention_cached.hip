// Attention of new tokens over the 4-bit paged cache.
#include "attention_rows.h"

namespace apgemv {

namespace {

struct CachedArgs {
    CacheShape cache;
    const _Float16 *q;
    int64_t q_token, q_head, tokens, table_width, max_length;
    const int32_t *q_starts, *lengths, *tables;
    int heads, sequences;
    float scale;
    _Float16 *out;
};

template <int D> struct CachedRows {
    typedef CacheLayout<D> L;
    CacheShape cache;
    const int32_t *table;
    int head;
    __device__ const uint8_t *block(int64_t j, int *t, bool *known) const
    {
        const int page = table[j >> cache.log_page];
        *t = (int)(j & ((1 << cache.log_page) - 1));
        *known = page >= 0 && page < cache.pages;
        return L::block(cache, *known ? page : 0, head);
    }
    __device__ float score(int64_t j, const float *q) const
    {
        int t;
        bool known;
        const uint8_t *b = block(j, &t, &known);
        const _Float16 *p = reinterpret_cast<const _Float16 *>(b + L::key_scale(cache.log_page, t));
        float sum = 0;
        for (int d = 0; d < D; ++d) sum += q[d] * ((float)p[0] + (float)p[1] * (b[L::key(t) + d / 2] >> (4 * (d & 1)) & 15));
        return known ? sum : -INFINITY;
    }
    __device__ float value(int64_t j, int d) const
    {
        int t;
        bool known;
        const uint8_t *b = block(j, &t, &known);
        const _Float16 *p = reinterpret_cast<const _Float16 *>(b + L::value_scale(cache.log_page, t));
        const int c = d / (D / 16), i = d % (D / 16);
        const int code = *reinterpret_cast<const uint16_t *>(b + L::value(cache.log_page, t, c, i / 4)) >> (4 * (i & 3)) & 15;
        return known ? (float)p[0] + (float)p[1] * code : 0.0f;
    }
};

template <int D> __global__ __launch_bounds__(64) void attention_cached_kernel(const CachedArgs a)
{
    const int64_t rows = a.tokens * a.heads;
    for (int64_t row = blockIdx.x; row < rows; row += gridDim.x) {
        const int64_t token = row / a.heads;
        const int head = (int)(row - token * a.heads);
        const int s = sequence_of(a.q_starts, token, a.tokens, a.sequences);
        if (s < 0) continue;
        int64_t begin, end;
        token_range(a.q_starts, s, a.tokens, a.sequences, &begin, &end);
        const int64_t length = a.lengths[s] < a.max_length ? a.lengths[s] : a.max_length;
        const CachedRows<D> source{a.cache, a.tables + s * a.table_width, head / (a.heads / a.cache.kv_heads)};
        attend_row<D>(source, length - (end - 1 - token), a.q + token * a.q_token + head * a.q_head, a.scale, a.out + row * D);
    }
}

} // namespace

size_t attention_cached_work(const ap_cache &, const ap_cached &) { return 0; }

hipError_t launch_attention_cached(const ap_cache &c, const ap_cached &a, hipStream_t stream)
{
    CachedArgs k;
    k.cache = cache_shape(c);
    k.q = static_cast<const _Float16 *>(a.q.data);
    k.q_token = a.q.token_stride, k.q_head = a.q.head_stride;
    k.tokens = a.tokens, k.table_width = a.table_width, k.max_length = a.max_length;
    k.q_starts = a.q_starts, k.lengths = a.lengths, k.tables = a.tables;
    k.heads = a.heads, k.sequences = a.sequences;
    k.scale = a.scale;
    k.out = static_cast<_Float16 *>(a.out);
    const int64_t rows = a.tokens * a.heads;
    const dim3 grid((unsigned)(rows < (1 << 22) ? rows : 1 << 22));
    if (c.head_dim == 64) attention_cached_kernel<64><<<grid, 64, 0, stream>>>(k);
    else attention_cached_kernel<128><<<grid, 64, 0, stream>>>(k);
    return hipGetLastError();
}

} // namespace apgemv
