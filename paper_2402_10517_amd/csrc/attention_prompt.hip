// Causal attention over packed sequences of binary16 keys and values.
#include "attention_rows.h"

namespace apgemv {

namespace {

struct PromptArgs {
    const _Float16 *q, *k, *v;
    int64_t q_token, q_head, k_token, k_head, v_token, v_head, tokens, keys;
    const int32_t *q_starts, *k_starts;
    int heads, kv_heads, sequences;
    float scale;
    _Float16 *out;
};

template <int D> struct PromptRows {
    const _Float16 *k, *v;
    int64_t k_token, v_token;
    __device__ float score(int64_t j, const float *q) const
    {
        float sum = 0;
        for (int d = 0; d < D; ++d) sum += q[d] * (float)k[j * k_token + d];
        return sum;
    }
    __device__ float value(int64_t j, int d) const { return (float)v[j * v_token + d]; }
};

template <int D> __global__ __launch_bounds__(64) void attention_prompt_kernel(const PromptArgs a)
{
    const int64_t rows = a.tokens * a.heads;
    for (int64_t row = blockIdx.x; row < rows; row += gridDim.x) {
        const int64_t token = row / a.heads;
        const int head = (int)(row - token * a.heads), kv = head / (a.heads / a.kv_heads);
        const int s = sequence_of(a.q_starts, token, a.tokens, a.sequences);
        if (s < 0) continue;
        int64_t begin, end, k0, k1;
        token_range(a.q_starts, s, a.tokens, a.sequences, &begin, &end);
        token_range(a.k_starts, s, a.keys, a.sequences, &k0, &k1);
        const PromptRows<D> source{a.k + k0 * a.k_token + kv * a.k_head, a.v + k0 * a.v_token + kv * a.v_head, a.k_token, a.v_token};
        attend_row<D>(source, (k1 - k0) - (end - 1 - token), a.q + token * a.q_token + head * a.q_head, a.scale, a.out + row * D);
    }
}

} // namespace

hipError_t launch_attention_prompt(const ap_prompt &a, hipStream_t stream)
{
    PromptArgs k;
    k.q = static_cast<const _Float16 *>(a.q.data);
    k.k = static_cast<const _Float16 *>(a.k.data);
    k.v = static_cast<const _Float16 *>(a.v.data);
    k.q_token = a.q.token_stride, k.q_head = a.q.head_stride;
    k.k_token = a.k.token_stride, k.k_head = a.k.head_stride;
    k.v_token = a.v.token_stride, k.v_head = a.v.head_stride;
    k.tokens = a.tokens, k.keys = a.keys;
    k.q_starts = a.q_starts, k.k_starts = a.k_starts;
    k.heads = a.heads, k.kv_heads = a.kv_heads, k.sequences = a.sequences;
    k.scale = a.scale;
    k.out = static_cast<_Float16 *>(a.out);
    const int64_t rows = a.tokens * a.heads;
    const dim3 grid((unsigned)(rows < (1 << 22) ? rows : 1 << 22));
    if (a.head_dim == 64) attention_prompt_kernel<64><<<grid, 64, 0, stream>>>(k);
    else attention_prompt_kernel<128><<<grid, 64, 0, stream>>>(k);
    return hipGetLastError();
}

} // namespace apgemv
