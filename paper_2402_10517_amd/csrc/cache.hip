// Rotation of q and k, append of k and v to the 4-bit cache, and its values read back.
#include "decode_device.h"

namespace apgemv {

namespace {

struct AppendArgs {
    CacheShape cache;
    const _Float16 *q, *k, *v;
    _Float16 *q_out, *k_out;
    int64_t q_token, q_head, k_token, k_head, v_token, v_head, qo_token, qo_head, ko_token, ko_head;
    const int64_t *slots, *positions;
    const float *rotary;
    int64_t rotary_rows, tokens;
    int heads, rot_dim, interleaved, page_mask;
};

constexpr int kThreads = 256;
constexpr int kRowsPerGroup = kThreads / 16; // 16 lanes per row of head_dim values

template <int V> __device__ __forceinline__ void load_row(const _Float16 *p, float (&x)[V])
{
    typedef _Float16 vec __attribute__((ext_vector_type(V)));
    const vec h = *reinterpret_cast<const vec *>(p);
#pragma unroll
    for (int i = 0; i < V; ++i) x[i] = (float)h[i];
}

template <int V> __device__ __forceinline__ void store_row(_Float16 *p, const float (&x)[V])
{
    typedef _Float16 vec __attribute__((ext_vector_type(V)));
    vec h;
#pragma unroll
    for (int i = 0; i < V; ++i) h[i] = (_Float16)x[i];
    *reinterpret_cast<vec *>(p) = h;
}

// The lane's V channels c * V .. of one row, rotated.  Every product and sum is rounded by itself: the codes of the cache jump where a rounded key
// does, and should not depend on which products a compiler fuses with a sum.
template <int V> __device__ __forceinline__ void rotate(const AppendArgs &a, const _Float16 *row, int c, int64_t position, float (&x)[V])
{
#pragma clang fp contract(off)
    const int d = c * V, half = a.rot_dim / 2;
    if (!a.rotary || d >= a.rot_dim) return;
    const bool known = position >= 0 && position < a.rotary_rows;
    const float *table = a.rotary + (known ? position : 0) * a.rot_dim;
    if (a.interleaved) {
#pragma unroll
        for (int i = 0; i < V; i += 2) {
            const float cosine = table[(d + i) / 2], sine = table[half + (d + i) / 2];
            const float first = x[i] * cosine - x[i + 1] * sine, second = x[i + 1] * cosine + x[i] * sine;
            x[i] = known ? first : __builtin_nanf("");
            x[i + 1] = known ? second : __builtin_nanf("");
        }
        return;
    }
    const bool upper = d >= half;
    float other[V];
    load_row<V>(row + (upper ? d - half : d + half), other);
    const int at = upper ? d - half : d;
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const float cosine = table[at + i], sine = table[half + at + i];
        const float along = x[i] * cosine, across = other[i] * sine;
        const float r = upper ? along + across : along - across;
        x[i] = known ? r : __builtin_nanf("");
    }
}

// Codes of a row held by 16 lanes, V values each; the row's (low, scale)
template <int V> __device__ __forceinline__ uint32_t encode(const float (&x)[V], _Float16 *low, _Float16 *scale)
{
    float least = x[0], most = x[0];
    bool finite = true;
#pragma unroll
    for (int i = 0; i < V; ++i) {
        least = fminf(least, x[i]);
        most = fmaxf(most, x[i]);
        finite = finite && fabsf(x[i]) <= 65504.0f;
    }
#pragma unroll
    for (int m = 1; m < 16; m <<= 1) {
        least = fminf(least, __shfl_xor(least, m));
        most = fmaxf(most, __shfl_xor(most, m));
    }
    const uint64_t whole = __ballot(finite);
    const bool ok = ((whole >> (threadIdx.x & 48)) & 0xffff) == 0xffff;
    const _Float16 step16 = (_Float16)((most - least) / 15.0f);
    const float step = (float)step16;
    uint32_t codes = 0;
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const float r = step > 0 ? rintf((x[i] - least) / step) : 0.0f; // a step that rounded down makes the last quotient exceed 15
        codes |= (uint32_t)fminf(fmaxf(r, 0.0f), 15.0f) << (4 * i);
    }
    *low = ok ? (_Float16)least : (_Float16)__builtin_nanf("");
    *scale = ok ? step16 : (_Float16)__builtin_nanf("");
    return ok ? codes : 0;
}

// (low, scale) and a code as a value.  A step that rounded up can take the greatest code beyond the range of binary16, whose end it then stands for.
__device__ __forceinline__ float decoded(const _Float16 *p, int code)
{
    const float x = (float)p[0] + (float)p[1] * code;
    return x > 65504.0f ? 65504.0f : x;
}

template <int D> __global__ __launch_bounds__(kThreads) void cache_append_kernel(const AppendArgs a)
{
    typedef CacheLayout<D> L;
    constexpr int V = D / 16;
    const int c = threadIdx.x & 15, G = a.cache.kv_heads, rows = a.heads + 2 * G;
    const int groups = (rows + kRowsPerGroup - 1) / kRowsPerGroup;
    const int64_t items = a.tokens * groups;
    for (int64_t item = blockIdx.x; item < items; item += gridDim.x) {
        const int64_t token = item / groups;
        const int row = (int)(item - token * groups) * kRowsPerGroup + (threadIdx.x >> 4);
        if (row >= rows) continue; // 16 lanes leave together
        const int64_t position = a.rotary ? a.positions[token] : 0;
        float x[V];
        if (row < a.heads) {
            const _Float16 *in = a.q + token * a.q_token + row * a.q_head;
            load_row<V>(in + c * V, x);
            rotate<V>(a, in, c, position, x);
            store_row<V>(a.q_out + token * a.qo_token + row * a.qo_head + c * V, x);
            continue;
        }
        const bool value = row >= a.heads + G;
        const int head = row - a.heads - (value ? G : 0);
        if (value) {
            load_row<V>(a.v + token * a.v_token + head * a.v_head + c * V, x);
        } else {
            const _Float16 *in = a.k + token * a.k_token + head * a.k_head;
            load_row<V>(in + c * V, x);
            rotate<V>(a, in, c, position, x);
#pragma unroll
            for (int i = 0; i < V; ++i) x[i] = (float)(_Float16)x[i];
            if (a.k_out) store_row<V>(a.k_out + token * a.ko_token + head * a.ko_head + c * V, x);
        }
        const int64_t slot = a.slots[token];
        _Float16 low, scale;
        const uint32_t codes = encode<V>(x, &low, &scale);
        const int64_t page = slot >> a.cache.log_page;
        if (slot < 0 || page >= a.cache.pages) continue;
        const int t = (int)(slot & a.page_mask), lp = a.cache.log_page;
        uint8_t *block = L::block(a.cache, page, head);
        if (value) {
#pragma unroll
            for (int h = 0; h < L::kHalves; ++h) *reinterpret_cast<uint16_t *>(block + L::value(lp, t, c, h)) = (uint16_t)(codes >> (16 * h));
        } else if constexpr (V == 8) {
            *reinterpret_cast<uint32_t *>(block + L::key(t) + c * 4) = codes;
        } else {
            *reinterpret_cast<uint16_t *>(block + L::key(t) + c * 2) = (uint16_t)codes;
        }
        if (c == 0) {
            _Float16 *p = reinterpret_cast<_Float16 *>(block + (value ? L::value_scale(lp, t) : L::key_scale(lp, t)));
            p[0] = low;
            p[1] = scale;
        }
    }
}

template <int D>
__global__ __launch_bounds__(kThreads) void cache_read_kernel(const CacheShape cache, const int64_t *slots, int64_t tokens, _Float16 *k, _Float16 *v)
{
    typedef CacheLayout<D> L;
    constexpr int V = D / 16;
    const int c = threadIdx.x & 15, lp = cache.log_page;
    const int64_t rows = tokens * cache.kv_heads;
    for (int64_t row = (int64_t)blockIdx.x * kRowsPerGroup + (threadIdx.x >> 4); row < rows; row += (int64_t)gridDim.x * kRowsPerGroup) {
        const int64_t token = row / cache.kv_heads, slot = slots[token], page = slot >> lp;
        const int head = (int)(row - token * cache.kv_heads), t = (int)(slot & ((1 << lp) - 1));
        float x[V] = {}, y[V] = {};
        if (slot >= 0 && page < cache.pages) {
            const uint8_t *block = L::block(cache, page, head);
            const _Float16 *kp = reinterpret_cast<const _Float16 *>(block + L::key_scale(lp, t));
            const _Float16 *vp = reinterpret_cast<const _Float16 *>(block + L::value_scale(lp, t));
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const int code = block[L::key(t) + (c * V + i) / 2] >> (4 * (i & 1)) & 15;
                const int vcode = *reinterpret_cast<const uint16_t *>(block + L::value(lp, t, c, i / 4)) >> (4 * (i & 3)) & 15;
                x[i] = decoded(kp, code);
                y[i] = decoded(vp, vcode);
            }
        }
        store_row<V>(k + row * D + c * V, x);
        store_row<V>(v + row * D + c * V, y);
    }
}

} // namespace

hipError_t launch_cache_append(const ap_cache &c, const ap_append &a, hipStream_t stream)
{
    AppendArgs k;
    k.cache = cache_shape(c);
    k.q = static_cast<const _Float16 *>(a.q.data);
    k.k = static_cast<const _Float16 *>(a.k.data);
    k.v = static_cast<const _Float16 *>(a.v.data);
    k.q_out = static_cast<_Float16 *>(a.q_out.data);
    k.k_out = static_cast<_Float16 *>(a.k_out.data);
    k.q_token = a.q.token_stride, k.q_head = a.q.head_stride;
    k.k_token = a.k.token_stride, k.k_head = a.k.head_stride;
    k.v_token = a.v.token_stride, k.v_head = a.v.head_stride;
    k.qo_token = a.q_out.token_stride, k.qo_head = a.q_out.head_stride;
    k.ko_token = a.k_out.token_stride, k.ko_head = a.k_out.head_stride;
    k.slots = a.slots, k.positions = a.positions, k.rotary = a.rotary;
    k.rotary_rows = a.rotary_rows, k.tokens = a.tokens;
    k.heads = a.q.data ? a.heads : 0;
    k.rot_dim = a.rot_dim, k.interleaved = a.interleaved;
    k.page_mask = c.page_tokens - 1;
    const int64_t groups = (k.heads + 2 * c.kv_heads + kRowsPerGroup - 1) / kRowsPerGroup, items = a.tokens * groups;
    const dim3 grid((unsigned)(items < (1 << 20) ? items : 1 << 20));
    if (c.head_dim == 64) cache_append_kernel<64><<<grid, kThreads, 0, stream>>>(k);
    else cache_append_kernel<128><<<grid, kThreads, 0, stream>>>(k);
    return hipGetLastError();
}

hipError_t launch_cache_read(const ap_cache &c, const int64_t *slots, int64_t tokens, void *k, void *v, hipStream_t stream)
{
    const int64_t groups = (tokens * c.kv_heads + kRowsPerGroup - 1) / kRowsPerGroup;
    const dim3 grid((unsigned)(groups < (1 << 20) ? groups : 1 << 20));
    if (c.head_dim == 64)
        cache_read_kernel<64><<<grid, kThreads, 0, stream>>>(cache_shape(c), slots, tokens, static_cast<_Float16 *>(k), static_cast<_Float16 *>(v));
    else
        cache_read_kernel<128><<<grid, kThreads, 0, stream>>>(cache_shape(c), slots, tokens, static_cast<_Float16 *>(k), static_cast<_Float16 *>(v));
    return hipGetLastError();
}

} // namespace apgemv
