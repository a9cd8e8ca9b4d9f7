// Rotation of q and k, append of k and v to the 4-bit cache, and its values read back.
//
// Bound by HBM: rows in, rotated rows and 4-bit codes out, each once. 16 lanes hold a row of head_dim values, so that the least and the greatest of
// it are four exchanges away. 8347 tokens of 64 + 2 x 8 heads take 68 us and their read-back 10 (381 MB in all, 4.8 TB/s; a copy reaches 5.15); a
// single token 4.9 and 2.1, the time of a launch and of three dependent loads.
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
    int parts, rounds; // workgroups per token or 16 adjacent tokens, rows of a group of 16 lanes
};

constexpr int kThreads = 256;
constexpr int kRowsPerGroup = kThreads / 16; // 16 lanes per row of head_dim values
constexpr int kAhead = 4;                    // rows whose loads a group has in flight

template <int V> using halves = _Float16 __attribute__((ext_vector_type(V)));

template <int V> __device__ __forceinline__ void store_row(_Float16 *p, const float (&x)[V])
{
    halves<V> h;
#pragma unroll
    for (int i = 0; i < V; ++i) h[i] = (_Float16)x[i];
    *reinterpret_cast<halves<V> *>(p) = h;
}

// Cosines and sines of the lane's V channels c * V .. at a token's position, for all its rows: of channel i, the sine with the sign it enters with,
// or (interleaved) of channels 2 i, 2 i + 1
template <int V> struct Turn {
    float cosine[V], sine[V];
    bool stays; // channels beyond the rotation: not 1 x + 0 y, which is NaN for an infinity and +0 for -0
    __device__ void load(const AppendArgs &a, int c, int64_t token)
    {
        const int d = c * V, half = a.rot_dim / 2;
        const bool upper = d >= half;
        stays = d >= a.rot_dim;
#pragma unroll
        for (int i = 0; i < V; ++i) cosine[i] = sine[i] = 0;
        if (stays) return;
        const int64_t position = a.positions[token];
        if (position < 0 || position >= a.rotary_rows) {
#pragma unroll
            for (int i = 0; i < V; ++i) cosine[i] = sine[i] = __builtin_nanf("");
            return;
        }
        const float *table = a.rotary + position * a.rot_dim;
        if (a.interleaved) {
            typedef float vec __attribute__((ext_vector_type(V / 2)));
            const vec x = *reinterpret_cast<const vec *>(table + d / 2), y = *reinterpret_cast<const vec *>(table + half + d / 2);
#pragma unroll
            for (int i = 0; i < V / 2; ++i) cosine[i] = x[i], sine[i] = y[i];
        } else {
            table += upper ? d - half : d;
#pragma unroll
            for (int i = 0; i < V; i += 4) {
                const float4_t x = *reinterpret_cast<const float4_t *>(table + i), y = *reinterpret_cast<const float4_t *>(table + half + i);
#pragma unroll
                for (int j = 0; j < 4; ++j) cosine[i + j] = x[j], sine[i + j] = upper ? y[j] : -y[j];
            }
        }
    }
};

enum { kNoTurn, kWholeTurn, kPartTurn, kInterleaved };

// What channel i of the lane turns with: its partner's lane is 8 away in the 16 where the whole row turns, else it is loaded
template <int V, int TURN> __device__ __forceinline__ halves<V> partner(halves<V> own, const _Float16 *row, int across)
{
    if constexpr (TURN == kWholeTurn) {
        typedef int words __attribute__((ext_vector_type(V / 2)));
        words w = __builtin_bit_cast(words, own);
#pragma unroll
        for (int i = 0; i < V / 2; ++i) w[i] = __builtin_amdgcn_mov_dpp(w[i], 0x128, 0xf, 0xf, true); // row_ror:8
        return __builtin_bit_cast(halves<V>, w);
    } else if constexpr (TURN == kPartTurn) {
        return *reinterpret_cast<const halves<V> *>(row + across);
    } else {
        return own;
    }
}

// The lane's V channels of one row, rotated.  Every product and sum is rounded by itself: the codes of the cache jump where a rounded key does, and
// should not depend on which products a compiler fuses with a sum.
template <int V, int TURN> __device__ __forceinline__ void rotate(const Turn<V> &turn, halves<V> own, halves<V> other, float (&x)[V])
{
#pragma clang fp contract(off)
    if constexpr (TURN == kInterleaved) {
#pragma unroll
        for (int i = 0; i < V; i += 2) {
            const float cosine = turn.cosine[i / 2], sine = turn.sine[i / 2], first = (float)own[i], second = (float)own[i + 1];
            x[i] = first * cosine - second * sine;
            x[i + 1] = second * cosine + first * sine;
        }
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i) x[i] = TURN == kNoTurn ? (float)own[i] : (float)own[i] * turn.cosine[i] + (float)other[i] * turn.sine[i];
    }
    if constexpr (TURN == kPartTurn || TURN == kInterleaved) {
#pragma unroll
        for (int i = 0; i < V; ++i) x[i] = turn.stays ? (float)own[i] : x[i];
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
    const float inverse = step > 0 ? 1.0f / step : 0.0f;
    uint32_t codes = 0;
#pragma unroll
    for (int i = 0; i < V; ++i) {
        // the product is within 3e-6 of the quotient (at most 22, where a step of one subnormal unit rounded down): only near the middle between two codes does it take the division
        const float y = (x[i] - least) * inverse;
        float r = rintf(y);
        if (fabsf(fabsf(y - r) - 0.5f) < 1e-5f) r = rintf((x[i] - least) / step);
        codes |= (uint32_t)fminf(r, 15.0f) << (4 * i); // a step that rounded down makes the last quotient exceed 15
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

// Rows of a token are taken by groups of 16 lanes, kAhead at a time.  TOGETHER: the groups of a workgroup are adjacent tokens at the same row, so
// that their codes are whole lines of the cache; else rows of one token.
template <int D, int TURN, bool TOGETHER> __global__ __launch_bounds__(kThreads) void cache_append_kernel(const AppendArgs a)
{
    typedef CacheLayout<D> L;
    constexpr int V = D / 16, kStep = TOGETHER ? 1 : kRowsPerGroup, kTokens = kRowsPerGroup / kStep;
    const int c = threadIdx.x & 15, place = threadIdx.x >> 4, G = a.cache.kv_heads, rows = a.heads + 2 * G, lp = a.cache.log_page;
    const int64_t items = (a.tokens + kTokens - 1) / kTokens * a.parts;
    for (int64_t item = blockIdx.x; item < items; item += gridDim.x) {
        const int64_t block_of = item / a.parts, token = block_of * kTokens + (TOGETHER ? place : 0);
        if (token >= a.tokens) continue; // 16 lanes leave together, here and below
        const int begin = (int)(item - block_of * a.parts) * a.rounds * kStep, stop = begin + a.rounds * kStep, end = stop < rows ? stop : rows;
        const int across = c * V >= a.rot_dim ? 0 : c * V >= a.rot_dim / 2 ? -a.rot_dim / 2 : a.rot_dim / 2;
        const _Float16 *q = a.q + token * a.q_token + c * V, *k = a.k + token * a.k_token + c * V, *v = a.v + token * a.v_token + c * V;
        _Float16 *q_out = a.q_out + token * a.qo_token + c * V, *k_out = a.k_out ? a.k_out + token * a.ko_token + c * V : nullptr;
        const auto source = [&](int row) {
            return row < a.heads ? q + row * a.q_head : row < a.heads + G ? k + (row - a.heads) * a.k_head : v + (row - a.heads - G) * a.v_head;
        };
        const int64_t slot = a.slots[token], page = slot >> lp;
        const bool kept = slot >= 0 && page < a.cache.pages;
        const int t = (int)(slot & a.page_mask);
        Turn<V> turn;
        if (TURN != kNoTurn) turn.load(a, c, token);
        for (int first = begin; first < end; first += kAhead * kStep) {
            halves<V> own[kAhead], other[kAhead];
#pragma unroll
            for (int i = 0; i < kAhead; ++i) {
                const int at = first + i * kStep + (TOGETHER ? 0 : place), row = at < end ? at : end - 1;
                own[i] = *reinterpret_cast<const halves<V> *>(source(row));
                if (TURN == kPartTurn) other[i] = partner<V, TURN>(own[i], source(row), across);
            }
#pragma unroll
            for (int i = 0; i < kAhead; ++i) {
                const int row = first + i * kStep + (TOGETHER ? 0 : place);
                if (row >= end) break;
                if (TURN != kPartTurn) other[i] = partner<V, TURN>(own[i], nullptr, 0);
                float x[V];
                if (row < a.heads) {
                    rotate<V, TURN>(turn, own[i], other[i], x);
                    store_row<V>(q_out + row * a.qo_head, x);
                    continue;
                }
                const bool value = row >= a.heads + G;
                const int head = row - a.heads - (value ? G : 0);
                if (value) {
#pragma unroll
                    for (int j = 0; j < V; ++j) x[j] = (float)own[i][j];
                } else {
                    rotate<V, TURN>(turn, own[i], other[i], x);
#pragma unroll
                    for (int j = 0; j < V; ++j) x[j] = (float)(_Float16)x[j];
                    if (k_out) store_row<V>(k_out + head * a.ko_head, x);
                }
                _Float16 low, scale;
                const uint32_t codes = encode<V>(x, &low, &scale);
                if (!kept) continue;
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
                    const uint32_t pair = __builtin_bit_cast(uint16_t, low) | (uint32_t)__builtin_bit_cast(uint16_t, scale) << 16;
                    *reinterpret_cast<uint32_t *>(block + (value ? L::value_scale(lp, t) : L::key_scale(lp, t))) = pair;
                }
            }
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

template <int D, int TURN> void launch(const AppendArgs &k, bool together, dim3 grid, hipStream_t stream)
{
    if (together) cache_append_kernel<D, TURN, true><<<grid, kThreads, 0, stream>>>(k);
    else cache_append_kernel<D, TURN, false><<<grid, kThreads, 0, stream>>>(k);
}
template <int D> void launch(const AppendArgs &k, int turn, bool together, dim3 grid, hipStream_t stream)
{
    switch (turn) {
    case kNoTurn: launch<D, kNoTurn>(k, together, grid, stream); break;
    case kWholeTurn: launch<D, kWholeTurn>(k, together, grid, stream); break;
    case kPartTurn: launch<D, kPartTurn>(k, together, grid, stream); break;
    default: launch<D, kInterleaved>(k, together, grid, stream);
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
    k.rot_dim = a.rotary ? a.rot_dim : 0, k.interleaved = a.interleaved;
    k.page_mask = c.page_tokens - 1;
    // With many tokens a workgroup takes 16 adjacent ones.  A group of lanes keeps its cosines and sines for up to 8 rows, all in flight at once by
    // fours, where that leaves the card two workgroups per CU.  8347 tokens of 64 + 2 x 8 heads, us with the values read back, at 1 / 2 / 4 / 8 / 10
    // / 16 / 40 rows: 113 / 98 / 82 / 80 / 99 / 90 / 108 (381 MB, 4.8 TB/s at 8).
    const bool together = a.tokens >= 256;
    const int64_t step = together ? 1 : kRowsPerGroup, rows = k.heads + 2 * c.kv_heads, blocks = together ? (a.tokens + kRowsPerGroup - 1) / kRowsPerGroup : a.tokens;
    const int64_t each = (rows + step - 1) / step;
    k.rounds = 1;
    while (k.rounds < 2 * kAhead && blocks * each >= 2 * k.rounds * 512) k.rounds *= 2;
    k.parts = (int)((each + k.rounds - 1) / k.rounds);
    const int64_t items = blocks * k.parts;
    const dim3 grid((unsigned)(items < (1 << 20) ? items : 1 << 20));
    const int turn = !a.rotary ? kNoTurn : a.interleaved ? kInterleaved : a.rot_dim == c.head_dim ? kWholeTurn : kPartTurn;
    if (c.head_dim == 64) launch<64>(k, turn, together, grid, stream);
    else launch<128>(k, turn, together, grid, stream);
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
