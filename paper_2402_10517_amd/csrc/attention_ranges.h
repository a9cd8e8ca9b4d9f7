// The kernels of attention over the 4-bit paged cache: ranges of keys for tiles of query rows, and the join of the ranges.  attention_cached.hip says
// how they work; attention_shared.hip launches them with prefixes that sequences share (SHARED).
#ifndef APGEMV_ATTENTION_RANGES_H
#define APGEMV_ATTENTION_RANGES_H

#include <type_traits>

#include "decode_device.h"

namespace apgemv {

namespace {

typedef __bf16 bf8_t __attribute__((ext_vector_type(8)));

struct CachedArgs {
    CacheShape cache;
    const _Float16 *q;
    int64_t q_token, q_head, table_width;
    const int32_t *q_starts, *lengths, *tables;
    int tokens, heads, sequences, max_length;
    int items, splits, chunk; // row tiles (at most), ranges of `chunk` keys
    float scale, slack;
    _Float16 *out;
    float *part;  // splits x rows x D: sums of range s
    float2 *stat; // splits x rows: their maximum and sum of weights
};

constexpr int kThreads = 256;
constexpr int kWaves = 4;
constexpr int kTile = 32;                   // keys per wave and step
constexpr int kStep = kTile * kWaves;       // keys per workgroup and step
constexpr int kPiece = 64 / 2 * kStep;      // keys whose pages a wave holds, those of one 16-key half per lane: 32 steps
constexpr float kCodeUnit = 0x1p-24f;       // a code as the low bits of a binary16 number; scores are in this unit
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kSlack = 8.0f;
// Exponents are fma(score, scale, -rounded product of maximum and scale): off by that rounding, up to 2^-11 of a weight at this size.  From there on the
// maximum is taken from the scores first: at 2^31 the rounding alone would be an exponent of 128.
constexpr float kFar = 0x1p14f;

struct Item {
    int sequence, tile, begin, tokens, length;
};

__device__ __forceinline__ int length_of(const CachedArgs &a, int sequence)
{
    const int length = a.lengths[sequence];
    return length < 0 ? 0 : length > a.max_length ? a.max_length : length;
}

// With prefixes: they are sequences of their own whose query rows are those of all their sequences, each of which sees all keys.  A row's sums of every range are
// kept, the prefix's behind its own, for the join.
struct SharedArgs : CachedArgs {
    const int32_t *prefix_starts, *prefix_lengths, *prefix_tables;
    int64_t prefix_width;
    int prefixes, max_prefix;
    int prefix_items, prefix_splits, prefix_chunk;
    // or the prefixes' rows are in tiles of kTileRows (attention_shared.hip), whose ranges are decided on the device: up to prefix_groups workgroups, whose
    // sums lie behind those of the sequences' own keys
    bool wide;
    int prefix_groups;
    struct Share {
        int first, tiles, ranges; // its first workgroup, tiles of rows, ranges of keys
        int begin, end;           // tokens
        int from, to;             // sequences
        int unused;
    };
    Share *shares; // of each prefix, for the join
};
constexpr int kTileRows = 128;

// The sequence and row tile of an item (64 lanes call together); false: there are fewer.  Where sequences have different numbers of tokens a lane
// looks at one sequence, its length with it.
__device__ __forceinline__ bool find_item(const CachedArgs &a, int rows_per_tile, int item, Item *out)
{
    const int lane = threadIdx.x & 63, group = a.heads / a.cache.kv_heads;
    if (!a.q_starts) {
        const int tiles = a.items / a.sequences, s = item / tiles;
        *out = Item{s, item - s * tiles, s * (a.tokens / a.sequences), a.tokens / a.sequences, length_of(a, s)};
        return true;
    }
    int before = 0;
    Apart apart;
    for (int first = 0; first < a.sequences; first += 64) {
        int length = 0;
        int64_t begin = 0, end = 0;
        bool ok = true;
        if (first + lane < a.sequences) {
            length = length_of(a, first + lane);
            ok = token_range(a.q_starts, first + lane, a.tokens, a.sequences, &begin, &end);
        }
        apart.cut(ok, &begin, &end);
        const int tiles = (int)(((end - begin) * group + rows_per_tile - 1) / rows_per_tile);
        int upto = tiles;
        for (int d = 1; d < 64; d <<= 1) {
            const int other = __shfl_up(upto, d);
            if (lane >= d) upto += other;
        }
        const uint64_t found = __ballot(before + upto > item);
        if (found) {
            const int l = __builtin_ctzll(found);
            *out = Item{first + l, item - before - (__builtin_amdgcn_readlane(upto, l) - __builtin_amdgcn_readlane(tiles, l)),
                        __builtin_amdgcn_readlane((int)begin, l), __builtin_amdgcn_readlane((int)(end - begin), l), __builtin_amdgcn_readlane(length, l)};
            return true;
        }
        before += __builtin_amdgcn_readlane(upto, 63);
    }
    return false;
}

// The sequences [from, to) of a prefix and their tokens [begin, end); none, and false, where starts descend or leave their range
__device__ __forceinline__ bool prefix_tokens(const SharedArgs &a, int p, int64_t *begin, int64_t *end, int64_t *from, int64_t *to)
{
    const bool ok = token_range(a.prefix_starts, p, a.sequences, a.prefixes, from, to);
    int64_t first, last;
    if (a.q_starts) {
        first = a.q_starts[*from], last = a.q_starts[*to]; // up to a.sequences
    } else {
        const int64_t each = a.tokens / a.sequences;
        first = *from * each, last = *to * each;
    }
    const bool some = *from < *to, there = first >= 0 && first <= last && last <= a.tokens;
    *begin = some && there ? first : 0;
    *end = some && there ? last : 0;
    return ok && (there || !some);
}

__device__ __forceinline__ int prefix_length(const SharedArgs &a, int p)
{
    const int length = a.prefix_lengths[p];
    return length < 0 ? 0 : length > a.max_prefix ? a.max_prefix : length;
}

// The prefix and row tile of an item (64 lanes call together); false: there are fewer
__device__ __forceinline__ bool find_prefix_item(const SharedArgs &a, int rows_per_tile, int item, Item *out)
{
    const int lane = threadIdx.x & 63, group = a.heads / a.cache.kv_heads;
    int before = 0;
    Apart apart;
    for (int first = 0; first < a.prefixes; first += 64) {
        int length = 0;
        int64_t begin = 0, end = 0, from, to;
        bool ok = true;
        if (first + lane < a.prefixes) {
            length = prefix_length(a, first + lane);
            ok = prefix_tokens(a, first + lane, &begin, &end, &from, &to);
        }
        if (a.prefix_starts || a.q_starts) apart.cut(ok, &begin, &end);
        const int tiles = (int)(((end - begin) * group + rows_per_tile - 1) / rows_per_tile);
        int upto = tiles;
        for (int d = 1; d < 64; d <<= 1) {
            const int other = __shfl_up(upto, d);
            if (lane >= d) upto += other;
        }
        const uint64_t found = __ballot(before + upto > item);
        if (found) {
            const int l = __builtin_ctzll(found);
            *out = Item{first + l, item - before - (__builtin_amdgcn_readlane(upto, l) - __builtin_amdgcn_readlane(tiles, l)),
                        __builtin_amdgcn_readlane((int)begin, l), __builtin_amdgcn_readlane((int)(end - begin), l), __builtin_amdgcn_readlane(length, l)};
            return true;
        }
        before += __builtin_amdgcn_readlane(upto, 63);
    }
    return false;
}

// Codes and (low, step) pairs of 16 keys as a lane (c = lane % 16, g = lane / 16) needs them: key c's channels g * D/4 .., the values of keys 4 g ..
// 4 g + 3 in channels c * D/16 .., the pairs of those four keys
template <int D> struct Half {
    typedef uint32_t words_t __attribute__((ext_vector_type(D / 32)));
    words_t k, v;
    uint4_t kp, vp;
};

// Byte offsets of a lane in them: from where the codes and where the pairs of the 16 keys start
struct Lane {
    uint32_t k, v, kp, vp;
};

// They are read once: past the caches' usual order.  section: where the (page, key head) starts; t: the first of the 16 keys in it.  Both starts are
// kept in scalar registers.
template <int D> __device__ __forceinline__ Half<D> load_half(const uint8_t *section, int log_page, int t, const Lane &at)
{
    typedef typename Half<D>::words_t words_t;
    uintptr_t codes_at = reinterpret_cast<uintptr_t>(section + t * CacheLayout<D>::kRow), pairs_at = reinterpret_cast<uintptr_t>(section + (D << log_page) + 4 * t);
    asm("" : "+s"(codes_at), "+s"(pairs_at));
    typedef const __attribute__((address_space(1))) uint8_t *global_t; // memory, and not LDS
    const global_t codes = (global_t)codes_at, pairs = (global_t)pairs_at;
    Half<D> h;
    h.k = __builtin_nontemporal_load((const __attribute__((address_space(1))) words_t *)(codes + at.k));
    h.v = __builtin_nontemporal_load((const __attribute__((address_space(1))) words_t *)(codes + at.v));
    h.kp = __builtin_nontemporal_load((const __attribute__((address_space(1))) uint4_t *)(pairs + at.kp));
    h.vp = __builtin_nontemporal_load((const __attribute__((address_space(1))) uint4_t *)(pairs + at.vp));
    return h;
}

__device__ __forceinline__ _Float16 low_of(uint32_t pair) { return __builtin_bit_cast(_Float16, (uint16_t)pair); }
__device__ __forceinline__ _Float16 step_of(uint32_t pair) { return __builtin_bit_cast(_Float16, (uint16_t)(pair >> 16)); }

// A binary16 number times a binary32 one in one mixed-precision instruction
__device__ __forceinline__ float times(_Float16 x, float y) { return __builtin_fmaf((float)x, y, 0.0f); }

// A constant in a vector register: (w & a constant) | it is then one v_and_or_b32, which takes one scalar operand, and w & it needs no literal.  The
// instructions themselves are the compiler's, who knows how far it has to stay from the matrix instruction that reads its result.
__device__ __forceinline__ uint32_t in_vector(uint32_t x)
{
    asm("" : "+v"(x));
    return x;
}

// 8 codes as binary16 code * kCodeUnit, in the order 0 4 1 5 2 6 3 7
__device__ __forceinline__ half8_t key_operand(uint32_t w, uint32_t mask)
{
    return __builtin_bit_cast(half8_t, uint4_t{w & mask, w >> 4 & mask, w >> 8 & mask, w >> 12 & mask});
}

__device__ __forceinline__ uint32_t pack_bf16(float x, float y)
{
    typedef __bf16 bf2_t __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(uint32_t, bf2_t{(__bf16)x, (__bf16)y});
}

// Channel n of four keys of both halves as bfloat16 16 + code
template <int D> __device__ __forceinline__ bf8_t value_operand(const Half<D> (&h)[2], int n, uint32_t mask, uint32_t bits)
{
    constexpr int kH = D / 64;
    uint4_t x;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t w = h[i >> 1].v[(i & 1) * kH + n / 4];
        x[i] = ((n & 3) == 0 ? w << 3 : w >> (4 * (n & 3) - 3)) & mask | bits;
    }
    return __builtin_bit_cast(bf8_t, x);
}

template <bool SHARED> using RangeArgs = std::conditional_t<SHARED, SharedArgs, CachedArgs>;

// The waves' sums of a row tile, where they meet
template <int D> struct RangeSums {
    float sums[kWaves][16][D + 4];
    float4_t stats[kWaves][16];
};

template <int D, int NR, bool SHARED> __device__ __forceinline__ void attend_ranges(const RangeArgs<SHARED> &a, int block, RangeSums<D> &lds)
{
    typedef CacheLayout<D> L;
    constexpr int kSteps = D / 32;    // products of 32 channels per score
    constexpr int kN = D / 16;        // channels of a lane's chunk
    constexpr int kRows = 16 * NR;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), c = lane & 15, g = lane >> 4;
    const int kv = a.cache.kv_heads, group = a.heads / kv;
    const int head = block % kv, rest = block / kv;
    int item, split, chunk = a.chunk, most = a.max_length, range;
    const int32_t *tables = a.tables;
    int64_t width = a.table_width;
    bool whole_prefix = false; // an item of a prefix: every row sees all keys
    if constexpr (SHARED) {
        const int groups = a.wide ? 0 : a.prefix_items * a.prefix_splits; // the prefixes' come first: they are the longest
        whole_prefix = rest < groups;
        const int at = whole_prefix ? rest : rest - groups, items = whole_prefix ? a.prefix_items : a.items;
        item = at % items, split = at / items;
        range = split;
        if (whole_prefix) chunk = a.prefix_chunk, most = a.max_prefix, tables = a.prefix_tables, width = a.prefix_width, range += a.splits;
    } else {
        item = rest % a.items, range = split = rest / a.items;
    }
    Item it;
    if constexpr (SHARED) {
        if (!(whole_prefix ? find_prefix_item(a, kRows, item, &it) : find_item(a, kRows, item, &it))) return;
    } else {
        if (!find_item(a, kRows, item, &it)) return;
    }
    const int sequence = it.sequence, tile = it.tile, begin = it.begin, n = it.tokens, c0 = split * chunk;
    // pages of the wave's keys in a piece, one half of 16 per lane; the first ones are asked for before the length is known
    const auto pages_of = [&](int piece) {
        const int t = piece + kTile * (wave + kWaves * (lane >> 1)) + 16 * (lane & 1);
        return t < most ? tables[(int64_t)sequence * width + (t >> a.cache.log_page)] : -1;
    };
    int pages = pages_of(c0);
    const int length = __builtin_amdgcn_readfirstlane(it.length);
    if ((int64_t)pages >= a.cache.pages) pages = -1;
    // keys that the tile's first and last row see
    const int first_token = tile * kRows / group, last = (tile * kRows + kRows - 1) / group, last_token = last < n ? last : n - 1;
    const int sees_first = whole_prefix ? length : length - n + 1, later = whole_prefix ? 0 : 1; // what token i sees: sees_first + later * i
    const int sees_least = sees_first + later * first_token, sees_most = sees_first + later * last_token;
    if (split > 0 && sees_most <= c0) return;
    const int c1 = sees_most < c0 + chunk ? sees_most : c0 + chunk;

    half8_t q[NR][kSteps];
    float q_sum[NR];
    int sees[NR];
#pragma unroll
    for (int r = 0; r < NR; ++r) {
        const int row = tile * kRows + 16 * r + c, token = row / group, h = row - token * group;
        const bool valid = token < n;
        sees[r] = valid ? sees_first + later * token : 0;
        const _Float16 *p = a.q + (int64_t)(valid ? begin + token : begin) * a.q_token + (int64_t)(head * group + (valid ? h : 0)) * a.q_head + g * (D / 4);
        float sum = 0;
#pragma unroll
        for (int s = 0; s < kSteps; ++s) {
            half8_t x = *reinterpret_cast<const half8_t *>(p + 8 * s);
            if (a.scale < 0) x = -x;
#pragma unroll
            for (int i = 0; i < 8; ++i) sum += (float)x[i];
            q[r][s] = half8_t{x[0], x[4], x[1], x[5], x[2], x[6], x[3], x[7]};
        }
        sum += __shfl_xor(sum, 16);
        sum += __shfl_xor(sum, 32);
        q_sum[r] = sum * kCodeUnit;
    }

    const float scale = fabsf(a.scale) * kLog2e;
    float4_t o[NR][kN], offset[NR]; // offset: 16 sum p step, on every channel
    float m[NR], l[NR], bias[NR];
    bool far[NR]; // scores whose product with the scale is too large to be rounded by itself
    const uint32_t key_mask = in_vector(0x000f000fu), value_mask = 0x00780078u;
    const uint32_t value_bits = in_vector(0x41804180u);
    const uint32_t ones = 0x41804180u; // bfloat16 16
    const bf8_t all = __builtin_bit_cast(bf8_t, uint4_t{ones, ones, ones, ones});
#pragma unroll
    for (int r = 0; r < NR; ++r) {
        m[r] = -INFINITY;
        offset[r] = float4_t{0, 0, 0, 0};
        l[r] = bias[r] = 0;
        far[r] = false;
#pragma unroll
        for (int i = 0; i < kN; ++i) o[r][i] = float4_t{0, 0, 0, 0};
    }

    const int lp = a.cache.log_page, page_mask = (1 << lp) - 1;
    const Lane at{(uint32_t)(c * L::kRow + g * (D / 8)), (uint32_t)((L::kRow << lp) + g * 4 * L::kRow + c * 8 * L::kHalves), (uint32_t)g * 16, (uint32_t)((4 << lp) + g * 16)};
    int piece = c0;
    const auto load = [&](int step, Half<D> (&h)[2]) {
        const int t = piece + kTile * (wave + kWaves * step);
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            const int page = __builtin_amdgcn_readlane(pages, 2 * step + half);
            h[half] = load_half<D>(L::block(a.cache, page < 0 ? 0 : page, head), lp, (t + 16 * half) & page_mask, at);
        }
    };
    Half<D> next[2];
    // A range of more than a piece starts anew in each, a wait for pages and keys in 32 steps.  Only with 32 rows: with 16 the loop around costs short
    // ranges 3 to 5 %, and their sums are few.
    for (;;) {
        const int mine = (NR == 2 && c1 - piece > kPiece ? kPiece : c1 - piece) - kTile * wave, steps = mine > 0 ? (mine + kStep - 1) / kStep : 0;
        if (steps > 0) load(0, next);
#pragma unroll 1
        for (int step = 0; step < steps; ++step) {
            Half<D> h[2] = {next[0], next[1]};
            if (step + 1 < steps) load(step + 1, next);
            const int t0 = piece + kTile * (wave + kWaves * step);
            const bool known0 = __builtin_amdgcn_readlane(pages, 2 * step) >= 0, known1 = __builtin_amdgcn_readlane(pages, 2 * step + 1) >= 0;
            const bool whole = known0 && known1 && t0 + kTile <= sees_least && t0 + kTile <= c1;

            float4_t s[NR][2];
#pragma unroll
            for (int half = 0; half < 2; ++half) {
#pragma unroll
                for (int k = 0; k < kSteps; ++k) {
                    const half8_t x = key_operand(h[half].k[k], key_mask);
#pragma unroll
                    for (int r = 0; r < NR; ++r) s[r][half] = __builtin_amdgcn_mfma_f32_16x16x32_f16(x, q[r][k], k == 0 ? float4_t{0, 0, 0, 0} : s[r][half], 0, 0, 0);
                }
            }
            bf8_t high[NR], low[NR];
#pragma unroll
            for (int r = 0; r < NR; ++r) {
                uint32_t pairs[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const uint32_t kp = h[i >> 2].kp[i & 3];
                    s[r][i >> 2][i & 3] = __builtin_fmaf((float)step_of(kp), s[r][i >> 2][i & 3], times(low_of(kp), q_sum[r]));
                    pairs[i] = h[i >> 2].vp[i & 3];
                }
                if (!whole) {
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const int t = t0 + 16 * (i >> 2) + 4 * g + (i & 3);
                        const bool seen = (i < 4 ? known0 : known1) && t < sees[r] && t < c1;
                        s[r][i >> 2][i & 3] = seen ? s[r][i >> 2][i & 3] : -INFINITY;
                        pairs[i] = seen ? pairs[i] : 0; // keys that are not seen may hold anything
                    }
                }
                float top = s[r][0][0];
#pragma unroll
                for (int i = 1; i < 8; ++i) top = fmaxf(top, s[r][i >> 2][i & 3]);
                if (__any(top - m[r] > a.slack)) { // also from -inf; a sum could round a difference of large scores away
                    top = fmaxf(top, __shfl_xor(top, 16));
                    top = fmaxf(top, __shfl_xor(top, 32));
                    const float next_m = fmaxf(m[r], top), keep = next_m == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f((m[r] - next_m) * scale);
                    m[r] = next_m;
                    far[r] = __any(next_m != -INFINITY && fabsf(next_m) * scale > kFar);
                    l[r] *= keep;
                    bias[r] *= keep;
                    offset[r] *= keep;
#pragma unroll
                    for (int i = 0; i < kN; ++i) o[r][i] *= keep;
                }
                const float from = m[r] == -INFINITY ? 0.0f : m[r];
                float base = from * scale;
                if (far[r]) {
#pragma unroll
                    for (int i = 0; i < 8; ++i) s[r][i >> 2][i & 3] -= from;
                    base = 0.0f;
                }
                uint4_t hi, lo;
#pragma unroll
                for (int i = 0; i < 8; i += 2) {
                    float ps[2];
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        const float p = __builtin_amdgcn_exp2f(__builtin_fmaf(s[r][(i + j) >> 2][(i + j) & 3], scale, -base));
                        l[r] += p;
                        bias[r] = __builtin_fmaf(p, (float)low_of(pairs[i + j]), bias[r]);
                        ps[j] = times(step_of(pairs[i + j]), p);
                    }
                    hi[i / 2] = pack_bf16(ps[0], ps[1]);
                    lo[i / 2] = pack_bf16(ps[0] - __builtin_bit_cast(float, hi[i / 2] << 16), ps[1] - __builtin_bit_cast(float, hi[i / 2] & 0xffff0000u));
                }
                high[r] = __builtin_bit_cast(bf8_t, hi);
                low[r] = __builtin_bit_cast(bf8_t, lo);
            }
#pragma unroll
            for (int r = 0; r < NR; ++r) {
                offset[r] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(all, high[r], offset[r], 0, 0, 0);
                offset[r] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(all, low[r], offset[r], 0, 0, 0);
            }
#pragma unroll
            for (int i = 0; i < kN; ++i) {
                const bf8_t v = value_operand<D>(h, i, value_mask, value_bits);
#pragma unroll
                for (int r = 0; r < NR; ++r) {
                    o[r][i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, high[r], o[r][i], 0, 0, 0);
                    o[r][i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, low[r], o[r][i], 0, 0, 0);
                }
            }
        }
        if (NR == 1 || c1 - piece <= kPiece) break;
        piece += kPiece;
        pages = pages_of(piece);
        if ((int64_t)pages >= a.cache.pages) pages = -1;
    }

    // join the waves: all sums to the common maximum, then every thread takes D / 16 channels of a row
    auto &sums = lds.sums;
    auto &stats = lds.stats;
    const int row_of = threadIdx.x >> 4, chunk_of = threadIdx.x & 15;
#pragma unroll
    for (int r = 0; r < NR; ++r) {
        l[r] += __shfl_xor(l[r], 16);
        l[r] += __shfl_xor(l[r], 32);
        bias[r] += __shfl_xor(bias[r], 16);
        bias[r] += __shfl_xor(bias[r], 32);
        bias[r] -= offset[r][0];
        if (r > 0) __syncthreads();
        if (g == 0) stats[wave][c] = float4_t{m[r], l[r], bias[r], 0};
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int k = 0; k < kN; ++k) sums[wave][c][(4 * g + i) * kN + k] = o[r][k][i];
        __syncthreads();
        float top = -INFINITY;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) top = fmaxf(top, stats[w][row_of][0]);
        float total = 0, x[kN] = {};
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
            const float4_t st = stats[w][row_of];
            // a wave without a finite maximum has seen no key, or only NaN: its sums are 0 or NaN and go in as they are
            const float keep = st[0] == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f((st[0] - top) * scale);
            total += keep * st[1];
#pragma unroll
            for (int k = 0; k < kN; ++k) x[k] += keep * (sums[w][row_of][chunk_of * kN + k] + st[2]);
        }
        const int row = tile * kRows + 16 * r + row_of, token = row / group, h = row - token * group;
        if (token < n) {
            const int64_t at = (int64_t)(begin + token) * a.heads + head * group + h;
            if (!SHARED && length - n + 1 + token <= a.chunk) {
                typedef _Float16 vec __attribute__((ext_vector_type(kN)));
                vec y;
#pragma unroll
                for (int k = 0; k < kN; ++k) y[k] = (_Float16)(total == 0.0f ? 0.0f : x[k] / total);
                if (split == 0) *reinterpret_cast<vec *>(a.out + at * D + chunk_of * kN) = y;
            } else {
                const int64_t place = (int64_t)range * a.tokens * a.heads + at;
#pragma unroll
                for (int k = 0; k < kN; k += 4) *reinterpret_cast<float4_t *>(a.part + place * D + chunk_of * kN + k) = float4_t{x[k], x[k + 1], x[k + 2], x[k + 3]};
                if (chunk_of == 0) a.stat[place] = make_float2(top, total);
            }
        }
    }
}

template <int D, int NR, bool SHARED> __global__ __launch_bounds__(kThreads, NR == 1 ? D == 64 ? 4 : 3 : 2) void attention_cached_kernel(const RangeArgs<SHARED> a)
{
    __shared__ RangeSums<D> lds;
    attend_ranges<D, NR, SHARED>(a, blockIdx.x, lds);
}

// Where the sums of a row's ranges are (64 lanes call together; false: the row has no sequence): its own keys', then its prefix's behind those of all sequences
template <bool WIDE> struct RowRanges {
    int64_t row, rows, at, step;
    int own, all, splits;
    __device__ int64_t place(int i) const // beyond the last any place
    {
        if (WIDE && i >= own) return i < all ? at + (int64_t)(i - own) * step : row;
        return (int64_t)(i < own ? i : i < all ? i - own + splits : 0) * rows + row;
    }
};
// What a lane knows of a prefix: its tokens, its sequences and its keys, or its share as find_part has left it
struct PrefixLane {
    int64_t begin = 0, end = 0, from = 0, to = 0;
    int length = 0;
    bool ok = true;
    __device__ __forceinline__ PrefixLane(const SharedArgs &a, int p)
    {
        if (p >= a.prefixes) return;
        length = prefix_length(a, p);
        ok = prefix_tokens(a, p, &begin, &end, &from, &to);
    }
};
struct ShareLane : SharedArgs::Share {
    __device__ __forceinline__ ShareLane(const SharedArgs &a, int p) : Share{}
    {
        if (p < a.prefixes) static_cast<Share &>(*this) = a.shares[p];
    }
};
template <bool WIDE> __device__ __forceinline__ bool ranges_of_row(const SharedArgs &a, int token, int head, RowRanges<WIDE> *out)
{
    RowRanges<WIDE> r{(int64_t)token * a.heads + head, (int64_t)a.tokens * a.heads, 0, 0, 0, 0, a.splits};
    const int lane = threadIdx.x & 63;
    // the first 64 sequences' numbers and prefixes' are asked for together
    int starts = 0, ends = 0, lengths = 0;
    const auto ask = [&](int first) {
        const int i = first + lane < a.sequences ? first + lane : a.sequences - 1;
        starts = a.q_starts[i], ends = a.q_starts[i + 1], lengths = a.lengths[i];
    };
    if (a.q_starts) ask(0);
    std::conditional_t<WIDE, ShareLane, PrefixLane> prefix(a, lane);
    int s = -1, sees = 0;
    if (!a.q_starts) {
        const int each = a.tokens / a.sequences;
        s = token / each;
        sees = length_of(a, s) - ((s + 1) * each - 1 - token);
    }
    Apart own;
    for (int first = 0; a.q_starts && first < a.sequences; first += 64) {
        if (first > 0) ask(first);
        const bool there = first + lane < a.sequences, ok = starts >= 0 && starts <= ends && ends <= a.tokens;
        int64_t begin = there && ok ? starts : 0, end = there && ok ? ends : 0;
        own.cut(ok || !there, &begin, &end);
        const uint64_t found = __ballot(token >= begin && token < end);
        if (!found) continue;
        const int l = __builtin_ctzll(found), length = __builtin_amdgcn_readlane(lengths, l);
        s = first + l;
        sees = (length < 0 ? 0 : length > a.max_length ? a.max_length : length) - (__builtin_amdgcn_readlane(ends, l) - 1 - token);
        break;
    }
    if (s < 0) return false;
    r.own = r.all = sees > a.chunk ? (sees + a.chunk - 1) / a.chunk : 1; // the first is there even where it holds no key
    Apart apart;
    for (int first = 0; first < a.prefixes; first += 64) {
        if (first > 0) prefix = decltype(prefix)(a, first + lane);
        if constexpr (!WIDE) apart.cut(prefix.ok, &prefix.begin, &prefix.end);
        const uint64_t found = __ballot(token >= prefix.begin && token < prefix.end && s >= prefix.from && s < prefix.to);
        if (!found) continue;
        const int l = __builtin_ctzll(found);
        const auto of = [&](int x) { return __builtin_amdgcn_readlane(x, l); };
        if constexpr (WIDE) {
            const int kv = a.cache.kv_heads, group = a.heads / kv, row = (token - of(prefix.begin)) * group + head % group;
            r.all += of(prefix.ranges);
            r.at = a.splits * r.rows + ((int64_t)of(prefix.first) + (int64_t)(row / kTileRows) * kv + head / group) * kTileRows + row % kTileRows;
            r.step = (int64_t)of(prefix.tiles) * kv * kTileRows;
        } else {
            const int length = of(prefix.length);
            r.all += length > a.prefix_chunk ? (length + a.prefix_chunk - 1) / a.prefix_chunk : 1;
        }
        break;
    }
    *out = r;
    return true;
}

// Joins the ranges of a row that sees more than one: D / 4 lanes take every kParts-th range with a running maximum, and one in kParts of the
// workgroup the rest. The sums are asked for before it is known how many ranges the row has; what is beyond them is dropped.  WIDE: of SharedArgs that say so
template <int D, bool SHARED, bool WIDE = false> __global__ __launch_bounds__(kThreads) void attention_join_kernel(const RangeArgs<SHARED> a)
{
    constexpr int kLanes = D / 4, kParts = kThreads / kLanes;
    const int token = blockIdx.x / a.heads, lane = threadIdx.x % kLanes, part = threadIdx.x / kLanes;
    const int64_t row = blockIdx.x, rows = (int64_t)a.tokens * a.heads;
    const float scale = fabsf(a.scale) * kLog2e;
    int ranges = 0;
    RowRanges<WIDE> found{};
    const auto place_of = [&](int i) {
        if constexpr (SHARED) return found.place(i);
        else return (int64_t)(i < a.splits ? i : 0) * rows + row;
    };
    const auto stat_of = [&](int i) { return a.stat[place_of(i)]; };
    const auto part_of = [&](int i) { return *reinterpret_cast<const float4_t *>(a.part + place_of(i) * D + lane * 4); };
    float2 st;
    float4_t y;
    if constexpr (SHARED) {
        if (!ranges_of_row(a, token, (int)(row - (int64_t)token * a.heads), &found)) return;
        ranges = found.all;
        st = stat_of(part), y = part_of(part);
    } else {
        st = stat_of(part), y = part_of(part);
        const int s = sequence_of(a.q_starts, token, a.tokens, a.sequences);
        if (s < 0) return;
        int64_t begin, end;
        token_range(a.q_starts, s, a.tokens, a.sequences, &begin, &end);
        const int sees = length_of(a, s) - (int)(end - 1 - token);
        if (sees <= a.chunk) return;
        ranges = (sees + a.chunk - 1) / a.chunk;
    }
    float top = -INFINITY, total = 0;
    float4_t x = {0, 0, 0, 0};
    // a range without a finite maximum has no key that the row sees, or only NaN: its sums are 0 or NaN and go in as they are
    const auto keep_of = [&](float from, float to) { return from == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f((from - to) * scale); };
    for (int i = part; i < ranges; i += kParts) {
        const float2 next_st = stat_of(i + kParts);
        const float4_t next_y = part_of(i + kParts);
        const float next = fmaxf(top, st.x), old = keep_of(top, next), keep = keep_of(st.x, next);
        total = total * old + st.y * keep;
        x = x * old + y * keep;
        top = next;
        st = next_st;
        y = next_y;
    }
    __shared__ float4_t sums[kParts][kLanes];
    __shared__ float2 stats[kParts];
    sums[part][lane] = x;
    if (lane == 0) stats[part] = make_float2(top, total);
    __syncthreads();
    if (part > 0) return;
    for (int i = 0; i < kParts; ++i) top = fmaxf(top, stats[i].x);
    x = float4_t{0, 0, 0, 0};
    total = 0;
    for (int i = 0; i < kParts; ++i) {
        const float keep = keep_of(stats[i].x, top);
        x += keep * sums[i][lane];
        total += keep * stats[i].y;
    }
    half4_t out;
#pragma unroll
    for (int k = 0; k < 4; ++k) out[k] = (_Float16)(total == 0.0f ? 0.0f : x[k] / total);
    *reinterpret_cast<half4_t *>(a.out + row * D + lane * 4) = out;
}

} // namespace
} // namespace apgemv
#endif
