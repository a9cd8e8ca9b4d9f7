// Causal attention over packed sequences of binary16 keys and values, on the matrix cores.
//
// A workgroup takes 128 query rows (token, head of the group) of one sequence and key head and walks the keys they see, 64 at a time; a wave has 32
// of the rows.  v_mfma_f32_32x32x16_f16 twice, both transposed:  S^T = K Q^T,  O^T = V^T P^T,  P = e^(scale s - m). With keys as rows and queries as
// columns a lane holds scores of one query row throughout, and the scores' registers, rounded to binary16, are the weights' operand as they stand:
// the order of the keys inside a product is free, and the values are read in the same order from LDS, transposed by ds_read_b64_tr_b16.  Row
// statistics are one number per lane; the running maximum moves only when a score exceeds it by 2^8, so weights stay below 2^8 and the accumulators
// are seldom rescaled. Keys and values go from memory into LDS without registers, 16 bytes a lane, one tile ahead.  Rows of LDS have their 16-byte
// chunks exchanged (the lanes ask memory for the chunk that belongs at their place) so that the reads of both operands meet every bank once.
//
// 4 D operations and one exponential per pair of query and key: bound by the matrix cores and the vector instructions beside them. 8192 tokens of 64
// heads and 8 key heads of 128 take 1.07 to 1.20 ms from card to card, 920 to 1020 TFLOP/s, where a library product of 8192^3 reaches 1177: the matrix
// cores are busy for 54 % of the time and the vector units for 38 %, and the two waves of a SIMD overlap them but little. Two workgroups per CU (212
// registers, 64 KB of LDS); no bank conflicts. Shorter prompts lose to the tiles on the diagonal and to the start of a workgroup: six of up to 2047 tokens
// and 40 heads run at 655 to 670.
//
// The weights are rounded to binary16, and their sum is of the rounded ones: errors of up to 2^-11 each add 1.7e-4 of the result to the 2.0e-4 that its own
// rounding is off by (2.65e-4 together, 8192 tokens).  With a second part of the weights, a second product per value, nothing of that is left, and the
// same tokens take 1.57 ms instead of 1.13, the six prompts 235 us instead of 184, pieces at head_dim 64 63.5 instead of 44.6.
#include "decode_device.h"

namespace apgemv {

namespace {

typedef float float16_t __attribute__((ext_vector_type(16)));
typedef float float2_t __attribute__((ext_vector_type(2)));
typedef _Float16 half2_t __attribute__((ext_vector_type(2)));
typedef __fp16 fp4_t __attribute__((ext_vector_type(4)));

struct PromptArgs {
    const _Float16 *q, *k, *v;
    int64_t q_token, q_head, k_token, k_head, v_token, v_head;
    const int32_t *q_starts, *k_starts;
    int tokens, keys, heads, kv_heads, sequences, items, splits;
    float scale, slack;
    _Float16 *out;
    float *part;  // splits x rows x D: sums of range s
    float2 *stat; // splits x rows: their maximum and sum of weights
};

constexpr int kThreads = 256;
constexpr int kWaveRows = 32;
constexpr int kRows = kWaveRows * kThreads / 64;
constexpr int kKeys = 64; // keys of a tile
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kSlack = 8.0f;
// Weights are 2^7 e^(..): up to 2^15, and above the subnormal numbers of binary16 down to 2^-21 of the greatest
constexpr float kRaise = 7.0f;
constexpr int kLeastTiles = 4;    // of a range of keys
constexpr int64_t kMostRanges = 64;
constexpr int kJoinThreads = 256;
// instruction classes of the scheduler's groups
constexpr int kProducts = 0x8, kLdsReads = 0x100;

// A tile of kKeys rows of D values in LDS.  chunk(row, i): where the 16-byte chunk i of a row is
template <int D> struct Tile {
    static constexpr int kChunks = D / 8;
    static constexpr int kBytes = kKeys * D * 2;
    static constexpr int kLoads = kBytes / (kThreads * 16); // of 16 bytes per lane
    __device__ static int key_chunk(int row, int i) { return D == 128 ? i ^ (row & 15) : i ^ (row >> 1 & 7); }
    __device__ static int value_chunk(int row, int i) { return D == 128 ? i ^ (row & 3) << 2 : i ^ (row >> 1 & 1) << 2; }
};

typedef __attribute__((address_space(3))) uint8_t lds_byte;

// Where a lane's 16-byte pieces of a tile come from in memory, as offsets from the tile's first row
template <int D, bool VALUES> struct Source {
    typedef Tile<D> T;
    const uint8_t *rows;
    uint32_t stride; // bytes
    uint32_t at[T::kLoads];

    // rows beyond the last key are the last's (they are not seen); present: keys from the tile's first on
    __device__ void place(int present, int wave, int lane)
    {
#pragma unroll
        for (int i = 0; i < T::kLoads; ++i) {
            const int row = ((wave * T::kLoads + i) * 64 + lane) / T::kChunks, chunk = VALUES ? T::value_chunk(row, lane % T::kChunks) : T::key_chunk(row, lane % T::kChunks);
            at[i] = (uint32_t)(row < present ? row : present - 1) * stride + chunk * 16;
        }
    }
    // the tile of keys key ..
    __device__ void fetch(int key, int keys, lds_byte *tile, int wave, int lane)
    {
        if (key + kKeys > keys) place(keys - key, wave, lane);
        const uint8_t *from = rows + (int64_t)key * stride;
        const uint32_t to = (uint32_t)(uintptr_t)tile + wave * T::kLoads * 1024;
        // In assembly, as the compiler would have every later read of LDS wait for these loads; the loop waits for them before its barrier.  The
        // s_nop's are the distances from a vector instruction that may have written the scalar operands, and from m0 to its use.
        if constexpr (T::kLoads == 4)
            asm volatile("s_nop 4\n\ts_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %5\n\ts_add_i32 m0, %0, 0x400\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %2, %5\n\t"
                         "s_add_i32 m0, %0, 0x800\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %3, %5\n\ts_add_i32 m0, %0, 0xc00\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %4, %5"
                         :
                         : "s"(to), "v"(at[0]), "v"(at[1]), "v"(at[T::kLoads - 2]), "v"(at[T::kLoads - 1]), "s"(from)
                         : "memory", "m0", "scc");
        else
            asm volatile("s_nop 4\n\ts_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %3\n\ts_add_i32 m0, %0, 0x400\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %2, %3"
                         :
                         : "s"(to), "v"(at[0]), "v"(at[1]), "s"(from)
                         : "memory", "m0", "scc");
    }
};
__device__ __forceinline__ void arrived() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }

// Four keys (4 h .. of 8, from `key`) of channel 32 block + lane % 32, transposed on the way from LDS; at: value_base
template <int D> __device__ __forceinline__ int value_base(int block, int lane)
{
    const int row = 4 * (lane >> 5) + (lane >> 2 & 3), d = block * 32 + (lane & 16) + 4 * (lane & 3);
    return row * D * 2 + Tile<D>::value_chunk(row, d >> 3) * 16 + (d & 4) * 2;
}
template <int D> __device__ __forceinline__ half4_t read_values(const lds_byte *at, int key)
{
    return __builtin_bit_cast(half4_t, __builtin_amdgcn_ds_read_tr16_b64_v4f16((__attribute__((address_space(3))) fp4_t *)(at + key * D * 2)));
}

__device__ __forceinline__ bool finite16(_Float16 x) { return (__builtin_bit_cast(uint16_t, x) & 0x7c00) != 0x7c00; }

__device__ __forceinline__ uint32_t max_halves(uint32_t a, uint32_t b)
{
    typedef uint16_t u2_t __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u2_t, a), __builtin_bit_cast(u2_t, b)));
}

// How the keys that a row tile's last row sees are divided among `splits` workgroups: ranges of whole tiles
struct Range {
    int count, keys;
};
__device__ __forceinline__ Range range_of(int most, int splits)
{
    const int tiles = most > 0 ? (most + kKeys - 1) / kKeys : 1, each = (tiles + splits - 1) / splits, of = each < kLeastTiles ? kLeastTiles : each;
    return Range{(tiles + of - 1) / of, of * kKeys};
}

// Item -> sequence and row tile (64 lanes call together); the items of a sequence come last tile first, its longest
__device__ __forceinline__ bool find_tile(const PromptArgs &a, int item, int *sequence, int *tile)
{
    const int lane = threadIdx.x & 63, group = a.heads / a.kv_heads;
    int before = 0;
    Apart apart;
    for (int first = 0; first < a.sequences; first += 64) {
        int64_t begin = 0, end = 0;
        const bool ok = first + lane >= a.sequences || token_range(a.q_starts, first + lane, a.tokens, a.sequences, &begin, &end);
        apart.cut(ok, &begin, &end);
        const int tiles = (int)(((end - begin) * group + kRows - 1) / kRows);
        int upto = tiles;
        for (int d = 1; d < 64; d <<= 1) {
            const int other = __shfl_up(upto, d);
            if (lane >= d) upto += other;
        }
        const uint64_t found = __ballot(before + upto > item);
        if (found) {
            const int l = __builtin_ctzll(found);
            *sequence = first + l;
            *tile = before + __shfl(upto, l) - 1 - item;
            return true;
        }
        before += __shfl(upto, 63);
    }
    return false;
}

template <int D> __global__ __launch_bounds__(kThreads, D == 64 ? 4 : 2) void attention_prompt_kernel(const PromptArgs a)
{
    typedef Tile<D> T;
    constexpr int kParts = D / 16; // products of 16 channels per score
    constexpr int kBlocks = D / 32; // blocks of 32 channels of the output
    __shared__ __attribute__((aligned(16))) uint8_t tiles[2][2][T::kBytes];
    __shared__ int flags[kThreads / 64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), c = lane & 31, h = lane >> 5;
    const int group = a.heads / a.kv_heads, head = blockIdx.x % a.kv_heads;
    int sequence, tile;
    const int rest = blockIdx.x / a.kv_heads, item = rest % a.items, split = rest / a.items;
    if (!find_tile(a, item, &sequence, &tile)) return;
    sequence = __builtin_amdgcn_readfirstlane(sequence);
    tile = __builtin_amdgcn_readfirstlane(tile);
    int64_t q0, q1, k0, k1;
    token_range(a.q_starts, sequence, a.tokens, a.sequences, &q0, &q1);
    token_range(a.k_starts, sequence, a.keys, a.sequences, &k0, &k1);
    const int n = (int)(q1 - q0), keys = (int)(k1 - k0), ahead = keys - n + 1; // token i sees ahead + i keys

    const int row = tile * kRows + wave * kWaveRows + c, token = row / group;
    const bool valid = token < n;
    const int sees = valid ? ahead + token : 0;
    half8_t q[kParts];
    {
        const _Float16 *p = a.q + (q0 + (valid ? token : 0)) * a.q_token + (int64_t)(head * group + (valid ? row - token * group : 0)) * a.q_head + 8 * h;
#pragma unroll
        for (int i = 0; i < kParts; ++i) {
            q[i] = *reinterpret_cast<const half8_t *>(p + 16 * i);
            if (a.scale < 0) q[i] = -q[i];
        }
    }
    const float scale = fabsf(a.scale) * kLog2e;
    // keys that the workgroup's last row, and the wave's first and last, see
    const auto token_of = [&](int r) { return r / group < n ? r / group : n - 1; };
    const int most = ahead + token_of(tile * kRows + kRows - 1), first_row = tile * kRows + wave * kWaveRows;
    const int wave_least = ahead + token_of(first_row), wave_most = first_row / group < n ? ahead + token_of(first_row + kWaveRows - 1) : 0;

    const Range range = range_of(most, a.splits);
    const int begin = split * range.keys, to = most < begin + range.keys ? most : begin + range.keys;
    if (split >= range.count) return;

    const _Float16 *k = a.k + k0 * a.k_token + head * a.k_head, *v = a.v + k0 * a.v_token + head * a.v_head;
    float16_t o[kBlocks];
#pragma unroll
    for (int i = 0; i < kBlocks; ++i)
#pragma unroll
        for (int j = 0; j < 16; ++j) o[i][j] = 0;
    float m = -INFINITY, l = 0;

    // places in a tile: of the lane's key in the chunks of the products, of its values in the blocks of channels
    int key_at[kParts], value_at[kBlocks];
#pragma unroll
    for (int i = 0; i < kParts; ++i) key_at[i] = c * D * 2 + T::key_chunk(c, 2 * i + h) * 16;
#pragma unroll
    for (int b = 0; b < kBlocks; ++b) value_at[b] = value_base<D>(b, lane);
    lds_byte *const lds = (lds_byte *)&tiles[0][0][0];
    Source<D, false> k_source{reinterpret_cast<const uint8_t *>(k), (uint32_t)a.k_token * 2, {}};
    Source<D, true> v_source{reinterpret_cast<const uint8_t *>(v), (uint32_t)a.v_token * 2, {}};
    k_source.place(kKeys, wave, lane);
    v_source.place(kKeys, wave, lane);
    if (to > begin) {
        k_source.fetch(begin, keys, lds, wave, lane);
        v_source.fetch(begin, keys, lds + T::kBytes, wave, lane);
    }
    const int least = ahead + tile * kRows / group; // what the workgroup's first row sees
#pragma unroll 1
    for (int key = begin, turn = 0; key < to; key += kKeys, turn ^= 1) {
        arrived();
        __syncthreads(); // this tile has arrived, the other one is free
        if (key + kKeys < to) {
            lds_byte *next = lds + (turn ^ 1) * 2 * T::kBytes;
            k_source.fetch(key + kKeys, keys, next, wave, lane);
            v_source.fetch(key + kKeys, keys, next + T::kBytes, wave, lane);
        }
        lds_byte *const kt = lds + turn * 2 * T::kBytes, *const vt = kt + T::kBytes;
        bool odd = false; // a value that is not finite, in a tile that some row does not see whole: 0 * infinity is NaN
        if (key + kKeys > least) {
            uint32_t worst = 0;
#pragma unroll
            for (int i = 0; i < T::kLoads; ++i) {
                const uint4_t x = *(const __attribute__((address_space(3))) uint4_t *)(vt + (i * kThreads + threadIdx.x) * 16);
#pragma unroll
                for (int j = 0; j < 4; ++j) worst = max_halves(worst, x[j] & 0x7fff7fffu);
            }
            const bool bad = __any((worst & 0xffff) >= 0x7c00 || worst >= 0x7c000000u);
            if (lane == 0) flags[wave] = bad;
            __syncthreads();
            odd = flags[0] | flags[1] | flags[2] | flags[3];
            if (odd) { // such values leave the tile and are added to the rows that see them
#pragma unroll
                for (int i = 0; i < T::kLoads; ++i) {
                    __attribute__((address_space(3))) half8_t *x = (__attribute__((address_space(3))) half8_t *)(vt + (i * kThreads + threadIdx.x) * 16);
                    half8_t y = *x;
#pragma unroll
                    for (int j = 0; j < 8; ++j)
                        if (!finite16(y[j])) y[j] = 0;
                    *x = y;
                }
                __syncthreads();
            }
        }
        if (key >= wave_most) continue;
        float16_t s[2];
        __builtin_amdgcn_s_setprio(1);
#pragma unroll
        for (int i = 0; i < kParts; ++i)
#pragma unroll
            for (int b = 0; b < 2; ++b) {
                const half8_t x = *(const __attribute__((address_space(3))) half8_t *)(kt + key_at[i] + b * 32 * D * 2);
                s[b] = __builtin_amdgcn_mfma_f32_32x32x16_f16(x, q[i], i == 0 ? float16_t{} : s[b], 0, 0, 0);
            }
        if constexpr (D == 128) { // operands of the scores six reads ahead; at head_dim 64 four waves per SIMD do better without
            __builtin_amdgcn_sched_group_barrier(kLdsReads, 6, 0);
#pragma unroll
            for (int i = 0; i < 2 * kParts - 6; ++i) {
                __builtin_amdgcn_sched_group_barrier(kProducts, 1, 0);
                __builtin_amdgcn_sched_group_barrier(kLdsReads, 1, 0);
            }
            __builtin_amdgcn_sched_group_barrier(kProducts, 6, 0);
        }
        __builtin_amdgcn_s_setprio(0);
        if (key + kKeys > wave_least) {
            const int seen = sees - key - 4 * h;
#pragma unroll
            for (int b = 0; b < 2; ++b)
#pragma unroll
                for (int j = 0; j < 16; ++j)
                    if (b * 32 + 8 * (j >> 2) + (j & 3) >= seen) s[b][j] = -INFINITY;
        }
        float top = s[0][0];
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
            for (int j = 0; j < 16; ++j) top = fmaxf(top, s[b][j]);
        if (__any(top - m > a.slack)) { // also from -inf; a sum could round a difference of large scores away
            const float next = fmaxf(m, fmaxf(top, __shfl_xor(top, 32))), keep = next == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f((m - next) * scale);
            m = next;
            l *= keep;
#pragma unroll
            for (int i = 0; i < kBlocks; ++i) o[i] *= keep;
        }
        const float from = m == -INFINITY ? 0.0f : m;
        float base = from * scale - kRaise;
        if (__any(fabsf(base) > 0x1p18f)) { // the rounding of the product would take weights past the end of binary16
#pragma unroll
            for (int b = 0; b < 2; ++b)
#pragma unroll
                for (int j = 0; j < 16; ++j) s[b][j] -= from;
            base = -kRaise;
        }
        half8_t p[4];
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int j = 0; j < 8; j += 2) {
                const float2_t x = {__builtin_amdgcn_exp2f(__builtin_fmaf(s[i >> 1][8 * (i & 1) + j], scale, -base)),
                                    __builtin_amdgcn_exp2f(__builtin_fmaf(s[i >> 1][8 * (i & 1) + j + 1], scale, -base))};
                const half2_t y = __builtin_convertvector(x, half2_t);
                l = __builtin_amdgcn_fdot2(y, half2_t{1, 1}, l, false); // the weights as they are used
                p[i][j] = y[0];
                p[i][j + 1] = y[1];
            }
        __builtin_amdgcn_s_setprio(1);
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int b = 0; b < kBlocks; ++b) {
                const half4_t lo = read_values<D>(vt + value_at[b], 16 * i), hi = read_values<D>(vt + value_at[b], 16 * i + 8);
                o[b] = __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7), p[i], o[b], 0, 0, 0);
            }
        // operands of the values 32 keys ahead
        __builtin_amdgcn_sched_group_barrier(kLdsReads, 4 * kBlocks, 0);
#pragma unroll
        for (int i = 0; i < 2 * kBlocks; ++i) {
            __builtin_amdgcn_sched_group_barrier(kProducts, 1, 0);
            __builtin_amdgcn_sched_group_barrier(kLdsReads, 2, 0);
        }
        __builtin_amdgcn_sched_group_barrier(kProducts, 2 * kBlocks, 0);
        __builtin_amdgcn_s_setprio(0);
        if (odd) {
            const _Float16 *row_of = v + key * a.v_token + 4 * h;
            for (int j = 0; j < kKeys && key + j < sees; ++j, row_of += a.v_token) {
#pragma unroll
                for (int b = 0; b < kBlocks; ++b)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const half4_t x = *reinterpret_cast<const half4_t *>(row_of + 32 * b + 8 * i);
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            if (!finite16(x[e])) o[b][4 * i + e] += (float)x[e];
                    }
            }
        }
    }
    l += __shfl_xor(l, 32);
    if (!valid) return;
    const int64_t place = (q0 + token) * a.heads + head * group + (row - token * group);
    if (range.count > 1) {
        float *part = a.part + ((int64_t)split * a.tokens * a.heads + place) * D + 4 * h;
#pragma unroll
        for (int b = 0; b < kBlocks; ++b)
#pragma unroll
            for (int i = 0; i < 4; ++i)
                *reinterpret_cast<float4_t *>(part + 32 * b + 8 * i) = float4_t{o[b][4 * i], o[b][4 * i + 1], o[b][4 * i + 2], o[b][4 * i + 3]};
        if (h == 0) a.stat[(int64_t)split * a.tokens * a.heads + place] = make_float2(m, l);
        return;
    }
    _Float16 *out = a.out + place * D + 4 * h;
    const float scale_out = l == 0.0f ? 0.0f : 1.0f / l;
#pragma unroll
    for (int b = 0; b < kBlocks; ++b)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            half4_t x;
#pragma unroll
            for (int e = 0; e < 4; ++e) x[e] = (_Float16)(l == 0.0f ? 0.0f : o[b][4 * i + e] * scale_out);
            *reinterpret_cast<half4_t *>(out + 32 * b + 8 * i) = x;
        }
}

// Joins the ranges of rows whose tile has more than one: D / 4 lanes a row
template <int D> __global__ __launch_bounds__(kJoinThreads) void attention_prompt_join_kernel(const PromptArgs a)
{
    constexpr int kLanes = D / 4, kEach = kJoinThreads / kLanes;
    const int groups = (a.heads + kEach - 1) / kEach, token = blockIdx.x / groups, lane = threadIdx.x % kLanes, group = a.heads / a.kv_heads;
    const int head = (blockIdx.x - token * groups) * kEach + threadIdx.x / kLanes;
    const int s = sequence_of(a.q_starts, token, a.tokens, a.sequences);
    if (s < 0 || head >= a.heads) return;
    int64_t q0, q1, k0, k1;
    token_range(a.q_starts, s, a.tokens, a.sequences, &q0, &q1);
    token_range(a.k_starts, s, a.keys, a.sequences, &k0, &k1);
    // what the last row of this row's tile sees, as in the kernel above
    const int n = (int)(q1 - q0), row = (int)(token - q0) * group + head % group, last = (row / kRows * kRows + kRows - 1) / group;
    const Range range = range_of((int)(k1 - k0) - n + 1 + (last < n ? last : n - 1), a.splits);
    if (range.count == 1) return;
    const int64_t place = (int64_t)token * a.heads + head, rows = (int64_t)a.tokens * a.heads;
    const float scale = fabsf(a.scale) * kLog2e;
    float top = -INFINITY;
    for (int i = 0; i < range.count; ++i) top = fmaxf(top, a.stat[i * rows + place].x);
    float total = 0;
    float4_t x = {0, 0, 0, 0};
#pragma unroll 4
    for (int i = 0; i < range.count; ++i) {
        const float2 st = a.stat[i * rows + place];
        // a range without a finite maximum has no key that the row sees, or only NaN: its sums are 0 or NaN and go in as they are
        const float keep = st.x == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f((st.x - top) * scale);
        total += keep * st.y;
        x += keep * *reinterpret_cast<const float4_t *>(a.part + (i * rows + place) * D + lane * 4);
    }
    half4_t y;
#pragma unroll
    for (int e = 0; e < 4; ++e) y[e] = (_Float16)(total == 0.0f ? 0.0f : x[e] / total);
    *reinterpret_cast<half4_t *>(a.out + place * D + lane * 4) = y;
}

struct PromptPlan {
    int64_t items;
    int splits;
};

// Row tiles (at most), and the ranges of keys that they are divided into: as many as fill the places that the card has for workgroups (two per CU at
// head_dim 128, four at 64), of four tiles at least and 64 in number at most, where that saves more than it costs: a workgroup takes about 0.9 us for a tile of 64 keys (0.6
// at head_dim 64), the second launch 5 us, and the sums go through memory, written and read, at 4 TB/s.  us without / with ranges: 1 query of 8 heads
// over 4000 keys 72 / 16, 200 of 32 over 8000 141 / 48, 3 x 500 of 16 x 64 over 7500 109 / 74; where the rule keeps to one: 512 of 32 over 512 16 /
// 21, 2000 of 16 x 64 over 2000 32 / 34.  More ranges make the join longer than they make the ranges shorter; us of 1 query of 8 heads and one key head
// with 32 / 64 / 128 / 256 / 512 ranges: 32768 keys 32 / 30 / 41, 65536 50 / 40 / 46 / 75, 131000 85 / 57 / 55 / 80 / 121; heads of 64, 131072 keys 64 / 46
// / 46 / 72 / 128.
PromptPlan plan_of(const ap_prompt &a)
{
    PromptPlan p;
    p.items = a.tokens * (a.heads / a.kv_heads) / kRows + a.sequences;
    const int64_t places = a.head_dim == 64 ? 1024 : 512, units = p.items * a.kv_heads, each = a.keys / a.sequences, room = each / (kKeys * kLeastTiles);
    int64_t splits = places / units;
    splits = splits < room ? splits : room;
    splits = splits < kMostRanges ? splits : kMostRanges;
    if (splits > 1) {
        const double alone = (double)each / kKeys * (a.head_dim == 64 ? 0.6 : 0.9), sums = 2.0 * splits * a.tokens * a.heads * a.head_dim * sizeof(float);
        if (alone * (1.0 - 1.0 / splits) < 5.0 + sums / 4e6) splits = 1;
    }
    p.splits = (int)(splits < 1 ? 1 : splits);
    return p;
}

} // namespace

size_t attention_prompt_work(const ap_prompt &a)
{
    const PromptPlan p = plan_of(a);
    return p.splits == 1 ? 0 : (size_t)p.splits * a.tokens * a.heads * (a.head_dim * sizeof(float) + sizeof(float2));
}

hipError_t launch_attention_prompt(const ap_prompt &a, hipStream_t stream)
{
    PromptArgs k;
    k.q = static_cast<const _Float16 *>(a.q.data);
    k.k = static_cast<const _Float16 *>(a.k.data);
    k.v = static_cast<const _Float16 *>(a.v.data);
    k.q_token = a.q.token_stride, k.q_head = a.q.head_stride;
    k.k_token = a.k.token_stride, k.k_head = a.k.head_stride;
    k.v_token = a.v.token_stride, k.v_head = a.v.head_stride;
    k.tokens = (int)a.tokens, k.keys = (int)a.keys;
    k.q_starts = a.q_starts, k.k_starts = a.k_starts;
    k.heads = a.heads, k.kv_heads = a.kv_heads, k.sequences = a.sequences;
    k.scale = scale_in_range(a.scale);
    k.slack = kSlack / (fabsf(k.scale) * kLog2e);
    k.out = static_cast<_Float16 *>(a.out);
    const PromptPlan p = plan_of(a);
    const int64_t blocks = p.items * a.kv_heads * p.splits; // within kMostGroups: the caller has looked
    k.items = (int)p.items, k.splits = p.splits;
    k.part = static_cast<float *>(a.work);
    k.stat = reinterpret_cast<float2 *>(k.part + (size_t)p.splits * a.tokens * a.heads * a.head_dim);
    if (a.head_dim == 64) attention_prompt_kernel<64><<<dim3((unsigned)blocks), kThreads, 0, stream>>>(k);
    else attention_prompt_kernel<128><<<dim3((unsigned)blocks), kThreads, 0, stream>>>(k);
    if (p.splits > 1) {
        const int each = kJoinThreads / (a.head_dim / 4);
        const dim3 join((unsigned)(a.tokens * ((a.heads + each - 1) / each)));
        if (a.head_dim == 64) attention_prompt_join_kernel<64><<<join, kJoinThreads, 0, stream>>>(k);
        else attention_prompt_join_kernel<128><<<join, kJoinThreads, 0, stream>>>(k);
    }
    return hipGetLastError();
}

} // namespace apgemv
