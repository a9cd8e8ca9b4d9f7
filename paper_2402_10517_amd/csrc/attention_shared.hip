// Attention of new tokens over the 4-bit paged cache where sequences share prefixes.
//
// softmax over a prefix's keys and a sequence's own is joined from ranges of keys: of each the maximum m, the sum l of weights e^(s - m) and the sum o of weighted values;
// out = sum o e^(m - max) / sum l e^(m - max).  The query rows of all sequences of a prefix are one long tile list over its keys, so that a prefix is read once; a
// sequence's own keys are a second list in the same launch.  Both leave (m, l, o) per range, which the second launch joins.
//
// A key of one head is D + 8 bytes and 4 D operations for each row: with hundreds of rows the matrix cores bound it, not HBM.  A tile of 128 rows takes 64 keys a turn,
// prepared once for its four waves.  Two prefixes of up to 65536 keys, 48 sequences of up to 3 tokens, 64 heads and 8 key heads of 128: 272 us (153 GFLOP, 561
// TFLOP/s; of the cycles matrix cores 41 %, a third of that for the second part of the weights, vector instructions 49 %, hardly overlapped), of which the join 9.
// 64 sequences behind 8192 keys with up to 1023 of their own: 51 us, 7 of them the join; 24 sequences with up to 5 tokens behind 3001 keys 18.4, a chain of latencies (start,
// lengths, pages, a turn's 64 keys 1.8 us, sums) twice.
#include "attention_ranges.h"

namespace apgemv {

namespace {

typedef float float16_t __attribute__((ext_vector_type(16)));
typedef float float2_t __attribute__((ext_vector_type(2)));
typedef _Float16 half2_t __attribute__((ext_vector_type(2)));

constexpr int kWaveRows = 32;
static_assert(kTileRows == kWaveRows * kWaves, "query rows of a workgroup");
constexpr int kTileKeys = 64;                 // keys in LDS, 16 from each wave
constexpr int kPageKeys = 64 * 16;            // keys whose pages a wave holds
// The division of the prefixes among workgroups.  Steps (of 64 keys, for a tile of rows and a key head) of a workgroup, at least: us at 1 / 2 / 4, heads of 128,
// 8 key heads: 96 rows over 2000 keys 22.2 / 19.2 / 21.0, 128 over 4096 24.9 / 25.0 / 24.5, over 8192 27.9 / 27.5 / 27.9; heads of 64, 4 key heads: 96 rows over 3000 keys
// 15.5 / 15.4 / 17.6, 3 x 128 over 3000 19.6 each.  2 would be the better for the shortest; 4 halves what the join of these reads at most.
constexpr int kLeastSteps = 4;
// Steps per CU from which on two workgroups for each share it, one at work while the other waits, at the price of twice as many sums.  us with one / two, 16 steps
// (128 rows of 16 prefixes, 2048 keys) 76.1 / 83.2, (256 rows, 16384 keys) 47.7 / 51.0; 32 steps (256 rows, 32768 keys) 75.9 / 73.4, (512, 16384) 78.1 / 77.9;
// 64 steps (512, 32768) 136.9 / 128.7, 128 steps (1024, 32768) 258 / 238.
constexpr int kStepsForTwo = 32;
constexpr int kTried = 16; // prefixes
// Rows (token and head) from which on the join takes a wave for each instead of a workgroup.  us of the whole call with workgroups / waves: 64 rows 18.4 / 20.7 (32768 keys),
// 256 13.8 / 14.0, 512 14.5 / 15.5 and 28.4 / 29.9, 1024 20.7 / 20.2 (1000 keys), 24.9 / 25.0 (4096) and 35.5 / 33.2 (16384), 1920 22.2 / 20.6, 4096 55.2 / 50.3.
constexpr int kRowsForWaves = 1024;
// Weights are 2^7 e^(..): up to 2^15, and above the subnormal numbers of binary16 down to 2^-21 of the greatest.  They go in as two binary16 parts, at twice the products
// for the values: what is left is the rounding of the values, low + step * code, to binary16.  One part, whose roundings are as large as the result's own: relative error
// 3.4e-4 against 2.9e-4 with two and 2.1e-4 of the result's rounding alone (64 sequences behind 8192 keys, heads of 128); 1024 rows over 32768 keys, 8 key heads of 128, 187 us
// against 238.
constexpr float kRaise = 7.0f;
// instruction classes of the scheduler's groups
constexpr int kProducts = 0x8, kLdsReads = 0x100;

// A tile of keys and values in LDS, as operands of v_mfma_f32_32x32x16_f16: 16 bytes per lane (column or row c = lane % 32, half h = lane / 32), in the order of the
// lanes, so that reads meet every bank once.  Keys: per block of 32 keys and part of 16 channels, key c's channels 8 h .. of the part; padded between parts for those
// who write.  Values: per 16 keys and block of 32 channels, channel c of keys 4 h .. and 8 + 4 h ..
template <int D> struct Staged {
    static constexpr int kParts = D / 16, kBlocks = D / 32, kN = D / 16; // kN: channels of a chunk
    static constexpr int kPart = 64 * 16 + 32;
    static constexpr int kKeyBytes = 2 * kParts * kPart, kValueBytes = 4 * kBlocks * 64 * 16;
    static constexpr int kBytes = kKeyBytes + kValueBytes + kTileKeys * 4; // and the keys' (low, step) pairs
    static constexpr int kSums = kTileRows * (D + 4) * 4;                   // the rows' sums, at the end
    __device__ static int key(int block, int part, int h, int c) { return (block * kParts + part) * kPart + (h * 32 + c) * 16; }
    __device__ static int value(int keys16, int block, int h, int c) { return kKeyBytes + ((keys16 * kBlocks + block) * 64 + h * 32 + c) * 16; }
    __device__ static int pair(int t) { return kKeyBytes + kValueBytes + t * 4; }
};

// A barrier for LDS alone: loads from memory stay in flight
__device__ __forceinline__ void lds_barrier()
{
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

// What a wave loads of a tile: 16 keys.  A lane has a quarter of key lane / 4's codes, chunk lane % 16 of the values of quad lane / 16 and that quad's pairs.
template <int D> struct Raw {
    typedef uint32_t words_t __attribute__((ext_vector_type(D / 32)));
    words_t k, v;
    uint4_t vp;
    uint32_t kp; // key lane's, of the first 16 lanes
};

// What a workgroup does: a row tile of a prefix and key head, and a range of its keys
struct Part {
    Item item;
    int head, from, to;
};

// The prefixes' tiles of keys (of 64, for each tile of rows and key head) are divided evenly among the workgroups that the card has room for: what they really hold is known
// on the device alone.  (64 lanes call together.)  The first workgroup leaves for the join how.  False: there is nothing left for this one.
__device__ __forceinline__ bool find_part(const SharedArgs &a, int block, Part *out)
{
    const int lane = threadIdx.x & 63, kv = a.cache.kv_heads, group = a.heads / kv;
    struct Prefix {
        int64_t begin, tokens, from, to;
        int length, tiles, steps;
    };
    const auto prefix_at = [&](int first, Apart &apart) {
        Prefix x{};
        int64_t end = 0;
        bool ok = true;
        if (first + lane < a.prefixes) {
            x.length = prefix_length(a, first + lane);
            ok = prefix_tokens(a, first + lane, &x.begin, &end, &x.from, &x.to);
        }
        apart.cut(ok, &x.begin, &end);
        x.tokens = end - x.begin;
        x.tiles = (int)((x.tokens * group + kTileRows - 1) / kTileRows);
        x.steps = (x.length + kTileKeys - 1) / kTileKeys;
        return x;
    };
    Apart apart, again;
    Prefix x = prefix_at(0, apart);
    int64_t steps = 0, units = 0;
    for (int first = 0; first < a.prefixes; first += 64) {
        if (first > 0) x = prefix_at(first, apart);
        int64_t s = (int64_t)x.tiles * kv * x.steps, u = x.steps > 0 ? (int64_t)x.tiles * kv : 0;
        for (int m = 1; m < 64; m <<= 1) s += __shfl_xor(s, m), u += __shfl_xor(u, m);
        steps += s;
        units += u;
    }
    if (a.prefixes > 64) x = prefix_at(0, again);
    // Each unit's last range may be short: with as many workgroups less there is no second round.  Few prefixes are tried at 64 lengths from there down.
    const int64_t slots = steps >= 256 * kStepsForTwo ? 512 : 256, divided = units < slots / 2 ? slots - units : slots / 2, each = (steps + divided - 1) / divided,
                  all = ((int64_t)a.max_prefix + kTileKeys - 1) / kTileKeys;
    int chunk = (int)(each < kLeastSteps ? kLeastSteps : each > all ? all : each);
    if (a.prefixes <= kTried && chunk > kLeastSteps) {
        const int least = (int)((steps + slots - 1) / slots), from = least < kLeastSteps ? kLeastSteps : least;
        if (from < chunk) {
            const int mine = from + (int)((int64_t)(chunk - from) * lane >> 6);
            int64_t groups = 0;
            for (int i = 0; i < a.prefixes; ++i) groups += (int64_t)__builtin_amdgcn_readlane(x.tiles, i) * kv * ((__builtin_amdgcn_readlane(x.steps, i) + mine - 1) / mine);
            const uint64_t fit = __ballot(groups <= slots);
            if (fit) chunk = __builtin_amdgcn_readlane(mine, __builtin_ctzll(fit));
        }
    }
    int before = 0;
    bool found = false;
    for (int first = 0; first < a.prefixes; first += 64) {
        if (first > 0) x = prefix_at(first, again);
        const int ranges = (x.steps + chunk - 1) / chunk, mine = x.tiles * kv * ranges;
        int upto = mine;
        for (int d = 1; d < 64; d <<= 1) {
            const int other = __shfl_up(upto, d);
            if (lane >= d) upto += other;
        }
        if (block == 0 && threadIdx.x < 64 && first + lane < a.prefixes)
            a.shares[first + lane] = {before + upto - mine, x.tiles, ranges, (int)x.begin, (int)(x.begin + x.tokens), (int)x.from, (int)x.to, 0};
        const uint64_t here = __ballot(before + upto > block);
        if (!found && here) {
            found = true;
            const int l = __builtin_ctzll(here), at = block - before - (__builtin_amdgcn_readlane(upto, l) - __builtin_amdgcn_readlane(mine, l)),
                      tiles = __builtin_amdgcn_readlane(x.tiles, l), rest = at / kv, split = rest / tiles, length = __builtin_amdgcn_readlane(x.length, l);
            out->head = at - rest * kv;
            out->item = Item{first + l, rest - split * tiles, __builtin_amdgcn_readlane((int)x.begin, l), __builtin_amdgcn_readlane((int)x.tokens, l), length};
            out->from = split * chunk * kTileKeys;
            out->to = length - out->from > (int64_t)chunk * kTileKeys ? out->from + chunk * kTileKeys : length;
        }
        before += __builtin_amdgcn_readlane(upto, 63);
    }
    return found;
}

// The keys of a prefix for 128 rows of one key head: codes become operands once for all four waves.
template <int D> __device__ __forceinline__ void attend_prefix(const SharedArgs &a, int block, uint8_t *lds)
{
    typedef CacheLayout<D> L;
    typedef Staged<D> T;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), c = lane & 31, h = lane >> 5;
    Part part;
    if (!find_part(a, block, &part)) return;
    const Item it = part.item;
    const int group = a.heads / a.cache.kv_heads, head = __builtin_amdgcn_readfirstlane(part.head), prefix = it.sequence, n = it.tokens,
              c0 = __builtin_amdgcn_readfirstlane(part.from), c1 = __builtin_amdgcn_readfirstlane(part.to);

    const int row = it.tile * kTileRows + wave * kWaveRows + c, token = row / group;
    const bool valid = token < n;
    half8_t q[T::kParts];
    float q_sum = 0;
    {
        const _Float16 *p = a.q + (int64_t)(it.begin + (valid ? token : 0)) * a.q_token + (int64_t)(head * group + (valid ? row - token * group : 0)) * a.q_head + 8 * h;
#pragma unroll
        for (int i = 0; i < T::kParts; ++i) {
            half8_t x = *reinterpret_cast<const half8_t *>(p + 16 * i);
            if (a.scale < 0) x = -x;
#pragma unroll
            for (int j = 0; j < 8; ++j) q_sum += (float)x[j];
            q[i] = half8_t{x[0], x[4], x[1], x[5], x[2], x[6], x[3], x[7]}; // the order that codes come in
        }
        q_sum += __shfl_xor(q_sum, 32);
        q_sum *= kCodeUnit;
    }
    const float scale = fabsf(a.scale) * kLog2e;
    float16_t o[T::kBlocks];
#pragma unroll
    for (int b = 0; b < T::kBlocks; ++b)
#pragma unroll
        for (int j = 0; j < 16; ++j) o[b][j] = 0;
    float m = -INFINITY, l = 0;

    // pages of 16 keys each, from `piece` on, and of the next piece
    const auto pages_of = [&](int from) {
        const int t = from + 16 * lane;
        const int page = t < c1 ? a.prefix_tables[(int64_t)prefix * a.prefix_width + (t >> a.cache.log_page)] : -1;
        return (int64_t)page < a.cache.pages ? page : -1;
    };
    int piece = c0, pages = pages_of(c0), later = pages_of(c0 + kPageKeys);
    const int lp = a.cache.log_page, page_mask = (1 << lp) - 1;
    // the tile's 16 keys of the wave; which of its four 16 keys are in the cache
    const auto load = [&](int key, int *known) {
        if (key - piece == kPageKeys) {
            piece = key;
            pages = later;
            later = pages_of(piece + kPageKeys);
        }
        const int at = (key - piece) >> 4;
        *known = (int)(__ballot(pages >= 0) >> at) & 15;
        const int page = __builtin_amdgcn_readlane(pages, at + wave), t = (key + 16 * wave) & page_mask;
        const uint8_t *section = L::block(a.cache, page < 0 ? 0 : page, head);
        uintptr_t codes_at = reinterpret_cast<uintptr_t>(section + t * L::kRow), pairs_at = reinterpret_cast<uintptr_t>(section + (D << lp) + 4 * t);
        asm("" : "+s"(codes_at), "+s"(pairs_at));
        typedef const __attribute__((address_space(1))) uint8_t *global_t;
        typedef typename Raw<D>::words_t words_t;
        const global_t codes = (global_t)codes_at, pairs = (global_t)pairs_at;
        Raw<D> r;
        r.k = *(const __attribute__((address_space(1))) words_t *)(codes + lane * (D / 8));
        r.v = *(const __attribute__((address_space(1))) words_t *)(codes + (L::kRow << lp) + lane * (D / 8));
        r.vp = *(const __attribute__((address_space(1))) uint4_t *)(pairs + (4 << lp) + (lane >> 4) * 16);
        r.kp = *(const __attribute__((address_space(1))) uint32_t *)(pairs + (lane & 15) * 4);
        return r;
    };
    const uint32_t key_mask = in_vector(0x000f000fu), value_bits = in_vector(0x64006400u);
    // The lanes take the channels of their chunks in different orders, n ^ turned for n = 0, 1, ..: their writes then meet every bank equally often
    const int turned = (lane & 15) / (D == 128 ? 2 : 4);
    int shifts[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) shifts[i] = 4 * (i ^ (turned & 3));
    const auto stage = [&](uint8_t *to, const Raw<D> &r, int key, int known) {
        const int of = lane >> 2, quarter = lane & 3;
#pragma unroll
        for (int j = 0; j < D / 32; ++j) {
            const int eight = quarter * (D / 32) + j;
            *reinterpret_cast<half8_t *>(to + T::key(wave >> 1, eight >> 1, eight & 1, (wave & 1) * 16 + of)) = key_operand(r.k[j], key_mask);
        }
        if (lane < 16) *reinterpret_cast<uint32_t *>(to + T::pair(16 * wave + lane)) = r.kp;
        // values: low + step * code rounded once; 0 for keys that are not there
        const int quad = lane >> 4, chunk = lane & 15, first = key + 16 * wave + 4 * quad;
        uint4_t pairs = r.vp;
        if (known != 15 || key + kTileKeys > c1) {
            int end = c1 - first, in = known >> wave & 1;
            asm volatile("" : "+v"(end), "+s"(in)); // stays a branch: the compiler would select in every turn
#pragma unroll
            for (int i = 0; i < 4; ++i) pairs[i] = in && i < end ? pairs[i] : 0;
        }
        half2_t low[2], step[2], last[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            low[i] = half2_t{low_of(pairs[2 * i]), low_of(pairs[2 * i + 1])};
            step[i] = half2_t{step_of(pairs[2 * i]), step_of(pairs[2 * i + 1])};
            last[i] = __builtin_elementwise_fma(half2_t{15, 15}, step[i], low[i]);
        }
        const half2_t most = __builtin_elementwise_max(last[0], last[1]);
        const bool over = most[0] > (_Float16)65504 || most[1] > (_Float16)65504;
        constexpr int kH = D / 64;
        const int at = T::value(wave, chunk / (512 / D), quad & 1, chunk % (512 / D) * T::kN + turned) + (quad >> 1) * 8;
        uint32_t words[2][kH];
#pragma unroll
        for (int p = 0; p < 2; ++p) {
            if constexpr (kH == 2) {
                words[p][0] = turned & 4 ? r.v[2 * p + 1] : r.v[2 * p];
                words[p][1] = turned & 4 ? r.v[2 * p] : r.v[2 * p + 1];
            } else {
                words[p][0] = r.v[p];
            }
        }
        const auto values = [&](const auto &last) {
#pragma unroll
            for (int i = 0; i < T::kN; ++i) {
                uint2_t x;
#pragma unroll
                for (int p = 0; p < 2; ++p) {
                    const half2_t code = __builtin_bit_cast(half2_t, words[p][i / 4] >> shifts[i & 3] & key_mask | value_bits) - half2_t{1024, 1024};
                    x[p] = __builtin_bit_cast(uint32_t, last(__builtin_elementwise_fma(code, step[p], low[p])));
                }
                *reinterpret_cast<uint2_t *>(to + (at ^ 16 * i)) = x;
            }
        };
        if (__any(over)) { // 15 steps may pass the end of binary16 by the rounding of the step
            asm volatile(""); // stays a branch: the compiler would take the greater of each value and its end, always
            values([](half2_t y) {
#pragma unroll
                for (int e = 0; e < 2; ++e) y[e] = y[e] > (_Float16)65504 ? (_Float16)65504 : y[e];
                return y;
            });
        } else {
            values([](half2_t y) { return y; });
        }
    };

    // Memory is asked for a tile two turns before its products, which leaves a turn for it to arrive; its codes become operands in the turn before, behind the
    // products of the scores.  Behind the last tile it is asked for nothing new: what is loaded is not used.
    int known = 0, next_known = 0;
    Raw<D> r;
    if (c0 < c1) {
        r = load(c0, &known);
        stage(lds, r, c0, known);
        r = load(c0 + kTileKeys, &next_known);
    }
#pragma unroll 1
    for (int key = c0, turn = 0; key < c1; key += kTileKeys, turn ^= 1) {
        lds_barrier(); // this tile is there, the other one is free
        const uint8_t *const tile = lds + turn * T::kBytes;
        float16_t s[2];
#pragma unroll
        for (int i = 0; i < T::kParts; ++i)
#pragma unroll
            for (int b = 0; b < 2; ++b) {
                const half8_t x = *reinterpret_cast<const half8_t *>(tile + T::key(b, i, h, c));
                s[b] = __builtin_amdgcn_mfma_f32_32x32x16_f16(x, q[i], i == 0 ? float16_t{} : s[b], 0, 0, 0);
            }
        // operands kAhead reads ahead of their products
        constexpr int kAhead = 6;
        __builtin_amdgcn_sched_group_barrier(kLdsReads, kAhead, 0);
#pragma unroll
        for (int i = 0; i < 2 * T::kParts - kAhead; ++i) {
            __builtin_amdgcn_sched_group_barrier(kProducts, 1, 0);
            __builtin_amdgcn_sched_group_barrier(kLdsReads, 1, 0);
        }
        __builtin_amdgcn_sched_group_barrier(kProducts, kAhead, 0);
        const int now = known;
        stage(lds + (turn ^ 1) * T::kBytes, r, key + kTileKeys, next_known);
        known = next_known;
        r = load(key + 2 * kTileKeys, &next_known);
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const uint4_t pairs = *reinterpret_cast<const uint4_t *>(tile + T::pair(32 * b + 8 * g + 4 * h));
#pragma unroll
                for (int e = 0; e < 4; ++e) s[b][4 * g + e] = __builtin_fmaf((float)step_of(pairs[e]), s[b][4 * g + e], times(low_of(pairs[e]), q_sum));
            }
        if (now != 15 || key + kTileKeys > c1) {
            int end = c1 - key - 4 * h, there = now;
            asm volatile("" : "+v"(end), "+s"(there)); // and so stays a branch
#pragma unroll
            for (int b = 0; b < 2; ++b)
#pragma unroll
                for (int g = 0; g < 4; ++g)
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if (!(there >> (2 * b + (g >> 1)) & 1) || 32 * b + 8 * g + e >= end) s[b][4 * g + e] = -INFINITY;
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
            for (int b = 0; b < T::kBlocks; ++b) o[b] *= keep;
        }
        const float from = m == -INFINITY ? 0.0f : m;
        float base = from * scale - kRaise;
        if (__any(fabsf(base) > kFar)) { // the rounding of the product would be part of the exponent
#pragma unroll
            for (int b = 0; b < 2; ++b)
#pragma unroll
                for (int j = 0; j < 16; ++j) s[b][j] -= from;
            base = -kRaise;
        }
        half8_t p[4], rest[4];
        float minus = -1.0f;
        asm("" : "+v"(minus)); // for a sum that takes a binary16 number as it is
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int j = 0; j < 8; j += 2) {
                const float2_t x = {__builtin_amdgcn_exp2f(__builtin_fmaf(s[i >> 1][8 * (i & 1) + j], scale, -base)),
                                    __builtin_amdgcn_exp2f(__builtin_fmaf(s[i >> 1][8 * (i & 1) + j + 1], scale, -base))};
                const half2_t y = __builtin_convertvector(x, half2_t);
                const half2_t z = __builtin_convertvector(float2_t{__builtin_fmaf((float)y[0], minus, x[0]), __builtin_fmaf((float)y[1], minus, x[1])}, half2_t);
                l = __builtin_amdgcn_fdot2(z, half2_t{1, 1}, __builtin_amdgcn_fdot2(y, half2_t{1, 1}, l, false), false); // the weights as they are used
                p[i][j] = y[0];
                p[i][j + 1] = y[1];
                rest[i][j] = z[0];
                rest[i][j + 1] = z[1];
            }
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int b = 0; b < T::kBlocks; ++b) {
                const half8_t x = *reinterpret_cast<const half8_t *>(tile + T::value(i, b, h, c));
                o[b] = __builtin_amdgcn_mfma_f32_32x32x16_f16(x, p[i], o[b], 0, 0, 0);
                o[b] = __builtin_amdgcn_mfma_f32_32x32x16_f16(x, rest[i], o[b], 0, 0, 0);
            }
        __builtin_amdgcn_sched_group_barrier(kLdsReads, kAhead, 0);
#pragma unroll
        for (int i = 0; i < 4 * T::kBlocks - kAhead; ++i) {
            __builtin_amdgcn_sched_group_barrier(kProducts, 2, 0);
            __builtin_amdgcn_sched_group_barrier(kLdsReads, 1, 0);
        }
        __builtin_amdgcn_sched_group_barrier(kProducts, 2 * kAhead, 0);
    }

    // the rows' sums, in whole lines: through LDS, a wave its own rows
    constexpr float kLower = 0.0078125f; // 2^-kRaise
    l = (l + __shfl_xor(l, 32)) * kLower;
    __syncthreads();
    float *const sums = reinterpret_cast<float *>(lds) + wave * kWaveRows * (D + 4);
#pragma unroll
    for (int b = 0; b < T::kBlocks; ++b)
#pragma unroll
        for (int g = 0; g < 4; ++g)
            *reinterpret_cast<float4_t *>(sums + c * (D + 4) + 32 * b + 8 * g + 4 * h) = float4_t{o[b][4 * g], o[b][4 * g + 1], o[b][4 * g + 2], o[b][4 * g + 3]} * kLower;
    const int64_t place = (int64_t)a.splits * a.tokens * a.heads + (int64_t)block * kTileRows + wave * kWaveRows;
    if (h == 0) a.stat[place + c] = make_float2(m, l);
    __syncthreads();
    // rows that are not there as well: the join does not look at them
#pragma unroll 4
    for (int i = 0; i < kWaveRows * D / 256; ++i) {
        const int at = i * 64 + lane, r = at / (D / 4), channel = at % (D / 4) * 4;
        *reinterpret_cast<float4_t *>(a.part + (place + r) * D + channel) = *reinterpret_cast<const float4_t *>(sums + r * (D + 4) + channel);
    }
}

// Both: workgroups of prefixes, then of the sequences' own keys, which wait for memory where the others wait for the matrix cores
template <int D, int NR> __global__ __launch_bounds__(kThreads, 2) void attention_shared_kernel(const SharedArgs a)
{
    constexpr int kPrefix = 2 * Staged<D>::kBytes > Staged<D>::kSums ? 2 * Staged<D>::kBytes : Staged<D>::kSums, kOwn = sizeof(RangeSums<D>);
    __shared__ __attribute__((aligned(16))) uint8_t lds[kPrefix > kOwn ? kPrefix : kOwn];
    if ((int)blockIdx.x < a.prefix_groups) attend_prefix<D>(a, blockIdx.x, lds);
    else attend_ranges<D, NR, true>(a, blockIdx.x - a.prefix_groups, *reinterpret_cast<RangeSums<D> *>(lds));
}

// The join where rows are many and their ranges few: a wave for a row, whose ranges go to its 64 / (D / 4) parts, kAtOnce of each asked for at once.
template <int D, bool WIDE> __global__ __launch_bounds__(kThreads) void join_rows_kernel(const SharedArgs a)
{
    constexpr int kLanes = D / 4, kParts = 64 / kLanes, kAtOnce = 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & (kLanes - 1), part = (threadIdx.x & 63) / kLanes;
    const int64_t row = (int64_t)blockIdx.x * kWaves + wave;
    if (row >= (int64_t)a.tokens * a.heads) return;
    const int token = (int)row / a.heads;
    RowRanges<WIDE> r;
    if (!ranges_of_row(a, token, (int)row - token * a.heads, &r)) return;
    const float scale = fabsf(a.scale) * kLog2e;
    // a range without a finite maximum has no key that the row sees, or only NaN: its sums are 0 or NaN and go in as they are
    const auto keep_of = [&](float from, float to) { return from == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f((from - to) * scale); };
    float top = -INFINITY, total = 0;
    float4_t x = {0, 0, 0, 0};
    for (int first = part; first - part < r.all; first += kAtOnce * kParts) {
        float2 st[kAtOnce];
        float4_t y[kAtOnce];
#pragma unroll
        for (int j = 0; j < kAtOnce; ++j) {
            const int64_t place = r.place(first + j * kParts);
            st[j] = a.stat[place];
            y[j] = *reinterpret_cast<const float4_t *>(a.part + place * D + lane * 4);
        }
#pragma unroll
        for (int j = 0; j < kAtOnce; ++j)
            if (first + j * kParts < r.all) {
                const float next = fmaxf(top, st[j].x), old = keep_of(top, next), keep = keep_of(st[j].x, next);
                total = total * old + st[j].y * keep;
                x = x * old + y[j] * keep;
                top = next;
            }
    }
#pragma unroll
    for (int m = kLanes; m < 64; m <<= 1) {
        const float other = __shfl_xor(top, m), next = fmaxf(top, other), keep = keep_of(top, next), keep_other = keep_of(other, next);
        total = total * keep + __shfl_xor(total, m) * keep_other;
#pragma unroll
        for (int k = 0; k < 4; ++k) x[k] = x[k] * keep + __shfl_xor(x[k], m) * keep_other;
        top = next;
    }
    half4_t out;
#pragma unroll
    for (int k = 0; k < 4; ++k) out[k] = (_Float16)(total == 0.0f ? 0.0f : x[k] / total);
    if (part == 0) *reinterpret_cast<half4_t *>(a.out + row * D + lane * 4) = out;
}

struct Plan {
    int rows;  // 16-row tiles per workgroup
    bool wide; // a prefix's rows in tiles of 128
    int64_t items, prefix_items = 0;
    int chunk, prefix_chunk = 0, splits, prefix_splits = 0;
    int64_t prefix_groups;
    int64_t sums(const ap_shared &a) const // rows' sums in the workspace
    {
        return (int64_t)(splits + prefix_splits) * a.own.tokens * a.own.heads + prefix_groups * kTileRows;
    }
};

Plan plan_of(const ap_cache &c, const ap_shared &a)
{
    Plan p;
    const ap_cached &o = a.own;
    const int64_t group = o.heads / c.kv_heads, each = (o.tokens + o.sequences - 1) / o.sequences, longest = o.max_length > 0 ? o.max_length : 1,
                  longest_prefix = a.max_prefix > 0 ? a.max_prefix : 1, most = longest > longest_prefix ? longest : longest_prefix;
    const auto items_of = [&](int64_t tile) { return o.q_starts ? o.tokens * group / tile + o.sequences : (each * group + tile - 1) / tile * o.sequences; };
    const auto prefix_items_of = [&](int64_t tile) { return a.prefixes > 0 ? o.tokens * group / tile + a.prefixes : 0; };
    const int64_t prefix_rows = a.prefixes > 0 ? (o.tokens + a.prefixes - 1) / a.prefixes * group : 0;
    const auto round_up = [](int64_t x, int64_t to) { return (int)((x + to - 1) / to * to); };
    // Tiles of 128 rows read and prepare a key once where the others do so for every 32 rows, and wait longer before their first.  us with tiles of 32 / 128, 8 key
    // heads of 128: 48 rows over 2000 keys 14.0 / 19.9, over 32768 33.2 / 45.2, 64 over 1000 13.6 / 19.3, over 8192 22.1 / 24.5, 128 over 8192 27.6 / 27.6, over 32768
    // 56.7 / 47.1, 256 over 8192 36.8 / 34.6, over 32768 89.2 / 74.1, 1024 over 1000 43.0 / 36.1, over 8192 91.9 / 85.8; 4 key heads of 64: 3 x 96 over 3000 20.3 / 18.4, 256 over
    // 8192 22.3 / 20.9, 1024 52.2 / 40.6.  The rule is by rows alone and does not meet the crossing, which depends on the keys too: above it tiles of 32 are ahead at 72 rows (over
    // 1000 keys 14.0 / 19.7, over 8192 22.6 / 25.3), 96 over 2000 (15.4 / 21.0), 128 and 256 over 1000 (15.3 / 19.8, 17.5 / 21.6; heads of 64 13.0 / 17.4).
    p.wide = prefix_rows > 64;
    if (p.wide) {
        p.rows = each * group <= 16 && longest / kPiece * items_of(16) * c.kv_heads < 1 << 20 ? 1 : 2;
        p.items = items_of(16 * p.rows);
        const int64_t units = p.items * c.kv_heads;
        int64_t chunk = (longest * units + 511) / 512;
        if (p.rows == 1 && chunk > kPiece) chunk = kPiece;
        chunk = chunk < 2 * kStep ? 2 * kStep : chunk;
        p.chunk = round_up(chunk < longest ? chunk : longest, kStep);
        p.splits = (int)((longest + p.chunk - 1) / p.chunk);
        // at most as many workgroups as find_part divides the prefixes among: slots, and a short range of each row tile and key head
        const int64_t prefix_units = prefix_items_of(kTileRows) * c.kv_heads, ranges = (longest_prefix + kLeastSteps * kTileKeys - 1) / (kLeastSteps * kTileKeys);
        p.prefix_groups = ranges * prefix_units < 512 + prefix_units ? ranges * prefix_units : 512 + prefix_units;
        return p;
    }
    p.prefix_groups = 0;
    p.rows = each * group <= 16 && prefix_rows <= 16 && most / kPiece * (items_of(16) + prefix_items_of(16)) * c.kv_heads < 1 << 20 ? 1 : 2;
    p.items = items_of(16 * p.rows);
    p.prefix_items = prefix_items_of(16 * p.rows);
    // Ranges of keys of the same length for both, so that there are two workgroups per CU in all
    const int64_t keys = (longest * p.items + longest_prefix * p.prefix_items) * c.kv_heads;
    int64_t chunk = (keys + 511) / 512;
    if (p.rows == 1 && chunk > kPiece) chunk = kPiece;
    if (chunk < 2 * kStep) chunk = 2 * kStep;
    p.chunk = round_up(chunk < longest ? chunk : longest, kStep);
    p.prefix_chunk = round_up(chunk < longest_prefix ? chunk : longest_prefix, kStep);
    p.splits = (int)((longest + p.chunk - 1) / p.chunk);
    p.prefix_splits = a.prefixes > 0 ? (int)((longest_prefix + p.prefix_chunk - 1) / p.prefix_chunk) : 0;
    return p;
}

} // namespace

size_t attention_shared_work(const ap_cache &c, const ap_shared &a)
{
    const Plan p = plan_of(c, a);
    return (size_t)p.sums(a) * (c.head_dim * sizeof(float) + sizeof(float2)) + (p.wide ? a.prefixes * sizeof(SharedArgs::Share) + 32 : 0);
}

hipError_t launch_attention_shared(const ap_cache &c, const ap_shared &a, hipStream_t stream)
{
    const Plan p = plan_of(c, a);
    const ap_cached &o = a.own;
    SharedArgs k;
    k.cache = cache_shape(c);
    k.q = static_cast<const _Float16 *>(o.q.data);
    k.q_token = o.q.token_stride, k.q_head = o.q.head_stride;
    k.table_width = o.table_width;
    k.q_starts = o.q_starts, k.lengths = o.lengths, k.tables = o.tables;
    k.tokens = (int)o.tokens, k.heads = o.heads, k.sequences = o.sequences, k.max_length = (int)o.max_length;
    k.items = (int)p.items, k.splits = p.splits, k.chunk = p.chunk;
    k.scale = scale_in_range(o.scale) / kCodeUnit;
    k.slack = kSlack / (fabsf(k.scale) * kLog2e);
    k.out = static_cast<_Float16 *>(o.out);
    k.part = static_cast<float *>(o.work);
    k.stat = reinterpret_cast<float2 *>(k.part + p.sums(a) * c.head_dim);
    k.shares = reinterpret_cast<SharedArgs::Share *>((reinterpret_cast<uintptr_t>(k.stat + p.sums(a)) + 31) & ~(uintptr_t)31);
    k.prefix_starts = a.prefix_starts, k.prefix_lengths = a.prefix_lengths, k.prefix_tables = a.prefix_tables;
    k.prefix_width = a.prefix_width;
    k.prefixes = a.prefixes, k.max_prefix = (int)a.max_prefix;
    k.prefix_items = (int)p.prefix_items, k.prefix_splits = p.prefix_splits, k.prefix_chunk = p.prefix_chunk;
    k.wide = p.wide, k.prefix_groups = (int)p.prefix_groups;
    const dim3 grid((unsigned)((p.items * p.splits + p.prefix_items * p.prefix_splits) * c.kv_heads + p.prefix_groups));
    const int64_t rows = o.tokens * o.heads;
    const bool waves = rows >= kRowsForWaves;
    const dim3 join((unsigned)(waves ? (rows + kWaves - 1) / kWaves : rows));
    const auto launch = [&](auto narrow, auto wide) {
        if (p.wide) wide<<<grid, kThreads, 0, stream>>>(k);
        else narrow<<<grid, kThreads, 0, stream>>>(k);
    };
    const auto launch_join = [&](auto narrow, auto wide) {
        if (p.wide) wide<<<join, kThreads, 0, stream>>>(k);
        else narrow<<<join, kThreads, 0, stream>>>(k);
    };
    if (c.head_dim == 64) {
        if (p.rows == 1) launch(attention_cached_kernel<64, 1, true>, attention_shared_kernel<64, 1>);
        else launch(attention_cached_kernel<64, 2, true>, attention_shared_kernel<64, 2>);
        if (waves) launch_join(join_rows_kernel<64, false>, join_rows_kernel<64, true>);
        else launch_join(attention_join_kernel<64, true>, attention_join_kernel<64, true, true>);
    } else {
        if (p.rows == 1) launch(attention_cached_kernel<128, 1, true>, attention_shared_kernel<128, 1>);
        else launch(attention_cached_kernel<128, 2, true>, attention_shared_kernel<128, 2>);
        if (waves) launch_join(join_rows_kernel<128, false>, join_rows_kernel<128, true>);
        else launch_join(attention_join_kernel<128, true>, attention_join_kernel<128, true, true>);
    }
    return hipGetLastError();
}

} // namespace apgemv
