// Attention of new tokens over the 4-bit paged cache, on the matrix cores.
//
// A workgroup takes a tile of query rows (token, head of the group) of one sequence and key head and a range of its keys; a wave takes 32 keys at a
// time:
//   S^T = C Q^T with C the key codes, v_mfma_f32_16x16x32_f16: a code as the low bits of a binary16 number is code * 2^-24, exact (the instruction takes
//         subnormal numbers as they are), and s = scale (step S + low sum q) in binary32, in the unit 2^-24 until it meets the scale;
//   O^T = V^T P^T, v_mfma_f32_16x16x32_bf16: codes enter as bfloat16 16 + code, exact (the nibble set into the mantissa of 16), the weights as p * step in
//         two bfloat16 parts (high + rest); what is the same for all channels of a row, sum p low - 16 sum p step, is one number.
// Rounding: the two parts keep 16 bits of a weight and the range of binary32 for any step, 2^-17 of it, a 64th of the result's own rounding; a third part
// would cost half as many products again.  The offset is the least that bfloat16 has room for: products of 16
// to 31 steps where the code alone would be 0 to 15 (mean of 2048 values that cancel, steps of 1.5: off by 2.1e-6; with an offset of 128, 1.2e-5).
// With keys as rows and queries as columns a lane holds scores of one query row throughout, the scores' registers are the weights' operand as they
// stand (the order of the keys inside a product is free, and the cache's value layout follows it), and the statistics are one number per lane. The
// running maximum moves only when a score exceeds it by 2^8: weights stay below 2^8 and the accumulators are seldom rescaled.
//
// A key of one head is D + 8 bytes and 4 (heads / kv_heads) D operations: HBM bounds the work, and a wave has its next 32 keys' loads in flight while
// it works. Long sequences reach it: two of 131072 keys and 8 key heads of 128 take 51 us (285 MB, 5.5 TB/s; ap_probe_read reads as much in 44) and
// the join 5. Short ones are bound by what happens once per workgroup (start, length, page and first key one after the other, the join of the waves,
// the second launch: some 10 us in all), and by the vector instructions per 32 keys, about 250: 4-bit codes to operands 120, softmax and weights 100.
// Codes staged through LDS two to four tiles ahead, or two sets of registers without moves, came out the same within 5 % on all of them.
#include "attention_ranges.h"

namespace apgemv {

namespace {

struct Plan {
    int rows; // 16-row tiles per workgroup
    int64_t items;
    int chunk, splits;
};

Plan plan_of(const ap_cache &c, const ap_cached &a)
{
    Plan p;
    const int64_t group = a.heads / c.kv_heads, each = (a.tokens + a.sequences - 1) / a.sequences, longest = a.max_length > 0 ? a.max_length : 1;
    const auto items_of = [&](int64_t tile) { return a.q_starts ? a.tokens * group / tile + a.sequences : (each * group + tile - 1) / tile * a.sequences; };
    // 16 rows where that is enough for a sequence's queries, in ranges of one piece at most.  2^20 such ranges are more keys than the card's memory can
    // hold: max_length is then far above the lengths, and the other kernel's ranges of any length keep the workgroups few.  So rows that are joined are
    // fewer than 2^24, a workgroup each.
    p.rows = each * group <= 16 && longest / kPiece * items_of(16) * c.kv_heads < 1 << 20 ? 1 : 2;
    p.items = items_of(16 * p.rows);
    // Ranges of keys.  Two workgroups per CU in all, of 256 keys at least; four where two would have more than 1024 keys each, as longer ranges leave
    // the card waiting for the last.  One, and no second launch, where every CU has a workgroup of up to 2048 keys.  us at 1 / 2 / 4 / 8 / 16 / 32 /
    // 64 ranges, heads of 128: 32 sequences of 2000 keys and 8 key heads 18.4 / 20.7 / 24.0, up to 4099 keys (ragged) - / 29.0 / 25.8 / 27.6, 4 of
    // 3000 and 32 - / 16.9 / 15.6 / 17.6, 16 up to 8000 and 8 - / - / 28.2 / 24.1, 1 of 1000 and 32 10.1 / 9.9 / 8.6 / 8.4, 2 of 131072 and 8 at 32
    // 62.7, at 64 57.9; heads of 64: 8 of 8000 and 4 at 8 12.9, at 16 12.6, at 32 14.6.
    const int64_t units = p.items * c.kv_heads, keys = longest * units, two = (keys + 511) / 512, four = (keys + 1023) / 1024;
    int64_t chunk = two <= 1024 ? two : four > 1024 ? four : 1024;
    if (units >= 256 && longest <= 2048) chunk = longest;
    // Longer ones are cut all the same, which fills the last round of workgroups; with 32 rows up to some 8192 workgroups, so that their sums are 280 MB
    // at most.  ms with ranges of 4096 keys / longer ones, 64 heads and 8 key heads of 128: 1 x 4096 queries over 32768 keys 7.78 / 7.13 (1.1 GB of
    // sums / none), 8 x 512 over 16384 4.20 / 3.78, over up to 16384 2.72 / 2.40.
    const int64_t cut = (keys + 8191) / 8192, most = p.rows == 2 && cut > kPiece ? cut : kPiece;
    chunk = chunk > most ? most : chunk;
    chunk = chunk > longest ? longest : chunk;
    chunk = chunk < 2 * kStep ? 2 * kStep : chunk;
    p.chunk = (int)((chunk + kStep - 1) / kStep * kStep);
    p.splits = (int)((longest + p.chunk - 1) / p.chunk);
    return p;
}

} // namespace

size_t attention_cached_work(const ap_cache &c, const ap_cached &a)
{
    const Plan p = plan_of(c, a);
    return p.splits == 1 ? 0 : (size_t)p.splits * a.tokens * a.heads * (c.head_dim * sizeof(float) + sizeof(float2));
}

hipError_t launch_attention_cached(const ap_cache &c, const ap_cached &a, hipStream_t stream)
{
    const Plan p = plan_of(c, a);
    CachedArgs k;
    k.cache = cache_shape(c);
    k.q = static_cast<const _Float16 *>(a.q.data);
    k.q_token = a.q.token_stride, k.q_head = a.q.head_stride;
    k.table_width = a.table_width;
    k.q_starts = a.q_starts, k.lengths = a.lengths, k.tables = a.tables;
    k.tokens = (int)a.tokens, k.heads = a.heads, k.sequences = a.sequences, k.max_length = (int)a.max_length;
    k.items = (int)p.items, k.splits = p.splits, k.chunk = p.chunk;
    k.scale = scale_in_range(a.scale) / kCodeUnit;
    k.slack = kSlack / (fabsf(k.scale) * kLog2e);
    k.out = static_cast<_Float16 *>(a.out);
    k.part = static_cast<float *>(a.work);
    k.stat = reinterpret_cast<float2 *>(k.part + (size_t)p.splits * a.tokens * a.heads * c.head_dim);
    const dim3 grid((unsigned)(p.items * c.kv_heads * p.splits)); // within kMostGroups: the caller has looked
    if (c.head_dim == 64) {
        if (p.rows == 1) attention_cached_kernel<64, 1, false><<<grid, kThreads, 0, stream>>>(k);
        else attention_cached_kernel<64, 2, false><<<grid, kThreads, 0, stream>>>(k);
    } else {
        if (p.rows == 1) attention_cached_kernel<128, 1, false><<<grid, kThreads, 0, stream>>>(k);
        else attention_cached_kernel<128, 2, false><<<grid, kThreads, 0, stream>>>(k);
    }
    if (p.splits > 1) {
        const dim3 join((unsigned)(a.tokens * a.heads));
        if (c.head_dim == 64) attention_join_kernel<64, false><<<join, kThreads, 0, stream>>>(k);
        else attention_join_kernel<128, false><<<join, kThreads, 0, stream>>>(k);
    }
    return hipGetLastError();
}

} // namespace apgemv
