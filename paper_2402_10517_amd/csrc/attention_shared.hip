// Attention of new tokens over the 4-bit paged cache where sequences share prefixes.
//
// The query rows of all sequences of a prefix are one long tile list over its keys, so that a prefix is read once; a sequence's own keys are a second list in the
// same launch.  Both leave maximum, sum of weights and sums of values per range of keys, which the second launch joins.
#include "attention_ranges.h"

namespace apgemv {

namespace {

struct Plan {
    int rows; // 16-row tiles per workgroup
    int64_t items, prefix_items;
    int chunk, prefix_chunk, splits, prefix_splits;
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
    p.rows = each * group <= 16 && prefix_rows <= 16 && most / kPiece * (items_of(16) + prefix_items_of(16)) * c.kv_heads < 1 << 20 ? 1 : 2;
    p.items = items_of(16 * p.rows);
    p.prefix_items = prefix_items_of(16 * p.rows);
    // Ranges of keys of the same length for both, so that there are two workgroups per CU in all
    const int64_t keys = (longest * p.items + longest_prefix * p.prefix_items) * c.kv_heads;
    int64_t chunk = (keys + 511) / 512;
    if (p.rows == 1 && chunk > kPiece) chunk = kPiece;
    if (chunk < 2 * kStep) chunk = 2 * kStep;
    const auto round_up = [](int64_t x) { return (int)((x + kStep - 1) / kStep * kStep); };
    p.chunk = round_up(chunk < longest ? chunk : longest);
    p.prefix_chunk = round_up(chunk < longest_prefix ? chunk : longest_prefix);
    p.splits = (int)((longest + p.chunk - 1) / p.chunk);
    p.prefix_splits = a.prefixes > 0 ? (int)((longest_prefix + p.prefix_chunk - 1) / p.prefix_chunk) : 0;
    return p;
}

} // namespace

size_t attention_shared_work(const ap_cache &c, const ap_shared &a)
{
    const Plan p = plan_of(c, a);
    return (size_t)(p.splits + p.prefix_splits) * a.own.tokens * a.own.heads * (c.head_dim * sizeof(float) + sizeof(float2));
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
    k.stat = reinterpret_cast<float2 *>(k.part + (size_t)(p.splits + p.prefix_splits) * o.tokens * o.heads * c.head_dim);
    k.prefix_starts = a.prefix_starts, k.prefix_lengths = a.prefix_lengths, k.prefix_tables = a.prefix_tables;
    k.prefix_width = a.prefix_width;
    k.prefixes = a.prefixes, k.max_prefix = (int)a.max_prefix;
    k.prefix_items = (int)p.prefix_items, k.prefix_splits = p.prefix_splits, k.prefix_chunk = p.prefix_chunk;
    const dim3 grid((unsigned)((p.items * p.splits + p.prefix_items * p.prefix_splits) * c.kv_heads)), join((unsigned)(o.tokens * o.heads));
    if (c.head_dim == 64) {
        if (p.rows == 1) attention_cached_kernel<64, 1, true><<<grid, kThreads, 0, stream>>>(k);
        else attention_cached_kernel<64, 2, true><<<grid, kThreads, 0, stream>>>(k);
        attention_join_kernel<64, true><<<join, kThreads, 0, stream>>>(k);
    } else {
        if (p.rows == 1) attention_cached_kernel<128, 1, true><<<grid, kThreads, 0, stream>>>(k);
        else attention_cached_kernel<128, 2, true><<<grid, kThreads, 0, stream>>>(k);
        attention_join_kernel<128, true><<<join, kThreads, 0, stream>>>(k);
    }
    return hipGetLastError();
}

} // namespace apgemv
