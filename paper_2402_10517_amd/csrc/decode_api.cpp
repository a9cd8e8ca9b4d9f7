// C-ABI entry points of the decoder operators (include/apdecode.h): argument checks, then one launcher each.
#include <cmath>

#include "decode.h"

using namespace apgemv;

namespace {

bool aligned(const void *p, uintptr_t n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }

// A row of 64 or 128 values at any head and token: strides in 16-byte steps, and no offset near the end of 64 bits
bool rows_ok(const ap_heads &r)
{
    const int64_t most = (int64_t)1 << 40;
    return r.data && aligned(r.data, 16) && r.token_stride % 8 == 0 && r.head_stride % 8 == 0 && r.token_stride > -most && r.token_stride < most &&
           r.head_stride > -most && r.head_stride < most;
}

bool head_dim_ok(int d) { return d == 64 || d == 128; }

constexpr int64_t kMaxTokens = 0x7fffff00; // tokens of a call: the starts of sequences are 32-bit
constexpr int64_t kMaxKeys = (int64_t)1 << 30; // of a sequence: the ends of ranges behind its last key are 32-bit too

ap_status check_cache_shape(const ap_cache *c)
{
    if (!c) return AP_ERR_INVALID_ARG;
    if (!head_dim_ok(c->head_dim) || cache_log_page(c->page_tokens) < 0 || c->kv_heads < 1 || c->kv_heads > 1024) return AP_ERR_SHAPE;
    if (c->pages < 1 || c->pages >= (int64_t)1 << 40 || c->pages * c->page_tokens >= (int64_t)1 << 40) return AP_ERR_SHAPE;
    return AP_OK;
}

ap_status check_cache(const ap_cache *c)
{
    const ap_status s = check_cache_shape(c);
    if (s != AP_OK) return s;
    return c->data && aligned(c->data, AP_BLOB_ALIGN) ? AP_OK : AP_ERR_INVALID_ARG;
}

ap_status check_heads(int heads, int kv_heads)
{
    return heads >= 1 && kv_heads >= 1 && kv_heads <= 1024 && heads <= 4096 && heads % kv_heads == 0 ? AP_OK : AP_ERR_SHAPE;
}

ap_status check_cached(const ap_cache *c, const ap_cached *a)
{
    ap_status s = check_cache_shape(c);
    if (s != AP_OK) return s;
    if (!a) return AP_ERR_INVALID_ARG;
    s = check_heads(a->heads, c->kv_heads);
    if (s != AP_OK) return s;
    if (a->tokens < 0 || a->tokens > kMaxTokens || a->sequences < 0 || a->sequences > (1 << 20)) return AP_ERR_SHAPE;
    if ((a->tokens > 0 && a->sequences < 1) || a->tokens * a->heads > kMaxTokens) return AP_ERR_SHAPE;
    if (!groups_ok(a->tokens * a->heads, 16, a->sequences, c->kv_heads)) return AP_ERR_SHAPE;
    if (!a->q_starts && a->sequences > 0 && a->tokens % a->sequences) return AP_ERR_SHAPE;
    if (a->table_width < 0 || a->table_width >= (int64_t)1 << 31 || a->max_length < 0 || a->max_length > kMaxKeys ||
        a->max_length > a->table_width * c->page_tokens)
        return AP_ERR_SHAPE;
    return AP_OK;
}

ap_status done(hipError_t e) { return e == hipSuccess ? AP_OK : AP_ERR_HIP; }

} // namespace

extern "C" ap_status ap_cache_size(const ap_cache *c, size_t *bytes)
{
    const ap_status s = check_cache_shape(c);
    if (s != AP_OK) return s;
    if (!bytes) return AP_ERR_INVALID_ARG;
    *bytes = (size_t)c->pages * c->page_tokens * c->kv_heads * (c->head_dim + 8);
    return AP_OK;
}

extern "C" ap_status ap_cache_append(const ap_cache *c, const ap_append *a, void *stream)
{
    ap_status s = check_cache(c);
    if (s != AP_OK) return s;
    if (!a) return AP_ERR_INVALID_ARG;
    if (a->tokens < 0 || a->tokens > kMaxTokens) return AP_ERR_SHAPE;
    if (a->q.data && (a->heads < 1 || a->heads > 4096)) return AP_ERR_SHAPE;
    if (a->rotary && (a->rot_dim < 16 || a->rot_dim > c->head_dim || a->rot_dim % 16 || a->rotary_rows < 0)) return AP_ERR_SHAPE;
    if (a->tokens == 0) return AP_OK;
    if (!rows_ok(a->k) || !rows_ok(a->v) || !a->slots || !aligned(a->slots, 8)) return AP_ERR_INVALID_ARG;
    if (a->q.data && (!rows_ok(a->q) || !rows_ok(a->q_out))) return AP_ERR_INVALID_ARG;
    if (a->k_out.data && !rows_ok(a->k_out)) return AP_ERR_INVALID_ARG;
    if (a->rotary && (!a->positions || !aligned(a->positions, 8) || !aligned(a->rotary, 16))) return AP_ERR_INVALID_ARG;
    return done(launch_cache_append(*c, *a, static_cast<hipStream_t>(stream)));
}

extern "C" ap_status ap_cache_read(const ap_cache *c, const int64_t *slots, int64_t tokens, void *k_out, void *v_out, void *stream)
{
    ap_status s = check_cache(c);
    if (s != AP_OK) return s;
    if (tokens < 0 || tokens > kMaxTokens) return AP_ERR_SHAPE;
    if (tokens == 0) return AP_OK;
    if (!slots || !aligned(slots, 8) || !k_out || !v_out || !aligned(k_out, 16) || !aligned(v_out, 16)) return AP_ERR_INVALID_ARG;
    return done(launch_cache_read(*c, slots, tokens, k_out, v_out, static_cast<hipStream_t>(stream)));
}

extern "C" ap_status ap_attention_cached_size(const ap_cache *c, const ap_cached *a, size_t *bytes)
{
    const ap_status s = check_cached(c, a);
    if (s != AP_OK) return s;
    if (!bytes) return AP_ERR_INVALID_ARG;
    *bytes = a->tokens == 0 ? 0 : attention_cached_work(*c, *a);
    return AP_OK;
}

extern "C" ap_status ap_attention_cached(const ap_cache *c, const ap_cached *a, void *stream)
{
    ap_status s = check_cached(c, a);
    if (s != AP_OK) return s;
    s = check_cache(c);
    if (s != AP_OK) return s;
    if (a->tokens == 0) return AP_OK;
    if (!rows_ok(a->q) || !a->lengths || !a->out || !aligned(a->out, 16) || !aligned(a->lengths, 4) || !aligned(a->q_starts, 4) ||
        !aligned(a->tables, 4) || (!a->tables && a->max_length > 0) || !std::isfinite(a->scale))
        return AP_ERR_INVALID_ARG;
    const size_t need = attention_cached_work(*c, *a);
    if (need && (!a->work || !aligned(a->work, 16))) return AP_ERR_INVALID_ARG;
    if (a->work_bytes < need) return AP_ERR_BUFFER_TOO_SMALL;
    return done(launch_attention_cached(*c, *a, static_cast<hipStream_t>(stream)));
}

static ap_status check_prompt(const ap_prompt *a)
{
    if (!a) return AP_ERR_INVALID_ARG;
    if (!head_dim_ok(a->head_dim)) return AP_ERR_SHAPE;
    const ap_status s = check_heads(a->heads, a->kv_heads);
    if (s != AP_OK) return s;
    if (a->tokens < 0 || a->tokens > kMaxTokens || a->keys < 0 || a->keys > kMaxKeys || a->sequences < 0 || a->sequences > (1 << 20) ||
        (a->tokens > 0 && a->sequences < 1) || a->tokens * a->heads > kMaxTokens || !groups_ok(a->tokens * a->heads, 128, a->sequences, a->kv_heads))
        return AP_ERR_SHAPE;
    // a tile of 64 rows of k or v is addressed by 32 bits from its first
    if (a->k.token_stride < 0 || a->k.token_stride > 1 << 24 || a->v.token_stride < 0 || a->v.token_stride > 1 << 24) return AP_ERR_SHAPE;
    return AP_OK;
}

extern "C" ap_status ap_attention_prompt_size(const ap_prompt *a, size_t *bytes)
{
    const ap_status s = check_prompt(a);
    if (s != AP_OK) return s;
    if (!bytes) return AP_ERR_INVALID_ARG;
    *bytes = a->tokens == 0 ? 0 : attention_prompt_work(*a);
    return AP_OK;
}

extern "C" ap_status ap_attention_prompt(const ap_prompt *a, void *stream)
{
    const ap_status s = check_prompt(a);
    if (s != AP_OK) return s;
    if (a->tokens == 0) return AP_OK;
    if (!rows_ok(a->q) || (a->keys > 0 && (!rows_ok(a->k) || !rows_ok(a->v))) || !a->q_starts || !a->k_starts || !aligned(a->q_starts, 4) ||
        !aligned(a->k_starts, 4) || !a->out || !aligned(a->out, 16) || !std::isfinite(a->scale))
        return AP_ERR_INVALID_ARG;
    const size_t need = attention_prompt_work(*a);
    if (need && (!a->work || !aligned(a->work, 16))) return AP_ERR_INVALID_ARG;
    if (a->work_bytes < need) return AP_ERR_BUFFER_TOO_SMALL;
    return done(launch_attention_prompt(*a, static_cast<hipStream_t>(stream)));
}

static ap_status check_verify(const ap_verification *a)
{
    if (!a) return AP_ERR_INVALID_ARG;
    if (a->sequences < 0 || a->sequences > (1 << 20) || a->drafts < 0 || a->drafts > 1024 || a->vocabulary < 1 || a->vocabulary >= (int64_t)1 << 31)
        return AP_ERR_SHAPE;
    return AP_OK;
}

extern "C" ap_status ap_verify_size(const ap_verification *a, size_t *bytes)
{
    const ap_status s = check_verify(a);
    if (s != AP_OK) return s;
    if (!bytes) return AP_ERR_INVALID_ARG;
    *bytes = a->sequences == 0 ? 0 : verify_work(*a);
    return AP_OK;
}

extern "C" ap_status ap_verify(const ap_verification *a, void *stream)
{
    const ap_status s = check_verify(a);
    if (s != AP_OK) return s;
    if (a->sequences == 0) return AP_OK;
    const uintptr_t element = a->half ? 2 : 4;
    if (!a->target || !aligned(a->target, element) || !a->noise || !aligned(a->noise, 4) || !a->tokens || !aligned(a->tokens, 8) || !a->accepted ||
        !aligned(a->accepted, 4) || !aligned(a->counts, 4))
        return AP_ERR_INVALID_ARG;
    if (a->drafts > 0 && (!a->draft || !aligned(a->draft, element) || !a->drafted || !aligned(a->drafted, 8) || !a->uniform || !aligned(a->uniform, 4)))
        return AP_ERR_INVALID_ARG;
    const size_t need = verify_work(*a);
    if (need && (!a->work || !aligned(a->work, 16))) return AP_ERR_INVALID_ARG;
    if (a->work_bytes < need) return AP_ERR_BUFFER_TOO_SMALL;
    return done(launch_verify(*a, static_cast<hipStream_t>(stream)));
}

static ap_status check_shared(const ap_cache *c, const ap_shared *a)
{
    if (!a) return c ? AP_ERR_INVALID_ARG : check_cache_shape(c);
    const ap_status s = check_cached(c, &a->own);
    if (s != AP_OK) return s;
    if (a->own.tokens * a->own.heads >= (int64_t)1 << 24) return AP_ERR_SHAPE; // a launch has no more workgroups, and one of the two joins takes one for each row
    if (a->prefixes < 0 || a->prefixes > (1 << 20)) return AP_ERR_SHAPE;
    if (!a->prefix_starts && a->prefixes > 0 && a->own.sequences % a->prefixes) return AP_ERR_SHAPE;
    // besides the row tiles' workgroups there are up to 512 for the prefixes
    if (!groups_ok(a->own.tokens * a->own.heads, 8, (int64_t)a->own.sequences + a->prefixes + 512, c->kv_heads)) return AP_ERR_SHAPE;
    if (a->prefix_width < 0 || a->prefix_width >= (int64_t)1 << 31 || a->max_prefix < 0 || a->max_prefix > kMaxKeys ||
        a->max_prefix > a->prefix_width * c->page_tokens)
        return AP_ERR_SHAPE;
    return AP_OK;
}

extern "C" ap_status ap_attention_shared_size(const ap_cache *c, const ap_shared *a, size_t *bytes)
{
    const ap_status s = check_shared(c, a);
    if (s != AP_OK) return s;
    if (!bytes) return AP_ERR_INVALID_ARG;
    *bytes = a->own.tokens == 0 ? 0 : attention_shared_work(*c, *a);
    return AP_OK;
}

extern "C" ap_status ap_attention_shared(const ap_cache *c, const ap_shared *a, void *stream)
{
    ap_status s = check_shared(c, a);
    if (s != AP_OK) return s;
    s = check_cache(c);
    if (s != AP_OK) return s;
    const ap_cached &o = a->own;
    if (o.tokens == 0) return AP_OK;
    if (!rows_ok(o.q) || !o.lengths || !o.out || !aligned(o.out, 16) || !aligned(o.lengths, 4) || !aligned(o.q_starts, 4) || !aligned(o.tables, 4) ||
        (!o.tables && o.max_length > 0) || !std::isfinite(o.scale))
        return AP_ERR_INVALID_ARG;
    if (!aligned(a->prefix_starts, 4) || !aligned(a->prefix_lengths, 4) || !aligned(a->prefix_tables, 4) || (a->prefixes > 0 && !a->prefix_lengths) ||
        (a->prefixes > 0 && a->max_prefix > 0 && !a->prefix_tables))
        return AP_ERR_INVALID_ARG;
    const size_t need = attention_shared_work(*c, *a);
    if (need && (!o.work || !aligned(o.work, 16))) return AP_ERR_INVALID_ARG;
    if (o.work_bytes < need) return AP_ERR_BUFFER_TOO_SMALL;
    return done(launch_attention_shared(*c, *a, static_cast<hipStream_t>(stream)));
}

extern "C" ap_status ap_norm(const ap_normed *a, void *stream)
{
    if (!a) return AP_ERR_INVALID_ARG;
    if (a->tokens < 0 || a->tokens > kMaxTokens || a->columns < 1 || a->columns > 32768) return AP_ERR_SHAPE;
    if (a->tokens == 0) return AP_OK;
    const int64_t most = (int64_t)1 << 40;
    const uintptr_t wide = a->half ? 2 : 4;
    const auto ok = [&](const ap_rows &r, uintptr_t element) { return aligned(r.data, element) && r.stride > -most && r.stride < most; };
    if ((!a->x.data && !a->residual.data) || !ok(a->x, 2) || !ok(a->gate, 2) || !ok(a->out, 2) || !ok(a->residual, wide) || !ok(a->residual_out, wide))
        return AP_ERR_INVALID_ARG;
    if (!aligned(a->weight, 2) || !aligned(a->bias, 2) || !aligned(a->post_weight, 2) || !aligned(a->post_bias, 2)) return AP_ERR_INVALID_ARG;
    if (!std::isfinite(a->scale) || !(a->eps >= 0) || !std::isfinite(a->eps)) return AP_ERR_INVALID_ARG;
    // rows that are written lie apart
    const auto apart = [&](const ap_rows &r) { return !r.data || a->tokens < 2 || r.stride >= a->columns || -r.stride >= a->columns; };
    if (!apart(a->out) || !apart(a->residual_out)) return AP_ERR_INVALID_ARG;
    if (!a->out.data && !a->residual_out.data) return AP_OK;
    return done(launch_norm(*a, static_cast<hipStream_t>(stream)));
}

static ap_status check_sample(const ap_sampling *a)
{
    if (!a) return AP_ERR_INVALID_ARG;
    const int64_t most = (int64_t)1 << 40;
    // a workgroup of up to 1024 threads per row
    if (a->rows < 0 || a->rows > 1 << 21 || a->vocabulary < 1 || a->vocabulary > 1 << 20 || a->stride <= -most || a->stride >= most) return AP_ERR_SHAPE;
    return AP_OK;
}

extern "C" ap_status ap_sample_size(const ap_sampling *a, size_t *bytes)
{
    const ap_status s = check_sample(a);
    if (s != AP_OK) return s;
    if (!bytes) return AP_ERR_INVALID_ARG;
    *bytes = 0; // a workgroup has a row and keeps its sums in LDS
    return AP_OK;
}

// Whether a row of logits lies in the probabilities' memory, which is written before the last logit is read
static bool overlaps(const ap_sampling *a)
{
    if (!a->probabilities) return false;
    typedef __int128 wide_t; // |rows * stride| is up to 2^63 bytes
    const wide_t element = a->half ? 2 : 4, row = a->vocabulary * element, begin = reinterpret_cast<uintptr_t>(a->probabilities),
                 end = begin + (wide_t)a->rows * a->vocabulary * (a->half_probabilities ? 2 : 4);
    wide_t first = reinterpret_cast<uintptr_t>(a->logits), stride = a->stride * element;
    if (stride < 0) first += (a->rows - 1) * stride, stride = -stride;
    // the first row that ends behind the beginning
    wide_t i = 0;
    if (first + row <= begin) {
        if (stride == 0) return false;
        i = (begin - row - first) / stride + 1;
    }
    return i < a->rows && first + i * stride < end;
}

extern "C" ap_status ap_sample(const ap_sampling *a, void *stream)
{
    const ap_status s = check_sample(a);
    if (s != AP_OK) return s;
    if (a->rows == 0) return AP_OK;
    if (!a->logits || !aligned(a->logits, a->half ? 2 : 4) || !a->uniform || !aligned(a->uniform, 4) || !a->tokens || !aligned(a->tokens, 8) ||
        !aligned(a->temperature, 4) || !aligned(a->top_p, 4) || !aligned(a->min_p, 4) || !aligned(a->top_k, 4) ||
        !aligned(a->probabilities, a->half_probabilities ? 2 : 4) || overlaps(a))
        return AP_ERR_INVALID_ARG;
    return done(launch_sample(*a, static_cast<hipStream_t>(stream)));
}
