// The Python binding's calls of the decoder operators as native functions: argument checks, output and workspace tensors, the current stream and
// the call of the C-ABI entry point (include/apdecode.h).  They hold no logic of the library.
#include <climits>
#include <cmath>

#include <ATen/hip/HIPContext.h>

#include "torch_args.h"

#include "../../include/apdecode.h"

namespace apgemv_torch {

namespace {

// Thrown where a Python error is set; caught at the entry of the call
struct Refused {};

[[noreturn]] void refuse(const char *what, const char *why)
{
    PyErr_Format(PyExc_AssertionError, "%s %s", what, why);
    throw Refused{};
}

struct Call {
    CallStream stream;
    at::Device device{at::kCUDA, 0};

    // the cache of a call: its memory and (pages, page_tokens, kv_heads, head_dim)
    ap_cache cache(PyObject *buffer, PyObject *shape)
    {
        const at::Tensor &b = tensor(buffer, "the cache");
        if (!b.is_cuda() || b.scalar_type() != at::kByte || !b.is_contiguous()) refuse("the cache", "must be a contiguous uint8 tensor on the GPU");
        if (!PyTuple_Check(shape) || PyTuple_GET_SIZE(shape) != 4) refuse("the cache's shape", "must be a tuple of 4");
        on(b.device());
        ap_cache c;
        c.data = b.data_ptr();
        c.pages = integer(PyTuple_GET_ITEM(shape, 0));
        c.page_tokens = small(PyTuple_GET_ITEM(shape, 1));
        c.kv_heads = small(PyTuple_GET_ITEM(shape, 2));
        c.head_dim = small(PyTuple_GET_ITEM(shape, 3));
        size_t bytes = 0;
        if (ap_cache_size(&c, &bytes) == AP_OK && (size_t)room(b) < bytes) refuse("the cache", "holds fewer bytes than its pages");
        return c;
    }

    // All tensors of a call are on the current device, whose stream it runs on
    void on(at::Device d)
    {
        device = d;
        if (d.index() != c10::hip::current_device()) refuse("the tensors", "must be on the current device");
    }

    // The stream of the call, once its tensors have been looked at: the current one is not to be had without a GPU
    void start(PyObject *o)
    {
        if (!stream_of(o, &stream)) throw Refused{};
    }

    const at::Tensor &tensor(PyObject *o, const char *what)
    {
        const at::Tensor *t = tensor_of(o, what);
        if (!t) throw Refused{};
        return *t;
    }

    float scale(PyObject *o, int64_t head_dim)
    {
        const double v = o == Py_None ? 1.0 / std::sqrt((double)head_dim) : PyFloat_AsDouble(o);
        if (PyErr_Occurred()) throw Refused{};
        return (float)v;
    }

    int64_t integer(PyObject *o)
    {
        const long long v = PyLong_AsLongLong(o);
        if (v == -1 && PyErr_Occurred()) throw Refused{};
        return v;
    }

    // -1, which no size may be, for what an int cannot hold
    int small(PyObject *o)
    {
        const int64_t v = integer(o);
        return v < INT_MIN || v > INT_MAX ? -1 : (int)v;
    }

    // (tokens, heads, head_dim) binary16 rows with contiguous heads; tokens or heads < 0: any
    ap_heads rows(PyObject *o, const char *what, int64_t tokens, int64_t heads, int64_t head_dim, const at::Tensor **out = nullptr)
    {
        const at::Tensor &t = tensor(o, what);
        if (t.device() != device || t.scalar_type() != at::kHalf || t.dim() != 3) refuse(what, "must be a float16 tensor (tokens, heads, head_dim) on the cache's or q's GPU");
        if ((tokens >= 0 && t.size(0) != tokens) || (heads >= 0 && t.size(1) != heads) || t.size(2) != head_dim) refuse(what, "has another shape than the call");
        if (t.size(2) > 1 && t.stride(2) != 1) refuse(what, "must have contiguous head_dim values");
        if (out) *out = &t;
        return ap_heads{t.data_ptr(), t.size(0) > 1 ? t.stride(0) : 0, t.size(1) > 1 ? t.stride(1) : 0};
    }

    // a contiguous tensor of `type` with `count` values
    void *array(PyObject *o, const char *what, at::ScalarType type, int64_t count)
    {
        const at::Tensor &t = tensor(o, what);
        if (t.device() != device || t.scalar_type() != type || !t.is_contiguous() || t.numel() != count)
            refuse(what, type == at::kLong  ? "must be a contiguous int64 tensor of the call's size on its GPU"
                         : type == at::kInt ? "must be a contiguous int32 tensor of the call's size on its GPU"
                         : type == at::kHalf ? "must be a contiguous float16 tensor of the call's size on its GPU"
                                             : "must be a contiguous float32 tensor of the call's size on its GPU");
        return t.data_ptr();
    }

    // (tokens, columns) rows of `type` with contiguous columns; `rows` of them, or one for all where `shared` allows
    ap_rows matrix(PyObject *o, const char *what, at::ScalarType type, int64_t count, int64_t columns, bool shared = false)
    {
        const at::Tensor &t = tensor(o, what);
        if (t.device() != device || t.scalar_type() != type || t.dim() != 2 || t.size(1) != columns || (t.size(0) != count && !(shared && t.size(0) == 1)) ||
            (columns > 1 && t.stride(1) != 1))
            refuse(what, type == at::kHalf ? "must be a float16 tensor (tokens, columns) of the call's size on its GPU, with contiguous columns"
                                           : "must be a float32 tensor (tokens, columns) of the call's size on its GPU, with contiguous columns");
        return ap_rows{t.data_ptr(), t.size(0) > 1 ? t.stride(0) : 0};
    }

    // the output that was given, or a new one
    at::Tensor output(PyObject *given, const char *what, at::IntArrayRef sizes, at::ScalarType type)
    {
        if (given == Py_None) return allocate(sizes, type, device, stream, true);
        int64_t count = 1;
        for (const int64_t n : sizes) count *= n;
        array(given, what, type, count);
        return tensor(given, what);
    }

    // workspace: what was given, or new memory of the call's stream
    at::Tensor workspace(PyObject *given, size_t bytes, void **data, size_t *room_bytes)
    {
        *data = nullptr;
        *room_bytes = 0;
        if (given == Py_None && bytes == 0) return at::Tensor();
        at::Tensor w = given == Py_None ? allocate({(int64_t)bytes}, at::kByte, device, stream, false) : tensor(given, "work");
        if (w.device() != device || !w.is_contiguous()) refuse("work", "must be a contiguous tensor on the call's GPU");
        *data = w.data_ptr();
        *room_bytes = (size_t)std::min(w.numel() * (int64_t)w.element_size(), room(w));
        return w;
    }
};

template <class F> PyObject *guarded(PyObject *const *, Py_ssize_t n, Py_ssize_t want, const F &call)
{
    HANDLE_TH_ERRORS
    if (n != want) {
        PyErr_Format(PyExc_TypeError, "takes %d arguments", (int)want);
        return nullptr;
    }
    try {
        return call();
    } catch (const Refused &) {
        return nullptr;
    }
    END_HANDLE_TH_ERRORS
}

template <class F> ap_status without_gil(const F &f)
{
    ap_status status;
    Py_BEGIN_ALLOW_THREADS
    status = f();
    Py_END_ALLOW_THREADS
    return status;
}

PyObject *pair(const at::Tensor &a, const at::Tensor &b)
{
    PyObject *x = a.defined() ? THPVariable_Wrap(a) : Py_NewRef(Py_None);
    PyObject *y = b.defined() ? THPVariable_Wrap(b) : Py_NewRef(Py_None);
    PyObject *t = x && y ? PyTuple_Pack(2, x, y) : nullptr;
    Py_XDECREF(x);
    Py_XDECREF(y);
    return t;
}

} // namespace

// cache_append(buffer, shape, k, v, slots, q, positions, rotary, interleaved, q_out, k_out, stream) -> (q_out, k_out), or a status
PyObject *cache_append(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    return guarded(args, n, 12, [&]() -> PyObject * {
        Call c;
        const ap_cache cache = c.cache(args[0], args[1]);
        const int64_t D = cache.head_dim;
        ap_append a = {};
        const at::Tensor *k = nullptr, *q = nullptr;
        a.k = c.rows(args[2], "k", -1, cache.kv_heads, D, &k);
        a.tokens = k->size(0);
        a.v = c.rows(args[3], "v", a.tokens, cache.kv_heads, D);
        a.slots = static_cast<const int64_t *>(c.array(args[4], "slots", at::kLong, a.tokens));
        c.start(args[11]);
        at::Tensor q_out, k_out;
        const auto out = [&](PyObject *given, const char *what, int64_t heads, ap_heads *rows) {
            if (given == Py_None) {
                const at::Tensor t = allocate({a.tokens, heads, D}, at::kHalf, c.device, c.stream, true);
                *rows = ap_heads{t.data_ptr(), heads * D, D};
                return t;
            }
            *rows = c.rows(given, what, a.tokens, heads, D);
            return c.tensor(given, what);
        };
        if (args[5] != Py_None) {
            a.q = c.rows(args[5], "q", a.tokens, -1, D, &q);
            a.heads = (int)std::min<int64_t>(q->size(1), INT_MAX);
            q_out = out(args[9], "q_out", q->size(1), &a.q_out);
        }
        k_out = out(args[10], "k_out", cache.kv_heads, &a.k_out);
        if (args[7] != Py_None) {
            const at::Tensor &r = c.tensor(args[7], "rotary");
            if (r.dim() != 2) refuse("rotary", "must have two dimensions");
            a.rotary = static_cast<const float *>(c.array(args[7], "rotary", at::kFloat, r.numel()));
            a.rotary_rows = r.size(0);
            a.rot_dim = (int)std::min<int64_t>(r.size(1), INT_MAX);
            if (!a.rotary) refuse("rotary", "must have rows and columns");
            if (args[6] == Py_None) refuse("positions", "are needed with rotary");
            a.positions = static_cast<const int64_t *>(c.array(args[6], "positions", at::kLong, a.tokens));
            a.interleaved = PyObject_IsTrue(args[8]);
            if (a.interleaved < 0) throw Refused{};
        }
        const ap_status status = without_gil([&] { return ap_cache_append(&cache, &a, c.stream.address); });
        return status == AP_OK ? pair(q_out, k_out) : PyLong_FromLong(status);
    });
}

// cache_read(buffer, shape, slots, stream) -> (k, v), or a status
PyObject *cache_read(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    return guarded(args, n, 4, [&]() -> PyObject * {
        Call c;
        const ap_cache cache = c.cache(args[0], args[1]);
        const at::Tensor &slots = c.tensor(args[2], "slots");
        const int64_t tokens = slots.numel();
        const int64_t *s = static_cast<const int64_t *>(c.array(args[2], "slots", at::kLong, tokens));
        c.start(args[3]);
        const at::Tensor k = allocate({tokens, cache.kv_heads, cache.head_dim}, at::kHalf, c.device, c.stream, true);
        const at::Tensor v = allocate({tokens, cache.kv_heads, cache.head_dim}, at::kHalf, c.device, c.stream, true);
        void *kp = k.data_ptr(), *vp = v.data_ptr();
        const ap_status status = without_gil([&] { return ap_cache_read(&cache, s, tokens, kp, vp, c.stream.address); });
        return status == AP_OK ? pair(k, v) : PyLong_FromLong(status);
    });
}

// attention_cached(buffer, shape, q, tables, lengths, q_starts, scale, max_length, out, work, stream) -> out, or a status
PyObject *attention_cached(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    return guarded(args, n, 11, [&]() -> PyObject * {
        Call c;
        const ap_cache cache = c.cache(args[0], args[1]);
        ap_cached a = {};
        const at::Tensor *q = nullptr;
        a.q = c.rows(args[2], "q", -1, -1, cache.head_dim, &q);
        a.tokens = q->size(0);
        a.heads = (int)std::min<int64_t>(q->size(1), INT_MAX);
        const at::Tensor &tables = c.tensor(args[3], "tables");
        if (tables.dim() != 2 || tables.size(0) > INT_MAX) refuse("tables", "must have two dimensions");
        a.sequences = (int)tables.size(0);
        a.table_width = tables.size(1);
        a.tables = static_cast<const int32_t *>(c.array(args[3], "tables", at::kInt, tables.numel()));
        a.lengths = static_cast<const int32_t *>(c.array(args[4], "lengths", at::kInt, a.sequences));
        if (args[5] != Py_None) a.q_starts = static_cast<const int32_t *>(c.array(args[5], "q_starts", at::kInt, (int64_t)a.sequences + 1));
        a.scale = c.scale(args[6], cache.head_dim);
        a.max_length = args[7] == Py_None ? a.table_width * cache.page_tokens : c.integer(args[7]);
        size_t bytes = 0;
        ap_status status = ap_attention_cached_size(&cache, &a, &bytes);
        if (status != AP_OK) return PyLong_FromLong(-(long)status);
        c.start(args[10]);
        const at::Tensor out = c.output(args[8], "out", {a.tokens, a.heads, cache.head_dim}, at::kHalf);
        const at::Tensor work = c.workspace(args[9], bytes, &a.work, &a.work_bytes);
        a.out = out.data_ptr();
        status = without_gil([&] { return ap_attention_cached(&cache, &a, c.stream.address); });
        return status == AP_OK ? THPVariable_Wrap(out) : PyLong_FromLong(status);
    });
}

// attention_prompt(q, k, v, q_starts, k_starts, scale, out, work, stream) -> out, or a status
PyObject *attention_prompt(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    return guarded(args, n, 9, [&]() -> PyObject * {
        Call c;
        const at::Tensor &q = c.tensor(args[0], "q"), &k = c.tensor(args[1], "k");
        if (!q.is_cuda() || q.dim() != 3 || k.dim() != 3) refuse("q and k", "must be float16 tensors (tokens, heads, head_dim) on the GPU");
        c.on(q.device());
        ap_prompt a = {};
        const int64_t D = q.size(2);
        a.q = c.rows(args[0], "q", -1, -1, D);
        a.k = c.rows(args[1], "k", -1, -1, D);
        a.v = c.rows(args[2], "v", k.size(0), k.size(1), D);
        a.tokens = q.size(0);
        a.keys = k.size(0);
        a.heads = (int)std::min<int64_t>(q.size(1), INT_MAX);
        a.kv_heads = (int)std::min<int64_t>(k.size(1), INT_MAX);
        a.head_dim = (int)std::min<int64_t>(D, INT_MAX);
        const at::Tensor &starts = c.tensor(args[3], "q_starts");
        if (starts.dim() != 1 || starts.size(0) < 1 || starts.size(0) > INT_MAX) refuse("q_starts", "must have one dimension and a value");
        a.sequences = (int)starts.size(0) - 1;
        a.q_starts = static_cast<const int32_t *>(c.array(args[3], "q_starts", at::kInt, starts.size(0)));
        a.k_starts = static_cast<const int32_t *>(c.array(args[4], "k_starts", at::kInt, starts.size(0)));
        a.scale = c.scale(args[5], D);
        size_t bytes = 0;
        ap_status status = ap_attention_prompt_size(&a, &bytes);
        if (status != AP_OK) return PyLong_FromLong(-(long)status);
        c.start(args[8]);
        const at::Tensor out = c.output(args[6], "out", {a.tokens, a.heads, D}, at::kHalf);
        const at::Tensor work = c.workspace(args[7], bytes, &a.work, &a.work_bytes);
        a.out = out.data_ptr();
        status = without_gil([&] { return ap_attention_prompt(&a, c.stream.address); });
        return status == AP_OK ? THPVariable_Wrap(out) : PyLong_FromLong(status);
    });
}

// verify(target, draft, drafted, uniform, noise, counts, work, stream) -> (tokens, accepted), or a status
PyObject *verify(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    return guarded(args, n, 8, [&]() -> PyObject * {
        Call c;
        const at::Tensor &target = c.tensor(args[0], "target"), &draft = c.tensor(args[1], "draft");
        if (!target.is_cuda() || target.dim() != 3 || draft.dim() != 3) refuse("target and draft", "must have three dimensions and be on the GPU");
        c.on(target.device());
        ap_verification a = {};
        const int64_t S = target.size(0), N = draft.size(1), V = target.size(2);
        if (draft.size(0) != S || target.size(1) != N + 1 || draft.size(2) != V) refuse("target and draft", "must be (sequences, drafts + 1, vocabulary) and (sequences, drafts, vocabulary)");
        a.half = target.scalar_type() == at::kHalf;
        const at::ScalarType type = a.half ? at::kHalf : at::kFloat;
        a.target = c.array(args[0], "target", type, S * (N + 1) * V);
        a.draft = c.array(args[1], "draft", type, S * N * V);
        if (S > INT_MAX || N > INT_MAX) refuse("target", "has too many sequences or drafts");
        a.sequences = (int)S;
        a.drafts = (int)N;
        a.vocabulary = V;
        a.drafted = static_cast<const int64_t *>(c.array(args[2], "drafted", at::kLong, S * N));
        a.uniform = static_cast<const float *>(c.array(args[3], "uniform", at::kFloat, S * N));
        a.noise = static_cast<const float *>(c.array(args[4], "noise", at::kFloat, S * V));
        if (args[5] != Py_None) a.counts = static_cast<const int32_t *>(c.array(args[5], "counts", at::kInt, S));
        size_t bytes = 0;
        ap_status status = ap_verify_size(&a, &bytes);
        if (status != AP_OK) return PyLong_FromLong(-(long)status);
        c.start(args[7]);
        const at::Tensor tokens = allocate({S, N + 1}, at::kLong, c.device, c.stream, true);
        const at::Tensor accepted = allocate({S}, at::kInt, c.device, c.stream, true);
        const at::Tensor work = c.workspace(args[6], bytes, &a.work, &a.work_bytes);
        a.tokens = static_cast<int64_t *>(tokens.data_ptr());
        a.accepted = static_cast<int32_t *>(accepted.data_ptr());
        status = without_gil([&] { return ap_verify(&a, c.stream.address); });
        return status == AP_OK ? pair(tokens, accepted) : PyLong_FromLong(status);
    });
}

// attention_shared(buffer, shape, q, prefix_tables, prefix_lengths, tables, lengths, prefix_starts, q_starts, scale, max_prefix, max_length, out, work, stream) ->
// out, or a status
PyObject *attention_shared(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    return guarded(args, n, 15, [&]() -> PyObject * {
        Call c;
        const ap_cache cache = c.cache(args[0], args[1]);
        ap_shared a = {};
        ap_cached &o = a.own;
        const at::Tensor *q = nullptr;
        o.q = c.rows(args[2], "q", -1, -1, cache.head_dim, &q);
        o.tokens = q->size(0);
        o.heads = (int)std::min<int64_t>(q->size(1), INT_MAX);
        const auto table = [&](PyObject *given, const char *what, int *rows, int64_t *width) {
            const at::Tensor &t = c.tensor(given, what);
            if (t.dim() != 2 || t.size(0) > INT_MAX) refuse(what, "must have two dimensions");
            *rows = (int)t.size(0);
            *width = t.size(1);
            return static_cast<const int32_t *>(c.array(given, what, at::kInt, t.numel()));
        };
        const auto ints = [&](PyObject *given, const char *what, int64_t count) { return static_cast<const int32_t *>(c.array(given, what, at::kInt, count)); };
        a.prefix_tables = table(args[3], "prefix_tables", &a.prefixes, &a.prefix_width);
        o.tables = table(args[5], "tables", &o.sequences, &o.table_width);
        a.prefix_lengths = ints(args[4], "prefix_lengths", a.prefixes);
        o.lengths = ints(args[6], "lengths", o.sequences);
        if (args[7] != Py_None) a.prefix_starts = ints(args[7], "prefix_starts", (int64_t)a.prefixes + 1);
        if (args[8] != Py_None) o.q_starts = ints(args[8], "q_starts", (int64_t)o.sequences + 1);
        o.scale = c.scale(args[9], cache.head_dim);
        a.max_prefix = args[10] == Py_None ? a.prefix_width * cache.page_tokens : c.integer(args[10]);
        o.max_length = args[11] == Py_None ? o.table_width * cache.page_tokens : c.integer(args[11]);
        size_t bytes = 0;
        ap_status status = ap_attention_shared_size(&cache, &a, &bytes);
        if (status != AP_OK) return PyLong_FromLong(-(long)status);
        c.start(args[14]);
        const at::Tensor out = c.output(args[12], "out", {o.tokens, o.heads, cache.head_dim}, at::kHalf);
        const at::Tensor work = c.workspace(args[13], bytes, &o.work, &o.work_bytes);
        o.out = out.data_ptr();
        status = without_gil([&] { return ap_attention_shared(&cache, &a, c.stream.address); });
        return status == AP_OK ? THPVariable_Wrap(out) : PyLong_FromLong(status);
    });
}

// norm(x, residual, weight, bias, post_weight, post_bias, post, gate, scale, eps, centred, normed, out, residual_out, stream) -> (out, residual_out), or a status
PyObject *norm(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    return guarded(args, n, 15, [&]() -> PyObject * {
        Call c;
        const bool has_x = args[0] != Py_None, has_residual = args[1] != Py_None;
        const at::Tensor &first = c.tensor(has_x ? args[0] : args[1], has_x ? "x" : "residual");
        if (!first.is_cuda() || first.dim() != 2) refuse(has_x ? "x" : "residual", "must be a tensor (tokens, columns) on the GPU");
        c.on(first.device());
        ap_normed a = {};
        const int64_t T = a.tokens = first.size(0), K = a.columns = first.size(1);
        const auto truth = [&](PyObject *o) {
            const int t = PyObject_IsTrue(o);
            if (t < 0) throw Refused{};
            return t;
        };
        // the residual's type: that of the one given, else of the output given, else binary32
        at::ScalarType wide = at::kFloat;
        if (has_residual) wide = c.tensor(args[1], "residual").scalar_type();
        else if (args[13] != Py_None) wide = c.tensor(args[13], "residual_out").scalar_type();
        if (wide != at::kFloat && wide != at::kHalf) refuse("residual", "must be a float32 or float16 tensor");
        a.half = wide == at::kHalf;
        if (has_x) a.x = c.matrix(args[0], "x", at::kHalf, T, K);
        if (has_residual) a.residual = c.matrix(args[1], "residual", wide, T, K);
        if (args[7] != Py_None) a.gate = c.matrix(args[7], "gate", at::kHalf, T, K, true);
        const auto vector = [&](PyObject *o, const char *what) -> const void * { return o == Py_None ? nullptr : c.array(o, what, at::kHalf, K); };
        a.weight = vector(args[2], "weight");
        a.bias = vector(args[3], "bias");
        a.post_weight = vector(args[4], "post_weight");
        a.post_bias = vector(args[5], "post_bias");
        a.post = truth(args[6]);
        a.scale = c.scale(args[8], 1);
        a.eps = c.scale(args[9], 1);
        a.centred = truth(args[10]);
        const bool normed = truth(args[11]);
        c.start(args[14]);
        at::Tensor out, residual_out;
        const auto given = [&](PyObject *o, const char *what, at::ScalarType type, ap_rows *rows) {
            *rows = c.matrix(o, what, type, T, K);
            return c.tensor(o, what);
        };
        const auto fresh = [&](at::ScalarType type, ap_rows *rows) {
            const at::Tensor t = allocate({T, K}, type, c.device, c.stream, true);
            *rows = ap_rows{t.data_ptr(), K};
            return t;
        };
        if (args[12] != Py_None) out = given(args[12], "out", at::kHalf, &a.out);
        else if (normed) out = fresh(at::kHalf, &a.out);
        if (args[13] != Py_None) residual_out = given(args[13], "residual_out", wide, &a.residual_out);
        else if (has_x && has_residual) residual_out = fresh(wide, &a.residual_out);
        const ap_status status = without_gil([&] { return ap_norm(&a, c.stream.address); });
        return status == AP_OK ? pair(out, residual_out) : PyLong_FromLong(status);
    });
}

// sample(logits, uniform, temperature, top_k, top_p, min_p, probabilities (a tensor, 0 = none, 1 = float32, 2 = float16), work, stream) -> (tokens, probabilities),
// or a status
PyObject *sample(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    return guarded(args, n, 9, [&]() -> PyObject * {
        Call c;
        const at::Tensor &logits = c.tensor(args[0], "logits");
        if (!logits.is_cuda() || logits.dim() != 2 || (logits.scalar_type() != at::kHalf && logits.scalar_type() != at::kFloat))
            refuse("logits", "must be a float32 or float16 tensor (rows, vocabulary) on the GPU");
        c.on(logits.device());
        ap_sampling a = {};
        const int64_t S = a.rows = logits.size(0), V = a.vocabulary = logits.size(1);
        a.half = logits.scalar_type() == at::kHalf;
        const ap_rows rows = c.matrix(args[0], "logits", logits.scalar_type(), S, V);
        a.logits = rows.data;
        a.stride = rows.stride;
        const auto floats = [&](PyObject *o, const char *what) { return o == Py_None ? nullptr : static_cast<const float *>(c.array(o, what, at::kFloat, S)); };
        a.uniform = static_cast<const float *>(c.array(args[1], "uniform", at::kFloat, S));
        a.temperature = floats(args[2], "temperature");
        if (args[3] != Py_None) a.top_k = static_cast<const int32_t *>(c.array(args[3], "top_k", at::kInt, S));
        a.top_p = floats(args[4], "top_p");
        a.min_p = floats(args[5], "min_p");
        size_t bytes = 0;
        ap_status status = ap_sample_size(&a, &bytes);
        if (status != AP_OK) return PyLong_FromLong(-(long)status);
        c.start(args[8]);
        const at::Tensor tokens = allocate({S}, at::kLong, c.device, c.stream, true);
        at::Tensor probabilities;
        if (PyLong_Check(args[6])) {
            const int64_t kind = c.integer(args[6]);
            if (kind) probabilities = allocate({S, V}, kind == 2 ? at::kHalf : at::kFloat, c.device, c.stream, true);
        } else {
            probabilities = c.tensor(args[6], "probabilities");
            if (probabilities.dim() != 2 || probabilities.size(0) != S || probabilities.size(1) != V || (probabilities.scalar_type() != at::kHalf && probabilities.scalar_type() != at::kFloat))
                refuse("probabilities", "must be a float32 or float16 tensor (rows, vocabulary)");
            c.array(args[6], "probabilities", probabilities.scalar_type(), S * V);
        }
        const at::Tensor work = c.workspace(args[7], bytes, &a.work, &a.work_bytes);
        a.tokens = static_cast<int64_t *>(tokens.data_ptr());
        if (probabilities.defined()) {
            a.probabilities = probabilities.data_ptr();
            a.half_probabilities = probabilities.scalar_type() == at::kHalf;
        }
        status = without_gil([&] { return ap_sample(&a, c.stream.address); });
        return status == AP_OK ? pair(tokens, probabilities) : PyLong_FromLong(status);
    });
}

} // namespace apgemv_torch
