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

} // namespace apgemv_torch
