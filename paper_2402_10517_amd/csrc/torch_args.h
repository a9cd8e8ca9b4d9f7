// What the binding's native calls share: tensors, addresses and streams from Python's arguments, and memory of a call's stream.
#ifndef APGEMV_TORCH_ARGS_H
#define APGEMV_TORCH_ARGS_H

#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <ATen/hip/impl/HIPStreamMasqueradingAsCUDA.h>
#include <ATen/ops/empty.h>

#include <algorithm>
#include <vector>

namespace apgemv_torch {

// `o` as a tensor, or an error set
inline const at::Tensor *tensor_of(PyObject *o, const char *what)
{
    if (THPVariable_Check(o)) return &THPVariable_Unpack(o);
    PyErr_Format(PyExc_TypeError, "%s must be a torch.Tensor", what);
    return nullptr;
}

// An address given as an int or None (0); false with an error set otherwise
inline bool address_of(PyObject *o, void **out)
{
    *out = nullptr;
    if (o == Py_None) return true;
    *out = PyLong_AsVoidPtr(o);
    return !PyErr_Occurred();
}

// The stream of a call: a named one, or (None) the current one
struct CallStream {
    void *address;
    bool named;
};

inline bool stream_of(PyObject *o, CallStream *out)
{
    out->named = o != Py_None;
    if (out->named) return address_of(o, &out->address);
    out->address = c10::hip::getCurrentHIPStream().stream();
    return true;
}

// Bytes of a given tensor's memory from its first element on; 0 for memory that the GPU cannot write
inline int64_t room(const at::Tensor &t)
{
    if (!t.is_cuda() && !t.is_pinned()) return 0;
    return (int64_t)t.storage().nbytes() - t.storage_offset() * (int64_t)t.element_size();
}

// Memory that work on the call's stream writes.  The caching allocator hands a block out in the order of the stream that is current,
// and again as soon as it is released there.  For a named stream it is therefore asked in that stream's order: from the current
// stream's blocks, work still queued there could use a block that the call overwrites, or be given one that the call still
// uses.  A tensor that is returned is read by the caller on the current stream, so its release waits for that one too.
inline at::Tensor allocate(at::IntArrayRef sizes, at::ScalarType type, at::Device device, const CallStream &stream, bool returned)
{
    const auto options = at::TensorOptions().dtype(type).device(device);
    if (!stream.named) return at::empty(sizes, options);
    const auto current = c10::hip::getCurrentHIPStreamMasqueradingAsCUDA(device.index());
    if (current.stream() == stream.address) return at::empty(sizes, options);
    struct Restore {
        decltype(current) &stream;
        ~Restore() { c10::hip::setCurrentHIPStreamMasqueradingAsCUDA(stream); }
    } restore{current};
    c10::hip::setCurrentHIPStreamMasqueradingAsCUDA(
        stream.address ? c10::hip::getStreamFromExternalMasqueradingAsCUDA(static_cast<hipStream_t>(stream.address), current.device_index())
                       : c10::hip::getDefaultHIPStreamMasqueradingAsCUDA(current.device_index()));
    at::Tensor t = at::empty(sizes, options);
    if (returned) t.record_stream(current.unwrap());
    return t;
}

// Native calls of the decoder operators (torch_decode.cpp)
PyObject *cache_append(PyObject *, PyObject *const *args, Py_ssize_t n);
PyObject *cache_read(PyObject *, PyObject *const *args, Py_ssize_t n);
PyObject *attention_cached(PyObject *, PyObject *const *args, Py_ssize_t n);
PyObject *attention_prompt(PyObject *, PyObject *const *args, Py_ssize_t n);
PyObject *verify(PyObject *, PyObject *const *args, Py_ssize_t n);

} // namespace apgemv_torch
#endif
