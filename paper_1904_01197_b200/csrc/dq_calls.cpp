// Python calls of the device entry points: unpacks tensors, messages and integers and calls the C ABI.
//
// A ctypes call of an encoder costs 9 us of Python (attribute look-ups on three tensors, a Stream object, nine
// argument conversions), five times what the library call itself takes; a kernel for a small gradient is done in
// less.  Here the same work takes 0.3 us for an encode, and 0.4 us plus 0.1 us per message for a decode.  The GIL is
// released around the library call, which may block while the stream's launch queue is full.  A list of gradients costs
// 14 ns per tensor, and 9 more where it is written.
//
// Every function returns the dq_status; errors of the arguments' types raise TypeError, as the ctypes calls do.  What torch
// throws while a tensor is looked at (one under vmap has no storage, for instance) is raised as the Python exception
// that the tensor's own methods raise.
#include <Python.h>

#include <ATen/core/grad_mode.h>
#include <ATen/ops/empty.h>
#include <c10/core/InferenceMode.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <optional>
#include <vector>

#include "dq.h"

namespace {

PyObject *s_packed, *s_scale, *s_seed, *s_worker, *s_kind, *s_params, *s_cuda_stream;

// An owned reference.
struct Ref {
    PyObject* v;
    explicit Ref(PyObject* owned) : v(owned) {}
    ~Ref() { Py_XDECREF(v); }
    Ref(const Ref&) = delete;
    Ref& operator=(const Ref&) = delete;
};

// The GIL is released while one of these lives.
struct WithoutGil {
    PyThreadState* state = PyEval_SaveThread();
    ~WithoutGil() { PyEval_RestoreThread(state); }
};

const char* type_name(at::ScalarType t)
{
    return t == at::kFloat ? "torch.float32" : t == at::kInt ? "torch.int32" : t == at::kLong ? "torch.int64"
                                                                                             : "torch.uint8";
}

// Address of a contiguous CUDA tensor of the given type; None is a null pointer, which the library judges -- but not where
// the call's length is the tensor's (`numel` given).  False: an exception is set.
bool device_pointer(PyObject* o, at::ScalarType type, const char* what, void** out, int64_t* numel = nullptr)
{
    *out = nullptr;
    if (o == Py_None && !numel) return true;
    if (THPVariable_Check(o)) {
        const at::Tensor& t = THPVariable_Unpack(o);
        if (t.is_cuda() && t.is_contiguous() && t.scalar_type() == type) {
            *out = t.data_ptr();
            if (numel) *numel = t.numel();
            return true;
        }
    }
    PyErr_Format(PyExc_TypeError, "%s: expected a contiguous CUDA tensor of %s", what, type_name(type));
    return false;
}

// Integers wrap to their width, as ctypes converts them.
bool as_u64(PyObject* o, uint64_t* out)
{
    *out = PyLong_AsUnsignedLongLongMask(o);
    return !(*out == (uint64_t)-1 && PyErr_Occurred());
}

bool as_u32(PyObject* o, uint32_t* out)
{
    uint64_t v;
    if (!as_u64(o, &v)) return false;
    *out = (uint32_t)v;
    return true;
}

bool as_params(PyObject* o, dq_params* out)
{
    Py_buffer b;
    if (PyObject_GetBuffer(o, &b, PyBUF_SIMPLE) != 0) return false;
    const bool fits = b.len == (Py_ssize_t)sizeof(dq_params);
    if (fits) memcpy(out, b.buf, sizeof(dq_params));
    PyBuffer_Release(&b);
    if (!fits) PyErr_SetString(PyExc_TypeError, "params: expected a DqParams");
    return fits;
}

// None: the current device's current stream; else an object with a cuda_stream address.
bool as_stream(PyObject* o, void** out)
{
    if (o == Py_None) {
        *out = c10::cuda::getCurrentCUDAStream().stream();
        return true;
    }
    Ref a(PyObject_GetAttr(o, s_cuda_stream));
    uint64_t v;
    if (!a.v || !as_u64(a.v, &v)) return false;
    *out = reinterpret_cast<void*>(v);
    return true;
}

bool as_message(PyObject* o, dq_msg* m)
{
    void* p;
    uint32_t kind;
    {
        Ref a(PyObject_GetAttr(o, s_packed));
        if (!a.v || !device_pointer(a.v, at::kInt, "packed", &p)) return false;
        m->packed = static_cast<const uint32_t*>(p);
    }
    {
        Ref a(PyObject_GetAttr(o, s_scale));
        if (!a.v || !device_pointer(a.v, at::kFloat, "scale", &p)) return false;
        m->scale = static_cast<const float*>(p);
    }
    Ref seed(PyObject_GetAttr(o, s_seed));
    if (!seed.v) return false;
    Ref worker(PyObject_GetAttr(o, s_worker));
    if (!worker.v) return false;
    Ref k(PyObject_GetAttr(o, s_kind));
    if (!k.v) return false;
    Ref params(PyObject_GetAttr(o, s_params));
    if (!params.v) return false;
    if (!as_u64(seed.v, &m->seed) || !as_u32(worker.v, &m->worker) || !as_u32(k.v, &kind)) return false;
    m->kind = static_cast<dq_kind>(kind);
    return as_params(params.v, &m->p);
}

PyObject* wrong_count(const char* name)
{
    PyErr_Format(PyExc_TypeError, "%s: wrong number of arguments", name);
    return nullptr;
}

// encode(kind, grad, first_element, seed, worker, step, params, out_packed, out_scale, stream); -1: an output buffer is
// too small.
PyObject* encode(PyObject*, PyObject* const* a, Py_ssize_t n_args)
{
    if (n_args != 10) return wrong_count("encode");
    uint32_t kind, worker;
    uint64_t first, seed, step;
    int64_t n = 0, have_words = 0, have_scales = 0;
    void *grad, *packed, *scale, *stream;
    dq_params p;
    if (!as_u32(a[0], &kind) || !device_pointer(a[1], at::kFloat, "grad", &grad, &n) || !as_u64(a[2], &first) ||
        !as_u64(a[3], &seed) || !as_u32(a[4], &worker) || !as_u64(a[5], &step) || !as_params(a[6], &p) ||
        !device_pointer(a[7], at::kInt, "out_packed", &packed, &have_words) ||
        !device_pointer(a[8], at::kFloat, "out_scale", &scale, &have_scales) || !as_stream(a[9], &stream))
        return nullptr;
    if ((uint64_t)have_words < dq_packed_words((uint64_t)n, p.bits) ||
        (uint64_t)have_scales < dq_num_buckets((uint64_t)n, p.bucket))
        return PyLong_FromLong(-1);
    dq_status s;
    {
        WithoutGil released;
        s = (kind == DQ_KIND_DQSG ? dqsg_encode_range : ndqsg_encode_range)(
            static_cast<const float*>(grad), (uint64_t)n, first, seed, worker, step, &p, static_cast<uint32_t*>(packed),
            static_cast<float*>(scale), stream);
    }
    return PyLong_FromLong(s);
}

enum Decode : uint32_t { kDqsg = 0, kNdqsg = 1, kRange = 2, kHalfDithered = 3, kRunning = 4, kSideFirst = 5 };

// decode(how, msgs, n, first_element, step, side_info, out_avg, status_word, stream)
PyObject* decode(PyObject*, PyObject* const* a, Py_ssize_t n_args)
{
    if (n_args != 9) return wrong_count("decode");
    uint32_t how;
    uint64_t n, first, step;
    void *side, *out, *status, *stream;
    if (!as_u32(a[0], &how) || !as_u64(a[2], &n) || !as_u64(a[3], &first) || !as_u64(a[4], &step) ||
        !device_pointer(a[5], at::kFloat, "side_info", &side) || !device_pointer(a[6], at::kFloat, "out_avg", &out) ||
        !device_pointer(a[7], at::kInt, "status_word", &status) || !as_stream(a[8], &stream))
        return nullptr;
    Ref seq(PySequence_Tuple(a[1]));         // (a list could change while its messages' attributes are read)
    if (!seq.v) return nullptr;
    const Py_ssize_t W = PyTuple_GET_SIZE(seq.v);
    dq_msg few[DQ_MAX_WORKERS];
    std::vector<dq_msg> many;
    dq_msg* m = few;
    if (W > (Py_ssize_t)DQ_MAX_WORKERS) {
        many.resize((size_t)W);
        m = many.data();
    }
    for (Py_ssize_t w = 0; w < W; ++w) {
        if (!as_message(PyTuple_GET_ITEM(seq.v, w), m + w)) return nullptr;
    }
    float* o = static_cast<float*>(out);
    uint32_t* st = static_cast<uint32_t*>(status);
    dq_status s = DQ_ERR_INVALID_ARG;
    {
        WithoutGil released;
        switch (how) {
            case kDqsg: s = dqsg_decode_aggregate(m, (uint32_t)W, n, step, o, stream); break;
            case kNdqsg:
                s = ndqsg_decode_aggregate(m, (uint32_t)W, n, step, static_cast<const float*>(side), o, st, stream);
                break;
            case kRange:
                s = ndqsg_decode_aggregate_range(m, (uint32_t)W, n, first, step, static_cast<const float*>(side), o, st,
                                                 stream);
                break;
            case kHalfDithered: s = dqsg_decode_aggregate_half_dithered(m, (uint32_t)W, n, o, stream); break;
            case kRunning: s = ndqsg_decode_aggregate_running(m, (uint32_t)W, n, step, o, st, stream); break;
            case kSideFirst: s = ndqsg_decode_aggregate_side_first(m, (uint32_t)W, n, step, o, st, stream); break;
            default: break;
        }
    }
    return PyLong_FromLong(s);
}

// code_histogram(packed, n, bits, hist, stream)
PyObject* code_histogram(PyObject*, PyObject* const* a, Py_ssize_t n_args)
{
    if (n_args != 5) return wrong_count("code_histogram");
    uint64_t n;
    uint32_t bits;
    void *packed, *hist, *stream;
    if (!device_pointer(a[0], at::kInt, "packed", &packed) || !as_u64(a[1], &n) || !as_u32(a[2], &bits) ||
        !device_pointer(a[3], at::kLong, "hist", &hist) || !as_stream(a[4], &stream))
        return nullptr;
    dq_status s;
    {
        WithoutGil released;
        s = dq_code_histogram(static_cast<const uint32_t*>(packed), n, bits, static_cast<uint64_t*>(hist), stream);
    }
    return PyLong_FromLong(s);
}

// ternary_pack(packed, n, out, status_word, stream)
PyObject* ternary_pack(PyObject*, PyObject* const* a, Py_ssize_t n_args)
{
    if (n_args != 5) return wrong_count("ternary_pack");
    uint64_t n;
    void *packed, *out, *status, *stream;
    if (!device_pointer(a[0], at::kInt, "packed", &packed) || !as_u64(a[1], &n) ||
        !device_pointer(a[2], at::kByte, "out", &out) || !device_pointer(a[3], at::kInt, "status_word", &status) ||
        !as_stream(a[4], &stream))
        return nullptr;
    dq_status s;
    {
        WithoutGil released;
        s = dq_ternary_pack(static_cast<const uint32_t*>(packed), n, static_cast<uint8_t*>(out),
                            static_cast<uint32_t*>(status), stream);
    }
    return PyLong_FromLong(s);
}

// ternary_unpack(data, n, out, stream)
PyObject* ternary_unpack(PyObject*, PyObject* const* a, Py_ssize_t n_args)
{
    if (n_args != 4) return wrong_count("ternary_unpack");
    uint64_t n;
    void *data, *out, *stream;
    if (!device_pointer(a[0], at::kByte, "data", &data) || !as_u64(a[1], &n) ||
        !device_pointer(a[2], at::kInt, "out", &out) || !as_stream(a[3], &stream))
        return nullptr;
    dq_status s;
    {
        WithoutGil released;
        s = dq_ternary_unpack(static_cast<const uint8_t*>(data), n, static_cast<uint32_t*>(out), stream);
    }
    return PyLong_FromLong(s);
}

// ------------------------------------------------------------------------------------------ gradients of many tensors
// A tensor that a call is about to write.  No graph could tell of it: where torch would record one, a tensor that requires a
// gradient is refused, as torch's own out= and in-place operations refuse it, and an inference tensor wherever it may not
// be written.  False: an exception is set.
bool may_be_written(const at::Tensor& t, const char* what)
{
    if (t.requires_grad() && at::GradMode::is_enabled())
        PyErr_Format(PyExc_RuntimeError, "%s: a tensor that requires a gradient is written under torch.no_grad() only", what);
    else if (t.is_inference() && !c10::InferenceMode::is_enabled())
        PyErr_Format(PyExc_RuntimeError, "%s: an inference tensor is written under torch.inference_mode() only", what);
    else
        return true;
    return false;
}

// Autograd notices that a tensor it has saved was written.  (None: nothing was.)
void mark_written(const at::Tensor& t) { t.unsafeGetTensorImpl()->bump_version(); }
void mark_written(PyObject* o)
{
    if (o != Py_None) mark_written(THPVariable_Unpack(o));
}

// What the library refuses, it has not touched.
bool was_refused(dq_status s) { return s != DQ_OK && s != DQ_ERR_CUDA; }

// Which elements a tensor's description has to keep in order.
enum class Order { kNone, kRows };

// Rows of contiguous elements at one distance, in the tensor's own order.  False: its strides are of another kind.
bool as_rows(const at::Tensor& t, dq_tensor* d)
{
    d->row = d->row_stride = 0;
    if (t.is_contiguous() || d->n == 0) return true;
    const auto sizes = t.sizes(), strides = t.strides();
    int64_t i = t.dim() - 1, row = 1;
    for (; i >= 0 && (sizes[i] == 1 || strides[i] == row); --i) row *= sizes[i];
    if (i < 0) return true;
    const int64_t step = strides[i];
    if (step < row) return false;
    int64_t rows = sizes[i];
    for (--i; i >= 0; --i) {
        if (sizes[i] == 1) continue;
        if (strides[i] != step * rows) return false;
        rows *= sizes[i];
    }
    d->row = (uint64_t)row;
    d->row_stride = (uint64_t)step;
    return true;
}

// Whether a call reads a tensor or writes it.
enum class Use { kRead, kWrite };

// A gradient tensor.  Where the order of its elements does not matter, any dense tensor is contiguous.  All tensors of a
// call lie on one device.  False: an exception is set.
bool as_gradient(PyObject* o, const char* what, Order order, Use use, c10::DeviceIndex* device, dq_tensor* d)
{
    if (!THPVariable_Check(o)) {
        PyErr_Format(PyExc_TypeError, "%s: expected CUDA tensors", what);
        return false;
    }
    const at::Tensor& t = THPVariable_Unpack(o);
    const at::ScalarType type = t.scalar_type();
    if (!t.is_cuda() || t.layout() != at::kStrided || t.is_neg() ||
        (type != at::kFloat && type != at::kBFloat16 && type != at::kHalf)) {
        PyErr_Format(PyExc_TypeError, "%s: expected strided CUDA tensors of torch.float32, torch.bfloat16 or torch.float16",
                     what);
        return false;
    }
    if (*device >= 0 && t.get_device() != *device) {
        PyErr_Format(PyExc_TypeError, "%s: the tensors of a call lie on one device", what);
        return false;
    }
    *device = t.get_device();
    if (use == Use::kWrite && !may_be_written(t, what)) return false;
    d->data = t.data_ptr();
    d->n = (uint64_t)t.numel();
    d->dtype = type == at::kFloat ? DQ_F32 : type == at::kBFloat16 ? DQ_BF16 : DQ_F16;
    d->reserved = 0;
    d->row = d->row_stride = 0;
    if (order == Order::kNone && t.is_non_overlapping_and_dense()) return true;
    if (as_rows(t, d)) return true;
    PyErr_Format(PyExc_TypeError, "%s: a tensor of strides that are not rows of contiguous elements at one distance", what);
    return false;
}

// A list or tuple of gradients; `seq` keeps the tensors for the call.
struct GradientList {
    PyObject* seq = nullptr;
    std::vector<dq_tensor> t;
    ~GradientList() { Py_XDECREF(seq); }

    bool take(PyObject* o, const char* what, Order order, Use use, c10::DeviceIndex* device)
    {
        if (THPVariable_Check(o)) {
            PyErr_Format(PyExc_TypeError, "%s: expected a list of tensors", what);
            return false;
        }
        seq = PySequence_Tuple(o);           // (a list could change while it is read)
        if (!seq) return false;
        const Py_ssize_t count = PyTuple_GET_SIZE(seq);
        t.resize((size_t)count);
        for (Py_ssize_t i = 0; i < count; ++i) {
            // A program does other things between two calls: a long list's tensors are no longer in the nearest caches (norm of
            // 2000 in turn with other lists 60 us, 55 with these).
            if (i + 12 < count) __builtin_prefetch(PyTuple_GET_ITEM(seq, i + 12));
            if (i + 6 < count && THPVariable_Check(PyTuple_GET_ITEM(seq, i + 6))) {
                const char* next = reinterpret_cast<const char*>(THPVariable_Unpack(PyTuple_GET_ITEM(seq, i + 6)).unsafeGetTensorImpl());
                for (int line = 0; line < 192; line += 64) __builtin_prefetch(next + line);
            }
            if (!as_gradient(PyTuple_GET_ITEM(seq, i), what, order, use, device, &t[(size_t)i])) return false;
        }
        return true;
    }
    const at::Tensor& tensor(size_t i) const { return THPVariable_Unpack(PyTuple_GET_ITEM(seq, (Py_ssize_t)i)); }
    uint32_t count() const { return (uint32_t)std::min<size_t>(t.size(), UINT32_MAX); }
    uint64_t total() const
    {
        uint64_t n = 0;
        for (const dq_tensor& x : t) n += x.n;
        return n;
    }
    void mark_all_written() const
    {
        for (size_t i = 0; i < t.size(); ++i) mark_written(tensor(i));
    }
};

// A contiguous tensor of at least `least` elements on the call's device; None is a null pointer.
bool buffer_pointer(PyObject* o, at::ScalarType type, const char* what, Use use, uint64_t least, c10::DeviceIndex* device,
                    void** out)
{
    int64_t have = 0;
    *out = nullptr;
    if (o == Py_None) return true;
    if (!device_pointer(o, type, what, out, &have)) return false;
    const c10::DeviceIndex on = THPVariable_Unpack(o).get_device();
    if (*device >= 0 && on != *device) {
        PyErr_Format(PyExc_TypeError, "%s: the tensors of a call lie on one device", what);
        return false;
    }
    *device = on;
    if ((uint64_t)have < least) {
        PyErr_Format(PyExc_ValueError, "%s: too small", what);
        return false;
    }
    return use == Use::kRead || may_be_written(THPVariable_Unpack(o), what);
}

// The call's device is current while one of these lives, the stream is resolved on it (None: its current stream), and the
// workspace belongs to that stream.
struct OnDevice {
    std::optional<c10::cuda::CUDAGuard> guard;
    std::optional<at::Tensor> memory;
    void* stream = nullptr;
    void* workspace = nullptr;

    bool enter(c10::DeviceIndex device, PyObject* s)
    {
        if (device >= 0) guard.emplace(device);
        return as_stream(s, &stream);
    }
    void allocate(uint64_t bytes)
    {
        if (bytes == 0) return;
        const c10::DeviceIndex device = c10::cuda::current_device();
        c10::cuda::CUDAStreamGuard on(c10::cuda::getStreamFromExternal(static_cast<cudaStream_t>(stream), device));
        memory = at::empty({(int64_t)bytes}, at::TensorOptions().dtype(at::kByte).device(at::kCUDA, device));
        workspace = memory->data_ptr();
    }
};

// kind, norm, out_norm, status_word and max_norm of a call (None: nothing is clipped).
bool as_clip(PyObject* max_norm, PyObject* norm, PyObject* kind, PyObject* out_norm, PyObject* status,
             c10::DeviceIndex* device, dq_clip* clip, bool* clips)
{
    void *given, *out, *st;
    uint32_t k;
    if (!as_u32(kind, &k) || !buffer_pointer(norm, at::kFloat, "norm", Use::kRead, 1, device, &given) ||
        !buffer_pointer(out_norm, at::kFloat, "out_norm", Use::kWrite, 1, device, &out) ||
        !buffer_pointer(status, at::kInt, "status_word", Use::kWrite, 1, device, &st))
        return false;
    *clips = max_norm != Py_None;
    clip->max_norm = 0.0f;
    if (*clips) {
        const double limit = PyFloat_AsDouble(max_norm);
        if (limit == -1.0 && PyErr_Occurred()) return false;
        clip->max_norm = (float)limit;
    } else if (given || out || st) {
        PyErr_SetString(PyExc_ValueError, "norm, out_norm and status_word go with max_norm");
        return false;
    }
    clip->kind = static_cast<dq_norm>(k);
    clip->norm = static_cast<const float*>(given);
    clip->out_norm = static_cast<float*>(out);
    clip->status_word = static_cast<uint32_t*>(st);
    return true;
}

// The flat vector of a gather or scatter.
bool as_flat(PyObject* o, const char* what, Use use, uint64_t total, c10::DeviceIndex* device, void** out)
{
    if (o == Py_None) {
        PyErr_Format(PyExc_TypeError, "%s: expected a contiguous CUDA tensor of torch.float32", what);
        return false;
    }
    if (!buffer_pointer(o, at::kFloat, what, use, total, device, out)) return false;
    if (total != 0 && (uint64_t)THPVariable_Unpack(o).numel() != total) {
        PyErr_Format(PyExc_ValueError, "%s: has %lld elements, the list has %llu", what,
                     (long long)THPVariable_Unpack(o).numel(), (unsigned long long)total);
        return false;
    }
    return true;
}

// grad_norm(grads, kind, out_norm, out_norms, status_word, stream)
PyObject* grad_norm(PyObject*, PyObject* const* a, Py_ssize_t n_args)
{
    if (n_args != 6) return wrong_count("grad_norm");
    c10::DeviceIndex device = -1;
    GradientList g;
    uint32_t kind;
    void *norm, *norms, *status;
    OnDevice on;
    if (!g.take(a[0], "grads", Order::kNone, Use::kRead, &device) || !as_u32(a[1], &kind) ||
        !buffer_pointer(a[2], at::kFloat, "out_norm", Use::kWrite, 1, &device, &norm) ||
        !buffer_pointer(a[3], at::kFloat, "out_norms", Use::kWrite, g.t.size(), &device, &norms) ||
        !buffer_pointer(a[4], at::kInt, "status_word", Use::kWrite, 1, &device, &status) || !on.enter(device, a[5]))
        return nullptr;
    on.allocate(dq_grad_workspace_bytes(g.t.data(), g.count(), norms != nullptr));
    dq_status s;
    {
        WithoutGil released;
        s = dq_grad_norm(g.t.data(), g.count(), static_cast<dq_norm>(kind), static_cast<float*>(norm),
                         static_cast<float*>(norms), static_cast<uint32_t*>(status), on.workspace,
                         on.memory ? (uint64_t)on.memory->numel() : 0, on.stream);
    }
    if (!was_refused(s)) {
        for (int i = 2; i < 5; ++i) mark_written(a[i]);
    }
    return PyLong_FromLong(s);
}

// grad_clip(grads, max_norm, out, norm, kind, out_norm, status_word, stream)
PyObject* grad_clip(PyObject*, PyObject* const* a, Py_ssize_t n_args)
{
    if (n_args != 8) return wrong_count("grad_clip");
    c10::DeviceIndex device = -1;
    const bool in_place = a[2] == Py_None;
    GradientList g, o;
    dq_clip clip;
    bool clips;
    OnDevice on;
    if (a[1] == Py_None) {
        PyErr_SetString(PyExc_TypeError, "max_norm: expected a number");
        return nullptr;
    }
    if (!g.take(a[0], "grads", Order::kNone, in_place ? Use::kWrite : Use::kRead, &device)) return nullptr;
    if (!in_place) {
        if (!o.take(a[2], "out", Order::kNone, Use::kWrite, &device)) return nullptr;
        if (o.t.size() != g.t.size()) {
            PyErr_SetString(PyExc_ValueError, "out: one tensor for each of grads");
            return nullptr;
        }
        for (size_t i = 0; i < g.t.size(); ++i) {
            const at::Tensor &x = g.tensor(i), &y = o.tensor(i);
            if (x.sizes() != y.sizes()) {
                PyErr_SetString(PyExc_ValueError, "out: a tensor of another shape than its gradient");
                return nullptr;
            }
            if ((x.is_contiguous() && y.is_contiguous()) ||
                (x.strides() == y.strides() && g.t[i].row == 0 && o.t[i].row == 0))
                continue;
            // the two are walked in the order of their indices
            if (!as_rows(x, &g.t[i]) || !as_rows(y, &o.t[i])) {
                PyErr_SetString(PyExc_TypeError,
                                "out: a tensor or its gradient has strides that are not rows of contiguous elements at one "
                                "distance");
                return nullptr;
            }
        }
    }
    if (!as_clip(a[1], a[3], a[4], a[5], a[6], &device, &clip, &clips) || !on.enter(device, a[7])) return nullptr;
    if (!clip.norm) on.allocate(dq_grad_workspace_bytes(g.t.data(), g.count(), 0));
    dq_status s;
    {
        WithoutGil released;
        s = dq_grad_clip(g.t.data(), g.count(), &clip, in_place ? nullptr : o.t.data(), on.workspace,
                         on.memory ? (uint64_t)on.memory->numel() : 0, on.stream);
    }
    if (!was_refused(s)) {
        (in_place ? g : o).mark_all_written();
        mark_written(a[5]);
        mark_written(a[6]);
    }
    return PyLong_FromLong(s);
}

// grad_gather(grads, out_flat, max_norm, norm, kind, out_norm, status_word, stream)
PyObject* grad_gather(PyObject*, PyObject* const* a, Py_ssize_t n_args)
{
    if (n_args != 8) return wrong_count("grad_gather");
    c10::DeviceIndex device = -1;
    GradientList g;
    dq_clip clip;
    bool clips;
    void* flat;
    OnDevice on;
    if (!g.take(a[0], "grads", Order::kRows, Use::kRead, &device) ||
        !as_flat(a[1], "out_flat", Use::kWrite, g.total(), &device, &flat) ||
        !as_clip(a[2], a[3], a[4], a[5], a[6], &device, &clip, &clips) || !on.enter(device, a[7]))
        return nullptr;
    if (clips && !clip.norm) on.allocate(dq_grad_workspace_bytes(g.t.data(), g.count(), 0));
    dq_status s;
    {
        WithoutGil released;
        s = dq_grad_gather(g.t.data(), g.count(), clips ? &clip : nullptr, static_cast<float*>(flat), on.workspace,
                           on.memory ? (uint64_t)on.memory->numel() : 0, on.stream);
    }
    if (!was_refused(s)) {
        for (int i : {1, 5, 6}) mark_written(a[i]);
    }
    return PyLong_FromLong(s);
}

// grad_scatter(flat, out, max_norm, norm, kind, out_norm, status_word, stream)
PyObject* grad_scatter(PyObject*, PyObject* const* a, Py_ssize_t n_args)
{
    if (n_args != 8) return wrong_count("grad_scatter");
    c10::DeviceIndex device = -1;
    GradientList o;
    dq_clip clip;
    bool clips;
    void* flat;
    OnDevice on;
    if (!o.take(a[1], "out", Order::kRows, Use::kWrite, &device) ||
        !as_flat(a[0], "flat", Use::kRead, o.total(), &device, &flat) ||
        !as_clip(a[2], a[3], a[4], a[5], a[6], &device, &clip, &clips) || !on.enter(device, a[7]))
        return nullptr;
    if (clips && !clip.norm) on.allocate(dq_grad_workspace_bytes(o.t.data(), o.count(), 0));
    dq_status s;
    {
        WithoutGil released;
        s = dq_grad_scatter(static_cast<const float*>(flat), clips ? &clip : nullptr, o.t.data(), o.count(), on.workspace,
                            on.memory ? (uint64_t)on.memory->numel() : 0, on.stream);
    }
    if (!was_refused(s)) {
        o.mark_all_written();
        mark_written(a[5]);
        mark_written(a[6]);
    }
    return PyLong_FromLong(s);
}

// No C++ exception may leave through the interpreter's C frames.
template <PyObject* (*F)(PyObject*, PyObject* const*, Py_ssize_t)>
PyObject* guarded(PyObject* self, PyObject* const* a, Py_ssize_t n_args)
{
    HANDLE_TH_ERRORS
    return F(self, a, n_args);
    END_HANDLE_TH_ERRORS
}

#define DQ_METHOD(f) {#f, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(guarded<f>)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {DQ_METHOD(encode),       DQ_METHOD(decode),         DQ_METHOD(code_histogram),
                         DQ_METHOD(ternary_pack), DQ_METHOD(ternary_unpack), DQ_METHOD(grad_norm),
                         DQ_METHOD(grad_clip),    DQ_METHOD(grad_gather),    DQ_METHOD(grad_scatter),
                         {nullptr, nullptr, 0, nullptr}};
#undef DQ_METHOD

PyModuleDef module = {PyModuleDef_HEAD_INIT, "dq_calls", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit_dq_calls()
{
    s_packed = PyUnicode_InternFromString("packed");
    s_scale = PyUnicode_InternFromString("scale");
    s_seed = PyUnicode_InternFromString("seed");
    s_worker = PyUnicode_InternFromString("worker");
    s_kind = PyUnicode_InternFromString("kind");
    s_params = PyUnicode_InternFromString("params");
    s_cuda_stream = PyUnicode_InternFromString("cuda_stream");
    return PyModule_Create(&module);
}
