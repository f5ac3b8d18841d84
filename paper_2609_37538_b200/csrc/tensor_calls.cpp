// avsg_append and avsg_attend with torch's tensors as arguments: their checks, the outputs' allocation and the argument block
// in native code, since the host bounds the small calls.  Host time of a queued attend(), marshalled in Python / here:
// 14.6 / 6.0 us, of an append() 9.6 / 3.9.
//
// Handled here: plain tensors (no subclass) of the documented types, shapes and places, and for append() a cache in one CUDA tensor
// without row_stride or kv_rows.  Anything else answers NotImplemented, and the binding's own conversions decide what is accepted and
// what is raised: a list of caches, as avsg_step takes them, and a cache in pinned memory too (52 us for an append() to 64 of them, 12 to one).
#include <ATen/ops/empty.h>
#include <c10/cuda/CUDACachingAllocator.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cmath>
#include <limits>
#include <vector>

#include "avsg.h"

namespace {

using AppendFn = int (*)(avsg_ctx*, const avsg_append_args*, void*);
using AttendFn = int (*)(avsg_ctx*, const avsg_attend_args*, void*);
AppendFn append_fn;
AttendFn attend_fn;

using BytesFn = uint32_t (*)(uint32_t);
BytesFn row_bytes;

PyObject* not_handled() { Py_RETURN_NOTIMPLEMENTED; }

const at::Tensor* tensor(PyObject* o)
{
    if (!THPVariable_CheckExact(o)) return nullptr;
    const at::Tensor& t = THPVariable_Unpack(o);
    return t.layout() == at::kStrided && t.has_storage() && !t.is_neg() && !t.is_conj() ? &t : nullptr;
}

// A CUDA tensor of `dims` dimensions with its last numbers side by side.
const at::Tensor* strided(PyObject* o, at::ScalarType type, int64_t dims)
{
    const at::Tensor* t = tensor(o);
    return t && t->is_cuda() && t->scalar_type() == type && t->dim() == dims && t->stride(dims - 1) == 1 ? t : nullptr;
}

// The address of a contiguous tensor of that type and shape on that device; 0 for None.  False: something else.
bool packed(PyObject* o, at::ScalarType type, at::IntArrayRef shape, c10::DeviceIndex device, uint64_t* at)
{
    *at = 0;
    if (o == Py_None) return true;
    const at::Tensor* t = tensor(o);
    if (!t || !t->is_cuda() || t->get_device() != device || t->scalar_type() != type || t->sizes() != shape || !t->is_contiguous()) return false;
    *at = reinterpret_cast<uint64_t>(t->data_ptr());
    return true;
}

// Bytes between the elements of the first dimensions (one of a single element may have any stride).
void steps(const at::Tensor& t, int dims, uint64_t* out)
{
    for (int i = 0; i < dims; ++i) out[i] = t.size(i) > 1 ? (uint64_t)t.stride(i) * t.element_size() : 0;
}

bool fits(int64_t v) { return v >= 0 && v <= (int64_t)std::numeric_limits<uint32_t>::max(); }

bool word(PyObject* o, uint32_t* v)
{
    if (!PyLong_CheckExact(o)) return false;
    int over = 0;
    const long long x = PyLong_AsLongLongAndOverflow(o, &over);
    *v = (uint32_t)x;
    return !over && fits(x);
}
bool address(PyObject* o, uint64_t* v)                              // an integer, or None: 0
{
    *v = 0;
    if (o == Py_None) return true;
    if (!PyLong_CheckExact(o)) return false;
    *v = PyLong_AsUnsignedLongLong(o);
    if (!PyErr_Occurred()) return true;
    PyErr_Clear();
    return false;
}
bool number(PyObject* o, float* v)
{
    double d;
    if (PyFloat_CheckExact(o)) {
        d = PyFloat_AS_DOUBLE(o);
    } else {
        uint32_t w;
        if (!word(o, &w)) return false;
        d = w;
    }
    *v = (float)d;
    return std::isfinite(*v);
}
bool tables(PyObject* o, int64_t n, std::vector<uint32_t>* out)
{
    if ((!PyList_CheckExact(o) && !PyTuple_CheckExact(o)) || PySequence_Fast_GET_SIZE(o) != n) return false;
    out->resize(n);
    for (int64_t i = 0; i < n; ++i)
        if (!word(PySequence_Fast_GET_ITEM(o, i), out->data() + i)) return false;
    return true;
}
// The stream of a call whose tensors lie on `device`: by default that device's current one.
bool stream_of(PyObject* o, c10::DeviceIndex device, uint64_t* v)
{
    if (o != Py_None) return address(o, v);
    *v = reinterpret_cast<uint64_t>(c10::cuda::getCurrentCUDAStream(device).stream());
    return true;
}

// An output of a call on that stream.  Its block is one of that stream's (another stream's may still be in use by what is queued
// there), and when the tensor is dropped it waits for what the current stream has queued by then, which reads it.
at::Tensor output(at::IntArrayRef shape, at::ScalarType type, const at::Tensor& like, uint64_t stream)
{
    const at::TensorOptions options = at::TensorOptions(type).device(like.device());
    const c10::cuda::CUDAStream current = c10::cuda::getCurrentCUDAStream(like.get_device());
    if (reinterpret_cast<uint64_t>(current.stream()) == stream) return at::empty(shape, options);
    at::Tensor t;
    {
        // (1: the handle that CUDA itself has for the default stream)
        c10::cuda::CUDAStreamGuard guard(stream <= 1 ? c10::cuda::getDefaultCUDAStream(like.get_device())
                                                     : c10::cuda::getStreamFromExternal(reinterpret_cast<cudaStream_t>(stream), like.get_device()));
        t = at::empty(shape, options);
    }
    c10::cuda::CUDACachingAllocator::recordStream(t.storage().data_ptr(), current);
    return t;
}

// Answers (code, result): a code of avsg.h and the call's result.
PyObject* answer(int rc, PyObject* result)
{
    if (!result) return nullptr;
    PyObject* code = PyLong_FromLong(rc);
    PyObject* both = code ? PyTuple_Pack(2, code, result) : nullptr;
    Py_XDECREF(code);
    Py_DECREF(result);
    return both;
}

// ctx, table_ids, q, buffer, slots, row_format, scale, out, lse, want_lse, softcap, ids, positions, spans, slopes, rope, status, stream
PyObject* attend(PyObject*, PyObject* const* a, Py_ssize_t nargs)
{
    if (nargs != 18 || !attend_fn) return not_handled();
    HANDLE_TH_ERRORS
    const at::Tensor* q = strided(a[2], at::kBFloat16, 4);
    const at::Tensor* slots = tensor(a[4]);
    uint64_t ctx, stream, at, status, rope;
    avsg_attend_args s = {};
    if (!q || !slots || slots->dim() != 3 || q->size(3) != AVSG_LATENT_DIMS + AVSG_ROPE_DIMS || !address(a[0], &ctx)) return not_handled();
    const int64_t n = q->size(0), T = q->size(1), H = q->size(2), K = slots->size(2);
    const c10::DeviceIndex device = q->get_device();
    if (!fits(n) || !fits(T) || !fits(H) || !fits(K) || !word(a[5], &s.row_format)) return not_handled();
    s.n = n; s.n_tokens = T; s.heads = H; s.topk = K;
    std::vector<uint32_t> ids;
    if (a[3] == Py_None) {
        if (!ctx || !tables(a[1], n, &ids)) return not_handled();
        s.table_ids = ids.data();
    } else {
        const at::Tensor* b = strided(a[3], at::kByte, 3);
        if (ctx || a[1] != Py_None || !b || b->get_device() != device || b->size(0) != n || !fits(b->size(1)) ||
            b->size(2) != row_bytes(s.row_format) || (n > 1 && b->size(1) > 1 && b->stride(0) != b->stride(1) * b->size(1)) ||
            (b->size(1) > 1 && b->stride(1) < b->size(2)) || (n > 1 && b->stride(0) < b->size(2)))
            return not_handled();
        s.buffer = b->data_ptr();
        s.buffer_slots = b->size(1);
        // (tables of one row are as far apart as their rows; the stride between rows says nothing then)
        s.buffer_row_bytes = b->size(1) > 1 ? b->stride(1) : n > 1 ? b->stride(0) : 0;
    }
    if (!packed(a[4], at::kInt, {n, T, K}, device, &at) || !at) return not_handled();
    s.slots = reinterpret_cast<const int32_t*>(at);
    s.q = q->data_ptr();
    steps(*q, 3, s.q_stride);
    if (!number(a[6], &s.scale) || !number(a[10], &s.softcap)) return not_handled();
    if (!packed(a[11], at::kInt, {n, T, K}, device, &at)) return not_handled();
    s.ids = reinterpret_cast<const int32_t*>(at);
    if (!packed(a[12], at::kInt, {n, T}, device, &at)) return not_handled();
    s.positions = reinterpret_cast<const int32_t*>(at);
    if (!packed(a[13], at::kInt, {n, T, 2}, device, &at)) return not_handled();
    s.spans = reinterpret_cast<const int32_t*>(at);
    if (!packed(a[14], at::kFloat, {H}, device, &at)) return not_handled();
    s.slopes = reinterpret_cast<const float*>(at);
    if (!address(a[15], &rope) || !address(a[16], &status) || !stream_of(a[17], device, &stream)) return not_handled();
    s.rope = reinterpret_cast<const avsg_rope*>(rope);
    s.status = reinterpret_cast<uint32_t*>(status);
    if (!packed(a[8], at::kFloat, {n, T, H}, device, &at)) return not_handled();
    const bool with_lse = at || a[9] == Py_True;
    at::Tensor out, lse;
    if (a[7] != Py_None) {
        const at::Tensor* o = strided(a[7], at::kBFloat16, 4);
        if (!o || o->get_device() != device || o->sizes() != at::IntArrayRef({n, T, H, (int64_t)AVSG_LATENT_DIMS})) return not_handled();
        out = *o;
    } else {
        out = output({n, T, H, (int64_t)AVSG_LATENT_DIMS}, at::kBFloat16, *q, stream);
    }
    s.out = out.data_ptr();
    steps(out, 3, s.out_stride);
    if (with_lse && !at) {
        lse = output({n, T, H}, at::kFloat, *q, stream);
        at = reinterpret_cast<uint64_t>(lse.data_ptr());
    }
    s.lse = reinterpret_cast<float*>(at);
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = attend_fn(reinterpret_cast<avsg_ctx*>(ctx), &s, reinterpret_cast<void*>(stream));
    Py_END_ALLOW_THREADS
    PyObject* first = a[7] != Py_None ? Py_NewRef(a[7]) : THPVariable_Wrap(out);
    if (!first || !with_lse) return answer(rc, first);
    PyObject* second = a[8] != Py_None ? Py_NewRef(a[8]) : THPVariable_Wrap(lse);
    PyObject* pair = second ? PyTuple_Pack(2, first, second) : nullptr;
    Py_DECREF(first);
    Py_XDECREF(second);
    return answer(rc, pair);
    END_HANDLE_TH_ERRORS
}

// ctx, table_ids, latent, rope_part, positions, kv, row_format, rope, rows, want_values, values, status, stream
PyObject* append(PyObject*, PyObject* const* a, Py_ssize_t nargs)
{
    if (nargs != 13 || !append_fn) return not_handled();
    HANDLE_TH_ERRORS
    const at::Tensor* latent = tensor(a[2]);
    const at::Tensor* kv = tensor(a[5]);
    if (!latent || !latent->is_cuda() || !kv || !kv->is_cuda()) return not_handled();
    const at::ScalarType type = latent->scalar_type();
    const at::Tensor* rope_part = strided(a[3], type, 3);
    avsg_append_args s = {};
    uint64_t ctx, stream, at, status, rope;
    if (type == at::kBFloat16) s.type = AVSG_TYPE_BF16;
    else if (type == at::kHalf) s.type = AVSG_TYPE_FP16;
    else if (type == at::kFloat) s.type = AVSG_TYPE_FP32;
    else return not_handled();
    if (!strided(a[2], type, 3) || !rope_part || !address(a[0], &ctx)) return not_handled();
    const int64_t n = latent->size(0), T = latent->size(1);
    const c10::DeviceIndex device = latent->get_device();
    if (!fits(n) || !fits(T) || n > 2048 || latent->size(2) != AVSG_LATENT_DIMS || rope_part->get_device() != device ||
        rope_part->sizes() != at::IntArrayRef({n, T, (int64_t)AVSG_ROPE_DIMS}) || !word(a[6], &s.row_format))
        return not_handled();
    s.n = n; s.n_tokens = T;
    std::vector<uint32_t> ids;
    if (ctx) {
        if (!tables(a[1], n, &ids)) return not_handled();
        s.table_ids = ids.data();
    } else if (a[1] != Py_None) {
        return not_handled();
    }
    s.latent = latent->data_ptr();
    s.rope_part = rope_part->data_ptr();
    steps(*latent, 2, s.latent_stride);
    steps(*rope_part, 2, s.rope_stride);
    if (!packed(a[4], at::kInt, {n, T}, device, &at) || !at) return not_handled();
    s.positions = reinterpret_cast<const int32_t*>(at);
    if (!packed(a[8], at::kInt, {n, T}, device, &at)) return not_handled();
    s.rows = reinterpret_cast<const int32_t*>(at);
    // the cache: [n, rows, bytes], or [rows, bytes] that all tables share
    const int64_t d = kv->dim(), bytes = row_bytes(s.row_format);
    if ((d != 2 && d != 3) || kv->scalar_type() != at::kByte || kv->get_device() != device || kv->size(d - 1) != bytes || kv->stride(d - 1) != 1 ||
        (d == 3 && kv->size(0) != n) || !fits(kv->size(d - 2)))
        return not_handled();
    s.kv = kv->data_ptr();
    s.kv_table_stride = d == 3 && n > 1 ? kv->stride(0) : 0;
    const std::vector<uint32_t> limits(n, (uint32_t)kv->size(d - 2));
    s.kv_rows = limits.data();
    std::vector<uint64_t> strides;
    if (kv->size(d - 2) > 1 && kv->stride(d - 2) != bytes) {
        strides.assign(n, kv->stride(d - 2));
        s.row_stride = strides.data();
    }
    if (!address(a[7], &rope) || !address(a[11], &status) || !stream_of(a[12], device, &stream)) return not_handled();
    s.rope = reinterpret_cast<const avsg_rope*>(rope);
    s.status = reinterpret_cast<uint32_t*>(status);
    const int64_t wide[3] = {n, T, (int64_t)(AVSG_LATENT_DIMS + AVSG_ROPE_DIMS)};
    if (!packed(a[10], at::kBFloat16, at::IntArrayRef(wide, 3), device, &at)) return not_handled();
    at::Tensor values;
    const bool made = !at && a[10] == Py_None && a[9] == Py_True;
    if (made) {
        values = output(at::IntArrayRef(wide, 3), at::kBFloat16, *latent, stream);
        at = reinterpret_cast<uint64_t>(values.data_ptr());
    }
    s.values = reinterpret_cast<void*>(at);
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = append_fn(reinterpret_cast<avsg_ctx*>(ctx), &s, reinterpret_cast<void*>(stream));
    Py_END_ALLOW_THREADS
    return answer(rc, made ? THPVariable_Wrap(values) : Py_NewRef(a[10]));
    END_HANDLE_TH_ERRORS
}

// addresses of avsg_append, avsg_attend, avsg_row_bytes
PyObject* set_library(PyObject*, PyObject* args)
{
    unsigned long long append_at, attend_at, bytes_at;
    if (!PyArg_ParseTuple(args, "KKK", &append_at, &attend_at, &bytes_at)) return nullptr;
    row_bytes = reinterpret_cast<BytesFn>(bytes_at);
    append_fn = reinterpret_cast<AppendFn>(append_at);
    attend_fn = reinterpret_cast<AttendFn>(attend_at);
    Py_RETURN_NONE;
}

PyMethodDef methods[] = {
    {"append", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(append)), METH_FASTCALL, nullptr},
    {"attend", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(attend)), METH_FASTCALL, nullptr},
    {"set_library", set_library, METH_VARARGS, nullptr},
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_tensor_calls", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__tensor_calls()
{
    PyObject* m = PyModule_Create(&module);
    if (!m || PyModule_AddStringConstant(m, "built_for", BUILT_FOR) < 0) return nullptr;          // (this version of torch)
    return m;
}
