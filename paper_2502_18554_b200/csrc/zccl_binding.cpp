// CPython module over the C boundary for the calls a program makes per message: argument checks and marshalling in
// native code.  A codec call on a small message is a few microseconds of GPU work, so the host's share decides how many
// such calls fit a second: through ctypes and torch's Python-level stream objects a call's marshalling took 5.5 us
// (3.3 us of it the look-up of the current stream), here it takes 0.4 us.  The calls themselves are the C boundary's.
#include <Python.h>

#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/Dtype.h>
#include <torch/csrc/DynamicTypes.h>
#include <torch/csrc/autograd/python_variable.h>

#include <algorithm>
#include <vector>

#include "../../include/zccl.h"

namespace {

// The data pointer of a contiguous CUDA tensor of type `dt`; false with a Python error set otherwise.
bool dev_ptr(PyObject* o, c10::ScalarType dt, void** p, size_t* numel = nullptr)
{
    if (!THPVariable_Check(o)) {
        PyErr_SetString(PyExc_ValueError, "expected a contiguous CUDA tensor");
        return false;
    }
    const at::Tensor& t = THPVariable_Unpack(o);
    if (!t.is_cuda() || !t.is_contiguous()) {
        PyErr_SetString(PyExc_ValueError, "expected a contiguous CUDA tensor");
        return false;
    }
    if (t.scalar_type() != dt) {
        PyErr_Format(PyExc_ValueError, "expected dtype %S, got %S", (PyObject*)torch::getTHPDtype(dt), (PyObject*)torch::getTHPDtype(t.scalar_type()));
        return false;
    }
    *p = t.data_ptr();
    if (numel) *numel = (size_t)t.numel();
    return true;
}
bool opt_dev_ptr(PyObject* o, c10::ScalarType dt, void** p, size_t* numel = nullptr)
{
    *p = nullptr;
    if (numel) *numel = 0;
    return o == Py_None || dev_ptr(o, dt, p, numel);
}
size_t numel_of(PyObject* o)
{
    return THPVariable_Check(o) ? (size_t)THPVariable_Unpack(o).numel() : 1;
}
// An empty input or output tensor need not be anything in particular: it counts as a null pointer.
bool ptr_unless_empty(PyObject* o, c10::ScalarType dt, void** p, size_t* numel)
{
    *p = nullptr;
    *numel = numel_of(o);
    return *numel == 0 || dev_ptr(o, dt, p, numel);
}

bool stream_of(PyObject* o, void** st)
{
    if (o == Py_None) {
        *st = (void*)c10::cuda::getCurrentCUDAStream().stream();
        return true;
    }
    PyObject* h = PyObject_GetAttrString(o, "cuda_stream");
    if (!h) return false;
    *st = PyLong_AsVoidPtr(h);
    Py_DECREF(h);
    return !PyErr_Occurred();
}

zccl_ctx* ctx_of(PyObject* o) { return (zccl_ctx*)PyLong_AsVoidPtr(o); }

bool nargs_are(Py_ssize_t n, Py_ssize_t want)
{
    if (n == want) return true;
    PyErr_Format(PyExc_TypeError, "expected %zd arguments, got %zd", want, n);
    return false;
}

// Runs a boundary call without the interpreter lock and hands its status back.
template <class F>
PyObject* status(F&& f)
{
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = f();
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(rc);
}

using Args = PyObject* const*;

PyObject* current_stream(PyObject*, PyObject*)
{
    return PyLong_FromVoidPtr((void*)c10::cuda::getCurrentCUDAStream().stream());
}

// (ctx, x, eb_mode, eb, out, out_bytes, stream, n)
PyObject* compress(PyObject*, Args a, Py_ssize_t na)
{
    if (!nargs_are(na, 8)) return nullptr;
    zccl_ctx* c = ctx_of(a[0]);
    size_t n = a[7] == Py_None ? numel_of(a[1]) : PyLong_AsSize_t(a[7]), cap;
    const int mode = (int)PyLong_AsLong(a[2]);
    const float eb = (float)PyFloat_AsDouble(a[3]);
    if (PyErr_Occurred()) return nullptr;
    void *x = nullptr, *out, *nb, *st;
    if (n && !dev_ptr(a[1], c10::kFloat, &x)) return nullptr;
    if (!dev_ptr(a[4], c10::kByte, &out, &cap) || !dev_ptr(a[5], c10::kLong, &nb) || !stream_of(a[6], &st)) return nullptr;
    return status([&] { return zccl_compress(c, (const float*)x, n, mode, eb, out, cap, (size_t*)nb, st); });
}

// (ctx, stream_bytes, in_bytes_max, y, stream)
PyObject* decompress(PyObject*, Args a, Py_ssize_t na)
{
    if (!nargs_are(na, 5)) return nullptr;
    zccl_ctx* c = ctx_of(a[0]);
    void *in, *y, *st;
    size_t cap, n;
    if (!dev_ptr(a[1], c10::kByte, &in, &cap)) return nullptr;
    if (a[2] != Py_None) cap = PyLong_AsSize_t(a[2]);
    if (PyErr_Occurred() || !ptr_unless_empty(a[3], c10::kFloat, &y, &n) || !stream_of(a[4], &st)) return nullptr;
    return status([&] { return zccl_decompress(c, in, cap, (float*)y, n, st); });
}

// (ctx, in_c, n, out_c, out_bytes, local, local_c, raw_out, flags, stream)
PyObject* hop(PyObject*, Args a, Py_ssize_t na)
{
    if (!nargs_are(na, 10)) return nullptr;
    zccl_ctx* c = ctx_of(a[0]);
    const size_t n = PyLong_AsSize_t(a[2]);
    const unsigned flags = (unsigned)PyLong_AsUnsignedLong(a[8]);
    if (PyErr_Occurred()) return nullptr;
    void *in, *out, *nb, *local, *local_c, *raw, *st;
    size_t in_cap, out_cap, local_cap;
    if (!dev_ptr(a[1], c10::kByte, &in, &in_cap) || !dev_ptr(a[3], c10::kByte, &out, &out_cap) || !dev_ptr(a[4], c10::kLong, &nb) ||
        !opt_dev_ptr(a[5], c10::kFloat, &local) || !opt_dev_ptr(a[6], c10::kByte, &local_c, &local_cap) ||
        !opt_dev_ptr(a[7], c10::kFloat, &raw) || !stream_of(a[9], &st))
        return nullptr;
    return status([&] {
        return zccl_decompress_reduce_compress(c, in, in_cap, (const float*)local, local_c, local_cap, n, out, out_cap, (size_t*)nb, (float*)raw, flags, st);
    });
}

// (ctx, x, eb_mode, eb, out, out_bytes, stream)
PyObject* compress_f64(PyObject*, Args a, Py_ssize_t na)
{
    if (!nargs_are(na, 7)) return nullptr;
    zccl_ctx* c = ctx_of(a[0]);
    const int mode = (int)PyLong_AsLong(a[2]);
    const double eb = PyFloat_AsDouble(a[3]);
    if (PyErr_Occurred()) return nullptr;
    void *x, *out, *nb, *st;
    size_t n, cap;
    if (!ptr_unless_empty(a[1], c10::kDouble, &x, &n) || !dev_ptr(a[4], c10::kByte, &out, &cap) || !dev_ptr(a[5], c10::kLong, &nb) || !stream_of(a[6], &st))
        return nullptr;
    return status([&] { return zccl_compress_f64(c, (const double*)x, n, mode, eb, out, cap, (size_t*)nb, st); });
}

// (ctx, in_c, y, stream)
PyObject* decompress_f64(PyObject*, Args a, Py_ssize_t na)
{
    if (!nargs_are(na, 4)) return nullptr;
    zccl_ctx* c = ctx_of(a[0]);
    void *in, *y, *st;
    size_t cap, n;
    if (!dev_ptr(a[1], c10::kByte, &in, &cap) || !ptr_unless_empty(a[2], c10::kDouble, &y, &n) || !stream_of(a[3], &st)) return nullptr;
    return status([&] { return zccl_decompress_f64(c, in, cap, (double*)y, n, st); });
}

// (ctx, x, eb_mode, eb, tile, out, out_bytes, stream)
PyObject* compress_tiled(PyObject*, Args a, Py_ssize_t na)
{
    if (!nargs_are(na, 8)) return nullptr;
    zccl_ctx* c = ctx_of(a[0]);
    const int mode = (int)PyLong_AsLong(a[2]);
    const float eb = (float)PyFloat_AsDouble(a[3]);
    const unsigned tile = (unsigned)PyLong_AsUnsignedLong(a[4]);
    if (PyErr_Occurred()) return nullptr;
    void *x, *out, *nb, *st;
    size_t n, cap;
    if (!ptr_unless_empty(a[1], c10::kFloat, &x, &n) || !dev_ptr(a[5], c10::kByte, &out, &cap) || !dev_ptr(a[6], c10::kLong, &nb) || !stream_of(a[7], &st))
        return nullptr;
    return status([&] { return zccl_compress_tiled(c, (const float*)x, n, mode, eb, tile, out, cap, (size_t*)nb, st); });
}

// (ctx, stream_bytes, tile, y, stream)
PyObject* decompress_tiled(PyObject*, Args a, Py_ssize_t na)
{
    if (!nargs_are(na, 5)) return nullptr;
    zccl_ctx* c = ctx_of(a[0]);
    const unsigned tile = (unsigned)PyLong_AsUnsignedLong(a[2]);
    if (PyErr_Occurred()) return nullptr;
    void *in, *y, *st;
    size_t cap, n;
    if (!dev_ptr(a[1], c10::kByte, &in, &cap) || !ptr_unless_empty(a[3], c10::kFloat, &y, &n) || !stream_of(a[4], &st)) return nullptr;
    return status([&] { return zccl_decompress_tiled(c, in, cap, tile, (float*)y, n, st); });
}

// The float pointers of a sequence of tensors.
struct Pointers {
    void* p[ZCCL_MAX_RANKS];
    int count = 0;
    size_t first = 0;   // elements of the first
};
bool pointers(PyObject* seq, Pointers& out)
{
    PyObject* f = PySequence_Fast(seq, "expected a sequence of tensors");
    if (!f) return false;
    const Py_ssize_t k = PySequence_Fast_GET_SIZE(f);
    bool ok = true;
    // more buffers than the library knows ranks: the boundary call refuses the count
    for (Py_ssize_t i = 0; ok && i < k && i < ZCCL_MAX_RANKS; ++i)
        ok = dev_ptr(PySequence_Fast_GET_ITEM(f, i), c10::kFloat, &out.p[i], i == 0 ? &out.first : nullptr);
    out.count = (int)k;
    Py_DECREF(f);
    return ok;
}

bool same_count(const Pointers& s, const Pointers& r)
{
    if (r.count >= s.count) return true;
    PyErr_SetString(PyExc_ValueError, "fewer receive buffers than send buffers");
    return false;
}

using SimFn = int (*)(zccl_ctx*, const float* const*, float* const*, int, size_t, int, float, void*);
// (ctx, send, recv, eb_mode, eb, stream)
template <SimFn FN>
PyObject* sim(PyObject*, Args a, Py_ssize_t na)
{
    if (!nargs_are(na, 6)) return nullptr;
    zccl_ctx* c = ctx_of(a[0]);
    const int mode = (int)PyLong_AsLong(a[3]);
    const float eb = (float)PyFloat_AsDouble(a[4]);
    if (PyErr_Occurred()) return nullptr;
    Pointers s, r;
    void* st;
    if (!pointers(a[1], s) || !pointers(a[2], r) || !same_count(s, r) || !stream_of(a[5], &st)) return nullptr;
    return status([&] { return FN(c, (const float* const*)s.p, (float* const*)r.p, s.count, s.first, mode, eb, st); });
}
// (ctx, send, recv, eb_mode, eb, flags, stream)
PyObject* sim_allreduce(PyObject*, Args a, Py_ssize_t na)
{
    if (!nargs_are(na, 7)) return nullptr;
    zccl_ctx* c = ctx_of(a[0]);
    const int mode = (int)PyLong_AsLong(a[3]);
    const float eb = (float)PyFloat_AsDouble(a[4]);
    const unsigned flags = (unsigned)PyLong_AsUnsignedLong(a[5]);
    if (PyErr_Occurred()) return nullptr;
    Pointers s, r;
    void* st;
    if (!pointers(a[1], s) || !pointers(a[2], r) || !same_count(s, r) || !stream_of(a[6], &st)) return nullptr;
    return status([&] { return zccl_sim_allreduce(c, (const float* const*)s.p, (float* const*)r.p, s.count, s.first, mode, eb, flags, st); });
}

// ---- calls without a context: they run on their tensors' device, whichever is the current one

bool refuse(const char* what)
{
    PyErr_SetString(PyExc_ValueError, what);
    return false;
}
int type_of(const at::Tensor& t)
{
    switch (t.scalar_type()) {
        case c10::kFloat: return ZCCL_F32;
        case c10::kBFloat16: return ZCCL_BF16;
        case c10::kHalf: return ZCCL_F16;
        default: return -1;
    }
}
bool cuda_tensor(PyObject* o, const at::Tensor** t)
{
    if (!THPVariable_Check(o) || !THPVariable_Unpack(o).is_cuda()) return refuse("expected a CUDA tensor");
    *t = &THPVariable_Unpack(o);
    return true;
}
// A matrix of float32, bfloat16 or float16 whose rows are contiguous; `pitch` elements from row to row.
bool matrix(PyObject* o, const at::Tensor** t, int* type, size_t* pitch)
{
    if (!cuda_tensor(o, t)) return false;
    *type = type_of(**t);
    if (*type < 0) return refuse("expected float32, bfloat16 or float16");
    if ((*t)->dim() != 2 || ((*t)->size(1) > 1 && (*t)->stride(1) != 1) || ((*t)->size(0) > 1 && (*t)->stride(0) < (*t)->size(1)))
        return refuse("expected a matrix with contiguous rows");
    *pitch = (*t)->size(0) > 1 ? (size_t)(*t)->stride(0) : (size_t)(*t)->size(1);
    return true;
}
// Bytes of exactly this number on the same device.
bool bytes_of(PyObject* o, size_t bytes, const at::Tensor& like, void** p)
{
    const at::Tensor* t;
    if (!cuda_tensor(o, &t)) return false;
    if (t->scalar_type() != c10::kByte || !t->is_contiguous() || (size_t)t->numel() != bytes) {
        PyErr_Format(PyExc_ValueError, "expected %zu contiguous bytes (uint8)", bytes);
        return false;
    }
    if (t->device() != like.device()) return refuse("all tensors of a call are on one device");
    *p = t->data_ptr();
    return true;
}
// The stream to run on: the one given, which has to be of that device, or the device's current one.
bool stream_on(PyObject* o, const at::Tensor& t, void** st)
{
    if (o == Py_None) {
        *st = (void*)c10::cuda::getCurrentCUDAStream(t.device().index()).stream();
        return true;
    }
    PyObject* d = PyObject_GetAttrString(o, "device_index");
    if (!d) return false;
    const long index = PyLong_AsLong(d);
    Py_DECREF(d);
    if (PyErr_Occurred()) return false;
    if (index != t.device().index()) return refuse("the stream is of another device than the tensors");
    return stream_of(o, st);
}
template <class F>
PyObject* status_on(const at::Tensor& t, F&& f)
{
    try {
        const c10::cuda::CUDAGuard guard(t.device());
        return status(f);
    } catch (const std::exception& e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
        return nullptr;
    }
}

// (rows, cols) -> bytes of codes and of scales
PyObject* mx4_sizes(PyObject*, Args a, Py_ssize_t na)
{
    if (!nargs_are(na, 2)) return nullptr;
    const size_t rows = PyLong_AsSize_t(a[0]), cols = PyLong_AsSize_t(a[1]);
    if (PyErr_Occurred()) return nullptr;
    return Py_BuildValue("nn", (Py_ssize_t)zccl_mx4_code_bytes(rows, cols), (Py_ssize_t)zccl_mx4_scale_bytes(rows, cols));
}

// (x, transpose, codes, scales, stream)
PyObject* mx4_quantize(PyObject*, Args a, Py_ssize_t na)
{
    if (!nargs_are(na, 5)) return nullptr;
    const at::Tensor* x;
    int type;
    size_t pitch;
    void *codes, *scales, *st;
    if (!matrix(a[0], &x, &type, &pitch)) return nullptr;
    const int transpose = PyObject_IsTrue(a[1]);
    const size_t rows = x->size(0), cols = x->size(1), r = transpose ? cols : rows, c = transpose ? rows : cols;
    if (!bytes_of(a[2], zccl_mx4_code_bytes(r, c), *x, &codes) || !bytes_of(a[3], zccl_mx4_scale_bytes(r, c), *x, &scales) || !stream_on(a[4], *x, &st)) return nullptr;
    return status_on(*x, [&] { return zccl_mx4_quantize(x->data_ptr(), type, rows, cols, pitch, transpose, codes, scales, st); });
}

// (codes, scales, y, stream)
PyObject* mx4_dequantize(PyObject*, Args a, Py_ssize_t na)
{
    if (!nargs_are(na, 4)) return nullptr;
    const at::Tensor* y;
    int type;
    size_t pitch;
    void *codes, *scales, *st;
    if (!matrix(a[2], &y, &type, &pitch)) return nullptr;
    const size_t rows = y->size(0), cols = y->size(1);
    if (!bytes_of(a[0], zccl_mx4_code_bytes(rows, cols), *y, &codes) || !bytes_of(a[1], zccl_mx4_scale_bytes(rows, cols), *y, &scales) || !stream_on(a[3], *y, &st)) return nullptr;
    return status_on(*y, [&] { return zccl_mx4_dequantize(codes, scales, rows, cols, y->data_ptr(), type, pitch, st); });
}

// (a_codes, a_scales, b_codes, b_scales, k, y, stream)
PyObject* mx4_matmul(PyObject*, Args a, Py_ssize_t na)
{
    if (!nargs_are(na, 7)) return nullptr;
    const size_t k = PyLong_AsSize_t(a[4]);
    if (PyErr_Occurred()) return nullptr;
    const at::Tensor* y;
    int type;
    size_t pitch;
    void *ac, *as, *bc, *bs, *st;
    if (!matrix(a[5], &y, &type, &pitch)) return nullptr;
    const size_t m = y->size(0), n = y->size(1);
    if (!bytes_of(a[0], zccl_mx4_code_bytes(m, k), *y, &ac) || !bytes_of(a[1], zccl_mx4_scale_bytes(m, k), *y, &as) || !bytes_of(a[2], zccl_mx4_code_bytes(n, k), *y, &bc) ||
        !bytes_of(a[3], zccl_mx4_scale_bytes(n, k), *y, &bs) || !stream_on(a[6], *y, &st)) return nullptr;
    return status_on(*y, [&] { return zccl_mx4_matmul(ac, as, m, bc, bs, n, k, y->data_ptr(), type, pitch, st); });
}

// A list or tuple of tensors, kept alive by its caller.
struct Tensors {
    PyObject* seq = nullptr;
    ~Tensors() { Py_XDECREF(seq); }
    bool take(PyObject* o)
    {
        seq = PySequence_Fast(o, "expected a sequence of tensors");
        return seq != nullptr;
    }
    size_t count() const { return seq ? (size_t)PySequence_Fast_GET_SIZE(seq) : 0; }
    bool at(size_t i, const at::Tensor** t) const { return cuda_tensor(PySequence_Fast_GET_ITEM(seq, (Py_ssize_t)i), t); }
};
// Entry i of a list that belongs to `like`: contiguous, of type `dt`, `n` elements, on the same device.
bool entry(const Tensors& list, size_t i, c10::ScalarType dt, size_t n, const at::Tensor& like, const at::Tensor** t)
{
    if (!list.at(i, t)) return false;
    if (!(*t)->is_contiguous() || (*t)->scalar_type() != dt || (size_t)(*t)->numel() != n) {
        PyErr_Format(PyExc_ValueError, "tensor %zu of a list: expected %zu contiguous elements of %S", i, n, (PyObject*)torch::getTHPDtype(dt));
        return false;
    }
    return (*t)->device() == like.device() || refuse("all tensors of a call are on one device");
}
// Whether no two of these ranges share a byte.
bool apart(std::vector<std::pair<uintptr_t, uintptr_t>>& ranges)
{
    const auto clash = [&] {
        for (size_t i = 1; i < ranges.size(); ++i)
            if (ranges[i].first < ranges[i - 1].second) return true;
        return false;
    };
    if (!clash()) return true;
    std::sort(ranges.begin(), ranges.end());
    return !clash();
}

// (params, grads, m, v, m_scales, v_scales, copies, lr, beta1, beta2, eps, weight_decay, step, seed, norm, max_norm, stream)
// m_scales, v_scales, copies, norm: or None; lr: a number or a float32 tensor; step: a number or an int64 tensor
PyObject* adamw(PyObject*, Args a, Py_ssize_t na)
{
    if (!nargs_are(na, 17)) return nullptr;
    Tensors p, g, m, v, ms, vs, copies;
    if (!p.take(a[0]) || !g.take(a[1]) || !m.take(a[2]) || !v.take(a[3])) return nullptr;
    const bool eight = a[4] != Py_None;
    if (eight != (a[5] != Py_None)) return refuse("scales of both states or of none"), nullptr;
    if (eight && (!ms.take(a[4]) || !vs.take(a[5]))) return nullptr;
    const bool copied = a[6] != Py_None;
    if (copied && !copies.take(a[6])) return nullptr;
    const size_t count = p.count();
    if (g.count() != count || m.count() != count || v.count() != count || (eight && (ms.count() != count || vs.count() != count)) || (copied && copies.count() != count))
        return refuse("lists of different lengths"), nullptr;
    if (count == 0) return PyLong_FromLong(ZCCL_OK);
    zccl_adamw_config k{};
    const at::Tensor *first, *t, *grad, *copy = nullptr;
    if (!p.at(0, &first) || !g.at(0, &grad) || (copied && !copies.at(0, &copy))) return nullptr;
    k.param_type = type_of(*first);
    k.grad_type = type_of(*grad);
    k.copy_type = copied ? type_of(*copy) : 0;
    k.state_bits = eight ? 8 : 32;
    if (k.param_type < 0 || k.grad_type < 0 || k.copy_type < 0) return refuse("expected float32, bfloat16 or float16"), nullptr;
    if (copied && (k.param_type != ZCCL_F32 || k.copy_type == ZCCL_F32)) return refuse("copies are bfloat16 or float16 ones of float32 parameters"), nullptr;
    const c10::ScalarType pt = first->scalar_type(), gt = grad->scalar_type(), state = eight ? c10::ScalarType::Float8_e4m3fn : c10::kFloat;
    std::vector<zccl_adamw_tensor> list(count);
    std::vector<const at::Tensor*> written;
    std::vector<std::pair<uintptr_t, uintptr_t>> ranges[6];
    written.reserve(6 * count);
    const auto put = [&](int kind, const at::Tensor* x) {
        written.push_back(x);
        const uintptr_t at = (uintptr_t)x->data_ptr();
        if (x->numel()) ranges[kind].emplace_back(at, at + (uintptr_t)x->nbytes());
        return x->data_ptr();
    };
    for (size_t i = 0; i < count; ++i) {
        zccl_adamw_tensor& s = list[i];
        if (!p.at(i, &t)) return nullptr;
        const size_t n = (size_t)t->numel(), blocks = (n + ZCCL_BLOCK - 1) / ZCCL_BLOCK;
        s.n = n;
        if (!entry(p, i, pt, n, *first, &t)) return nullptr;
        s.p = put(0, t);
        if (!entry(g, i, gt, n, *first, &t)) return nullptr;
        s.g = t->data_ptr();
        if (!entry(m, i, state, n, *first, &t)) return nullptr;
        s.m = put(1, t);
        if (!entry(v, i, state, n, *first, &t)) return nullptr;
        s.v = put(2, t);
        if (eight) {
            if (!entry(ms, i, c10::kByte, blocks, *first, &t)) return nullptr;
            s.m_scale = put(3, t);
            if (!entry(vs, i, c10::kByte, blocks, *first, &t)) return nullptr;
            s.v_scale = put(4, t);
        }
        if (copied) {
            if (!entry(copies, i, copy->scalar_type(), n, *first, &t)) return nullptr;
            s.copy = put(5, t);
        }
    }
    for (auto& r : ranges)
        if (!apart(r)) return refuse("two tensors of a list overlap"), nullptr;
    const auto scalar = [&](PyObject* o, c10::ScalarType dt, const at::Tensor** x) {
        if (!cuda_tensor(o, x)) return false;
        if ((*x)->numel() != 1 || (*x)->scalar_type() != dt || (*x)->device() != first->device()) {
            PyErr_Format(PyExc_ValueError, "expected one element of %S on the tensors' device", (PyObject*)torch::getTHPDtype(dt));
            return false;
        }
        return true;
    };
    if (THPVariable_Check(a[7])) {
        if (!scalar(a[7], c10::kFloat, &t)) return nullptr;
        k.lr_device = (const float*)t->data_ptr();
    } else k.lr = PyFloat_AsDouble(a[7]);
    k.beta1 = PyFloat_AsDouble(a[8]);
    k.beta2 = PyFloat_AsDouble(a[9]);
    k.eps = PyFloat_AsDouble(a[10]);
    k.weight_decay = PyFloat_AsDouble(a[11]);
    if (THPVariable_Check(a[12])) {
        if (!scalar(a[12], c10::kLong, &t)) return nullptr;
        k.step_device = (const long long*)t->data_ptr();
    } else k.step = PyLong_AsLongLong(a[12]);
    k.seed = PyLong_AsUnsignedLongLongMask(a[13]);
    if (a[14] != Py_None) {
        if (!scalar(a[14], c10::kFloat, &t)) return nullptr;
        k.norm = (const float*)t->data_ptr();
        k.max_norm = PyFloat_AsDouble(a[15]);
    }
    void* st;
    if (PyErr_Occurred() || !stream_on(a[16], *first, &st)) return nullptr;
    PyObject* rc = status_on(*first, [&] { return zccl_adamw(list.data(), count, &k, st); });
    for (const at::Tensor* x : written)
        if (!x->is_inference()) x->unsafeGetTensorImpl()->bump_version();
    return rc;
}

// (grads, norm, work, stream)
PyObject* grad_norm(PyObject*, Args a, Py_ssize_t na)
{
    if (!nargs_are(na, 4)) return nullptr;
    Tensors g;
    const at::Tensor *norm, *work, *t;
    if (!g.take(a[0]) || !cuda_tensor(a[1], &norm) || !cuda_tensor(a[2], &work)) return nullptr;
    const size_t count = g.count();
    if (norm->scalar_type() != c10::kFloat || norm->numel() != 1) return refuse("the norm is one float32"), nullptr;
    if (work->scalar_type() != c10::kByte || !work->is_contiguous() || (size_t)work->numel() < zccl_grad_norm_work(count) || work->device() != norm->device())
        return refuse("the workspace is contiguous uint8, of grad_norm_work(count) bytes at least, on the norm's device"), nullptr;
    std::vector<const void*> at(count);
    std::vector<size_t> n(count);
    int type = ZCCL_F32;
    const at::Tensor* first = nullptr;
    for (size_t i = 0; i < count; ++i) {
        if (!g.at(i, &t)) return nullptr;
        if (!first) {
            first = t;
            type = type_of(*t);
            if (type < 0) return refuse("expected float32, bfloat16 or float16"), nullptr;
        }
        if (!entry(g, i, first->scalar_type(), (size_t)t->numel(), *norm, &t)) return nullptr;
        at[i] = t->data_ptr();
        n[i] = (size_t)t->numel();
    }
    void* st;
    if (!stream_on(a[3], *norm, &st)) return nullptr;
    return status_on(*norm, [&] { return zccl_grad_norm(at.data(), n.data(), count, type, (float*)norm->data_ptr(), work->data_ptr(), st); });
}

#define FAST(name) {#name, (PyCFunction)(void (*)(void))name, METH_FASTCALL, nullptr}
PyMethodDef methods[] = {
    {"current_stream", current_stream, METH_NOARGS, nullptr},
    FAST(compress), FAST(decompress), FAST(hop), FAST(compress_f64), FAST(decompress_f64), FAST(compress_tiled), FAST(decompress_tiled), FAST(sim_allreduce),
    {"sim_allgather", (PyCFunction)(void (*)(void))sim<zccl_sim_allgather>, METH_FASTCALL, nullptr},
    {"sim_reduce_scatter", (PyCFunction)(void (*)(void))sim<zccl_sim_reduce_scatter>, METH_FASTCALL, nullptr},
    FAST(mx4_sizes), FAST(mx4_quantize), FAST(mx4_dequantize), FAST(mx4_matmul), FAST(adamw), FAST(grad_norm),
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_zccl", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__zccl(void) { return PyModule_Create(&module); }
