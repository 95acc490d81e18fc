// CPython module over the C boundary for the calls a program makes per message: argument checks and marshalling in
// native code.  A codec call on a small message is a few microseconds of GPU work, so the host's share decides how many
// such calls fit a second: through ctypes and torch's Python-level stream objects a call's marshalling took 5.5 us
// (3.3 us of it the look-up of the current stream), here it takes 0.4 us.  The calls themselves are the C boundary's.
#include <Python.h>

#include <ATen/cuda/EmptyTensor.h>
#include <c10/cuda/CUDACachingAllocator.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>
#include <c10/util/SmallVector.h>
#include <torch/csrc/Dtype.h>
#include <torch/csrc/DynamicTypes.h>
#include <torch/csrc/autograd/python_variable.h>
#include <torch/csrc/jit/frontend/tracer.h>

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
// Whether an object is true; false with a Python error set where it has no answer.
bool truth(PyObject* o, bool* is)
{
    const int t = PyObject_IsTrue(o);
    *is = t == 1;
    return t >= 0;
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
    if ((*t)->layout() != c10::kStrided || (*t)->is_neg()) return refuse("expected a dense tensor");
    if ((*t)->_fw_grad(0).defined()) return refuse("a tensor with a forward-mode tangent, which would be lost here");
    const bool some = (*t)->numel() > 0;     // without elements any strides are good
    if ((*t)->dim() != 2 || (some && (((*t)->size(1) > 1 && (*t)->stride(1) != 1) || ((*t)->size(0) > 1 && (*t)->stride(0) < (*t)->size(1)))))
        return refuse("expected a matrix with contiguous rows");
    *pitch = some && (*t)->size(0) > 1 ? (size_t)(*t)->stride(0) : (size_t)(*t)->size(1);
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
// Tells autograd that a tensor has been written, which may have been saved for a backward pass.
void written(const at::Tensor& t)
{
    if (!t.is_inference()) t.unsafeGetTensorImpl()->bump_version();
}
// A boundary call without the interpreter lock: a launch waits where the GPU's queue is full, and other threads go on meanwhile.
template <class F>
int unlocked(F&& f)
{
    struct Lock {
        PyThreadState* const state = PyEval_SaveThread();
        ~Lock() { PyEval_RestoreThread(state); }
    } lock;
    return f();
}
// The tensors of a sequence, held for the call: another thread may change a list while the lock is not held.
struct Tensors {
    c10::SmallVector<PyObject*, 48> held;
    Tensors() = default;
    Tensors(const Tensors&) = delete;
    Tensors& operator=(const Tensors&) = delete;
    ~Tensors()
    {
        for (PyObject* o : held) Py_DECREF(o);
    }
    bool take(PyObject* o)
    {
        PyObject* const seq = PySequence_Fast(o, "expected a sequence of tensors");
        if (!seq) return false;
        PyObject** const items = PySequence_Fast_ITEMS(seq);
        held.assign(items, items + PySequence_Fast_GET_SIZE(seq));
        for (PyObject* t : held) Py_INCREF(t);
        Py_DECREF(seq);
        return true;
    }
    size_t count() const { return held.size(); }
    bool at(size_t i, const at::Tensor** t) const { return cuda_tensor(held[i], t); }
};
// ---- microscaled 4-bit floating point.  Outputs are allocated here, on the stream that the call runs on: through Python the small
// allocations of a call took longer than its kernels.

// The device and stream of a call, current for its duration where they are not already.
struct Place {
    c10::cuda::OptionalCUDAStreamGuard guard;
    void* st = nullptr;
    bool take(PyObject* stream, const at::Tensor& t)
    {
        if (!stream_on(stream, t, &st)) return false;
        if (stream != Py_None || c10::cuda::current_device() != t.device().index())
            guard.reset_stream(c10::cuda::getStreamFromExternal((cudaStream_t)st, t.device().index()));
        return true;
    }
};
at::Tensor new_bytes(size_t n, const at::Tensor& like) { return at::detail::empty_cuda({(int64_t)n}, at::kByte, like.device(), c10::nullopt); }
at::Tensor new_matrix(size_t rows, size_t cols, c10::ScalarType dt, const at::Tensor& like) { return at::detail::empty_cuda({(int64_t)rows, (int64_t)cols}, dt, like.device(), c10::nullopt); }
struct Form {
    at::Tensor codes, scales;
};
Form new_form(size_t rows, size_t cols, const at::Tensor& like) { return {new_bytes(zccl_mx4_code_bytes(rows, cols), like), new_bytes(zccl_mx4_scale_bytes(rows, cols), like)}; }

struct Matrix {
    const at::Tensor* t = nullptr;
    int type = 0;
    size_t pitch = 0, rows = 0, cols = 0;
    bool take(PyObject* o)
    {
        if (!matrix(o, &t, &type, &pitch)) return false;
        rows = (size_t)t->size(0);
        cols = (size_t)t->size(1);
        return true;
    }
    zccl_mx4_job job(bool transpose, void* codes, void* scales) const { return {t->data_ptr(), rows, cols, pitch, transpose, codes, scales}; }
    int quantize(bool transpose, void* codes, void* scales, void* st) const
    {
        void* const x = t->data_ptr();
        return unlocked([&] { return zccl_mx4_quantize(x, type, rows, cols, pitch, transpose, codes, scales, st); });
    }
};
// Forms that a call needs for itself, out of one allocation: each costs the host as much as a small kernel costs the GPU.
struct Inner {
    void *codes = nullptr, *scales = nullptr;
};
struct InnerForms {
    size_t bytes = 0;
    struct { size_t codes, scales; } at[4];
    int count = 0;
    void add(size_t rows, size_t cols)
    {
        const auto whole = [](size_t n) { return (n + 511) / 512 * 512; };
        at[count].codes = bytes;
        bytes += whole(zccl_mx4_code_bytes(rows, cols));
        at[count++].scales = bytes;
        bytes += whole(zccl_mx4_scale_bytes(rows, cols));
    }
    at::Tensor memory;
    void take(const at::Tensor& like) { memory = new_bytes(bytes, like); }
    Inner operator[](int i) const
    {
        char* const base = (char*)memory.data_ptr();
        return {base + at[i].codes, base + at[i].scales};
    }
};
int multiply(const Inner& a, size_t m, const Inner& b, size_t n, size_t k, const at::Tensor& y, void* st)
{
    void* const out = y.data_ptr();
    return unlocked([&] { return zccl_mx4_matmul(a.codes, a.scales, m, b.codes, b.scales, n, k, out, type_of(y), n, st); });
}
// A form that the caller has: bytes of the right number on the right device.
bool take_form(PyObject* codes, PyObject* scales, size_t rows, size_t cols, const at::Tensor& like, Form* f)
{
    void* p;
    if (!bytes_of(codes, zccl_mx4_code_bytes(rows, cols), like, &p) || !bytes_of(scales, zccl_mx4_scale_bytes(rows, cols), like, &p)) return false;
    f->codes = THPVariable_Unpack(codes);
    f->scales = THPVariable_Unpack(scales);
    return true;
}
bool element_type(PyObject* o, c10::ScalarType* dt)
{
    if (!THPDtype_Check(o)) return refuse("expected a dtype");
    *dt = ((THPDtype*)o)->scalar_type;
    return *dt == c10::kFloat || *dt == c10::kBFloat16 || *dt == c10::kHalf || refuse("expected float32, bfloat16 or float16");
}
PyObject* wrapped(int rc, const at::Tensor& t) { return rc == ZCCL_OK ? THPVariable_Wrap(t) : PyLong_FromLong(rc); }

// (rows, cols) -> bytes of codes and of scales
PyObject* mx4_sizes(PyObject*, Args a, Py_ssize_t na)
{
    if (!nargs_are(na, 2)) return nullptr;
    const size_t rows = PyLong_AsSize_t(a[0]), cols = PyLong_AsSize_t(a[1]);
    if (PyErr_Occurred()) return nullptr;
    return Py_BuildValue("nn", (Py_ssize_t)zccl_mx4_code_bytes(rows, cols), (Py_ssize_t)zccl_mx4_scale_bytes(rows, cols));
}

// (x, transpose, codes or None, scales or None, stream) -> (codes, scales, rows, cols) or a status
PyObject* mx4_quantize(PyObject*, Args a, Py_ssize_t na)
{
    if (!nargs_are(na, 5)) return nullptr;
    Matrix x;
    if (!x.take(a[0])) return nullptr;
    bool transpose;
    if (!truth(a[1], &transpose)) return nullptr;
    const size_t rows = transpose ? x.cols : x.rows, cols = transpose ? x.rows : x.cols;
    Form f;
    const bool given = a[2] != Py_None;
    if (given && !take_form(a[2], a[3], rows, cols, *x.t, &f)) return nullptr;
    Place place;
    if (!place.take(a[4], *x.t)) return nullptr;
    if (!given) f = new_form(rows, cols, *x.t);
    const int rc = x.quantize(transpose, f.codes.data_ptr(), f.scales.data_ptr(), place.st);
    if (rc != ZCCL_OK) return PyLong_FromLong(rc);
    if (given) {
        written(f.codes);
        written(f.scales);
    }
    return Py_BuildValue("NNnn", THPVariable_Wrap(f.codes), THPVariable_Wrap(f.scales), (Py_ssize_t)rows, (Py_ssize_t)cols);
}

// (matrices, transposes, stream) -> list of (codes, scales) or a status
PyObject* mx4_quantize_all(PyObject*, Args a, Py_ssize_t na)
{
    if (!nargs_are(na, 3)) return nullptr;
    Tensors xs, ts;
    if (!xs.take(a[0]) || !ts.take(a[1])) return nullptr;
    const size_t count = xs.count();
    if (ts.count() != count) return refuse("lists of different lengths"), nullptr;
    std::vector<Matrix> x(count);
    std::vector<Form> f(count);
    std::vector<zccl_mx4_job> jobs(count);
    for (size_t i = 0; i < count; ++i) {
        if (!x[i].take(xs.held[i])) return nullptr;
        if (x[i].type != x[0].type || x[i].t->device() != x[0].t->device()) return refuse("all matrices of a call are of one type and on one device"), nullptr;
    }
    if (count == 0) return PyList_New(0);
    Place place;
    if (!place.take(a[2], *x[0].t)) return nullptr;
    for (size_t i = 0; i < count; ++i) {
        bool transpose;
        if (!truth(ts.held[i], &transpose)) return nullptr;
        f[i] = transpose ? new_form(x[i].cols, x[i].rows, *x[0].t) : new_form(x[i].rows, x[i].cols, *x[0].t);
        jobs[i] = x[i].job(transpose, f[i].codes.data_ptr(), f[i].scales.data_ptr());
    }
    const int rc = unlocked([&] { return zccl_mx4_quantize_all(jobs.data(), (int)count, x[0].type, place.st); });
    if (rc != ZCCL_OK) return PyLong_FromLong(rc);
    PyObject* const out = PyList_New((Py_ssize_t)count);
    for (size_t i = 0; out && i < count; ++i) PyList_SET_ITEM(out, (Py_ssize_t)i, Py_BuildValue("NN", THPVariable_Wrap(f[i].codes), THPVariable_Wrap(f[i].scales)));
    return out;
}

// (codes, scales, rows, cols, dtype, y or None, stream) -> y or a status
PyObject* mx4_dequantize(PyObject*, Args a, Py_ssize_t na)
{
    if (!nargs_are(na, 7)) return nullptr;
    const at::Tensor* codes;
    Form f;
    const size_t rows = PyLong_AsSize_t(a[2]), cols = PyLong_AsSize_t(a[3]);
    if (PyErr_Occurred() || !cuda_tensor(a[0], &codes) || !take_form(a[0], a[1], rows, cols, *codes, &f)) return nullptr;
    Matrix y;
    c10::ScalarType dt = c10::kFloat;
    const bool given = a[5] != Py_None;
    if (given) {
        if (!y.take(a[5])) return nullptr;
        if (y.rows != rows || y.cols != cols || y.t->device() != codes->device()) return refuse("the output is of another size or device than the form"), nullptr;
    } else if (!element_type(a[4], &dt)) return nullptr;
    Place place;
    if (!place.take(a[6], *codes)) return nullptr;
    const at::Tensor out = given ? *y.t : new_matrix(rows, cols, dt, *codes);
    const int rc = unlocked([&] { return zccl_mx4_dequantize(f.codes.data_ptr(), f.scales.data_ptr(), rows, cols, out.data_ptr(), type_of(out), given ? y.pitch : cols, place.st); });
    if (given && rc == ZCCL_OK) written(out);
    return wrapped(rc, out);
}

// (a_codes, a_scales, m, b_codes, b_scales, n, k, dtype, y or None, stream) -> y or a status
PyObject* mx4_matmul(PyObject*, Args a, Py_ssize_t na)
{
    if (!nargs_are(na, 10)) return nullptr;
    const size_t m = PyLong_AsSize_t(a[2]), n = PyLong_AsSize_t(a[5]), k = PyLong_AsSize_t(a[6]);
    const at::Tensor* codes;
    Form l, r;
    if (PyErr_Occurred() || !cuda_tensor(a[0], &codes) || !take_form(a[0], a[1], m, k, *codes, &l) || !take_form(a[3], a[4], n, k, *codes, &r)) return nullptr;
    Matrix y;
    c10::ScalarType dt = c10::kFloat;
    const bool given = a[8] != Py_None;
    if (given) {
        if (!y.take(a[8])) return nullptr;
        if (y.rows != m || y.cols != n || y.t->device() != codes->device()) return refuse("the output is of another size or device than the operands"), nullptr;
    } else if (!element_type(a[7], &dt)) return nullptr;
    Place place;
    if (!place.take(a[9], *codes)) return nullptr;
    const at::Tensor out = given ? *y.t : new_matrix(m, n, dt, *codes);
    const int rc = unlocked([&] {
        return zccl_mx4_matmul(l.codes.data_ptr(), l.scales.data_ptr(), m, r.codes.data_ptr(), r.scales.data_ptr(), n, k, out.data_ptr(), type_of(out), given ? y.pitch : n, place.st);
    });
    if (given && rc == ZCCL_OK) written(out);
    return wrapped(rc, out);
}

// (x, w) or (x, codes, scales, n) -> x W^T in x's type, or a status
PyObject* mx4_linear(PyObject*, Args a, Py_ssize_t na)
{
    if (na != 2 && !nargs_are(na, 4)) return nullptr;
    Matrix x, w;
    Form held;
    size_t n = 0;
    if (!x.take(a[0])) return nullptr;
    if (na == 2) {
        if (!w.take(a[1])) return nullptr;
        if (w.cols != x.cols || w.type != x.type || w.t->device() != x.t->device()) return refuse("x and the weights differ in type, device or the length of their rows"), nullptr;
        n = w.rows;
    } else {
        n = PyLong_AsSize_t(a[3]);
        if (PyErr_Occurred() || !take_form(a[1], a[2], n, x.cols, *x.t, &held)) return nullptr;
    }
    Place place;
    if (!place.take(Py_None, *x.t)) return nullptr;
    InnerForms inner;
    inner.add(x.rows, x.cols);
    if (na == 2) inner.add(n, x.cols);
    inner.take(*x.t);
    const Inner f = inner[0];
    const at::Tensor y = new_matrix(x.rows, n, x.t->scalar_type(), *x.t);
    int rc;
    if (na == 2) {
        const Inner g = inner[1];
        const zccl_mx4_job both[2] = {w.job(false, g.codes, g.scales), x.job(false, f.codes, f.scales)};
        rc = unlocked([&] { return zccl_mx4_quantize_all(both, 2, x.type, place.st); });
        if (rc == ZCCL_OK) rc = multiply(f, x.rows, g, n, x.cols, y, place.st);
    } else
        rc = unlocked([&] {
            return zccl_mx4_linear(x.t->data_ptr(), x.type, x.rows, x.cols, x.pitch, held.codes.data_ptr(), held.scales.data_ptr(), n, f.codes, f.scales, y.data_ptr(), n, place.st);
        });
    return wrapped(rc, y);
}

// (dy, x, w, dx wanted, dw wanted) -> (dx or None, dw or None), or a status
PyObject* mx4_linear_backward(PyObject*, Args a, Py_ssize_t na)
{
    if (!nargs_are(na, 5)) return nullptr;
    Matrix dy, x, w;
    if (!dy.take(a[0]) || !x.take(a[1]) || !w.take(a[2])) return nullptr;
    const size_t m = x.rows, k = x.cols, n = w.rows;
    if (dy.rows != m || dy.cols != n || w.cols != k) return refuse("sizes of the gradient, the input and the weights do not belong together"), nullptr;
    if (dy.t->device() != x.t->device() || w.t->device() != x.t->device()) return refuse("all tensors of a call are on one device"), nullptr;
    bool want_x, want_w;
    if (!truth(a[3], &want_x) || !truth(a[4], &want_w)) return nullptr;
    Place place;
    if (!place.take(Py_None, *x.t)) return nullptr;
    at::Tensor dx, dw;
    InnerForms inner;
    if (want_x) {
        inner.add(m, n);
        inner.add(k, n);
        dx = new_matrix(m, k, x.t->scalar_type(), *x.t);
    }
    if (want_w) {
        inner.add(n, m);
        inner.add(k, m);
        dw = new_matrix(n, k, w.t->scalar_type(), *x.t);
    }
    inner.take(*x.t);
    const struct { const Matrix* from; bool transpose, wanted; } operands[4] = {{&dy, false, want_x}, {&w, true, want_x}, {&dy, true, want_w}, {&x, true, want_w}};
    zccl_mx4_job jobs[4];
    int types[4], count = 0;
    for (const auto& o : operands)
        if (o.wanted) {
            const Inner f = inner[count];
            types[count] = o.from->type;
            jobs[count++] = o.from->job(o.transpose, f.codes, f.scales);
        }
    int rc = ZCCL_OK;
    if (dy.type == x.type && w.type == x.type) rc = unlocked([&] { return zccl_mx4_quantize_all(jobs, count, x.type, place.st); });
    else
        for (int i = 0; i < count && rc == ZCCL_OK; ++i) rc = unlocked([&] { return zccl_mx4_quantize_all(&jobs[i], 1, types[i], place.st); });
    if (want_x && rc == ZCCL_OK) rc = multiply(inner[0], m, inner[1], k, n, dx, place.st);
    if (want_w && rc == ZCCL_OK) rc = multiply(inner[count - 2], n, inner[count - 1], k, m, dw, place.st);
    if (rc != ZCCL_OK) return PyLong_FromLong(rc);
    Py_INCREF(Py_None);
    Py_INCREF(Py_None);
    PyObject* const ox = want_x ? THPVariable_Wrap(dx) : Py_None;
    PyObject* const ow = want_w ? THPVariable_Wrap(dw) : Py_None;
    if (want_x) Py_DECREF(Py_None);
    if (want_w) Py_DECREF(Py_None);
    return Py_BuildValue("NN", ox, ow);
}

// Entry i of a list that belongs to `like`: contiguous, of type `dt`, `n` elements, on the same device.
bool refuse_entry(const Tensors& list, size_t i, c10::ScalarType dt, size_t n, const at::Tensor& like)
{
    const at::Tensor* t;
    if (!list.at(i, &t)) return false;
    if (t->device() != like.device()) return refuse("all tensors of a call are on one device");
    PyErr_Format(PyExc_ValueError, "tensor %zu of a list: expected %zu contiguous elements of %S", i, n, (PyObject*)torch::getTHPDtype(dt));
    return false;
}
inline bool entry(const Tensors& list, size_t i, c10::ScalarType dt, size_t n, const at::Tensor& like, const at::Tensor** t)
{
    PyObject* const o = list.held[i];
    if (THPVariable_Check(o)) {
        const at::Tensor& x = THPVariable_Unpack(o);
        if (x.scalar_type() == dt && (size_t)x.numel() == n && x.is_contiguous() && x.device() == like.device()) {
            *t = &x;
            return true;
        }
    }
    return refuse_entry(list, i, dt, n, like);
}
// Whether the tensors of a list share no byte.  Lists are in the order of memory more often than not: only others are sorted.
struct Apart {
    uintptr_t begin = 0, end = 0;
    bool ordered = true;
    void add(const void* p, size_t bytes)
    {
        ordered &= bytes == 0 || (uintptr_t)p >= end;
        if (end == 0) begin = (uintptr_t)p;
        if (bytes) end = (uintptr_t)p + bytes;
    }
    // Lists in the order of memory, one behind the other: none of their tensors can overlap.
    bool clear_of(const Apart& o) const { return ordered && o.ordered && (end <= o.begin || o.end <= begin); }
    // `at(i)` and `bytes(i)`: where tensor i is and how long
    template <class F, class G>
    bool ok(size_t count, F&& at, G&& bytes) const
    {
        if (ordered) return true;
        std::vector<std::pair<uintptr_t, uintptr_t>> ranges;
        for (size_t i = 0; i < count; ++i)
            if (bytes(i)) ranges.emplace_back((uintptr_t)at(i), (uintptr_t)at(i) + bytes(i));
        std::sort(ranges.begin(), ranges.end());
        for (size_t i = 1; i < ranges.size(); ++i)
            if (ranges[i].first < ranges[i - 1].second) return false;
        return true;
    }
};

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
    Apart apart[7];
    const size_t wide = c10::elementSize(pt), grad_bytes = c10::elementSize(gt), state_bytes = c10::elementSize(state);
    for (size_t i = 0; i < count; ++i) {
        zccl_adamw_tensor& s = list[i];
        if (!p.at(i, &t)) return nullptr;
        const size_t n = (size_t)t->numel(), blocks = (n + ZCCL_BLOCK - 1) / ZCCL_BLOCK;
        s.n = n;
        if (!entry(p, i, pt, n, *first, &t)) return nullptr;
        s.p = t->data_ptr();
        if (!entry(g, i, gt, n, *first, &t)) return nullptr;
        s.g = t->data_ptr();
        if (!entry(m, i, state, n, *first, &t)) return nullptr;
        s.m = t->data_ptr();
        if (!entry(v, i, state, n, *first, &t)) return nullptr;
        s.v = t->data_ptr();
        if (eight) {
            if (!entry(ms, i, c10::kByte, blocks, *first, &t)) return nullptr;
            s.m_scale = t->data_ptr();
            if (!entry(vs, i, c10::kByte, blocks, *first, &t)) return nullptr;
            s.v_scale = t->data_ptr();
            apart[3].add(s.m_scale, blocks);
            apart[4].add(s.v_scale, blocks);
        }
        if (copied) {
            if (!entry(copies, i, copy->scalar_type(), n, *first, &t)) return nullptr;
            s.copy = t->data_ptr();
            apart[5].add(s.copy, 2 * n);
        }
        apart[0].add(s.p, n * wide);
        apart[6].add(s.g, n * grad_bytes);
        apart[1].add(s.m, n * state_bytes);
        apart[2].add(s.v, n * state_bytes);
    }
    const auto blocks = [&](size_t i) { return (list[i].n + ZCCL_BLOCK - 1) / ZCCL_BLOCK; };
    const auto states = [&](size_t i) { return list[i].n * state_bytes; };
    if (!apart[0].ok(count, [&](size_t i) { return list[i].p; }, [&](size_t i) { return list[i].n * wide; }) || !apart[1].ok(count, [&](size_t i) { return list[i].m; }, states) ||
        !apart[2].ok(count, [&](size_t i) { return list[i].v; }, states) || !apart[3].ok(count, [&](size_t i) { return list[i].m_scale; }, blocks) ||
        !apart[4].ok(count, [&](size_t i) { return list[i].v_scale; }, blocks) || !apart[5].ok(count, [&](size_t i) { return list[i].copy; }, [&](size_t i) { return 2 * list[i].n; }))
        return refuse("two tensors of a list overlap"), nullptr;
    bool clear = true;
    for (int i = 1; i < 7; ++i)
        for (int j = 0; j < i; ++j) clear = clear && apart[i].clear_of(apart[j]);
    for (const zccl_adamw_tensor& s : list) {
        if (clear) break;
        const size_t n = s.n, scales = eight ? (n + ZCCL_BLOCK - 1) / ZCCL_BLOCK : 0;
        const struct { const void* p; size_t bytes; } arrays[7] = {{s.p, n * wide},          {s.g, n * grad_bytes}, {s.m, n * state_bytes}, {s.v, n * state_bytes},
                                                                   {s.copy, copied ? 2 * n : 0}, {s.m_scale, scales},             {s.v_scale, scales}};
        for (int i = 1; i < 7; ++i)
            for (int j = 0; j < i; ++j)
                if ((uintptr_t)arrays[i].p < (uintptr_t)arrays[j].p + arrays[j].bytes && (uintptr_t)arrays[j].p < (uintptr_t)arrays[i].p + arrays[i].bytes)
                    return refuse("a parameter, its gradient, states and copy overlap"), nullptr;
    }
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
    if (PyErr_Occurred()) return nullptr;
    Place place;
    if (!place.take(a[16], *first)) return nullptr;
    const int rc = unlocked([&] { return zccl_adamw(list.data(), count, &k, place.st); });
    for (size_t i = 0; rc == ZCCL_OK && i < count; ++i)
        for (const Tensors* l : {&p, copied ? &copies : nullptr})
            if (l) written(THPVariable_Unpack(l->held[i]));
    return PyLong_FromLong(rc);
}

// (grads, norm or None, stream) -> norm or a status
PyObject* grad_norm(PyObject*, Args a, Py_ssize_t na)
{
    if (!nargs_are(na, 3)) return nullptr;
    Tensors g;
    const at::Tensor *norm = nullptr, *first = nullptr, *t;
    const bool given = a[1] != Py_None;
    if (!g.take(a[0]) || (given && !cuda_tensor(a[1], &norm))) return nullptr;
    const size_t count = g.count();
    if (given && (norm->scalar_type() != c10::kFloat || norm->numel() != 1)) return refuse("the norm is one float32"), nullptr;
    if (count && !g.at(0, &first)) return nullptr;
    if (!given && !count) return refuse("no gradients to take a device from: pass an output"), nullptr;
    const at::Tensor& like = given ? *norm : *first;
    const int type = first ? type_of(*first) : ZCCL_F32;
    if (type < 0) return refuse("expected float32, bfloat16 or float16"), nullptr;
    std::vector<const void*> at(count);
    std::vector<size_t> n(count);
    for (size_t i = 0; i < count; ++i) {
        if (!g.at(i, &t) || !entry(g, i, first->scalar_type(), (size_t)t->numel(), like, &t)) return nullptr;
        at[i] = t->data_ptr();
        n[i] = (size_t)t->numel();
    }
    Place place;
    if (!place.take(a[2], like)) return nullptr;
    const at::Tensor out = given ? *norm : at::Tensor(at::detail::empty_cuda({1}, c10::kFloat, like.device(), c10::nullopt));
    const c10::DataPtr work = c10::cuda::CUDACachingAllocator::get()->allocate(zccl_grad_norm_work(count));   // of the stream that place made current
    const int rc = unlocked([&] { return zccl_grad_norm(at.data(), n.data(), count, type, (float*)out.data_ptr(), work.get(), place.st); });
    if (given && rc == ZCCL_OK) written(out);
    return wrapped(rc, out);
}

// What torch throws (a tensor without memory or strides of its own, no memory left) ends here as a Python exception.  A trace would take the outputs for constants.
template <PyObject* (*F)(PyObject*, Args, Py_ssize_t)>
PyObject* guarded(PyObject* self, Args a, Py_ssize_t na)
{
    try {
        if (torch::jit::tracer::isTracing()) return refuse("this call cannot be recorded in a trace"), nullptr;
        return F(self, a, na);
    } catch (const std::exception& e) {
        if (!PyErr_Occurred()) PyErr_SetString(PyExc_RuntimeError, e.what());
        return nullptr;
    }
}

#define GUARDED(name) {#name, (PyCFunction)(void (*)(void))guarded<name>, METH_FASTCALL, nullptr}
#define FAST(name) {#name, (PyCFunction)(void (*)(void))name, METH_FASTCALL, nullptr}
PyMethodDef methods[] = {
    {"current_stream", current_stream, METH_NOARGS, nullptr},
    FAST(compress), FAST(decompress), FAST(hop), FAST(compress_f64), FAST(decompress_f64), FAST(compress_tiled), FAST(decompress_tiled), FAST(sim_allreduce),
    {"sim_allgather", (PyCFunction)(void (*)(void))sim<zccl_sim_allgather>, METH_FASTCALL, nullptr},
    {"sim_reduce_scatter", (PyCFunction)(void (*)(void))sim<zccl_sim_reduce_scatter>, METH_FASTCALL, nullptr},
    GUARDED(mx4_sizes), GUARDED(mx4_quantize), GUARDED(mx4_quantize_all), GUARDED(mx4_dequantize), GUARDED(mx4_matmul), GUARDED(mx4_linear), GUARDED(mx4_linear_backward), GUARDED(adamw), GUARDED(grad_norm),
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_zccl", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__zccl(void) { return PyModule_Create(&module); }
