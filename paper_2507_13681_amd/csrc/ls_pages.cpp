// Marshalling of the calls on pages and packed sequences: tensors of any strides in, the C ABI call out.  What the library cannot see of a tensor (its type, its
// sizes, its device) is checked here.  Against the C++ tensor: asked for one by one through Python, as ls_py.c does for the two things it needs, type, sizes, strides, device and
// address of a tensor are half a microsecond, and a call has eight tensors (a token's rows written for four sequences: 5.9 us a call, 4.4 so).
#include <Python.h>
#include <torch/csrc/autograd/python_variable.h>

#include <initializer_list>

#include "../../include/loopserve.h"

namespace {

PyObject* get_raw_stream;                                  // torch._C._cuda_getCurrentRawStream

struct Wrong {};                                           // a Python error is set
[[noreturn]] void wrong(const char* name, const char* what) {
    PyErr_Format(PyExc_ValueError, "%s: %s", name, what);
    throw Wrong{};
}

// A tensor on GPU `device` of this type; null for None
const at::Tensor* tensor(PyObject* o, const char* name, at::ScalarType type, long device) {
    if (o == Py_None) return nullptr;
    if (!THPVariable_Check(o)) wrong(name, "must be a tensor");
    const at::Tensor& t = THPVariable_Unpack(o);
    if (!t.is_cuda()) wrong(name, "must be a device tensor");
    if (t.scalar_type() != type) wrong(name, "has another type than the call takes");
    if (t.get_device() != device) wrong(name, "is not on the context's GPU");
    return &t;
}
// The address of a contiguous tensor of these sizes (-1: any)
void* plain(PyObject* o, const char* name, at::ScalarType type, long device, std::initializer_list<int64_t> want, int32_t* last = nullptr) {
    const at::Tensor* t = tensor(o, name, type, device);
    if (!t) return nullptr;
    bool ok = t->dim() == (int64_t)want.size();
    int64_t i = 0;
    for (const int64_t w : want) { ok = ok && (w < 0 ? t->size(i) <= INT32_MAX : t->size(i) == w); ++i; }
    if (!ok) wrong(name, "has other sizes than the call takes");
    if (!t->is_contiguous()) wrong(name, "must be contiguous");
    if (last) *last = (int32_t)t->size(t->dim() - 1);
    return t->data_ptr();
}
// Rows: packed [rows,H,d], else [B,H,rows,d], of any strides but the last, which is one
ls_rows rows_of(PyObject* o, const char* name, const ls_shape& s, long device, bool packed, int64_t rows, int64_t H) {
    const at::Tensor* t = tensor(o, name, s.dtype == LS_BF16 ? at::kBFloat16 : at::kFloat, device);
    if (!t) wrong(name, "must be a tensor");
    const bool ok = packed ? t->dim() == 3 && t->size(0) == rows && t->size(1) == H && t->size(2) == s.d
                           : t->dim() == 4 && t->size(0) == s.B && t->size(1) == H && t->size(2) == rows && t->size(3) == s.d;
    if (!ok) wrong(name, packed ? "must be [rows, heads, d] of the shape's numbers" : "must be [B, heads, rows, d] of the shape's numbers");
    if (t->stride(t->dim() - 1) != 1) wrong(name, "the values of a row must be neighbours");
    auto step = [&](int64_t i) { return t->size(i) == 1 ? 0 : t->stride(i); };               // (of one alone it is never taken, whatever it says)
    if (packed) return ls_rows{t->data_ptr(), 0, step(0), step(1)};
    return ls_rows{t->data_ptr(), step(0), step(2), step(1)};
}
// A ctypes structure (it exports its bytes as a buffer), copied
template <typename T>
T struct_of(PyObject* o, const char* what) {
    Py_buffer b;
    if (PyObject_GetBuffer(o, &b, PyBUF_SIMPLE) != 0) throw Wrong{};
    const bool ok = b.len == (Py_ssize_t)sizeof(T);
    T x{};
    if (ok) memcpy(&x, b.buf, sizeof(T));
    PyBuffer_Release(&b);
    if (!ok) { PyErr_Format(PyExc_TypeError, "not an %s", what); throw Wrong{}; }
    return x;
}
struct Call {
    ls_ctx* ctx;
    long device;
    ls_shape sh;
    void* stream;
    Call(PyObject* const* a, Py_ssize_t nargs, Py_ssize_t want) {                  // ctx, device, shape, ..
        if (nargs != want) { PyErr_Format(PyExc_TypeError, "%d arguments instead of %d", (int)nargs, (int)want); throw Wrong{}; }
        ctx = static_cast<ls_ctx*>(PyLong_AsVoidPtr(a[0]));
        device = PyLong_AsLong(a[1]);
        if (PyErr_Occurred()) throw Wrong{};
        sh = struct_of<ls_shape>(a[2], "LsShape");
        PyObject* r = PyObject_CallOneArg(get_raw_stream, a[1]);                   // the one that PyTorch issues to on the context's GPU
        if (!r) throw Wrong{};
        stream = PyLong_AsVoidPtr(r);
        Py_DECREF(r);
        if (PyErr_Occurred()) throw Wrong{};
    }
};
template <typename F>
PyObject* guarded(F f) {                                   // no C++ exception leaves
    int rc = 0;
    try {
        rc = f();
    } catch (const Wrong&) {
        return nullptr;
    } catch (const std::exception& e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
        return nullptr;
    }
    return PyLong_FromLong(rc);
}
template <typename F>
int released(F f) {
    int rc;
    Py_BEGIN_ALLOW_THREADS rc = f();
    Py_END_ALLOW_THREADS return rc;
}
const auto I32 = at::kInt;
const auto F32 = at::kFloat;
const auto BF16 = at::kBFloat16;

PyObject* packed_prefill(PyObject*, PyObject* const* a, Py_ssize_t nargs) {       // ctx, device, shape, q, k, v, q_starts, k_starts, out, lse
    return guarded([&] {
        const Call c(a, nargs, 10);
        const ls_shape& s = c.sh;
        const bool packed = a[6] != Py_None;
        const ls_rows q = rows_of(a[3], "q", s, c.device, packed, s.n_hat, s.Hq), k = rows_of(a[4], "k", s, c.device, packed, s.n, s.Hkv),
                      v = rows_of(a[5], "v", s, c.device, packed, s.n, s.Hkv), out = rows_of(a[8], "out", s, c.device, packed, s.n_hat, s.Hq);
        const int32_t* qs = static_cast<int32_t*>(plain(a[6], "q_starts", I32, c.device, {(int64_t)s.B + 1}));
        const int32_t* ks = static_cast<int32_t*>(plain(a[7], "k_starts", I32, c.device, {(int64_t)s.B + 1}));
        float* lse = static_cast<float*>(packed ? plain(a[9], "lse", F32, c.device, {s.Hq, s.n_hat}) : plain(a[9], "lse", F32, c.device, {s.B, s.Hq, s.n_hat}));
        return released([&] { return ls_packed_prefill(c.ctx, &s, &q, &k, &v, qs, ks, &out, lse, c.stream); });
    });
}
template <typename F>
PyObject* move(PyObject* const* a, Py_ssize_t nargs, F call) {                     // ctx, device, shape, cache, k, v, table, pos, starts, count
    return guarded([&] {
        const Call c(a, nargs, 10);
        const ls_shape& s = c.sh;
        const ls_cache cache = struct_of<ls_cache>(a[3], "LsCache");
        const bool packed = a[8] != Py_None;
        const ls_rows k = rows_of(a[4], "k", s, c.device, packed, s.n_hat, s.Hkv), v = rows_of(a[5], "v", s, c.device, packed, s.n_hat, s.Hkv);
        int32_t pages = 0;
        const int32_t* table = static_cast<int32_t*>(plain(a[6], "table", I32, c.device, {s.B, -1}, &pages));
        const int32_t* pos = static_cast<int32_t*>(plain(a[7], "pos", I32, c.device, {s.B}));
        const int32_t* starts = static_cast<int32_t*>(plain(a[8], "starts", I32, c.device, {(int64_t)s.B + 1}));
        const int32_t* count = static_cast<int32_t*>(plain(a[9], "count", I32, c.device, {s.B}));
        return released([&] { return call(c.ctx, &s, &cache, &k, &v, starts, count, table, pages, pos, c.stream); });
    });
}
PyObject* cache_write(PyObject*, PyObject* const* a, Py_ssize_t nargs) { return move(a, nargs, ls_cache_write); }
PyObject* cache_read(PyObject*, PyObject* const* a, Py_ssize_t nargs) { return move(a, nargs, ls_cache_read); }
PyObject* paged_attend(PyObject*, PyObject* const* a, Py_ssize_t nargs) {          // ctx, device, shape, cache, q, table, lens, out, lse
    return guarded([&] {
        const Call c(a, nargs, 9);
        const ls_shape& s = c.sh;
        const ls_cache cache = struct_of<ls_cache>(a[3], "LsCache");
        int32_t pages = 0;
        const void* q = plain(a[4], "q", BF16, c.device, {s.B, s.Hq, s.d});
        const int32_t* table = static_cast<int32_t*>(plain(a[5], "table", I32, c.device, {s.B, -1}, &pages));
        const int32_t* lens = static_cast<int32_t*>(plain(a[6], "lens", I32, c.device, {s.B}));
        void* out = plain(a[7], "out", BF16, c.device, {s.B, s.Hq, s.d});
        float* lse = static_cast<float*>(plain(a[8], "lse", F32, c.device, {s.B, s.Hq}));
        return released([&] { return ls_paged_attend(c.ctx, &s, &cache, q, table, pages, lens, out, lse, c.stream); });
    });
}

template <PyObject* (*F)(PyObject*, PyObject* const*, Py_ssize_t)>
PyMethodDef method(const char* name) { return {name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(F)), METH_FASTCALL, nullptr}; }
PyMethodDef methods[] = {method<packed_prefill>("packed_prefill"), method<cache_write>("cache_write"), method<cache_read>("cache_read"),
                         method<paged_attend>("paged_attend"), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_lspages", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__lspages() {
    // Tensors are read by functions that the compiler took from PyTorch's headers: of another PyTorch they would read other places.
    PyObject* torch = PyImport_ImportModule("torch");
    PyObject* version = torch ? PyObject_GetAttrString(torch, "__version__") : nullptr;
    Py_XDECREF(torch);
    if (!version) return nullptr;
    PyObject* text = PyObject_Str(version);
    Py_DECREF(version);
    if (!text) return nullptr;
    const bool same = PyUnicode_CompareWithASCIIString(text, LS_TORCH) == 0;
    if (!same) PyErr_Format(PyExc_ImportError, "built against PyTorch %s, and this is %U", LS_TORCH, text);
    Py_DECREF(text);
    if (!same) return nullptr;
    PyObject* c = PyImport_ImportModule("torch._C");
    if (!c) return nullptr;
    get_raw_stream = PyObject_GetAttrString(c, "_cuda_getCurrentRawStream");
    Py_DECREF(c);
    return get_raw_stream ? PyModule_Create(&module) : nullptr;
}
