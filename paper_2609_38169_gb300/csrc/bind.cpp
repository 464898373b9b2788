// Argument marshalling of the paged cache's calls, which a serving loop makes for every layer of
// every token: tensors to pointers and strides, with the checks of shapes, types and devices,
// in half a microsecond where the same in Python takes four. Nothing is computed here.
// api.py's functions of the same names call these with every argument, and raise StepqError on
// a status; errors of arguments are raised here as ValueError.
#include <Python.h>

#include <cmath>

#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include "stepq.h"

namespace {

decltype(&stepq_kv_append) kv_append;
decltype(&stepq_kv_read) kv_read;
decltype(&stepq_kv_attend) kv_attend;
decltype(&stepq_kv_page_bytes) kv_page_bytes;

struct Raised {};                      // a Python error is set

[[noreturn]] void refuse(const char *format, ...) {
    va_list args;
    va_start(args, format);
    PyErr_FormatV(PyExc_ValueError, format, args);
    va_end(args);
    throw Raised{};
}

long long number(PyObject *o) {
    const long long v = PyLong_AsLongLong(o);
    if (v == -1 && PyErr_Occurred()) throw Raised{};
    return v;
}
int integer(PyObject *o, const char *what) {
    const long long v = number(o);
    if (v < INT32_MIN || v > INT32_MAX) refuse("%s: %lld does not fit 32 bits", what, v);
    return (int)v;
}

const at::Tensor &tensor(PyObject *o, const char *what) {
    if (!THPVariable_Check(o)) refuse("%s: expected a tensor", what);
    return THPVariable_Unpack(o);
}

const char *name_of(at::ScalarType t) { return c10::toString(t); }

int dtype_code(at::ScalarType t) {
    switch (t) {
    case at::kFloat: return STEPQ_F32;
    case at::kBFloat16: return STEPQ_BF16;
    case at::kHalf: return STEPQ_F16;
    default: refuse("expected float32, bfloat16 or float16, got %s", name_of(t));
    }
}

// What a call's tensors have in common: the device that is current.
struct Call {
    int device = -1;
    // Where t lies; written: the call writes there, so that a tensor that still shares another's memory gets its own.
    void *on(const at::Tensor &t, const char *what, bool written = false) {
        if (!t.is_cuda()) refuse("%s: expected a CUDA tensor", what);
        if (device < 0) device = c10::cuda::current_device();
        if (t.get_device() != device)
            refuse("%s: expected a CUDA tensor on the current device, got one on cuda:%d", what, (int)t.get_device());
        return written ? t.mutable_data_ptr() : const_cast<void *>(t.const_data_ptr());
    }
    const int32_t *int32s(PyObject *o, int64_t n, const char *what) {
        const at::Tensor &t = tensor(o, what);
        const void *p = on(t, what);
        if (t.scalar_type() != at::kInt || !t.is_contiguous()) refuse("%s: expected contiguous int32", what);
        if (t.numel() != n) refuse("%s: expected %lld values, got %lld", what, (long long)n, (long long)t.numel());
        return (const int32_t *)p;
    }
    // Rows [rows][heads][dim] or [rows][heads * dim], heads next to each other, and the stride of rows.
    void *rows(PyObject *o, at::ScalarType type, int64_t n, int64_t heads, int64_t dim, int64_t &stride, const char *what,
               bool written) {
        const at::Tensor &t = tensor(o, what);
        void *p = on(t, what, written);
        if (t.scalar_type() != type) refuse("%s: expected %s, got %s", what, name_of(type), name_of(t.scalar_type()));
        const auto size = t.sizes(), step = t.strides();
        const bool ok = size.size() == 3 ? size[1] == heads && size[2] == dim && step[2] == 1 && (heads == 1 || step[1] == dim)
                                         : size.size() == 2 && size[1] == heads * dim && step[1] == 1;
        if (!ok || size[0] != n)
            refuse("%s: expected %lld contiguous rows of %lld x %lld", what, (long long)n, (long long)heads, (long long)dim);
        stride = n > 1 ? step[0] : heads * dim;              // that of a single row is arbitrary
        return p;
    }
};

stepq_kv_config config(PyObject *kv) {
    static PyObject *names[5];
    static const char *const text[5] = {"n_layers", "n_heads", "head_dim", "page_tokens", "format"};
    int v[5];
    for (int i = 0; i < 5; i++) {
        if (!names[i] && !(names[i] = PyUnicode_InternFromString(text[i]))) throw Raised{};
        PyObject *o = PyObject_GetAttr(kv, names[i]);
        if (!o) throw Raised{};
        const long long x = PyLong_AsLongLong(o);
        Py_DECREF(o);
        if (x == -1 && PyErr_Occurred()) throw Raised{};
        if (x < INT32_MIN || x > INT32_MAX) refuse("%s: %lld does not fit 32 bits", text[i], x);
        v[i] = (int)x;
    }
    return {v[0], v[1], v[2], v[3], v[4]};
}

stepq_kv_pages pages_of(Call &call, const stepq_kv_config &c, PyObject *pages_, PyObject *table_, int64_t B, bool written) {
    stepq_kv_pages p{};
    const at::Tensor &table = tensor(table_, "table");
    const auto size = table.sizes();
    if (size.size() != 2 || size[0] != B) refuse("table: expected %lld rows", (long long)B);
    p.table = (const int32_t *)call.on(table, "table");
    if (table.scalar_type() != at::kInt || (size[1] > 1 && table.strides()[1] != 1) || size[1] > INT32_MAX)
        refuse("table: expected rows of contiguous int32");
    p.table_width = (int)size[1];
    p.table_stride = B > 1 ? table.strides()[0] : size[1];
    const at::Tensor &pages = tensor(pages_, "pages");
    p.pages = call.on(pages, "pages", written);
    if (!pages.is_contiguous()) refuse("pages: expected a contiguous tensor");
    const size_t each = kv_page_bytes(&c);                   // 0: the library refuses the configuration
    const size_t n = each ? pages.nbytes() / each : 1;
    p.n_pages = n > INT32_MAX ? INT32_MAX : (int)n;
    return p;
}

stepq_stream_t stream_of(PyObject *stream, int device) {
    if (stream == Py_None) return device < 0 ? nullptr : (stepq_stream_t)c10::cuda::getCurrentCUDAStream((c10::DeviceIndex)device).stream();
    PyObject *o = PyObject_GetAttrString(stream, "cuda_stream");
    if (!o) throw Raised{};
    const unsigned long long v = PyLong_AsUnsignedLongLong(o);
    Py_DECREF(o);
    if (v == (unsigned long long)-1 && PyErr_Occurred()) throw Raised{};
    return (stepq_stream_t)v;
}

// Runs f() -> status; a C++ error becomes a Python one.
template <class F>
PyObject *guarded(Py_ssize_t n, Py_ssize_t want, F &&f) {
    if (n != want) {
        PyErr_Format(PyExc_TypeError, "expected %zd arguments, got %zd", want, n);
        return nullptr;
    }
    try {
        return PyLong_FromLong((long)f());
    } catch (const Raised &) {
    } catch (const std::exception &e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
    }
    return nullptr;
}

// The library's call without Python's lock: a launch waits where the queue is full, and what is queued may be a
// host function that takes the lock.
template <class F>
stepq_status unlocked(F &&call) {
    stepq_status status;
    Py_BEGIN_ALLOW_THREADS
    status = call();
    Py_END_ALLOW_THREADS
    return status;
}

// kv, layer, pages, table, starts, k, v, cu_seqlens, stream
stepq_status transfer(bool append, PyObject *const *a) {
    const stepq_kv_config c = config(a[0]);
    Call call;
    const int64_t B = tensor(a[4], "starts").numel();
    const at::Tensor &k = tensor(a[5], "k");
    const int64_t n = k.dim() ? k.sizes()[0] : 0;
    const at::ScalarType type = k.scalar_type();
    if (B > INT32_MAX || n > INT32_MAX) refuse("too many rows");
    if (a[7] != Py_None && tensor(a[7], "cu_seqlens").numel() != B + 1)
        refuse("cu_seqlens: expected %lld values, got %lld", (long long)(B + 1), (long long)tensor(a[7], "cu_seqlens").numel());
    const stepq_kv_pages p = pages_of(call, c, a[2], a[3], B, append);
    stepq_kv_rows r{};
    r.dtype = dtype_code(type);
    r.k = call.rows(a[5], type, n, c.n_heads, c.head_dim, r.k_stride, "k", !append);
    r.v = call.rows(a[6], type, n, c.n_heads, c.head_dim, r.v_stride, "v", !append);
    const int32_t *starts = call.int32s(a[4], B, "starts");
    const int32_t *cu = a[7] == Py_None ? nullptr : call.int32s(a[7], B + 1, "cu_seqlens");
    const int layer = integer(a[1], "layer");
    const stepq_stream_t stream = stream_of(a[8], call.device);
    return unlocked([&] { return (append ? kv_append : kv_read)(&c, layer, &p, starts, cu, (int)B, (int)n, &r, stream); });
}

PyObject *py_append(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return guarded(n, 9, [&] { return transfer(true, a); });
}
PyObject *py_read(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return guarded(n, 9, [&] { return transfer(false, a); });
}

// kv, layer, pages, table, lens, q, y, scale, window, lse, max_len, workspace, stream
PyObject *py_attend(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return guarded(n, 13, [&]() -> stepq_status {
        const stepq_kv_config c = config(a[0]);
        Call call;
        const int64_t B = tensor(a[4], "lens").numel();
        if (B > INT32_MAX) refuse("too many rows");
        const stepq_kv_pages p = pages_of(call, c, a[2], a[3], B, false);
        const at::Tensor &q = tensor(a[5], "q");
        if (q.dim() != 2 && q.dim() != 3) refuse("q: expected rows of heads");
        const int64_t heads = q.dim() == 3 ? q.sizes()[1] : c.head_dim > 0 ? q.sizes()[1] / c.head_dim : 0;
        if (heads > INT32_MAX) refuse("q: too many heads");
        const at::ScalarType type = q.scalar_type();
        stepq_kv_query io{};
        io.dtype = dtype_code(type);
        io.n_heads = (int)heads;
        io.y = call.rows(a[6], type, B, heads, c.head_dim, io.y_stride, "y", true);         // first: q may be the same tensor
        io.q = call.rows(a[5], type, B, heads, c.head_dim, io.q_stride, "q", false);
        if (a[7] == Py_None) {
            io.scale = c.head_dim > 0 ? (float)(1.0 / std::sqrt((double)c.head_dim)) : 0.f;
        } else {
            const double s = PyFloat_AsDouble(a[7]);
            if (s == -1.0 && PyErr_Occurred()) throw Raised{};
            io.scale = (float)s;
        }
        io.window = integer(a[8], "window");
        io.max_len = integer(a[10], "max_len");
        if (a[9] != Py_None) {
            const at::Tensor &lse = tensor(a[9], "lse");
            io.lse = (float *)call.on(lse, "lse", true);
            if (lse.scalar_type() != at::kFloat || !lse.is_contiguous()) refuse("lse: expected contiguous float32");
            if (lse.numel() != B * heads) refuse("lse: expected %lld values, got %lld", (long long)(B * heads), (long long)lse.numel());
        }
        void *ws = nullptr;
        size_t have = 0;
        if (a[11] != Py_None) {
            const at::Tensor &t = tensor(a[11], "workspace");
            ws = call.on(t, "workspace", true);
            if (!t.is_contiguous()) refuse("workspace: expected a contiguous tensor");
            have = t.nbytes();
        }
        const int32_t *lens = call.int32s(a[4], B, "lens");
        const int layer = integer(a[1], "layer");
        const stepq_stream_t stream = stream_of(a[12], call.device);
        return unlocked([&] { return kv_attend(&c, layer, &p, lens, (int)B, &io, ws, have, stream); });
    });
}

// The library's functions, by address: append, read, attend, page_bytes.
PyObject *py_use(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return guarded(n, 4, [&] {
        kv_append = (decltype(kv_append))number(a[0]);
        kv_read = (decltype(kv_read))number(a[1]);
        kv_attend = (decltype(kv_attend))number(a[2]);
        kv_page_bytes = (decltype(kv_page_bytes))number(a[3]);
        return 0;
    });
}

PyMethodDef methods[] = {{"use", (PyCFunction)(void (*)())py_use, METH_FASTCALL, nullptr},
                         {"kv_append", (PyCFunction)(void (*)())py_append, METH_FASTCALL, nullptr},
                         {"kv_read", (PyCFunction)(void (*)())py_read, METH_FASTCALL, nullptr},
                         {"kv_attend", (PyCFunction)(void (*)())py_attend, METH_FASTCALL, nullptr},
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_stepq_bind", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__stepq_bind() { return PyModule_Create(&module); }
