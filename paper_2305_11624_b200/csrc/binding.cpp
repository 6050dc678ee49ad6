// Python entry to the C calls that a training step makes, beside the ctypes binding of convbn.py.
// ctypes and the Python code that turned thirteen tensors into addresses took 2.8 us of a call of 5.9 us (forward of a 3x3
// 64 -> 64 layer, 1.4 of them for data_ptr alone).  With this, the plans of a layer kept (convbn_api.cu) and three allocations less
// per layer of a backbone (backbone.py): a ResNet-50 iteration that waits for the host 1820 -> 1300 us, 1x1 128 -> 256 at 9 x 13,
// N = 36 21.8 -> 18.3, depthwise 128 at 18 x 24 18.6 -> 16.4.  Arguments are converted by the declared parameter types
// of the C function: a descriptor is the object's buffer (ctypes structures export theirs), a pointer is None, an integer
// address or what data_ptr() returns.  The two arguments that every call ends with are resolved as the Python functions
// document them: workspace_bytes None is the workspace's nbytes, stream None is torch's current stream.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <cstdint>
#include <tuple>
#include <type_traits>
#include <utility>

#include "../../include/convbn.h"

namespace {

PyObject *s_data_ptr, *s_nbytes, *s_cuda_stream, *s_dtype, *s_numel, *s_itemsize, *s_is_contiguous, *s_get_device;      // attribute names
PyObject *g_get_device, *g_get_stream;                // torch._C._cuda_getDevice, _cuda_getCurrentRawStream

bool address(PyObject *o, void **out) {
    if (o == Py_None) { *out = nullptr; return true; }
    if (PyLong_Check(o)) {
        *out = PyLong_AsVoidPtr(o);
        return *out || !PyErr_Occurred();
    }
    PyObject *v = PyObject_CallMethodNoArgs(o, s_data_ptr);
    if (!v) return false;
    *out = PyLong_AsVoidPtr(v);
    Py_DECREF(v);
    return *out || !PyErr_Occurred();
}

bool stream(PyObject *o, void **out) {
    if (PyLong_Check(o)) { *out = PyLong_AsVoidPtr(o); return *out || !PyErr_Occurred(); }
    PyObject *v;
    if (o == Py_None) {
        if (!g_get_stream) {
            PyObject *m = PyImport_ImportModule("torch._C");
            if (!m) return false;
            g_get_device = PyObject_GetAttrString(m, "_cuda_getDevice");
            if (g_get_device) g_get_stream = PyObject_GetAttrString(m, "_cuda_getCurrentRawStream");
            Py_DECREF(m);
            if (!g_get_stream) return false;
        }
        PyObject *d = PyObject_CallNoArgs(g_get_device);
        if (!d) return false;
        v = PyObject_CallOneArg(g_get_stream, d);
        Py_DECREF(d);
    } else {
        v = PyObject_GetAttr(o, s_cuda_stream);
    }
    if (!v) return false;
    *out = PyLong_AsVoidPtr(v);
    Py_DECREF(v);
    return *out || !PyErr_Occurred();
}

template <class T>
bool convert(PyObject *o, T *out) {
    if constexpr (std::is_same_v<T, const convbn_desc *>) {
        if (o == Py_None) { *out = nullptr; return true; }
        Py_buffer b;
        if (PyObject_GetBuffer(o, &b, PyBUF_SIMPLE) != 0) return false;
        const bool fits = (size_t)b.len == sizeof(convbn_desc);
        *out = (const convbn_desc *)b.buf;            // (the caller holds the descriptor for the length of the call)
        PyBuffer_Release(&b);
        if (!fits) PyErr_SetString(PyExc_TypeError, "a convolution descriptor is expected");
        return fits;
    } else if constexpr (std::is_pointer_v<T>) {
        void *p = nullptr;
        if (!address(o, &p)) return false;
        *out = (T)p;
        return true;
    } else {
        // (as ctypes does: integers only, and cut to the parameter's width)
        if (!PyLong_Check(o)) {
            PyErr_Format(PyExc_TypeError, "an integer is expected, not %.100s", Py_TYPE(o)->tp_name);
            return false;
        }
        const unsigned long long v = PyLong_AsUnsignedLongLongMask(o);
        if (v == (unsigned long long)-1 && PyErr_Occurred()) return false;
        *out = (T)v;
        return true;
    }
}

// f(arguments ..., [workspace, workspace_bytes,] stream)
template <class... P, size_t... I>
PyObject *call(int (*f)(P...), PyObject *const *a, Py_ssize_t n, std::index_sequence<I...>) {
    constexpr size_t N = sizeof...(P);
    if (n != (Py_ssize_t)N) return PyErr_Format(PyExc_TypeError, "%zu arguments are expected", N);
    std::tuple<P...> v;
    using Bytes = std::tuple_element_t<N >= 2 ? N - 2 : 0, std::tuple<P...>>;
    bool ok = true;
    auto one = [&](auto index) {
        constexpr size_t K = decltype(index)::value;
        if (!ok) return;
        if constexpr (K == N - 1) {
            ok = stream(a[K], &std::get<K>(v));
        } else if constexpr (K + 2 == N && std::is_same_v<Bytes, size_t>) {
            if (a[K] != Py_None) { ok = convert(a[K], &std::get<K>(v)); return; }
            std::get<K>(v) = 0;
            if (a[K - 1] == Py_None) return;
            PyObject *b = PyObject_GetAttr(a[K - 1], s_nbytes);
            ok = b && convert(b, &std::get<K>(v));
            Py_XDECREF(b);
        } else {
            ok = convert(a[K], &std::get<K>(v));
        }
    };
    (one(std::integral_constant<size_t, I>()), ...);
    if (!ok) return nullptr;
    int status;
    Py_BEGIN_ALLOW_THREADS
    status = std::apply(f, v);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(status);
}

template <auto F>
struct Entry;
template <class... P, int (*F)(P...)>
struct Entry<F> {
    static PyObject *go(PyObject *, PyObject *const *a, Py_ssize_t n) { return call(F, a, n, std::index_sequence_for<P...>()); }
};

// ---- packed tensors: what the library reads and writes by address alone is looked at here ------------------------------------------
// An integer that an attribute or a method gives; -1 where there is none.
long long number(PyObject *o, PyObject *name, bool method) {
    PyObject *v = method ? PyObject_CallMethodNoArgs(o, name) : PyObject_GetAttr(o, name);
    long long r = -1;
    if (v && PyLong_Check(v)) r = PyLong_AsLongLong(v);
    Py_XDECREF(v);
    if (PyErr_Occurred()) { PyErr_Clear(); return -1; }
    return r;
}
bool contiguous(PyObject *o) {
    PyObject *v = PyObject_CallMethodNoArgs(o, s_is_contiguous);
    const bool r = v == Py_True;
    Py_XDECREF(v);
    if (PyErr_Occurred()) { PyErr_Clear(); return false; }
    return r;
}
bool room(PyObject *codes, PyObject *steps, long long count) {
    return number(codes, s_itemsize, false) == 1 && number(steps, s_itemsize, false) == 1 && number(codes, s_numel, true) >= count &&
           number(steps, s_numel, true) >= (count + 31) / 32 && contiguous(codes) && contiguous(steps);
}
int storage_type(PyObject *x) {           // -1: none of the three
    static PyObject *types[3];            // by CONVBN_F32, CONVBN_BF16, CONVBN_F16
    if (!types[CONVBN_F16]) {
        PyObject *m = PyImport_ImportModule("torch");
        if (m) {
            types[CONVBN_F32] = PyObject_GetAttrString(m, "float32");
            types[CONVBN_BF16] = PyObject_GetAttrString(m, "bfloat16");
            types[CONVBN_F16] = PyObject_GetAttrString(m, "float16");
            Py_DECREF(m);
        }
    }
    PyObject *t = PyObject_GetAttr(x, s_dtype);
    int r = -1;
    for (int k = 0; t && k < 3; ++k)
        if (t == types[k]) r = k;
    Py_XDECREF(t);
    PyErr_Clear();
    return r;
}
// convbn_pack(x, codes, steps, stream) and convbn_unpack(codes, steps, out, stream) for contiguous tensors of one GPU with room
// enough; None for anything else, which convbn.py then looks at.  (The checks in Python took 1.3 us of a call of 4.8.)
template <auto F, bool UNPACK>
PyObject *packed(PyObject *, PyObject *const *a, Py_ssize_t n) {
    if (n != 4) return PyErr_Format(PyExc_TypeError, "4 arguments are expected");
    PyObject *x = a[UNPACK ? 2 : 0], *codes = a[UNPACK ? 0 : 1], *steps = a[UNPACK ? 1 : 2];
    const int type = storage_type(x);
    const long long count = type < 0 ? -1 : number(x, s_numel, true), device = count < 0 ? -1 : number(x, s_get_device, true);
    if (device < 0 || !contiguous(x) || !room(codes, steps, count) || number(codes, s_get_device, true) != device ||
        number(steps, s_get_device, true) != device)
        Py_RETURN_NONE;
    void *p[3], *st = nullptr;
    for (int i = 0; i < 3; ++i)
        if (!address(a[i], &p[i])) return nullptr;
    if (!stream(a[3], &st)) return nullptr;
    int status;
    Py_BEGIN_ALLOW_THREADS
    status = F(type, p[0], p[1], p[2], count, st);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(status);
}
// convbn_tune_bwd_packed for codes and steps with room enough for the descriptor's X; None for others.
PyObject *packed_bwd(PyObject *self, PyObject *const *a, Py_ssize_t n) {
    const convbn_desc *d = nullptr;
    if (n > 3 && !convert(a[0], &d)) return nullptr;
    if (d && (d->n < 0 || d->c_in < 0 || d->h_in < 0 || d->w_in < 0 || !room(a[2], a[3], (long long)d->n * d->c_in * d->h_in * d->w_in)))
        Py_RETURN_NONE;
    return Entry<&convbn_tune_bwd_packed>::go(self, a, n);
}

#define ENTRY(name) {#name, (PyCFunction)(void (*)(void))Entry<&name>::go, METH_FASTCALL, nullptr}
PyMethodDef g_methods[] = {
    ENTRY(convbn_tune_fwd), ENTRY(convbn_tune_bwd_data), ENTRY(convbn_tune_bwd_weight), ENTRY(convbn_tune_bwd),
    ENTRY(convbn_tune_bwd_begin), ENTRY(convbn_tune_bwd_join), ENTRY(convbn_tune_fwd_glue), ENTRY(convbn_tune_bwd_glue),
    ENTRY(convbn_tconv_tune_fwd), ENTRY(convbn_tconv_tune_bwd), ENTRY(convbn_eval_fwd), ENTRY(convbn_eval_bwd),
    ENTRY(convbn_deploy_fwd), ENTRY(convbn_deploy_bwd), ENTRY(convbn_pack), ENTRY(convbn_unpack), ENTRY(convbn_tune_bwd_packed),
    ENTRY(convbn_deploy_fwd_quant),
    {"pack", (PyCFunction)(void (*)(void))packed<&convbn_pack, false>, METH_FASTCALL, nullptr},
    {"unpack", (PyCFunction)(void (*)(void))packed<&convbn_unpack, true>, METH_FASTCALL, nullptr},
    {"tune_bwd_packed", (PyCFunction)(void (*)(void))packed_bwd, METH_FASTCALL, nullptr}, {nullptr, nullptr, 0, nullptr}};
PyModuleDef g_module = {PyModuleDef_HEAD_INIT, "_binding", nullptr, -1, g_methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__binding(void) {
    s_data_ptr = PyUnicode_InternFromString("data_ptr");
    s_nbytes = PyUnicode_InternFromString("nbytes");
    s_cuda_stream = PyUnicode_InternFromString("cuda_stream");
    s_dtype = PyUnicode_InternFromString("dtype");
    s_numel = PyUnicode_InternFromString("numel");
    s_itemsize = PyUnicode_InternFromString("itemsize");
    s_is_contiguous = PyUnicode_InternFromString("is_contiguous");
    s_get_device = PyUnicode_InternFromString("get_device");
    return s_data_ptr && s_nbytes && s_cuda_stream && s_dtype && s_numel && s_itemsize && s_is_contiguous && s_get_device
               ? PyModule_Create(&g_module) : nullptr;
}
