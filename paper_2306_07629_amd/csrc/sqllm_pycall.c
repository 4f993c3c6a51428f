/* One call of sqllm_dense_sparse_matvec, or of one of the sqllm_mx_* entry points, from Python without ctypes: takes the arguments apart, asks the tensors for their addresses and the
 * runtime for the current stream, and calls the library.  The call of a small layer is bound by the host: through ctypes 256x4096 takes
 * 5.6 us and 4096x4096 at 4 bits 5.8, this way 4.5 and 4.5 (their kernels run for 3.0 and 4.4).  Arguments that are not plain ints, None or
 * objects with data_ptr() are left to the ctypes path (None is returned), which accepts or refuses them as it always has. */
#define PY_SSIZE_T_CLEAN
#include <Python.h>
#include <string.h>

typedef int (*matvec_fn)(int, int, int, long long, int, const void*, const void*, const int*, const int*, const void*, const void*, const void*, void*, void*);

static matvec_fn g_matvec;
static PyObject *g_device, *g_stream;      /* torch.cuda.current_device, device -> raw handle of its current stream */
static PyObject *s_data_ptr, *s_cuda_stream;

static PyObject* bind(PyObject* self, PyObject* args) {
    unsigned long long address;
    PyObject *device, *stream;
    (void)self;
    if (!PyArg_ParseTuple(args, "KOO", &address, &device, &stream)) return NULL;
    Py_INCREF(device);
    Py_INCREF(stream);
    Py_XSETREF(g_device, device);
    Py_XSETREF(g_stream, stream);
    g_matvec = (matvec_fn)(uintptr_t)address;
    Py_RETURN_NONE;
}

/* 1: *out is set, 0: not for this path, -1: an error is set */
static int address_of(PyObject* o, PyObject* method, int call, void** out) {
    PyObject* v;
    if (o == Py_None) { *out = NULL; return 1; }
    if (PyLong_Check(o)) { Py_INCREF(o); v = o; }
    else {
        v = call ? PyObject_CallMethodNoArgs(o, method) : PyObject_GetAttr(o, method);
        if (!v) return -1;
        if (!PyLong_Check(v)) { Py_DECREF(v); return 0; }
    }
    *out = (void*)(uintptr_t)PyLong_AsUnsignedLongLongMask(v);        /* as ctypes takes integers: the low bits */
    Py_DECREF(v);
    return PyErr_Occurred() ? -1 : 1;
}

/* handle of a stream, None: the current one of the current device; returns as address_of */
static int stream_of(PyObject* o, PyObject* device, PyObject* stream, void** out) {
    PyObject *dev, *s;
    int st;
    if (o != Py_None) return address_of(o, s_cuda_stream, 0, out);
    dev = PyObject_CallNoArgs(device);
    if (!dev) return -1;
    s = PyObject_CallOneArg(stream, dev);
    Py_DECREF(dev);
    if (!s) return -1;
    st = PyLong_Check(s) ? address_of(s, NULL, 0, out) : 0;
    Py_DECREF(s);
    return st;
}

/* matvec(M, N, bits, nnz, B, qidx, lut, rowptr, cols, vals, plan, x, y, stream) -> status, or None */
static PyObject* matvec(PyObject* self, PyObject* const* a, Py_ssize_t n) {
    long long v[5];
    void* p[9];
    int i, st;
    (void)self;
    if (n != 14 || !g_matvec) Py_RETURN_NONE;
    for (i = 0; i < 5; ++i) {
        if (!PyLong_Check(a[i])) Py_RETURN_NONE;
        v[i] = (long long)PyLong_AsUnsignedLongLongMask(a[i]);
        if (PyErr_Occurred()) return NULL;
    }
    for (i = 0; i < 8; ++i) {
        st = address_of(a[5 + i], s_data_ptr, 1, &p[i]);
        if (st < 0) return NULL;
        if (st == 0) Py_RETURN_NONE;
    }
    st = stream_of(a[13], g_device, g_stream, &p[8]);
    if (st < 0) return NULL;
    if (st == 0) Py_RETURN_NONE;
    Py_BEGIN_ALLOW_THREADS
    st = g_matvec((int)v[0], (int)v[1], (int)v[2], v[3], (int)v[4], p[0], p[1], (const int*)p[2], (const int*)p[3], p[4], p[5], p[6], p[7], p[8]);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(st);
}

/* The sqllm_mx_* entry points: i an int, l a long long, p a pointer, s the stream. */
enum { kQuantize, kDequantize, kGemv, kGemm, kEntries };
static const char* const g_kinds[kEntries] = {"iiiplpppps", "iiipppls", "iiippppis", "iiiippppplis"};
static void* g_mx[kEntries];
static PyObject *g_mx_device, *g_mx_stream;      /* as g_device and g_stream */
typedef int (*quantize_fn)(int, int, int, const void*, long long, void*, void*, void*, void*, void*);
typedef int (*dequantize_fn)(int, int, int, const void*, const void*, void*, long long, void*);
typedef int (*gemv_fn)(int, int, int, const void*, const void*, const void*, void*, int, void*);
typedef int (*gemm_fn)(int, int, int, int, const void*, const void*, const void*, const void*, void*, long long, int, void*);

static PyObject* bind_mx(PyObject* self, PyObject* args) {
    unsigned long long a[kEntries];
    PyObject *device, *stream;
    int i;
    (void)self;
    if (!PyArg_ParseTuple(args, "KKKKOO", &a[0], &a[1], &a[2], &a[3], &device, &stream)) return NULL;
    Py_INCREF(device);
    Py_INCREF(stream);
    Py_XSETREF(g_mx_device, device);
    Py_XSETREF(g_mx_stream, stream);
    for (i = 0; i < kEntries; ++i) g_mx[i] = (void*)(uintptr_t)a[i];
    Py_RETURN_NONE;
}

/* mx(entry, its arguments...) -> status, or None */
static PyObject* mx(PyObject* self, PyObject* const* a, Py_ssize_t n) {
    long long v[12];                                                  /* integers and pointers by position */
    void* p[12];
    long entry;
    const char* kinds;
    int i, st;
    (void)self;
    if (n < 1 || !PyLong_Check(a[0])) Py_RETURN_NONE;
    entry = PyLong_AsLong(a[0]);
    if (entry < 0 || entry >= kEntries) {
        if (PyErr_Occurred()) return NULL;
        Py_RETURN_NONE;
    }
    kinds = g_kinds[entry];
    if (!g_mx[entry] || n != 1 + (Py_ssize_t)strlen(kinds)) Py_RETURN_NONE;
    for (i = 0; kinds[i]; ++i) {
        PyObject* o = a[1 + i];
        if (kinds[i] == 'i' || kinds[i] == 'l') {
            if (!PyLong_Check(o)) Py_RETURN_NONE;
            v[i] = (long long)PyLong_AsUnsignedLongLongMask(o);
            if (PyErr_Occurred()) return NULL;
            continue;
        }
        st = kinds[i] == 's' ? stream_of(o, g_mx_device, g_mx_stream, &p[i]) : address_of(o, s_data_ptr, 1, &p[i]);
        if (st < 0) return NULL;
        if (st == 0) Py_RETURN_NONE;
    }
    Py_BEGIN_ALLOW_THREADS
    switch (entry) {
        case kQuantize: st = ((quantize_fn)g_mx[entry])((int)v[0], (int)v[1], (int)v[2], p[3], v[4], p[5], p[6], p[7], p[8], p[9]); break;
        case kDequantize: st = ((dequantize_fn)g_mx[entry])((int)v[0], (int)v[1], (int)v[2], p[3], p[4], p[5], v[6], p[7]); break;
        case kGemv: st = ((gemv_fn)g_mx[entry])((int)v[0], (int)v[1], (int)v[2], p[3], p[4], p[5], p[6], (int)v[7], p[8]); break;
        default: st = ((gemm_fn)g_mx[entry])((int)v[0], (int)v[1], (int)v[2], (int)v[3], p[4], p[5], p[6], p[7], p[8], v[9], (int)v[10], p[11]); break;
    }
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(st);
}

static PyMethodDef methods[] = {
    {"bind_mx", bind_mx, METH_VARARGS, NULL},
    {"mx", (PyCFunction)(void (*)(void))mx, METH_FASTCALL, NULL},
    {"bind", bind, METH_VARARGS, NULL},
    {"matvec", (PyCFunction)(void (*)(void))matvec, METH_FASTCALL, NULL},
    {NULL, NULL, 0, NULL},
};
static struct PyModuleDef module = {PyModuleDef_HEAD_INIT, "_pycall", NULL, -1, methods, NULL, NULL, NULL, NULL};

PyMODINIT_FUNC PyInit__pycall(void) {
    s_data_ptr = PyUnicode_InternFromString("data_ptr");
    s_cuda_stream = PyUnicode_InternFromString("cuda_stream");
    if (!s_data_ptr || !s_cuda_stream) return NULL;
    return PyModule_Create(&module);
}
