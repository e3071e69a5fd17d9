/* Argument marshalling of the hot calls for CPython: the same checks and conversions as binding.py's helpers, without
 * ctypes.  A call on a few tokens takes the GPU 5 to 10 us, and ctypes with the checks written in Python took the host
 * 6 to 7 us of every call (4 attribute reads per tensor, 11 to 22 argument conversions); this takes about 1 us.
 *
 * Call(name, address, spec, names, float_types, on_error, stream_of, sizes, device_of) is a callable object.  spec has one letter per
 * positional argument, in the order of the C function's parameters:
 *   t  tensor of the storage dtype (the first one decides which)      f  float32 tensor       q  int64 tensor
 *   i  integer     d  float (double)     w  workspace: object with ptr and nbytes, or (ptr, nbytes); two C parameters
 *   v  workspace pointer, or None     s  stream: None (the current one), an integer, or an object with cuda_stream
 *   D  (no argument) the dtype code
 * sizes is None, or for each argument a tuple of the positions of up to three integer arguments (none: an empty tuple): a tensor
 * has to have at least their product of values, and to be on the device that device_of() says is the current one.
 * None as a tensor is a null pointer.  A non-zero status is given to on_error(status, name). */
#define PY_SSIZE_T_CLEAN
#include <Python.h>
#include <stdint.h>
#include <string.h>

#include "monarch.h"

#define MAX_ARGS 24

typedef int (*apply_fn)(void *, const uint64_t *);
#define P(k) ((void *)(uintptr_t)a[k])
#define F(k) ((float *)(uintptr_t)a[k])
#define I(k) ((int32_t)a[k])
#define L(k) ((int64_t)a[k])
#define Z(k) ((size_t)a[k])
#define Q(k) ((const int64_t *)(uintptr_t)a[k])
static double as_double(uint64_t bits)
{
    double v;
    memcpy(&v, &bits, sizeof v);
    return v;
}
#define D(k) as_double(a[k])
#define APPLY(name, ...) \
    static int apply_##name(void *fn, const uint64_t *a) { return ((__typeof__(name) *)fn)(__VA_ARGS__); }
APPLY(monarch_fwd, P(0), P(1), P(2), P(3), L(4), I(5), I(6), I(7), P(8), Z(9), P(10))
APPLY(monarch_bwd_dx, P(0), P(1), P(2), P(3), L(4), I(5), I(6), I(7), P(8), Z(9), P(10))
APPLY(monarch_bwd_dw, P(0), P(1), P(2), P(3), F(4), F(5), I(6), L(7), I(8), I(9), I(10), P(11), Z(12), P(13))
APPLY(monarch_bwd, P(0), P(1), P(2), P(3), P(4), P(5), F(6), F(7), I(8), L(9), I(10), I(11), I(12), P(13), Z(14), P(15))
APPLY(monarch_mlp_fwd, P(0), P(1), P(2), P(3), P(4), P(5), P(6), P(7), L(8), I(9), I(10), I(11), P(12), Z(13), P(14))
APPLY(monarch_mlp_bwd, P(0), P(1), P(2), P(3), P(4), P(5), P(6), P(7), F(8), F(9), F(10), F(11), F(12), F(13), I(14), L(15),
      I(16), I(17), I(18), P(19), Z(20), P(21))
APPLY(monarch_rect_fwd, P(0), P(1), P(2), P(3), L(4), I(5), I(6), I(7), I(8), I(9), P(10), Z(11), P(12))
APPLY(monarch_rect_bwd, P(0), P(1), P(2), P(3), P(4), P(5), F(6), F(7), I(8), L(9), I(10), I(11), I(12), I(13), I(14), P(15),
      Z(16), P(17))
APPLY(monarch_cplx_fwd, P(0), P(1), P(2), P(3), I(4), L(5), I(6), I(7), I(8), P(9), Z(10), P(11))
APPLY(monarch_dense, P(0), P(1), P(2), I(3), I(4), I(5), P(6))
APPLY(monarch_project, P(0), P(1), P(2), I(3), I(4), I(5), (unsigned long long *)P(6), P(7))
APPLY(monarch_xent_fwd, P(0), P(1), Q(2), F(3), F(4), L(5), I(6), I(7), L(8), I(9), P(10), Z(11), P(12))
APPLY(monarch_xent_bwd, P(0), P(1), Q(2), F(3), F(4), P(5), F(6), I(7), L(8), I(9), I(10), L(11), I(12), P(13), Z(14), P(15))
APPLY(monarch_orthogonalize, P(0), P(1), L(2), I(3), I(4), I(5), I(6), P(7), Z(8), P(9))
APPLY(monarch_muon_step, P(0), F(1), F(2), L(3), I(4), I(5), D(6), D(7), D(8), I(9), D(10), I(11), I(12), P(13), Z(14), P(15))

static const struct { const char *name; apply_fn apply; int params; } kCalls[] = {
    {"monarch_fwd", apply_monarch_fwd, 11},         {"monarch_bwd_dx", apply_monarch_bwd_dx, 11},
    {"monarch_bwd_dw", apply_monarch_bwd_dw, 14},   {"monarch_bwd", apply_monarch_bwd, 16},
    {"monarch_mlp_fwd", apply_monarch_mlp_fwd, 15}, {"monarch_mlp_bwd", apply_monarch_mlp_bwd, 22},
    {"monarch_rect_fwd", apply_monarch_rect_fwd, 13}, {"monarch_rect_bwd", apply_monarch_rect_bwd, 18},
    {"monarch_cplx_fwd", apply_monarch_cplx_fwd, 12}, {"monarch_dense", apply_monarch_dense, 7},
    {"monarch_project", apply_monarch_project, 8},  {"monarch_xent_fwd", apply_monarch_xent_fwd, 13},
    {"monarch_xent_bwd", apply_monarch_xent_bwd, 16}, {"monarch_orthogonalize", apply_monarch_orthogonalize, 10},
    {"monarch_muon_step", apply_monarch_muon_step, 16},
};

typedef struct {
    PyObject_HEAD
    vectorcallfunc vectorcall;
    void *fn;
    apply_fn apply;
    char spec[MAX_ARGS];
    int n_spec, n_args;
    PyObject *name, *names, *types, *on_error, *stream_of;   /* types: (float32, bfloat16, int64) */
    PyObject *device_of;                                     /* null: sizes are not checked */
    signed char need[MAX_ARGS][3];                           /* positions of the factors, -1: no more; first -2: not checked */
} Call;

static PyObject *s_is_cuda, *s_is_contiguous, *s_dtype, *s_data_ptr, *s_ptr, *s_nbytes, *s_cuda_stream, *s_numel, *s_get_device;

static int to_u64(PyObject *o, uint64_t *out)
{
    PyObject *n = PyNumber_Index(o);
    if (n == NULL) return -1;
    *out = PyLong_AsUnsignedLongLongMask(n);
    Py_DECREF(n);
    return *out == (uint64_t)-1 && PyErr_Occurred() ? -1 : 0;
}

static int attr_u64(PyObject *o, PyObject *attr, uint64_t *out)
{
    PyObject *v = PyObject_GetAttr(o, attr);
    if (v == NULL) return -1;
    const int r = to_u64(v, out);
    Py_DECREF(v);
    return r;
}

/* 1 / 0 / -1 for a truth-valued attribute (call: method) */
static int flag_of(PyObject *o, PyObject *attr, int call)
{
    PyObject *v = call ? PyObject_CallMethodNoArgs(o, attr) : PyObject_GetAttr(o, attr);
    if (v == NULL) return -1;
    const int r = PyObject_IsTrue(v);
    Py_DECREF(v);
    return r;
}

static int tensor_ptr(Call *c, int k, PyObject *t, char kind, PyObject **storage, int *code, uint64_t *out)
{
    PyObject *name = PyTuple_GET_ITEM(c->names, k), *f32 = PyTuple_GET_ITEM(c->types, 0);
    if (t == Py_None && !(kind == 't' && *storage == NULL)) {
        *out = 0;
        return 0;
    }
    PyObject *dt = PyObject_GetAttr(t, s_dtype);
    if (dt == NULL) return -1;
    int r = flag_of(t, s_is_cuda, 0);
    if (r == 0) PyErr_Format(PyExc_ValueError, "%U must be a CUDA tensor", name);
    if (r > 0 && (r = flag_of(t, s_is_contiguous, 1)) == 0) PyErr_Format(PyExc_ValueError, "%U must be contiguous", name);
    if (r > 0) {
        PyObject *want = kind == 'f' ? f32 : kind == 'q' ? PyTuple_GET_ITEM(c->types, 2) : *storage;
        if (want == NULL) {
            if (dt == f32) *code = MONARCH_F32;
            else if (dt == PyTuple_GET_ITEM(c->types, 1)) *code = MONARCH_BF16;
            else { PyErr_Format(PyExc_TypeError, "unsupported tensor dtype %S", dt); r = 0; }
            *storage = *code == MONARCH_F32 ? f32 : PyTuple_GET_ITEM(c->types, 1);
        } else if (dt != want) {
            PyErr_Format(PyExc_TypeError, "%U must have dtype %S, got %S", name, want, dt);
            r = 0;
        }
    }
    Py_DECREF(dt);
    if (r <= 0) return -1;
    PyObject *p = PyObject_CallMethodNoArgs(t, s_data_ptr);
    if (p == NULL) return -1;
    r = to_u64(p, out);
    Py_DECREF(p);
    return r;
}

static int workspace_of(PyObject *w, uint64_t *ptr, uint64_t *bytes)
{
    if (PyTuple_Check(w)) {
        if (PyTuple_GET_SIZE(w) != 2) { PyErr_SetString(PyExc_ValueError, "workspace is a Workspace or (pointer, bytes)"); return -1; }
        return to_u64(PyTuple_GET_ITEM(w, 0), ptr) || to_u64(PyTuple_GET_ITEM(w, 1), bytes) ? -1 : 0;
    }
    return attr_u64(w, s_ptr, ptr) || attr_u64(w, s_nbytes, bytes) ? -1 : 0;
}

static int method_i64(PyObject *o, PyObject *method, long long *out)
{
    PyObject *v = PyObject_CallMethodNoArgs(o, method);
    if (v == NULL) return -1;
    *out = PyLong_AsLongLong(v);
    Py_DECREF(v);
    return *out == -1 && PyErr_Occurred() ? -1 : 0;
}

/* every tensor is large enough for what the integer arguments say, and on the current device */
static int check_sizes(Call *c, PyObject *const *args)
{
    long long device = 0;
    PyObject *v = PyObject_CallNoArgs(c->device_of);
    if (v == NULL) return -1;
    device = PyLong_AsLongLong(v);
    Py_DECREF(v);
    if (device == -1 && PyErr_Occurred()) return -1;
    for (int i = 0; i < c->n_args; ++i) {
        if (c->need[i][0] == -2 || args[i] == Py_None) continue;
        unsigned long long n = 1;
        for (int k = 0; k < 3 && c->need[i][k] >= 0; ++k) {
            uint64_t f;
            if (to_u64(args[(int)c->need[i][k]], &f)) return -1;
            if ((int64_t)f < 0) { n = 0; break; }                    /* the call itself refuses it */
            if (__builtin_mul_overflow(n, (unsigned long long)f, &n)) n = ~0ull;
        }
        long long have, at;
        if (method_i64(args[i], s_numel, &have)) return -1;
        PyObject *name = PyTuple_GET_ITEM(c->names, i);
        if ((unsigned long long)have < n) {
            PyErr_Format(PyExc_ValueError, "%U: %U must have at least %llu values, got %lld", c->name, name, n, have);
            return -1;
        }
        if (method_i64(args[i], s_get_device, &at)) return -1;
        if (at >= 0 && at != device) {
            PyErr_Format(PyExc_ValueError, "%U: %U is on device %lld, the current one is %lld", c->name, name, at, device);
            return -1;
        }
    }
    return 0;
}

static PyObject *call_it(PyObject *self, PyObject *const *args, size_t nargsf, PyObject *kw)
{
    Call *c = (Call *)self;
    const Py_ssize_t n = PyVectorcall_NARGS(nargsf);
    if (n != c->n_args || (kw != NULL && PyTuple_GET_SIZE(kw) != 0))
        return PyErr_Format(PyExc_TypeError, "%U takes %d positional arguments (%zd given)", c->name, c->n_args, n);
    if (c->device_of != NULL && check_sizes(c, args)) return NULL;
    uint64_t a[MAX_ARGS], ignored;
    PyObject *storage = NULL;
    int code = 0, out = 0, in = 0, dtype_at = -1;
    for (int i = 0; i < c->n_spec; ++i) {
        const char kind = c->spec[i];
        PyObject *v = kind == 'D' ? NULL : args[in];
        switch (kind) {
            case 'D': dtype_at = out++; break;
            case 'i': if (to_u64(v, &a[out++])) return NULL; break;
            case 'd': {
                const double f = PyFloat_AsDouble(v);
                if (f == -1.0 && PyErr_Occurred()) return NULL;
                memcpy(&a[out++], &f, sizeof f);
                break;
            }
            case 'w': if (workspace_of(v, &a[out], &a[out + 1])) return NULL; out += 2; break;
            case 'v':
                a[out] = 0;
                if (v != Py_None && workspace_of(v, &a[out], &ignored)) return NULL;
                ++out;
                break;
            case 's':
                if (v == Py_None) {
                    PyObject *s = PyObject_CallNoArgs(c->stream_of);
                    if (s == NULL) return NULL;
                    const int r = to_u64(s, &a[out]);
                    Py_DECREF(s);
                    if (r) return NULL;
                } else if (PyLong_Check(v) ? to_u64(v, &a[out]) : attr_u64(v, s_cuda_stream, &a[out])) {
                    return NULL;
                }
                ++out;
                break;
            default: if (tensor_ptr(c, in, v, kind, &storage, &code, &a[out++])) return NULL;
        }
        if (kind != 'D') ++in;
    }
    if (dtype_at >= 0) a[dtype_at] = (uint64_t)code;
    int status;
    Py_BEGIN_ALLOW_THREADS
    status = c->apply(c->fn, a);
    Py_END_ALLOW_THREADS
    if (status != 0) return PyObject_CallFunction(c->on_error, "iO", status, c->name);
    Py_RETURN_NONE;
}

static PyObject *call_new(PyTypeObject *type, PyObject *args, PyObject *kw)
{
    PyObject *name, *names, *types, *on_error, *stream_of, *sizes, *device_of;
    unsigned long long fn;
    const char *spec;
    Py_ssize_t len;
    if (kw != NULL && PyDict_GET_SIZE(kw) != 0) { PyErr_SetString(PyExc_TypeError, "Call takes no keywords"); return NULL; }
    if (!PyArg_ParseTuple(args, "UKs#O!O!OOOO", &name, &fn, &spec, &len, &PyTuple_Type, &names, &PyTuple_Type, &types, &on_error, &stream_of, &sizes,
                          &device_of))
        return NULL;
    if (len > MAX_ARGS || PyTuple_GET_SIZE(types) != 3) { PyErr_SetString(PyExc_ValueError, "bad spec"); return NULL; }
    int n_args = 0, params = 0;
    for (Py_ssize_t i = 0; i < len; ++i) {
        if (strchr("tfqidwvsD", spec[i]) == NULL) { PyErr_SetString(PyExc_ValueError, "bad spec"); return NULL; }
        n_args += spec[i] != 'D';
        params += spec[i] == 'w' ? 2 : 1;
    }
    apply_fn apply = NULL;
    for (size_t k = 0; k < sizeof(kCalls) / sizeof(kCalls[0]); ++k)
        if (PyUnicode_CompareWithASCIIString(name, kCalls[k].name) == 0 && kCalls[k].params == params) apply = kCalls[k].apply;
    if (apply == NULL || fn == 0 || PyTuple_GET_SIZE(names) != n_args) { PyErr_SetString(PyExc_ValueError, "spec does not fit the function"); return NULL; }
    if (sizes != Py_None && (!PyTuple_Check(sizes) || PyTuple_GET_SIZE(sizes) != n_args)) { PyErr_SetString(PyExc_ValueError, "bad sizes"); return NULL; }
    Call *c = (Call *)type->tp_alloc(type, 0);
    if (c == NULL) return NULL;
    for (int i = 0; sizes != Py_None && i < n_args; ++i) {
        PyObject *t = PyTuple_GET_ITEM(sizes, i);
        const Py_ssize_t n = PyTuple_Check(t) ? PyTuple_GET_SIZE(t) : 4;
        c->need[i][0] = n == 0 ? -2 : -1;
        for (Py_ssize_t k = 0; k < 3 && n <= 3; ++k) {
            const long at = k < n ? PyLong_AsLong(PyTuple_GET_ITEM(t, k)) : -1;
            if (k < n) c->need[i][k] = at >= 0 && at < n_args ? (signed char)at : -1;
            else if (k > 0) c->need[i][k] = -1;
        }
    }
    c->device_of = sizes != Py_None ? Py_NewRef(device_of) : NULL;
    c->vectorcall = call_it;
    c->fn = (void *)(uintptr_t)fn;
    c->apply = apply;
    memcpy(c->spec, spec, (size_t)len);
    c->n_spec = (int)len;
    c->n_args = n_args;
    c->name = Py_NewRef(name);
    c->names = Py_NewRef(names);
    c->types = Py_NewRef(types);
    c->on_error = Py_NewRef(on_error);
    c->stream_of = Py_NewRef(stream_of);
    return (PyObject *)c;
}

static void call_dealloc(PyObject *self)
{
    Call *c = (Call *)self;
    Py_XDECREF(c->name);
    Py_XDECREF(c->names);
    Py_XDECREF(c->types);
    Py_XDECREF(c->on_error);
    Py_XDECREF(c->stream_of);
    Py_XDECREF(c->device_of);
    Py_TYPE(self)->tp_free(self);
}

static PyTypeObject CallType = {
    PyVarObject_HEAD_INIT(NULL, 0)
    .tp_name = "paper_2204_00595_b200._pycalls.Call",
    .tp_basicsize = sizeof(Call),
    .tp_dealloc = call_dealloc,
    .tp_vectorcall_offset = offsetof(Call, vectorcall),
    .tp_call = PyVectorcall_Call,
    .tp_flags = Py_TPFLAGS_DEFAULT | Py_TPFLAGS_HAVE_VECTORCALL,
    .tp_new = call_new,
};

static struct PyModuleDef module = {PyModuleDef_HEAD_INIT, "_pycalls", "native argument marshalling", -1, NULL, NULL, NULL, NULL, NULL};

PyMODINIT_FUNC PyInit__pycalls(void)
{
    if (PyType_Ready(&CallType) < 0) return NULL;
    s_is_cuda = PyUnicode_InternFromString("is_cuda");
    s_is_contiguous = PyUnicode_InternFromString("is_contiguous");
    s_dtype = PyUnicode_InternFromString("dtype");
    s_data_ptr = PyUnicode_InternFromString("data_ptr");
    s_ptr = PyUnicode_InternFromString("ptr");
    s_nbytes = PyUnicode_InternFromString("nbytes");
    s_cuda_stream = PyUnicode_InternFromString("cuda_stream");
    s_numel = PyUnicode_InternFromString("numel");
    s_get_device = PyUnicode_InternFromString("get_device");
    PyObject *m = PyModule_Create(&module);
    if (m == NULL || PyModule_AddObjectRef(m, "Call", (PyObject *)&CallType) < 0) return NULL;
    return m;
}
