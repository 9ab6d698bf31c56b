/* The shortest way from Python to the calls that a model makes per layer on parts of the cache: the checks of
 * Pool.select_blocks and Pool.sparse_attention, and the call, without ctypes. A selection for one session takes the
 * GPU 5.7 us; a pass took 11.3 with the checks in Python, as the host needed that long, and takes 8.2 here.
 *
 * A method returns the library's code, or None where an argument is not plainly what the call takes: then nothing was
 * called, and Pool's own checks say what is wrong (or take what is unusual). An interrupt or a lack of memory that comes
 * up meanwhile is passed on. */
#define PY_SSIZE_T_CLEAN
#include <Python.h>
#include <stdint.h>

typedef int (*select_fn)(void *, int32_t, const void *, int64_t, const void *, const int32_t *, const int32_t *, int32_t,
                         int32_t, int32_t, int32_t, int32_t, int32_t *, float *, void *);
typedef int (*sparse_fn)(void *, int32_t, const void *, int64_t, const void *, const void *, int64_t, const int32_t *,
                         int32_t, const int32_t *, const int32_t *, int32_t, int32_t, float, void *, uint32_t, void *);

enum { kDim = 128, kOutBf16 = 2 };

typedef struct {
    PyObject_HEAD
    void *pool;
    select_fn select;
    sparse_fn sparse;
    long index;                          /* the device number of the pool's tensors */
    int64_t Hq, Hkv, bounds_bytes;
    PyObject *bf16, *i32, *f32;          /* torch's dtypes */
} Calls;

static PyObject *s_dtype, *s_shape, *s_stride, *s_contiguous, *s_numel, *s_nbytes, *s_device, *s_ptr, *s_stream;

static int as_int64(PyObject *x, int64_t *to) {   /* takes the reference */
    int over = 0;
    if (!x) return 0;
    *to = PyLong_Check(x) ? PyLong_AsLongLongAndOverflow(x, &over) : (over = 1, 0);
    Py_DECREF(x);
    return !over && !PyErr_Occurred();
}

static int as_int32(PyObject *x, int32_t *to) {
    int64_t y;
    Py_INCREF(x);
    if (!as_int64(x, &y) || y < INT32_MIN || y > INT32_MAX) return 0;
    *to = (int32_t)y;
    return 1;
}

static int is_dtype(PyObject *x, PyObject *dtype) {
    PyObject *d = PyObject_GetAttr(x, s_dtype);
    Py_XDECREF(d);
    return d == dtype;
}

static int is_contiguous(PyObject *x) {
    PyObject *y = PyObject_CallMethodNoArgs(x, s_contiguous);
    Py_XDECREF(y);
    return y == Py_True;
}

/* On the pool's device; its address. */
static int place(const Calls *c, PyObject *x, void **ptr) {
    int64_t dev, at;
    if (!as_int64(PyObject_CallMethodNoArgs(x, s_device), &dev) || dev != c->index) return 0;
    PyObject *p = PyObject_CallMethodNoArgs(x, s_ptr);
    if (!p) return 0;
    at = (int64_t)PyLong_AsUnsignedLongLong(p);
    Py_DECREF(p);
    *ptr = (void *)(uintptr_t)at;
    return !PyErr_Occurred();
}

/* A tuple of three numbers, from a new reference. */
static int three_of(PyObject *t, int64_t *to) {
    int ok = t && PyTuple_Check(t) && PyTuple_GET_SIZE(t) == 3;
    for (int i = 0; ok && i < 3; ++i) {
        to[i] = PyLong_AsLongLong(PyTuple_GET_ITEM(t, i));
        ok = !PyErr_Occurred();
    }
    Py_XDECREF(t);
    return ok;
}

static int has_shape(PyObject *x, int64_t a, int64_t b, int64_t n) {
    int64_t s[3];
    return three_of(PyObject_GetAttr(x, s_shape), s) && s[0] == a && s[1] == b && s[2] == n;
}

/* int32, contiguous, at least n. */
static int row(const Calls *c, PyObject *x, int64_t n, void **ptr) {
    int64_t have;
    return is_dtype(x, c->i32) && as_int64(PyObject_CallMethodNoArgs(x, s_numel), &have) && have >= n && is_contiguous(x) &&
           place(c, x, ptr);
}

/* bf16 [B][heads][D] with contiguous heads; its row stride (0: one row). */
static int heads(const Calls *c, PyObject *x, int64_t B, int64_t n, int64_t *stride, void **ptr) {
    int64_t s[3];
    if (!is_dtype(x, c->bf16) || !has_shape(x, B, n, kDim) || !three_of(PyObject_CallMethodNoArgs(x, s_stride), s)) return 0;
    if (s[2] != 1 || s[1] != kDim || (B > 1 && s[0] == 0)) return 0;
    *stride = B > 1 ? s[0] : 0;
    return place(c, x, ptr);
}

/* int32 [B][Hkv][top]. */
static int list(const Calls *c, PyObject *x, int64_t B, int32_t *top, void **ptr) {
    int64_t s[3];
    if (!is_dtype(x, c->i32) || !three_of(PyObject_GetAttr(x, s_shape), s) || s[0] != B || s[1] != c->Hkv || s[2] > INT32_MAX ||
        !is_contiguous(x))
        return 0;
    *top = (int32_t)s[2];
    return place(c, x, ptr);
}

static int stream_of(PyObject *x, void **to) {
    PyObject *y;
    if (x == Py_None) {
        *to = NULL;
        return 1;
    }
    y = PyLong_Check(x) ? Py_NewRef(x) : PyObject_GetAttr(x, s_stream);
    if (!y) return 0;
    *to = PyLong_AsVoidPtr(y);
    Py_DECREF(y);
    return !PyErr_Occurred();
}

static PyObject *declined(void) {
    if (PyErr_Occurred() && (!PyErr_ExceptionMatches(PyExc_Exception) || PyErr_ExceptionMatches(PyExc_MemoryError))) return NULL;
    PyErr_Clear();
    Py_RETURN_NONE;
}

/* (layer, q, bounds, block_tables, seq_lens, B, max_blocks, selected, first, last, scores, stream) */
static PyObject *calls_select(Calls *c, PyObject *const *a, Py_ssize_t n) {
    int32_t layer, B, max_blocks, first, last, top;
    int64_t stride, bytes;
    void *q, *bounds, *tables, *lens, *selected, *scores = NULL, *stream;
    if (n != 12 || !as_int32(a[0], &layer) || !as_int32(a[5], &B) || !as_int32(a[6], &max_blocks) || !as_int32(a[8], &first) ||
        !as_int32(a[9], &last))
        return declined();
    if (!row(c, a[3], (int64_t)B * max_blocks, &tables) || !row(c, a[4], B, &lens) || !heads(c, a[1], B, c->Hq, &stride, &q) ||
        !list(c, a[7], B, &top, &selected))
        return declined();
    if (!as_int64(PyObject_GetAttr(a[2], s_nbytes), &bytes) || bytes < c->bounds_bytes || !is_contiguous(a[2]) ||
        !place(c, a[2], &bounds))
        return declined();
    if (a[10] != Py_None && (!is_dtype(a[10], c->f32) || !has_shape(a[10], B, c->Hkv, max_blocks) || !is_contiguous(a[10]) ||
                             !place(c, a[10], &scores)))
        return declined();
    if (!stream_of(a[11], &stream)) return declined();
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = c->select(c->pool, layer, q, stride, bounds, tables, lens, B, max_blocks, first, last, top, selected, scores, stream);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(rc);
}

/* (layer, q, selected, block_tables, seq_lens, B, max_blocks, scale, out, k_new, v_new, stream) */
static PyObject *calls_sparse(Calls *c, PyObject *const *a, Py_ssize_t n) {
    int32_t layer, B, max_blocks, top;
    int64_t stride, kv_stride = 0, v_stride = 0;
    void *q, *k = NULL, *v = NULL, *tables, *lens, *selected, *out, *stream;
    if (n != 12 || !as_int32(a[0], &layer) || !as_int32(a[5], &B) || !as_int32(a[6], &max_blocks) || !PyFloat_Check(a[7]))
        return declined();
    if (!row(c, a[3], (int64_t)B * max_blocks, &tables) || !row(c, a[4], B, &lens) || !heads(c, a[1], B, c->Hq, &stride, &q) ||
        !list(c, a[2], B, &top, &selected))
        return declined();
    if (a[9] != Py_None && (!heads(c, a[9], B, c->Hkv, &kv_stride, &k) || !heads(c, a[10], B, c->Hkv, &v_stride, &v) ||
                            kv_stride != v_stride))
        return declined();
    if (a[9] == Py_None && a[10] != Py_None) return declined();
    const int half = is_dtype(a[8], c->bf16);
    if (PyErr_Occurred() || (!half && !is_dtype(a[8], c->f32)) || !has_shape(a[8], B, c->Hq, kDim) || !is_contiguous(a[8]) || !place(c, a[8], &out))
        return declined();
    if (!stream_of(a[11], &stream)) return declined();
    const float scale = (float)PyFloat_AS_DOUBLE(a[7]);
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = c->sparse(c->pool, layer, q, stride, k, v, kv_stride, selected, top, tables, lens, B, max_blocks, scale, out,
                   half ? kOutBf16 : 0, stream);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(rc);
}

/* Calls(pool, index, Hq, Hkv, bounds_bytes, bf16, int32, float32, address of select_blocks, of sparse_attention) */
static int calls_init(Calls *c, PyObject *args, PyObject *kw) {
    unsigned long long pool, select, sparse;
    long long hq, hkv, bytes;
    PyObject *bf16, *i32, *f32;
    (void)kw;
    if (!PyArg_ParseTuple(args, "KlLLLOOOKK", &pool, &c->index, &hq, &hkv, &bytes, &bf16, &i32, &f32, &select, &sparse)) return -1;
    c->pool = (void *)(uintptr_t)pool;
    c->Hq = hq;
    c->Hkv = hkv;
    c->bounds_bytes = bytes;
    c->select = (select_fn)(uintptr_t)select;
    c->sparse = (sparse_fn)(uintptr_t)sparse;
    Py_XSETREF(c->bf16, Py_NewRef(bf16));
    Py_XSETREF(c->i32, Py_NewRef(i32));
    Py_XSETREF(c->f32, Py_NewRef(f32));
    return 0;
}

static void calls_free(Calls *c) {
    Py_XDECREF(c->bf16);
    Py_XDECREF(c->i32);
    Py_XDECREF(c->f32);
    Py_TYPE(c)->tp_free((PyObject *)c);
}

static PyMethodDef calls_methods[] = {
    {"select_blocks", (PyCFunction)(void (*)(void))calls_select, METH_FASTCALL, NULL},
    {"sparse_attention", (PyCFunction)(void (*)(void))calls_sparse, METH_FASTCALL, NULL},
    {NULL, NULL, 0, NULL},
};

static PyTypeObject calls_type = {
    PyVarObject_HEAD_INIT(NULL, 0).tp_name = "_calls.Calls",
    .tp_basicsize = sizeof(Calls),
    .tp_flags = Py_TPFLAGS_DEFAULT,
    .tp_new = PyType_GenericNew,
    .tp_init = (initproc)calls_init,
    .tp_dealloc = (destructor)calls_free,
    .tp_methods = calls_methods,
};

static struct PyModuleDef calls_module = {PyModuleDef_HEAD_INIT, "_calls", NULL, -1, NULL, NULL, NULL, NULL, NULL};

PyMODINIT_FUNC PyInit__calls(void) {
    PyObject **names[] = {&s_dtype, &s_shape, &s_stride, &s_contiguous, &s_numel, &s_nbytes, &s_device, &s_ptr, &s_stream};
    const char *texts[] = {"dtype", "shape", "stride", "is_contiguous", "numel", "nbytes", "get_device", "data_ptr", "cuda_stream"};
    for (int i = 0; i < 9; ++i)
        if (!(*names[i] = PyUnicode_InternFromString(texts[i]))) return NULL;
    if (PyType_Ready(&calls_type) < 0) return NULL;
    PyObject *m = PyModule_Create(&calls_module);
    if (m && PyModule_AddObjectRef(m, "Calls", (PyObject *)&calls_type) < 0) Py_CLEAR(m);
    return m;
}
