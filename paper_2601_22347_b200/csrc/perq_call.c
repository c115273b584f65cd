/* CPython entries to the calls of the online path, the 8-bit layers and the 8-bit cache: integers to C arguments, and the call without the interpreter lock.
 *
 * Small calls are bound by the host.  Of 4.8 us for one row, the general converter of foreign functions took 0.95 (its own call, one
 * object for each argument); this takes 0.2 (one row of 2048: 4.84 -> 4.1 us between calls).  Arguments that are not plain integers (None: a null pointer) are refused with a
 * TypeError, upon which the caller takes the general converter, so that what is accepted and what is raised stay its own. */
#define PY_SSIZE_T_CLEAN
#include <Python.h>
#include <stdint.h>

typedef int (*rotate_fn)(const void *, const int32_t *, int64_t, int32_t, int32_t, int32_t, int32_t, void *, void *, void *);
typedef int (*swiglu_fn)(const void *, const void *, const int32_t *, int64_t, int32_t, int32_t, int32_t, int32_t, void *, void *, void *);

typedef int (*rows_fn)(const void *, const int32_t *, int64_t, int32_t, int32_t, void *, void *, void *);
typedef int (*product_fn)(const void *, const void *, int32_t, const void *, const void *, int32_t, const void *, int64_t, int32_t, int32_t, void *, int32_t, void *,
                          size_t, void *);
typedef int (*grouped_fn)(const void *, const void *, int32_t, const void *, const void *, int32_t, const void *, const void *, int64_t, int32_t, int32_t, int32_t,
                          void *, int32_t, void *, size_t, void *);

typedef int (*cache_write_fn)(const void *, const void *, int32_t, int64_t, int64_t, const void *, const void *, const void *, int64_t, int32_t, int32_t, int32_t, int32_t, int32_t,
                              int64_t, int32_t, void *, void *, void *, void *, void *);
typedef int (*cache_read_fn)(const void *, const void *, const void *, const void *, const void *, const void *, const void *, int64_t, int32_t, int32_t, int32_t, int32_t, int32_t, int64_t,
                             int32_t, void *, void *, int32_t, void *);
typedef int (*attention_fn)(const void *, int32_t, int64_t, const void *, const void *, const void *, const void *, const void *, const void *, const void *, int64_t, int32_t, int32_t, int32_t,
                            int32_t, int32_t, int32_t, int64_t, int32_t, int32_t, float, int32_t, int32_t, void *, int32_t, void *, size_t, void *);

static rotate_fn rotate = NULL;
static swiglu_fn swiglu = NULL;
static rows_fn rows = NULL;
static product_fn product = NULL;
static grouped_fn grouped = NULL;
static cache_write_fn cache_write = NULL;
static cache_read_fn cache_read = NULL;
static attention_fn attention = NULL;

/* n arguments: numbers where `numbers` has a bit, the others addresses. */
static int convert_mixed(PyObject *const *args, Py_ssize_t n, Py_ssize_t expected, unsigned numbers, unsigned long long *a)
{
    if (n != expected) { PyErr_SetString(PyExc_TypeError, "number of arguments"); return 0; }
    for (int i = 0; i < n; ++i) {
        const int number = (numbers >> i) & 1u;
        if (args[i] == Py_None && !number) { a[i] = 0; continue; }
        if (!PyLong_Check(args[i])) { PyErr_SetString(PyExc_TypeError, "an integer is required"); return 0; }
        a[i] = PyLong_AsUnsignedLongLongMask(args[i]);
    }
    return 1;
}
/* (five numbers from `first` on) */
static int convert(PyObject *const *args, Py_ssize_t n, Py_ssize_t expected, int first, unsigned long long *a)
{
    return convert_mixed(args, n, expected, 31u << first, a);
}
#define ADDRESS(v) ((void *)(uintptr_t)(v))

static PyObject *rotate_quantize(PyObject *self, PyObject *const *args, Py_ssize_t n)
{
    unsigned long long a[10];
    int rc;
    (void)self;
    if (!convert(args, n, 10, 2, a)) return NULL;
    Py_BEGIN_ALLOW_THREADS
    rc = rotate(ADDRESS(a[0]), ADDRESS(a[1]), (int64_t)a[2], (int32_t)a[3], (int32_t)a[4], (int32_t)a[5], (int32_t)a[6], ADDRESS(a[7]), ADDRESS(a[8]),
                ADDRESS(a[9]));
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(rc);
}

static PyObject *swiglu_rotate_quantize(PyObject *self, PyObject *const *args, Py_ssize_t n)
{
    unsigned long long a[11];
    int rc;
    (void)self;
    if (!convert(args, n, 11, 3, a)) return NULL;
    Py_BEGIN_ALLOW_THREADS
    rc = swiglu(ADDRESS(a[0]), ADDRESS(a[1]), ADDRESS(a[2]), (int64_t)a[3], (int32_t)a[4], (int32_t)a[5], (int32_t)a[6], (int32_t)a[7], ADDRESS(a[8]),
                ADDRESS(a[9]), ADDRESS(a[10]));
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(rc);
}

static PyObject *rotate_quantize_i8(PyObject *self, PyObject *const *args, Py_ssize_t n)
{
    unsigned long long a[8];
    int rc;
    (void)self;
    if (!convert_mixed(args, n, 8, 0x1cu, a)) return NULL;
    Py_BEGIN_ALLOW_THREADS
    rc = rows(ADDRESS(a[0]), ADDRESS(a[1]), (int64_t)a[2], (int32_t)a[3], (int32_t)a[4], ADDRESS(a[5]), ADDRESS(a[6]), ADDRESS(a[7]));
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(rc);
}

static PyObject *matmul_i8(PyObject *self, PyObject *const *args, Py_ssize_t n)
{
    unsigned long long a[15];
    int rc;
    (void)self;
    if (!convert_mixed(args, n, 15, 0x2ba4u, a)) return NULL;
    Py_BEGIN_ALLOW_THREADS
    rc = product(ADDRESS(a[0]), ADDRESS(a[1]), (int32_t)a[2], ADDRESS(a[3]), ADDRESS(a[4]), (int32_t)a[5], ADDRESS(a[6]), (int64_t)a[7], (int32_t)a[8],
                 (int32_t)a[9], ADDRESS(a[10]), (int32_t)a[11], ADDRESS(a[12]), (size_t)a[13], ADDRESS(a[14]));
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(rc);
}

static PyObject *grouped_matmul_i8(PyObject *self, PyObject *const *args, Py_ssize_t n)
{
    unsigned long long a[17];
    int rc;
    (void)self;
    if (!convert_mixed(args, n, 17, 0xaf24u, a)) return NULL;
    Py_BEGIN_ALLOW_THREADS
    rc = grouped(ADDRESS(a[0]), ADDRESS(a[1]), (int32_t)a[2], ADDRESS(a[3]), ADDRESS(a[4]), (int32_t)a[5], ADDRESS(a[6]), ADDRESS(a[7]), (int64_t)a[8],
                 (int32_t)a[9], (int32_t)a[10], (int32_t)a[11], ADDRESS(a[12]), (int32_t)a[13], ADDRESS(a[14]), (size_t)a[15], ADDRESS(a[16]));
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(rc);
}

static PyObject *cache_write_i8(PyObject *self, PyObject *const *args, Py_ssize_t n)
{
    unsigned long long a[21];
    int rc;
    (void)self;
    if (!convert_mixed(args, n, 21, 0xff1cu, a)) return NULL;
    Py_BEGIN_ALLOW_THREADS
    rc = cache_write(ADDRESS(a[0]), ADDRESS(a[1]), (int32_t)a[2], (int64_t)a[3], (int64_t)a[4], ADDRESS(a[5]), ADDRESS(a[6]), ADDRESS(a[7]), (int64_t)a[8], (int32_t)a[9], (int32_t)a[10],
                     (int32_t)a[11], (int32_t)a[12], (int32_t)a[13], (int64_t)a[14], (int32_t)a[15], ADDRESS(a[16]), ADDRESS(a[17]), ADDRESS(a[18]), ADDRESS(a[19]), ADDRESS(a[20]));
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(rc);
}

static PyObject *cache_read_i8(PyObject *self, PyObject *const *args, Py_ssize_t n)
{
    unsigned long long a[19];
    int rc;
    (void)self;
    if (!convert_mixed(args, n, 19, 0x27f80u, a)) return NULL;
    Py_BEGIN_ALLOW_THREADS
    rc = cache_read(ADDRESS(a[0]), ADDRESS(a[1]), ADDRESS(a[2]), ADDRESS(a[3]), ADDRESS(a[4]), ADDRESS(a[5]), ADDRESS(a[6]), (int64_t)a[7], (int32_t)a[8], (int32_t)a[9], (int32_t)a[10],
                    (int32_t)a[11], (int32_t)a[12], (int64_t)a[13], (int32_t)a[14], ADDRESS(a[15]), ADDRESS(a[16]), (int32_t)a[17], ADDRESS(a[18]));
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(rc);
}

/* (argument 20, the logits' scale, is a float) */
static PyObject *attention_i8(PyObject *self, PyObject *const *args, Py_ssize_t n)
{
    unsigned long long a[28];
    PyObject *plain[28];
    double scale;
    int rc;
    (void)self;
    if (n != 28 || !PyFloat_Check(args[20])) { PyErr_SetString(PyExc_TypeError, "number of arguments, or a float"); return NULL; }
    scale = PyFloat_AS_DOUBLE(args[20]);
    for (int i = 0; i < 28; ++i) plain[i] = i == 20 ? args[1] : args[i];
    if (!convert_mixed(plain, n, 28, 0x57ffc06u, a)) return NULL;
    Py_BEGIN_ALLOW_THREADS
    rc = attention(ADDRESS(a[0]), (int32_t)a[1], (int64_t)a[2], ADDRESS(a[3]), ADDRESS(a[4]), ADDRESS(a[5]), ADDRESS(a[6]), ADDRESS(a[7]), ADDRESS(a[8]), ADDRESS(a[9]), (int64_t)a[10],
                   (int32_t)a[11], (int32_t)a[12], (int32_t)a[13], (int32_t)a[14], (int32_t)a[15], (int32_t)a[16], (int64_t)a[17], (int32_t)a[18], (int32_t)a[19], (float)scale,
                   (int32_t)a[21], (int32_t)a[22], ADDRESS(a[23]), (int32_t)a[24], ADDRESS(a[25]), (size_t)a[26], ADDRESS(a[27]));
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(rc);
}

static PyObject *bind_cache(PyObject *self, PyObject *const *args, Py_ssize_t n)
{
    (void)self;
    if (n != 3) { PyErr_SetString(PyExc_TypeError, "number of arguments"); return NULL; }
    void *const w = PyLong_AsVoidPtr(args[0]), *const r = PyLong_AsVoidPtr(args[1]), *const t = PyLong_AsVoidPtr(args[2]);
    if (PyErr_Occurred()) return NULL;
    cache_write = (cache_write_fn)w;
    cache_read = (cache_read_fn)r;
    attention = (attention_fn)t;
    Py_RETURN_NONE;
}

static PyObject *bind_i8(PyObject *self, PyObject *const *args, Py_ssize_t n)
{
    (void)self;
    if (n != 3) { PyErr_SetString(PyExc_TypeError, "number of arguments"); return NULL; }
    void *const r = PyLong_AsVoidPtr(args[0]), *const m = PyLong_AsVoidPtr(args[1]), *const g = PyLong_AsVoidPtr(args[2]);
    if (PyErr_Occurred()) return NULL;
    rows = (rows_fn)r;
    product = (product_fn)m;
    grouped = (grouped_fn)g;
    Py_RETURN_NONE;
}

static PyObject *bind(PyObject *self, PyObject *const *args, Py_ssize_t n)
{
    (void)self;
    if (n != 2) { PyErr_SetString(PyExc_TypeError, "number of arguments"); return NULL; }
    void *const r = PyLong_AsVoidPtr(args[0]), *const s = PyLong_AsVoidPtr(args[1]);
    if (PyErr_Occurred()) return NULL;
    rotate = (rotate_fn)r;
    swiglu = (swiglu_fn)s;
    Py_RETURN_NONE;
}

static PyMethodDef methods[] = {
    {"rotate_quantize", (PyCFunction)(void (*)(void))rotate_quantize, METH_FASTCALL, "perq_rotate_quantize(x, perm, T, d, b, fmt, group, codes, scales, stream)"},
    {"swiglu_rotate_quantize", (PyCFunction)(void (*)(void))swiglu_rotate_quantize, METH_FASTCALL, "perq_swiglu_rotate_quantize(gate, up, perm, T, d, b, fmt, group, codes, scales, stream)"},
    {"rotate_quantize_i8", (PyCFunction)(void (*)(void))rotate_quantize_i8, METH_FASTCALL, "perq_rotate_quantize_i8(x, perm, T, d, b, codes, scales, stream)"},
    {"matmul_i8", (PyCFunction)(void (*)(void))matmul_i8, METH_FASTCALL, "perq_matmul_i8(a, a_scales, a_fmt, w, w_scales, w_fmt, w_sums, T, N, d, out, type, workspace, bytes, stream)"},
    {"grouped_matmul_i8", (PyCFunction)(void (*)(void))grouped_matmul_i8, METH_FASTCALL, "perq_grouped_matmul_i8(a, a_scales, a_fmt, w, w_scales, w_fmt, w_sums, offsets, T, E, N, d, out, type, workspace, bytes, stream)"},
    {"cache_write_i8", (PyCFunction)(void (*)(void))cache_write_i8, METH_FASTCALL, "perq_cache_write_i8(...), its 21 arguments in their order"},
    {"cache_read_i8", (PyCFunction)(void (*)(void))cache_read_i8, METH_FASTCALL, "perq_cache_read_i8(...), its 19 arguments in their order"},
    {"attention_i8", (PyCFunction)(void (*)(void))attention_i8, METH_FASTCALL, "perq_attention_i8(...), its 28 arguments in their order"},
    {"bind_cache", (PyCFunction)(void (*)(void))bind_cache, METH_FASTCALL, "The addresses of these three; before any call of theirs."},
    {"bind_i8", (PyCFunction)(void (*)(void))bind_i8, METH_FASTCALL, "The addresses of these three; before any call of theirs."},
    {"bind", (PyCFunction)(void (*)(void))bind, METH_FASTCALL, "The addresses of both; before any call."},
    {NULL, NULL, 0, NULL},
};
static struct PyModuleDef module = {PyModuleDef_HEAD_INIT, "_perq_call", NULL, -1, methods, NULL, NULL, NULL, NULL};

PyMODINIT_FUNC PyInit__perq_call(void) { return PyModule_Create(&module); }
