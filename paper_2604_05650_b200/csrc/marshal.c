/* Python's side of the calls that a decoding loop makes by the dozen: arguments turned into the C ABI's and the
 * library's function called, without ctypes' conversions.  A pointer is None, an address, an object with
 * data_ptr() (a tensor) or a numpy array; a structure is any object with a buffer of its size.  Returns the status.
 *
 * A call of seventeen arguments, eleven of them tensors: 6.4 us by ctypes, of a call's 10 in all; 1.6 us by this.  The stream, which such a
 * loop sets before each call: 0.44 us and 0.05. */
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include "lvspec.h"

static PyObject *name_data_ptr, *name_ctypes, *name_data;
static __typeof__(&lvspec_set_stream) f_set_stream;
static __typeof__(&lvspec_plan_pages) f_plan_pages;
static __typeof__(&lvspec_append_paged_fp8) f_append;
static __typeof__(&lvspec_verify_attention_paged_fp8) f_attention;
static __typeof__(&lvspec_sample) f_sample;

enum { kMostArgs = 20, kMostBuffers = 2 };
typedef struct {
    uint64_t w[kMostArgs];
    Py_buffer held[kMostBuffers];
    int n_held;
} Args;

static int as_word(PyObject *o, uint64_t *w)
{
    if (!o) return -1;
    *w = PyLong_AsUnsignedLongLong(o);
    return *w == (uint64_t)-1 && PyErr_Occurred() ? -1 : 0;
}
static int pointer(PyObject *o, uint64_t *w)
{
    if (o == Py_None) {
        *w = 0;
        return 0;
    }
    if (PyLong_Check(o)) return as_word(o, w);
    PyObject *a = PyObject_CallMethodNoArgs(o, name_data_ptr);
    if (!a && PyErr_ExceptionMatches(PyExc_AttributeError)) {
        PyErr_Clear();
        PyObject *c = PyObject_GetAttr(o, name_ctypes);
        if (!c) return -1;
        a = PyObject_GetAttr(c, name_data);
        Py_DECREF(c);
    }
    const int bad = as_word(a, w);
    Py_XDECREF(a);
    return bad;
}
static int whole(PyObject *o, uint64_t *w)
{
    PyObject *a = PyNumber_Long(o);
    if (!a) return -1;
    const long long x = PyLong_AsLongLong(a);
    Py_DECREF(a);
    *w = (uint64_t)x;
    return x == -1 && PyErr_Occurred() ? -1 : 0;
}

static PyObject *finish(Args *a, int status)
{
    while (a->n_held > 0) PyBuffer_Release(&a->held[--a->n_held]);
    return PyErr_Occurred() ? NULL : PyLong_FromLong(status);
}
/* kinds: p pointer, i 32-bit and l 64-bit integer, c cache description, s attention shape */
static int take(Args *a, const void *function, const char *kinds, PyObject *const *args, Py_ssize_t n)
{
    a->n_held = 0;
    if (!function || n != (Py_ssize_t)strlen(kinds)) {
        PyErr_Format(PyExc_TypeError, function ? "%zd arguments given, %zu expected" : "not bound to the library", n, strlen(kinds));
        return -1;
    }
    for (Py_ssize_t i = 0; i < n; ++i) {
        int bad;
        if (kinds[i] == 'p') {
            bad = pointer(args[i], &a->w[i]);
        } else if (kinds[i] == 'i' || kinds[i] == 'l') {
            bad = whole(args[i], &a->w[i]);
        } else {
            const size_t size = kinds[i] == 'c' ? sizeof(lvspec_paged_fp8_t) : sizeof(lvspec_attn_shape_t);
            Py_buffer *b = &a->held[a->n_held];
            bad = PyObject_GetBuffer(args[i], b, PyBUF_SIMPLE);
            if (!bad) {
                ++a->n_held;
                a->w[i] = (uint64_t)(uintptr_t)b->buf;
                if ((size_t)b->len != size) {
                    PyErr_SetString(PyExc_TypeError, "a structure of another size");
                    bad = -1;
                }
            }
        }
        if (bad) {
            finish(a, 0);
            return -1;
        }
    }
    return 0;
}
#define P(T, k) ((T)(uintptr_t)a.w[k])
#define I(k) ((int32_t)a.w[k])
#define L(k) ((int64_t)a.w[k])

static PyObject *set_stream(PyObject *self, PyObject *const *args, Py_ssize_t n)
{
    (void)self;
    Args a;
    if (take(&a, f_set_stream, "pp", args, n)) return NULL;
    return finish(&a, f_set_stream(P(void *, 0), P(void *, 1)));
}
static PyObject *plan_pages(PyObject *self, PyObject *const *args, Py_ssize_t n)
{
    (void)self;
    Args a;
    int st;
    if (take(&a, f_plan_pages, "piiiiippppppppppp", args, n)) return NULL;
    Py_BEGIN_ALLOW_THREADS
    st = f_plan_pages(P(void *, 0), I(1), I(2), I(3), I(4), I(5), P(void *, 6), P(void *, 7), P(void *, 8), P(void *, 9), P(void *, 10),
                      P(void *, 11), P(void *, 12), P(void *, 13), P(void *, 14), P(void *, 15), P(void *, 16));
    Py_END_ALLOW_THREADS
    return finish(&a, st);
}
static PyObject *append_paged_fp8(PyObject *self, PyObject *const *args, Py_ssize_t n)
{
    (void)self;
    Args a;
    int st;
    if (take(&a, f_append, "piiicppllppppp", args, n)) return NULL;
    Py_BEGIN_ALLOW_THREADS
    st = f_append(P(void *, 0), I(1), I(2), I(3), P(void *, 4), P(void *, 5), P(void *, 6), L(7), L(8), P(void *, 9), P(void *, 10),
                  P(void *, 11), P(void *, 12), P(void *, 13));
    Py_END_ALLOW_THREADS
    return finish(&a, st);
}
static PyObject *verify_attention_paged_fp8(PyObject *self, PyObject *const *args, Py_ssize_t n)
{
    (void)self;
    Args a;
    int st;
    if (take(&a, f_attention, "pscii" "pppppppppp", args, n)) return NULL;
    Py_BEGIN_ALLOW_THREADS
    st = f_attention(P(void *, 0), P(void *, 1), P(void *, 2), I(3), I(4), P(void *, 5), P(void *, 6), P(void *, 7), P(void *, 8),
                     P(void *, 9), P(void *, 10), P(void *, 11), P(void *, 12), P(void *, 13), P(void *, 14));
    Py_END_ALLOW_THREADS
    return finish(&a, st);
}
static PyObject *sample(PyObject *self, PyObject *const *args, Py_ssize_t n)
{
    (void)self;
    Args a;
    int st;
    if (take(&a, f_sample, "piiiplppppppp", args, n)) return NULL;
    Py_BEGIN_ALLOW_THREADS
    st = f_sample(P(void *, 0), I(1), I(2), I(3), P(void *, 4), L(5), P(void *, 6), P(void *, 7), P(void *, 8), P(void *, 9),
                  P(void *, 10), P(void *, 11), P(void *, 12));
    Py_END_ALLOW_THREADS
    return finish(&a, st);
}
/* bind(addresses of the functions, in the order of the methods below) */
static PyObject *bind(PyObject *self, PyObject *args)
{
    (void)self;
    unsigned long long f[5];
    if (!PyArg_ParseTuple(args, "KKKKK", &f[0], &f[1], &f[2], &f[3], &f[4])) return NULL;
    f_set_stream = (__typeof__(f_set_stream))(uintptr_t)f[0];
    f_plan_pages = (__typeof__(f_plan_pages))(uintptr_t)f[1];
    f_append = (__typeof__(f_append))(uintptr_t)f[2];
    f_attention = (__typeof__(f_attention))(uintptr_t)f[3];
    f_sample = (__typeof__(f_sample))(uintptr_t)f[4];
    Py_RETURN_NONE;
}

static PyMethodDef methods[] = {
    {"set_stream", (PyCFunction)(void (*)(void))set_stream, METH_FASTCALL, NULL},
    {"plan_pages", (PyCFunction)(void (*)(void))plan_pages, METH_FASTCALL, NULL},
    {"append_paged_fp8", (PyCFunction)(void (*)(void))append_paged_fp8, METH_FASTCALL, NULL},
    {"verify_attention_paged_fp8", (PyCFunction)(void (*)(void))verify_attention_paged_fp8, METH_FASTCALL, NULL},
    {"sample", (PyCFunction)(void (*)(void))sample, METH_FASTCALL, NULL},
    {"bind", bind, METH_VARARGS, NULL},
    {NULL, NULL, 0, NULL}};
static struct PyModuleDef module = {PyModuleDef_HEAD_INIT, "_marshal", NULL, -1, methods, NULL, NULL, NULL, NULL};

PyMODINIT_FUNC PyInit__marshal(void)
{
    name_data_ptr = PyUnicode_InternFromString("data_ptr");
    name_ctypes = PyUnicode_InternFromString("ctypes");
    name_data = PyUnicode_InternFromString("data");
    return name_data_ptr && name_ctypes && name_data ? PyModule_Create(&module) : NULL;
}
