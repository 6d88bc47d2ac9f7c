/* Native argument marshalling for the entry points that are called several times per layer: torch tensors (anything with
 * data_ptr()), ints and None become pointers, and the C function is called without the GIL.  The same job through ctypes takes
 * 6-8 us a call for these argument lists -- longer than most of their kernels run; this takes about one.
 *
 * bind(path) looks the functions up in the library the package has loaded; the wrappers take the C function's arguments by
 * position and return its status code. */
#define PY_SSIZE_T_CLEAN
#include <Python.h>
#include <dlfcn.h>
#include <limits.h>
#include <stdint.h>

typedef union {
    void* p;
    int i;
    int64_t l;
    float f;
} arg_t;

static PyObject* s_data_ptr;

/* One argument by its kind: p pointer, i int, l int64, f float.  0, or -1 with an exception set. */
static int convert(PyObject* o, char kind, arg_t* out) {
    if (kind == 'f') {
        const double d = PyFloat_AsDouble(o);
        if (d == -1.0 && PyErr_Occurred()) return -1;
        out->f = (float)d;
        return 0;
    }
    if (kind == 'p') {
        if (o == Py_None) {
            out->p = NULL;
            return 0;
        }
        if (PyLong_Check(o)) {
            out->p = PyLong_AsVoidPtr(o);
        } else {
            PyObject* v = PyObject_CallMethodNoArgs(o, s_data_ptr);
            if (!v) return -1;
            out->p = PyLong_AsVoidPtr(v);
            Py_DECREF(v);
        }
        return out->p == NULL && PyErr_Occurred() ? -1 : 0;
    }
    const long long v = PyLong_AsLongLong(o);
    if (v == -1 && PyErr_Occurred()) return -1;
    if (kind == 'l') {
        out->l = v;
        return 0;
    }
    if (v < INT_MIN || v > INT_MAX) {
        PyErr_SetString(PyExc_OverflowError, "argument does not fit a C int");
        return -1;
    }
    out->i = (int)v;
    return 0;
}

static int convert_all(const char* name, const char* kinds, PyObject* const* args, Py_ssize_t n, arg_t* a) {
    Py_ssize_t k = 0;
    for (; kinds[k]; ++k) {
        if (k >= n) break;
        if (convert(args[k], kinds[k], &a[k]) != 0) return -1;
    }
    if (kinds[k] || k != n) {
        PyErr_Format(PyExc_TypeError, "%s: wrong number of arguments (%zd)", name, n);
        return -1;
    }
    return 0;
}

typedef int (*reserve_fn)(void*, int, int, void*, void*, void*, void*, void*, void*, void*, void*, void*, void*, int, void*, void*, void*);
typedef int (*rope_fn)(void*, int, void*, int64_t, void*, void*, float, void*, int, int, int, void*, void*, void*, void*, int, int, float, float, void*);
typedef int (*append_fn)(void*, int, int, void*, void*, void*, int, void*, void*, void*, float, float, void*);
typedef int (*read_fn)(void*, int, int, void*, int, void*, void*, void*, float, float, void*, void*, void*);
typedef int (*attn_fn)(void*, int, int, void*, void*, int, void*, void*, void*, void*, void*, float, float, void*, void*);

static reserve_fn f_reserve;
static rope_fn f_rope;
static append_fn f_append;
static read_fn f_read;
static attn_fn f_attn;

#define WRAPPER(NAME, FN, KINDS, CALL)                                                              \
    static PyObject* NAME(PyObject* self, PyObject* const* args, Py_ssize_t n) {                    \
        arg_t a[24];                                                                                \
        int code;                                                                                   \
        (void)self;                                                                                 \
        if (!FN) {                                                                                  \
            PyErr_SetString(PyExc_RuntimeError, #NAME ": bind() has not been called");              \
            return NULL;                                                                            \
        }                                                                                           \
        if (convert_all(#NAME, KINDS, args, n, a) != 0) return NULL;                                \
        Py_BEGIN_ALLOW_THREADS                                                                      \
        code = CALL;                                                                                \
        Py_END_ALLOW_THREADS                                                                        \
        return PyLong_FromLong(code);                                                               \
    }

WRAPPER(fd_kv_reserve, f_reserve, "piippppppppppippp",
        f_reserve(a[0].p, a[1].i, a[2].i, a[3].p, a[4].p, a[5].p, a[6].p, a[7].p, a[8].p, a[9].p, a[10].p, a[11].p, a[12].p, a[13].i, a[14].p,
                  a[15].p, a[16].p))
WRAPPER(fd_qk_norm_rope_append, f_rope, "piplppfpiiippppiiffp",
        f_rope(a[0].p, a[1].i, a[2].p, a[3].l, a[4].p, a[5].p, a[6].f, a[7].p, a[8].i, a[9].i, a[10].i, a[11].p, a[12].p, a[13].p, a[14].p, a[15].i,
               a[16].i, a[17].f, a[18].f, a[19].p))
WRAPPER(fd_kv_append_fp4, f_append, "piipppipppffp",
        f_append(a[0].p, a[1].i, a[2].i, a[3].p, a[4].p, a[5].p, a[6].i, a[7].p, a[8].p, a[9].p, a[10].f, a[11].f, a[12].p))
WRAPPER(fd_kv_read_fp4, f_read, "piipipppffppp",
        f_read(a[0].p, a[1].i, a[2].i, a[3].p, a[4].i, a[5].p, a[6].p, a[7].p, a[8].f, a[9].f, a[10].p, a[11].p, a[12].p))
WRAPPER(fd_attn_draft_verify_fp4, f_attn, "piippipppppffpp",
        f_attn(a[0].p, a[1].i, a[2].i, a[3].p, a[4].p, a[5].i, a[6].p, a[7].p, a[8].p, a[9].p, a[10].p, a[11].f, a[12].f, a[13].p, a[14].p))

static PyObject* bind(PyObject* self, PyObject* path) {
    const char* s = PyUnicode_AsUTF8(path);
    void* lib;
    (void)self;
    if (!s) return NULL;
    lib = dlopen(s, RTLD_NOW);
    if (!lib) {
        PyErr_SetString(PyExc_OSError, dlerror());
        return NULL;
    }
    f_reserve = (reserve_fn)dlsym(lib, "fd_kv_reserve");
    f_rope = (rope_fn)dlsym(lib, "fd_qk_norm_rope_append");
    f_append = (append_fn)dlsym(lib, "fd_kv_append_fp4");
    f_read = (read_fn)dlsym(lib, "fd_kv_read_fp4");
    f_attn = (attn_fn)dlsym(lib, "fd_attn_draft_verify_fp4");
    if (!f_reserve || !f_rope || !f_append || !f_read || !f_attn) {
        PyErr_SetString(PyExc_OSError, "the library lacks an entry point");
        return NULL;
    }
    Py_RETURN_NONE;
}

#define METHOD(NAME) {#NAME, (PyCFunction)(void (*)(void))NAME, METH_FASTCALL, NULL}
static PyMethodDef methods[] = {METHOD(fd_kv_reserve), METHOD(fd_qk_norm_rope_append), METHOD(fd_kv_append_fp4), METHOD(fd_kv_read_fp4),
                                METHOD(fd_attn_draft_verify_fp4), {"bind", bind, METH_O, NULL}, {NULL, NULL, 0, NULL}};
static struct PyModuleDef module = {PyModuleDef_HEAD_INIT, "_marshal", NULL, -1, methods, NULL, NULL, NULL, NULL};

PyMODINIT_FUNC PyInit__marshal(void) {
    s_data_ptr = PyUnicode_InternFromString("data_ptr");
    return s_data_ptr ? PyModule_Create(&module) : NULL;
}
