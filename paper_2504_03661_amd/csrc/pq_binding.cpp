// The per-step calls of the Python binding (pq_attn_decode, pq_encode_append, the five of the paged cache) without ctypes:
// arguments are taken apart here, the library's functions are called through the addresses that binding.py hands over.  A
// decoding step of one short sequence (32 heads, 1K tokens) is bound by the host: with ctypes the two calls took 13 us of the step, marshalling
// ten pointers each through Python helpers; with this module the step takes 16.1 us, before 22.8.
//
// As binding.py's helpers do it: a pointer argument is None (NULL), an int, or an object with data_ptr(); a stream is
// None (torch's current stream, through the callable handed over), an int, or an object with a cuda_stream attribute.
// The calls run without the interpreter lock and return the library's status.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <stdint.h>

namespace {

typedef int (*decode_fn)(void *, const void *, const uint8_t *, const uint8_t *, const int32_t *, const void *, const void *,
                         const void *, const void *, const int32_t *, float, float *, void *);
typedef int (*append_fn)(void *, const void *, const void *, int32_t, const void *, const void *, uint8_t *, uint8_t *,
                         int32_t *, void *);

PyObject *s_data_ptr, *s_cuda_stream, *s_value;

// false: a Python exception is set
bool pointer(PyObject *o, void **out)
{
    if (o == Py_None) {
        *out = nullptr;
        return true;
    }
    if (PyLong_Check(o)) {
        *out = (void *)(uintptr_t)PyLong_AsUnsignedLongLongMask(o);
        return !PyErr_Occurred();
    }
    PyObject *p = PyObject_CallMethodNoArgs(o, s_data_ptr);
    if (p == nullptr)
        return false;
    PyObject *n = PyNumber_Long(p);
    Py_DECREF(p);
    if (n == nullptr)
        return false;
    *out = (void *)(uintptr_t)PyLong_AsUnsignedLongLongMask(n);
    Py_DECREF(n);
    return !PyErr_Occurred();
}

// the context: None, an int, or a ctypes.c_void_p (binding.py hands over no other)
bool handle(PyObject *o, void **out)
{
    if (o == Py_None || PyLong_Check(o))
        return pointer(o, out);
    PyObject *v = PyObject_GetAttr(o, s_value);
    if (v == nullptr)
        return false;
    const bool ok = pointer(v, out);
    Py_DECREF(v);
    return ok;
}

bool integer(PyObject *o, uint64_t *out)
{
    PyObject *n = PyNumber_Long(o);
    if (n == nullptr)
        return false;
    *out = PyLong_AsUnsignedLongLongMask(n);
    Py_DECREF(n);
    return !PyErr_Occurred();
}

// `current`: called for None; returns the raw stream as an int
bool stream(PyObject *o, PyObject *current, void **out)
{
    PyObject *v = o == Py_None ? PyObject_CallNoArgs(current) : PyLong_Check(o) ? Py_NewRef(o) : PyObject_GetAttr(o, s_cuda_stream);
    if (v == nullptr)
        return false;
    uint64_t n = 0;
    const bool ok = integer(v, &n);
    Py_DECREF(v);
    *out = (void *)(uintptr_t)n;
    return ok;
}

bool count(Py_ssize_t n, Py_ssize_t want)
{
    if (n != want)
        PyErr_Format(PyExc_TypeError, "expected %zd arguments, got %zd", want, n);
    return n == want;
}

// decode(function address, current-stream callable, <the 13 arguments of pq_attn_decode>)
PyObject *decode(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    void *f, *p[11], *s;
    if (!count(n, 15) || !pointer(a[0], &f) || !handle(a[2], &p[0]))
        return nullptr;
    for (int i = 1; i < 10; ++i)  // q, k_codes, v_codes, ctx_len, k_codebook, v_codebook, recent_k, recent_v, recent_len
        if (!pointer(a[2 + i], &p[i]))
            return nullptr;
    PyObject *number = PyNumber_Float(a[12]);
    if (number == nullptr)
        return nullptr;
    const double scale = PyFloat_AS_DOUBLE(number);
    Py_DECREF(number);
    if (!pointer(a[13], &p[10]) || !stream(a[14], a[1], &s))
        return nullptr;
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = ((decode_fn)f)(p[0], p[1], (const uint8_t *)p[2], (const uint8_t *)p[3], (const int32_t *)p[4], p[5], p[6], p[7], p[8],
                        (const int32_t *)p[9], (float)scale, (float *)p[10], s);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(rc);
}

// append(function address, current-stream callable, <the 10 arguments of pq_encode_append>)
PyObject *append(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    void *f, *p[10], *s;
    uint64_t n_new;
    if (!count(n, 12) || !pointer(a[0], &f) || !handle(a[2], &p[0]) || !integer(a[5], &n_new))
        return nullptr;
    for (int i = 1; i < 9; ++i)  // new_k, new_v, (n_new), k_codebook, v_codebook, k_codes, v_codes, ctx_len
        if (i != 3 && !pointer(a[2 + i], &p[i]))
            return nullptr;
    if (!stream(a[11], a[1], &s))
        return nullptr;
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = ((append_fn)f)(p[0], p[1], p[2], (int32_t)(uint32_t)n_new, p[4], p[5], (uint8_t *)p[6], (uint8_t *)p[7],
                        (int32_t *)p[8], s);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(rc);
}

// The five calls of the paged cache: their arguments by kind, in the order of pq_attn.h (h context, p pointer, i int32, l int64,
// f float; the stream comes last).
constexpr int MOST = 16;

union argument {
    void *p;
    int32_t i;
    int64_t l;
    float f;
};

// a: function address, current-stream callable, the arguments
bool arguments(const char *kinds, PyObject *const *a, Py_ssize_t n, void **f, argument *to)
{
    const Py_ssize_t want = (Py_ssize_t)__builtin_strlen(kinds);
    if (!count(n, want + 3) || !pointer(a[0], f))
        return false;
    for (Py_ssize_t k = 0; k < want; ++k) {
        PyObject *o = a[2 + k];
        uint64_t whole;
        bool ok = true;
        if (kinds[k] == 'h') {
            ok = handle(o, &to[k].p);
        } else if (kinds[k] == 'p') {
            ok = pointer(o, &to[k].p);
        } else if (kinds[k] == 'f') {
            PyObject *number = PyNumber_Float(o);
            ok = number != nullptr;
            if (ok) {
                to[k].f = (float)PyFloat_AS_DOUBLE(number);
                Py_DECREF(number);
            }
        } else {
            ok = integer(o, &whole);
            if (ok && kinds[k] == 'i')
                to[k].i = (int32_t)(uint32_t)whole;
            else if (ok)
                to[k].l = (int64_t)whole;
        }
        if (!ok)
            return false;
    }
    return stream(a[2 + want], a[1], &to[want].p);
}

#define PAGED_CALL(NAME, KINDS, TYPE, CALL)                                          \
    PyObject *NAME(PyObject *, PyObject *const *args, Py_ssize_t n)                  \
    {                                                                                \
        void *f;                                                                     \
        argument a[MOST];                                                            \
        if (!arguments(KINDS, args, n, &f, a))                                       \
            return nullptr;                                                          \
        int rc;                                                                      \
        Py_BEGIN_ALLOW_THREADS                                                       \
        rc = ((int (*)TYPE)f)CALL;                                                   \
        Py_END_ALLOW_THREADS                                                         \
        return PyLong_FromLong(rc);                                                  \
    }

typedef void *P;
PAGED_CALL(paged_plan, "hiipppppppppp", (P, int32_t, int32_t, P, P, P, P, P, P, P, P, P, P, P),
           (a[0].p, a[1].i, a[2].i, a[3].p, a[4].p, a[5].p, a[6].p, a[7].p, a[8].p, a[9].p, a[10].p, a[11].p, a[12].p, a[13].p))
PAGED_CALL(paged_append, "hipplppppp", (P, int32_t, P, P, int64_t, P, P, P, P, P, P),
           (a[0].p, a[1].i, a[2].p, a[3].p, a[4].l, a[5].p, a[6].p, a[7].p, a[8].p, a[9].p, a[10].p))
PAGED_CALL(paged_read, "hiippppppppp", (P, int32_t, int32_t, P, P, P, P, P, P, P, P, P, P),
           (a[0].p, a[1].i, a[2].i, a[3].p, a[4].p, a[5].p, a[6].p, a[7].p, a[8].p, a[9].p, a[10].p, a[11].p, a[12].p))
PAGED_CALL(paged_decode, "hiplppppppfp", (P, int32_t, P, int64_t, P, P, P, P, P, P, float, P, P),
           (a[0].p, a[1].i, a[2].p, a[3].l, a[4].p, a[5].p, a[6].p, a[7].p, a[8].p, a[9].p, a[10].f, a[11].p, a[12].p))
PAGED_CALL(paged_prefill, "hiiplppppppppfp", (P, int32_t, int32_t, P, int64_t, P, P, P, P, P, P, P, P, float, P, P),
           (a[0].p, a[1].i, a[2].i, a[3].p, a[4].l, a[5].p, a[6].p, a[7].p, a[8].p, a[9].p, a[10].p, a[11].p, a[12].p, a[13].f,
            a[14].p, a[15].p))

#define METHOD(NAME) {#NAME, (PyCFunction)(void (*)(void))NAME, METH_FASTCALL, nullptr}
PyMethodDef methods[] = {METHOD(decode), METHOD(append), METHOD(paged_plan), METHOD(paged_append), METHOD(paged_read),
                         METHOD(paged_decode), METHOD(paged_prefill), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_pq_calls", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__pq_calls(void)
{
    s_data_ptr = PyUnicode_InternFromString("data_ptr");
    s_cuda_stream = PyUnicode_InternFromString("cuda_stream");
    s_value = PyUnicode_InternFromString("value");
    if (s_data_ptr == nullptr || s_cuda_stream == nullptr || s_value == nullptr)
        return nullptr;
    return PyModule_Create(&module);
}
