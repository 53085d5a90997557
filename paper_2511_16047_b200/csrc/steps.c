/* Python side of the calls of a generation step (amskv_append, amskv_attend, amskv_append_attend, amskv_rotary, amskv_cross_attend): takes addresses and strides
 * out of the tensors and calls the library, without the argument conversions of ctypes.  Marshalling only, and only of the
 * usual forms: a call with any other argument returns None without having called the library, and the binding makes it
 * through ctypes, which decides what is accepted and what the error is.
 *
 * These calls are made layers x scales times per image; through ctypes their Python side took 2.1 us with contiguous tensors
 * and 3.3 us with views, about what the launch itself takes; here 0.8 and 1.4.
 *
 * The usual forms: a handle, layer, scale or address that is exactly an int (None as an address), a tensor with data_ptr(),
 * is_contiguous() and stride() (a torch tensor), a stream that is None, an int or has an int as .cuda_stream.
 * The library's functions are handed over by bind() as addresses, so this module is independent of where it was loaded from.
 */
#define PY_SSIZE_T_CLEAN
#include <Python.h>
#include <stdint.h>

#include "../../include/amskv.h"

typedef int (*rotary_fn)(const amskv_rotary_spec*, const float*, int64_t, int64_t, const int32_t*, int64_t, int, int, int, int, const void*,
                         const int64_t*, void*, const int64_t*, int, const void*, const int64_t*, void*, const int64_t*, uint32_t, void*);
typedef int (*cross_fn)(void*, int, const amskv_encoder*, const void*, const void*, const int64_t*, const void*, void*, const int64_t*,
                        const int64_t*, void*);
static rotary_fn f_rotary;
static cross_fn f_cross;
typedef int (*append_fn)(void*, int, int, const void*, const void*, const int64_t*, void*);
typedef int (*attend_fn)(void*, int, int, const void*, void*, const int64_t*, const int64_t*, void*);
typedef int (*append_attend_fn)(void*, int, int, const void*, const void*, const int64_t*, const void*, void*, const int64_t*,
                                const int64_t*, void*);
static append_fn f_append;
static attend_fn f_attend;
static append_attend_fn f_append_attend;
static PyObject *s_data_ptr, *s_is_contiguous, *s_stride, *s_cuda_stream, *s_dtype, *s_numel, *s_shape, *s_torch;
static PyObject *torch_int32, *torch_float32; /* looked up when a tensor is first checked for them */

/* The helpers below return 0, or -1 for an argument that is left to ctypes (with or without an error set). */

static int as_pointer(PyObject* o, void** out) /* an int, or None */
{
    if (o == Py_None) {
        *out = NULL;
        return 0;
    }
    if (!PyLong_CheckExact(o)) return -1;
    *out = (void*)(uintptr_t)PyLong_AsUnsignedLongLongMask(o);
    return 0;
}

/* address of a tensor argument; strides[3] and *strided = 1 when it is a view that is not contiguous */
static int tensor(PyObject* x, void** addr, int64_t* strides, int* strided)
{
    *strided = 0;
    if (x == Py_None || PyLong_CheckExact(x)) return as_pointer(x, addr);
    PyObject* r = PyObject_CallMethodNoArgs(x, s_data_ptr);
    if (!r) return -1;
    const int bad = as_pointer(r, addr);
    Py_DECREF(r);
    if (bad) return -1;
    r = PyObject_CallMethodNoArgs(x, s_is_contiguous);
    if (!r) return -1;
    const int contiguous = r == Py_True ? 1 : r == Py_False ? 0 : -1;
    Py_DECREF(r);
    if (contiguous) return contiguous < 0 ? -1 : 0;
    r = PyObject_CallMethodNoArgs(x, s_stride);
    if (!r) return -1;
    int ok = PyTuple_Check(r) && PyTuple_GET_SIZE(r) == 4;
    for (int i = 0; ok && i < 4; ++i) {
        const long long v = PyLong_AsLongLong(PyTuple_GET_ITEM(r, i));
        if (i < 3) strides[i] = v;
        ok = i < 3 ? !PyErr_Occurred() : v == 1;
    }
    Py_DECREF(r);
    *strided = 1;
    return ok ? 0 : -1;
}

static int as_int(PyObject* o, int* out)
{
    if (!PyLong_CheckExact(o)) return -1;
    const long v = PyLong_AsLong(o);
    *out = (int)v;
    return PyErr_Occurred() || v != *out ? -1 : 0;
}

static int as_int64(PyObject* o, int64_t* out)
{
    if (!PyLong_CheckExact(o)) return -1;
    *out = PyLong_AsLongLong(o);
    return PyErr_Occurred() ? -1 : 0;
}

/* whether a tensor's elements are of the type `name` of torch */
static int is_of(PyObject* x, PyObject** type, const char* name)
{
    if (!*type) {
        PyObject* torch = PyImport_GetModule(s_torch);
        if (!torch) return -1;
        *type = PyObject_GetAttrString(torch, name);
        Py_DECREF(torch);
        if (!*type) return -1;
    }
    PyObject* d = PyObject_GetAttr(x, s_dtype);
    if (!d) return -1;
    const int same = d == *type;
    Py_DECREF(d);
    return same ? 0 : -1;
}

/* address of a contiguous list of at least `count` numbers of a type: None, an int or a tensor */
static int list_of(PyObject* x, PyObject** type, const char* name, int64_t count, void** out)
{
    int64_t s[3], n = 0;
    int strided;
    if (tensor(x, out, s, &strided) || strided) return -1;
    if (x == Py_None || PyLong_CheckExact(x)) return 0;
    if (is_of(x, type, name)) return -1;
    PyObject* r = PyObject_CallMethodNoArgs(x, s_numel);
    if (!r) return -1;
    const int bad = as_int64(r, &n);
    Py_DECREF(r);
    return bad || n < count ? -1 : 0;
}

/* extents of a tensor into shape[most]; the number of dimensions, or -1 */
static int shape_of(PyObject* x, int64_t* shape, int most)
{
    PyObject* r = PyObject_GetAttr(x, s_shape);
    if (!r) return -1;
    int n = PyTuple_Check(r) && PyTuple_GET_SIZE(r) <= most ? (int)PyTuple_GET_SIZE(r) : -1;
    for (int i = 0; i < n; ++i)
        if (as_int64(PyTuple_GET_ITEM(r, i), &shape[i])) n = -1;
    Py_DECREF(r);
    return n;
}

/* address of a list of table rows, and the stride of its rows: None, an int with `given`, or a tensor [T] or [rows, T] */
static int index_of(PyObject* x, PyObject* given, int rows, int T, void** addr, int64_t* row_stride)
{
    *row_stride = 0;
    if (given != Py_None && as_int64(given, row_stride)) return -1;
    if (x == Py_None || PyLong_CheckExact(x)) return as_pointer(x, addr);
    int64_t shape[2];
    if (is_of(x, &torch_int32, "int32") || shape_of(x, shape, 2) < 1) return -1;
    PyObject* r = PyObject_CallMethodNoArgs(x, s_data_ptr);
    if (!r) return -1;
    const int bad = as_pointer(r, addr);
    Py_DECREF(r);
    if (bad) return -1;
    r = PyObject_CallMethodNoArgs(x, s_stride);
    if (!r) return -1;
    const Py_ssize_t n = PyTuple_Check(r) ? PyTuple_GET_SIZE(r) : 0;
    int64_t last = 0, first = 0;
    int ok = (n == 1 || n == 2) && !as_int64(PyTuple_GET_ITEM(r, n - 1), &last) && last == 1 && !as_int64(PyTuple_GET_ITEM(r, 0), &first);
    Py_DECREF(r);
    if (!ok) return -1;
    if (given == Py_None) {
        *row_stride = n == 2 ? first : 0;
        return shape[n - 1] >= T && (n == 1 || shape[0] >= rows) ? 0 : -1;
    }
    const __int128 there = shape[0] < 1 || shape[n - 1] < 1 ? 0 : (n == 2 ? (__int128)(shape[0] - 1) * first : 0) + shape[n - 1];
    return (__int128)(rows - 1) * *row_stride + T <= there ? 0 : -1;
}

static int stream_of(PyObject* s, void** out) /* None, an address, or something with .cuda_stream */
{
    if (s == Py_None || PyLong_CheckExact(s)) return as_pointer(s, out);
    PyObject* a = PyObject_GetAttr(s, s_cuda_stream);
    if (!a) return -1;
    const int bad = as_pointer(a, out);
    Py_DECREF(a);
    return bad;
}

static int head(PyObject* const* args, void** cache, int* layer, int* scale)
{
    if (as_pointer(args[0], cache) || !PyLong_CheckExact(args[1]) || !PyLong_CheckExact(args[2])) return -1;
    const long l = PyLong_AsLong(args[1]), s = PyLong_AsLong(args[2]);
    *layer = (int)l;
    *scale = (int)s;
    return PyErr_Occurred() || l != *layer || s != *scale ? -1 : 0;
}

static int key_value(PyObject* K, PyObject* V, void** k, void** v, int64_t* ks, int* strided)
{
    int64_t vs[3];
    int v_strided;
    if (tensor(K, k, ks, strided) || tensor(V, v, vs, &v_strided)) return -1;
    return *strided != v_strided || (*strided && (ks[0] != vs[0] || ks[1] != vs[1] || ks[2] != vs[2])) ? -1 : 0;
}

static int count(Py_ssize_t n, Py_ssize_t want)
{
    if (n == want && f_append) return 0;
    PyErr_SetString(PyExc_TypeError, f_append ? "wrong number of arguments" : "bind() has not been called");
    return -1;
}

static PyObject* left_to_ctypes(void)
{
    PyErr_Clear();
    Py_RETURN_NONE;
}

/* append(cache, layer, scale, K, V, stream) -> return code, or None */
static PyObject* py_append(PyObject* self, PyObject* const* args, Py_ssize_t n)
{
    void *cache, *k, *v, *stream;
    int layer, scale, kv, rc;
    int64_t ks[3];
    if (count(n, 6)) return NULL;
    if (head(args, &cache, &layer, &scale) || key_value(args[3], args[4], &k, &v, ks, &kv) || stream_of(args[5], &stream))
        return left_to_ctypes();
    Py_BEGIN_ALLOW_THREADS
    rc = f_append(cache, layer, scale, k, v, kv ? ks : NULL, stream);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(rc);
}

/* attend(cache, layer, scale, Q, out, stream) -> return code, or None */
static PyObject* py_attend(PyObject* self, PyObject* const* args, Py_ssize_t n)
{
    void *cache, *q, *o, *stream;
    int layer, scale, qv, ov, rc;
    int64_t qs[3], os[3];
    if (count(n, 6)) return NULL;
    if (head(args, &cache, &layer, &scale) || tensor(args[3], &q, qs, &qv) || tensor(args[4], &o, os, &ov) ||
        stream_of(args[5], &stream))
        return left_to_ctypes();
    Py_BEGIN_ALLOW_THREADS
    rc = f_attend(cache, layer, scale, q, o, qv ? qs : NULL, ov ? os : NULL, stream);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(rc);
}

/* append_attend(cache, layer, scale, K, V, Q, out, stream) -> return code, or None */
static PyObject* py_append_attend(PyObject* self, PyObject* const* args, Py_ssize_t n)
{
    void *cache, *k, *v, *q, *o, *stream;
    int layer, scale, kv, qv, ov, rc;
    int64_t ks[3], qs[3], os[3];
    if (count(n, 8)) return NULL;
    if (head(args, &cache, &layer, &scale) || key_value(args[3], args[4], &k, &v, ks, &kv) || tensor(args[5], &q, qs, &qv) ||
        tensor(args[6], &o, os, &ov) || stream_of(args[7], &stream))
        return left_to_ctypes();
    Py_BEGIN_ALLOW_THREADS
    rc = f_append_attend(cache, layer, scale, k, v, kv ? ks : NULL, q, o, qv ? qs : NULL, ov ? os : NULL, stream);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(rc);
}

/* floats in `rows` rows of a table (arguments that make no sense are the library's to refuse) */
static int64_t floats_of(const amskv_rotary_spec* spec, int64_t rows)
{
    const int64_t d = spec->rotary_dim;
    return rows < 1 || d < 1 ? 0 : rows > INT64_MAX / d ? INT64_MAX : rows * d;
}

/* rotary(spec, table, table_rows, first, index, index_row_stride, rows, T, head_dim, q_heads, Q, Q_out, k_heads, K, K_out, transposed, stream) */
static PyObject* py_rotary(PyObject* self, PyObject* const* a, Py_ssize_t n)
{
    void *table, *index, *q, *qo, *k, *ko, *stream;
    int64_t table_rows, first, index_row, qs[3], qos[3], ks[3], kos[3];
    int rows, T, d, qh, kh, qv, qov, kv, kov, rc;
    Py_buffer spec;
    if (count(n, 17)) return NULL;
    if (!PyObject_CheckBuffer(a[0]) || PyObject_GetBuffer(a[0], &spec, PyBUF_SIMPLE)) return left_to_ctypes();
    if (spec.len != (Py_ssize_t)sizeof(amskv_rotary_spec) || as_int64(a[2], &table_rows) ||
        list_of(a[1], &torch_float32, "float32", floats_of(spec.buf, table_rows), &table) || as_int64(a[3], &first) || as_int(a[6], &rows) ||
        as_int(a[7], &T) || index_of(a[4], a[5], rows, T, &index, &index_row) || as_int(a[8], &d) || as_int(a[9], &qh) || tensor(a[10], &q, qs, &qv) || tensor(a[11], &qo, qos, &qov) || as_int(a[12], &kh) || tensor(a[13], &k, ks, &kv) ||
        tensor(a[14], &ko, kos, &kov) || (a[15] != Py_True && a[15] != Py_False) || stream_of(a[16], &stream)) {
        PyBuffer_Release(&spec);
        return left_to_ctypes();
    }
    Py_BEGIN_ALLOW_THREADS
    rc = f_rotary(spec.buf, table, table_rows, first, index, index_row, rows, T, d, qh, q, qv ? qs : NULL, qo, qov ? qos : NULL, kh, k,
                  kv ? ks : NULL, ko, kov ? kos : NULL, a[15] == Py_True ? AMSKV_ROTARY_TRANSPOSED : 0u, stream);
    Py_END_ALLOW_THREADS
    PyBuffer_Release(&spec);
    return PyLong_FromLong(rc);
}

/* cross_attend(cache, scale, kv_heads, keys, K, V, Q, out, lengths, offsets, max_keys, stream) -> return code, or None */
static PyObject* py_cross_attend(PyObject* self, PyObject* const* a, Py_ssize_t n)
{
    void *cache, *k, *v, *q, *o, *stream, *lengths, *offsets;
    int64_t ks[3], qs[3], os[3], shape[4], rows = 0;
    int scale, kv, qv, ov, rc, heads, keys, max_keys;
    amskv_encoder enc;
    if (count(n, 12)) return NULL;
    if (as_pointer(a[0], &cache) || as_int(a[1], &scale) || as_int(a[2], &heads) || as_int(a[3], &keys) || key_value(a[4], a[5], &k, &v, ks, &kv) ||
        tensor(a[6], &q, qs, &qv) || tensor(a[7], &o, os, &ov) || as_int(a[10], &max_keys) || stream_of(a[11], &stream))
        return left_to_ctypes();
    /* how many rows there are the queries tell, where they are a tensor */
    if ((a[8] != Py_None || a[9] != Py_None) && a[6] != Py_None && !PyLong_CheckExact(a[6])) {
        if (shape_of(a[6], shape, 4) != 4) return left_to_ctypes();
        rows = shape[0];
    }
    if (list_of(a[8], &torch_int32, "int32", rows, &lengths) || list_of(a[9], &torch_int32, "int32", rows ? rows + 1 : 0, &offsets))
        return left_to_ctypes();
    enc.lengths = lengths;
    enc.offsets = offsets;
    enc.kv_heads = heads;
    enc.keys = keys;
    enc.max_keys = max_keys;
    Py_BEGIN_ALLOW_THREADS
    rc = f_cross(cache, scale, &enc, k, v, kv ? ks : NULL, q, o, qv ? qs : NULL, ov ? os : NULL, stream);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(rc);
}

/* bind(append, attend, append_attend, rotary, cross_attend): addresses of the library's functions */
static PyObject* py_bind(PyObject* self, PyObject* const* args, Py_ssize_t n)
{
    void* f[5];
    if (n != 5) {
        PyErr_SetString(PyExc_TypeError, "bind(append, attend, append_attend, rotary, cross_attend)");
        return NULL;
    }
    for (int i = 0; i < 5; ++i) {
        if (as_pointer(args[i], &f[i]) || !f[i]) {
            PyErr_SetString(PyExc_ValueError, "bind() wants addresses");
            return NULL;
        }
    }
    f_attend = (attend_fn)f[1];
    f_append_attend = (append_attend_fn)f[2];
    f_rotary = (rotary_fn)f[3];
    f_cross = (cross_fn)f[4];
    f_append = (append_fn)f[0];
    Py_RETURN_NONE;
}

static PyMethodDef methods[] = {
    {"bind", (PyCFunction)(void (*)(void))py_bind, METH_FASTCALL, NULL},
    {"append", (PyCFunction)(void (*)(void))py_append, METH_FASTCALL, NULL},
    {"attend", (PyCFunction)(void (*)(void))py_attend, METH_FASTCALL, NULL},
    {"append_attend", (PyCFunction)(void (*)(void))py_append_attend, METH_FASTCALL, NULL},
    {"rotary", (PyCFunction)(void (*)(void))py_rotary, METH_FASTCALL, NULL},
    {"cross_attend", (PyCFunction)(void (*)(void))py_cross_attend, METH_FASTCALL, NULL},
    {NULL, NULL, 0, NULL}};
static struct PyModuleDef module = {PyModuleDef_HEAD_INIT, "_steps", NULL, -1, methods, NULL, NULL, NULL, NULL};

PyMODINIT_FUNC PyInit__steps(void)
{
    s_data_ptr = PyUnicode_InternFromString("data_ptr");
    s_is_contiguous = PyUnicode_InternFromString("is_contiguous");
    s_stride = PyUnicode_InternFromString("stride");
    s_cuda_stream = PyUnicode_InternFromString("cuda_stream");
    s_dtype = PyUnicode_InternFromString("dtype");
    s_numel = PyUnicode_InternFromString("numel");
    s_shape = PyUnicode_InternFromString("shape");
    s_torch = PyUnicode_InternFromString("torch");
    if (!s_data_ptr || !s_is_contiguous || !s_stride || !s_cuda_stream || !s_dtype || !s_numel || !s_shape || !s_torch) return NULL;
    return PyModule_Create(&module);
}
