/* The calls that a training loop makes once per step or per layer, for Python: the arguments of zi_grad_norm, zi_grad_norm_noalloc,
 * zi_adamw_step and the operators of zi_fp8.h and zi_epilogue.h are taken out of their objects here.  On a short tensor such a call is bound by the host, and ctypes
 * spends on its arguments what the library spends on the launch: norm and step on 1003 elements 9.5 us through ctypes, 7.0
 * without any binding.
 *
 * Only the usual forms are taken: a list made by make_tensors (or any ctypes array of zi_tensor with its length), a
 * zi_adamw_config, numbers that are Python's own int and float, addresses as int, None or an object with data_ptr(), a
 * stream as int, None or an object with cuda_stream.  For anything else, and for whatever raises on the way, a function
 * here returns None and the caller goes the general way, which accepts and refuses as it always has.  The GIL is released
 * during the call as ctypes does it. */
#define PY_SSIZE_T_CLEAN
#include <Python.h>
#include <stdint.h>

#include "zi.h"
#include "zi_epilogue.h"
#include "zi_fp8.h"

static zi_status (*grad_norm)(const zi_tensor*, int32_t, zi_lp_dtype, float, zi_norm_result*, void*, size_t, void*);
static zi_status (*grad_norm_noalloc)(const zi_tensor*, int32_t, zi_lp_dtype, float, zi_norm_result*, void*);
static zi_status (*adamw_step)(const zi_tensor*, int32_t, zi_lp_dtype, const zi_adamw_config*, const zi_norm_result*, void*);
typedef zi_status quantize_type(const void*, int32_t, int64_t, int64_t, int64_t, const zi_fp8_matrix*, const zi_fp8_matrix*, void*);
typedef zi_status matmul_type(const zi_fp8_matrix*, const zi_fp8_matrix*, void*, int32_t, int64_t, const void*, void*, size_t, void*);
typedef zi_status rms_norm_type(const zi_rms_norm_args*, const zi_fp8_matrix*, void*);
typedef zi_status rms_norm_backward_type(const zi_rms_norm_backward_args*, void*, size_t, void*);
static quantize_type* quantize;
static matmul_type* matmul;
static rms_norm_type* rms_norm;
static rms_norm_backward_type* rms_norm_backward;
typedef zi_status epilogue_type(const void*, int64_t, int64_t, int64_t, const zi_epilogue_args*, const zi_fp8_matrix*, const zi_fp8_matrix*, void*);
typedef zi_status matmul_epilogue_type(const zi_fp8_matrix*, const zi_fp8_matrix*, const zi_epilogue_args*, const zi_fp8_matrix*, const zi_fp8_matrix*, void*, size_t, void*);
typedef zi_status epilogue_backward_type(const zi_epilogue_backward_args*, const zi_fp8_matrix*, const zi_fp8_matrix*, void*, size_t, void*);
static epilogue_type* epilogue;
static matmul_epilogue_type* matmul_epilogue;
static epilogue_backward_type* epilogue_backward;
static PyObject *s_data_ptr, *s_cuda_stream, *s_numel, *s_element_size;
/* how ctypes describes the structures */
static char tensor_format[256], config_format[256], matrix_format[256], norm_format[512], backward_format[512], epilogue_format[512], epilogue_backward_format[512],
    epilogue_matrix_format[256];

/* 1 and the value, or 0 without an error set. */
static int as_int(PyObject* x, long long lo, long long hi, long long* out)
{
    int over = 0;
    if (!PyLong_CheckExact(x)) return 0;
    *out = PyLong_AsLongLongAndOverflow(x, &over);
    return !over && *out >= lo && *out <= hi;
}
static int as_float(PyObject* x, float* out)
{
    if (!PyFloat_CheckExact(x)) return 0;
    *out = (float)PyFloat_AS_DOUBLE(x);
    return 1;
}
static int as_pointer(PyObject* x, PyObject* method, PyObject* attribute, void** out)
{
    if (x == Py_None) {
        *out = NULL;
        return 1;
    }
    if (PyLong_CheckExact(x)) {
        Py_INCREF(x);
    } else {
        x = method ? PyObject_CallMethodNoArgs(x, method) : PyObject_GetAttr(x, attribute);
        if (!x) goto no;
        if (!PyLong_CheckExact(x)) goto drop;
    }
    *out = (void*)PyLong_AsUnsignedLongLong(x);
    if (PyErr_Occurred()) goto drop;
    Py_DECREF(x);
    return 1;
drop:
    Py_DECREF(x);
no:
    PyErr_Clear();
    return 0;
}
static int view_of(PyObject* x, const char* format, Py_buffer* view)
{
    if (PyObject_GetBuffer(x, view, PyBUF_FORMAT | PyBUF_ND | PyBUF_WRITABLE) != 0) {
        PyErr_Clear();
        return 0;
    }
    if (view->format && strcmp(view->format, format) == 0) return 1;
    PyBuffer_Release(view);
    return 0;
}
/* The pair (array, length) of make_tensors. */
static int tensors_of(PyObject* x, Py_buffer* view, long long* n)
{
    if (!PyTuple_CheckExact(x) || PyTuple_GET_SIZE(x) != 2) return 0;
    if (!as_int(PyTuple_GET_ITEM(x, 1), INT32_MIN, INT32_MAX, n)) return 0;
    if (!view_of(PyTuple_GET_ITEM(x, 0), tensor_format, view)) return 0;
    if (view->ndim == 1) return 1;
    PyBuffer_Release(view);
    return 0;
}

static PyObject* call_grad_norm(PyObject* self, PyObject* const* a, Py_ssize_t n_args)
{
    long long n, dt, bytes;
    float scale;
    void *out, *ws, *stream;
    Py_buffer list;
    zi_status st;
    if (n_args != 7 || !as_int(a[1], INT32_MIN, INT32_MAX, &dt) || !as_float(a[2], &scale) || !as_pointer(a[3], s_data_ptr, NULL, &out) ||
        !as_pointer(a[4], s_data_ptr, NULL, &ws) || !as_pointer(a[6], NULL, s_cuda_stream, &stream))
        Py_RETURN_NONE;
    if (a[5] == Py_None) {
        PyObject* count = PyObject_CallMethodNoArgs(a[4], s_numel);
        PyObject* size = count ? PyObject_CallMethodNoArgs(a[4], s_element_size) : NULL;
        long long c = 0, s = 0;
        const int ok = count && size && as_int(count, 0, (long long)1 << 40, &c) && as_int(size, 1, 64, &s);
        Py_XDECREF(count);
        Py_XDECREF(size);
        PyErr_Clear();
        if (!ok) Py_RETURN_NONE;
        bytes = c * s;
    } else if (!as_int(a[5], 0, INT64_MAX, &bytes)) {
        Py_RETURN_NONE;
    }
    if (!tensors_of(a[0], &list, &n)) Py_RETURN_NONE;
    Py_BEGIN_ALLOW_THREADS
    st = grad_norm((const zi_tensor*)list.buf, (int32_t)n, (zi_lp_dtype)dt, scale, (zi_norm_result*)out, ws, (size_t)bytes, stream);
    Py_END_ALLOW_THREADS
    PyBuffer_Release(&list);
    return PyLong_FromLong((long)st);
}

static PyObject* call_grad_norm_noalloc(PyObject* self, PyObject* const* a, Py_ssize_t n_args)
{
    long long n, dt;
    float scale;
    void *out, *stream;
    Py_buffer list;
    zi_status st;
    if (n_args != 5 || !as_int(a[1], INT32_MIN, INT32_MAX, &dt) || !as_float(a[2], &scale) || !as_pointer(a[3], s_data_ptr, NULL, &out) ||
        !as_pointer(a[4], NULL, s_cuda_stream, &stream) || !tensors_of(a[0], &list, &n))
        Py_RETURN_NONE;
    Py_BEGIN_ALLOW_THREADS
    st = grad_norm_noalloc((const zi_tensor*)list.buf, (int32_t)n, (zi_lp_dtype)dt, scale, (zi_norm_result*)out, stream);
    Py_END_ALLOW_THREADS
    PyBuffer_Release(&list);
    return PyLong_FromLong((long)st);
}

static PyObject* call_adamw_step(PyObject* self, PyObject* const* a, Py_ssize_t n_args)
{
    long long n, dt;
    void *norm, *stream;
    Py_buffer list, cfg;
    zi_status st;
    if (n_args != 5 || !as_int(a[1], INT32_MIN, INT32_MAX, &dt) || !as_pointer(a[3], s_data_ptr, NULL, &norm) ||
        !as_pointer(a[4], NULL, s_cuda_stream, &stream) || !view_of(a[2], config_format, &cfg))
        Py_RETURN_NONE;
    if (cfg.ndim != 0 || !tensors_of(a[0], &list, &n)) {
        PyBuffer_Release(&cfg);
        Py_RETURN_NONE;
    }
    Py_BEGIN_ALLOW_THREADS
    st = adamw_step((const zi_tensor*)list.buf, (int32_t)n, (zi_lp_dtype)dt, (const zi_adamw_config*)cfg.buf, (const zi_norm_result*)norm, stream);
    Py_END_ALLOW_THREADS
    PyBuffer_Release(&list);
    PyBuffer_Release(&cfg);
    return PyLong_FromLong((long)st);
}

/* A structure or None: 1 with view->buf set, or NULL. */
static int struct_of(PyObject* x, const char* format, Py_buffer* view)
{
    view->obj = NULL;
    view->buf = NULL;
    if (x == Py_None) return 1;
    if (!view_of(x, format, view)) return 0;
    if (view->ndim == 0) return 1;
    PyBuffer_Release(view);
    return 0;
}
/* Bytes of a buffer, as given or as it says (none: 0). */
static int bytes_of(PyObject* buffer, PyObject* given, long long* out)
{
    *out = 0;
    if (given != Py_None) return as_int(given, 0, INT64_MAX, out);
    if (buffer == Py_None) return 1;
    PyObject* count = PyObject_CallMethodNoArgs(buffer, s_numel);
    PyObject* size = count ? PyObject_CallMethodNoArgs(buffer, s_element_size) : NULL;
    long long c = 0, s = 0;
    const int ok = count && size && as_int(count, 0, (long long)1 << 40, &c) && as_int(size, 1, 64, &s);
    Py_XDECREF(count);
    Py_XDECREF(size);
    PyErr_Clear();
    *out = c * s;
    return ok;
}

/* x, dtype, rows, cols, ld, out, turned, stream */
static PyObject* call_fp8_quantize(PyObject* self, PyObject* const* a, Py_ssize_t n_args)
{
    long long dt, rows, cols, ld;
    void *x, *stream;
    Py_buffer out, turned;
    zi_status st;
    if (n_args != 8 || !as_pointer(a[0], s_data_ptr, NULL, &x) || !as_int(a[1], INT32_MIN, INT32_MAX, &dt) || !as_int(a[2], INT64_MIN, INT64_MAX, &rows) ||
        !as_int(a[3], INT64_MIN, INT64_MAX, &cols) || !as_int(a[4], INT64_MIN, INT64_MAX, &ld) || !as_pointer(a[7], NULL, s_cuda_stream, &stream) ||
        !struct_of(a[5], matrix_format, &out))
        Py_RETURN_NONE;
    if (!struct_of(a[6], matrix_format, &turned)) {
        PyBuffer_Release(&out);
        Py_RETURN_NONE;
    }
    Py_BEGIN_ALLOW_THREADS
    st = quantize(x, (int32_t)dt, rows, cols, ld, (const zi_fp8_matrix*)out.buf, (const zi_fp8_matrix*)turned.buf, stream);
    Py_END_ALLOW_THREADS
    PyBuffer_Release(&out);
    PyBuffer_Release(&turned);
    return PyLong_FromLong((long)st);
}

/* a, b, d, dtype, ldd, c, workspace, its bytes, stream */
static PyObject* call_fp8_matmul(PyObject* self, PyObject* const* a, Py_ssize_t n_args)
{
    long long dt, ldd, bytes;
    void *d, *c, *ws, *stream;
    Py_buffer x, y;
    zi_status st;
    if (n_args != 9 || !as_pointer(a[2], s_data_ptr, NULL, &d) || !as_int(a[3], INT32_MIN, INT32_MAX, &dt) || !as_int(a[4], INT64_MIN, INT64_MAX, &ldd) ||
        !as_pointer(a[5], s_data_ptr, NULL, &c) || !as_pointer(a[6], s_data_ptr, NULL, &ws) || !bytes_of(a[6], a[7], &bytes) ||
        !as_pointer(a[8], NULL, s_cuda_stream, &stream) || !struct_of(a[0], matrix_format, &x))
        Py_RETURN_NONE;
    if (!struct_of(a[1], matrix_format, &y)) {
        PyBuffer_Release(&x);
        Py_RETURN_NONE;
    }
    Py_BEGIN_ALLOW_THREADS
    st = matmul((const zi_fp8_matrix*)x.buf, (const zi_fp8_matrix*)y.buf, d, (int32_t)dt, ldd, c, ws, (size_t)bytes, stream);
    Py_END_ALLOW_THREADS
    PyBuffer_Release(&x);
    PyBuffer_Release(&y);
    return PyLong_FromLong((long)st);
}

/* args, y8, stream */
static PyObject* call_rms_norm(PyObject* self, PyObject* const* a, Py_ssize_t n_args)
{
    void* stream;
    Py_buffer args, y8;
    zi_status st;
    if (n_args != 3 || !as_pointer(a[2], NULL, s_cuda_stream, &stream) || !struct_of(a[0], norm_format, &args)) Py_RETURN_NONE;
    if (!struct_of(a[1], matrix_format, &y8)) {
        PyBuffer_Release(&args);
        Py_RETURN_NONE;
    }
    Py_BEGIN_ALLOW_THREADS
    st = rms_norm((const zi_rms_norm_args*)args.buf, (const zi_fp8_matrix*)y8.buf, stream);
    Py_END_ALLOW_THREADS
    PyBuffer_Release(&args);
    PyBuffer_Release(&y8);
    return PyLong_FromLong((long)st);
}

/* args, workspace, its bytes, stream */
static PyObject* call_rms_norm_backward(PyObject* self, PyObject* const* a, Py_ssize_t n_args)
{
    long long bytes;
    void *ws, *stream;
    Py_buffer args;
    zi_status st;
    if (n_args != 4 || !as_pointer(a[1], s_data_ptr, NULL, &ws) || !bytes_of(a[1], a[2], &bytes) || !as_pointer(a[3], NULL, s_cuda_stream, &stream) ||
        !struct_of(a[0], backward_format, &args))
        Py_RETURN_NONE;
    Py_BEGIN_ALLOW_THREADS
    st = rms_norm_backward((const zi_rms_norm_backward_args*)args.buf, ws, (size_t)bytes, stream);
    Py_END_ALLOW_THREADS
    PyBuffer_Release(&args);
    return PyLong_FromLong((long)st);
}

/* bind_fp8(addresses of zi_fp8_quantize, zi_fp8_matmul, zi_rms_norm, zi_rms_norm_backward, a zi_fp8_matrix, a zi_rms_norm_args, a
 * zi_rms_norm_backward_args): as bind. */
static PyObject* bind_fp8(PyObject* self, PyObject* const* a, Py_ssize_t n_args)
{
    void* f[4];
    Py_buffer view;
    char* const formats[3] = {matrix_format, norm_format, backward_format};
    const size_t room[3] = {sizeof matrix_format, sizeof norm_format, sizeof backward_format};
    const Py_ssize_t sizes[3] = {(Py_ssize_t)sizeof(zi_fp8_matrix), (Py_ssize_t)sizeof(zi_rms_norm_args), (Py_ssize_t)sizeof(zi_rms_norm_backward_args)};
    int ok = n_args == 7;
    for (int i = 0; ok && i < 4; ++i) ok = as_pointer(a[i], s_data_ptr, NULL, &f[i]) && f[i];
    for (int i = 0; ok && i < 3; ++i) {
        if (PyObject_GetBuffer(a[4 + i], &view, PyBUF_FORMAT | PyBUF_ND) != 0) return NULL;
        ok = view.itemsize == sizes[i] && view.format && strlen(view.format) < room[i];
        if (ok) strcpy(formats[i], view.format);
        PyBuffer_Release(&view);
    }
    if (!ok) Py_RETURN_FALSE;
    quantize = (quantize_type*)f[0];
    matmul = (matmul_type*)f[1];
    rms_norm = (rms_norm_type*)f[2];
    rms_norm_backward = (rms_norm_backward_type*)f[3];
    Py_RETURN_TRUE;
}

/* Structures or None, as struct_of takes each of them: all or none. */
static int structs_of(PyObject* const* x, const char* const* format, Py_buffer* view, int count)
{
    for (int i = 0; i < count; ++i) {
        if (struct_of(x[i], format[i], &view[i])) continue;
        while (i-- > 0) PyBuffer_Release(&view[i]);
        return 0;
    }
    return 1;
}
static void release(Py_buffer* view, int count)
{
    for (int i = 0; i < count; ++i) PyBuffer_Release(&view[i]);
}

/* x, rows, cols, ld, args, y8, turned, stream */
static PyObject* call_epilogue(PyObject* self, PyObject* const* a, Py_ssize_t n_args)
{
    const char* const formats[3] = {epilogue_format, epilogue_matrix_format, epilogue_matrix_format};
    long long rows, cols, ld;
    void *x, *stream;
    Py_buffer v[3];
    zi_status st;
    if (n_args != 8 || !as_pointer(a[0], s_data_ptr, NULL, &x) || !as_int(a[1], INT64_MIN, INT64_MAX, &rows) || !as_int(a[2], INT64_MIN, INT64_MAX, &cols) ||
        !as_int(a[3], INT64_MIN, INT64_MAX, &ld) || !as_pointer(a[7], NULL, s_cuda_stream, &stream) || !structs_of(a + 4, formats, v, 3))
        Py_RETURN_NONE;
    Py_BEGIN_ALLOW_THREADS
    st = epilogue(x, rows, cols, ld, (const zi_epilogue_args*)v[0].buf, (const zi_fp8_matrix*)v[1].buf, (const zi_fp8_matrix*)v[2].buf, stream);
    Py_END_ALLOW_THREADS
    release(v, 3);
    return PyLong_FromLong((long)st);
}

/* a, b, args, y8, turned, workspace, its bytes, stream */
static PyObject* call_matmul_epilogue(PyObject* self, PyObject* const* a, Py_ssize_t n_args)
{
    const char* const formats[5] = {epilogue_matrix_format, epilogue_matrix_format, epilogue_format, epilogue_matrix_format, epilogue_matrix_format};
    long long bytes;
    void *ws, *stream;
    Py_buffer v[5];
    zi_status st;
    if (n_args != 8 || !as_pointer(a[5], s_data_ptr, NULL, &ws) || !bytes_of(a[5], a[6], &bytes) || !as_pointer(a[7], NULL, s_cuda_stream, &stream) ||
        !structs_of(a, formats, v, 5))
        Py_RETURN_NONE;
    Py_BEGIN_ALLOW_THREADS
    st = matmul_epilogue((const zi_fp8_matrix*)v[0].buf, (const zi_fp8_matrix*)v[1].buf, (const zi_epilogue_args*)v[2].buf, (const zi_fp8_matrix*)v[3].buf,
                         (const zi_fp8_matrix*)v[4].buf, ws, (size_t)bytes, stream);
    Py_END_ALLOW_THREADS
    release(v, 5);
    return PyLong_FromLong((long)st);
}

/* args, dz8, turned, workspace, its bytes, stream */
static PyObject* call_epilogue_backward(PyObject* self, PyObject* const* a, Py_ssize_t n_args)
{
    const char* const formats[3] = {epilogue_backward_format, epilogue_matrix_format, epilogue_matrix_format};
    long long bytes;
    void *ws, *stream;
    Py_buffer v[3];
    zi_status st;
    if (n_args != 6 || !as_pointer(a[3], s_data_ptr, NULL, &ws) || !bytes_of(a[3], a[4], &bytes) || !as_pointer(a[5], NULL, s_cuda_stream, &stream) ||
        !structs_of(a, formats, v, 3))
        Py_RETURN_NONE;
    Py_BEGIN_ALLOW_THREADS
    st = epilogue_backward((const zi_epilogue_backward_args*)v[0].buf, (const zi_fp8_matrix*)v[1].buf, (const zi_fp8_matrix*)v[2].buf, ws, (size_t)bytes, stream);
    Py_END_ALLOW_THREADS
    release(v, 3);
    return PyLong_FromLong((long)st);
}

/* bind_epilogue(addresses of zi_epilogue, zi_fp8_matmul_epilogue, zi_epilogue_backward, a zi_fp8_matrix, a zi_epilogue_args, a zi_epilogue_backward_args): as
 * bind. */
static PyObject* bind_epilogue(PyObject* self, PyObject* const* a, Py_ssize_t n_args)
{
    void* f[3];
    Py_buffer view;
    char* const formats[3] = {epilogue_matrix_format, epilogue_format, epilogue_backward_format};
    const size_t room[3] = {sizeof epilogue_matrix_format, sizeof epilogue_format, sizeof epilogue_backward_format};
    const Py_ssize_t sizes[3] = {(Py_ssize_t)sizeof(zi_fp8_matrix), (Py_ssize_t)sizeof(zi_epilogue_args), (Py_ssize_t)sizeof(zi_epilogue_backward_args)};
    int ok = n_args == 6;
    for (int i = 0; ok && i < 3; ++i) ok = as_pointer(a[i], s_data_ptr, NULL, &f[i]) && f[i];
    for (int i = 0; ok && i < 3; ++i) {
        if (PyObject_GetBuffer(a[3 + i], &view, PyBUF_FORMAT | PyBUF_ND) != 0) return NULL;
        ok = view.itemsize == sizes[i] && view.format && strlen(view.format) < room[i];
        if (ok) strcpy(formats[i], view.format);
        PyBuffer_Release(&view);
    }
    if (!ok) Py_RETURN_FALSE;
    epilogue = (epilogue_type*)f[0];
    matmul_epilogue = (matmul_epilogue_type*)f[1];
    epilogue_backward = (epilogue_backward_type*)f[2];
    Py_RETURN_TRUE;
}

/* bind(address of zi_grad_norm, of zi_grad_norm_noalloc, of zi_adamw_step, a zi_tensor, a zi_adamw_config): True if these
 * are the structures that this module was compiled with. */
static PyObject* bind(PyObject* self, PyObject* const* a, Py_ssize_t n_args)
{
    void* f[3];
    Py_buffer view;
    char* const formats[2] = {tensor_format, config_format};
    const Py_ssize_t sizes[2] = {(Py_ssize_t)sizeof(zi_tensor), (Py_ssize_t)sizeof(zi_adamw_config)};
    int ok = n_args == 5;
    for (int i = 0; ok && i < 3; ++i) ok = as_pointer(a[i], s_data_ptr, NULL, &f[i]) && f[i];
    for (int i = 0; ok && i < 2; ++i) {
        if (PyObject_GetBuffer(a[3 + i], &view, PyBUF_FORMAT | PyBUF_ND) != 0) return NULL;
        ok = view.itemsize == sizes[i] && view.format && strlen(view.format) < sizeof tensor_format;
        if (ok) strcpy(formats[i], view.format);
        PyBuffer_Release(&view);
    }
    if (!ok) Py_RETURN_FALSE;
    grad_norm = (zi_status(*)(const zi_tensor*, int32_t, zi_lp_dtype, float, zi_norm_result*, void*, size_t, void*))f[0];
    grad_norm_noalloc = (zi_status(*)(const zi_tensor*, int32_t, zi_lp_dtype, float, zi_norm_result*, void*))f[1];
    adamw_step = (zi_status(*)(const zi_tensor*, int32_t, zi_lp_dtype, const zi_adamw_config*, const zi_norm_result*, void*))f[2];
    Py_RETURN_TRUE;
}

static PyMethodDef methods[] = {
    {"bind", (PyCFunction)(void (*)(void))bind, METH_FASTCALL, NULL},
    {"grad_norm", (PyCFunction)(void (*)(void))call_grad_norm, METH_FASTCALL, NULL},
    {"grad_norm_noalloc", (PyCFunction)(void (*)(void))call_grad_norm_noalloc, METH_FASTCALL, NULL},
    {"adamw_step", (PyCFunction)(void (*)(void))call_adamw_step, METH_FASTCALL, NULL},
    {"bind_fp8", (PyCFunction)(void (*)(void))bind_fp8, METH_FASTCALL, NULL},
    {"fp8_quantize", (PyCFunction)(void (*)(void))call_fp8_quantize, METH_FASTCALL, NULL},
    {"fp8_matmul", (PyCFunction)(void (*)(void))call_fp8_matmul, METH_FASTCALL, NULL},
    {"rms_norm", (PyCFunction)(void (*)(void))call_rms_norm, METH_FASTCALL, NULL},
    {"rms_norm_backward", (PyCFunction)(void (*)(void))call_rms_norm_backward, METH_FASTCALL, NULL},
    {"bind_epilogue", (PyCFunction)(void (*)(void))bind_epilogue, METH_FASTCALL, NULL},
    {"epilogue", (PyCFunction)(void (*)(void))call_epilogue, METH_FASTCALL, NULL},
    {"matmul_epilogue", (PyCFunction)(void (*)(void))call_matmul_epilogue, METH_FASTCALL, NULL},
    {"epilogue_backward", (PyCFunction)(void (*)(void))call_epilogue_backward, METH_FASTCALL, NULL},
    {NULL, NULL, 0, NULL}};
static struct PyModuleDef module = {PyModuleDef_HEAD_INIT, "_zi_call", NULL, -1, methods, NULL, NULL, NULL, NULL};

PyMODINIT_FUNC PyInit__zi_call(void)
{
    s_data_ptr = PyUnicode_InternFromString("data_ptr");
    s_cuda_stream = PyUnicode_InternFromString("cuda_stream");
    s_numel = PyUnicode_InternFromString("numel");
    s_element_size = PyUnicode_InternFromString("element_size");
    if (!s_data_ptr || !s_cuda_stream || !s_numel || !s_element_size) return NULL;
    return PyModule_Create(&module);
}
