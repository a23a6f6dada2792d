/* Argument marshalling of the calls that a program makes once per layer and step, where ctypes is a large part of the
 * call: a cache update + attention of two rows takes the device 7.0 us, and its nineteen arguments cost 7.3 us through
 * ctypes (conversions and temporary pointer objects) against 0.8-2.8 us here (two hosts). Together with attribute
 * lookups that no longer import, the call went from 16.4 us (host-bound) to 8.0 us (device-bound). Plain CPython C API; the library's functions
 * are handed over as addresses at import, so this module links against nothing.
 *
 * Tensors are asked for data_ptr(), shape and nbytes by name: no dependence on torch's headers or layout. */
/* Only the stable ABI (Python 3.10 and later): the module's file name says nothing about the interpreter it was built
 * with, so nothing of that interpreter's object layout may be compiled in. */
#define Py_LIMITED_API 0x030A0000
#define PY_SSIZE_T_CLEAN
#include <Python.h>
#include <stddef.h>
#include <stdint.h>
#include <stdio.h>

#include "../../include/dkv.h"

typedef int (*attn_update_fn)(void *, void *, const void *, const void *, const void *, const int32_t *, const int32_t *, void *,
                              int32_t, int32_t, int32_t, int32_t, int32_t, int32_t, int32_t, int32_t, void *, size_t, void *);
typedef int (*attn_update_static_fn)(void *, void *, const void *, const void *, const void *, const int32_t *, const int32_t *,
                                     void *, int32_t, int32_t, int32_t, int32_t, int32_t, int32_t, int32_t, int32_t, void *);

static attn_update_fn f_attn_update;
static attn_update_static_fn f_attn_update_static;
static PyObject *s_data_ptr, *s_shape, *s_nbytes, *s_value;
static PyObject *c_int_type;      /* ctypes.c_int32 */

/* address of a tensor's first element, NULL for None; -1 with an exception set on failure */
static int get_ptr(PyObject *t, void **p) {
    *p = NULL;
    if (t == Py_None) return 0;
    PyObject *v = PyObject_CallMethodObjArgs(t, s_data_ptr, NULL);
    if (!v) return -1;
    *p = PyLong_AsVoidPtr(v);
    Py_DECREF(v);
    return PyErr_Occurred() ? -1 : 0;
}

/* a whole number of 32 bits, as ctypes takes it for an int32 argument: int, anything with __index__, or a ctypes int; a
 * number that does not fit is an error (it would name other sizes than the caller's) */
static int get_i32(PyObject *o, int32_t *v) {
    PyObject *held = NULL;
    if (!PyLong_Check(o) && c_int_type) {
        const int is_c_int = PyObject_IsInstance(o, c_int_type);
        if (is_c_int < 0) return -1;
        if (is_c_int) {
            if (!(held = PyObject_GetAttr(o, s_value))) return -1;
            o = held;
        }
    }
    const long x = PyLong_AsLong(o);
    Py_XDECREF(held);
    if (x == -1 && PyErr_Occurred()) return -1;
    if (x < INT32_MIN || x > INT32_MAX) {
        PyErr_SetString(PyExc_OverflowError, "argument does not fit 32 bits");
        return -1;
    }
    *v = (int32_t)x;
    return 0;
}

/* up to `max` sizes of a tensor; returns the number of dimensions, -1 with an exception set on failure */
static Py_ssize_t get_shape(PyObject *t, int32_t *dims, Py_ssize_t max) {
    PyObject *s = PyObject_GetAttr(t, s_shape);
    if (!s) return -1;
    if (!PyTuple_Check(s)) {
        PyObject *seq = PySequence_Tuple(s);
        Py_DECREF(s);
        if (!(s = seq)) return -1;
    }
    Py_ssize_t n = PyTuple_Size(s);
    for (Py_ssize_t i = 0; i < n && i < max; ++i)
        if (get_i32(PyTuple_GetItem(s, i), &dims[i])) {
            n = -1;
            break;
        }
    Py_DECREF(s);
    return n;
}

/* (k_cache, v_cache, q, k_new, v_new, active_idx, active_off, out, rows, max_rows_per_seq, dtype, workspace, stream) for
 * `with_workspace`, without `workspace` else: the status code of the library call */
static PyObject *call_attn_update(PyObject *const *a, Py_ssize_t n, int with_workspace) {
    if (n != (with_workspace ? 13 : 12)) {
        PyErr_SetString(PyExc_TypeError, "wrong number of arguments");
        return NULL;
    }
    if (!f_attn_update) {
        PyErr_SetString(PyExc_RuntimeError, "bind() has not been called");
        return NULL;
    }
    void *p[8], *ws = NULL, *stream;
    int32_t c[4], h[4], rows, max_rows, dtype;
    size_t ws_bytes = 0;
    Py_ssize_t d = get_shape(a[0], c, 4);
    if (d < 0) return NULL;
    if (d != 4) {
        PyErr_SetString(PyExc_ValueError, "the cache has four dimensions: batch, kv heads, positions, head_dim");
        return NULL;
    }
    /* query heads: from q, or from the output when there is no q of three dimensions */
    d = a[2] == Py_None ? 0 : get_shape(a[2], h, 4);
    if (d < 0) return NULL;
    if (d != 3) {
        d = get_shape(a[7], h, 4);
        if (d < 0) return NULL;
        if (d < 2) {
            PyErr_SetString(PyExc_IndexError, "out has too few dimensions");
            return NULL;
        }
    }
    for (int i = 0; i < 8; ++i)
        if (get_ptr(a[i], &p[i])) return NULL;
    if (get_i32(a[8], &rows) || get_i32(a[9], &max_rows) || get_i32(a[10], &dtype)) return NULL;
    if (with_workspace && a[11] != Py_None) {
        if (get_ptr(a[11], &ws)) return NULL;
        PyObject *b = PyObject_GetAttr(a[11], s_nbytes);
        if (!b) return NULL;
        ws_bytes = PyLong_AsSize_t(b);
        Py_DECREF(b);
    }
    stream = PyLong_AsVoidPtr(a[n - 1]);
    if (PyErr_Occurred()) return NULL;
    int rc;
    Py_BEGIN_ALLOW_THREADS      /* as ctypes does: other threads may run while a launch is enqueued */
    rc = with_workspace ? f_attn_update(p[0], p[1], p[2], p[3], p[4], p[5], p[6], p[7], rows, max_rows, c[0], h[1], c[1], c[2], c[3],
                                        dtype, ws, ws_bytes, stream)
                        : f_attn_update_static(p[0], p[1], p[2], p[3], p[4], p[5], p[6], p[7], rows, max_rows, c[0], h[1], c[1], c[2],
                                               c[3], dtype, stream);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(rc);
}

static PyObject *py_attn_update(PyObject *self, PyObject *const *a, Py_ssize_t n) { return call_attn_update(a, n, 1); }
static PyObject *py_attn_update_static(PyObject *self, PyObject *const *a, Py_ssize_t n) { return call_attn_update(a, n, 0); }

/* bind(address of dkv_attn_update, address of dkv_attn_update_static, ctypes.c_int32) */
static PyObject *py_bind(PyObject *self, PyObject *const *a, Py_ssize_t n) {
    if (n != 3) {
        PyErr_SetString(PyExc_TypeError, "two addresses and the integer type are expected");
        return NULL;
    }
    void *x = PyLong_AsVoidPtr(a[0]), *y = PyLong_AsVoidPtr(a[1]);
    if (PyErr_Occurred()) return NULL;
    f_attn_update = (attn_update_fn)x;
    f_attn_update_static = (attn_update_static_fn)y;
    PyObject *old = c_int_type;
    Py_INCREF(a[2]);
    c_int_type = a[2];
    Py_XDECREF(old);
    Py_RETURN_NONE;
}

/* ---- the paged cache: the checks of what a kernel would read are made here, with the marshalling (through ctypes and Python
 * a store of 64 rows took 27 us of the host, its kernel 4) ---- */
typedef int (*paged_store_fn)(const dkv_paged_cache *, const void *, const void *, int64_t, const int32_t *, const int32_t *, int32_t,
                              int32_t, void *);
typedef int (*paged_load_fn)(const dkv_paged_cache *, void *, void *, const int32_t *, const int32_t *, int32_t, int32_t, void *);
typedef size_t (*paged_bytes_fn)(const dkv_paged_cache *, int32_t, int32_t, int32_t, int32_t);
typedef int (*paged_attn_fn)(const dkv_paged_cache *, const void *, int64_t, const int32_t *, void *, int32_t, int32_t, int32_t, int32_t,
                             void *, size_t, void *);

static paged_store_fn f_paged_store;
static paged_load_fn f_paged_load;
static paged_bytes_fn f_paged_bytes;
static paged_attn_fn f_paged_attn;
typedef int (*paged_resize_fn)(const dkv_paged_tables *, const int32_t *, int32_t *, int32_t *, int64_t *, int32_t, void *, size_t, void *);
typedef int (*rope_fn)(const dkv_rope_desc *, const void *, int64_t, void *, int64_t, int32_t, const void *, int64_t, void *, int64_t, int32_t,
                       const int32_t *, const int32_t *, int32_t, int32_t, int32_t, int32_t, void *);
static paged_resize_fn f_paged_resize;
static rope_fn f_rope;
enum { T_BF16 = DKV_BF16, T_FP32 = DKV_FP32, T_E4M3 = DKV_E4M3, T_E8M0, T_E2M1 = DKV_E2M1, T_I32, T_I64, T_COUNT };
static PyObject *dtypes[T_COUNT];
static PyObject *s_dtype, *s_is_contiguous, *s_get_device, *s_stride, *s_current, *s_stream;
static PyObject *place_of;        /* has _cuda_getDevice() and _cuda_getCurrentRawStream(device) */

typedef struct {
    void *ptr;
    int32_t dims[4];
    int n_dims, dtype, device, whole;     /* dtype: T_*, or -1; device: -1 on the host */
} tensor_info;

/* where it is, and whether it is contiguous */
static int look_memory(PyObject *t, tensor_info *i) {
    PyObject *v = PyObject_CallMethodObjArgs(t, s_is_contiguous, NULL);
    if (!v) return -1;
    i->whole = (int)PyLong_AsLong(v);      /* a bool is a whole number */
    Py_DECREF(v);
    if (!(v = PyObject_CallMethodObjArgs(t, s_get_device, NULL))) return -1;
    i->device = (int)PyLong_AsLong(v);
    Py_DECREF(v);
    if (PyErr_Occurred()) return -1;
    return get_ptr(t, &i->ptr);
}

static int look(PyObject *t, tensor_info *i) {
    const Py_ssize_t d = get_shape(t, i->dims, 4);
    if (d < 0) return -1;
    i->n_dims = (int)d;
    PyObject *v = PyObject_GetAttr(t, s_dtype);
    if (!v) return -1;
    for (i->dtype = T_COUNT - 1; i->dtype >= 0 && dtypes[i->dtype] != v; --i->dtype);
    Py_DECREF(v);
    return look_memory(t, i);
}

static int refuse(const char *name, const char *text) {
    char all[160];
    snprintf(all, sizeof all, "%s: %s", name, text);
    PyErr_SetString(PyExc_ValueError, all);
    return -1;
}

/* a contiguous tensor of this type and of these sizes (n < 0: any, of -n dimensions), where the cache is */
static int look_whole(PyObject *t, const char *name, int dtype, int n, const int32_t *dims, int device, tensor_info *i) {
    if (look(t, i)) return -1;
    if (i->dtype != dtype || !i->whole) return refuse(name, "a contiguous tensor of the documented type is expected");
    if (i->n_dims != (n < 0 ? -n : n)) return refuse(name, "wrong number of dimensions");
    for (int k = 0; k < n; ++k)
        if (i->dims[k] != dims[k]) return refuse(name, "sizes do not fit those of the cache and the rows");
    return i->device == device ? 0 : refuse(name, "not on the device of the other tensors");
}

/* (k_pages, v_pages, page_table, seq_len, k_scale, v_scale) */
static int look_cache(PyObject *o, dkv_paged_cache *c, int *device) {
    if (!PyTuple_Check(o) || PyTuple_Size(o) != 6) {
        PyErr_SetString(PyExc_TypeError, "a PagedCache is expected");
        return -1;
    }
    PyObject *t[6];
    for (int i = 0; i < 6; ++i) t[i] = PyTuple_GetItem(o, i);
    tensor_info k, v, x;
    if (look(t[0], &k)) return -1;
    if (k.n_dims != 4) return refuse("k_pages", "pages have four dimensions: pages, kv heads, slots, head_dim");
    const int four_bits = k.dtype == T_E2M1;
    if (k.dtype < 0 || (k.dtype > T_E4M3 && !four_bits)) return refuse("k_pages", "pages of this type are not supported");
    if (!k.whole) return refuse("k_pages", "a contiguous tensor is expected");
    if (look_whole(t[1], "v_pages", k.dtype, 4, k.dims, k.device, &v)) return -1;
    if (look_whole(t[2], "page_table", T_I32, -2, NULL, k.device, &x)) return -1;
    if (four_bits && k.dims[3] > INT32_MAX / 2) return refuse("k_pages", "sizes do not fit 32 bits");
    *c = (dkv_paged_cache){k.ptr, v.ptr, NULL, NULL, x.ptr, NULL, x.dims[0], k.dims[0], x.dims[1], k.dims[2], k.dims[1], four_bits ? 2 * k.dims[3] : k.dims[3], k.dtype};
    if (t[3] != Py_None) {
        if (look_whole(t[3], "seq_len", T_I32, 1, &c->batch, k.device, &x)) return -1;
        c->seq_len = x.ptr;
    }
    if (k.dtype != T_E4M3 && !four_bits) {
        if (t[4] != Py_None || t[5] != Py_None) return refuse("k_scale, v_scale", "scales go with pages of float8_e4m3fn and float4_e2m1fn_x2 only");
    } else {
        if (t[4] == Py_None || t[5] == Py_None) return refuse("k_scale, v_scale", "pages of float8_e4m3fn and float4_e2m1fn_x2 need k_scale and v_scale");
        const int32_t dims[4] = {k.dims[0], k.dims[1], k.dims[2], k.dims[3] / 16};      /* e2m1: one for each 32 dims */
        if (look_whole(t[4], "k_scale", T_E8M0, four_bits ? 4 : 3, dims, k.device, &x)) return -1;
        c->k_scale = x.ptr;
        if (look_whole(t[5], "v_scale", T_E8M0, four_bits ? 4 : 3, dims, k.device, &x)) return -1;
        c->v_scale = x.ptr;
    }
    *device = k.device;
    return 0;
}

/* [rows, heads, head_dim] of bfloat16 or float32 (heads < 0: any number of them), rows `*stride` elements apart */
static int look_rows(PyObject *t, const char *name, int32_t heads, int32_t head_dim, int device, tensor_info *i, int64_t *stride) {
    if (look(t, i)) return -1;
    if (i->n_dims != 3 || (heads >= 0 && i->dims[1] != heads) || i->dims[2] != head_dim || (i->dtype != T_BF16 && i->dtype != T_FP32))
        return refuse(name, "[rows, heads, head_dim] of bfloat16 or float32 with the head_dim at hand is expected");
    if (i->device != device) return refuse(name, "not on the device of the other tensors");
    *stride = (int64_t)i->dims[1] * head_dim;
    if (i->whole) return 0;
    PyObject *s = PyObject_CallMethodObjArgs(t, s_stride, NULL);
    if (!s) return -1;
    long n[3];
    for (int k = 0; k < 3; ++k) n[k] = PyLong_AsLong(PyTuple_GetItem(s, k));
    Py_DECREF(s);
    if (PyErr_Occurred()) return -1;
    if (n[2] != 1 || (i->dims[1] > 1 && n[1] != head_dim) || (i->dims[0] > 1 && n[0] < *stride))
        return refuse(name, "rows of heads one behind the other are expected");
    if (i->dims[0] > 1) *stride = n[0];
    return 0;
}

/* None: one row per sequence */
static int look_offsets(PyObject *t, int32_t batch, int32_t rows, int device, const int32_t **p) {
    *p = NULL;
    if (t == Py_None) return rows == batch ? 0 : refuse("row_off", "without row offsets there is one row per sequence");
    tensor_info x;
    const int32_t n = batch + 1;
    if (look_whole(t, "row_off", T_I32, 1, &n, device, &x)) return -1;
    *p = x.ptr;
    return 0;
}

/* the current stream of the tensors' device, which has to be the current one: asked of torch only where there is a GPU */
static int look_place(const char *name, int device, void **s) {
    if (device < 0) return refuse(name, "not on a GPU");
    PyObject *at = PyObject_CallMethodObjArgs(place_of, s_current, NULL);
    if (!at) return -1;
    const long current = PyLong_AsLong(at);
    if (current == device) {
        PyObject *stream = PyObject_CallMethodObjArgs(place_of, s_stream, at, NULL);
        if (stream) *s = PyLong_AsVoidPtr(stream);
        Py_XDECREF(stream);
    }
    Py_DECREF(at);
    if (PyErr_Occurred()) return -1;
    return current == device ? 0 : refuse(name, "not on the current device");
}

static int ready(Py_ssize_t n, Py_ssize_t want) {
    if (n != want) PyErr_SetString(PyExc_TypeError, "wrong number of arguments");
    else if (!f_paged_store) PyErr_SetString(PyExc_RuntimeError, "bind_paged() has not been called");
    else return 1;
    return 0;
}

/* (cache, k, v, positions, row_off): the status code of the library call */
static PyObject *rows_call(PyObject *const *a, Py_ssize_t n, int storing) {
    if (!ready(n, 5)) return NULL;
    dkv_paged_cache c;
    tensor_info k, v, pos;
    int64_t stride, v_stride;
    const int32_t *off;
    void *stream;
    int device;
    const char *kn = storing ? "k_new" : "k_out", *vn = storing ? "v_new" : "v_out";
    if (look_cache(a[0], &c, &device) || look_rows(a[1], kn, c.n_kv_heads, c.head_dim, device, &k, &stride) ||
        look_rows(a[2], vn, c.n_kv_heads, c.head_dim, device, &v, &v_stride))
        return NULL;
    if (v.dtype != k.dtype || v.dims[0] != k.dims[0] || v_stride != stride) {
        refuse(vn, "same shape, type and distance between rows as of the keys is expected");
        return NULL;
    }
    if (!storing && !(k.whole && v.whole)) {
        refuse(kn, "contiguous results are expected");
        return NULL;
    }
    if (look_whole(a[3], "positions", T_I32, 1, &k.dims[0], device, &pos) || look_offsets(a[4], c.batch, k.dims[0], device, &off) ||
        look_place("k_pages", device, &stream))
        return NULL;
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = storing ? f_paged_store(&c, k.ptr, v.ptr, stride, pos.ptr, off, k.dims[0], k.dtype, stream)
                 : f_paged_load(&c, k.ptr, v.ptr, pos.ptr, off, k.dims[0], k.dtype, stream);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(rc);
}

static PyObject *py_paged_store(PyObject *self, PyObject *const *a, Py_ssize_t n) { return rows_call(a, n, 1); }
static PyObject *py_paged_load(PyObject *self, PyObject *const *a, Py_ssize_t n) { return rows_call(a, n, 0); }

/* (cache, n_q_heads, rows, max_rows_per_seq, dtype): bytes */
static PyObject *py_paged_attn_workspace_bytes(PyObject *self, PyObject *const *a, Py_ssize_t n) {
    if (!ready(n, 5)) return NULL;
    dkv_paged_cache c;
    int device;
    int32_t x[4];
    if (look_cache(a[0], &c, &device)) return NULL;
    for (int i = 0; i < 4; ++i)
        if (get_i32(a[1 + i], &x[i])) return NULL;
    return PyLong_FromLong((long)f_paged_bytes(&c, x[0], x[1], x[2], x[3]));
}

/* None, or memory of any type and shape: its sizes may pass 32 bits */
static int look_workspace(PyObject *t, int device, tensor_info *ws, size_t *bytes) {
    if (t == Py_None) return 0;
    if (look_memory(t, ws)) return -1;
    if (!ws->whole || ws->device != device) return refuse("workspace", "a contiguous tensor on the device of the others is expected");
    PyObject *b = PyObject_GetAttr(t, s_nbytes);
    if (!b) return -1;
    *bytes = PyLong_AsSize_t(b);
    Py_DECREF(b);
    return PyErr_Occurred() ? -1 : 0;
}

/* (cache, q, row_off, out, max_rows_per_seq, workspace): the status code of the library call */
static PyObject *py_paged_attn(PyObject *self, PyObject *const *a, Py_ssize_t n) {
    if (!ready(n, 6)) return NULL;
    dkv_paged_cache c;
    tensor_info q, out, ws = {0};
    int64_t stride;
    const int32_t *off;
    void *stream;
    int device;
    int32_t most;
    size_t bytes = 0;
    if (look_cache(a[0], &c, &device)) return NULL;
    if (!c.seq_len) {
        refuse("seq_len", "attention needs the lengths");
        return NULL;
    }
    if (look_rows(a[1], "q", -1, c.head_dim, device, &q, &stride) || look_offsets(a[2], c.batch, q.dims[0], device, &off) ||
        look_whole(a[3], "out", q.dtype, 3, q.dims, device, &out) || get_i32(a[4], &most))
        return NULL;
    if (look_workspace(a[5], device, &ws, &bytes)) return NULL;
    if (look_place("k_pages", device, &stream)) return NULL;
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = f_paged_attn(&c, q.ptr, stride, off, out.ptr, q.dims[0], most, q.dims[1], q.dtype, ws.ptr, bytes, stream);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(rc);
}

/* ((page_table, seq_len, free_pages, free_at, page_size), lengths, workspace, row_off, positions, slots): the status code of the library call */
static PyObject *py_paged_resize(PyObject *self, PyObject *const *a, Py_ssize_t n) {
    if (!ready(n, 6)) return NULL;
    if (!PyTuple_Check(a[0]) || PyTuple_Size(a[0]) != 5) {
        PyErr_SetString(PyExc_TypeError, "PagedTables are expected");
        return NULL;
    }
    PyObject *t[5];
    for (int i = 0; i < 5; ++i) t[i] = PyTuple_GetItem(a[0], i);
    tensor_info table, len, ring, at, x, off = {0}, pos = {0}, slots = {0}, ws = {0};
    int32_t page_size;
    size_t bytes = 0;
    void *stream;
    if (look(t[0], &table)) return NULL;
    if (table.dtype != T_I32 || table.n_dims != 2 || !table.whole) {
        refuse("page_table", "a contiguous int32 tensor [batch, max_pages] is expected");
        return NULL;
    }
    const int device = table.device;
    const int32_t batch = table.dims[0], two = 2, many = batch < INT32_MAX ? batch + 1 : batch;
    if (look_whole(t[1], "seq_len", T_I32, 1, &batch, device, &len) || look_whole(t[2], "free_pages", T_I32, -1, NULL, device, &ring) ||
        look_whole(t[3], "free_at", T_I32, 1, &two, device, &at) || get_i32(t[4], &page_size) ||
        look_whole(a[1], "lengths", T_I32, 1, &batch, device, &x) || look_workspace(a[2], device, &ws, &bytes))
        return NULL;
    int32_t rows = 0;
    if (a[3] != Py_None && look_whole(a[3], "row_off", T_I32, 1, &many, device, &off)) return NULL;
    if (a[4] != Py_None) {
        if (look_whole(a[4], "positions", T_I32, -1, NULL, device, &pos)) return NULL;
        rows = pos.dims[0];
    }
    if (a[5] != Py_None) {
        if (look_whole(a[5], "slots", T_I64, -1, NULL, device, &slots)) return NULL;
        if (a[4] != Py_None && slots.dims[0] != rows) {
            refuse("slots", "as many as positions are expected");
            return NULL;
        }
        rows = slots.dims[0];
    }
    if (a[3] != Py_None && a[4] == Py_None && a[5] == Py_None) {
        refuse("row_off", "positions or slots say how many rows there may be");
        return NULL;
    }
    if (look_place("page_table", device, &stream)) return NULL;
    const dkv_paged_tables c = {table.ptr, len.ptr, ring.ptr, at.ptr, batch, ring.dims[0], table.dims[1], page_size};
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = f_paged_resize(&c, x.ptr, off.ptr, pos.ptr, slots.ptr, rows, ws.ptr, bytes, stream);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(rc);
}

/* rows of one of the two tensors that are rotated, None for none, and where they go (None: where they are) */
static int look_rotated(PyObject *t, PyObject *to, const char *name, const char *to_name, int32_t head_dim, int device, tensor_info *in,
                        int64_t *in_stride, tensor_info *out, int64_t *out_stride) {
    if (look_rows(t, name, -1, head_dim, device, in, in_stride)) return -1;
    *out = *in;
    *out_stride = *in_stride;
    if (to == Py_None) return 0;
    if (look_rows(to, to_name, in->dims[1], head_dim, device, out, out_stride)) return -1;
    return out->dtype == in->dtype && out->dims[0] == in->dims[0] ? 0 : refuse(to_name, "the input's type and rows are expected");
}

/* (address of a dkv_rope_desc, q, k, positions, row_off, q_out, k_out, inverse): the status code of the library call */
static PyObject *py_rope(PyObject *self, PyObject *const *a, Py_ssize_t n) {
    if (!ready(n, 8)) return NULL;
    const dkv_rope_desc *rope = PyLong_AsVoidPtr(a[0]);
    if (PyErr_Occurred()) return NULL;
    tensor_info pos, off = {0}, q = {0}, k = {0}, q_out = {0}, k_out = {0};
    int64_t strides[4] = {0};
    int32_t inverse;
    void *stream;
    if (look(a[3], &pos)) return NULL;
    if (pos.dtype != T_I32 || pos.n_dims != 1 || !pos.whole) {
        refuse("positions", "a contiguous int32 tensor [rows] is expected");
        return NULL;
    }
    const int device = pos.device, has_q = a[1] != Py_None, has_k = a[2] != Py_None;
    if ((!has_q && a[5] != Py_None) || (!has_k && a[6] != Py_None)) {
        refuse(has_q ? "k_out" : "q_out", "there is nothing that goes there");
        return NULL;
    }
    if ((has_q && look_rotated(a[1], a[5], "q", "q_out", rope->head_dim, device, &q, &strides[0], &q_out, &strides[1])) ||
        (has_k && look_rotated(a[2], a[6], "k", "k_out", rope->head_dim, device, &k, &strides[2], &k_out, &strides[3])) || get_i32(a[7], &inverse))
        return NULL;
    if ((has_q && q.dims[0] != pos.dims[0]) || (has_k && k.dims[0] != pos.dims[0])) {
        refuse("positions", "one for each row is expected");
        return NULL;
    }
    if (has_q && has_k && q.dtype != k.dtype) {
        refuse("k", "the type of q is expected");
        return NULL;
    }
    if (a[4] != Py_None) {
        if (look_whole(a[4], "row_off", T_I32, -1, NULL, device, &off)) return NULL;
        if (off.dims[0] < 2) {
            refuse("row_off", "a number more than there are sequences is expected");
            return NULL;
        }
    }
    if (look_place("positions", device, &stream)) return NULL;
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = f_rope(rope, q.ptr, strides[0], q_out.ptr, strides[1], has_q ? q.dims[1] : 0, k.ptr, strides[2], k_out.ptr, strides[3], has_k ? k.dims[1] : 0,
                pos.ptr, off.ptr, off.ptr ? off.dims[0] - 1 : 0, pos.dims[0], has_q ? q.dtype : has_k ? k.dtype : DKV_FP32, inverse, stream);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(rc);
}

/* bind_paged(addresses of dkv_paged_store, _load, _attn_workspace_bytes, _attn, _resize and dkv_rope, then the types bfloat16, float32, float8_e4m3fn,
 * float8_e8m0fnu, float4_e2m1fn_x2, int32, int64, and what tells the current device and stream) */
static PyObject *py_bind_paged(PyObject *self, PyObject *const *a, Py_ssize_t n) {
    enum { FUNCTIONS = 6 };
    if (n != FUNCTIONS + T_COUNT + 1) {
        PyErr_SetString(PyExc_TypeError, "six addresses, seven types and a source of streams are expected");
        return NULL;
    }
    void *f[FUNCTIONS];
    for (int i = 0; i < FUNCTIONS; ++i) f[i] = PyLong_AsVoidPtr(a[i]);
    if (PyErr_Occurred()) return NULL;
    for (int i = 0; i < T_COUNT; ++i) {
        PyObject *old = dtypes[i];
        Py_INCREF(a[FUNCTIONS + i]);
        dtypes[i] = a[FUNCTIONS + i];
        Py_XDECREF(old);
    }
    PyObject *before = place_of;
    Py_INCREF(a[FUNCTIONS + T_COUNT]);
    place_of = a[FUNCTIONS + T_COUNT];
    Py_XDECREF(before);
    f_paged_store = (paged_store_fn)f[0];
    f_paged_load = (paged_load_fn)f[1];
    f_paged_bytes = (paged_bytes_fn)f[2];
    f_paged_attn = (paged_attn_fn)f[3];
    f_paged_resize = (paged_resize_fn)f[4];
    f_rope = (rope_fn)f[5];
    Py_RETURN_NONE;
}

static PyMethodDef methods[] = {
    {"attn_update", (PyCFunction)(void (*)(void))py_attn_update, METH_FASTCALL, NULL},
    {"attn_update_static", (PyCFunction)(void (*)(void))py_attn_update_static, METH_FASTCALL, NULL},
    {"paged_store", (PyCFunction)(void (*)(void))py_paged_store, METH_FASTCALL, NULL},
    {"paged_load", (PyCFunction)(void (*)(void))py_paged_load, METH_FASTCALL, NULL},
    {"paged_attn_workspace_bytes", (PyCFunction)(void (*)(void))py_paged_attn_workspace_bytes, METH_FASTCALL, NULL},
    {"paged_attn", (PyCFunction)(void (*)(void))py_paged_attn, METH_FASTCALL, NULL},
    {"paged_resize", (PyCFunction)(void (*)(void))py_paged_resize, METH_FASTCALL, NULL},
    {"rope", (PyCFunction)(void (*)(void))py_rope, METH_FASTCALL, NULL},
    {"bind_paged", (PyCFunction)(void (*)(void))py_bind_paged, METH_FASTCALL, NULL},
    {"bind", (PyCFunction)(void (*)(void))py_bind, METH_FASTCALL, NULL},
    {NULL, NULL, 0, NULL}};

static struct PyModuleDef module = {PyModuleDef_HEAD_INIT, "_marshal", NULL, -1, methods, NULL, NULL, NULL, NULL};

PyMODINIT_FUNC PyInit__marshal(void) {
    s_data_ptr = PyUnicode_InternFromString("data_ptr");
    s_shape = PyUnicode_InternFromString("shape");
    s_nbytes = PyUnicode_InternFromString("nbytes");
    s_value = PyUnicode_InternFromString("value");
    s_dtype = PyUnicode_InternFromString("dtype");
    s_is_contiguous = PyUnicode_InternFromString("is_contiguous");
    s_get_device = PyUnicode_InternFromString("get_device");
    s_stride = PyUnicode_InternFromString("stride");
    s_current = PyUnicode_InternFromString("_cuda_getDevice");
    s_stream = PyUnicode_InternFromString("_cuda_getCurrentRawStream");
    return s_data_ptr && s_shape && s_nbytes && s_value && s_dtype && s_is_contiguous && s_get_device && s_stride && s_current && s_stream ? PyModule_Create(&module) : NULL;
}
