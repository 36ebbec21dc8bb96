/* Argument marshalling of the calls whose launches are short enough for the host to bound them (rmm_product, rmm_reduced_attn, and
 * those on rows of heads and the 4-bit cache) as one native call each: reading three or four tensors, asking for the workspace size
 * and calling the library through ctypes took about as long as the GPU needs for a small product twice over.
 *
 * Only the plain form is taken (torch.Tensor or Parameter, no buffer passed in).  Whatever else it meets, and every
 * argument that would be refused, is answered with None: the caller's Python code then does the whole call, and raises what
 * it always raised.  Outputs and workspaces come from the same torch calls as there. */
#define PY_SSIZE_T_CLEAN
#include <Python.h>
#include <dlfcn.h>

#include "rmm.h"

static PyTypeObject *type_tensor, *type_parameter;
static PyObject *dt_bf16, *dt_f32, *dt_i32, *dt_u8;
static PyObject *fn_stream, *fn_device, *names;   /* names: the Python module's, looked up at every call */
static PyObject *s_is_cuda, *s_dtype, *s_shape, *s_stride, *s_data_ptr, *s_new_empty, *s_get_device, *s_numel, *s_device, *s_cuda, *s_ws_cache, *s_workspace, *s_check, *s_out, *kw_dtype;
static int poison;

static int (*p_keep_count)(double, int64_t, int64_t *);
static size_t (*p_product_ws)(const rmm_mat_t *, const rmm_mat_t *, const rmm_mat_t *);
static size_t (*p_score_ws)(const rmm_mat_t *, int);
static size_t (*p_gemm_ws)(const rmm_mat_t *, const rmm_mat_t *, int64_t, const rmm_mat_t *);
static int (*p_product)(const rmm_mat_t *, const rmm_mat_t *, double, int64_t, float, const rmm_mat_t *, int32_t *, float *, void *, size_t, void *);
static size_t (*p_attn_ws)(const rmm_attn_desc_t *);
static int (*p_attn)(const rmm_attn_desc_t *, const void *, const void *, const void *, void *, int32_t *, int32_t *, void *, size_t, void *);
static int (*p_norm_rope)(const rmm_heads_t *, const rmm_heads_t *, const void *, const void *, const rmm_rope_t *, const rmm_heads_t *, const rmm_heads_t *, void *, size_t, void *);
static int (*p_append)(const rmm_heads_t *, const rmm_heads_t *, const rmm_kv4_t *, const void *, const rmm_rope_t *, const rmm_heads_t *, const rmm_heads_t *, void *, size_t, void *);
static int (*p_read)(const rmm_kv4_t *, const rmm_heads_t *, const rmm_heads_t *, void *, size_t, void *);
static size_t (*p_kv4_attn_ws)(const rmm_heads_t *, const rmm_kv4_t *);
static int (*p_kv4_attn)(const rmm_heads_t *, const rmm_kv4_t *, int, double, const rmm_heads_t *, int32_t *, void *, size_t, void *);

/* 1: read; 0: not a plain CUDA tensor of a known dtype (no exception is left set) */
typedef struct {
    void *ptr;
    PyObject *dtype;   /* borrowed: one of the dtypes above */
    int dims;
    int64_t shape[4], stride[4];
    long device;       /* set by read_on */
} tensor_t;

static void find_exchange(PyObject *tensor_type);

static int read_tensor(PyObject *t, tensor_t *o)
{
    PyObject *v, *shape = NULL, *stride = NULL;
    int ok = 0;
    if (Py_TYPE(t) != type_tensor && Py_TYPE(t) != type_parameter) return 0;
    if ((v = PyObject_GetAttr(t, s_is_cuda)) == NULL) goto out;
    ok = v == Py_True;
    Py_DECREF(v);
    if (!ok) return 0;
    ok = 0;
    if ((v = PyObject_GetAttr(t, s_dtype)) == NULL) goto out;
    o->dtype = v == dt_bf16 ? dt_bf16 : v == dt_f32 ? dt_f32 : v == dt_i32 ? dt_i32 : v == dt_u8 ? dt_u8 : NULL;
    Py_DECREF(v);
    if (o->dtype == NULL) return 0;
    if ((shape = PyObject_GetAttr(t, s_shape)) == NULL || (stride = PyObject_CallMethodNoArgs(t, s_stride)) == NULL) goto out;
    if (!PyTuple_Check(shape) || !PyTuple_Check(stride) || PyTuple_GET_SIZE(shape) > 4 || PyTuple_GET_SIZE(shape) != PyTuple_GET_SIZE(stride)) goto out;
    o->dims = (int)PyTuple_GET_SIZE(shape);
    for (int i = 0; i < o->dims; ++i) {
        if (!PyLong_CheckExact(PyTuple_GET_ITEM(shape, i)) || !PyLong_CheckExact(PyTuple_GET_ITEM(stride, i))) goto out;
        o->shape[i] = PyLong_AsLongLong(PyTuple_GET_ITEM(shape, i));
        o->stride[i] = PyLong_AsLongLong(PyTuple_GET_ITEM(stride, i));
    }
    if ((v = PyObject_CallMethodNoArgs(t, s_data_ptr)) == NULL) goto out;
    o->ptr = PyLong_AsVoidPtr(v);
    Py_DECREF(v);
    ok = !PyErr_Occurred();
out:
    Py_XDECREF(shape);
    Py_XDECREF(stride);
    PyErr_Clear();
    return ok;
}

static int read_mat(PyObject *t, rmm_mat_t *m, int *dims)
{
    tensor_t r;
    if (!read_tensor(t, &r) || (r.dims != 2 && r.dims != 3) || (r.dtype != dt_bf16 && r.dtype != dt_f32)) return 0;
    const int b = r.dims - 2;
    m->ptr = r.ptr;
    m->dtype = r.dtype == dt_bf16 ? RMM_BF16 : RMM_F32;
    m->batch = b ? r.shape[0] : 1;
    m->rows = r.shape[b]; m->cols = r.shape[b + 1];
    m->stride_batch = b ? r.stride[0] : 0;
    m->stride_row = r.stride[b]; m->stride_col = r.stride[b + 1];
    *dims = r.dims;
    return 1;
}

static PyObject *named(PyObject *name)   /* borrowed */
{
    PyObject *v = PyDict_GetItemWithError(names, name);
    if (v == NULL && !PyErr_Occurred()) PyErr_SetObject(PyExc_NameError, name);
    return v;
}

static int number(PyObject *o, double *v)
{
    if (!PyFloat_CheckExact(o) && !PyLong_CheckExact(o)) return 0;
    *v = PyFloat_AsDouble(o);
    if (PyErr_Occurred()) { PyErr_Clear(); return 0; }
    return 1;
}

/* A new tensor on `like`'s device, of the given sizes; its address through *ptr.  NULL with an exception on failure. */
static PyObject *new_out(PyObject *like, int dims, const int64_t *size, PyObject *dtype, void **ptr)
{
    PyObject *shape = PyTuple_New(dims), *t = NULL, *v;
    if (shape == NULL) return NULL;
    for (int i = 0; i < dims; ++i) {
        if ((v = PyLong_FromLongLong(size[i])) == NULL) { Py_DECREF(shape); return NULL; }
        PyTuple_SET_ITEM(shape, i, v);
    }
    if (poison) {
        PyObject *args[3] = {shape, dtype, like}, *out = named(s_out);
        t = out != NULL ? PyObject_Vectorcall(out, args, 3, NULL) : NULL;
    } else {
        PyObject *args[3] = {like, shape, dtype};
        t = PyObject_VectorcallMethod(s_new_empty, args, 2, kw_dtype);
    }
    Py_DECREF(shape);
    if (t == NULL) return NULL;
    if ((v = PyObject_CallMethodNoArgs(t, s_data_ptr)) == NULL) { Py_DECREF(t); return NULL; }
    *ptr = PyLong_AsVoidPtr(v);
    Py_DECREF(v);
    return t;
}

/* The cached workspace of `like`'s device, at least `need` bytes: a new reference, its 256-byte aligned part through *ptr, *bytes */
static PyObject *workspace_of(PyObject *like, size_t need, void **ptr, size_t *bytes)
{
    PyObject *ws = NULL, *v, *key, *cache, *make;
    if (need < RMM_WS_HEADER_BYTES) need = RMM_WS_HEADER_BYTES;
    if ((v = PyObject_CallMethodNoArgs(like, s_get_device)) == NULL) return NULL;
    key = PyTuple_Pack(2, s_cuda, v);
    Py_DECREF(v);
    if (key == NULL) return NULL;
    /* (borrowed names are used at once: a tensor's methods may run Python code, which may bind them anew) */
    if ((cache = named(s_ws_cache)) != NULL && !PyDict_Check(cache)) PyErr_SetString(PyExc_TypeError, "_ws_cache must be a dict");
    ws = cache != NULL && PyDict_Check(cache) ? PyDict_GetItemWithError(cache, key) : NULL;
    Py_DECREF(key);
    if (ws == NULL && PyErr_Occurred()) return NULL;
    Py_XINCREF(ws);
    size_t have = 0;
    for (int pass = 0; pass < 2; ++pass) {
        if (ws != NULL) {
            if ((v = PyObject_CallMethodNoArgs(ws, s_numel)) == NULL) goto fail;
            have = PyLong_AsSize_t(v);
            Py_DECREF(v);
        }
        if (ws != NULL && have >= need) break;
        Py_XDECREF(ws);
        PyObject *dev = PyObject_GetAttr(like, s_device), *n = PyLong_FromSize_t(need);
        PyObject *args[2] = {n, dev};
        make = dev != NULL && n != NULL ? named(s_workspace) : NULL;
        ws = make != NULL ? PyObject_Vectorcall(make, args, 2, NULL) : NULL;
        Py_XDECREF(dev);
        Py_XDECREF(n);
        if (ws == NULL) return NULL;
    }
    if ((v = PyObject_CallMethodNoArgs(ws, s_data_ptr)) == NULL) goto fail;
    {
        const uintptr_t p = (uintptr_t)PyLong_AsVoidPtr(v), a = (p + 255) / 256 * 256;
        Py_DECREF(v);
        *ptr = (void *)a;
        *bytes = have - (size_t)(a - p);
    }
    if (PyErr_Occurred()) goto fail;
    return ws;
fail:
    Py_XDECREF(ws);
    return NULL;
}

static int stream_of(void **stream)
{
    PyObject *dev = PyObject_CallNoArgs(fn_device), *v;
    if (dev == NULL) return 0;
    v = PyObject_CallOneArg(fn_stream, dev);
    Py_DECREF(dev);
    if (v == NULL) return 0;
    *stream = PyLong_AsVoidPtr(v);
    Py_DECREF(v);
    return !PyErr_Occurred();
}

static int raise_status(int rc)   /* the library's text belongs to this thread, as in the Python code */
{
    PyObject *n = PyLong_FromLong(rc), *check = named(s_check), *v = n != NULL && check != NULL ? PyObject_CallOneArg(check, n) : NULL;
    Py_XDECREF(n);
    Py_XDECREF(v);
    return v != NULL;
}

/* product(A, B, rho, k, scale) -> (Y, idx) or None */
static PyObject *product(PyObject *self, PyObject *const *args, Py_ssize_t n)
{
    rmm_mat_t a, b, y;
    int da, db;
    double rho, scale;
    int64_t k;
    (void)self;
    if (n != 5 || !read_mat(args[0], &a, &da) || !read_mat(args[1], &b, &db) || !number(args[2], &rho) || !PyLong_CheckExact(args[3]) ||
        !number(args[4], &scale))
        Py_RETURN_NONE;
    k = PyLong_AsLongLong(args[3]);
    if (PyErr_Occurred()) { PyErr_Clear(); Py_RETURN_NONE; }
    int64_t kk = k;
    if (k <= 0 && p_keep_count(rho, a.cols, &kk) != RMM_OK) Py_RETURN_NONE;

    PyObject *Y = NULL, *idx = NULL, *ws = NULL, *ret = NULL;
    const int64_t ys[3] = {a.batch, a.rows, b.cols}, is[2] = {a.batch, kk};
    void *ip, *wp, *stream;
    size_t bytes, need;
    PyObject *dtype = a.dtype == RMM_BF16 ? dt_bf16 : dt_f32;
    if ((Y = new_out(args[0], da, ys + (da == 3 ? 0 : 1), dtype, &y.ptr)) == NULL) goto out;
    if ((idx = new_out(args[0], da - 1, is + (da == 3 ? 0 : 1), dt_i32, &ip)) == NULL) goto out;
    y.dtype = a.dtype; y.batch = a.batch; y.rows = a.rows; y.cols = b.cols;
    y.stride_col = 1;
    y.stride_row = b.cols > 0 ? b.cols : 1;   /* as torch describes a new tensor */
    y.stride_batch = da == 3 ? (a.rows > 0 ? a.rows : 1) * y.stride_row : 0;
    if (a.dtype == RMM_F32) {
        const size_t s = p_score_ws(&a, 1), g = p_gemm_ws(&a, &b, kk, &y);
        need = s == 0 || g == 0 ? 0 : s > g ? s : g;
    } else {
        need = p_product_ws(&a, &b, &y);
    }
    if (need == 0) { ret = Py_None; Py_INCREF(ret); goto out; }
    if ((ws = workspace_of(args[0], need, &wp, &bytes)) == NULL || !stream_of(&stream)) goto out;
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = p_product(&a, &b, rho, k, (float)scale, &y, (int32_t *)ip, NULL, wp, bytes, stream);
    if (rc != RMM_OK) { Py_BLOCK_THREADS raise_status(rc); Py_UNBLOCK_THREADS }
    Py_END_ALLOW_THREADS
    if (rc == RMM_OK) ret = PyTuple_Pack(2, Y, idx);
out:
    Py_XDECREF(Y);
    Py_XDECREF(idx);
    Py_XDECREF(ws);
    return ret;
}

/* attn(Q, K, V, causal, rho_d, rho_t) -> O or None */
static PyObject *attn(PyObject *self, PyObject *const *args, Py_ssize_t n)
{
    tensor_t t[3];
    rmm_attn_desc_t d = {0};
    (void)self;
    if (n != 6) Py_RETURN_NONE;
    for (int i = 0; i < 3; ++i)
        if (!read_tensor(args[i], &t[i]) || t[i].dims != 4 || t[i].dtype != dt_bf16 || t[i].stride[3] != 1) Py_RETURN_NONE;
    if ((args[3] != Py_True && args[3] != Py_False) || !number(args[4], &d.rho_d) || !number(args[5], &d.rho_t)) Py_RETURN_NONE;
    d.B = t[0].shape[0]; d.Hq = t[0].shape[1]; d.Lq = t[0].shape[2]; d.Dh = t[0].shape[3];
    d.Hkv = t[1].shape[1]; d.Lk = t[1].shape[2];
    if (d.B < 1 || d.Hq < 1 || d.Lq < 1 || d.Dh < 1) Py_RETURN_NONE;
    if (t[1].shape[0] < d.B || t[1].shape[3] < d.Dh || t[2].shape[0] < d.B || t[2].shape[1] < d.Hkv || t[2].shape[2] < d.Lk ||
        t[2].shape[3] < d.Dh)
        Py_RETURN_NONE;   /* refused there: the library sees strides only */
    d.causal = args[3] == Py_True;
    for (int i = 0; i < 3; ++i) {
        d.q_stride[i] = t[0].stride[i];
        d.k_stride[i] = t[1].stride[i];
        d.v_stride[i] = t[2].stride[i];
    }
    d.o_stride[2] = d.Dh; d.o_stride[1] = d.Lq * d.Dh; d.o_stride[0] = d.Hq * d.o_stride[1];
    const size_t need = p_attn_ws(&d);
    if (need == 0) Py_RETURN_NONE;
    PyObject *O = NULL, *ws = NULL, *ret = NULL;
    const int64_t os[4] = {d.B, d.Hq, d.Lq, d.Dh};
    void *op, *wp, *stream;
    size_t bytes;
    int rc;
    if ((O = new_out(args[0], 4, os, dt_bf16, &op)) == NULL) goto out;
    if ((ws = workspace_of(args[0], need, &wp, &bytes)) == NULL || !stream_of(&stream)) goto out;
    Py_BEGIN_ALLOW_THREADS
    rc = p_attn(&d, t[0].ptr, t[1].ptr, t[2].ptr, op, NULL, NULL, wp, bytes, stream);
    if (rc != RMM_OK) { Py_BLOCK_THREADS raise_status(rc); Py_UNBLOCK_THREADS }
    Py_END_ALLOW_THREADS
    if (rc == RMM_OK) { ret = O; Py_INCREF(ret); }
out:
    Py_XDECREF(O);
    Py_XDECREF(ws);
    return ret;
}

/* ---- rows of heads and the 4-bit cache.  What is not plain here: a tensor of another device than the current one, and whatever the
 * Python code would refuse. */

static int current_device(long *index)
{
    PyObject *v = PyObject_CallNoArgs(fn_device);
    if (v == NULL) { PyErr_Clear(); return 0; }
    *index = PyLong_AsLong(v);
    Py_DECREF(v);
    if (PyErr_Occurred()) { PyErr_Clear(); return 0; }
    return 1;
}

/* The tensors' exchange table of the DLPack protocol (its published C structures): a description of a tensor in one C call.
 * NULL where this torch has none: the attributes are then read one by one. */
typedef struct { int32_t type, id; } dl_device;
typedef struct { uint8_t code, bits; uint16_t lanes; } dl_dtype;
typedef struct { void *data; dl_device device; int32_t ndim; dl_dtype dtype; int64_t *shape, *strides; uint64_t byte_offset; } dl_tensor;
typedef struct dl_header { struct { uint32_t major, minor; } version; struct dl_header *prev; } dl_header;
typedef struct {
    dl_header header;
    void *managed_tensor_allocator, *managed_tensor_from_py_object, *managed_tensor_to_py_object;
    int (*dltensor_from_py_object)(void *, dl_tensor *);
    void *current_work_stream;
} dl_exchange;
enum { DL_CUDA = 2, DL_INT = 0, DL_UINT = 1, DL_FLOAT = 2, DL_BFLOAT = 4, DL_MAJOR = 1 };
static const dl_exchange *exchange;

static void find_exchange(PyObject *tensor_type)
{
    PyObject *capsule = PyObject_GetAttrString(tensor_type, "__dlpack_c_exchange_api__");
    if (capsule != NULL && PyCapsule_CheckExact(capsule)) {
        const dl_exchange *e = PyCapsule_GetPointer(capsule, "dlpack_exchange_api");
        if (e != NULL && e->header.version.major == DL_MAJOR && e->dltensor_from_py_object != NULL) exchange = e;
    }
    Py_XDECREF(capsule);   /* (the table lives as long as the process) */
    PyErr_Clear();
}

/* 1: read, and on the given device */
static int read_on(PyObject *t, tensor_t *o, long device)
{
    PyObject *v;
    if (exchange != NULL) {
        dl_tensor d;
        if (Py_TYPE(t) != type_tensor && Py_TYPE(t) != type_parameter) return 0;
        if (exchange->dltensor_from_py_object(t, &d) != 0) { PyErr_Clear(); return 0; }
        if (d.device.type != DL_CUDA || d.device.id != device || d.ndim < 1 || d.ndim > 4 || d.dtype.lanes != 1 || d.strides == NULL) return 0;
        o->dtype = d.dtype.code == DL_BFLOAT && d.dtype.bits == 16  ? dt_bf16
                   : d.dtype.code == DL_FLOAT && d.dtype.bits == 32 ? dt_f32
                   : d.dtype.code == DL_INT && d.dtype.bits == 32   ? dt_i32
                   : d.dtype.code == DL_UINT && d.dtype.bits == 8   ? dt_u8
                                                                    : NULL;
        if (o->dtype == NULL) return 0;
        o->ptr = (char *)d.data + d.byte_offset;
        o->dims = d.ndim;
        for (int i = 0; i < d.ndim; ++i) {
            o->shape[i] = d.shape[i];
            o->stride[i] = d.strides[i];
        }
        o->device = device;
        return 1;
    }
    if (!read_tensor(t, o)) return 0;
    if ((v = PyObject_CallMethodNoArgs(t, s_get_device)) == NULL) { PyErr_Clear(); return 0; }
    o->device = PyLong_AsLong(v);
    Py_DECREF(v);
    if (PyErr_Occurred()) { PyErr_Clear(); return 0; }
    return o->device == device;
}

static int read_heads(PyObject *t, rmm_heads_t *h, long device)
{
    tensor_t r;
    if (!read_on(t, &r, device) || r.dims != 4 || (r.dtype != dt_bf16 && r.dtype != dt_f32) || (r.stride[3] != 1 && r.shape[3] > 1)) return 0;
    h->ptr = r.ptr;
    h->dtype = r.dtype == dt_bf16 ? RMM_BF16 : RMM_F32;
    h->B = r.shape[0]; h->H = r.shape[1]; h->L = r.shape[2]; h->D = r.shape[3];
    for (int i = 0; i < 3; ++i) h->stride[i] = r.stride[i];
    return h->B > 0 && h->H > 0 && h->L > 0 && h->D > 0;
}

/* A weight [D] (None: NULL); *dtype: -1 before the first, the same for all */
static int read_weight(PyObject *t, int64_t D, const void **ptr, int *dtype, long device)
{
    tensor_t r;
    *ptr = NULL;
    if (t == Py_None) return 1;
    if (!read_on(t, &r, device) || r.dims != 1 || r.shape[0] != D || (r.stride[0] != 1 && D > 1) || (r.dtype != dt_bf16 && r.dtype != dt_f32)) return 0;
    const int dt = r.dtype == dt_bf16 ? RMM_BF16 : RMM_F32;
    if (*dtype >= 0 && *dtype != dt) return 0;
    *dtype = dt;
    *ptr = r.ptr;
    return 1;
}

static int read_rope(PyObject *table, PyObject *eps, PyObject *interleaved, rmm_rope_t *r, long device)
{
    tensor_t t;
    if (!number(eps, &r->eps) || (interleaved != Py_True && interleaved != Py_False)) return 0;
    r->interleaved = interleaved == Py_True;
    if (table == Py_None) return 1;
    if (!read_on(table, &t, device) || t.dims != 2 || t.dtype != dt_f32 || t.stride[1] != 1 || t.shape[0] < 1 || t.shape[1] < 1) return 0;
    r->table = t.ptr;
    r->table_rows = t.shape[0];
    r->rot = t.shape[1];
    r->table_stride = t.shape[0] > 1 ? t.stride[0] : t.shape[1];
    return 1;
}

static int read_ints(PyObject *t, int64_t n, const int32_t **ptr, long device)
{
    tensor_t r;
    if (!read_on(t, &r, device) || r.dims != 1 || r.dtype != dt_i32 || r.shape[0] != n || (r.stride[0] != 1 && n > 1)) return 0;
    *ptr = r.ptr;
    return 1;
}

static int read_cache(PyObject *pool, PyObject *pages, PyObject *lengths, PyObject *new_len, rmm_kv4_t *c, long device)
{
    tensor_t p, t;
    if (!read_on(pool, &p, device) || p.dims != 4 || p.dtype != dt_u8 || p.stride[3] != 1 || p.shape[0] < 1 || p.shape[1] < 1 || p.shape[2] < 1 ||
        p.shape[3] < 18 || p.shape[3] % 18 != 0 || (p.shape[2] > 1 && p.stride[2] != p.shape[3]))
        return 0;
    if (!read_on(pages, &t, device) || t.dims != 2 || t.dtype != dt_i32 || (t.stride[1] != 1 && t.shape[1] > 1)) return 0;
    c->pool = p.ptr;
    c->n_pages = p.shape[0]; c->Hkv = p.shape[1]; c->page = 16 * p.shape[2]; c->Dh = p.shape[3] / 18;
    c->page_stride = c->n_pages > 1 ? p.stride[0] : c->Hkv * p.shape[2] * p.shape[3];
    c->head_stride = c->Hkv > 1 ? p.stride[1] : p.shape[2] * p.shape[3];
    c->pages = t.ptr;
    c->B = t.shape[0]; c->max_pages = t.shape[1]; c->pages_stride = c->B > 1 ? t.stride[0] : c->max_pages;
    return read_ints(lengths, c->B, &c->lengths, device) && (new_len == Py_None || read_ints(new_len, c->B, &c->new_len, device));
}

static PyObject *new_heads(PyObject *like, const rmm_heads_t *shape, PyObject *dtype, rmm_heads_t *out)
{
    const int64_t size[4] = {shape->B, shape->H, shape->L, shape->D};
    *out = *shape;
    out->dtype = dtype == dt_bf16 ? RMM_BF16 : RMM_F32;
    out->stride[2] = shape->D; out->stride[1] = shape->L * shape->D; out->stride[0] = shape->H * out->stride[1];
    return new_out(like, 4, size, dtype, &out->ptr);
}

/* 1: done; 0: an exception is set */
#define CALL(expression)                                                        \
    do {                                                                        \
        Py_BEGIN_ALLOW_THREADS                                                  \
        rc = (expression);                                                      \
        if (rc != RMM_OK) { Py_BLOCK_THREADS raise_status(rc); Py_UNBLOCK_THREADS } \
        Py_END_ALLOW_THREADS                                                    \
    } while (0)

/* norm_rope(Q, K, q_weight, k_weight, rope, positions, eps, interleaved) -> Q', (Q', K') or None */
static PyObject *norm_rope(PyObject *self, PyObject *const *args, Py_ssize_t n)
{
    rmm_heads_t q, k, qo, ko;
    rmm_rope_t r = {0};
    const void *qw, *kw;
    int dtype = -1, rc;
    long device;
    (void)self;
    if (n != 8 || !current_device(&device) || !read_heads(args[0], &q, device)) Py_RETURN_NONE;
    const int has_k = args[1] != Py_None;
    if ((has_k && (!read_heads(args[1], &k, device) || k.dtype != q.dtype)) || !read_weight(args[2], q.D, &qw, &dtype, device) ||
        !read_weight(args[3], q.D, &kw, &dtype, device) || !read_rope(args[4], args[6], args[7], &r, device))
        Py_RETURN_NONE;
    r.weight_dtype = dtype < 0 ? RMM_F32 : dtype;
    if (args[5] != Py_None) {
        tensor_t p;
        if (!read_on(args[5], &p, device) || p.dtype != dt_i32 || (p.dims != 1 && p.dims != 2) || p.shape[p.dims - 1] != q.L) Py_RETURN_NONE;
        if (p.dims == 2 && p.shape[0] != 1 && p.shape[0] != q.B) Py_RETURN_NONE;
        r.positions = p.ptr;
        r.pos_stride[0] = p.dims == 2 && p.shape[0] != 1 ? p.stride[0] : 0;
        r.pos_stride[1] = p.stride[p.dims - 1];
    }
    PyObject *Qo = NULL, *Ko = NULL, *ws = NULL, *ret = NULL, *dt = q.dtype == RMM_BF16 ? dt_bf16 : dt_f32;
    void *wp, *stream;
    size_t bytes;
    if ((Qo = new_heads(args[0], &q, dt, &qo)) == NULL || (has_k && (Ko = new_heads(args[1], &k, dt, &ko)) == NULL)) goto out;
    if ((ws = workspace_of(args[0], 0, &wp, &bytes)) == NULL || !stream_of(&stream)) goto out;
    CALL(p_norm_rope(&q, has_k ? &k : NULL, qw, kw, &r, &qo, has_k ? &ko : NULL, wp, bytes, stream));
    if (rc == RMM_OK) {
        if (has_k) ret = PyTuple_Pack(2, Qo, Ko);
        else { ret = Qo; Py_INCREF(ret); }
    }
out:
    Py_XDECREF(Qo);
    Py_XDECREF(Ko);
    Py_XDECREF(ws);
    return ret;
}

/* kv4_append(K, V, pool, pages, lengths, new_len, k_weight, rope, eps, interleaved, want_values) -> (K', V'), False (done, nothing asked for) or None */
static PyObject *kv4_append(PyObject *self, PyObject *const *args, Py_ssize_t n)
{
    rmm_heads_t k, v, ko, vo;
    rmm_rope_t r = {0};
    rmm_kv4_t c = {0};
    const void *kw;
    int dtype = -1, rc;
    long device;
    (void)self;
    if (n != 11 || !current_device(&device) || !read_heads(args[0], &k, device) || !read_heads(args[1], &v, device) ||
        !read_cache(args[2], args[3], args[4], args[5], &c, device) || !read_weight(args[6], k.D, &kw, &dtype, device) ||
        !read_rope(args[7], args[8], args[9], &r, device) || (args[10] != Py_True && args[10] != Py_False))
        Py_RETURN_NONE;
    r.weight_dtype = dtype < 0 ? RMM_F32 : dtype;
    const int held = args[10] == Py_True;
    PyObject *Ko = NULL, *Vo = NULL, *ws = NULL, *ret = NULL;
    void *wp, *stream;
    size_t bytes;
    if (held && ((Ko = new_heads(args[0], &k, dt_bf16, &ko)) == NULL || (Vo = new_heads(args[0], &k, dt_bf16, &vo)) == NULL)) goto out;
    if ((ws = workspace_of(args[0], 0, &wp, &bytes)) == NULL || !stream_of(&stream)) goto out;
    CALL(p_append(&k, &v, &c, kw, &r, held ? &ko : NULL, held ? &vo : NULL, wp, bytes, stream));
    if (rc == RMM_OK) {
        if (held) ret = PyTuple_Pack(2, Ko, Vo);
        else { ret = Py_False; Py_INCREF(ret); }
    }
out:
    Py_XDECREF(Ko);
    Py_XDECREF(Vo);
    Py_XDECREF(ws);
    return ret;
}

/* kv4_read(pool, pages, lengths, new_len, rows, dtype) -> (K, V) or None */
static PyObject *kv4_read(PyObject *self, PyObject *const *args, Py_ssize_t n)
{
    rmm_kv4_t c = {0};
    rmm_heads_t shape = {0}, k, v;
    int rc;
    long device;
    (void)self;
    if (n != 6 || !current_device(&device) || !read_cache(args[0], args[1], args[2], args[3], &c, device) || !PyLong_CheckExact(args[4]) ||
        (args[5] != dt_bf16 && args[5] != dt_f32))
        Py_RETURN_NONE;
    shape.B = c.B; shape.H = c.Hkv; shape.L = PyLong_AsLongLong(args[4]); shape.D = c.Dh;
    if (PyErr_Occurred()) { PyErr_Clear(); Py_RETURN_NONE; }
    if (shape.B < 1 || shape.L < 1) Py_RETURN_NONE;
    PyObject *K = NULL, *V = NULL, *ws = NULL, *ret = NULL;
    void *wp, *stream;
    size_t bytes;
    if ((K = new_heads(args[0], &shape, args[5], &k)) == NULL || (V = new_heads(args[0], &shape, args[5], &v)) == NULL) goto out;
    if ((ws = workspace_of(args[0], 0, &wp, &bytes)) == NULL || !stream_of(&stream)) goto out;
    CALL(p_read(&c, &k, &v, wp, bytes, stream));
    if (rc == RMM_OK) ret = PyTuple_Pack(2, K, V);
out:
    Py_XDECREF(K);
    Py_XDECREF(V);
    Py_XDECREF(ws);
    return ret;
}

/* kv4_attn(Q, pool, pages, lengths, new_len, causal, rho_d) -> O or None */
static PyObject *kv4_attn(PyObject *self, PyObject *const *args, Py_ssize_t n)
{
    rmm_kv4_t c = {0};
    rmm_heads_t q, o;
    double rho_d;
    int rc;
    long device;
    (void)self;
    if (n != 7 || !current_device(&device) || !read_heads(args[0], &q, device) || !read_cache(args[1], args[2], args[3], args[4], &c, device) ||
        (args[5] != Py_True && args[5] != Py_False) || !number(args[6], &rho_d))
        Py_RETURN_NONE;
    const size_t need = p_kv4_attn_ws(&q, &c);
    if (need == 0) Py_RETURN_NONE;
    PyObject *O = NULL, *ws = NULL, *ret = NULL;
    void *wp, *stream;
    size_t bytes;
    if ((O = new_heads(args[0], &q, dt_bf16, &o)) == NULL) goto out;
    if ((ws = workspace_of(args[0], need, &wp, &bytes)) == NULL || !stream_of(&stream)) goto out;
    CALL(p_kv4_attn(&q, &c, args[5] == Py_True, rho_d, &o, NULL, wp, bytes, stream));
    if (rc == RMM_OK) { ret = O; Py_INCREF(ret); }
out:
    Py_XDECREF(O);
    Py_XDECREF(ws);
    return ret;
}

static PyObject *set_poison(PyObject *self, PyObject *on)
{
    (void)self;
    poison = PyObject_IsTrue(on);
    Py_RETURN_NONE;
}

/* init(library path, (Tensor, Parameter), (bfloat16, float32, int32, uint8), (raw stream, current device), the module's names) */
static PyObject *init(PyObject *self, PyObject *args)
{
    const char *path;
    PyObject *tt, *tp;
    (void)self;
    if (!PyArg_ParseTuple(args, "s(OO)(OOOO)(OO)O!", &path, &tt, &tp, &dt_bf16, &dt_f32, &dt_i32, &dt_u8, &fn_stream, &fn_device, &PyDict_Type,
                          &names))
        return NULL;
    void *h = dlopen(path, RTLD_NOW);
    if (h == NULL) { PyErr_SetString(PyExc_RuntimeError, dlerror()); return NULL; }
    *(void **)&p_keep_count = dlsym(h, "rmm_keep_count");
    *(void **)&p_product_ws = dlsym(h, "rmm_product_workspace_bytes");
    *(void **)&p_score_ws = dlsym(h, "rmm_score_select_workspace_bytes");
    *(void **)&p_gemm_ws = dlsym(h, "rmm_reduced_gemm_workspace_bytes");
    *(void **)&p_product = dlsym(h, "rmm_product");
    *(void **)&p_attn_ws = dlsym(h, "rmm_reduced_attn_workspace_bytes");
    *(void **)&p_attn = dlsym(h, "rmm_reduced_attn");
    *(void **)&p_norm_rope = dlsym(h, "rmm_qk_norm_rope");
    *(void **)&p_append = dlsym(h, "rmm_kv4_append");
    *(void **)&p_read = dlsym(h, "rmm_kv4_read");
    *(void **)&p_kv4_attn_ws = dlsym(h, "rmm_kv4_attn_workspace_bytes");
    *(void **)&p_kv4_attn = dlsym(h, "rmm_kv4_attn");
    if (!p_keep_count || !p_product_ws || !p_score_ws || !p_gemm_ws || !p_product || !p_attn_ws || !p_attn || !p_norm_rope || !p_append || !p_read ||
        !p_kv4_attn_ws || !p_kv4_attn) {
        PyErr_SetString(PyExc_RuntimeError, "librmm_b200.so lacks an entry point");
        return NULL;
    }
    find_exchange(tt);
    type_tensor = (PyTypeObject *)tt;
    type_parameter = (PyTypeObject *)tp;
    PyObject *keep[] = {tt, tp, dt_bf16, dt_f32, dt_i32, dt_u8, fn_stream, fn_device, names};
    for (size_t i = 0; i < sizeof keep / sizeof *keep; ++i) Py_INCREF(keep[i]);   /* for the life of the process */
    Py_RETURN_NONE;
}

static PyMethodDef methods[] = {
    {"init", init, METH_VARARGS, NULL},
    {"set_poison", set_poison, METH_O, NULL},
    {"product", (PyCFunction)(void (*)(void))product, METH_FASTCALL, NULL},
    {"attn", (PyCFunction)(void (*)(void))attn, METH_FASTCALL, NULL},
    {"norm_rope", (PyCFunction)(void (*)(void))norm_rope, METH_FASTCALL, NULL},
    {"kv4_append", (PyCFunction)(void (*)(void))kv4_append, METH_FASTCALL, NULL},
    {"kv4_read", (PyCFunction)(void (*)(void))kv4_read, METH_FASTCALL, NULL},
    {"kv4_attn", (PyCFunction)(void (*)(void))kv4_attn, METH_FASTCALL, NULL},
    {NULL, NULL, 0, NULL},
};
static struct PyModuleDef module = {PyModuleDef_HEAD_INIT, "rmm_marshal", NULL, -1, methods, NULL, NULL, NULL, NULL};

PyMODINIT_FUNC PyInit_rmm_marshal(void)
{
    struct { PyObject **p; const char *s; } texts[] = {
        {&s_is_cuda, "is_cuda"}, {&s_dtype, "dtype"}, {&s_shape, "shape"}, {&s_stride, "stride"}, {&s_data_ptr, "data_ptr"},
        {&s_new_empty, "new_empty"}, {&s_get_device, "get_device"}, {&s_numel, "numel"}, {&s_device, "device"}, {&s_cuda, "cuda"},
        {&s_ws_cache, "_ws_cache"}, {&s_workspace, "workspace"}, {&s_check, "_check"}, {&s_out, "_out"}};
    for (size_t i = 0; i < sizeof texts / sizeof *texts; ++i)
        if ((*texts[i].p = PyUnicode_InternFromString(texts[i].s)) == NULL) return NULL;
    if ((kw_dtype = PyTuple_Pack(1, s_dtype)) == NULL) return NULL;
    return PyModule_Create(&module);
}
