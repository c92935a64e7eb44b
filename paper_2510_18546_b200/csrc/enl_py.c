/* The calls that a planner makes per layer or per group, for Python: argument marshalling in C over the C ABI.
 *
 * A planning step calls enl_attend once per layer; through ctypes the marshalling of one call (structure fields, array
 * conversions, pointer casts) took about 8 us of host time, longer than the kernel of a short decode step runs.  Here it
 * is about 1 us.  Nothing is computed and nothing is kept between calls; enl.py holds the signatures and raises the errors.
 *
 * Tensors are asked for data_ptr(), and for their sizes only where the caller has not given them.  Index lists are read in
 * place when they are contiguous int32 arrays; anything else goes through the converter that enl.py hands over once. */
#define PY_SSIZE_T_CLEAN
#include <Python.h>
#include <string.h>

#include "../../include/enl.h"

static PyObject *s_data_ptr, *s_shape, *s_dtype, *s_contiguous, *s_get_device, *to_int32;
static PyObject *t_bf16, *t_int32, *t_int64;                /* torch's dtypes (enl.py hands them over once) */

/* 0 and NULL for None */
static int tensor_ptr(PyObject *t, void **out)
{
    *out = NULL;
    if (t == Py_None) return 0;
    PyObject *v = PyObject_CallMethodNoArgs(t, s_data_ptr);
    if (!v) return -1;
    *out = PyLong_AsVoidPtr(v);
    Py_DECREF(v);
    return (!*out && PyErr_Occurred()) ? -1 : 0;
}

/* one dimension of a tensor, counted from the end if negative (by `shape`: len() and size() of a tensor take three times as long) */
static int dim_of(PyObject *t, Py_ssize_t at, int32_t *out)
{
    PyObject *shape = PyObject_GetAttr(t, s_shape);
    if (!shape) return -1;
    PyObject *v = NULL;
    if (PyTuple_Check(shape)) {
        const Py_ssize_t n = PyTuple_GET_SIZE(shape), i = at < 0 ? n + at : at;
        if (i >= 0 && i < n) {
            v = PyTuple_GET_ITEM(shape, i);
            Py_INCREF(v);
        } else {
            PyErr_SetString(PyExc_IndexError, "tensor has too few dimensions");
        }
    } else {
        v = PySequence_GetItem(shape, at);
    }
    Py_DECREF(shape);
    if (!v) return -1;
    *out = (int32_t)PyLong_AsLong(v);
    Py_DECREF(v);
    return (*out == -1 && PyErr_Occurred()) ? -1 : 0;
}
static int last_dim(PyObject *t, int32_t *out) { return dim_of(t, -1, out); }
static int first_dim(PyObject *t, int32_t *out) { return dim_of(t, 0, out); }

static int int_arg(PyObject *o, int32_t *out)
{
    const long v = PyLong_AsLong(o);
    if (v == -1 && PyErr_Occurred()) {
        /* numpy integers and the like */
        PyErr_Clear();
        PyObject *i = PyNumber_Index(o);
        if (!i) return -1;
        const long w = PyLong_AsLong(i);
        Py_DECREF(i);
        if (w == -1 && PyErr_Occurred()) return -1;
        *out = (int32_t)w;
        return 0;
    }
    *out = (int32_t)v;
    return 0;
}

static int handle_arg(PyObject *o, void **out)
{
    *out = NULL;
    if (o == Py_None) return 0;
    *out = PyLong_AsVoidPtr(o);
    return (!*out && PyErr_Occurred()) ? -1 : 0;
}

/* an index list as contiguous int32 */
typedef struct {
    const int32_t *p;
    Py_ssize_t n;
    Py_buffer view;
    int held;
} ints_t;

static int ints_get(PyObject *o, ints_t *a)
{
    a->p = NULL;
    a->n = 0;
    a->held = 0;
    if (o == Py_None) return 0;
    PyObject *conv = NULL;
    int got = PyObject_CheckBuffer(o) && PyObject_GetBuffer(o, &a->view, PyBUF_C_CONTIGUOUS | PyBUF_FORMAT) == 0;
    if (got && !(a->view.itemsize == 4 && a->view.ndim == 1 && a->view.format && strcmp(a->view.format, "i") == 0)) {
        PyBuffer_Release(&a->view);
        got = 0;
    }
    if (!got) {
        PyErr_Clear();
        conv = PyObject_CallOneArg(to_int32, o);
        if (!conv) return -1;
        const int rc = PyObject_GetBuffer(conv, &a->view, PyBUF_C_CONTIGUOUS | PyBUF_FORMAT);
        Py_DECREF(conv);                                    /* the view keeps it alive */
        if (rc != 0) return -1;
    }
    a->held = 1;
    a->p = (const int32_t *)a->view.buf;
    a->n = a->view.len / 4;
    return 0;
}

static void ints_free(ints_t *a)
{
    if (a->held) PyBuffer_Release(&a->view);
    a->held = 0;
}

static int want_args(Py_ssize_t n, Py_ssize_t want)
{
    if (n == want) return 0;
    PyErr_Format(PyExc_TypeError, "expected %zd arguments, got %zd", want, n);
    return -1;
}

/* attend(cache, layer, sel_ids, q, k_new, v_new, out, group_mass, cu_sel, cu_q, cu_new, n_q, n_new, mass_stride, sel_off,
 *        split_hint, flags, stream, group_mass_sum, obj_off) -> return code.  sel_off: a callable that makes the int32 array
 * for n entries and keeps it, or None. */
static PyObject *py_attend(PyObject *self, PyObject *const *v, Py_ssize_t nargs)
{
    (void)self;
    if (want_args(nargs, 20)) return NULL;
    enl_attend_args_t a;
    memset(&a, 0, sizeof a);
    ints_t sel, cs, cq, cn, oo, so;
    sel.held = cs.held = cq.held = cn.held = oo.held = so.held = 0;
    PyObject *so_obj = NULL, *ret = NULL;
    void *cache, *stream, *p;
    int32_t flags;
    if (handle_arg(v[0], &cache) || int_arg(v[1], &a.layer) || ints_get(v[2], &sel)) goto done;
    if (tensor_ptr(v[3], &p)) goto done;
    a.q = p;
    if (tensor_ptr(v[4], &p)) goto done;
    a.k_new = p;
    if (tensor_ptr(v[5], &p)) goto done;
    a.v_new = p;
    if (tensor_ptr(v[6], &a.out)) goto done;
    if (tensor_ptr(v[7], &p)) goto done;
    a.group_mass = (float *)p;
    if (ints_get(v[8], &cs) || ints_get(v[9], &cq) || ints_get(v[10], &cn)) goto done;
    a.batch = v[9] == Py_None ? 1 : (int32_t)cq.n - 1;
    a.sel_ids = sel.p;
    a.n_sel = (int32_t)sel.n;
    a.cu_sel = cs.p;
    a.cu_q = cq.p;
    a.cu_new = cn.p;
    if (v[11] != Py_None ? int_arg(v[11], &a.n_q) : first_dim(v[3], &a.n_q)) goto done;
    if (v[12] != Py_None ? int_arg(v[12], &a.n_new) : first_dim(v[4], &a.n_new)) goto done;
    if (v[13] != Py_None) {
        if (int_arg(v[13], &a.mass_stride)) goto done;
    } else if (v[7] != Py_None && last_dim(v[7], &a.mass_stride)) {
        goto done;
    }
    if (v[14] != Py_None) {
        so_obj = PyObject_CallFunction(v[14], "n", sel.n + (Py_ssize_t)a.batch);
        if (!so_obj || ints_get(so_obj, &so)) goto done;
        a.sel_off_out = (int32_t *)so.p;
    }
    if (int_arg(v[15], &a.split_hint) || int_arg(v[16], &flags) || handle_arg(v[17], &stream)) goto done;
    a.flags = (uint32_t)flags;
    if (v[18] != Py_None) {
        if (tensor_ptr(v[18], &p) || last_dim(v[18], &a.sum_stride)) goto done;
        a.group_mass_sum = (float *)p;
    }
    if (ints_get(v[19], &oo)) goto done;
    a.n_obj = v[19] == Py_None ? 0 : (int32_t)oo.n - 1;
    a.obj_off = oo.p;
    {
        int rc;
        Py_BEGIN_ALLOW_THREADS
        rc = enl_attend((enl_cache_t *)cache, &a, stream);
        Py_END_ALLOW_THREADS
        ret = PyLong_FromLong(rc);
    }
done:
    ints_free(&sel);
    ints_free(&cs);
    ints_free(&cq);
    ints_free(&cn);
    ints_free(&oo);
    ints_free(&so);
    Py_XDECREF(so_obj);
    return ret;
}

/* attend_static(seg_len, n_new, q, k, v, out, group_mass, stream) -> return code */
static PyObject *py_attend_static(PyObject *self, PyObject *const *v, Py_ssize_t nargs)
{
    (void)self;
    if (want_args(nargs, 8)) return NULL;
    enl_static_args_t a;
    memset(&a, 0, sizeof a);
    ints_t seg;
    seg.held = 0;
    PyObject *ret = NULL;
    void *stream, *p;
    if (ints_get(v[0], &seg) || int_arg(v[1], &a.n_new)) goto done;
    if (last_dim(v[2], &a.head_dim)) goto done;
    if (dim_of(v[2], -2, &a.n_q_heads) || dim_of(v[3], -2, &a.n_kv_heads)) goto done;
    a.n_seg = (int32_t)seg.n;
    a.seg_len = seg.n ? seg.p : NULL;
    if (tensor_ptr(v[2], &p)) goto done;
    a.q = p;
    if (tensor_ptr(v[3], &p)) goto done;
    a.k = p;
    if (tensor_ptr(v[4], &p)) goto done;
    a.v = p;
    if (tensor_ptr(v[5], &a.out) || tensor_ptr(v[6], &p)) goto done;
    a.group_mass = (float *)p;
    if (handle_arg(v[7], &stream)) goto done;
    {
        int rc;
        Py_BEGIN_ALLOW_THREADS
        rc = enl_attend_static(&a, stream);
        Py_END_ALLOW_THREADS
        ret = PyLong_FromLong(rc);
    }
done:
    ints_free(&seg);
    return ret;
}

/* store(cache, group_id, layer, n_tokens or None, k, v, mode, stream) -> return code */
static PyObject *py_store(PyObject *self, PyObject *const *v, Py_ssize_t nargs)
{
    (void)self;
    if (want_args(nargs, 8)) return NULL;
    void *cache, *stream, *k, *vv;
    int32_t group, layer, n, mode;
    if (handle_arg(v[0], &cache) || int_arg(v[1], &group) || int_arg(v[2], &layer)) return NULL;
    if (v[4] != Py_None ? first_dim(v[4], &n) : int_arg(v[3], &n)) return NULL;
    if (tensor_ptr(v[4], &k) || tensor_ptr(v[5], &vv) || int_arg(v[6], &mode) || handle_arg(v[7], &stream)) return NULL;
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = enl_group_store((enl_cache_t *)cache, group, layer, n, k, vv, mode, stream);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(rc);
}

/* store_all_layers(cache, group_id, ks, vs, mode, stream) -> return code; ks and vs are lists or tuples of equal length
 * whose tensors have the same number of rows (ValueError otherwise) */
static PyObject *py_store_all(PyObject *self, PyObject *const *v, Py_ssize_t nargs)
{
    (void)self;
    if (want_args(nargs, 6)) return NULL;
    void *cache, *stream;
    int32_t group, mode, n = 0;
    if (handle_arg(v[0], &cache) || int_arg(v[1], &group) || int_arg(v[4], &mode) || handle_arg(v[5], &stream)) return NULL;
    PyObject *ks = PySequence_Fast(v[2], "one K tensor per layer");
    PyObject *vs = ks ? PySequence_Fast(v[3], "one V tensor per layer") : NULL;
    PyObject *ret = NULL;
    const void **ptrs = NULL;
    if (!vs) goto done;
    const Py_ssize_t L = PySequence_Fast_GET_SIZE(ks);
    if (L < 1 || PySequence_Fast_GET_SIZE(vs) != L) {
        PyErr_SetString(PyExc_ValueError, "one K and one V tensor per layer of the cache");
        goto done;
    }
    ptrs = PyMem_Malloc(2 * (size_t)L * sizeof *ptrs);
    if (!ptrs) { PyErr_NoMemory(); goto done; }
    for (int kv = 0; kv < 2; ++kv)
        for (Py_ssize_t l = 0; l < L; ++l) {
            PyObject *t = PySequence_Fast_GET_ITEM(kv ? vs : ks, l);
            int32_t rows;
            void *p;
            if (first_dim(t, &rows) || tensor_ptr(t, &p)) goto done;
            if (kv == 0 && l == 0) n = rows;
            if (rows != n) {
                PyErr_SetString(PyExc_ValueError, "every layer must bring the same number of rows");
                goto done;
            }
            ptrs[kv * L + l] = p;
        }
    {
        int rc;
        Py_BEGIN_ALLOW_THREADS
        rc = enl_group_store_all_layers((enl_cache_t *)cache, group, n, ptrs, ptrs + L, mode, stream);
        Py_END_ALLOW_THREADS
        ret = PyLong_FromLong(rc);
    }
done:
    PyMem_Free((void *)ptrs);
    Py_XDECREF(ks);
    Py_XDECREF(vs);
    return ret;
}

/* What a tensor is made of, as the DLPack exchange interface of torch 2.10 and later tells it without a call into Python: five method calls
 * a tensor are 0.3 us, 48 us of an append over 40 layers.  (Declared here as far as it is used: the interface is a fixed binary one, versions 1.x.) */
typedef struct {
    void *data;
    struct { int32_t type, id; } device;
    int32_t ndim;
    struct { uint8_t code, bits; uint16_t lanes; } dtype;
    int64_t *shape, *strides;
    uint64_t byte_offset;
} view_t;
typedef struct {
    struct { uint32_t major, minor; void *older; } header;
    void *allocate, *to_managed, *from_managed;
    int (*view)(void *tensor, view_t *out);
} exchange_t;
enum { kCuda = 2, kInt = 0, kBfloat = 4 };
static PyTypeObject *t_tensor;                              /* torch.Tensor, whose exchange interface this is: */
static const exchange_t *exchange;                          /* NULL: the methods are asked */

/* A tensor whose type, number of dimensions, layout and device are checked (the lengths of these calls are device values: nothing behind the
 * binding could tell a tensor of another shape).  `dims` receives its shape; the first tensor of a call sets *device.  ValueError. */
static int checked(PyObject *t, const char *name, PyObject *dtype, int ndim, int64_t *dims, void **ptr, long *device, int optional)
{
    *ptr = NULL;
    if (t == Py_None) {
        if (optional) return 0;
        PyErr_Format(PyExc_ValueError, "%s is missing", name);
        return -1;
    }
    view_t w;
    if (exchange && Py_TYPE(t) == t_tensor && exchange->view(t, &w) == 0) {
        int fine = w.device.type == kCuda && (*device == -2 || w.device.id == *device) && w.ndim == ndim && w.dtype.lanes == 1 &&
                   (dtype == t_bf16 ? w.dtype.code == kBfloat && w.dtype.bits == 16 : w.dtype.code == kInt && w.dtype.bits == (dtype == t_int32 ? 32 : 64));
        int64_t step = 1;
        for (int i = ndim - 1; fine && i >= 0; --i) {
            fine = w.shape[i] > 0 && (w.shape[i] == 1 || w.strides[i] == step);
            step *= w.shape[i];
            dims[i] = w.shape[i];
        }
        if (fine) {
            *device = w.device.id;
            *ptr = (char *)w.data + w.byte_offset;
            return 0;
        }                                                   /* else what is wrong is said below */
    }
    PyErr_Clear();
    PyObject *v = PyObject_GetAttr(t, s_dtype);
    if (!v) return -1;
    Py_DECREF(v);                                           /* torch keeps its dtypes */
    if (v != dtype) {
        PyErr_Format(PyExc_ValueError, "%s has to be %S, not %S", name, dtype, v);
        return -1;
    }
    if (!(v = PyObject_GetAttr(t, s_shape))) return -1;
    if (!PyTuple_Check(v) || PyTuple_GET_SIZE(v) != ndim) {
        PyErr_Format(PyExc_ValueError, "%s has to have %d dimensions", name, ndim);
        Py_DECREF(v);
        return -1;
    }
    for (int i = 0; i < ndim; ++i) dims[i] = PyLong_AsLongLong(PyTuple_GET_ITEM(v, i));
    Py_DECREF(v);
    if (!(v = PyObject_CallMethodNoArgs(t, s_contiguous))) return -1;
    const int flat = v == Py_True;
    Py_DECREF(v);
    if (!flat) {
        PyErr_Format(PyExc_ValueError, "%s has to be contiguous", name);
        return -1;
    }
    if (!(v = PyObject_CallMethodNoArgs(t, s_get_device))) return -1;
    const long at = PyLong_AsLong(v);
    Py_DECREF(v);
    if (*device == -2) *device = at;
    if (at < 0 || at != *device) {
        PyErr_Format(PyExc_ValueError, at < 0 ? "%s has to be a CUDA tensor" : "%s is on another device", name);
        return -1;
    }
    return tensor_ptr(t, ptr);
}
static int same(const char *what, int64_t a, int64_t b)
{
    if (a == b) return 0;
    PyErr_Format(PyExc_ValueError, "%s: %lld where %lld is expected", what, (long long)a, (long long)b);
    return -1;
}
static int small(const char *what, int64_t a)
{
    if (a <= 0x7fffffff) return 0;
    PyErr_Format(PyExc_ValueError, "%s is too large", what);
    return -1;
}
/* an int32 array of a value per request, or of a value per row */
static int per_request(PyObject *t, const char *name, int64_t batch, void **ptr, long *device, int optional)
{
    int64_t d[1] = {batch};
    return checked(t, name, t_int32, 1, d, ptr, device, optional) || (*ptr && same(name, d[0], batch)) ? -1 : 0;
}
static int per_row(PyObject *t, const char *name, PyObject *dtype, int64_t batch, int64_t n_max, void **ptr, long *device, int optional)
{
    int64_t d[2] = {batch, n_max};
    return checked(t, name, dtype, 2, d, ptr, device, optional) || (*ptr && (same(name, d[0], batch) || same(name, d[1], n_max))) ? -1 : 0;
}

/* tail_tables(device, tail_len, block_table, n_blocks, free_pages, n_free, slot, position, mask, n_new, parent, pos_base, failed, stream) -> return code */
static PyObject *py_tail_tables(PyObject *self, PyObject *const *v, Py_ssize_t nargs)
{
    (void)self;
    if (want_args(nargs, 14)) return NULL;
    enl_tail_tables_args_t a;
    memset(&a, 0, sizeof a);
    int64_t tab[2] = {0, 0}, rows[2] = {0, 0}, free_n[1] = {0}, one[1] = {0};
    long dev = PyLong_AsLong(v[0]);
    void *p, *stream;
    if (checked(v[6], "slots", t_int32, 2, rows, &p, &dev, 0)) return NULL;
    a.slot = p;
    const int64_t B = rows[0], N = rows[1];
    if (per_request(v[1], "tail_len", B, &p, &dev, 0)) return NULL;
    a.tail_len = p;
    if (checked(v[2], "block_table", t_int32, 2, tab, &p, &dev, 0) || same("block_table", tab[0], B)) return NULL;
    a.block_table = p;
    if (per_request(v[3], "n_blocks", B, &p, &dev, 0)) return NULL;
    a.n_blocks = p;
    if (checked(v[4], "free_pages", t_int32, 1, free_n, &p, &dev, 0)) return NULL;
    a.free_pages = p;
    if (checked(v[5], "n_free", t_int32, 1, one, &p, &dev, 0) || same("n_free", one[0], 1)) return NULL;
    a.n_free = p;
    if (per_row(v[7], "positions", t_int32, B, N, &p, &dev, 1)) return NULL;
    a.position = p;
    if (per_row(v[8], "mask", t_int64, B, N, &p, &dev, 1)) return NULL;
    a.mask = p;
    if (per_request(v[9], "n_new", B, &p, &dev, 1)) return NULL;
    a.n_new = p;
    if (per_row(v[10], "parent", t_int32, B, N, &p, &dev, 1)) return NULL;
    a.parent = p;
    if (per_request(v[11], "pos_base", B, &p, &dev, 1)) return NULL;
    a.pos_base = p;
    if (per_request(v[12], "failed", 1, &p, &dev, 1)) return NULL;
    a.failed = p;
    if (handle_arg(v[13], &stream) || small("slots", B * N) || small("block_table", tab[1]) || small("free_pages", free_n[0])) return NULL;
    a.batch = (int32_t)B;
    a.n_max = (int32_t)N;
    a.max_blocks = (int32_t)tab[1];
    a.n_pages = (int32_t)free_n[0];
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = enl_tail_tables(&a, stream);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(rc);
}

/* attend_tree(device, cache, layer, sel_ids, q, k_new, v_new, k_tail, v_tail, block_table, tail_len, out, n_new, mask, cu_sel, n_q_heads, n_kv_heads,
 * head_dim, stream) -> return code */
static PyObject *py_attend_tree(PyObject *self, PyObject *const *v, Py_ssize_t nargs)
{
    (void)self;
    if (want_args(nargs, 19)) return NULL;
    enl_attend_tree_args_t a;
    memset(&a, 0, sizeof a);
    ints_t sel, cs;
    sel.held = cs.held = 0;
    int64_t q[4], t[4], tab[2];
    long dev = PyLong_AsLong(v[0]);
    int32_t Hq, Hkv, D;
    void *cache, *p, *stream;
    PyObject *ret = NULL;
    if (handle_arg(v[1], &cache) || int_arg(v[2], &a.layer) || int_arg(v[15], &Hq) || int_arg(v[16], &Hkv) || int_arg(v[17], &D)) return NULL;
    if (checked(v[4], "q", t_bf16, 4, q, &p, &dev, 0) || same("q heads", q[2], Hq) || same("q channels", q[3], D)) return NULL;
    a.q = p;
    for (int i = 0; i < 2; ++i) {
        const char *name = i ? "v_new" : "k_new";
        if (checked(v[5 + i], name, t_bf16, 4, t, &p, &dev, 0) || same(name, t[0], q[0]) || same(name, t[1], q[1]) || same(name, t[2], Hkv) ||
            same(name, t[3], D))
            return NULL;
        if (i) a.v_new = p; else a.k_new = p;
    }
    int64_t pages = 0;
    for (int i = 0; i < 2; ++i) {
        const char *name = i ? "v_tail" : "k_tail";
        if (checked(v[7 + i], name, t_bf16, 4, t, &p, &dev, 0) || same(name, t[1], Hkv) || same(name, t[2], 16) || same(name, t[3], D) ||
            (i && same(name, t[0], pages)))
            return NULL;
        pages = t[0];
        if (i) a.v_tail = p; else a.k_tail = p;
    }
    if (checked(v[9], "block_table", t_int32, 2, tab, &p, &dev, 0) || same("block_table", tab[0], q[0])) return NULL;
    a.block_table = p;
    if (per_request(v[10], "tail_len", q[0], &p, &dev, 0)) return NULL;
    a.tail_len = p;
    if (checked(v[11], "out", t_bf16, 4, t, &p, &dev, 0) || same("out", t[0], q[0]) || same("out", t[1], q[1]) || same("out", t[2], Hq) || same("out", t[3], D))
        return NULL;
    a.out = p;
    if (per_request(v[12], "n_new", q[0], &p, &dev, 1)) return NULL;
    a.n_new = p;
    if (per_row(v[13], "mask", t_int64, q[0], q[1], &p, &dev, 1)) return NULL;
    a.mask = p;
    if (handle_arg(v[18], &stream) || small("q", q[0] * q[1]) || small("block_table", tab[1]) || small("k_tail", pages)) return NULL;
    a.batch = (int32_t)q[0];
    a.n_max = (int32_t)q[1];
    a.max_blocks = (int32_t)tab[1];
    a.n_pages = (int32_t)pages;
    if (ints_get(v[3], &sel) || ints_get(v[14], &cs)) goto done;
    if (v[14] != Py_None && same("cu_sel", cs.n, q[0] + 1)) goto done;
    a.sel_ids = sel.p;
    a.n_sel = (int32_t)sel.n;
    a.cu_sel = cs.p;
    {
        int rc;
        Py_BEGIN_ALLOW_THREADS
        rc = enl_attend_tree((enl_cache_t *)cache, &a, stream);
        Py_END_ALLOW_THREADS
        ret = PyLong_FromLong(rc);
    }
done:
    ints_free(&sel);
    ints_free(&cs);
    return ret;
}

/* tree_accept(device, parent, token, target, accept, n_accept, next_token, n_new, first, stream) -> return code */
static PyObject *py_tree_accept(PyObject *self, PyObject *const *v, Py_ssize_t nargs)
{
    (void)self;
    if (want_args(nargs, 10)) return NULL;
    enl_tree_accept_args_t a;
    memset(&a, 0, sizeof a);
    int64_t rows[2];
    long dev = PyLong_AsLong(v[0]);
    void *p, *stream;
    if (checked(v[2], "token", t_int32, 2, rows, &p, &dev, 0)) return NULL;
    a.token = p;
    const int64_t B = rows[0], N = rows[1];
    if (per_row(v[1], "parent", t_int32, B, N, &p, &dev, 1)) return NULL;
    a.parent = p;
    if (per_row(v[3], "target", t_int32, B, N, &p, &dev, 0)) return NULL;
    a.target = p;
    if (per_row(v[4], "accept", t_int32, B, N, &p, &dev, 0)) return NULL;
    a.accept = p;
    if (per_request(v[5], "n_accept", B, &p, &dev, 0)) return NULL;
    a.n_accept = p;
    if (per_request(v[6], "next_token", B, &p, &dev, 0)) return NULL;
    a.next = p;
    if (per_request(v[7], "n_new", B, &p, &dev, 1)) return NULL;
    a.n_new = p;
    if (per_request(v[8], "first", B, &p, &dev, 1)) return NULL;
    a.first = p;
    if (handle_arg(v[9], &stream) || small("token", B * N)) return NULL;
    a.batch = (int32_t)B;
    a.n_max = (int32_t)N;
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = enl_tree_accept(&a, stream);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(rc);
}

/* tail_append(device, ks, vs, k_tails, v_tails, slot, tail_len, tail_len_out, accept, n_accept, stream) -> return code; the first four are lists or tuples
 * of a tensor per layer */
static PyObject *py_tail_append(PyObject *self, PyObject *const *v, Py_ssize_t nargs)
{
    (void)self;
    if (want_args(nargs, 11)) return NULL;
    enl_tail_append_args_t a;
    memset(&a, 0, sizeof a);
    int64_t rows[2], t[4];
    long dev = PyLong_AsLong(v[0]);
    void *p, *stream;
    if (checked(v[5], "slots", t_int32, 2, rows, &p, &dev, 0)) return NULL;
    a.slot = p;
    const int64_t B = rows[0], N = rows[1];
    if (per_request(v[6], "tail_len", B, &p, &dev, 0)) return NULL;
    a.tail_len = p;
    if (per_request(v[7], "tail_len_out", B, &p, &dev, 0)) return NULL;
    a.tail_len_out = p;
    if (per_row(v[8], "accept", t_int32, B, N, &p, &dev, 1)) return NULL;
    a.accept = p;
    if (per_request(v[9], "n_accept", B, &p, &dev, 1)) return NULL;
    a.n_accept = p;
    if (handle_arg(v[10], &stream) || small("slots", B * N)) return NULL;
    static const char *const names[4] = {"ks", "vs", "k_tails", "v_tails"};
    PyObject *seq[4] = {NULL, NULL, NULL, NULL}, *ret = NULL;
    void **ptrs = NULL;
    Py_ssize_t L = 0;
    int64_t heads = 0, dim = 0, pages = 0;
    for (int k = 0; k < 4; ++k) {
        if (!(seq[k] = PySequence_Fast(v[1 + k], "one tensor per layer"))) goto done;
        if (k == 0) {
            L = PySequence_Fast_GET_SIZE(seq[0]);
            if (L < 1 || L > 65535) { PyErr_SetString(PyExc_ValueError, "ks: one tensor per layer"); goto done; }
            if (!(ptrs = PyMem_Malloc(4 * (size_t)L * sizeof *ptrs))) { PyErr_NoMemory(); goto done; }
        }
        if (same(names[k], PySequence_Fast_GET_SIZE(seq[k]), L)) goto done;
        for (Py_ssize_t l = 0; l < L; ++l) {
            if (checked(PySequence_Fast_GET_ITEM(seq[k], l), names[k], t_bf16, 4, t, &ptrs[k * L + l], &dev, 0)) goto done;
            if (k < 2) {
                if (k == 0 && l == 0) { heads = t[2]; dim = t[3]; }
                if (same(names[k], t[0], B) || same(names[k], t[1], N) || same(names[k], t[2], heads) || same(names[k], t[3], dim)) goto done;
            } else {
                if (k == 2 && l == 0) pages = t[0];
                if (same(names[k], t[0], pages) || same(names[k], t[1], heads) || same(names[k], t[2], 16) || same(names[k], t[3], dim)) goto done;
            }
        }
    }
    if (small("heads", heads) || small("channels", dim) || small("pages", pages)) goto done;
    a.n_layers = (int32_t)L;
    a.batch = (int32_t)B;
    a.n_max = (int32_t)N;
    a.n_kv_heads = (int32_t)heads;
    a.head_dim = (int32_t)dim;
    a.n_pages = (int32_t)pages;
    a.k_new = (const void *const *)ptrs;
    a.v_new = (const void *const *)(ptrs + L);
    a.k_tail = ptrs + 2 * L;
    a.v_tail = ptrs + 3 * L;
    {
        int rc;
        Py_BEGIN_ALLOW_THREADS
        rc = enl_tail_append(&a, stream);
        Py_END_ALLOW_THREADS
        ret = PyLong_FromLong(rc);
    }
done:
    PyMem_Free(ptrs);
    for (int k = 0; k < 4; ++k) Py_XDECREF(seq[k]);
    return ret;
}

/* set_types(bfloat16, int32, int64, Tensor, exchange): torch's; exchange: the capsule of Tensor's DLPack exchange interface, or None */
static PyObject *py_set_types(PyObject *self, PyObject *const *v, Py_ssize_t nargs)
{
    (void)self;
    if (want_args(nargs, 5)) return NULL;
    if (!PyType_Check(v[3])) { PyErr_SetString(PyExc_TypeError, "the tensor type"); return NULL; }
    for (int i = 0; i < 4; ++i) Py_INCREF(v[i]);
    if (PyCapsule_IsValid(v[4], "dlpack_exchange_api")) {
        exchange = PyCapsule_GetPointer(v[4], "dlpack_exchange_api");
        if (exchange && (exchange->header.major != 1 || !exchange->view)) exchange = NULL;
    }
    Py_XSETREF(t_tensor, (PyTypeObject *)v[3]);
    Py_XSETREF(t_bf16, v[0]);
    Py_XSETREF(t_int32, v[1]);
    Py_XSETREF(t_int64, v[2]);
    Py_RETURN_NONE;
}

/* set_int32_converter(f): f(sequence) -> contiguous int32 array */
static PyObject *py_set_converter(PyObject *self, PyObject *f)
{
    (void)self;
    Py_INCREF(f);
    Py_XSETREF(to_int32, f);
    Py_RETURN_NONE;
}

static PyMethodDef methods[] = {
    {"attend", (PyCFunction)(void (*)(void))py_attend, METH_FASTCALL, NULL},
    {"attend_static", (PyCFunction)(void (*)(void))py_attend_static, METH_FASTCALL, NULL},
    {"store", (PyCFunction)(void (*)(void))py_store, METH_FASTCALL, NULL},
    {"store_all_layers", (PyCFunction)(void (*)(void))py_store_all, METH_FASTCALL, NULL},
    {"tail_tables", (PyCFunction)(void (*)(void))py_tail_tables, METH_FASTCALL, NULL},
    {"attend_tree", (PyCFunction)(void (*)(void))py_attend_tree, METH_FASTCALL, NULL},
    {"tree_accept", (PyCFunction)(void (*)(void))py_tree_accept, METH_FASTCALL, NULL},
    {"tail_append", (PyCFunction)(void (*)(void))py_tail_append, METH_FASTCALL, NULL},
    {"set_types", (PyCFunction)(void (*)(void))py_set_types, METH_FASTCALL, NULL},
    {"set_int32_converter", py_set_converter, METH_O, NULL},
    {NULL, NULL, 0, NULL},
};
static struct PyModuleDef module = {PyModuleDef_HEAD_INIT, "_enl", NULL, -1, methods, NULL, NULL, NULL, NULL};

PyMODINIT_FUNC PyInit__enl(void)
{
    s_data_ptr = PyUnicode_InternFromString("data_ptr");
    s_shape = PyUnicode_InternFromString("shape");
    s_dtype = PyUnicode_InternFromString("dtype");
    s_contiguous = PyUnicode_InternFromString("is_contiguous");
    s_get_device = PyUnicode_InternFromString("get_device");
    if (!s_data_ptr || !s_shape || !s_dtype || !s_contiguous || !s_get_device) return NULL;
    return PyModule_Create(&module);
}
