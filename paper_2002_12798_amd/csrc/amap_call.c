/* The way from a Python call to the library: tensors and integers in, one call of a C entry point, its status out.
 *
 * A call on tensors of some hundred kilobytes is bound by issuing it: through the interpreter and ctypes (a table of addresses built,
 * four arguments converted) that was 1.0 us of 4.4 to 5.3, here 0.3; the launch itself is 3.3 to 3.9.  Only the ordinary call is taken:
 * maps whose sources are known, lists or tuples of things with a data_ptr(), integers that fit.  Whatever else comes is answered
 * with NOT_TAKEN before the library has seen it, and goes the way through ctypes, which raises what there is to raise.  Nothing is kept
 * between calls but the addresses of the entry points and torch's functions. */
#define PY_SSIZE_T_CLEAN
#include <Python.h>
#include <math.h>
#include <pthread.h>
#include <stdint.h>
#include <string.h>

#include "amap.h"

enum { NOT_TAKEN = -1, MAX_TABLE = 16 };

typedef int (*execute_fn)(void *const *, void *, void *, void *);
typedef int (*multi_fn)(void *const *, void *const *, void *const *, int, void *);
typedef int (*fused_fn)(void *, void *, void *, int64_t, void *, void *);
typedef int (*store_fn)(void *, void *, void *, int64_t, void *, void *, void *);
typedef int (*mapped_fn)(void *, void *, void *, void *, void *, void *, void *);
typedef int (*gather_fn)(void *const *, void *, void *, void *, int64_t, void *, void *, void *);

static execute_fn p_execute;
static multi_fn p_multi;
static fused_fn p_fused;
static store_fn p_store;
static mapped_fn p_mapped;
static gather_fn p_gather;
static PyObject *raw_stream, *get_device, *is_initialized;   /* torch's; NULL: no current stream from here */
static PyObject *s_data_ptr, *s_at, *s_reads;
static int initialized;   /* torch said so in this process (a fork asks again) */

static void forked(void) { initialized = 0; }

/* Each of these is 1, or 0 for a call that is not taken.  An error is the other way's to raise again and is cleared; one that ends the
 * program (an interrupt, an exit: no Exception) stays, and the call returns with it. */

static int not_taken(void)
{
    if (PyErr_Occurred() && PyErr_ExceptionMatches(PyExc_Exception)) PyErr_Clear();
    return 0;
}

static int address(PyObject *o, void **at)
{
    if (o == Py_None) {
        *at = NULL;
        return 1;
    }
    if (!PyLong_CheckExact(o)) return 0;
    *at = PyLong_AsVoidPtr(o);
    return *at || !PyErr_Occurred() || not_taken();
}

static int integer(PyObject *o, void **at) { return o != Py_None && address(o, at); }

static int data_of(PyObject *tensor, void **at)
{
    PyObject *p = PyObject_CallMethodNoArgs(tensor, s_data_ptr);
    if (!p) return not_taken();
    const int ok = integer(p, at);
    Py_DECREF(p);
    return ok;
}

/* a source, which a map may not need; an output is always there */
static int source_of(PyObject *tensor, void **at)
{
    if (tensor != Py_None) return data_of(tensor, at);
    *at = NULL;
    return 1;
}

/* a map: the library's, how long a source table it expects and the last source that it reads (-1: none) */
static int map_of(PyObject *m, void **map, Py_ssize_t *n_src, Py_ssize_t *last)
{
    PyObject *at = PyObject_GetAttr(m, s_at), *reads = at ? PyObject_GetAttr(m, s_reads) : NULL;
    int ok = 0;
    if (reads && integer(at, map) && *map && PyTuple_CheckExact(reads) && PyTuple_GET_SIZE(reads) == 2 && PyTuple_CheckExact(PyTuple_GET_ITEM(reads, 1))) {
        PyObject *ids = PyTuple_GET_ITEM(reads, 1);
        const Py_ssize_t n = PyTuple_GET_SIZE(ids);
        *n_src = PyLong_AsSsize_t(PyTuple_GET_ITEM(reads, 0));
        *last = n ? PyLong_AsSsize_t(PyTuple_GET_ITEM(ids, n - 1)) : -1;
        ok = *n_src >= 0;
    }
    if (PyErr_Occurred()) ok = not_taken();
    Py_XDECREF(at);
    Py_XDECREF(reads);
    return ok;
}

/* what an object's attribute of this name says is the library's; None: NULL */
static int named_handle_of(PyObject *o, PyObject *name, void **at)
{
    if (o == Py_None) {
        *at = NULL;
        return 1;
    }
    PyObject *x = PyObject_GetAttr(o, name);
    const int ok = (x && integer(x, at) && *at) || not_taken();
    Py_XDECREF(x);
    return ok;
}

/* a map whose sources are not asked for */
static int handle_of(PyObject *m, void **map) { return named_handle_of(m, s_at, map); }

static int table(PyObject *list, void **tab, Py_ssize_t *given, int (*of)(PyObject *, void **))
{
    if (!PyList_CheckExact(list) && !PyTuple_CheckExact(list)) return 0;
    const Py_ssize_t n = PySequence_Fast_GET_SIZE(list);
    if (n > MAX_TABLE) return 0;
    for (Py_ssize_t i = 0; i < MAX_TABLE; ++i) tab[i] = NULL;
    for (Py_ssize_t i = 0; i < n; ++i) {
        if (i >= PySequence_Fast_GET_SIZE(list)) return 0;   /* (a data_ptr() may run anything) */
        PyObject *o = PySequence_Fast_GET_ITEM(list, i);
        Py_INCREF(o);
        const int ok = of(o, &tab[i]);
        Py_DECREF(o);
        if (!ok) return 0;
    }
    *given = n;
    return 1;
}

static int stream_of(PyObject *o, void **stream)
{
    if (o != Py_None) return address(o, stream);
    if (!raw_stream) return 0;
    PyObject *r;
    if (!initialized) {
        r = PyObject_CallNoArgs(is_initialized);
        initialized = r ? PyObject_IsTrue(r) == 1 : 0;
        Py_XDECREF(r);
        if (!initialized) return not_taken();
    }
    PyObject *dev = PyObject_CallNoArgs(get_device);
    r = dev ? PyObject_CallOneArg(raw_stream, dev) : NULL;
    const int ok = (r && integer(r, stream)) || not_taken();
    Py_XDECREF(dev);
    Py_XDECREF(r);
    return ok;
}

#define CALLED(expr)                \
    do {                            \
        int status_;                \
        Py_BEGIN_ALLOW_THREADS      \
        status_ = (expr);           \
        Py_END_ALLOW_THREADS        \
        return PyLong_FromLong(status_); \
    } while (0)
#define UNLESS(x) \
    if (!(x)) return PyErr_Occurred() ? NULL : PyLong_FromLong(NOT_TAKEN)

/* execute(map, tensors, tensor, stream or None) */
static PyObject *call_execute(PyObject *self, PyObject *const *a, Py_ssize_t n)
{
    void *tab[MAX_TABLE], *dst, *map, *stream;
    Py_ssize_t given, n_src, last;
    (void)self;
    UNLESS(p_execute && n == 4 && map_of(a[0], &map, &n_src, &last) && table(a[1], tab, &given, source_of));
    UNLESS(last < given && n_src <= MAX_TABLE && data_of(a[2], &dst) && stream_of(a[3], &stream));
    CALLED(p_execute(tab, dst, map, stream));
}

/* execute_multi(maps, tensors, tensors, stream or None) */
static PyObject *call_execute_multi(PyObject *self, PyObject *const *a, Py_ssize_t n)
{
    void *tab[MAX_TABLE], *dst[MAX_TABLE], *maps[MAX_TABLE], *stream;
    Py_ssize_t given, n_dst, n_maps, n_src, last;
    (void)self;
    UNLESS(p_multi && n == 4 && (PyList_CheckExact(a[0]) || PyTuple_CheckExact(a[0])) && table(a[1], tab, &given, source_of) && table(a[2], dst, &n_dst, data_of));
    n_maps = PySequence_Fast_GET_SIZE(a[0]);
    UNLESS(n_maps >= 1 && n_maps <= n_dst);
    for (Py_ssize_t i = 0; i < n_maps; ++i) {
        UNLESS(i < PySequence_Fast_GET_SIZE(a[0]));
        PyObject *m = PySequence_Fast_GET_ITEM(a[0], i);
        Py_INCREF(m);   /* (asking it for its attributes may take it out of the list) */
        const int ok = map_of(m, &maps[i], &n_src, &last);
        Py_DECREF(m);
        UNLESS(ok && last < given && n_src <= MAX_TABLE);
    }
    UNLESS(stream_of(a[3], &stream));
    CALLED(p_multi(tab, dst, maps, (int)n_maps, stream));
}

static int count_of(PyObject *o, int64_t *n)
{
    if (!PyLong_CheckExact(o)) return 0;
    *n = PyLong_AsLongLong(o);
    return *n != -1 || !PyErr_Occurred() || not_taken();
}

/* gemm(address of A, map, address of W, map or None, n, store map or None, address of the product, stream) */
static PyObject *call_gemm(PyObject *self, PyObject *const *a, Py_ssize_t n)
{
    void *src, *a_map, *w, *w_map, *out_map, *out, *stream;
    int64_t cols;
    (void)self;
    UNLESS(p_fused && n == 8 && integer(a[0], &src) && a[1] != Py_None && handle_of(a[1], &a_map) && integer(a[2], &w) && handle_of(a[3], &w_map) &&
           count_of(a[4], &cols) && handle_of(a[5], &out_map) && integer(a[6], &out) && integer(a[7], &stream));
    if (w_map) CALLED(p_mapped(src, a_map, w, w_map, out_map, out, stream));
    if (out_map) CALLED(p_store(src, a_map, w, cols, out_map, out, stream));
    CALLED(p_fused(src, a_map, w, cols, out, stream));
}

/* gather(addresses, map, address of W, map or None, n, store map or None, address of the product, stream) */
static PyObject *call_gather(PyObject *self, PyObject *const *a, Py_ssize_t n)
{
    void *tab[MAX_TABLE], *a_map, *w, *w_map, *out_map, *out, *stream;
    Py_ssize_t given, n_src, last;
    int64_t cols;
    (void)self;
    UNLESS(p_gather && n == 8 && table(a[0], tab, &given, address) && map_of(a[1], &a_map, &n_src, &last) && n_src <= MAX_TABLE && integer(a[2], &w) &&
           handle_of(a[3], &w_map) && count_of(a[4], &cols) && handle_of(a[5], &out_map) && integer(a[6], &out) && integer(a[7], &stream));
    CALLED(p_gather(tab, a_map, w, w_map, cols, out_map, out, stream));
}

/* the current stream's handle, or None where torch has to be asked in full */
static PyObject *call_current_stream(PyObject *self, PyObject *none)
{
    void *stream;
    (void)self;
    (void)none;
    if (!stream_of(Py_None, &stream)) {
        if (PyErr_Occurred()) return NULL;
        Py_RETURN_NONE;
    }
    return PyLong_FromVoidPtr(stream);
}

/* library(addresses of amap_execute, _execute_multi, _gemm_fused, _gemm_fused_store, _gemm_mapped, _gemm_gather) */
static PyObject *call_library(PyObject *self, PyObject *const *a, Py_ssize_t n)
{
    void *p[6];
    (void)self;
    for (Py_ssize_t i = 0; i < 6; ++i)
        if (n != 6 || !integer(a[i], &p[i])) {
            PyErr_SetString(PyExc_TypeError, "six addresses");
            return NULL;
        }
    p_execute = (execute_fn)(uintptr_t)p[0];
    p_multi = (multi_fn)(uintptr_t)p[1];
    p_fused = (fused_fn)(uintptr_t)p[2];
    p_store = (store_fn)(uintptr_t)p[3];
    p_mapped = (mapped_fn)(uintptr_t)p[4];
    p_gather = (gather_fn)(uintptr_t)p[5];
    Py_RETURN_NONE;
}

/* torch(stream handle of a device, current device, whether CUDA is initialised) */
static PyObject *call_torch(PyObject *self, PyObject *const *a, Py_ssize_t n)
{
    (void)self;
    if (n != 3) {
        PyErr_SetString(PyExc_TypeError, "three functions");
        return NULL;
    }
    Py_INCREF(a[0]);
    Py_INCREF(a[1]);
    Py_INCREF(a[2]);
    Py_XSETREF(raw_stream, a[0]);
    Py_XSETREF(get_device, a[1]);
    Py_XSETREF(is_initialized, a[2]);
    initialized = 0;
    Py_RETURN_NONE;
}

/* ---- the calls around the paged cache: tensors with their shapes and strides ---------------------------------------------- */

typedef amap_status (*assign_fn)(const amap_assign *, void *);
typedef amap_status (*rotary_fn)(const amap_heads *, const amap_heads *, int64_t, int, const amap_rope *, const int32_t *, int64_t, int, void *);
typedef amap_status (*append_fn)(const amap_cache *, const amap_heads *, const amap_heads *, int64_t, const int64_t *, const amap_rope *, const int32_t *, int64_t,
                                 const amap_heads *, const amap_heads *, void *);
typedef amap_status (*attend_fn)(const amap_cache *, const amap_heads *, int64_t, const int32_t *, int64_t, int, const int32_t *, float, int, const amap_heads *, float *,
                                 void *, int64_t, void *);
typedef amap_status (*room_fn)(const amap_cache *, int, int64_t, int, int64_t *);
static assign_fn p_assign;
static rotary_fn p_rotary;
static append_fn p_append;
static attend_fn p_attend;
static room_fn p_room;

/* torch's types, each one object: those of rows of heads with the library's name for them, and those of whole numbers */
enum { MAX_TYPES = 8 };
static PyObject *row_type[MAX_TYPES], *t_int32, *t_int64, *t_float32, *t_uint8;
static int row_code[MAX_TYPES], n_row_types;
static PyObject *s_shape, *s_stride, *s_dtype, *s_is_cuda, *s_cache_at, *s_rope_at;   /* (a map is neither a cache nor a rope) */

typedef struct {
    void *data;
    PyObject *dtype;   /* borrowed: torch keeps its types */
    int rank;
    int64_t size[4], stride[4];
} tensor_t;

static int whole_numbers(PyObject *tuple, int64_t *v, int *n)
{
    if (!tuple || !PyTuple_Check(tuple) || PyTuple_GET_SIZE(tuple) > 4) return 0;
    *n = (int)PyTuple_GET_SIZE(tuple);
    for (int i = 0; i < *n; ++i) {
        v[i] = PyLong_AsLongLong(PyTuple_GET_ITEM(tuple, i));
        if (v[i] == -1 && PyErr_Occurred()) return 0;
    }
    return 1;
}

/* a tensor on the GPU of this rank, its last dimension contiguous */
static int tensor_of(PyObject *o, int rank, tensor_t *t)
{
    PyObject *shape = NULL, *stride = NULL, *dtype = NULL, *on_gpu = NULL;
    int n = 0, ok = 0;
    if ((on_gpu = PyObject_GetAttr(o, s_is_cuda)) && on_gpu == Py_True && (dtype = PyObject_GetAttr(o, s_dtype)) && (shape = PyObject_GetAttr(o, s_shape)) &&
        (stride = PyObject_CallMethodNoArgs(o, s_stride)))
        ok = whole_numbers(shape, t->size, &t->rank) && whole_numbers(stride, t->stride, &n) && n == t->rank && n == rank &&
             (n == 0 || t->size[n - 1] <= 1 || t->stride[n - 1] == 1) && data_of(o, &t->data);
    if (PyErr_Occurred()) ok = not_taken();
    t->dtype = dtype;
    Py_XDECREF(on_gpu);
    Py_XDECREF(dtype);
    Py_XDECREF(shape);
    Py_XDECREF(stride);
    return ok;
}

static int of_type(PyObject *o, int rank, PyObject *dtype, tensor_t *t) { return tensor_of(o, rank, t) && t->dtype == dtype; }

/* [tokens, heads, head_dim] */
static int rows_of(PyObject *o, tensor_t *t, amap_heads *h)
{
    if (!tensor_of(o, 3, t) || t->size[1] > INT32_MAX || t->size[2] > INT32_MAX) return 0;
    for (int i = 0; i < n_row_types; ++i)
        if (row_type[i] == t->dtype) {
            h->data = t->data;
            h->type = (amap_type)row_code[i];
            h->heads = (int)t->size[1];
            h->token_stride = t->stride[0];
            h->head_stride = t->stride[1];
            return 1;
        }
    return 0;
}
static int same_shape(const tensor_t *a, const tensor_t *b) { return a->rank == b->rank && !memcmp(a->size, b->size, sizeof(int64_t) * (size_t)a->rank); }

/* positions of so many tokens for a rope's axes: [tokens], the same for all, or [axes, tokens] */
static int positions_of(PyObject *o, const amap_rope *rope, int64_t tokens, tensor_t *t, int64_t *step)
{
    if (of_type(o, 1, t_int32, t)) {
        *step = 0;
        return t->size[0] == tokens;
    }
    if (PyErr_Occurred() || !of_type(o, 2, t_int32, t)) return 0;
    *step = t->stride[0];
    return t->size[0] == rope->n_axes && t->size[1] == tokens;
}

/* rotary(x, rope, positions, out, inverse, stream or None) */
static PyObject *call_rotary(PyObject *self, PyObject *const *a, Py_ssize_t n)
{
    tensor_t tx, ty, tp;
    amap_heads x, y;
    void *rope, *stream;
    int64_t step;
    (void)self;
    UNLESS(p_rotary && n == 6 && a[1] != Py_None && named_handle_of(a[1], s_rope_at, &rope) && rows_of(a[0], &tx, &x) && rows_of(a[3], &ty, &y) && same_shape(&tx, &ty) &&
           positions_of(a[2], rope, tx.size[0], &tp, &step) && PyBool_Check(a[4]) && stream_of(a[5], &stream));
    CALLED(p_rotary(&x, &y, tx.size[0], (int)tx.size[2], rope, tp.data, step, a[4] == Py_True, stream));
}

/* append(cache, k, v, slots, rope or None, positions, q or None, q_out, stream or None) */
static PyObject *call_append(PyObject *self, PyObject *const *a, Py_ssize_t n)
{
    tensor_t tk, tv, ts, tp = {0}, tq, to;
    amap_heads k, v, q, out;
    void *cache, *rope, *stream;
    int64_t step = 0;
    int turned;
    (void)self;
    UNLESS(p_append && n == 9 && a[0] != Py_None && named_handle_of(a[0], s_cache_at, &cache) && named_handle_of(a[4], s_rope_at, &rope) && rows_of(a[1], &tk, &k) && rows_of(a[2], &tv, &v) &&
           of_type(a[3], 1, t_int64, &ts) && ts.size[0] == tk.size[0] && same_shape(&tk, &tv) && tk.size[2] == ((amap_cache *)cache)->head_dim);
    if (rope) UNLESS(positions_of(a[5], rope, tk.size[0], &tp, &step));
    turned = a[6] != Py_None;
    if (turned) UNLESS(rows_of(a[6], &tq, &q) && rows_of(a[7], &to, &out) && same_shape(&tq, &to) && tq.size[0] == tk.size[0] && tq.size[2] == tk.size[2]);
    UNLESS(stream_of(a[8], &stream));
    CALLED(p_append(cache, &k, &v, tk.size[0], ts.data, rope, tp.data, step, turned ? &q : NULL, turned ? &out : NULL, stream));
}

/* attend(cache, q, table, lengths, scale or None, window, out, lse, workspace or None, stream or None); a workspace that is too small: not taken */
static PyObject *call_attend(PyObject *self, PyObject *const *a, Py_ssize_t n)
{
    tensor_t tq, tt, tl, to, te, tw;
    amap_heads q, out;
    void *cache, *stream;
    int64_t window, need = 0;
    double scale = 0.0;
    (void)self;
    UNLESS(p_attend && n == 10 && a[0] != Py_None && named_handle_of(a[0], s_cache_at, &cache) && rows_of(a[1], &tq, &q) && of_type(a[2], 2, t_int32, &tt) &&
           of_type(a[3], 1, t_int32, &tl) && rows_of(a[6], &to, &out) && of_type(a[7], 2, t_float32, &te) && same_shape(&tq, &to));
    UNLESS(tt.size[0] == tq.size[0] && tl.size[0] == tq.size[0] && tq.size[2] == ((amap_cache *)cache)->head_dim && tt.size[1] <= INT32_MAX);
    UNLESS(te.size[0] == tq.size[0] && te.size[1] == tq.size[1] && (te.size[0] <= 1 || te.stride[0] == te.size[1]));
    UNLESS(PyLong_CheckExact(a[5]) && count_of(a[5], &window) && window >= 0 && window <= INT32_MAX && (a[4] == Py_None || PyFloat_CheckExact(a[4])));
    if (a[4] != Py_None) scale = PyFloat_AS_DOUBLE(a[4]);
    UNLESS(p_room(cache, q.heads, tq.size[0], (int)tt.size[1], &need) == AMAP_OK);
    tw.data = NULL;
    tw.size[0] = 0;
    if (a[8] != Py_None) UNLESS(of_type(a[8], 1, t_uint8, &tw));
    UNLESS(need <= tw.size[0] && stream_of(a[9], &stream));
    if (a[4] == Py_None) scale = 1.0 / sqrt((double)tq.size[2]);
    CALLED(p_attend(cache, &q, tq.size[0], tt.data, tt.stride[0], (int)tt.size[1], tl.data, (float)scale, (int)window, &out, te.data, tw.data, tw.size[0], stream));
}

/* assign(page size, cached or None, fresh, table, free pages, n_tokens, outputs, stream or None).  Outputs: begin, length, slot, position, owner, taken; or the
 * two buffers they are all parts of, int32 with begin, length, taken, position and owner one after the other, and int64 for the slots. */
static PyObject *call_assign(PyObject *self, PyObject *const *a, Py_ssize_t n)
{
    tensor_t tc, tf, tt, tp, out[6];
    amap_assign g;
    int64_t page, tokens;
    void *stream;
    (void)self;
    UNLESS(p_assign && n == 8 && of_type(a[2], 1, t_int32, &tf) && of_type(a[3], 2, t_int32, &tt) && of_type(a[4], 1, t_int32, &tp) && tt.size[0] == tf.size[0]);
    tc.data = NULL;
    if (a[1] != Py_None) UNLESS(of_type(a[1], 1, t_int32, &tc) && tc.size[0] == tf.size[0]);
    UNLESS(count_of(a[0], &page) && page >= 1 && page <= INT32_MAX && count_of(a[5], &tokens) && tokens >= 0 && tt.size[1] <= INT32_MAX && PyTuple_Check(a[6]));
    const int64_t size[6] = {tf.size[0] + 1, tf.size[0], tokens, tokens, tokens, 1};
    if (PyTuple_GET_SIZE(a[6]) == 2) {
        UNLESS(of_type(PyTuple_GET_ITEM(a[6], 0), 1, t_int32, &out[0]) && of_type(PyTuple_GET_ITEM(a[6], 1), 1, t_int64, &out[2]));
        UNLESS(tokens <= INT32_MAX && out[0].size[0] == 2 * tf.size[0] + 2 + 2 * tokens && out[2].size[0] == tokens);
        out[1].data = (int32_t *)out[0].data + size[0];
        out[5].data = (int32_t *)out[1].data + size[1];
        out[3].data = (int32_t *)out[5].data + 1;
        out[4].data = (int32_t *)out[3].data + tokens;
    } else {
        UNLESS(PyTuple_GET_SIZE(a[6]) == 6);
        for (int i = 0; i < 6; ++i) UNLESS(of_type(PyTuple_GET_ITEM(a[6], i), 1, i == 2 ? t_int64 : t_int32, &out[i]) && out[i].size[0] == size[i]);
    }
    UNLESS(stream_of(a[7], &stream));
    memset(&g, 0, sizeof(g));
    g.requests = tf.size[0];
    g.page_size = (int)page;
    g.cached = tc.data;
    g.fresh = tf.data;
    g.free_pages = tp.data;
    g.n_free = tp.size[0];
    g.table = tt.data;
    g.table_stride = tt.stride[0];
    g.table_width = (int)tt.size[1];
    g.begin = out[0].data;
    g.length = out[1].data;
    g.slot = out[2].data;
    g.position = out[3].data;
    g.owner = out[4].data;
    g.n_tokens = tokens;
    g.taken = out[5].data;
    CALLED(p_assign(&g, stream));
}

/* paged(addresses of amap_cache_assign, amap_rotary, amap_cache_append, _attend, _attend_workspace; int32, int64, float32, uint8; ((type, the library's name), ...)) */
static PyObject *call_paged(PyObject *self, PyObject *const *a, Py_ssize_t n)
{
    void *p[5];
    PyObject *const types = n == 10 ? a[9] : Py_None;
    int ok = PyTuple_CheckExact(types) && PyTuple_GET_SIZE(types) <= MAX_TYPES;
    (void)self;
    for (int i = 0; ok && i < 5; ++i) ok = integer(a[i], &p[i]);
    if (!ok) {
        PyErr_SetString(PyExc_TypeError, "five addresses, four types, and the types of rows");
        return NULL;
    }
    n_row_types = 0;
    for (Py_ssize_t i = 0; i < PyTuple_GET_SIZE(types); ++i) {
        PyObject *type;
        int code;
        if (!PyArg_ParseTuple(PyTuple_GET_ITEM(types, i), "Oi", &type, &code)) return NULL;
        Py_INCREF(type);
        Py_XSETREF(row_type[i], type);
        row_code[i] = code;
        n_row_types = (int)i + 1;
    }
    PyObject **const to[4] = {&t_int32, &t_int64, &t_float32, &t_uint8};
    for (int i = 0; i < 4; ++i) {
        Py_INCREF(a[5 + i]);
        Py_XSETREF(*to[i], a[5 + i]);
    }
    p_assign = (assign_fn)(uintptr_t)p[0];
    p_rotary = (rotary_fn)(uintptr_t)p[1];
    p_append = (append_fn)(uintptr_t)p[2];
    p_attend = (attend_fn)(uintptr_t)p[3];
    p_room = (room_fn)(uintptr_t)p[4];
    Py_RETURN_NONE;
}

static PyMethodDef methods[] = {
    {"rotary", (PyCFunction)(void (*)(void))call_rotary, METH_FASTCALL, NULL},
    {"append", (PyCFunction)(void (*)(void))call_append, METH_FASTCALL, NULL},
    {"attend", (PyCFunction)(void (*)(void))call_attend, METH_FASTCALL, NULL},
    {"assign", (PyCFunction)(void (*)(void))call_assign, METH_FASTCALL, NULL},
    {"paged", (PyCFunction)(void (*)(void))call_paged, METH_FASTCALL, NULL},
    {"execute", (PyCFunction)(void (*)(void))call_execute, METH_FASTCALL, NULL},
    {"execute_multi", (PyCFunction)(void (*)(void))call_execute_multi, METH_FASTCALL, NULL},
    {"gemm", (PyCFunction)(void (*)(void))call_gemm, METH_FASTCALL, NULL},
    {"gather", (PyCFunction)(void (*)(void))call_gather, METH_FASTCALL, NULL},
    {"current_stream", call_current_stream, METH_NOARGS, NULL},
    {"library", (PyCFunction)(void (*)(void))call_library, METH_FASTCALL, NULL},
    {"torch", (PyCFunction)(void (*)(void))call_torch, METH_FASTCALL, NULL},
    {NULL, NULL, 0, NULL},
};
static struct PyModuleDef module = {PyModuleDef_HEAD_INIT, "_amap_call", NULL, -1, methods, NULL, NULL, NULL, NULL};

PyMODINIT_FUNC PyInit__amap_call(void)
{
    s_data_ptr = PyUnicode_InternFromString("data_ptr");
    s_at = PyUnicode_InternFromString("_at");
    s_reads = PyUnicode_InternFromString("_reads");
    s_shape = PyUnicode_InternFromString("shape");
    s_stride = PyUnicode_InternFromString("stride");
    s_dtype = PyUnicode_InternFromString("dtype");
    s_is_cuda = PyUnicode_InternFromString("is_cuda");
    s_cache_at = PyUnicode_InternFromString("_cache_at");
    s_rope_at = PyUnicode_InternFromString("_rope_at");
    if (!s_cache_at || !s_rope_at || !s_shape || !s_stride || !s_dtype || !s_is_cuda || !s_data_ptr || !s_at || !s_reads || pthread_atfork(NULL, NULL, forked)) return NULL;
    return PyModule_Create(&module);
}
