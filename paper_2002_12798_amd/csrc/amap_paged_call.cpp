// The way from a Python call to the operators around the paged cache: torch's tensors taken as they are, outputs made, one call of a C entry point.
//
// These calls run for 4 to 10 us on the GPU where requests are few, and issuing a launch takes 3.5 of them; asked for through the interpreter, a tensor's
// type, shape, strides and address are 0.3 us, a new tensor is 1.7.  Here they are 0.01 and 0.5.  Only the ordinary call is taken:
// tensors on the GPU of the types and ranks that belong there.  Whatever else comes is answered with None before the library has seen it, and
// goes the way through ctypes, which says what is wrong with it; a status that the library returns comes back as an integer.  Built for
// one torch, whose objects it looks into: another one is told apart by its version, and does without.
#include <ATen/ATen.h>
#include <c10/core/impl/LocalDispatchKeySet.h>
#include <torch/csrc/autograd/python_variable.h>

#include <pthread.h>

#include <cmath>

#include "amap.h"

namespace {

decltype(&amap_cache_assign) p_assign;
decltype(&amap_rotary) p_rotary;
decltype(&amap_cache_append) p_append;
decltype(&amap_cache_attend) p_attend;
decltype(&amap_cache_attend_workspace) p_room;
PyObject *raw_stream, *get_device, *is_initialized, *is_capturing, *s_cache_at, *s_rope_at, *s_work, *assigned;
bool initialized;   // torch said so in this process (a fork asks again)

void forked() { initialized = false; }

// An error is the other way's to raise again and is cleared; one that ends the program (an interrupt, an exit: no Exception) stays.
bool not_taken() {
    if (PyErr_Occurred() && PyErr_ExceptionMatches(PyExc_Exception)) PyErr_Clear();
    return false;
}
PyObject *answer_none() {
    not_taken();
    if (PyErr_Occurred()) return nullptr;
    Py_RETURN_NONE;
}

struct Ref {   // an owned reference
    PyObject *o;
    explicit Ref(PyObject *o_ = nullptr) : o(o_) {}
    ~Ref() { Py_XDECREF(o); }
    Ref(const Ref &) = delete;
    Ref &operator=(const Ref &) = delete;
};

bool address(PyObject *o, void **at) {
    if (!o || !PyLong_CheckExact(o)) return false;
    *at = PyLong_AsVoidPtr(o);
    return *at || !PyErr_Occurred() || not_taken();
}
// what an object's attribute says is the library's
template <class X>
bool handle(PyObject *o, PyObject *name, X **at) {
    Ref x(PyObject_GetAttr(o, name));
    void *p = nullptr;
    if (!x.o || !address(x.o, &p) || !p) return not_taken();
    *at = static_cast<X *>(p);
    return true;
}
bool whole(PyObject *o, int64_t lo, int64_t hi, int64_t *n) {
    if (!PyLong_CheckExact(o)) return false;
    *n = PyLong_AsLongLong(o);
    if (*n == -1 && PyErr_Occurred()) return not_taken();
    return *n >= lo && *n <= hi;
}
bool stream_of(PyObject *o, void **stream) {
    if (o != Py_None) return address(o, stream);
    if (!raw_stream) return false;
    if (!initialized) {
        Ref r(PyObject_CallNoArgs(is_initialized));
        initialized = r.o && PyObject_IsTrue(r.o) == 1;
        if (!initialized) return not_taken();
    }
    Ref dev(PyObject_CallNoArgs(get_device));
    Ref r(dev.o ? PyObject_CallOneArg(raw_stream, dev.o) : nullptr);
    return (r.o && address(r.o, stream)) || not_taken();
}

// a tensor on the GPU of this rank and type, its last dimension contiguous
const at::Tensor *tensor(PyObject *o, int rank) {
    if (!THPVariable_Check(o)) return nullptr;
    const at::Tensor &t = THPVariable_Unpack(o);
    if (!t.defined() || !t.is_cuda() || t.layout() != at::kStrided || t.dim() != rank) return nullptr;
    if (rank && t.size(rank - 1) > 1 && t.stride(rank - 1) != 1) return nullptr;
    return &t;
}
const at::Tensor *tensor(PyObject *o, int rank, at::ScalarType type) {
    const at::Tensor *const t = tensor(o, rank);
    return t && t->scalar_type() == type ? t : nullptr;
}
template <class X>
X *data(const at::Tensor &t) {
    return static_cast<X *>(t.data_ptr());
}
// [tokens, heads, head_dim] (16-bit words are bf16 bits)
const at::Tensor *rows(PyObject *o, amap_heads &h) {
    const at::Tensor *const t = tensor(o, 3);
    if (!t || t->size(1) > INT32_MAX || t->size(2) > INT32_MAX) return nullptr;
    switch (t->scalar_type()) {
    case at::kFloat: h.type = AMAP_F32; break;
    case at::kBFloat16:
    case at::kShort: h.type = AMAP_BF16; break;
    case at::kHalf: h.type = AMAP_F16; break;
    default: return nullptr;
    }
    h.data = data<void>(*t);
    h.heads = (int)t->size(1);
    h.token_stride = t->stride(0);
    h.head_stride = t->stride(1);
    return t;
}
// positions of so many tokens for a rope's axes: [tokens], the same for all, or [axes, tokens]
const int32_t *positions(PyObject *o, const amap_rope &rope, int64_t tokens, int64_t &step) {
    step = 0;
    if (const at::Tensor *const t = tensor(o, 1, at::kInt)) return t->size(0) == tokens ? data<int32_t>(*t) : nullptr;
    const at::Tensor *const t = tensor(o, 2, at::kInt);
    if (!t || t->size(0) != rope.n_axes || t->size(1) != tokens) return nullptr;
    step = t->stride(0);
    return data<int32_t>(*t);
}

// New tensors beside another one, of which no gradient is asked.
struct Making {
    c10::impl::ExcludeDispatchKeyGuard without{c10::autograd_dispatch_keyset_with_ADInplaceOrView};
};
at::Tensor made(at::IntArrayRef size, const at::Tensor &beside, at::ScalarType type) { return at::empty(size, beside.options().dtype(type).requires_grad(false)); }

// A tensor of this type and size in a buffer, from its element `at` of that type on (through the dispatcher 0.4 us each)
at::Tensor part(const at::Tensor &buffer, at::ScalarType type, at::IntArrayRef size, int64_t at) {
    at::Tensor t = at::detail::make_tensor<c10::TensorImpl>(c10::TensorImpl::VIEW, c10::Storage(buffer.storage()), buffer.key_set(), c10::scalarTypeToTypeMeta(type));
    t.unsafeGetTensorImpl()->set_storage_offset(at);
    t.unsafeGetTensorImpl()->set_sizes_contiguous(size);
    return t;
}

template <class F>
amap_status called(F f) {
    amap_status st;
    Py_BEGIN_ALLOW_THREADS
    st = f();
    Py_END_ALLOW_THREADS
    return st;
}
PyObject *result(amap_status st, PyObject *value) {   // takes the value
    if (st == AMAP_OK) return value;
    Py_XDECREF(value);
    return PyLong_FromLong(st);
}
PyObject *again(PyObject *o) {
    Py_INCREF(o);
    return o;
}

// rotary(x, rope, positions, out or None, inverse, stream or None) -> out
PyObject *rotary(PyObject *const *a, Py_ssize_t n) {
    amap_heads x, y;
    amap_rope *rope;
    int64_t step;
    void *stream;
    if (n != 6 || !PyBool_Check(a[4])) return nullptr;
    const at::Tensor *const tx = rows(a[0], x);
    if (!tx || a[1] == Py_None || !handle(a[1], s_rope_at, &rope)) return nullptr;
    const int32_t *const position = positions(a[2], *rope, tx->size(0), step);
    if ((!position && tx->numel()) || (a[3] == Py_None && a[5] != Py_None) || !stream_of(a[5], &stream)) return nullptr;
    Ref out;
    if (a[3] != Py_None) {
        out.o = again(a[3]);
    } else {
        Making without;
        out.o = THPVariable_Wrap(made(tx->sizes(), *tx, tx->scalar_type()));
    }
    const at::Tensor *const ty = out.o ? rows(out.o, y) : nullptr;
    if (!ty || ty->sizes() != tx->sizes()) return nullptr;
    const int64_t tokens = tx->size(0);
    const int dim = (int)tx->size(2), inverse = a[4] == Py_True;
    return result(called([&] { return p_rotary(&x, &y, tokens, dim, rope, position, step, inverse, stream); }), again(out.o));
}

// append(cache, k, v, slots, rope or None, positions, q or None, q_out or None, stream or None) -> q_out, or True without a q
PyObject *append(PyObject *const *a, Py_ssize_t n) {
    amap_heads k, v, q, y;
    amap_cache *cache;
    amap_rope *rope = nullptr;
    int64_t step = 0;
    void *stream;
    if (n != 9) return nullptr;
    const at::Tensor *const tk = rows(a[1], k), *const tv = rows(a[2], v), *const ts = tensor(a[3], 1, at::kLong);
    if (!tk || !tv || !ts || tk->sizes() != tv->sizes() || ts->size(0) != tk->size(0) || a[0] == Py_None || !handle(a[0], s_cache_at, &cache)) return nullptr;
    const int64_t tokens = tk->size(0);
    if (tk->size(2) != cache->head_dim) return nullptr;
    const int32_t *position = nullptr;
    if (a[4] != Py_None) {
        if (!handle(a[4], s_rope_at, &rope)) return nullptr;
        position = positions(a[5], *rope, tokens, step);
        if (!position && tokens) return nullptr;
    }
    if (!stream_of(a[8], &stream)) return nullptr;
    Ref out;
    const bool turned = a[6] != Py_None;
    if (turned) {
        const at::Tensor *const tq = rows(a[6], q);
        if (!tq || tq->size(0) != tokens || tq->size(2) != tk->size(2) || (a[7] == Py_None && a[8] != Py_None)) return nullptr;
        if (a[7] != Py_None) {
            out.o = again(a[7]);
        } else {
            Making without;
            out.o = THPVariable_Wrap(made(tq->sizes(), *tq, tq->scalar_type()));
        }
        const at::Tensor *const ty = out.o ? rows(out.o, y) : nullptr;
        if (!ty || ty->sizes() != tq->sizes()) return nullptr;
    }
    const int64_t *const slot = data<int64_t>(*ts);
    return result(called([&] { return p_append(cache, &k, &v, tokens, slot, rope, position, step, turned ? &q : nullptr, turned ? &y : nullptr, stream); }),
                  again(turned ? out.o : Py_True));
}

// The workspace that a cache keeps for a stream, taken out of its dictionary for as long as a call issues its launches (they let other Python threads run)
// and put back behind them: a call of another thread finds none in the meantime and has one of its own, so no two calls whose launches may come one between
// the other's share one.  (Once both are on the stream, whichever was put back last is what the next call finds.)
struct Kept {
    Ref all, key, room;
    bool taken = false;
    // what is there, if it is large enough
    const at::Tensor *look(PyObject *cache, void *stream, int64_t need) {
        all.o = PyObject_GetAttr(cache, s_work);
        key.o = all.o ? PyLong_FromVoidPtr(stream) : nullptr;
        PyObject *const o = key.o && PyDict_CheckExact(all.o) ? PyDict_GetItemWithError(all.o, key.o) : nullptr;
        const at::Tensor *const t = o ? tensor(o, 1, at::kByte) : nullptr;
        if (!t || t->size(0) < need) return nullptr;
        Py_INCREF(o);
        room.o = o;
        return t;
    }
    bool take() { return taken = PyDict_DelItem(all.o, key.o) == 0; }
    ~Kept() {
        if (!taken) return;
        PyObject *type, *value, *trace;   // an error that is on its way stays
        PyErr_Fetch(&type, &value, &trace);
        if (PyDict_SetItem(all.o, key.o, room.o)) PyErr_Clear();
        PyErr_Restore(type, value, trace);
    }
};

// attend(cache, q, table, lengths, scale or None, window, out or None, lse or None, workspace or None, stream or None) -> (out, lse).  Without a workspace the
// one that the cache keeps for the stream is used, if there is one and it is large enough.
PyObject *attend(PyObject *const *a, Py_ssize_t n) {
    amap_heads q, y;
    amap_cache *cache;
    int64_t window, need = 0, have = 0;
    void *stream, *work = nullptr;
    if (n != 10 || (a[4] != Py_None && !PyFloat_CheckExact(a[4])) || !whole(a[5], 0, INT32_MAX, &window)) return nullptr;
    const at::Tensor *const tq = rows(a[1], q), *const tt = tensor(a[2], 2, at::kInt), *const tl = tensor(a[3], 1, at::kInt);
    if (!tq || !tt || !tl || tt->size(0) != tq->size(0) || tl->size(0) != tq->size(0) || tt->size(1) > INT32_MAX || a[0] == Py_None || !handle(a[0], s_cache_at, &cache))
        return nullptr;
    const int64_t requests = tq->size(0);
    const int width = (int)tt->size(1);
    if (tq->size(2) != cache->head_dim || ((a[6] == Py_None || a[7] == Py_None) && a[9] != Py_None) || !stream_of(a[9], &stream)) return nullptr;
    if (p_room(cache, q.heads, requests, width, &need) != AMAP_OK) return nullptr;
    Kept kept;
    if (need) {
        if (a[8] == Py_None && a[9] != Py_None) return nullptr;
        const at::Tensor *const tw = a[8] == Py_None ? kept.look(a[0], stream, need) : tensor(a[8], 1, at::kByte);
        if (!tw || tw->size(0) < need) return nullptr;
        if (a[8] == Py_None) {
            Ref capturing(PyObject_CallNoArgs(is_capturing));   // (a graph runs beside what its stream does later: it has one of its own)
            if (!capturing.o || PyObject_IsTrue(capturing.o) || !kept.take()) return nullptr;
        }
        work = data<void>(*tw);
        have = tw->size(0);
    }
    Ref out, lse;
    {
        Making without;
        if (a[6] == Py_None && a[7] == Py_None) {   // (one allocation, 0.7 us, for both: the sums behind the rows)
            const int64_t bytes = tq->numel() * (int64_t)tq->element_size(), behind = (bytes + 15) / 16 * 4, sums = requests * q.heads;
            const at::Tensor words = made({behind + sums}, *tq, at::kInt);
            out.o = THPVariable_Wrap(part(words, tq->scalar_type(), tq->sizes(), 0));
            lse.o = THPVariable_Wrap(part(words, at::kFloat, {requests, (int64_t)q.heads}, behind));
        } else {
            out.o = a[6] != Py_None ? again(a[6]) : THPVariable_Wrap(made(tq->sizes(), *tq, tq->scalar_type()));
            lse.o = a[7] != Py_None ? again(a[7]) : THPVariable_Wrap(made({requests, (int64_t)q.heads}, *tq, at::kFloat));
        }
    }
    const at::Tensor *const ty = out.o ? rows(out.o, y) : nullptr, *const te = lse.o ? tensor(lse.o, 2, at::kFloat) : nullptr;
    if (!ty || !te || ty->sizes() != tq->sizes() || te->size(0) != requests || te->size(1) != q.heads || !te->is_contiguous()) return nullptr;
    const float scale = a[4] == Py_None ? (float)(1.0 / std::sqrt((double)tq->size(2))) : (float)PyFloat_AS_DOUBLE(a[4]);
    const int32_t *const table = data<int32_t>(*tt), *const length = data<int32_t>(*tl);
    const int64_t stride = tt->stride(0);
    float *const sums = data<float>(*te);
    const amap_status st = called([&] { return p_attend(cache, &q, requests, table, stride, width, length, scale, (int)window, &y, sums, work, have, stream); });
    return st == AMAP_OK ? PyTuple_Pack(2, out.o, lse.o) : PyLong_FromLong(st);
}

// assign(page size, cached or None, fresh, table, free pages, n_tokens, outputs or None, stream or None) -> the outputs: begin, length, slot, position, owner, taken
PyObject *assign(PyObject *const *a, Py_ssize_t n) {
    int64_t page, tokens;
    void *stream;
    if (n != 8 || !whole(a[0], 1, INT32_MAX, &page) || !whole(a[5], 0, INT32_MAX, &tokens) || (a[6] == Py_None && a[7] != Py_None)) return nullptr;
    const at::Tensor *const tf = tensor(a[2], 1, at::kInt), *const tt = tensor(a[3], 2, at::kInt), *const tp = tensor(a[4], 1, at::kInt);
    const at::Tensor *const tc = a[1] != Py_None ? tensor(a[1], 1, at::kInt) : nullptr;
    if (!tf || !tt || !tp || (a[1] != Py_None && (!tc || tc->size(0) != tf->size(0))) || tt->size(0) != tf->size(0) || tt->size(1) > INT32_MAX) return nullptr;
    const int64_t requests = tf->size(0), size[6] = {requests + 1, requests, tokens, tokens, tokens, 1};
    if (!stream_of(a[7], &stream)) return nullptr;
    Ref out;
    if (a[6] != Py_None) {
        if (!PyTuple_Check(a[6]) || PyTuple_GET_SIZE(a[6]) != 6) return nullptr;
        out.o = again(a[6]);
    } else {
        Making without;
        const at::Tensor words = made({2 * requests + 2 + 4 * tokens}, *tf, at::kInt);   // (one buffer: the slots first, 8 bytes each)
        Ref all(PyTuple_New(6));
        if (!all.o) return nullptr;
        int64_t at = 2 * tokens;
        for (int i = 0; i < 6; ++i) {
            PyObject *const o = THPVariable_Wrap(i == 2 ? part(words, at::kLong, {tokens}, 0) : part(words, at::kInt, {size[i]}, at));
            if (!o) return nullptr;
            PyTuple_SET_ITEM(all.o, i, o);
            at += i == 2 ? 0 : size[i];
        }
        // (a named tuple's own constructor is a Python function that does this)
        Ref args(PyTuple_Pack(1, all.o));
        out.o = args.o ? PyTuple_Type.tp_new(reinterpret_cast<PyTypeObject *>(assigned), args.o, nullptr) : nullptr;
        if (!out.o || !PyTuple_Check(out.o)) return nullptr;
    }
    amap_assign g = {};
    void *to[6];
    for (int i = 0; i < 6; ++i) {
        const at::Tensor *const t = tensor(PyTuple_GET_ITEM(out.o, i), 1, i == 2 ? at::kLong : at::kInt);
        if (!t || t->size(0) != size[i]) return nullptr;
        to[i] = data<void>(*t);
    }
    g.requests = requests;
    g.page_size = (int)page;
    g.cached = tc ? data<int32_t>(*tc) : nullptr;
    g.fresh = data<int32_t>(*tf);
    g.free_pages = data<int32_t>(*tp);
    g.n_free = tp->size(0);
    g.table = data<int32_t>(*tt);
    g.table_stride = tt->stride(0);
    g.table_width = (int)tt->size(1);
    g.begin = static_cast<int32_t *>(to[0]);
    g.length = static_cast<int32_t *>(to[1]);
    g.slot = static_cast<int64_t *>(to[2]);
    g.position = static_cast<int32_t *>(to[3]);
    g.owner = static_cast<int32_t *>(to[4]);
    g.n_tokens = tokens;
    g.taken = static_cast<int32_t *>(to[5]);
    return result(called([&] { return p_assign(&g, stream); }), again(out.o));
}

// A call: what it returns; None where it is not taken, an exception of torch's or C++'s among the reasons (the other way meets it again).
template <PyObject *(*F)(PyObject *const *, Py_ssize_t)>
PyObject *entry(PyObject *, PyObject *const *a, Py_ssize_t n) {
    if (!p_rotary) Py_RETURN_NONE;
    try {
        if (PyObject *const r = F(a, n)) return r;
    } catch (...) {
    }
    return answer_none();
}

// library(addresses of amap_cache_assign, amap_rotary, amap_cache_append, _attend, _attend_workspace; the type of an assignment; torch's stream handle of a
// device, current device, whether CUDA is initialised, whether the current stream is being captured)
PyObject *library(PyObject *, PyObject *const *a, Py_ssize_t n) {
    void *p[5];
    bool ok = n == 10 && PyType_Check(a[5]) && PyType_IsSubtype(reinterpret_cast<PyTypeObject *>(a[5]), &PyTuple_Type);
    for (int i = 0; ok && i < 5; ++i) ok = address(a[i], &p[i]);
    if (!ok) {
        PyErr_SetString(PyExc_TypeError, "five addresses, a type and four functions");
        return nullptr;
    }
    PyObject **const to[5] = {&assigned, &raw_stream, &get_device, &is_initialized, &is_capturing};
    for (int i = 0; i < 5; ++i) {
        Py_INCREF(a[5 + i]);
        Py_XSETREF(*to[i], a[5 + i]);
    }
    initialized = false;
    p_assign = reinterpret_cast<decltype(p_assign)>(p[0]);
    p_rotary = reinterpret_cast<decltype(p_rotary)>(p[1]);
    p_append = reinterpret_cast<decltype(p_append)>(p[2]);
    p_attend = reinterpret_cast<decltype(p_attend)>(p[3]);
    p_room = reinterpret_cast<decltype(p_room)>(p[4]);
    Py_RETURN_NONE;
}

#define AMAP_METHOD(name, f) {name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(f)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {AMAP_METHOD("rotary", entry<rotary>), AMAP_METHOD("append", entry<append>), AMAP_METHOD("attend", entry<attend>), AMAP_METHOD("assign", entry<assign>),
                         AMAP_METHOD("library", library), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_amap_paged_call", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__amap_paged_call(void) {
    s_cache_at = PyUnicode_InternFromString("_cache_at");
    s_rope_at = PyUnicode_InternFromString("_rope_at");
    s_work = PyUnicode_InternFromString("_work");
    if (!s_cache_at || !s_rope_at || !s_work || pthread_atfork(nullptr, nullptr, forked)) return nullptr;
    PyObject *const m = PyModule_Create(&module);
    if (m && PyModule_AddStringConstant(m, "torch_version", AMAP_TORCH_VERSION)) {
        Py_DECREF(m);
        return nullptr;
    }
    return m;
}
