// The per-layer calls of the Python binding, from Python objects to the C ABI in one step (module _native).
//
// A layer of a few MB takes its kernels 3 us each, and ctypes with its argument objects took 5 us a call on the host.
// Here a call reads the tensors' addresses and sizes by the same attributes that binding.py reads, and calls the same
// entry point of the same library.  Whatever is not plainly in order (an argument of another type, a tensor that is not
// contiguous, a pool or a buffer too small, a plan destroyed) is left to binding.py, which says what is wrong with it or
// takes it: the functions return 1 for that, else what the library returned.  A hop of 4.6 MB 17.3 -> 8.3 us (6.3 of kernels;
// the same through the C ABI with arguments made before 7.9); the requests of a batch of 64 for kvl_plan 120 -> 2.3.
#define PY_SSIZE_T_CLEAN
#include <Python.h>
#include <structmember.h>

#include <cstdint>

#include "kvl_attn.h"
#include "kvl_pages.h"

namespace {

constexpr long kNotTaken = 1;

// What binding.py's Plan objects add to Python's own: the handle and what is asked of a pool on every call.
struct PlanObject {
    PyObject_HEAD
    void *handle;                              // null: destroyed, or not set
    Py_ssize_t planes;
    unsigned long long bytes[KVL_MAX_PLANES];
    Py_ssize_t dst_planes;                     // of paired plans
    unsigned long long dst_bytes[KVL_MAX_PLANES];
};

// The same of attn.py's AttnPlan objects.
constexpr Py_ssize_t kAttnPlanes = 4;
struct AttnPlanObject {
    PyObject_HEAD
    void *handle;
    Py_ssize_t planes;
    unsigned long long bytes[kAttnPlanes];
    unsigned long long tokens, q_heads, kv_heads, head_dim, rope_half;
    float scale;                               // where the caller names none
    PyObject *dtype;
};

struct Library {
    decltype(&kvl_pack_layer) pack;
    decltype(&kvl_unpack_layer) unpack;
    decltype(&kvl_move_layer) move;
    decltype(&kvl_fullblocks_to_pool_layer) to_pool;
    decltype(&kvl_pool_to_fullblocks_layer) to_blocks;
    decltype(&kvl_append_layer) append;
    decltype(&kvl_attn_layer) attn;
    decltype(&kvl_attn_scored_layer) scored;
    decltype(&kvl_attn_join) join;
    decltype(&kvl_pages_fork) fork;
    decltype(&kvl_pages_extend) extend;
    decltype(&kvl_pages_free) end;
    decltype(&kvl_pages_tables) tables;
    decltype(&kvl_copy_blocks) copy_blocks;
    decltype(&kvl_pages_compact) compact;
} g_lib;
PyObject *g_float32;
PyObject *g_tensor_type, *g_array_type, *g_raw_stream, *g_get_device, *g_is_initialized;
bool g_initialized;             // this process has a device context (a forked child starts anew)
PyObject *s_is_cuda, *s_is_contiguous, *s_is_pinned, *s_data_ptr, *s_nbytes, *s_cuda_stream, *s_dtype, *s_shape, *s_stride;

PyTypeObject *plan_type();
PyTypeObject *attn_plan_type();

// Python's attributes and methods by name; false (with no exception left) if anything is unlike what is expected.
bool get_true(PyObject *o, PyObject *name, bool *value) {
    PyObject *r = PyObject_GetAttr(o, name);
    if (r != Py_True && r != Py_False) {
        Py_XDECREF(r);
        PyErr_Clear();
        return false;
    }
    *value = r == Py_True;
    Py_DECREF(r);
    return true;
}
bool call_true(PyObject *o, PyObject *name) {
    PyObject *args[1] = {o};
    PyObject *r = PyObject_VectorcallMethod(name, args, 1 | PY_VECTORCALL_ARGUMENTS_OFFSET, nullptr);
    if (!r) PyErr_Clear();
    const bool yes = r == Py_True;
    Py_XDECREF(r);
    return yes;
}
bool number(PyObject *r, unsigned long long *value) {       // (takes the reference)
    if (!r || !PyLong_Check(r)) {
        Py_XDECREF(r);
        PyErr_Clear();
        return false;
    }
    *value = PyLong_AsUnsignedLongLong(r);
    Py_DECREF(r);
    if (*value == (unsigned long long)-1 && PyErr_Occurred()) {
        PyErr_Clear();
        return false;
    }
    return true;
}

struct Buffer {
    void *ptr;
    unsigned long long bytes;
};
// A contiguous tensor on the device or, where `host` is given, in pinned memory.
bool buffer(PyObject *t, bool host, Buffer *out) {
    if ((PyObject *)Py_TYPE(t) != g_tensor_type) return false;
    bool cuda;
    if (!get_true(t, s_is_cuda, &cuda) || (!cuda && !(host && call_true(t, s_is_pinned)))) return false;
    if (!call_true(t, s_is_contiguous)) return false;
    unsigned long long p;
    PyObject *args[1] = {t};
    if (!number(PyObject_VectorcallMethod(s_data_ptr, args, 1 | PY_VECTORCALL_ARGUMENTS_OFFSET, nullptr), &p)) return false;
    if (!number(PyObject_GetAttr(t, s_nbytes), &out->bytes)) return false;
    out->ptr = (void *)(uintptr_t)p;
    return true;
}

bool pool(PyObject *planes, Py_ssize_t n, const unsigned long long *need, void **out) {
    const bool list = PyList_CheckExact(planes);
    if (!list && !PyTuple_CheckExact(planes)) return false;
    if (n == 0 || (list ? PyList_GET_SIZE(planes) : PyTuple_GET_SIZE(planes)) != n) return false;
    for (Py_ssize_t p = 0; p < n; ++p) {
        // (the attributes run Python code at most for exotic tensors, but a list could be changed by it)
        if (list && PyList_GET_SIZE(planes) != n) return false;
        PyObject *t = list ? PyList_GET_ITEM(planes, p) : PyTuple_GET_ITEM(planes, p);
        Py_INCREF(t);
        Buffer b;
        const bool ok = buffer(t, false, &b) && b.bytes >= need[p];
        Py_DECREF(t);
        if (!ok) return false;
        out[p] = b.ptr;
    }
    return true;
}

bool stream(PyObject *s, void **out) {
    unsigned long long h;
    if (s == Py_None) {
        if (!g_initialized) {
            PyObject *r = PyObject_CallNoArgs(g_is_initialized);
            if (!r) PyErr_Clear();
            g_initialized = r == Py_True;
            Py_XDECREF(r);
            if (!g_initialized) return false;
        }
        PyObject *device = PyObject_CallNoArgs(g_get_device);
        if (!device) {
            PyErr_Clear();
            return false;
        }
        PyObject *r = PyObject_CallOneArg(g_raw_stream, device);
        Py_DECREF(device);
        if (!number(r, &h)) return false;
    } else if (PyLong_Check(s)) {
        Py_INCREF(s);
        if (!number(s, &h)) return false;
    } else if (!number(PyObject_GetAttr(s, s_cuda_stream), &h)) {
        return false;
    }
    *out = (void *)(uintptr_t)h;
    return true;
}

PlanObject *plan_of(PyObject *o) {
    if (!PyObject_TypeCheck(o, plan_type())) return nullptr;
    PlanObject *p = (PlanObject *)o;
    return p->handle ? p : nullptr;
}

// (As ctypes does, the interpreter goes on meanwhile.)
#define KVL_CALL(expr)              \
    do {                            \
        int rc;                     \
        Py_BEGIN_ALLOW_THREADS      \
        rc = (expr);                \
        Py_END_ALLOW_THREADS        \
        return PyLong_FromLong(rc); \
    } while (0)
#define KVL_NOT_TAKEN return PyLong_FromLong(kNotTaken)

PyObject *pack_layer(PyObject *, PyObject *const *a, Py_ssize_t n) {        // plan, pool planes, xfer, stream
    PlanObject *plan = n == 4 ? plan_of(a[0]) : nullptr;
    void *planes[KVL_MAX_PLANES], *s;
    Buffer x;
    if (!plan || !pool(a[1], plan->planes, plan->bytes, planes) || !buffer(a[2], true, &x) || !stream(a[3], &s)) KVL_NOT_TAKEN;
    void *handle = plan->handle;
    KVL_CALL(g_lib.pack((const kvl_plan_t *)handle, planes, x.ptr, x.bytes, s));
}

PyObject *unpack_layer(PyObject *, PyObject *const *a, Py_ssize_t n) {      // plan, xfer, pool planes, stream
    PlanObject *plan = n == 4 ? plan_of(a[0]) : nullptr;
    void *planes[KVL_MAX_PLANES], *s;
    Buffer x;
    if (!plan || !pool(a[2], plan->planes, plan->bytes, planes) || !buffer(a[1], true, &x) || !stream(a[3], &s)) KVL_NOT_TAKEN;
    void *handle = plan->handle;
    KVL_CALL(g_lib.unpack((const kvl_plan_t *)handle, x.ptr, x.bytes, planes, s));
}

PyObject *move_layer(PyObject *, PyObject *const *a, Py_ssize_t n) {        // plan, source planes, destination planes, stream
    PlanObject *plan = n == 4 ? plan_of(a[0]) : nullptr;
    void *src[KVL_MAX_PLANES], *dst[KVL_MAX_PLANES], *s;
    if (!plan || !pool(a[1], plan->planes, plan->bytes, src) || !pool(a[2], plan->dst_planes, plan->dst_bytes, dst) || !stream(a[3], &s))
        KVL_NOT_TAKEN;
    void *handle = plan->handle;
    KVL_CALL(g_lib.move((const kvl_plan_t *)handle, src, dst, s));
}

bool layer_of(PyObject *o, uint32_t *layer) {
    unsigned long long v;
    if (!PyLong_CheckExact(o)) return false;
    Py_INCREF(o);
    if (!number(o, &v) || v > UINT32_MAX) return false;
    *layer = (uint32_t)v;
    return true;
}

PyObject *fullblocks_to_pool_layer(PyObject *, PyObject *const *a, Py_ssize_t n) {      // plan, blocks, layer, planes, stream
    PlanObject *plan = n == 5 ? plan_of(a[0]) : nullptr;
    void *planes[KVL_MAX_PLANES], *s;
    Buffer b;
    uint32_t layer;
    if (!plan || !pool(a[3], plan->planes, plan->bytes, planes) || !buffer(a[1], true, &b) || !layer_of(a[2], &layer) || !stream(a[4], &s))
        KVL_NOT_TAKEN;
    void *handle = plan->handle;
    KVL_CALL(g_lib.to_pool((const kvl_plan_t *)handle, b.ptr, b.bytes, layer, planes, s));
}

PyObject *pool_to_fullblocks_layer(PyObject *, PyObject *const *a, Py_ssize_t n) {      // plan, planes, layer, blocks, stream
    PlanObject *plan = n == 5 ? plan_of(a[0]) : nullptr;
    void *planes[KVL_MAX_PLANES], *s;
    Buffer b;
    uint32_t layer;
    if (!plan || !pool(a[1], plan->planes, plan->bytes, planes) || !buffer(a[3], true, &b) || !layer_of(a[2], &layer) || !stream(a[4], &s))
        KVL_NOT_TAKEN;
    void *handle = plan->handle;
    KVL_CALL(g_lib.to_blocks((const kvl_plan_t *)handle, planes, layer, b.ptr, b.bytes, s));
}

bool is_type(PyObject *t, PyObject *dtype) {
    PyObject *r = PyObject_GetAttr(t, s_dtype);
    if (!r) PyErr_Clear();
    const bool yes = r == dtype;
    Py_XDECREF(r);
    return yes;
}
// A tuple of `n` numbers (takes the reference).
bool numbers(PyObject *r, Py_ssize_t n, unsigned long long *out) {
    bool ok = r && PyTuple_Check(r) && PyTuple_GET_SIZE(r) == n;
    for (Py_ssize_t k = 0; k < n && ok; ++k) {
        PyObject *x = PyTuple_GET_ITEM(r, k);
        Py_INCREF(x);
        ok = number(x, &out[k]);
    }
    Py_XDECREF(r);
    PyErr_Clear();
    return ok;
}

// [tokens, heads, head_dim] of the plan's type, a token's heads dense: its address and the elements between tokens.
bool rows_of(const AttnPlanObject *plan, PyObject *t, unsigned long long heads, const void **ptr, uint64_t *per) {
    if ((PyObject *)Py_TYPE(t) != g_tensor_type || !is_type(t, plan->dtype)) return false;
    bool cuda;
    unsigned long long shape[3], stride[3], p;
    PyObject *args[1] = {t};
    if (!get_true(t, s_is_cuda, &cuda) || !cuda || !numbers(PyObject_GetAttr(t, s_shape), 3, shape)) return false;
    if (!numbers(PyObject_VectorcallMethod(s_stride, args, 1 | PY_VECTORCALL_ARGUMENTS_OFFSET, nullptr), 3, stride)) return false;
    if (!number(PyObject_VectorcallMethod(s_data_ptr, args, 1 | PY_VECTORCALL_ARGUMENTS_OFFSET, nullptr), &p)) return false;
    const unsigned long long dense = heads * plan->head_dim;
    if (shape[0] != plan->tokens || shape[1] != heads || shape[2] != plan->head_dim) return false;
    if (stride[2] != 1 || (heads > 1 && stride[1] != plan->head_dim)) return false;
    *per = shape[0] == 1 ? dense : stride[0];
    *ptr = (const void *)(uintptr_t)p;
    return *per >= dense && *per % 8 == 0 && p % 16 == 0;
}

AttnPlanObject *attn_plan_of(PyObject *o) {
    if (!PyObject_TypeCheck(o, attn_plan_type())) return nullptr;
    AttnPlanObject *p = (AttnPlanObject *)o;
    return p->handle && p->tokens ? p : nullptr;
}

PyObject *append_layer(PyObject *, PyObject *const *a, Py_ssize_t n) {  // plan, k, v, pool planes, rope, q, q_out, stream
    AttnPlanObject *plan = n == 8 ? attn_plan_of(a[0]) : nullptr;
    void *planes[kAttnPlanes], *s;
    kvl_append_t t{};
    if (!plan || !pool(a[3], plan->planes, plan->bytes, planes)) KVL_NOT_TAKEN;
    if (!rows_of(plan, a[1], plan->kv_heads, &t.k, &t.k_stride) || !rows_of(plan, a[2], plan->kv_heads, &t.v, &t.v_stride)) KVL_NOT_TAKEN;
    if (a[4] != Py_None) {
        Buffer b;
        unsigned long long shape[3];
        if (!buffer(a[4], false, &b) || !is_type(a[4], g_float32) || !numbers(PyObject_GetAttr(a[4], s_shape), 3, shape)) KVL_NOT_TAKEN;
        if (shape[1] != plan->rope_half || shape[2] != 2) KVL_NOT_TAKEN;
        t.rope = (const float *)b.ptr;
        t.rope_positions = shape[0];
    } else if (plan->rope_half) {
        KVL_NOT_TAKEN;
    }
    if (a[5] != Py_None) {
        const void *to;
        if (!rows_of(plan, a[5], plan->q_heads, &t.q, &t.q_stride)) KVL_NOT_TAKEN;
        if (!rows_of(plan, a[6] == Py_None ? a[5] : a[6], plan->q_heads, &to, &t.q_out_stride)) KVL_NOT_TAKEN;
        t.q_out = const_cast<void *>(to);
    } else if (a[6] != Py_None) {
        KVL_NOT_TAKEN;
    }
    if (!stream(a[7], &s) || !plan->handle) KVL_NOT_TAKEN;
    void *handle = plan->handle;
    KVL_CALL(g_lib.append((const kvl_attn_plan_t *)handle, &t, planes, s));
}

// float32 [tokens, q_heads]
bool lse_of(AttnPlanObject *plan, PyObject *o, float **ptr) {
    Buffer b;
    unsigned long long shape[2];
    if (!buffer(o, false, &b) || !is_type(o, g_float32) || !numbers(PyObject_GetAttr(o, s_shape), 2, shape)) return false;
    *ptr = (float *)b.ptr;
    return shape[0] == plan->tokens && shape[1] == plan->q_heads;
}

// plan, q, pool planes, out, workspace, scale, lse, stream; and cap, slopes
PyObject *attn_layer(PyObject *, PyObject *const *a, Py_ssize_t n) {
    AttnPlanObject *plan = n == 8 || n == 10 ? attn_plan_of(a[0]) : nullptr;
    void *planes[kAttnPlanes], *s;
    const void *to;
    kvl_attn_t t{};
    if (!plan || !pool(a[2], plan->planes, plan->bytes, planes)) KVL_NOT_TAKEN;
    if (!rows_of(plan, a[1], plan->q_heads, &t.q, &t.q_stride) || !rows_of(plan, a[3], plan->q_heads, &to, &t.out_stride)) KVL_NOT_TAKEN;
    t.out = const_cast<void *>(to);
    if (a[4] != Py_None) {
        Buffer b;
        if (!buffer(a[4], false, &b)) KVL_NOT_TAKEN;
        t.workspace = b.ptr;
        t.workspace_bytes = b.bytes;
    }
    if (a[5] == Py_None) t.scale = plan->scale;
    else if (PyFloat_CheckExact(a[5])) t.scale = (float)PyFloat_AS_DOUBLE(a[5]);
    else KVL_NOT_TAKEN;
    if (a[6] != Py_None && !lse_of(plan, a[6], &t.lse)) KVL_NOT_TAKEN;
    kvl_attn_scores_t scores{};
    if (n == 10) {
        if (PyFloat_CheckExact(a[8])) scores.cap = (float)PyFloat_AS_DOUBLE(a[8]);
        else if (a[8] != Py_None) KVL_NOT_TAKEN;
        if (a[9] != Py_None) {
            Buffer b;
            unsigned long long shape[1];
            if (!buffer(a[9], false, &b) || !is_type(a[9], g_float32) || !numbers(PyObject_GetAttr(a[9], s_shape), 1, shape)) KVL_NOT_TAKEN;
            if (shape[0] != plan->q_heads) KVL_NOT_TAKEN;
            scores.slopes = (const float *)b.ptr;
        }
    }
    if (!stream(a[7], &s) || !plan->handle) KVL_NOT_TAKEN;
    void *handle = plan->handle;
    if (n == 10) KVL_CALL(g_lib.scored((const kvl_attn_plan_t *)handle, &t, &scores, planes, s));
    KVL_CALL(g_lib.attn((const kvl_attn_plan_t *)handle, &t, planes, s));
}

PyObject *attn_join(PyObject *, PyObject *const *a, Py_ssize_t n) {     // plan, parts, lses, out, lse, stream
    AttnPlanObject *plan = n == 6 ? attn_plan_of(a[0]) : nullptr;
    if (!plan || !PyList_CheckExact(a[1]) || !PyList_CheckExact(a[2])) KVL_NOT_TAKEN;
    const Py_ssize_t parts = PyList_GET_SIZE(a[1]);
    if (parts < 1 || parts > (Py_ssize_t)KVL_JOIN_MOST || PyList_GET_SIZE(a[2]) != parts) KVL_NOT_TAKEN;
    const void *from[KVL_JOIN_MOST], *to;
    float *lses[KVL_JOIN_MOST];
    uint64_t strides[KVL_JOIN_MOST];
    void *s;
    kvl_attn_join_t t{};
    for (Py_ssize_t i = 0; i < parts; ++i) {
        if (PyList_GET_SIZE(a[1]) != parts || PyList_GET_SIZE(a[2]) != parts) KVL_NOT_TAKEN;       // (as in pool())
        PyObject *part = PyList_GET_ITEM(a[1], i), *lse = PyList_GET_ITEM(a[2], i);
        Py_INCREF(part);
        Py_INCREF(lse);
        const bool ok = rows_of(plan, part, plan->q_heads, &from[i], &strides[i]) && lse_of(plan, lse, &lses[i]);
        Py_DECREF(part);
        Py_DECREF(lse);
        if (!ok) KVL_NOT_TAKEN;
    }
    if (!rows_of(plan, a[3], plan->q_heads, &to, &t.out_stride)) KVL_NOT_TAKEN;
    if (a[4] != Py_None && !lse_of(plan, a[4], &t.lse)) KVL_NOT_TAKEN;
    if (!stream(a[5], &s) || !plan->handle) KVL_NOT_TAKEN;
    void *handle = plan->handle;
    t.n_parts = (uint32_t)parts;
    t.parts = from;
    t.part_strides = strides;
    t.lses = lses;
    t.out = const_cast<void *>(to);
    KVL_CALL(g_lib.join((const kvl_attn_plan_t *)handle, &t, s));
}

// requests(hit, app, tables, out): a batch's kvl_request_t into `out`, from contiguous uint32 arrays and a list of contiguous
// int32 tables, all of them NumPy's.  False: not all of them are that.
bool array_of(PyObject *o, const char *formats, Py_buffer *view) {
    if (PyObject_GetBuffer(o, view, PyBUF_C_CONTIGUOUS | PyBUF_FORMAT) != 0) {
        PyErr_Clear();
        return false;
    }
    const char *f = view->format;
    if (view->itemsize == 4 && f && f[0] && !f[1] && (f[0] == formats[0] || f[0] == formats[1])) return true;
    PyBuffer_Release(view);
    return false;
}
PyObject *requests(PyObject *, PyObject *const *a, Py_ssize_t n) {
    if (n != 4 || !PyList_CheckExact(a[2])) Py_RETURN_FALSE;
    const Py_ssize_t count = PyList_GET_SIZE(a[2]);
    Py_buffer hit, app, out;
    if (!array_of(a[0], "IL", &hit)) Py_RETURN_FALSE;
    if (!array_of(a[1], "IL", &app)) {
        PyBuffer_Release(&hit);
        Py_RETURN_FALSE;
    }
    bool ok = hit.len / 4 == count && app.len / 4 == count;
    if (ok && PyObject_GetBuffer(a[3], &out, PyBUF_WRITABLE) != 0) {
        PyErr_Clear();
        ok = false;
    }
    if (ok) {
        ok = out.len >= (Py_ssize_t)sizeof(kvl_request_t) * count;
        kvl_request_t *r = (kvl_request_t *)out.buf;
        for (Py_ssize_t k = 0; k < count && ok; ++k) {
            Py_buffer t;
            PyObject *table = PyList_GET_ITEM(a[2], k);
            ok = (PyObject *)Py_TYPE(table) == g_array_type && array_of(table, "il", &t);
            if (!ok) break;
            ok = t.len / 4 <= (Py_ssize_t)UINT32_MAX;
            r[k].hit_tokens = ((const uint32_t *)hit.buf)[k];
            r[k].append_tokens = ((const uint32_t *)app.buf)[k];
            r[k].n_blocks = (uint32_t)(t.len / 4);
            r[k].block_table = t.len ? (const int32_t *)t.buf : nullptr;    // (the caller's list keeps the table)
            PyBuffer_Release(&t);
        }
        PyBuffer_Release(&out);
    }
    PyBuffer_Release(&hit);
    PyBuffer_Release(&app);
    return PyBool_FromLong(ok);
}

// The pages' calls, for arrays that pages.py has made or looked at: contiguous ones of numbers of the size named here.  They return what the library
// returned; a buffer that is not what it should be is a TypeError.
struct Array {
    Py_buffer view;
    bool held = false;
    ~Array() {
        if (held) PyBuffer_Release(&view);
    }
    bool get(PyObject *o, Py_ssize_t item, bool write) {
        if (PyObject_GetBuffer(o, &view, write ? PyBUF_CONTIG : PyBUF_CONTIG_RO) != 0) return false;
        held = true;
        if (view.itemsize == item) return true;
        PyErr_SetString(PyExc_TypeError, "an array of other numbers");
        return false;
    }
    uint64_t size() const { return (uint64_t)(view.len / view.itemsize); }
    template <typename T>
    T *as() const { return (T *)view.buf; }
};
void *handle_of(PyObject *o) { return PyLong_AsVoidPtr(o); }     // (0 where it is no number: the library refuses it)
#define KVL_ARRAY(name, at, type, write) \
    Array name;                          \
    if (!name.get(a[at], sizeof(type), write)) return nullptr
#define KVL_PAGES(count)                                                   \
    if (n != count) {                                                      \
        PyErr_SetString(PyExc_TypeError, "wrong number of arguments");     \
        return nullptr;                                                    \
    }                                                                      \
    void *pages = handle_of(a[0]);                                         \
    if (PyErr_Occurred()) return nullptr

PyObject *pages_fork(PyObject *, PyObject *const *a, Py_ssize_t n) {        // handle, sequences, numbers of the forks
    KVL_PAGES(3);
    KVL_ARRAY(from, 1, uint64_t, false);
    KVL_ARRAY(to, 2, uint64_t, true);
    if (to.size() < from.size()) return PyLong_FromLong(KVL_EINVAL);
    return PyLong_FromLong(g_lib.fork((kvl_pages_t *)pages, from.as<uint64_t>(), (uint32_t)from.size(), to.as<uint64_t>()));
}
// handle, sequences, tokens, copies; what is not negative is how many copies there are
PyObject *pages_extend(PyObject *, PyObject *const *a, Py_ssize_t n) {
    KVL_PAGES(4);
    KVL_ARRAY(sequences, 1, uint64_t, false);
    KVL_ARRAY(tokens, 2, uint32_t, false);
    KVL_ARRAY(copies, 3, int32_t, true);
    if (tokens.size() != sequences.size() || copies.size() < 2 * sequences.size()) return PyLong_FromLong(KVL_EINVAL);
    uint32_t made = 0;
    const int rc = g_lib.extend((kvl_pages_t *)pages, sequences.as<uint64_t>(), tokens.as<uint32_t>(), (uint32_t)sequences.size(),
                                copies.as<kvl_block_copy_t>(), &made);
    return PyLong_FromLong(rc != KVL_OK ? rc : (long)made);
}
PyObject *pages_compact(PyObject *, PyObject *const *a, Py_ssize_t n) {     // handle, copies; as above
    KVL_PAGES(2);
    KVL_ARRAY(copies, 1, int32_t, true);
    uint32_t made = 0;
    const int rc = g_lib.compact((kvl_pages_t *)pages, (uint32_t)(copies.size() / 2), copies.as<kvl_block_copy_t>(), &made);
    return PyLong_FromLong(rc != KVL_OK ? rc : (long)made);
}
PyObject *pages_free(PyObject *, PyObject *const *a, Py_ssize_t n) {        // handle, sequences
    KVL_PAGES(2);
    KVL_ARRAY(sequences, 1, uint64_t, false);
    return PyLong_FromLong(g_lib.end((kvl_pages_t *)pages, sequences.as<uint64_t>(), (uint32_t)sequences.size()));
}
PyObject *pages_tables(PyObject *, PyObject *const *a, Py_ssize_t n) {      // handle, sequences, table, first
    KVL_PAGES(4);
    KVL_ARRAY(sequences, 1, uint64_t, false);
    KVL_ARRAY(table, 2, int32_t, true);
    KVL_ARRAY(first, 3, uint64_t, true);
    if (first.size() <= sequences.size()) return PyLong_FromLong(KVL_EINVAL);
    return PyLong_FromLong(g_lib.tables((const kvl_pages_t *)pages, sequences.as<uint64_t>(), (uint32_t)sequences.size(), table.as<int32_t>(),
                                        table.size(), first.as<uint64_t>()));
}
PyObject *copy_blocks(PyObject *, PyObject *const *a, Py_ssize_t n) {       // handle, copies, stream
    KVL_PAGES(3);
    KVL_ARRAY(copies, 1, int32_t, false);
    void *s;
    if (!stream(a[2], &s)) KVL_NOT_TAKEN;
    KVL_CALL(g_lib.copy_blocks((const kvl_page_pools_t *)pages, copies.as<kvl_block_copy_t>(), copies.size() / 2, s));
}

// setup_pages(the addresses of the pages' six entry points)
PyObject *setup_pages(PyObject *, PyObject *args) {
    unsigned long long f[6];
    if (!PyArg_ParseTuple(args, "KKKKKK", &f[0], &f[1], &f[2], &f[3], &f[4], &f[5])) return nullptr;
    g_lib.compact = (decltype(g_lib.compact))(uintptr_t)f[5];
    g_lib.fork = (decltype(g_lib.fork))(uintptr_t)f[0];
    g_lib.extend = (decltype(g_lib.extend))(uintptr_t)f[1];
    g_lib.end = (decltype(g_lib.end))(uintptr_t)f[2];
    g_lib.tables = (decltype(g_lib.tables))(uintptr_t)f[3];
    g_lib.copy_blocks = (decltype(g_lib.copy_blocks))(uintptr_t)f[4];
    Py_RETURN_NONE;
}

// setup(torch.Tensor, numpy.ndarray, torch's three stream functions, the addresses of the library's five entry points)
PyObject *setup(PyObject *, PyObject *args) {
    PyObject *type, *array, *raw, *device, *initialized;
    unsigned long long f[5];
    if (!PyArg_ParseTuple(args, "OOOOOKKKKK", &type, &array, &raw, &device, &initialized, &f[0], &f[1], &f[2], &f[3], &f[4])) return nullptr;
    Py_INCREF(type);
    Py_INCREF(array);
    Py_INCREF(raw);
    Py_INCREF(device);
    Py_INCREF(initialized);
    g_tensor_type = type;
    g_array_type = array;
    g_raw_stream = raw;
    g_get_device = device;
    g_is_initialized = initialized;
    g_lib.pack = (decltype(g_lib.pack))(uintptr_t)f[0];
    g_lib.unpack = (decltype(g_lib.unpack))(uintptr_t)f[1];
    g_lib.move = (decltype(g_lib.move))(uintptr_t)f[2];
    g_lib.to_pool = (decltype(g_lib.to_pool))(uintptr_t)f[3];
    g_lib.to_blocks = (decltype(g_lib.to_blocks))(uintptr_t)f[4];
    Py_RETURN_NONE;
}

// setup_attn(torch.float32, the addresses of the attention operators' four entry points)
PyObject *setup_attn(PyObject *, PyObject *args) {
    PyObject *type;
    unsigned long long f[4];
    if (!PyArg_ParseTuple(args, "OKKKK", &type, &f[0], &f[1], &f[2], &f[3])) return nullptr;
    Py_INCREF(type);
    g_float32 = type;
    g_lib.append = (decltype(g_lib.append))(uintptr_t)f[0];
    g_lib.attn = (decltype(g_lib.attn))(uintptr_t)f[1];
    g_lib.scored = (decltype(g_lib.scored))(uintptr_t)f[2];
    g_lib.join = (decltype(g_lib.join))(uintptr_t)f[3];
    Py_RETURN_NONE;
}

PyObject *forked(PyObject *, PyObject *) {
    g_initialized = false;
    Py_RETURN_NONE;
}

PyObject *plan_set(PyObject *self, PyObject *args) {        // _set(handle, bytes of the pool's planes)
    PlanObject *p = (PlanObject *)self;
    unsigned long long handle, bytes[KVL_MAX_PLANES] = {};
    PyObject *t;
    if (!PyArg_ParseTuple(args, "KO!", &handle, &PyTuple_Type, &t)) return nullptr;
    const Py_ssize_t n = PyTuple_GET_SIZE(t);
    if (n > KVL_MAX_PLANES) {
        PyErr_SetString(PyExc_ValueError, "too many planes");
        return nullptr;
    }
    for (Py_ssize_t k = 0; k < n; ++k) {
        bytes[k] = PyLong_AsUnsignedLongLong(PyTuple_GET_ITEM(t, k));
        if (PyErr_Occurred()) return nullptr;
    }
    p->handle = (void *)(uintptr_t)handle;
    p->planes = n;
    for (Py_ssize_t k = 0; k < n; ++k) p->bytes[k] = bytes[k];
    Py_RETURN_NONE;
}
PyObject *plan_set_dst(PyObject *self, PyObject *t) {
    PlanObject *p = (PlanObject *)self;
    if (!PyTuple_CheckExact(t) || PyTuple_GET_SIZE(t) > KVL_MAX_PLANES) {
        PyErr_SetString(PyExc_TypeError, "need a tuple of plane sizes");
        return nullptr;
    }
    p->dst_planes = 0;
    for (Py_ssize_t k = 0; k < PyTuple_GET_SIZE(t); ++k) {
        p->dst_bytes[k] = PyLong_AsUnsignedLongLong(PyTuple_GET_ITEM(t, k));
        if (PyErr_Occurred()) return nullptr;
    }
    p->dst_planes = PyTuple_GET_SIZE(t);
    Py_RETURN_NONE;
}
PyObject *plan_clear(PyObject *self, PyObject *) {
    ((PlanObject *)self)->handle = nullptr;
    Py_RETURN_NONE;
}

// _set(handle, bytes of the pool's planes, dtype, tokens, q_heads, kv_heads, head_dim, rope_dim / 2, scale)
PyObject *attn_plan_set(PyObject *self, PyObject *args) {
    AttnPlanObject *p = (AttnPlanObject *)self;
    unsigned long long handle, size[5], bytes[kAttnPlanes] = {};
    PyObject *t, *dtype;
    double scale;
    if (!PyArg_ParseTuple(args, "KO!OKKKKKd", &handle, &PyTuple_Type, &t, &dtype, &size[0], &size[1], &size[2], &size[3], &size[4], &scale)) return nullptr;
    const Py_ssize_t n = PyTuple_GET_SIZE(t);
    if (n > kAttnPlanes) {
        PyErr_SetString(PyExc_ValueError, "too many planes");
        return nullptr;
    }
    for (Py_ssize_t k = 0; k < n; ++k) {
        bytes[k] = PyLong_AsUnsignedLongLong(PyTuple_GET_ITEM(t, k));
        if (PyErr_Occurred()) return nullptr;
    }
    Py_INCREF(dtype);
    Py_XSETREF(p->dtype, dtype);
    p->handle = (void *)(uintptr_t)handle;
    p->planes = n;
    for (Py_ssize_t k = 0; k < n; ++k) p->bytes[k] = bytes[k];
    p->tokens = size[0];
    p->q_heads = size[1];
    p->kv_heads = size[2];
    p->head_dim = size[3];
    p->rope_half = size[4];
    p->scale = (float)scale;
    Py_RETURN_NONE;
}
PyObject *attn_plan_clear(PyObject *self, PyObject *) {
    ((AttnPlanObject *)self)->handle = nullptr;
    Py_RETURN_NONE;
}
void attn_plan_dealloc(PyObject *self) {
    PyTypeObject *type = Py_TYPE(self);
    Py_XDECREF(((AttnPlanObject *)self)->dtype);
    type->tp_free(self);
}

PyMethodDef attn_plan_methods[] = {
    {"_set", attn_plan_set, METH_VARARGS, nullptr},
    {"_clear", attn_plan_clear, METH_NOARGS, nullptr},
    {nullptr, nullptr, 0, nullptr},
};

PyTypeObject g_attn_plan_type = {PyVarObject_HEAD_INIT(nullptr, 0)};
PyTypeObject *attn_plan_type() { return &g_attn_plan_type; }

PyMethodDef plan_methods[] = {
    {"_set", plan_set, METH_VARARGS, nullptr},
    {"_set_dst", plan_set_dst, METH_O, nullptr},
    {"_clear", plan_clear, METH_NOARGS, nullptr},
    {nullptr, nullptr, 0, nullptr},
};

PyTypeObject g_plan_type = {PyVarObject_HEAD_INIT(nullptr, 0)};
PyTypeObject *plan_type() { return &g_plan_type; }

PyMethodDef module_methods[] = {
    {"pack_layer", (PyCFunction)(void (*)(void))pack_layer, METH_FASTCALL, nullptr},
    {"unpack_layer", (PyCFunction)(void (*)(void))unpack_layer, METH_FASTCALL, nullptr},
    {"move_layer", (PyCFunction)(void (*)(void))move_layer, METH_FASTCALL, nullptr},
    {"fullblocks_to_pool_layer", (PyCFunction)(void (*)(void))fullblocks_to_pool_layer, METH_FASTCALL, nullptr},
    {"pool_to_fullblocks_layer", (PyCFunction)(void (*)(void))pool_to_fullblocks_layer, METH_FASTCALL, nullptr},
    {"append_layer", (PyCFunction)(void (*)(void))append_layer, METH_FASTCALL, nullptr},
    {"attn_layer", (PyCFunction)(void (*)(void))attn_layer, METH_FASTCALL, nullptr},
    {"attn_join", (PyCFunction)(void (*)(void))attn_join, METH_FASTCALL, nullptr},
    {"requests", (PyCFunction)(void (*)(void))requests, METH_FASTCALL, nullptr},
    {"setup", setup, METH_VARARGS, nullptr},
    {"setup_attn", setup_attn, METH_VARARGS, nullptr},
    {"pages_fork", (PyCFunction)(void (*)(void))pages_fork, METH_FASTCALL, nullptr},
    {"pages_extend", (PyCFunction)(void (*)(void))pages_extend, METH_FASTCALL, nullptr},
    {"pages_compact", (PyCFunction)(void (*)(void))pages_compact, METH_FASTCALL, nullptr},
    {"pages_free", (PyCFunction)(void (*)(void))pages_free, METH_FASTCALL, nullptr},
    {"pages_tables", (PyCFunction)(void (*)(void))pages_tables, METH_FASTCALL, nullptr},
    {"copy_blocks", (PyCFunction)(void (*)(void))copy_blocks, METH_FASTCALL, nullptr},
    {"setup_pages", setup_pages, METH_VARARGS, nullptr},
    {"forked", forked, METH_NOARGS, nullptr},
    {nullptr, nullptr, 0, nullptr},
};

// (found in the file by build.py, which takes no module built from other sources: the calls above go by raw addresses)
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_native", "The per-layer calls of the binding (" KVL_NATIVE_KEY ")", -1, module_methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__native(void) {
    const char *names[] = {"is_cuda", "is_contiguous", "is_pinned", "data_ptr", "nbytes", "cuda_stream", "dtype", "shape", "stride"};
    PyObject **where[] = {&s_is_cuda, &s_is_contiguous, &s_is_pinned, &s_data_ptr, &s_nbytes, &s_cuda_stream, &s_dtype, &s_shape, &s_stride};
    for (int i = 0; i < 9; ++i)
        if (!(*where[i] = PyUnicode_InternFromString(names[i]))) return nullptr;
    g_plan_type.tp_name = "paper_2602_21548_amd._native.PlanBase";
    g_plan_type.tp_basicsize = sizeof(PlanObject);
    g_plan_type.tp_flags = Py_TPFLAGS_DEFAULT | Py_TPFLAGS_BASETYPE;
    g_plan_type.tp_new = PyType_GenericNew;
    g_plan_type.tp_methods = plan_methods;
    g_attn_plan_type.tp_name = "paper_2602_21548_amd._native.AttnPlanBase";
    g_attn_plan_type.tp_basicsize = sizeof(AttnPlanObject);
    g_attn_plan_type.tp_flags = Py_TPFLAGS_DEFAULT | Py_TPFLAGS_BASETYPE;
    g_attn_plan_type.tp_new = PyType_GenericNew;
    g_attn_plan_type.tp_dealloc = attn_plan_dealloc;
    g_attn_plan_type.tp_methods = attn_plan_methods;
    if (PyType_Ready(&g_plan_type) < 0 || PyType_Ready(&g_attn_plan_type) < 0) return nullptr;
    PyObject *m = PyModule_Create(&module);
    if (!m) return nullptr;
    Py_INCREF(&g_plan_type);
    if (PyModule_AddObject(m, "PlanBase", (PyObject *)&g_plan_type) < 0) {
        Py_DECREF(&g_plan_type);
        Py_DECREF(m);
        return nullptr;
    }
    Py_INCREF(&g_attn_plan_type);
    if (PyModule_AddObject(m, "AttnPlanBase", (PyObject *)&g_attn_plan_type) < 0) {
        Py_DECREF(&g_attn_plan_type);
        Py_DECREF(m);
        return nullptr;
    }
    return m;
}
