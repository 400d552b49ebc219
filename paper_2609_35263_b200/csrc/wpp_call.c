/* The calls a stage makes once per layer, marshalled in C: a Python module `_wpp_call` whose functions take what the binding's
 * functions take and hand it to the library.  Through ctypes the fourteen to eighteen arguments of a call cost about as much
 * host time as its launches.  An argument that is memory is None (null) or an object with data_ptr(), never an integer; a
 * description is an instance of the binding's ctypes structure; contexts and streams are integers.  The library's functions
 * come from the loaded libwpp.so (init), so that this module links to nothing. */
#define PY_SSIZE_T_CLEAN
#include <Python.h>
#include <stdint.h>

#include "../../include/wpp.h"

static int (*p_append)(const wpp_ctx*, const wpp_batch_desc*, const void*, const void*, void*, void*, const int32_t*, const int32_t*,
                       const int32_t*, const void*, const void*, int32_t*, void*);
static int (*p_attention)(const wpp_ctx*, const wpp_batch_desc*, const void*, void*, float*, const void*, const void*, const int32_t*,
                          const int32_t*, const int32_t*, const void*, const void*, void*, size_t, int32_t*, void*);
static int (*p_kda)(const wpp_ctx*, const wpp_kda_desc*, const void*, const void*, const void*, const float*, const float*,
                    const int64_t*, const int32_t*, float*, const int32_t*, const int32_t*, const int32_t*, void*, void*, size_t,
                    int32_t*, void*);
static int (*p_linear)(const wpp_ctx*, const wpp_linear_desc*, const void*, const void*, const void*, const float*, const int64_t*,
                       const int32_t*, float*, const int32_t*, const int32_t*, const int32_t*, void*, void*, size_t, int32_t*, void*);
static int (*p_rope)(const wpp_ctx*, const wpp_rope_desc*, const void*, void*, const void*, void*, const uint64_t*, const int32_t*, void*);
static int (*p_rope_append)(const wpp_ctx*, const wpp_batch_desc*, const wpp_rope_desc*, const void*, void*, const void*, const void*, void*,
                            void*, const uint64_t*, const int32_t*, const int64_t*, int32_t*, void*);
static int (*p_pages)(const wpp_ctx*, const wpp_batch_desc*, const int32_t*, const int32_t*, const int32_t*, int32_t, const int32_t*, int32_t*,
                      int32_t*, int64_t*, int32_t*, int64_t*, int32_t, int32_t*, void*);
static PyObject *t_batch, *t_kda, *t_linear;                   /* the binding's BatchDesc, KdaDesc and LinearDesc */
static PyObject *o_bf16, *o_i32, *o_i64, *no_args;             /* torch's types; () */

/* A tensor's attributes and methods.  A torch.Tensor (t_tensor) is asked through its class's descriptors, which are looked up once; what
 * else has them (subclasses, which may have their own), by name.  Host time of a call, by name | so, us: wpp_assign_pages, which
 * looks at ten tensors, 9.7 | 9.2, wpp_rope 5.8 | 5.4, wpp_rope_append 6.4 | 6.0. */
typedef struct {
    const char* text;
    int method;                     /* called without arguments */
    PyObject *name, *descriptor;    /* descriptor: null where it is of no kind that is known here */
} member;
static member data_ptr = {"data_ptr", 1, NULL, NULL}, get_device = {"get_device", 1, NULL, NULL}, strides = {"stride", 1, NULL, NULL},
              element_size = {"element_size", 1, NULL, NULL}, shape = {"shape", 0, NULL, NULL}, dtype = {"dtype", 0, NULL, NULL};
static PyTypeObject* t_tensor;
static PyObject* ask(PyObject* o, const member* m) {
    if (Py_TYPE(o) == t_tensor && m->descriptor) {
        if (!m->method) {
            const PyGetSetDef* d = ((PyGetSetDescrObject*)m->descriptor)->d_getset;
            return d->get(o, d->closure);
        }
        const PyMethodDef* d = ((PyMethodDescrObject*)m->descriptor)->d_method;
        return d->ml_flags == METH_NOARGS ? d->ml_meth(o, NULL) : ((PyCFunctionWithKeywords)(void (*)(void))d->ml_meth)(o, no_args, NULL);
    }
    return m->method ? PyObject_CallMethodNoArgs(o, m->name) : PyObject_GetAttr(o, m->name);
}
/* looks one up: 0, or -1 with an exception set */
static int find(member* m) {
    PyObject* d = PyObject_GetAttrString((PyObject*)t_tensor, m->text);
    if (!d) return -1;
    int known = 0;
    if (m->method && Py_IS_TYPE(d, &PyMethodDescr_Type)) {
        const int flags = ((PyMethodDescrObject*)d)->d_method->ml_flags;
        known = flags == METH_NOARGS || flags == (METH_VARARGS | METH_KEYWORDS);
    } else if (!m->method && Py_IS_TYPE(d, &PyGetSetDescr_Type)) {
        known = ((PyGetSetDescrObject*)d)->d_getset->get != NULL;
    }
    known = known && PyType_IsSubtype(t_tensor, PyDescr_TYPE(d));
    Py_XSETREF(m->descriptor, known ? Py_NewRef(d) : NULL);
    Py_DECREF(d);
    return 0;
}

/* Each of these returns 0, or -1 with an exception set. */
static int integer(PyObject* o, void** out) {           /* a context, a stream, a function: None is null */
    *out = o == Py_None ? NULL : PyLong_AsVoidPtr(o);
    return *out == NULL && PyErr_Occurred() ? -1 : 0;
}
static int memory(PyObject* o, void** out) {            /* what has no data_ptr() raises AttributeError, an integer too */
    *out = NULL;
    PyObject* v = ask(o, &data_ptr);
    if (!v) return -1;
    if (PyLong_Check(v)) *out = PyLong_AsVoidPtr(v);
    else PyErr_SetString(PyExc_TypeError, "data_ptr() is not an integer");
    Py_DECREF(v);
    return *out == NULL && PyErr_Occurred() ? -1 : 0;
}
static int memories(PyObject* const* args, int n, void** out) {         /* None is null */
    for (int i = 0; i < n; ++i) {
        out[i] = NULL;
        if (args[i] != Py_None && memory(args[i], &out[i])) return -1;
    }
    return 0;
}
/* copies a ctypes structure: what the caller does with it while the call runs without the interpreter lock is the caller's */
static int description(PyObject* o, PyObject* type, void* out, Py_ssize_t size) {
    const int is = PyObject_IsInstance(o, type);
    if (is < 0) return -1;
    if (!is) {
        PyErr_Format(PyExc_TypeError, "a description has to be a %s, not %.100s", ((PyTypeObject*)type)->tp_name, Py_TYPE(o)->tp_name);
        return -1;
    }
    Py_buffer b;
    if (PyObject_GetBuffer(o, &b, PyBUF_SIMPLE)) return -1;
    if (b.len >= size) memcpy(out, b.buf, (size_t)size);      /* (a subclass may have fields of its own behind) */
    else PyErr_SetString(PyExc_TypeError, "description of another size");
    const int rc = b.len >= size ? 0 : -1;
    PyBuffer_Release(&b);
    return rc;
}
static int count(Py_ssize_t n, Py_ssize_t want) {
    if (n == want) return 0;
    PyErr_Format(PyExc_TypeError, "%zd arguments instead of %zd", n, want);
    return -1;
}

static int code_pools(const wpp_batch_desc* d, PyObject* k, PyObject* v);

/* kv_append(ctx, desc, k_new, v_new, k_cache, v_cache, tables, prefix, chunks, plan_host, plan_dev, status, stream) */
static PyObject* kv_append(PyObject* self, PyObject* const* args, Py_ssize_t n) {
    (void)self;
    void *ctx, *a[11];
    wpp_batch_desc d;
    if (count(n, 13) || integer(args[0], &ctx) || description(args[1], t_batch, &d, sizeof(d)) || memories(args + 2, 7, a) ||
        memory(args[9], &a[7]) || memories(args + 10, 2, a + 8) || integer(args[12], &a[10]))
        return NULL;
    int st = code_pools(&d, args[4], args[5]);
    if (st) return st < 0 ? NULL : PyLong_FromLong(st);
    Py_BEGIN_ALLOW_THREADS
    st = p_append(ctx, &d, a[0], a[1], a[2], a[3], a[4], a[5], a[6], a[7], a[8], a[9], a[10]);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(st);
}

/* attention(ctx, desc, q, out, lse, k_cache, v_cache, tables, prefix, chunks, plan_host, plan_dev, workspace, bytes, status, stream) */
static PyObject* attention(PyObject* self, PyObject* const* args, Py_ssize_t n) {
    (void)self;
    void *ctx, *a[11], *b[2];
    wpp_batch_desc d;
    if (count(n, 16) || integer(args[0], &ctx) || description(args[1], t_batch, &d, sizeof(d)) || memories(args + 2, 8, a) ||
        memory(args[10], &a[8]) || memories(args + 11, 2, a + 9))
        return NULL;
    const size_t bytes = PyLong_AsSize_t(args[13]);
    if ((bytes == (size_t)-1 && PyErr_Occurred()) || memories(args + 14, 1, b) || integer(args[15], &b[1])) return NULL;
    int st = code_pools(&d, args[5], args[6]);
    if (st) return st < 0 ? NULL : PyLong_FromLong(st);
    Py_BEGIN_ALLOW_THREADS
    st = p_attention(ctx, &d, a[0], a[1], a[2], a[3], a[4], a[5], a[6], a[7], a[8], a[9], a[10], bytes, b[0], b[1]);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(st);
}

/* kda_chunk(ctx, desc, q, k, v, alpha, beta, rows, prefix, pool, state_in, state_out, snaps, out, workspace, bytes, status, stream) */
static PyObject* kda_chunk(PyObject* self, PyObject* const* args, Py_ssize_t n) {
    (void)self;
    void *ctx, *a[13], *b[2];
    wpp_kda_desc d;
    if (count(n, 18) || integer(args[0], &ctx) || description(args[1], t_kda, &d, sizeof(d)) || memories(args + 2, 13, a)) return NULL;
    const size_t bytes = PyLong_AsSize_t(args[15]);
    if ((bytes == (size_t)-1 && PyErr_Occurred()) || memories(args + 16, 1, b) || integer(args[17], &b[1])) return NULL;
    int st;
    Py_BEGIN_ALLOW_THREADS
    st = p_kda(ctx, &d, a[0], a[1], a[2], a[3], a[4], a[5], a[6], a[7], a[8], a[9], a[10], a[11], a[12], bytes, b[0], b[1]);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(st);
}

/* linear_chunk(ctx, desc, q, k, v, decay, rows, prefix, pool, state_in, state_out, snaps, out, workspace, bytes, status, stream) */
static PyObject* linear_chunk(PyObject* self, PyObject* const* args, Py_ssize_t n) {
    (void)self;
    void *ctx, *a[12], *b[2];
    wpp_linear_desc d;
    if (count(n, 17) || integer(args[0], &ctx) || description(args[1], t_linear, &d, sizeof(d)) || memories(args + 2, 12, a)) return NULL;
    const size_t bytes = PyLong_AsSize_t(args[14]);
    if ((bytes == (size_t)-1 && PyErr_Occurred()) || memories(args + 15, 1, b) || integer(args[16], &b[1])) return NULL;
    int st;
    Py_BEGIN_ALLOW_THREADS
    st = p_linear(ctx, &d, a[0], a[1], a[2], a[3], a[4], a[5], a[6], a[7], a[8], a[9], a[10], a[11], bytes, b[0], b[1]);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(st);
}

/* ---- calls that take tensors as they are: what they have to be is looked at here (0; 1: they are not; -1: an exception is set) */
typedef struct {
    void* at;
    int dims;
    int64_t size[4], stride[4];
} tensor;
static int longs(PyObject* o, int64_t* out, int* n) {
    if (!o) return -1;
    int rc = -1;
    if (!PyTuple_Check(o)) {
        PyErr_SetString(PyExc_TypeError, "shape or strides that are no tuple");
    } else {
        const Py_ssize_t k = PyTuple_GET_SIZE(o);
        *n = (int)k;
        rc = k > 4;
        for (Py_ssize_t i = 0; rc == 0 && i < k; ++i) {
            out[i] = (int64_t)PyLong_AsLongLong(PyTuple_GET_ITEM(o, i));
            if (out[i] == -1 && PyErr_Occurred()) rc = -1;
        }
    }
    Py_DECREF(o);
    return rc;
}
/* a tensor of a type, on the device with this number, with `dims` dimensions */
static int tensor_of(PyObject* o, PyObject* type, long device, int dims, tensor* t) {
    if (memory(o, &t->at)) return -1;
    PyObject* x = ask(o, &dtype);
    if (!x) return -1;
    const int other = x != type;
    Py_DECREF(x);
    if (other) return 1;
    x = ask(o, &get_device);
    if (!x) return -1;
    const long on = PyLong_AsLong(x);
    Py_DECREF(x);
    if (on == -1 && PyErr_Occurred()) return -1;
    if (on != device) return 1;
    int n = 0, rc = longs(ask(o, &shape), t->size, &n);
    if (rc) return rc;
    t->dims = n;
    if ((rc = longs(ask(o, &strides), t->stride, &n))) return rc;
    return t->dims != dims;
}
/* numbers behind one another, `least` of them or more */
static int numbers(PyObject* o, PyObject* type, long device, int64_t least, tensor* t) {
    const int rc = tensor_of(o, type, device, 1, t);
    return rc ? rc : t->size[0] < least || (t->size[0] > 1 && t->stride[0] != 1);
}
/* rows [T, heads, d] of contiguous elements: the strides as the library wants them, 0 where there is but one */
static int rows(PyObject* o, long device, int64_t T, int64_t heads, int64_t d, tensor* t, int64_t* token, int64_t* head) {
    const int rc = tensor_of(o, o_bf16, device, 3, t);
    if (rc) return rc;
    if ((T >= 0 && t->size[0] != T) || (heads >= 0 && t->size[1] != heads) || (d >= 0 && t->size[2] != d)) return 1;
    *token = *head = 0;
    if (t->size[0] == 0 || t->size[1] == 0 || t->size[2] == 0) return 0;                   /* (strides of nothing say nothing) */
    if (t->size[2] > 1 && t->stride[2] != 1) return 1;
    *token = t->size[0] > 1 ? t->stride[0] : 0;
    *head = t->size[1] > 1 ? t->stride[1] : 0;
    if ((t->size[0] > 1 && *token == 0) || (t->size[1] > 1 && *head == 0)) return 1;      /* (one row for several; to the library 0 means dense) */
    if (*token && !*head) *head = t->size[2];
    if (!*token && *head) *token = *head * t->size[1];                                     /* (of a single token: any that is long enough) */
    return 0;
}
/* Elements (of a cache held in codes: bytes) from a pool's address to the end of its last row, as the library reads the description; 0 where
 * it refuses it. */
static __int128 pool_end(const wpp_batch_desc* d) {
    if (d->num_pages <= 0 || d->num_kv_heads <= 0 || d->page_size <= 0 || d->head_dim <= 0) return 0;
    if (d->kv_token_stride < 0 || d->kv_head_stride < 0 || d->kv_page_stride < 0) return 0;
    const __int128 B = d->page_size, token = d->kv_token_stride ? d->kv_token_stride : d->head_dim;
    if (d->dtype == WPP_KV8) {
        const __int128 block = B * d->head_dim + 16, head = d->kv_head_stride ? d->kv_head_stride : block;
        return (d->num_pages - 1) * (d->kv_page_stride ? d->kv_page_stride : head * d->num_kv_heads) + (d->num_kv_heads - 1) * head + block;
    }
    const __int128 block = (B - 1) * token + d->head_dim;
    const __int128 head = d->kv_head_stride ? d->kv_head_stride : token * B, page = d->kv_page_stride ? d->kv_page_stride : head * d->num_kv_heads;
    return (d->num_pages - 1) * page + (d->num_kv_heads - 1) * head + block;
}
/* a tensor of any shape that goes on for `end` elements: kernels read and write at computed places of it */
static int reaches(PyObject* o, __int128 end) {
    PyObject *size = ask(o, &shape), *stride = size ? ask(o, &strides) : NULL;
    int rc = -1;
    if (stride && PyTuple_Check(size) && PyTuple_Check(stride) && PyTuple_GET_SIZE(size) == PyTuple_GET_SIZE(stride)) {
        __int128 reach = 1;
        int none = 0;
        for (Py_ssize_t i = 0; i < PyTuple_GET_SIZE(size); ++i) {
            const int64_t n = (int64_t)PyLong_AsLongLong(PyTuple_GET_ITEM(size, i)), by = (int64_t)PyLong_AsLongLong(PyTuple_GET_ITEM(stride, i));
            none |= n <= 0;
            reach += (__int128)(n - 1) * by;
        }
        if (!PyErr_Occurred()) rc = (none ? 0 : reach) < end;
    } else if (stride) {
        PyErr_SetString(PyExc_TypeError, "shape or strides that are no tuple");
    }
    Py_XDECREF(size);
    Py_XDECREF(stride);
    return rc;
}
/* the same, of a type and on the device with this number */
static int pool_of(PyObject* o, PyObject* type, long device, __int128 end) {
    PyObject* x = ask(o, &dtype);
    if (!x) return -1;
    const int other = x != type;
    Py_DECREF(x);
    if (other) return 1;
    x = ask(o, &get_device);
    if (!x) return -1;
    const long on = PyLong_AsLong(x);
    Py_DECREF(x);
    if (on == -1 && PyErr_Occurred()) return -1;
    return on != device ? 1 : reaches(o, end);
}
/* The pools of a cache held in 8 bits, in calls that take addresses: tensors of one-byte elements that go on for as long as the description says.
 * (What is no tensor but has an address answers for itself; of the other kinds of cache nothing is looked at.) */
static int code_pools(const wpp_batch_desc* d, PyObject* k, PyObject* v) {
    if (d->dtype != WPP_KV8 || !t_tensor) return 0;
    PyObject* const pools[2] = {k, v};
    int st = 0;
    for (int i = 0; st == 0 && i < 2; ++i) {
        if (!PyObject_TypeCheck(pools[i], t_tensor)) continue;
        PyObject* x = ask(pools[i], &element_size);
        if (!x) return -1;
        const long bytes = PyLong_AsLong(x);
        Py_DECREF(x);
        if (bytes == -1 && PyErr_Occurred()) return -1;
        st = bytes != 1 ? 1 : reaches(pools[i], pool_end(d));
    }
    return st;
}
/* code_pools(desc, k, v): what those calls answer to such pools, for one that is not marshalled here */
static PyObject* pools_of(PyObject* self, PyObject* const* args, Py_ssize_t n) {
    (void)self;
    wpp_batch_desc d;
    if (count(n, 3) || description(args[0], t_batch, &d, sizeof(d))) return NULL;
    const int st = code_pools(&d, args[1], args[2]);
    return st < 0 ? NULL : PyLong_FromLong(st);
}
/* q, k (None: none), turns, positions and the options into a description: args[0 .. 7] are q, k, q_out, k_out or v, turns, positions,
 * interleaved, magnitude */
static int rope_desc(PyObject* const* args, long device, int with_v, wpp_rope_desc* d, tensor* t) {
    memset(d, 0, sizeof(*d));
    memset(t, 0, 6 * sizeof(*t));
    int rc = 0;
    int64_t T = -1, dim = -1;
    if (args[0] != Py_None) {
        if ((rc = rows(args[0], device, -1, -1, -1, &t[0], &d->q_token_stride, &d->q_head_stride))) return rc;
        T = t[0].size[0];
        dim = t[0].size[2];
        if ((rc = rows(args[2], device, T, t[0].size[1], dim, &t[2], &d->qo_token_stride, &d->qo_head_stride))) return rc;
        if (t[0].size[1] > 65535) return 1;
        d->num_q_heads = (int32_t)t[0].size[1];
    }
    if (args[1] != Py_None) {
        if ((rc = rows(args[1], device, T, -1, dim, &t[1], &d->k_token_stride, &d->k_head_stride))) return rc;
        T = t[1].size[0];
        dim = t[1].size[2];
        if ((rc = rows(args[3], device, T, t[1].size[1], dim, &t[3], with_v ? &d->v_token_stride : &d->ko_token_stride,
                       with_v ? &d->v_head_stride : &d->ko_head_stride)))
            return rc;
        if (t[1].size[1] > 65535) return 1;
        d->num_k_heads = (int32_t)t[1].size[1];
    }
    if (T < 0 || dim > 65535) return 1;
    if ((rc = numbers(args[4], o_i64, device, 0, &t[4])) || (rc = numbers(args[5], o_i32, device, T, &t[5]))) return rc;
    if (t[4].size[0] > 65535) return 1;
    d->head_dim = (int32_t)dim;
    d->rot_dim = (int32_t)(2 * t[4].size[0]);
    d->interleaved = PyObject_IsTrue(args[6]);
    d->magnitude = (float)PyFloat_AsDouble(args[7]);
    if (d->interleaved < 0 || PyErr_Occurred()) return -1;
    d->total_tokens = T;
    return 0;
}

/* rope(ctx, device, q, k, q_out, k_out, turns, positions, interleaved, magnitude, stream) */
static PyObject* rope(PyObject* self, PyObject* const* args, Py_ssize_t n) {
    (void)self;
    void *ctx, *stream;
    wpp_rope_desc d;
    tensor t[6];
    if (count(n, 11) || integer(args[0], &ctx) || integer(args[10], &stream)) return NULL;
    const long device = PyLong_AsLong(args[1]);
    if (device == -1 && PyErr_Occurred()) return NULL;
    int st = rope_desc(args + 2, device, 0, &d, t);
    if (st < 0) return NULL;
    if (st == 0) {
        Py_BEGIN_ALLOW_THREADS
        st = p_rope(ctx, &d, t[0].at, t[2].at, t[1].at, t[3].at, t[4].at, t[5].at, stream);
        Py_END_ALLOW_THREADS
    }
    return PyLong_FromLong(st);
}

/* rope_append(ctx, device, desc, q, k_new, q_out, v_new, turns, positions, interleaved, magnitude, k_cache, v_cache, slots, status, stream) */
static PyObject* rope_append(PyObject* self, PyObject* const* args, Py_ssize_t n) {
    (void)self;
    void *ctx, *stream, *pool[2], *status;
    wpp_batch_desc b;
    wpp_rope_desc d;
    tensor t[6], slots;
    if (count(n, 16) || integer(args[0], &ctx) || integer(args[15], &stream) || description(args[2], t_batch, &b, sizeof(b))) return NULL;
    const long device = PyLong_AsLong(args[1]);
    if (device == -1 && PyErr_Occurred()) return NULL;
    int st = args[4] == Py_None ? 1 : rope_desc(args + 3, device, 1, &d, t);
    if (st == 0) st = numbers(args[13], o_i64, device, d.total_tokens, &slots);
    for (int i = 0; st == 0 && i < 2; ++i)               /* (none, and a cache that is not of bf16 rows: the library says so) */
        if (args[11 + i] != Py_None && d.total_tokens > 0 && b.dtype == WPP_BF16) st = pool_of(args[11 + i], o_bf16, device, pool_end(&b));
    if (st < 0 || memories(args + 11, 2, pool) || memories(args + 14, 1, &status)) return NULL;
    if (st == 0) {
        Py_BEGIN_ALLOW_THREADS
        st = p_rope_append(ctx, &b, &d, t[0].at, t[2].at, t[1].at, t[3].at, pool[0], pool[1], t[4].at, t[5].at, slots.at, status, stream);
        Py_END_ALLOW_THREADS
    }
    return PyLong_FromLong(st);
}

/* pages(ctx, device, desc, prefix, chunks, free, cursor, cursor_out, tables, rows, positions, slots, status, stream) */
static PyObject* pages(PyObject* self, PyObject* const* args, Py_ssize_t n) {
    (void)self;
    void *ctx, *stream, *status;
    wpp_batch_desc b;
    tensor t[9];
    if (count(n, 14) || integer(args[0], &ctx) || integer(args[13], &stream) || description(args[2], t_batch, &b, sizeof(b))) return NULL;
    const long device = PyLong_AsLong(args[1]);
    if (device == -1 && PyErr_Occurred()) return NULL;
    memset(t, 0, sizeof(t));
    const int64_t R = b.num_requests < 0 ? 0 : b.num_requests;
    int64_t most = -1;
    int st;
    if ((st = numbers(args[3], o_i32, device, R, &t[0])) == 0 && (st = numbers(args[4], o_i32, device, R, &t[1])) == 0 &&
        (st = numbers(args[5], o_i32, device, 0, &t[2])) == 0 && (st = numbers(args[6], o_i32, device, 1, &t[3])) == 0 &&
        (st = numbers(args[7], o_i32, device, 2, &t[4])) == 0 && (st = tensor_of(args[8], o_i32, device, 2, &t[5])) == 0 &&
        (st = numbers(args[9], o_i64, device, R + 1, &t[6])) == 0) {
        st = t[2].size[0] > 0x7fffffff || t[5].size[0] < R || (R > 0 && t[5].size[1] != b.max_blocks_per_req) ||
             (R > 0 && t[5].size[1] > 1 && t[5].stride[1] != 1) || (R > 1 && t[5].stride[0] != t[5].size[1]);
        for (int i = 0; st == 0 && i < 2; ++i) {
            if (args[10 + i] == Py_None) continue;
            st = numbers(args[10 + i], i ? o_i64 : o_i32, device, 0, &t[7 + i]);
            if (st == 0 && (most < 0 || t[7 + i].size[0] < most)) most = t[7 + i].size[0];
            if (!t[7 + i].at) t[7 + i].at = t[3].at;      /* (of no rows, and no address: but asked for, and so tokens are too many) */
        }
    }
    if (st < 0 || memories(args + 12, 1, &status)) return NULL;
    if (most > 0x7fffffff) st = 1;
    if (st == 0) {
        Py_BEGIN_ALLOW_THREADS
        st = p_pages(ctx, &b, t[0].at, t[1].at, t[2].at, (int32_t)t[2].size[0], t[3].at, t[4].at, t[5].at, t[6].at, t[7].at, t[8].at,
                     most < 0 ? 0 : (int32_t)most, status, stream);
        Py_END_ALLOW_THREADS
    }
    return PyLong_FromLong(st);
}

/* init_tensors(rope, rope_append, pages, bfloat16, int32, int64): the functions' addresses, torch's types */
static PyObject* init_tensors(PyObject* self, PyObject* const* args, Py_ssize_t n) {
    (void)self;
    void* a[3];
    if (count(n, 6) || integer(args[0], &a[0]) || integer(args[1], &a[1]) || integer(args[2], &a[2])) return NULL;
    memcpy(&p_rope, &a[0], sizeof(void*));
    memcpy(&p_rope_append, &a[1], sizeof(void*));
    memcpy(&p_pages, &a[2], sizeof(void*));
    Py_XSETREF(o_bf16, Py_NewRef(args[3]));
    Py_XSETREF(o_i32, Py_NewRef(args[4]));
    Py_XSETREF(o_i64, Py_NewRef(args[5]));
    PyObject* torch = PyImport_ImportModule("torch");
    PyObject* type = torch ? PyObject_GetAttrString(torch, "Tensor") : NULL;
    Py_XDECREF(torch);
    if (type && !PyType_Check(type)) PyErr_SetString(PyExc_TypeError, "torch.Tensor is no class");
    if (PyErr_Occurred()) {
        Py_XDECREF(type);
        return NULL;
    }
    Py_XSETREF(t_tensor, (PyTypeObject*)type);
    if (find(&data_ptr) || find(&get_device) || find(&strides) || find(&element_size) || find(&shape) || find(&dtype)) return NULL;
    Py_RETURN_NONE;
}

/* init(append, attention, kda, linear, BatchDesc, KdaDesc, LinearDesc): the functions' addresses in the loaded library, the
 * descriptions' types */
static PyObject* init(PyObject* self, PyObject* const* args, Py_ssize_t n) {
    (void)self;
    void* a[4];
    if (count(n, 7) || integer(args[0], &a[0]) || integer(args[1], &a[1]) || integer(args[2], &a[2]) || integer(args[3], &a[3])) return NULL;
    if (!PyType_Check(args[4]) || !PyType_Check(args[5]) || !PyType_Check(args[6])) {
        PyErr_SetString(PyExc_TypeError, "the descriptions' types");
        return NULL;
    }
    memcpy(&p_append, &a[0], sizeof(void*));
    memcpy(&p_attention, &a[1], sizeof(void*));
    memcpy(&p_kda, &a[2], sizeof(void*));
    memcpy(&p_linear, &a[3], sizeof(void*));
    Py_XSETREF(t_batch, Py_NewRef(args[4]));
    Py_XSETREF(t_kda, Py_NewRef(args[5]));
    Py_XSETREF(t_linear, Py_NewRef(args[6]));
    Py_RETURN_NONE;
}

static PyMethodDef methods[] = {
    {"init", (PyCFunction)(void (*)(void))init, METH_FASTCALL, NULL},
    {"kv_append", (PyCFunction)(void (*)(void))kv_append, METH_FASTCALL, NULL},
    {"attention", (PyCFunction)(void (*)(void))attention, METH_FASTCALL, NULL},
    {"kda_chunk", (PyCFunction)(void (*)(void))kda_chunk, METH_FASTCALL, NULL},
    {"linear_chunk", (PyCFunction)(void (*)(void))linear_chunk, METH_FASTCALL, NULL},
    {"init_tensors", (PyCFunction)(void (*)(void))init_tensors, METH_FASTCALL, NULL},
    {"rope", (PyCFunction)(void (*)(void))rope, METH_FASTCALL, NULL},
    {"rope_append", (PyCFunction)(void (*)(void))rope_append, METH_FASTCALL, NULL},
    {"pages", (PyCFunction)(void (*)(void))pages, METH_FASTCALL, NULL},
    {"code_pools", (PyCFunction)(void (*)(void))pools_of, METH_FASTCALL, NULL},
    {NULL, NULL, 0, NULL},
};
static struct PyModuleDef module = {PyModuleDef_HEAD_INIT, "_wpp_call", NULL, -1, methods, NULL, NULL, NULL, NULL};
PyMODINIT_FUNC PyInit__wpp_call(void) {
    member* const all[] = {&data_ptr, &get_device, &strides, &element_size, &shape, &dtype};
    no_args = PyTuple_New(0);
    for (int i = 0; no_args && i < 6; ++i)
        if (!(all[i]->name = PyUnicode_InternFromString(all[i]->text))) return NULL;
    return no_args ? PyModule_Create(&module) : NULL;
}
