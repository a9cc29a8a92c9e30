/* Argument marshalling of model_ops.py for ordinary calls.
 *
 * On a few rows the operators' kernels take less time than the checks, attribute reads and ctypes
 * conversions of their calls do in Python (one token through a block's norms: 3 us of kernel behind 17 us
 * of Python).  These functions do the same reads and checks in C.  They take a call on only if everything
 * is as usual and return -1 otherwise, also where the library refuses it: the caller then goes through its
 * own checks, which say what is wrong.  No tensor data is touched here.
 */
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <stdint.h>

#include "../../include/detonation_model.h"

/* the library's entry points, in the order that setup() takes their addresses in */
static int (*f_logprobs)(int64_t, int64_t, const deto_rows*, float, const void*, int, float*, float*, float*,
                         int32_t, int32_t*, float*, float*, void*, void*);
static int (*f_logprobs_backward)(int64_t, int64_t, const deto_rows*, float, const void*, int, const float*,
                                  const float*, const float*, const float*, const deto_rows*, void*);
static int64_t (*f_logprobs_workspace)(int64_t, int64_t, int32_t);
static int (*f_norm)(const deto_norm_residual*, int64_t, int64_t, const deto_rows*, const deto_rows*,
                     const deto_rows*, const deto_rows*, const deto_act8*, void*);
static int (*f_norm_backward)(const deto_norm_residual*, int64_t, int64_t, const deto_rows*, const deto_rows*,
                              const deto_rows*, const deto_rows*, const deto_rows*, const deto_rows*,
                              const deto_norm_grads*, void*, void*);
static int64_t (*f_norm_workspace)(const deto_norm_residual*, int64_t, int64_t);
static int (*f_encode)(int64_t, int64_t, const deto_rows*, const deto_act8*, void*);
static int (*f_decode)(int64_t, int64_t, const deto_act8*, const deto_rows*, void*);
static int (*f_glu_forward)(int, int64_t, int64_t, const deto_rows*, const deto_rows*, const deto_rows*,
                            const deto_act8*, const deto_act8*, void*);
static int (*f_glu_backward)(int, int64_t, int64_t, const deto_rows*, const deto_act8*, const deto_act8*,
                             const deto_rows*, const deto_rows*, const deto_act8*, void*);
static int (*f_weight_grad)(int64_t, int64_t, int64_t, const deto_rows*, const deto_act8*, const deto_rows*,
                            int, void*, void*);
static int64_t (*f_weight_grad_workspace)(int64_t, int64_t, int64_t);

/* and in that of setup_block() */
static int (*f_rotary)(const deto_rotary*, int64_t, const deto_rows*, const double*, const void*, int, const deto_rows*,
                       void*);
static int (*f_attention_forward)(const deto_attention*, int64_t, int64_t, const deto_rows*, const deto_rows*,
                                  const deto_rows*, const deto_rows*, float*, void*, void*);
static int (*f_attention_backward)(const deto_attention*, int64_t, int64_t, const deto_rows*, const deto_rows*,
                                   const deto_rows*, const deto_rows*, const float*, const deto_rows*, const deto_rows*,
                                   const deto_rows*, const deto_rows*, void*, void*);
static int64_t (*f_attention_workspace)(const deto_attention*, int64_t, int64_t);
static int (*f_dropout)(const deto_dropout*, int64_t, int64_t, const deto_rows*, const deto_rows*, const deto_rows*,
                        void*);

enum dt { DT_F32, DT_BF16, DT_F16, DT_I32, DT_I64, DT_I8, DT_U8, DT_F64, DT_COUNT };   /* the first three: deto_dtype */
static PyObject* dtypes[DT_COUNT];
static const int dt_size[DT_COUNT] = {4, 2, 2, 4, 8, 1, 1, 8};

static PyObject *fn_device, *fn_stream;
static int several;          /* devices: tensors say which one they are on */

static PyObject *s_is_cuda, *s_is_contiguous, *s_shape, *s_stride, *s_numel, *s_dtype, *s_data_ptr,
    *s_get_device, *s_codes, *s_exps, *s_pre, *s_post, *s_eps_pre, *s_eps_post, *s_scale, *s_rows_per_gate,
    *s_heads, *s_kv_heads, *s_head_dim, *s_rotary_dim, *s_layout, *s_magnitude, *s_first, *s_period, *s_causal,
    *s_sequences, *s_rate, *s_seed;

/* ---- reads; 0 where something is not as usual (a Python error may be set) */

static int truth_of(PyObject* o, PyObject* name) {
    PyObject* v = PyObject_GetAttr(o, name);
    if (!v) return 0;
    const int t = v == Py_True || (v != Py_False && PyObject_IsTrue(v) > 0);
    Py_DECREF(v);
    return t;
}

static int long_of(PyObject* o, PyObject* name, long long* out) {
    PyObject* v = PyObject_GetAttr(o, name);
    if (!v) return 0;
    const int ok = PyLong_Check(v);
    if (ok) *out = PyLong_AsLongLong(v);
    Py_DECREF(v);
    return ok && !PyErr_Occurred();
}

static int float_of(PyObject* o, PyObject* name, float* out) {
    PyObject* v = PyObject_GetAttr(o, name);
    if (!v) return 0;
    *out = (float)PyFloat_AsDouble(v);
    Py_DECREF(v);
    return !PyErr_Occurred();
}

static int call_long(PyObject* o, PyObject* method, long long* out) {
    PyObject* v = PyObject_CallMethodNoArgs(o, method);
    if (!v) return 0;
    *out = PyLong_AsLongLong(v);
    Py_DECREF(v);
    return !PyErr_Occurred();
}

struct call {
    long long device;
    void* stream;
};

/* the current device, and a stream handle (None: the device's current stream) */
static int begin(struct call* c, PyObject* given) {
    PyObject* dev = PyObject_CallNoArgs(fn_device);
    if (!dev) return 0;
    c->device = PyLong_AsLongLong(dev);
    if (given == Py_None) {
        PyObject* h = PyObject_CallOneArg(fn_stream, dev);
        Py_DECREF(dev);
        if (!h) return 0;
        c->stream = PyLong_AsVoidPtr(h);
        Py_DECREF(h);
    } else {
        Py_DECREF(dev);
        c->stream = PyLong_AsVoidPtr(given);
    }
    return !PyErr_Occurred();
}

/* type, address and whether a device tensor is contiguous */
static int tensor_of(const struct call* c, PyObject* t, int* dt, void** ptr, int* contiguous) {
    if (!truth_of(t, s_is_cuda)) return 0;
    if (several) {
        long long d;
        if (!call_long(t, s_get_device, &d) || d != c->device) return 0;
    }
    PyObject* v = PyObject_GetAttr(t, s_dtype);
    if (!v) return 0;
    for (*dt = 0; *dt < DT_COUNT; ++*dt)
        if (dtypes[*dt] == v) break;
    Py_DECREF(v);
    if (*dt == DT_COUNT) return 0;
    v = PyObject_CallMethodNoArgs(t, s_is_contiguous);
    if (!v) return 0;
    *contiguous = v == Py_True;
    Py_DECREF(v);
    v = PyObject_CallMethodNoArgs(t, s_data_ptr);
    if (!v) return 0;
    *ptr = PyLong_AsVoidPtr(v);
    Py_DECREF(v);
    return !PyErr_Occurred();
}

static int two(PyObject* tuple, long long* a, long long* b) {
    if (!tuple) return 0;
    int ok = PyTuple_Check(tuple) && PyTuple_GET_SIZE(tuple) == 2;
    if (ok) {
        *a = PyLong_AsLongLong(PyTuple_GET_ITEM(tuple, 0));
        *b = PyLong_AsLongLong(PyTuple_GET_ITEM(tuple, 1));
        ok = !PyErr_Occurred();
    }
    Py_DECREF(tuple);
    return ok;
}

struct matrix {
    deto_rows m;
    long long T, D;
    int dt;
};

/* rows of consecutive elements that do not overlap */
static int matrix_of(const struct call* c, PyObject* t, struct matrix* out) {
    int contiguous;
    long long ld, step;
    if (!tensor_of(c, t, &out->dt, &out->m.data, &contiguous) ||
        !two(PyObject_GetAttr(t, s_shape), &out->T, &out->D))
        return 0;
    out->m.dtype = out->dt;
    out->m.reserved = 0;
    out->m.ld = out->D > 1 ? out->D : 1;
    if (!contiguous) {
        if (!two(PyObject_CallMethodNoArgs(t, s_stride), &ld, &step)) return 0;
        if ((out->D > 1 && step != 1) || (out->T > 1 && ld < out->D)) return 0;
        if (out->T > 1) out->m.ld = ld;
    }
    return 1;
}

/* [T, D] of a floating type (one of them, or any: -1); None is an absent one where that is allowed */
static int rows_of(const struct call* c, PyObject* t, long long T, long long D, int dt, int may_be_absent,
                   deto_rows* out) {
    struct matrix m;
    if (t == Py_None) {
        out->data = NULL;
        return may_be_absent;
    }
    if (!matrix_of(c, t, &m) || m.T != T || m.D != D || m.dt > DT_F16 || (dt >= 0 && m.dt != dt)) return 0;
    *out = m.m;
    return 1;
}

static int act8_of(const struct call* c, PyObject* o, long long T, long long D, deto_act8* out) {
    struct matrix q, e;
    out->codes = NULL;
    out->exps = NULL;
    if (o == Py_None) return 1;
    PyObject* v = PyObject_GetAttr(o, s_codes);
    if (!v) return 0;
    int ok = matrix_of(c, v, &q) && q.dt == DT_I8 && q.T == T && q.D == D;
    Py_DECREF(v);
    if (!ok) return 0;
    v = PyObject_GetAttr(o, s_exps);
    if (!v) return 0;
    ok = matrix_of(c, v, &e) && e.dt == DT_U8 && e.T == T && e.D == (D + DETO_ACT8_GROUP - 1) / DETO_ACT8_GROUP;
    Py_DECREF(v);
    out->codes = (int8_t*)q.m.data;
    out->ld_codes = q.m.ld;
    out->exps = (uint8_t*)e.m.data;
    out->ld_exps = e.m.ld;
    return ok;
}

/* a contiguous tensor of `numel` elements of type `dt`; None: NULL */
static int vector_of(const struct call* c, PyObject* t, long long numel, int dt, void* out) {
    int got, contiguous;
    long long n;
    void* p;
    *(void**)out = NULL;
    if (t == Py_None) return 1;
    if (!tensor_of(c, t, &got, &p, &contiguous) || got != dt || !contiguous || !call_long(t, s_numel, &n) ||
        n != numel)
        return 0;
    *(void**)out = p;
    return 1;
}

static int scratch_of(const struct call* c, PyObject* t, int64_t bytes, void** out) {
    int dt, contiguous;
    long long n;
    *out = NULL;
    if (bytes <= 0) return bytes == 0;
    return t != Py_None && tensor_of(c, t, &dt, out, &contiguous) && contiguous && call_long(t, s_numel, &n) &&
           n * dt_size[dt] >= bytes;
}

/* rows of memory, in bytes */
struct span {
    const char* at;
    int64_t rows, step, wide;
};

static struct span span_of(const deto_rows* m, long long T, long long D) {
    const struct span s = {m->data, T, m->ld * dt_size[m->dtype], D * dt_size[m->dtype]};
    return s;
}

/* whether two of them share memory (columns of one matrix lie side by side; rows a different step apart are taken to
 * meet where the memory from the first one to the last does) */
static int meet(const struct span* a, const struct span* b) {
    if (!a->at || !b->at || a->rows < 1 || b->rows < 1) return 0;
    if (a->at + (a->rows - 1) * a->step + a->wide <= b->at || b->at + (b->rows - 1) * b->step + b->wide <= a->at)
        return 0;
    if ((a->rows == 1 && b->rows == 1) || (a->rows > 1 && b->rows > 1 && a->step != b->step)) return 1;
    const int64_t step = a->rows > 1 ? a->step : b->step;
    int64_t d = (b->at - a->at) % step;
    if (d < 0) d += step;
    return d < a->wide || d + b->wide > step;
}

/* What a call writes, its workspace included, and the matrices that it reads.  `twin`: outputs that may be the very
 * rows of an input. */
struct memory {
    struct span outs[8], ins[12];
    int twin_out[8], twin_in[12], n_outs, n_ins;
};

static void writes(struct memory* m, struct span s, int twin) {
    m->outs[m->n_outs] = s;
    m->twin_out[m->n_outs++] = twin;
}
static void reads(struct memory* m, struct span s, int twin) {
    m->ins[m->n_ins] = s;
    m->twin_in[m->n_ins++] = twin;
}
static struct span bytes_of(const void* at, int64_t n) {
    const struct span s = {at, 1, 0, n};
    return s;
}
static struct span codes_of(const deto_act8* q, long long T, long long D) {
    const struct span s = {(const char*)q->codes, T, q->ld_codes, D};
    return s;
}
static struct span exps_of(const deto_act8* q, long long T, long long D) {
    const struct span s = {(const char*)q->exps, T, q->ld_exps, (D + DETO_ACT8_GROUP - 1) / DETO_ACT8_GROUP};
    return s;
}
static void writes8(struct memory* m, const deto_act8* q, long long T, long long D) {
    writes(m, codes_of(q, T, D), 0);
    writes(m, exps_of(q, T, D), 0);
}
static void reads8(struct memory* m, const deto_act8* q, long long T, long long D) {
    reads(m, codes_of(q, T, D), 0);
    reads(m, exps_of(q, T, D), 0);
}

/* no output meets another one, or an input, except as its twin */
static int apart(const struct memory* m) {
    for (int i = 0; i < m->n_outs; ++i) {
        const struct span* o = &m->outs[i];
        for (int j = i + 1; j < m->n_outs; ++j)
            if (meet(o, &m->outs[j])) return 0;
        for (int j = 0; j < m->n_ins; ++j) {
            const struct span* in = &m->ins[j];
            const int same = o->at == in->at && o->step == in->step && o->wide == in->wide;
            if (!(same && m->twin_out[i] && m->twin_in[j]) && meet(o, in)) return 0;
        }
    }
    return 1;
}

static PyObject* unusual(void) {
    PyErr_Clear();
    return PyLong_FromLong(-1);
}
static PyObject* answer(int rc) { return PyLong_FromLong(rc == DETO_OK || rc == DETO_ERR_HIP ? rc : -1); }

#define OPTIONAL(r) ((r).data ? &(r) : NULL)
#define OPTIONAL8(q) ((q).codes ? &(q) : NULL)
/* a call into the library, without the interpreter's lock */
#define RUN(expression)          \
    int rc;                      \
    Py_BEGIN_ALLOW_THREADS       \
    rc = (expression);           \
    Py_END_ALLOW_THREADS         \
    return answer(rc)

/* ---- the calls */

/* targets: int64 or int32 */
static int targets_of(const struct call* c, PyObject* t, long long T, void** out, int* bytes) {
    int dt, contiguous;
    long long n;
    if (!tensor_of(c, t, &dt, out, &contiguous) || !contiguous || (dt != DT_I64 && dt != DT_I32) ||
        !call_long(t, s_numel, &n) || n != T)
        return 0;
    *bytes = dt_size[dt];
    return 1;
}

/* (logits, targets, logp, lse, entropy, top_idx, top_logp, stats, logit_scale, workspace, stream) */
static PyObject* py_logprobs(PyObject* self, PyObject* const* a, Py_ssize_t count) {
    (void)self;
    struct call c;
    struct matrix x, best;
    void *y, *ws;
    float *logp, *lse, *entropy, *top_logp, *stats;
    int32_t* top_idx = NULL;
    int yb;
    long long top = 0;
    if (count != 11 || !begin(&c, a[10]) || !matrix_of(&c, a[0], &x) || x.dt > DT_F16 ||
        !targets_of(&c, a[1], x.T, &y, &yb) || a[2] == Py_None || !vector_of(&c, a[2], x.T, DT_F32, &logp) ||
        !vector_of(&c, a[3], x.T, DT_F32, &lse) || !vector_of(&c, a[4], x.T, DT_F32, &entropy))
        return unusual();
    if (a[5] != Py_None) {
        if (!matrix_of(&c, a[5], &best) || best.dt != DT_I32 || best.T != x.T || (best.T > 1 && best.m.ld != best.D))
            return unusual();
        top = best.D;
        top_idx = (int32_t*)best.m.data;
    } else if (a[6] != Py_None) {
        return unusual();
    }
    const double scale = PyFloat_AsDouble(a[8]);
    if (!vector_of(&c, a[6], x.T * top, DT_F32, &top_logp) || !vector_of(&c, a[7], 2 * x.T, DT_F32, &stats) ||
        PyErr_Occurred() || top > 32)
        return unusual();
    const int64_t need = f_logprobs_workspace(x.T, x.D, (int32_t)top);
    if (!scratch_of(&c, a[9], need, &ws)) return unusual();
    struct memory mem = {.n_outs = 0};
    writes(&mem, bytes_of(ws, need), 0);
    reads(&mem, span_of(&x.m, x.T, x.D), 0);
    if (!apart(&mem)) return unusual();
    RUN(f_logprobs(x.T, x.D, &x.m, (float)scale, y, yb, logp, lse, entropy, (int32_t)top, top_idx, top_logp, stats,
                   ws, c.stream));
}

/* (logits, targets, stats, dlogits, g_logp, entropy, g_entropy, logit_scale, stream) */
static PyObject* py_logprobs_backward(PyObject* self, PyObject* const* a, Py_ssize_t count) {
    (void)self;
    struct call c;
    struct memory mem = {.n_outs = 0};
    struct matrix x;
    deto_rows dx;
    void* y;
    float *stats, *g, *entropy, *ge;
    int yb;
    if (count != 9 || !begin(&c, a[8]) || !matrix_of(&c, a[0], &x) || x.dt > DT_F16 ||
        !targets_of(&c, a[1], x.T, &y, &yb) || a[2] == Py_None || !vector_of(&c, a[2], 2 * x.T, DT_F32, &stats) ||
        !rows_of(&c, a[3], x.T, x.D, x.dt, 0, &dx) ||
        !vector_of(&c, a[4], x.T, DT_F32, &g) || !vector_of(&c, a[5], x.T, DT_F32, &entropy) ||
        !vector_of(&c, a[6], x.T, DT_F32, &ge))
        return unusual();
    const double scale = PyFloat_AsDouble(a[7]);
    writes(&mem, span_of(&dx, x.T, x.D), 1);
    reads(&mem, span_of(&x.m, x.T, x.D), 1);
    if (PyErr_Occurred() || !apart(&mem)) return unusual();
    RUN(f_logprobs_backward(x.T, x.D, &x.m, (float)scale, y, yb, stats, entropy, g, ge, &dx, c.stream));
}

/* cfg, and gate, w_post, b_post, w_pre, b_pre in a[0 .. 4] (vectors and the gate of one type) */
static int norm_of(const struct call* c, PyObject* cfg, PyObject* const* a, long long T, long long D,
                   deto_norm_residual* s, long long* gates, struct memory* mem) {
    long long pre, post, per;
    if (!long_of(cfg, s_pre, &pre) || !long_of(cfg, s_post, &post) || !float_of(cfg, s_eps_pre, &s->eps_pre) ||
        !float_of(cfg, s_eps_post, &s->eps_post) || !float_of(cfg, s_scale, &s->scale) ||
        !long_of(cfg, s_rows_per_gate, &per) || per < 0 || pre < 0 || pre > 2 || post < 0 || post > 2)
        return 0;
    s->pre = (int32_t)pre;
    s->post = (int32_t)post;
    s->rows_per_gate = per;
    s->gate = NULL;
    s->ld_gate = D;
    s->param_dtype = DETO_F32;
    *gates = per ? (T + per - 1) / per : 1;
    const void** at[5] = {&s->gate, &s->w_post, &s->b_post, &s->w_pre, &s->b_pre};
    int dtype = -1;
    for (int i = 0; i < 5; ++i) {
        int dt, contiguous;
        void* p;
        long long n, rows, columns;
        *at[i] = NULL;
        if (a[i] == Py_None) continue;
        if (!tensor_of(c, a[i], &dt, &p, &contiguous) || dt > DT_F16 || !contiguous ||
            !call_long(a[i], s_numel, &n) || n != (i ? 1 : *gates) * D || (dtype >= 0 && dt != dtype))
            return 0;
        if (i == 0 && *gates > 1 &&          /* as many elements may lie the other way round */
            (!two(PyObject_GetAttr(a[i], s_shape), &rows, &columns) || rows != *gates || columns != D))
            return 0;
        *at[i] = p;
        dtype = dt;
        reads(mem, bytes_of(p, n * dt_size[dt]), 0);
    }
    if (dtype >= 0) s->param_dtype = dtype;
    return 1;
}

/* (cfg, x, f, x_out, y, y8, gate, w_post, b_post, w_pre, b_pre, stream) */
static PyObject* py_norm(PyObject* self, PyObject* const* a, Py_ssize_t count) {
    (void)self;
    struct call c;
    struct matrix x;
    deto_rows f, x_out, y;
    deto_act8 y8;
    deto_norm_residual s;
    struct memory mem = {.n_outs = 0};
    long long gates;
    if (count != 12 || !begin(&c, a[11]) || !matrix_of(&c, a[1], &x) || x.dt > DT_F16 ||
        !norm_of(&c, a[0], a + 6, x.T, x.D, &s, &gates, &mem) || !rows_of(&c, a[2], x.T, x.D, -1, 1, &f) ||
        !rows_of(&c, a[3], x.T, x.D, x.dt, 1, &x_out) ||
        !rows_of(&c, a[4], x.T, x.D, f.data ? f.dtype : -1, 1, &y) || !act8_of(&c, a[5], x.T, x.D, &y8))
        return unusual();
    if (x_out.data) writes(&mem, span_of(&x_out, x.T, x.D), 1);
    if (y.data) writes(&mem, span_of(&y, x.T, x.D), 0);
    if (y8.codes) writes8(&mem, &y8, x.T, x.D);
    reads(&mem, span_of(&x.m, x.T, x.D), 1);
    if (f.data) reads(&mem, span_of(&f, x.T, x.D), 0);
    if (!apart(&mem)) return unusual();
    RUN(f_norm(&s, x.T, x.D, &x.m, OPTIONAL(f), OPTIONAL(x_out), OPTIONAL(y), OPTIONAL8(y8), c.stream));
}

/* (cfg, x_out, f, dy, dx_out, dx, df, workspace, gate, w_post, b_post, w_pre, dgate, dw_post, db_post, dw_pre,
 * db_pre, stream) */
static PyObject* py_norm_backward(PyObject* self, PyObject* const* a, Py_ssize_t count) {
    (void)self;
    struct call c;
    struct matrix x;
    deto_rows f, dy, dxo, dx, df;
    deto_norm_residual s;
    deto_norm_grads g;
    struct memory mem = {.n_outs = 0};
    long long gates;
    void* ws = NULL;
    if (count != 18) return unusual();
    PyObject* const params[5] = {a[8], a[9], a[10], a[11], Py_None};
    if (!begin(&c, a[17]) || !matrix_of(&c, a[1], &x) || x.dt > DT_F16 ||
        !norm_of(&c, a[0], params, x.T, x.D, &s, &gates, &mem) || !rows_of(&c, a[2], x.T, x.D, -1, 1, &f) ||
        !rows_of(&c, a[3], x.T, x.D, f.data ? f.dtype : -1, 1, &dy) ||
        !rows_of(&c, a[4], x.T, x.D, x.dt, 1, &dxo) || !rows_of(&c, a[5], x.T, x.D, x.dt, 0, &dx) ||
        !rows_of(&c, a[6], x.T, x.D, f.data ? f.dtype : -1, 1, &df) ||
        !vector_of(&c, a[12], gates * x.D, DT_F32, &g.gate) || !vector_of(&c, a[13], x.D, DT_F32, &g.w_post) ||
        !vector_of(&c, a[14], x.D, DT_F32, &g.b_post) || !vector_of(&c, a[15], x.D, DT_F32, &g.w_pre) ||
        !vector_of(&c, a[16], x.D, DT_F32, &g.b_pre))
        return unusual();
    if (g.gate || g.w_post || g.b_post || g.w_pre || g.b_pre) {
        const int64_t need = f_norm_workspace(&s, x.T, x.D);
        if (!scratch_of(&c, a[7], need, &ws)) return unusual();
        writes(&mem, bytes_of(ws, need), 0);
    }
    writes(&mem, span_of(&dx, x.T, x.D), 1);
    if (df.data) writes(&mem, span_of(&df, x.T, x.D), 0);
    reads(&mem, span_of(&x.m, x.T, x.D), 0);
    if (f.data) reads(&mem, span_of(&f, x.T, x.D), 0);
    if (dy.data) reads(&mem, span_of(&dy, x.T, x.D), 0);
    if (dxo.data) reads(&mem, span_of(&dxo, x.T, x.D), 1);
    if (!apart(&mem)) return unusual();
    RUN(f_norm_backward(&s, x.T, x.D, &x.m, OPTIONAL(f), OPTIONAL(dy), OPTIONAL(dxo), &dx, OPTIONAL(df), &g, ws,
                        c.stream));
}

/* (x, x8, stream) and (x8, x, stream) */
static PyObject* codec(PyObject* x, PyObject* x8, PyObject* stream, int encode) {
    struct call c;
    struct matrix m;
    deto_act8 q;
    if (!begin(&c, stream) || !matrix_of(&c, x, &m) || m.dt > DT_F16 || x8 == Py_None ||
        !act8_of(&c, x8, m.T, m.D, &q))
        return unusual();
    struct memory mem = {.n_outs = 0};
    if (encode) {
        writes8(&mem, &q, m.T, m.D);
        reads(&mem, span_of(&m.m, m.T, m.D), 0);
    } else {
        writes(&mem, span_of(&m.m, m.T, m.D), 0);
        reads8(&mem, &q, m.T, m.D);
    }
    if (!apart(&mem)) return unusual();
    RUN(encode ? f_encode(m.T, m.D, &m.m, &q, c.stream) : f_decode(m.T, m.D, &q, &m.m, c.stream));
}
static PyObject* py_encode(PyObject* self, PyObject* const* a, Py_ssize_t count) {
    (void)self;
    return count == 3 ? codec(a[0], a[1], a[2], 1) : unusual();
}
static PyObject* py_decode(PyObject* self, PyObject* const* a, Py_ssize_t count) {
    (void)self;
    return count == 3 ? codec(a[1], a[0], a[2], 0) : unusual();
}

static int act_of(PyObject* o, int* out) {
    if (!PyLong_Check(o)) return 0;
    const long v = PyLong_AsLong(o);
    *out = (int)v;
    return !PyErr_Occurred() && v >= 0 && v <= 3;
}

/* (act, a, b, h, a8, b8, stream) */
static PyObject* py_glu_forward(PyObject* self, PyObject* const* a, Py_ssize_t count) {
    (void)self;
    struct call c;
    struct matrix m;
    deto_rows b, h;
    deto_act8 a8, b8;
    int act;
    if (count != 7 || !act_of(a[0], &act) || !begin(&c, a[6]) || !matrix_of(&c, a[1], &m) || m.dt > DT_F16 ||
        !rows_of(&c, a[2], m.T, m.D, m.dt, 1, &b) || !rows_of(&c, a[3], m.T, m.D, m.dt, 0, &h) ||
        !act8_of(&c, a[4], m.T, m.D, &a8) || !act8_of(&c, a[5], m.T, m.D, &b8))
        return unusual();
    struct memory mem = {.n_outs = 0};
    writes(&mem, span_of(&h, m.T, m.D), 1);
    if (a8.codes) writes8(&mem, &a8, m.T, m.D);
    if (b8.codes) writes8(&mem, &b8, m.T, m.D);
    reads(&mem, span_of(&m.m, m.T, m.D), 1);
    if (b.data) reads(&mem, span_of(&b, m.T, m.D), 1);
    if (!apart(&mem)) return unusual();
    RUN(f_glu_forward(act, m.T, m.D, &m.m, OPTIONAL(b), &h, OPTIONAL8(a8), OPTIONAL8(b8), c.stream));
}

/* (act, dh, a8, b8, da, db, h8, stream) */
static PyObject* py_glu_backward(PyObject* self, PyObject* const* a, Py_ssize_t count) {
    (void)self;
    struct call c;
    struct matrix m;
    deto_rows da, db;
    deto_act8 a8, b8, h8;
    int act;
    if (count != 8 || !act_of(a[0], &act) || !begin(&c, a[7]) || !matrix_of(&c, a[1], &m) || m.dt > DT_F16 ||
        a[2] == Py_None || !act8_of(&c, a[2], m.T, m.D, &a8) || !act8_of(&c, a[3], m.T, m.D, &b8) ||
        !rows_of(&c, a[4], m.T, m.D, m.dt, 0, &da) || !rows_of(&c, a[5], m.T, m.D, m.dt, 1, &db) ||
        !act8_of(&c, a[6], m.T, m.D, &h8))
        return unusual();
    struct memory mem = {.n_outs = 0};
    writes(&mem, span_of(&da, m.T, m.D), 1);
    if (db.data) writes(&mem, span_of(&db, m.T, m.D), 1);
    if (h8.codes) writes8(&mem, &h8, m.T, m.D);
    reads(&mem, span_of(&m.m, m.T, m.D), 1);
    reads8(&mem, &a8, m.T, m.D);
    if (b8.codes) reads8(&mem, &b8, m.T, m.D);
    if (!apart(&mem)) return unusual();
    RUN(f_glu_backward(act, m.T, m.D, &m.m, &a8, OPTIONAL8(b8), &da, OPTIONAL(db), OPTIONAL8(h8), c.stream));
}

/* (dy, x8, dw, accumulate, workspace, stream) */
static PyObject* py_weight_grad(PyObject* self, PyObject* const* a, Py_ssize_t count) {
    (void)self;
    struct call c;
    struct matrix dy, dw;
    deto_act8 x;
    void* ws;
    if (count != 6 || !PyBool_Check(a[3]) || !begin(&c, a[5]) || !matrix_of(&c, a[0], &dy) || dy.dt > DT_F16 ||
        !matrix_of(&c, a[2], &dw) || dw.dt > DT_F16 || dw.T != dy.D || a[1] == Py_None ||
        !act8_of(&c, a[1], dy.T, dw.D, &x))
        return unusual();
    const int64_t need = f_weight_grad_workspace(dy.T, dy.D, dw.D);
    if (!scratch_of(&c, a[4], need, &ws)) return unusual();
    struct memory mem = {.n_outs = 0};
    writes(&mem, span_of(&dw.m, dw.T, dw.D), 0);
    writes(&mem, bytes_of(ws, need), 0);
    reads(&mem, span_of(&dy.m, dy.T, dy.D), 0);
    reads8(&mem, &x, dy.T, dw.D);
    if (!apart(&mem)) return unusual();
    RUN(f_weight_grad(dy.T, dy.D, dw.D, &dy.m, &x, &dw.m, a[3] == Py_True, ws, c.stream));
}

/* a number of 32 bits */
static int int_of(PyObject* o, PyObject* name, int32_t* out) {
    long long v;
    if (!long_of(o, name, &v) || v != (int32_t)v) return 0;
    *out = (int32_t)v;
    return 1;
}

/* a matrix that the call reads, or writes */
static int part_of(const struct call* c, struct memory* mem, PyObject* t, long long T, long long D, int dt, int written,
                   deto_rows* out) {
    if (!rows_of(c, t, T, D, dt, 0, out)) return 0;
    if (written) writes(mem, span_of(out, T, D), 0);
    else reads(mem, span_of(out, T, D), 0);
    return 1;
}

/* (cfg, x, freqs, out, positions, inverse, stream) */
static PyObject* py_rotary(PyObject* self, PyObject* const* a, Py_ssize_t count) {
    (void)self;
    struct call c;
    struct matrix x;
    deto_rows out;
    deto_rotary s;
    struct memory mem = {.n_outs = 0};
    double* freqs;
    long long first, period;
    void* positions = NULL;
    int bytes = 0;
    if (count != 7 || !PyBool_Check(a[5]) || !int_of(a[0], s_heads, &s.heads) || !int_of(a[0], s_head_dim, &s.head_dim) ||
        !int_of(a[0], s_rotary_dim, &s.rotary_dim) || !int_of(a[0], s_layout, &s.layout) ||
        !float_of(a[0], s_magnitude, &s.magnitude) || !long_of(a[0], s_first, &first) ||
        !long_of(a[0], s_period, &period) || !begin(&c, a[6]) || !matrix_of(&c, a[1], &x) || x.dt > DT_F16 ||
        x.D != (long long)s.heads * s.head_dim || !rows_of(&c, a[3], x.T, x.D, x.dt, 0, &out))
        return unusual();
    if (!s.rotary_dim) s.rotary_dim = s.head_dim;
    s.inverse = a[5] == Py_True;
    s.first = first;
    s.period = period;
    if (a[2] == Py_None || !vector_of(&c, a[2], s.rotary_dim / 2, DT_F64, &freqs) ||
        (a[4] != Py_None && !targets_of(&c, a[4], x.T, &positions, &bytes)))
        return unusual();
    writes(&mem, span_of(&out, x.T, x.D), 1);
    reads(&mem, span_of(&x.m, x.T, x.D), 1);
    reads(&mem, bytes_of(freqs, s.rotary_dim / 2 * 8), 0);
    if (positions) reads(&mem, bytes_of(positions, x.T * bytes), 0);
    if (!apart(&mem)) return unusual();
    RUN(f_rotary(&s, x.T, &x.m, freqs, positions, bytes, &out, c.stream));
}

/* cfg, and q_starts and k_starts in a[0] and a[1] */
static int attention_of(const struct call* c, PyObject* cfg, PyObject* const* a, deto_attention* s, struct memory* mem) {
    long long sequences;
    int32_t *qs, *ks;
    if (!int_of(cfg, s_heads, &s->heads) || !int_of(cfg, s_kv_heads, &s->kv_heads) ||
        !int_of(cfg, s_head_dim, &s->head_dim) || !float_of(cfg, s_scale, &s->scale) ||
        !long_of(cfg, s_sequences, &sequences) || sequences < 1 || sequences > INT32_MAX ||
        !vector_of(c, a[0], sequences + 1, DT_I32, &qs) || !vector_of(c, a[1], sequences + 1, DT_I32, &ks))
        return 0;
    if (!s->kv_heads) s->kv_heads = s->heads;
    s->causal = truth_of(cfg, s_causal);
    s->reserved = 0;
    s->sequences = sequences;
    s->q_starts = qs;
    s->k_starts = ks;
    if (qs) reads(mem, bytes_of(qs, (sequences + 1) * 4), 0);
    if (ks) reads(mem, bytes_of(ks, (sequences + 1) * 4), 0);
    return !PyErr_Occurred();
}

/* (cfg, q, k, v, out, lse, q_starts, k_starts, workspace, stream) */
static PyObject* py_attention_forward(PyObject* self, PyObject* const* a, Py_ssize_t count) {
    (void)self;
    struct call c;
    struct matrix q, k;
    deto_rows v, out;
    deto_attention s;
    struct memory mem = {.n_outs = 0};
    float* lse;
    void* ws;
    if (count != 10 || !begin(&c, a[9]) || !attention_of(&c, a[0], a + 6, &s, &mem) || !matrix_of(&c, a[1], &q) ||
        q.dt > DT_F16 || q.D != (long long)s.heads * s.head_dim || !matrix_of(&c, a[2], &k) || k.dt != q.dt ||
        k.D != (long long)s.kv_heads * s.head_dim || !part_of(&c, &mem, a[3], k.T, k.D, q.dt, 0, &v) ||
        !part_of(&c, &mem, a[4], q.T, q.D, q.dt, 1, &out) || !vector_of(&c, a[5], s.heads * q.T, DT_F32, &lse))
        return unusual();
    const int64_t need = f_attention_workspace(&s, q.T, k.T);
    if (!scratch_of(&c, a[8], need, &ws)) return unusual();
    reads(&mem, span_of(&q.m, q.T, q.D), 0);
    reads(&mem, span_of(&k.m, k.T, k.D), 0);
    writes(&mem, bytes_of(lse, s.heads * q.T * 4), 0);
    writes(&mem, bytes_of(ws, need), 0);
    if (!apart(&mem)) return unusual();
    RUN(f_attention_forward(&s, q.T, k.T, &q.m, &k.m, &v, &out, lse, ws, c.stream));
}

/* (cfg, q, k, v, out, lse, dout, dq, dk, dv, q_starts, k_starts, workspace, stream) */
static PyObject* py_attention_backward(PyObject* self, PyObject* const* a, Py_ssize_t count) {
    (void)self;
    struct call c;
    struct matrix q, k;
    deto_rows v, out, dout, dq, dk, dv;
    deto_attention s;
    struct memory mem = {.n_outs = 0};
    float* lse;
    void* ws;
    if (count != 14 || !begin(&c, a[13]) || !attention_of(&c, a[0], a + 10, &s, &mem) || !matrix_of(&c, a[1], &q) ||
        q.dt > DT_F16 || q.D != (long long)s.heads * s.head_dim || !matrix_of(&c, a[2], &k) || k.dt != q.dt ||
        k.D != (long long)s.kv_heads * s.head_dim || !part_of(&c, &mem, a[3], k.T, k.D, q.dt, 0, &v) ||
        !part_of(&c, &mem, a[4], q.T, q.D, q.dt, 0, &out) || a[5] == Py_None ||
        !vector_of(&c, a[5], s.heads * q.T, DT_F32, &lse) || !part_of(&c, &mem, a[6], q.T, q.D, q.dt, 0, &dout) ||
        !part_of(&c, &mem, a[7], q.T, q.D, q.dt, 1, &dq) || !part_of(&c, &mem, a[8], k.T, k.D, q.dt, 1, &dk) ||
        !part_of(&c, &mem, a[9], k.T, k.D, q.dt, 1, &dv))
        return unusual();
    const int64_t need = f_attention_workspace(&s, q.T, k.T);
    if (!scratch_of(&c, a[12], need, &ws)) return unusual();
    reads(&mem, span_of(&q.m, q.T, q.D), 0);
    reads(&mem, span_of(&k.m, k.T, k.D), 0);
    reads(&mem, bytes_of(lse, s.heads * q.T * 4), 0);
    writes(&mem, bytes_of(ws, need), 0);
    if (!apart(&mem)) return unusual();
    RUN(f_attention_backward(&s, q.T, k.T, &q.m, &k.m, &v, &out, lse, &dout, &dq, &dk, &dv, ws, c.stream));
}

/* (cfg, x, out, residual, offset, device_offset, stream) */
static PyObject* py_dropout(PyObject* self, PyObject* const* a, Py_ssize_t count) {
    (void)self;
    struct call c;
    struct matrix x, out;
    deto_rows residual;
    deto_dropout s;
    struct memory mem = {.n_outs = 0};
    uint64_t* more;
    if (count != 7 || !PyLong_Check(a[4]) || !float_of(a[0], s_rate, &s.rate)) return unusual();
    PyObject* seed = PyObject_GetAttr(a[0], s_seed);
    if (!seed) return unusual();
    const int whole = PyLong_Check(seed);
    s.seed = whole ? PyLong_AsUnsignedLongLong(seed) : 0;
    Py_DECREF(seed);
    if (!whole || PyErr_Occurred()) return unusual();
    s.offset = PyLong_AsUnsignedLongLong(a[4]);
    s.reserved = 0;
    if (PyErr_Occurred() || !begin(&c, a[6]) || !matrix_of(&c, a[1], &x) || x.dt > DT_F16 ||
        !matrix_of(&c, a[2], &out) || out.dt > DT_F16 || out.T != x.T || out.D != x.D ||
        !rows_of(&c, a[3], x.T, x.D, out.dt, 1, &residual) || !vector_of(&c, a[5], 1, DT_I64, &more))
        return unusual();
    s.device_offset = more;
    /* in place where types are the same: an element's bytes are then its own */
    writes(&mem, span_of(&out.m, x.T, x.D), 1);
    reads(&mem, span_of(&x.m, x.T, x.D), x.dt == out.dt);
    if (residual.data) reads(&mem, span_of(&residual, x.T, x.D), 1);
    if (more) reads(&mem, bytes_of(more, 8), 0);
    if (!apart(&mem)) return unusual();
    RUN(f_dropout(&s, x.T, x.D, &x.m, OPTIONAL(residual), &out.m, c.stream));
}

/* setup_block(addresses of the entry points of an attention block, in the order of _MARSHALLED_BLOCK) */
static PyObject* py_setup_block(PyObject* self, PyObject* f) {
    (void)self;
    void** const at[] = {(void**)&f_rotary, (void**)&f_attention_forward, (void**)&f_attention_backward,
                         (void**)&f_attention_workspace, (void**)&f_dropout};
    const Py_ssize_t entries = (Py_ssize_t)(sizeof(at) / sizeof(at[0]));
    if (!PyTuple_Check(f) || PyTuple_GET_SIZE(f) != entries) {
        PyErr_SetString(PyExc_ValueError, "setup_block: wrong number of entry points");
        return NULL;
    }
    for (Py_ssize_t i = 0; i < entries; ++i) {
        *at[i] = PyLong_AsVoidPtr(PyTuple_GET_ITEM(f, i));
        if (PyErr_Occurred()) return NULL;
    }
    Py_RETURN_NONE;
}

/* setup(addresses of the entry points, torch's dtypes in the order of enum dt, current device, current stream of
 * a device, devices) */
static PyObject* py_setup(PyObject* self, PyObject* args) {
    (void)self;
    PyObject *f, *d, *device, *stream;
    int devices;
    if (!PyArg_ParseTuple(args, "O!O!OOi", &PyTuple_Type, &f, &PyTuple_Type, &d, &device, &stream, &devices))
        return NULL;
    void** const at[] = {(void**)&f_logprobs, (void**)&f_logprobs_backward, (void**)&f_logprobs_workspace,
                         (void**)&f_norm, (void**)&f_norm_backward, (void**)&f_norm_workspace,
                         (void**)&f_encode, (void**)&f_decode, (void**)&f_glu_forward,
                         (void**)&f_glu_backward, (void**)&f_weight_grad, (void**)&f_weight_grad_workspace};
    const Py_ssize_t entries = (Py_ssize_t)(sizeof(at) / sizeof(at[0]));
    if (PyTuple_GET_SIZE(f) != entries || PyTuple_GET_SIZE(d) != DT_COUNT) {
        PyErr_SetString(PyExc_ValueError, "setup: wrong number of entry points or types");
        return NULL;
    }
    for (Py_ssize_t i = 0; i < entries; ++i) {
        *at[i] = PyLong_AsVoidPtr(PyTuple_GET_ITEM(f, i));
        if (PyErr_Occurred()) return NULL;
    }
    for (int i = 0; i < DT_COUNT; ++i) {
        PyObject* t = PyTuple_GET_ITEM(d, i);
        Py_INCREF(t);
        Py_XSETREF(dtypes[i], t);
    }
    Py_INCREF(device);
    Py_INCREF(stream);
    Py_XSETREF(fn_device, device);
    Py_XSETREF(fn_stream, stream);
    several = devices != 1;
    Py_RETURN_NONE;
}

#define FAST(name, fn) {name, (PyCFunction)(void (*)(void))fn, METH_FASTCALL, "status, or -1"}
static PyMethodDef methods[] = {
    {"setup", py_setup, METH_VARARGS, "entry points and torch's dtypes"},
    FAST("logprobs", py_logprobs), FAST("logprobs_backward", py_logprobs_backward), FAST("norm", py_norm),
    FAST("norm_backward", py_norm_backward), FAST("encode", py_encode), FAST("decode", py_decode),
    FAST("glu_forward", py_glu_forward), FAST("glu_backward", py_glu_backward),
    FAST("weight_grad", py_weight_grad),
    {"setup_block", py_setup_block, METH_O, "entry points of an attention block"}, FAST("rotary", py_rotary),
    FAST("attention_forward", py_attention_forward), FAST("attention_backward", py_attention_backward),
    FAST("dropout", py_dropout), {NULL, NULL, 0, NULL}};

static struct PyModuleDef module = {PyModuleDef_HEAD_INIT, "_model_marshal", NULL, -1, methods,
                                    NULL, NULL, NULL, NULL};

PyMODINIT_FUNC PyInit__model_marshal(void) {
    struct { PyObject** at; const char* name; } names[] = {
        {&s_is_cuda, "is_cuda"}, {&s_is_contiguous, "is_contiguous"}, {&s_shape, "shape"},
        {&s_stride, "stride"}, {&s_numel, "numel"}, {&s_dtype, "dtype"}, {&s_data_ptr, "data_ptr"},
        {&s_get_device, "get_device"}, {&s_codes, "codes"}, {&s_exps, "exps"}, {&s_pre, "pre"},
        {&s_post, "post"}, {&s_eps_pre, "eps_pre"}, {&s_eps_post, "eps_post"}, {&s_scale, "scale"},
        {&s_rows_per_gate, "rows_per_gate"}, {&s_heads, "heads"}, {&s_kv_heads, "kv_heads"},
        {&s_head_dim, "head_dim"}, {&s_rotary_dim, "rotary_dim"}, {&s_layout, "layout"}, {&s_magnitude, "magnitude"},
        {&s_first, "first"}, {&s_period, "period"}, {&s_causal, "causal"}, {&s_sequences, "sequences"},
        {&s_rate, "rate"}, {&s_seed, "seed"}};
    for (size_t i = 0; i < sizeof(names) / sizeof(names[0]); ++i)
        if (!(*names[i].at = PyUnicode_InternFromString(names[i].name))) return NULL;
    return PyModule_Create(&module);
}
