/* The fused layer calls of binding.py as native functions: a small layer's kernels are shorter than its marshalling through ctypes
 * (4.8 us on the host for the 19 arguments of a linear; 1.7 here).  The functions take what the Python ones take, ask a
 * tensor for its address, shape, pitch and type through its Python attributes, and call the C entry points, whose addresses
 * binding.py hands over (bind): nothing is linked against either library, and the GIL is released during the call. */
#define PY_SSIZE_T_CLEAN
#include <Python.h>
#include <limits.h>
#include <stdint.h>

#include "../../include/hq.h"

typedef hq_status (*qlinear_fn)(const void*, hq_dtype, int64_t, int64_t, int64_t, const hq_weight_desc*, const void*, const float*,
                                const float*, int, hq_scale_mode, const float*, void*, hq_dtype, int64_t, void*, size_t, int32_t*, void*);
typedef hq_status (*qconv_fn)(const void*, hq_dtype, int64_t, int64_t, int64_t, int64_t, const hq_weight_desc*, const void*, int, int, int,
                              int, const float*, const float*, int, hq_scale_mode, const float*, void*, hq_dtype, void*, size_t, int32_t*,
                              void*);
typedef hq_status (*ln_qlinear_fn)(const void*, hq_dtype, int64_t, int64_t, int64_t, const float*, const float*, int64_t, float,
                                   const hq_weight_desc*, const void*, const float*, const float*, int, void*, hq_dtype, int64_t, void*,
                                   size_t, int32_t*, void*);
typedef hq_status (*quant_fn)(const void*, hq_dtype, int64_t, int64_t, int64_t, int, int, hq_scale_mode, const float*, void*, hq_container,
                              int64_t, float*, void*);
static qlinear_fn f_qlinear;
static qconv_fn f_qconv;
static ln_qlinear_fn f_ln_qlinear;
static quant_fn f_quant;

static PyObject *s_data_ptr, *s_shape, *s_stride, *s_dtype, *s_nbytes, *s_desc, *s_blob_dev, *s_s_w_dev, *zero;
static PyObject* dtype_code;              /* binding.py's function, asked once per type */
static PyObject* known_dtype[2];
static int known_code[2];

static int address(PyObject* t, void** out) {
    *out = NULL;
    if (t == Py_None) return 0;
    PyObject* v = PyObject_CallMethodNoArgs(t, s_data_ptr);
    if (v == NULL) return -1;
    *out = PyLong_AsVoidPtr(v);
    Py_DECREF(v);
    return PyErr_Occurred() ? -1 : 0;
}
static int attr_address(PyObject* o, PyObject* name, void** out) {
    PyObject* t = PyObject_GetAttr(o, name);
    if (t == NULL) return -1;
    const int r = address(t, out);
    Py_DECREF(t);
    return r;
}
static int shape(PyObject* t, int n, int64_t* out) {
    PyObject* s = PyObject_GetAttr(t, s_shape);
    if (s == NULL) return -1;
    PyObject* f = PySequence_Fast(s, "a shape is a sequence");
    Py_DECREF(s);
    if (f == NULL) return -1;
    if (PySequence_Fast_GET_SIZE(f) != n) {
        PyErr_Format(PyExc_ValueError, "expected a tensor of %d dimensions, got %zd", n, PySequence_Fast_GET_SIZE(f));
        Py_DECREF(f);
        return -1;
    }
    for (int i = 0; i < n; ++i) out[i] = PyLong_AsLongLong(PySequence_Fast_GET_ITEM(f, i));
    Py_DECREF(f);
    return PyErr_Occurred() ? -1 : 0;
}
static int integer(PyObject* v, int64_t* out) {
    *out = PyLong_AsLongLong(v);
    return *out == -1 && PyErr_Occurred() ? -1 : 0;
}
static int small(PyObject* v, int* out) {
    const long r = PyLong_AsLong(v);
    if (r == -1 && PyErr_Occurred()) return -1;
    if (r < INT_MIN || r > INT_MAX) {
        PyErr_Format(PyExc_OverflowError, "%ld is not a number of 32 bits", r);
        return -1;
    }
    *out = (int)r;
    return 0;
}
static int pitch(PyObject* t, int64_t* out) {
    PyObject* v = PyObject_CallMethodOneArg(t, s_stride, zero);
    if (v == NULL) return -1;
    const int r = integer(v, out);
    Py_DECREF(v);
    return r;
}
static int dtype(PyObject* t, hq_dtype* out) {
    PyObject* d = PyObject_GetAttr(t, s_dtype);
    if (d == NULL) return -1;
    for (int i = 0; i < 2; ++i)
        if (d == known_dtype[i]) {
            Py_DECREF(d);
            *out = (hq_dtype)known_code[i];
            return 0;
        }
    PyObject* c = PyObject_CallOneArg(dtype_code, t);        /* raises for a type that is not taken */
    int code;
    if (c == NULL || small(c, &code) != 0) {
        Py_XDECREF(c);
        Py_DECREF(d);
        return -1;
    }
    Py_DECREF(c);
    const int slot = known_dtype[0] == NULL ? 0 : 1;
    if (known_dtype[slot] == NULL) {
        known_code[slot] = code;
        known_dtype[slot] = d;                               /* kept */
    } else {
        Py_DECREF(d);
    }
    *out = (hq_dtype)code;
    return 0;
}
static int bytes_of(PyObject* t, size_t* out) {
    PyObject* v = PyObject_GetAttr(t, s_nbytes);
    if (v == NULL) return -1;
    *out = PyLong_AsSize_t(v);
    Py_DECREF(v);
    return PyErr_Occurred() ? -1 : 0;
}
typedef struct { Py_buffer desc; void* blob; void* s_w; } weight;
static int weight_of(PyObject* pw, weight* w) {
    PyObject* d = PyObject_GetAttr(pw, s_desc);
    if (d == NULL) return -1;
    const int r = PyObject_GetBuffer(d, &w->desc, PyBUF_SIMPLE);
    Py_DECREF(d);
    if (r != 0) return -1;
    if ((size_t)w->desc.len >= sizeof(hq_weight_desc) && attr_address(pw, s_blob_dev, &w->blob) == 0 && attr_address(pw, s_s_w_dev, &w->s_w) == 0)
        return 0;
    PyBuffer_Release(&w->desc);
    if (!PyErr_Occurred()) PyErr_SetString(PyExc_TypeError, "not a weight descriptor");
    return -1;
}
static int arguments(Py_ssize_t n, Py_ssize_t want, const void* fn) {
    if (n == want && fn != NULL) return 0;
    PyErr_Format(PyExc_TypeError, fn == NULL ? "not bound" : "expected %zd arguments, got %zd", want, n);
    return -1;
}
#define MODE(o) ((o) == Py_None ? HQ_SCALE_PER_ROW : HQ_SCALE_STATIC)

/* qlinear(x, pw, bias, a_bits, y, workspace, static_scale, dev_status, stream) */
static PyObject* py_qlinear(PyObject* self, PyObject* const* a, Py_ssize_t n) {
    (void)self;
    void *x, *bias, *y, *ws, *ss, *status;
    int64_t dim[2], ldx, ldy, stream;
    hq_dtype xdt, ydt;
    size_t ws_bytes;
    int bits;
    weight w;
    if (arguments(n, 9, f_qlinear) || shape(a[0], 2, dim) || address(a[0], &x) || dtype(a[0], &xdt) || pitch(a[0], &ldx) ||
        address(a[2], &bias) || small(a[3], &bits) || address(a[4], &y) || dtype(a[4], &ydt) || pitch(a[4], &ldy) || address(a[5], &ws) ||
        bytes_of(a[5], &ws_bytes) || address(a[6], &ss) || address(a[7], &status) || integer(a[8], &stream) || weight_of(a[1], &w))
        return NULL;
    hq_status s;
    Py_BEGIN_ALLOW_THREADS
    s = f_qlinear(x, xdt, dim[0], dim[1], ldx, w.desc.buf, w.blob, w.s_w, bias, bits, MODE(a[6]), ss, y, ydt, ldy, ws, ws_bytes, status,
                  (void*)(intptr_t)stream);
    Py_END_ALLOW_THREADS
    PyBuffer_Release(&w.desc);
    return PyLong_FromLong(s);
}

/* qconv(x, pw, R, S, stride, pad, bias, a_bits, y, workspace, static_scale, dev_status, stream) */
static PyObject* py_qconv(PyObject* self, PyObject* const* a, Py_ssize_t n) {
    (void)self;
    void *x, *bias, *y, *ws, *ss, *status;
    int64_t dim[4], stream;
    hq_dtype xdt, ydt;
    size_t ws_bytes;
    int R, S, stride, pad, bits;
    weight w;
    if (arguments(n, 13, f_qconv) || shape(a[0], 4, dim) || address(a[0], &x) || dtype(a[0], &xdt) || small(a[2], &R) || small(a[3], &S) ||
        small(a[4], &stride) || small(a[5], &pad) || address(a[6], &bias) || small(a[7], &bits) || address(a[8], &y) || dtype(a[8], &ydt) ||
        address(a[9], &ws) || bytes_of(a[9], &ws_bytes) || address(a[10], &ss) || address(a[11], &status) || integer(a[12], &stream) ||
        weight_of(a[1], &w))
        return NULL;
    hq_status s;
    Py_BEGIN_ALLOW_THREADS
    s = f_qconv(x, xdt, dim[0], dim[1], dim[2], dim[3], w.desc.buf, w.blob, R, S, stride, pad, w.s_w, bias, bits, MODE(a[10]), ss, y, ydt, ws,
                ws_bytes, status, (void*)(intptr_t)stream);
    Py_END_ALLOW_THREADS
    PyBuffer_Release(&w.desc);
    return PyLong_FromLong(s);
}

/* ln_qlinear(x, ln_weight, ln_bias, rows_per_group, eps, pw, bias, a_bits, y, workspace, dev_status, stream) */
static PyObject* py_ln_qlinear(PyObject* self, PyObject* const* a, Py_ssize_t n) {
    (void)self;
    void *x, *lw, *lb, *bias, *y, *ws, *status;
    int64_t dim[2], ldx, ldy, group, stream;
    hq_dtype xdt, ydt;
    size_t ws_bytes;
    int bits;
    weight w;
    if (arguments(n, 12, f_ln_qlinear)) return NULL;
    const double eps = PyFloat_AsDouble(a[4]);
    if (PyErr_Occurred() || shape(a[0], 2, dim) || address(a[0], &x) || dtype(a[0], &xdt) || pitch(a[0], &ldx) || address(a[1], &lw) ||
        address(a[2], &lb) || integer(a[3], &group) || address(a[6], &bias) || small(a[7], &bits) || address(a[8], &y) || dtype(a[8], &ydt) ||
        pitch(a[8], &ldy) || address(a[9], &ws) || bytes_of(a[9], &ws_bytes) || address(a[10], &status) || integer(a[11], &stream) ||
        weight_of(a[5], &w))
        return NULL;
    hq_status s;
    Py_BEGIN_ALLOW_THREADS
    s = f_ln_qlinear(x, xdt, dim[0], dim[1], ldx, lw, lb, group, (float)eps, w.desc.buf, w.blob, w.s_w, bias, bits, y, ydt, ldy, ws, ws_bytes,
                     status, (void*)(intptr_t)stream);
    Py_END_ALLOW_THREADS
    PyBuffer_Release(&w.desc);
    return PyLong_FromLong(s);
}

/* hadamard_quant(x, had_block, bits, codes, container, scales, static_scale, stream) */
static PyObject* py_quant(PyObject* self, PyObject* const* a, Py_ssize_t n) {
    (void)self;
    void *x, *codes, *scales, *ss;
    int64_t dim[2], ldx, ldc, stream;
    hq_dtype xdt;
    int block, bits, cont;
    if (arguments(n, 8, f_quant) || shape(a[0], 2, dim) || address(a[0], &x) || dtype(a[0], &xdt) || pitch(a[0], &ldx) || small(a[1], &block) ||
        small(a[2], &bits) || address(a[3], &codes) || pitch(a[3], &ldc) || small(a[4], &cont) || address(a[5], &scales) || address(a[6], &ss) ||
        integer(a[7], &stream))
        return NULL;
    hq_status s;
    Py_BEGIN_ALLOW_THREADS
    s = f_quant(x, xdt, dim[0], dim[1], ldx, block, bits, MODE(a[6]), ss, codes, (hq_container)cont, ldc, scales, (void*)(intptr_t)stream);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(s);
}

/* bind(dtype_code, qlinear, qconv, ln_qlinear, hadamard_quant): the type lookup and the addresses of the entry points */
static PyObject* py_bind(PyObject* self, PyObject* args) {
    (void)self;
    PyObject* code;
    unsigned long long p[4];
    if (!PyArg_ParseTuple(args, "OKKKK", &code, &p[0], &p[1], &p[2], &p[3])) return NULL;
    Py_INCREF(code);
    Py_XSETREF(dtype_code, code);
    f_qlinear = (qlinear_fn)(uintptr_t)p[0];
    f_qconv = (qconv_fn)(uintptr_t)p[1];
    f_ln_qlinear = (ln_qlinear_fn)(uintptr_t)p[2];
    f_quant = (quant_fn)(uintptr_t)p[3];
    Py_RETURN_NONE;
}

/* ---- the training attention and the norm + rotation of queries and keys: the same, and the tensors' sizes, types and device are checked
 * here (twenty look-ups of a call's eight matrices through Python took 15 us) ---- */
typedef hq_status (*rope_fn)(const void*, int64_t, const void*, int64_t, hq_dtype, int64_t, int, int, int, const float*, const float*, float,
                             const float*, const float*, int64_t, int, const int32_t*, int, void*, int64_t, void*, int64_t, void*);
typedef hq_status (*rope_bwd_fn)(const void*, int64_t, const void*, int64_t, hq_dtype, int64_t, int, int, int, const float*, const float*, float,
                                 const float*, const float*, int64_t, int, const int32_t*, int, const void*, int64_t, const void*, int64_t,
                                 void*, int64_t, void*, int64_t, float*, float*, void*, size_t, void*);
typedef hq_status (*attn_fwd_fn)(const void*, int64_t, const void*, int64_t, const void*, int64_t, int64_t, int64_t, int64_t, int, int, int,
                                 float, int, const int32_t*, const int32_t*, void*, int64_t, float*, void*, size_t, int32_t*, void*);
typedef hq_status (*attn_bwd_fn)(const void*, int64_t, const void*, int64_t, const void*, int64_t, const void*, int64_t, const float*,
                                 const void*, int64_t, int64_t, int64_t, int64_t, int, int, int, float, int, const int32_t*, const int32_t*,
                                 void*, int64_t, void*, int64_t, void*, int64_t, void*, size_t, int32_t*, void*);
static rope_fn f_rope;
static rope_bwd_fn f_rope_bwd;
static attn_fwd_fn f_attn_fwd;
static attn_bwd_fn f_attn_bwd;
static PyObject *s_get_device, *s_is_contiguous, *dt_f32, *dt_bf16, *dt_i32;

/* A tensor whose address is handed to a kernel lies on the current device: another's may fault there, the host's does. */
static int here(const char* name, PyObject* t, int64_t device) {
    PyObject* v = PyObject_CallMethodNoArgs(t, s_get_device);
    int64_t d;
    if (v == NULL) return -1;
    const int r = integer(v, &d);
    Py_DECREF(v);
    if (r != 0) return -1;
    if (d == device) return 0;
    PyErr_Format(PyExc_ValueError, d < 0 ? "%s: a tensor of the host, not on the current CUDA device" : "%s: a tensor on CUDA device %lld, not on the current one",
                 name, (long long)d);
    return -1;
}
static int is_type(const char* name, PyObject* t, PyObject* want) {
    PyObject* d = PyObject_GetAttr(t, s_dtype);
    if (d == NULL) return -1;
    const int same = d == want;
    if (!same) PyErr_Format(PyExc_ValueError, "%s: expected %R, got %R", name, want, d);
    Py_DECREF(d);
    return same ? 0 : -1;
}
/* [rows, width] whose columns are next to one another (rows may be further apart): address and pitch */
static int heads_matrix(const char* name, PyObject* t, PyObject* type, int64_t rows, int64_t width, int64_t device, void** p, int64_t* ld) {
    int64_t dim[2], st[2];
    if (is_type(name, t, type) || shape(t, 2, dim)) return -1;
    PyObject* v = PyObject_CallMethodNoArgs(t, s_stride);
    if (v == NULL) return -1;
    PyObject* f = PySequence_Fast(v, "strides are a sequence");
    Py_DECREF(v);
    if (f == NULL) return -1;
    for (int i = 0; i < 2; ++i) st[i] = PyLong_AsLongLong(PySequence_Fast_GET_ITEM(f, i));
    Py_DECREF(f);
    if (PyErr_Occurred()) return -1;
    if (dim[0] != rows || dim[1] != width || (st[1] != 1 && width > 1)) {
        PyErr_Format(PyExc_ValueError, "%s: expected [%lld, %lld] with contiguous columns, got [%lld, %lld] with strides (%lld, %lld)", name,
                     (long long)rows, (long long)width, (long long)dim[0], (long long)dim[1], (long long)st[0], (long long)st[1]);
        return -1;
    }
    *ld = rows > 1 ? st[0] : width;
    return here(name, t, device) || address(t, p) ? -1 : 0;
}
/* an optional dense tensor of n sizes */
static int dense(const char* name, PyObject* t, PyObject* type, int n, int64_t d0, int64_t d1, int64_t d2, int64_t device, void** p) {
    int64_t dim[3], want[3] = {d0, d1, d2};
    *p = NULL;
    if (t == Py_None) return 0;
    if (is_type(name, t, type) || shape(t, n, dim)) return -1;
    PyObject* v = PyObject_CallMethodNoArgs(t, s_is_contiguous);
    if (v == NULL) return -1;
    int ok = v == Py_True;
    Py_DECREF(v);
    for (int i = 0; i < n; ++i) ok = ok && dim[i] == want[i];
    if (!ok) {
        PyErr_Format(PyExc_ValueError, "%s: expected a dense tensor of %d sizes from %lld on", name, n, (long long)d0);
        return -1;
    }
    return here(name, t, device) || address(t, p) ? -1 : 0;
}
static int workspace_of(PyObject* t, int64_t device, void** p, size_t* bytes) {
    *p = NULL;
    *bytes = 0;
    if (t == Py_None) return 0;
    PyObject* v = PyObject_CallMethodNoArgs(t, s_is_contiguous);
    if (v == NULL) return -1;
    const int ok = v == Py_True;
    Py_DECREF(v);
    if (!ok) {
        PyErr_SetString(PyExc_ValueError, "workspace: a dense tensor");
        return -1;
    }
    return here("workspace", t, device) || address(t, p) || bytes_of(t, bytes) ? -1 : 0;
}

typedef struct { int64_t Nb, Lq, Lk; int heads, kv_heads, dh, causal; float scale; } attn_shape;
static int attn_shape_of(PyObject* q, PyObject* k, PyObject* Nb, PyObject* heads, PyObject* kv_heads, PyObject* causal, PyObject* scale, attn_shape* s) {
    int64_t dq[2], dk[2];
    if (shape(q, 2, dq) || shape(k, 2, dk) || integer(Nb, &s->Nb) || small(heads, &s->heads) || small(kv_heads, &s->kv_heads)) return -1;
    if (s->Nb <= 0 || s->heads <= 0 || s->kv_heads <= 0 || dq[0] % s->Nb || dk[0] % s->Nb || dq[1] % s->heads) {
        PyErr_Format(PyExc_ValueError, "queries [%lld, %lld] and keys [%lld, %lld] are not %lld samples of %d / %d heads", (long long)dq[0],
                     (long long)dq[1], (long long)dk[0], (long long)dk[1], (long long)s->Nb, s->heads, s->kv_heads);
        return -1;
    }
    s->Lq = dq[0] / s->Nb;
    s->Lk = dk[0] / s->Nb;
    s->dh = (int)(dq[1] / s->heads);
    s->causal = PyObject_IsTrue(causal);
    if (s->causal < 0) return -1;
    if (scale == Py_None) {
        double x = s->dh > 0 ? s->dh : 1, r = x;
        for (int i = 0; i < 60; ++i) r = 0.5 * (r + x / r);      /* the square root, without the math library */
        s->scale = (float)(1.0 / r);
    } else {
        s->scale = (float)PyFloat_AsDouble(scale);
        if (PyErr_Occurred()) return -1;
    }
    return 0;
}

/* attention_fwd(q, k, v, Nb, heads, kv_heads, out, lse, workspace, q_lens, k_lens, causal, scale, dev_status, stream, device) */
static PyObject* py_attn_fwd(PyObject* self, PyObject* const* a, Py_ssize_t n) {
    (void)self;
    attn_shape s;
    void *p[4], *lse, *ws, *ql, *kl, *status;
    int64_t ld[4], stream, dev;
    size_t ws_bytes;
    if (arguments(n, 16, f_attn_fwd) || attn_shape_of(a[0], a[1], a[3], a[4], a[5], a[11], a[12], &s) || integer(a[14], &stream) || integer(a[15], &dev)) return NULL;
    const int64_t wq = (int64_t)s.heads * s.dh, wk = (int64_t)s.kv_heads * s.dh, rq = s.Nb * s.Lq, rk = s.Nb * s.Lk;
    if (heads_matrix("q", a[0], dt_bf16, rq, wq, dev, &p[0], &ld[0]) || heads_matrix("k", a[1], dt_bf16, rk, wk, dev, &p[1], &ld[1]) ||
        heads_matrix("v", a[2], dt_bf16, rk, wk, dev, &p[2], &ld[2]) || heads_matrix("out", a[6], dt_bf16, rq, wq, dev, &p[3], &ld[3]) ||
        dense("lse", a[7], dt_f32, 3, s.Nb, s.heads, s.Lq, dev, &lse) || workspace_of(a[8], dev, &ws, &ws_bytes) ||
        dense("q_lens", a[9], dt_i32, 1, s.Nb, 0, 0, dev, &ql) || dense("k_lens", a[10], dt_i32, 1, s.Nb, 0, 0, dev, &kl) ||
        dense("dev_status", a[13], dt_i32, 1, 1, 0, 0, dev, &status))
        return NULL;
    hq_status r;
    Py_BEGIN_ALLOW_THREADS
    r = f_attn_fwd(p[0], ld[0], p[1], ld[1], p[2], ld[2], s.Nb, s.Lq, s.Lk, s.heads, s.kv_heads, s.dh, s.scale, s.causal, ql, kl, p[3], ld[3], lse, ws,
                   ws_bytes, status, (void*)(intptr_t)stream);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(r);
}

/* attention_bwd(q, k, v, out, lse, dout, Nb, heads, kv_heads, dq, dk, dv, workspace, q_lens, k_lens, causal, scale, dev_status, stream, device) */
static PyObject* py_attn_bwd(PyObject* self, PyObject* const* a, Py_ssize_t n) {
    (void)self;
    attn_shape s;
    void *p[8], *lse, *ws, *ql, *kl, *status;
    int64_t ld[8], stream, dev;
    size_t ws_bytes;
    if (arguments(n, 20, f_attn_bwd) || attn_shape_of(a[0], a[1], a[6], a[7], a[8], a[15], a[16], &s) || integer(a[18], &stream) || integer(a[19], &dev)) return NULL;
    const int64_t wq = (int64_t)s.heads * s.dh, wk = (int64_t)s.kv_heads * s.dh, rq = s.Nb * s.Lq, rk = s.Nb * s.Lk;
    if (heads_matrix("q", a[0], dt_bf16, rq, wq, dev, &p[0], &ld[0]) || heads_matrix("k", a[1], dt_bf16, rk, wk, dev, &p[1], &ld[1]) ||
        heads_matrix("v", a[2], dt_bf16, rk, wk, dev, &p[2], &ld[2]) || heads_matrix("out", a[3], dt_bf16, rq, wq, dev, &p[3], &ld[3]) ||
        heads_matrix("dout", a[5], dt_bf16, rq, wq, dev, &p[4], &ld[4]) || heads_matrix("dq", a[9], dt_bf16, rq, wq, dev, &p[5], &ld[5]) ||
        heads_matrix("dk", a[10], dt_bf16, rk, wk, dev, &p[6], &ld[6]) || heads_matrix("dv", a[11], dt_bf16, rk, wk, dev, &p[7], &ld[7]) ||
        dense("lse", a[4], dt_f32, 3, s.Nb, s.heads, s.Lq, dev, &lse) || workspace_of(a[12], dev, &ws, &ws_bytes) ||
        dense("q_lens", a[13], dt_i32, 1, s.Nb, 0, 0, dev, &ql) || dense("k_lens", a[14], dt_i32, 1, s.Nb, 0, 0, dev, &kl) ||
        dense("dev_status", a[17], dt_i32, 1, 1, 0, 0, dev, &status))
        return NULL;
    hq_status r;
    Py_BEGIN_ALLOW_THREADS
    r = f_attn_bwd(p[0], ld[0], p[1], ld[1], p[2], ld[2], p[3], ld[3], lse, p[4], ld[4], s.Nb, s.Lq, s.Lk, s.heads, s.kv_heads, s.dh, s.scale, s.causal,
                   ql, kl, p[5], ld[5], p[6], ld[6], p[7], ld[7], ws, ws_bytes, status, (void*)(intptr_t)stream);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(r);
}

typedef struct { int64_t rows, npos; int heads, kv_heads, dh, rot, interleaved; float eps; hq_dtype dt; PyObject* type; void *gq, *gk, *cos, *sin, *pos; } rope_shape;
/* q, k, heads, kv_heads, gamma_q, gamma_k, eps, cos, sin of both calls; the type is q's */
static int rope_shape_of(PyObject* const* a, PyObject* positions, PyObject* interleaved, int64_t dev, rope_shape* s) {
    int64_t dim[2], table[2] = {0, 0};
    if (shape(a[0], 2, dim) || small(a[2], &s->heads) || small(a[3], &s->kv_heads)) return -1;
    if (s->heads <= 0 || dim[1] % s->heads) {
        PyErr_Format(PyExc_ValueError, "%lld columns do not hold %d heads", (long long)dim[1], s->heads);
        return -1;
    }
    if ((a[1] == Py_None) != (s->kv_heads == 0)) {
        PyErr_SetString(PyExc_ValueError, "keys are given with their heads, or neither");
        return -1;
    }
    if ((a[7] == Py_None) != (a[8] == Py_None)) {
        PyErr_SetString(PyExc_ValueError, "cos and sin: two tables [positions, rot / 2]");
        return -1;
    }
    s->rows = dim[0];
    s->dh = (int)(dim[1] / s->heads);
    if (dtype(a[0], &s->dt)) return -1;
    s->type = s->dt == HQ_F32 ? dt_f32 : dt_bf16;
    s->eps = (float)PyFloat_AsDouble(a[6]);
    s->interleaved = PyObject_IsTrue(interleaved);
    if (PyErr_Occurred() || (a[7] != Py_None && shape(a[7], 2, table))) return -1;
    if (table[1] > INT_MAX / 2) {
        PyErr_Format(PyExc_OverflowError, "tables of %lld columns", (long long)table[1]);
        return -1;
    }
    s->npos = table[0];
    s->rot = (int)(2 * table[1]);
    return dense("gamma_q", a[4], dt_f32, 1, s->dh, 0, 0, dev, &s->gq) || dense("gamma_k", a[5], dt_f32, 1, s->dh, 0, 0, dev, &s->gk) ||
           dense("cos", a[7], dt_f32, 2, table[0], table[1], 0, dev, &s->cos) || dense("sin", a[8], dt_f32, 2, table[0], table[1], 0, dev, &s->sin) ||
           dense("positions", positions, dt_i32, 1, s->rows, 0, 0, dev, &s->pos) ? -1 : 0;
}

/* qk_rope(q, k, heads, kv_heads, gamma_q, gamma_k, eps, cos, sin, q_out, k_out, positions, interleaved, stream, device) */
static PyObject* py_rope(PyObject* self, PyObject* const* a, Py_ssize_t n) {
    (void)self;
    rope_shape s;
    void* p[4] = {NULL, NULL, NULL, NULL};
    int64_t ld[4] = {0, 0, 0, 0}, stream, dev;
    if (arguments(n, 15, f_rope) || integer(a[13], &stream) || integer(a[14], &dev) || rope_shape_of(a, a[11], a[12], dev, &s)) return NULL;
    const int64_t wq = (int64_t)s.heads * s.dh, wk = (int64_t)s.kv_heads * s.dh;
    if (heads_matrix("q", a[0], s.type, s.rows, wq, dev, &p[0], &ld[0]) || heads_matrix("q_out", a[9], s.type, s.rows, wq, dev, &p[2], &ld[2]) ||
        (a[1] != Py_None && (heads_matrix("k", a[1], s.type, s.rows, wk, dev, &p[1], &ld[1]) || heads_matrix("k_out", a[10], s.type, s.rows, wk, dev, &p[3], &ld[3]))))
        return NULL;
    hq_status r;
    Py_BEGIN_ALLOW_THREADS
    r = f_rope(p[0], ld[0], p[1], ld[1], s.dt, s.rows, s.heads, s.kv_heads, s.dh, s.gq, s.gk, s.eps, s.cos, s.sin, s.npos, s.rot, s.pos, s.interleaved,
               p[2], ld[2], p[3], ld[3], (void*)(intptr_t)stream);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(r);
}

/* qk_rope_bwd(q, k, heads, kv_heads, gamma_q, gamma_k, eps, cos, sin, dq_out, dk_out, dq, dk, dgamma_q, dgamma_k, workspace, positions, interleaved,
 *             stream, device) */
static PyObject* py_rope_bwd(PyObject* self, PyObject* const* a, Py_ssize_t n) {
    (void)self;
    rope_shape s;
    void *p[6] = {NULL, NULL, NULL, NULL, NULL, NULL}, *dgq, *dgk, *ws;
    int64_t ld[6] = {0, 0, 0, 0, 0, 0}, stream, dev;
    size_t ws_bytes;
    if (arguments(n, 20, f_rope_bwd) || integer(a[18], &stream) || integer(a[19], &dev) || rope_shape_of(a, a[16], a[17], dev, &s)) return NULL;
    const int64_t wq = (int64_t)s.heads * s.dh, wk = (int64_t)s.kv_heads * s.dh;
    if (heads_matrix("q", a[0], s.type, s.rows, wq, dev, &p[0], &ld[0]) || heads_matrix("dq_out", a[9], s.type, s.rows, wq, dev, &p[2], &ld[2]) ||
        heads_matrix("dq", a[11], s.type, s.rows, wq, dev, &p[4], &ld[4]) ||
        (a[1] != Py_None && (heads_matrix("k", a[1], s.type, s.rows, wk, dev, &p[1], &ld[1]) || heads_matrix("dk_out", a[10], s.type, s.rows, wk, dev, &p[3], &ld[3]) ||
                             heads_matrix("dk", a[12], s.type, s.rows, wk, dev, &p[5], &ld[5]))) ||
        dense("dgamma_q", a[13], dt_f32, 1, s.dh, 0, 0, dev, &dgq) || dense("dgamma_k", a[14], dt_f32, 1, s.dh, 0, 0, dev, &dgk) ||
        workspace_of(a[15], dev, &ws, &ws_bytes))
        return NULL;
    hq_status r;
    Py_BEGIN_ALLOW_THREADS
    r = f_rope_bwd(p[0], ld[0], p[1], ld[1], s.dt, s.rows, s.heads, s.kv_heads, s.dh, s.gq, s.gk, s.eps, s.cos, s.sin, s.npos, s.rot, s.pos, s.interleaved,
                   p[2], ld[2], p[3], ld[3], p[4], ld[4], p[5], ld[5], dgq, dgk, ws, ws_bytes, (void*)(intptr_t)stream);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(r);
}

/* ---- the gated residual with its norms, and the embedding: the same ---- */
typedef hq_status (*gate_norm_fn)(const void*, int64_t, hq_dtype, const void*, int64_t, hq_dtype, int64_t, int64_t, int64_t, const int32_t*, hq_norm,
                                  const float*, const float*, int64_t, float, hq_norm, const float*, int64_t, const float*, int64_t, float, float,
                                  void*, int64_t, void*, int64_t, float*, void*);
typedef hq_status (*gate_norm_bwd_fn)(const void*, int64_t, hq_dtype, const void*, int64_t, hq_dtype, const float*, int64_t, int64_t, int64_t,
                                      const int32_t*, hq_norm, const float*, const float*, int64_t, float, hq_norm, const float*, int64_t, float,
                                      const void*, int64_t, const void*, int64_t, void*, int64_t, void*, int64_t, float*, float*, int64_t, float*,
                                      int64_t, float*, int64_t, void*, size_t, void*);
typedef hq_status (*embedding_fn)(const void*, int, int64_t, const void*, hq_dtype, int64_t, int64_t, int64_t, float, void*, hq_dtype, int64_t, void*);
typedef hq_status (*embedding_bwd_fn)(const void*, int, int64_t, const void*, hq_dtype, int64_t, int64_t, int64_t, float, const void*, int64_t, void*,
                                      hq_dtype, int64_t, void*, size_t, void*);
static gate_norm_fn f_gate_norm;
static gate_norm_bwd_fn f_gate_norm_bwd;
static embedding_fn f_embedding;
static embedding_bwd_fn f_embedding_bwd;
static PyObject *dt_i64;

typedef struct { void* p; int64_t ld; } matrix;
static int optional(const char* name, PyObject* t, PyObject* type, int64_t rows, int64_t width, int64_t device, matrix* m) {
    m->p = NULL;
    m->ld = width;
    return t == Py_None ? 0 : heads_matrix(name, t, type, rows, width, device, &m->p, &m->ld);
}
/* [groups, cols] with contiguous columns, or [cols] where there is one group */
static int vectors(const char* name, PyObject* t, int64_t groups, int64_t cols, int64_t device, matrix* m) {
    if (t != Py_None && groups == 1) {
        PyObject* s = PyObject_GetAttr(t, s_shape);
        if (s == NULL) return -1;
        const Py_ssize_t n = PyObject_Length(s);
        Py_DECREF(s);
        if (n < 0) return -1;
        m->ld = cols;
        if (n == 1) return dense(name, t, dt_f32, 1, cols, 0, 0, device, &m->p);
    }
    return optional(name, t, dt_f32, groups, cols, device, m);
}
static PyObject* first_of(PyObject* a, PyObject* b, PyObject* c) { return a != Py_None ? a : b != Py_None ? b : c; }
static int real(PyObject* v, float* out) {
    *out = (float)PyFloat_AsDouble(v);
    return PyErr_Occurred() ? -1 : 0;
}
/* the types of both sides and the sizes: of the first matrix that is given */
typedef struct { hq_dtype xdt, hdt; PyObject *xtype, *htype; int64_t rows, cols, per, groups; int post, norm; } norm_shape;
static int norm_shape_of(PyObject* x, PyObject* h, PyObject* per, PyObject* post, PyObject* norm, norm_shape* s) {
    int64_t dim[2];
    PyObject* any = x != Py_None ? x : h;
    if (any == Py_None) {
        PyErr_SetString(PyExc_ValueError, "no matrix is given");
        return -1;
    }
    if (shape(any, 2, dim) || integer(per, &s->per) || small(post, &s->post) || small(norm, &s->norm)) return -1;
    if (dtype(any, &s->xdt)) return -1;
    s->hdt = s->xdt;
    if (h != Py_None && dtype(h, &s->hdt)) return -1;
    s->xtype = s->xdt == HQ_F32 ? dt_f32 : dt_bf16;
    s->htype = s->hdt == HQ_F32 ? dt_f32 : dt_bf16;
    s->rows = dim[0];
    s->cols = dim[1];
    if (s->per < 0) {
        PyErr_SetString(PyExc_ValueError, "rows_per_group: 0 or more");
        return -1;
    }
    s->groups = s->per > 0 ? s->rows / s->per + (s->rows % s->per != 0) : 1;
    return 0;
}

/* gate_norm(x, h, gate, weight, bias, x_out, y, stats, rows_per_group, lens, post, post_weight, norm, weight_plus, residual_scale, eps, stream, device) */
static PyObject* py_gate_norm(PyObject* self, PyObject* const* a, Py_ssize_t n) {
    (void)self;
    norm_shape s;
    matrix x, h, gate, weight, bias, x_out, y;
    void *stats, *lens, *pw;
    float plus, residual, eps;
    int64_t stream, dev;
    if (arguments(n, 18, f_gate_norm) || integer(a[16], &stream) || integer(a[17], &dev) || norm_shape_of(a[0], first_of(a[1], a[6], Py_None), a[8], a[10], a[12], &s) ||
        real(a[13], &plus) || real(a[14], &residual) || real(a[15], &eps) || optional("x", a[0], s.xtype, s.rows, s.cols, dev, &x) ||
        optional("h", a[1], s.htype, s.rows, s.cols, dev, &h) || vectors("gate", a[2], s.groups, s.cols, dev, &gate) ||
        vectors("weight", a[3], s.groups, s.cols, dev, &weight) || vectors("bias", a[4], s.groups, s.cols, dev, &bias) ||
        optional("x_out", a[5], s.xtype, s.rows, s.cols, dev, &x_out) || optional("y", a[6], s.htype, s.rows, s.cols, dev, &y) ||
        dense("stats", a[7], dt_f32, 2, s.rows, 4, 0, dev, &stats) || dense("lens", a[9], dt_i32, 1, s.groups, 0, 0, dev, &lens) ||
        dense("post_weight", a[11], dt_f32, 1, s.cols, 0, 0, dev, &pw))
        return NULL;
    hq_status r;
    Py_BEGIN_ALLOW_THREADS
    r = f_gate_norm(x.p, x.ld, s.xdt, h.p, h.ld, s.hdt, s.rows, s.cols, s.per, lens, (hq_norm)s.post, pw, gate.p, gate.ld, residual, (hq_norm)s.norm,
                    weight.p, weight.ld, bias.p, bias.ld, plus, eps, x_out.p, x_out.ld, y.p, y.ld, stats, (void*)(intptr_t)stream);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(r);
}

/* gate_norm_bwd(x_out, h, stats, gate, weight, dx_out, dy, dx, dh, dgate, dweight, dbias, workspace, rows_per_group, lens, post, post_weight, dpost_weight,
 *               norm, weight_plus, residual_scale, stream, device) */
static PyObject* py_gate_norm_bwd(PyObject* self, PyObject* const* a, Py_ssize_t n) {
    (void)self;
    norm_shape s;
    matrix x, h, gate, weight, dxo, dy, dx, dh, dgate, dweight, dbias;
    void *stats, *lens, *pw, *dpw, *ws;
    size_t ws_bytes;
    float plus, residual;
    int64_t stream, dev;
    if (arguments(n, 23, f_gate_norm_bwd) || integer(a[21], &stream) || integer(a[22], &dev) ||
        norm_shape_of(first_of(a[0], a[5], a[7]), first_of(a[1], a[6], a[8]), a[13], a[15], a[18], &s) || real(a[19], &plus) || real(a[20], &residual) ||
        optional("x_out", a[0], s.xtype, s.rows, s.cols, dev, &x) || optional("h", a[1], s.htype, s.rows, s.cols, dev, &h) ||
        dense("stats", a[2], dt_f32, 2, s.rows, 4, 0, dev, &stats) || vectors("gate", a[3], s.groups, s.cols, dev, &gate) ||
        vectors("weight", a[4], s.groups, s.cols, dev, &weight) || optional("dx_out", a[5], s.xtype, s.rows, s.cols, dev, &dxo) ||
        optional("dy", a[6], s.htype, s.rows, s.cols, dev, &dy) || optional("dx", a[7], s.xtype, s.rows, s.cols, dev, &dx) ||
        optional("dh", a[8], s.htype, s.rows, s.cols, dev, &dh) || vectors("dgate", a[9], s.groups, s.cols, dev, &dgate) ||
        vectors("dweight", a[10], s.groups, s.cols, dev, &dweight) || vectors("dbias", a[11], s.groups, s.cols, dev, &dbias) ||
        workspace_of(a[12], dev, &ws, &ws_bytes) || dense("lens", a[14], dt_i32, 1, s.groups, 0, 0, dev, &lens) ||
        dense("post_weight", a[16], dt_f32, 1, s.cols, 0, 0, dev, &pw) || dense("dpost_weight", a[17], dt_f32, 1, s.cols, 0, 0, dev, &dpw))
        return NULL;
    hq_status r;
    Py_BEGIN_ALLOW_THREADS
    r = f_gate_norm_bwd(x.p, x.ld, s.xdt, h.p, h.ld, s.hdt, stats, s.rows, s.cols, s.per, lens, (hq_norm)s.post, pw, gate.p, gate.ld, residual,
                        (hq_norm)s.norm, weight.p, weight.ld, plus, dxo.p, dxo.ld, dy.p, dy.ld, dx.p, dx.ld, dh.p, dh.ld, dpw, dgate.p, dgate.ld, dweight.p,
                        dweight.ld, dbias.p, dbias.ld, ws, ws_bytes, (void*)(intptr_t)stream);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(r);
}

/* dense ids of 32 or 64 bits */
static int ids_of(PyObject* t, int64_t tokens, int64_t dev, void** p, int* bytes) {
    PyObject* d = PyObject_GetAttr(t, s_dtype);
    if (d == NULL) return -1;
    const int wide = d == dt_i64;
    Py_DECREF(d);
    *bytes = wide ? 8 : 4;
    return dense("ids", t, wide ? dt_i64 : dt_i32, 1, tokens, 0, 0, dev, p);
}
/* embedding(ids, table, out, scale, stream, device) */
static PyObject* py_embedding(PyObject* self, PyObject* const* a, Py_ssize_t n) {
    (void)self;
    int64_t rows[2], tab[2], stream, dev;
    matrix table, out;
    void* ids;
    float scale;
    hq_dtype tdt, odt;
    int bytes;
    if (arguments(n, 6, f_embedding) || integer(a[4], &stream) || integer(a[5], &dev) || shape(a[2], 2, rows) || shape(a[1], 2, tab) || real(a[3], &scale) ||
        dtype(a[1], &tdt) || dtype(a[2], &odt) || ids_of(a[0], rows[0], dev, &ids, &bytes) ||
        optional("table", a[1], tdt == HQ_F32 ? dt_f32 : dt_bf16, tab[0], tab[1], dev, &table) ||
        optional("out", a[2], odt == HQ_F32 ? dt_f32 : dt_bf16, rows[0], tab[1], dev, &out))
        return NULL;
    hq_status r;
    Py_BEGIN_ALLOW_THREADS
    r = f_embedding(ids, bytes, rows[0], table.p, tdt, tab[0], tab[1], table.ld, scale, out.p, odt, out.ld, (void*)(intptr_t)stream);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(r);
}
/* embedding_bwd(ids, dout, dtable, workspace, scale, base, stream, device) */
static PyObject* py_embedding_bwd(PyObject* self, PyObject* const* a, Py_ssize_t n) {
    (void)self;
    int64_t rows[2], tab[2], stream, dev;
    matrix dout, base, dtable;
    void *ids, *ws;
    size_t ws_bytes;
    float scale;
    hq_dtype ddt, gdt;
    int bytes;
    if (arguments(n, 8, f_embedding_bwd) || integer(a[6], &stream) || integer(a[7], &dev) || shape(a[1], 2, rows) || shape(a[2], 2, tab) || real(a[4], &scale) ||
        dtype(a[1], &ddt) || dtype(a[2], &gdt) || ids_of(a[0], rows[0], dev, &ids, &bytes) ||
        optional("dout", a[1], ddt == HQ_F32 ? dt_f32 : dt_bf16, rows[0], tab[1], dev, &dout) ||
        optional("base", a[5], gdt == HQ_F32 ? dt_f32 : dt_bf16, tab[0], tab[1], dev, &base) ||
        optional("dtable", a[2], gdt == HQ_F32 ? dt_f32 : dt_bf16, tab[0], tab[1], dev, &dtable) || workspace_of(a[3], dev, &ws, &ws_bytes))
        return NULL;
    hq_status r;
    Py_BEGIN_ALLOW_THREADS
    r = f_embedding_bwd(ids, bytes, rows[0], dout.p, ddt, dout.ld, tab[0], tab[1], scale, base.p, base.ld, dtable.p, gdt, dtable.ld, ws, ws_bytes,
                        (void*)(intptr_t)stream);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(r);
}

typedef hq_status (*grad_norm_fn)(const hq_grad_tensor*, int64_t, float*, void*, size_t, void*);
typedef hq_status (*grad_clip_fn)(const hq_grad_tensor*, int64_t, float, float, float*, float*, void*, size_t, void*);
static grad_norm_fn f_grad_norm;
static grad_clip_fn f_grad_clip;
/* one value, of no dimension or one */
static int one_value(const char* name, PyObject* t, int64_t device, void** p) {
    int64_t dim[1];
    *p = NULL;
    if (t == Py_None) return 0;
    PyObject* s = PyObject_GetAttr(t, s_shape);
    if (s == NULL) return -1;
    const Py_ssize_t n = PyObject_Length(s);
    Py_DECREF(s);
    if (n < 0 || (n == 1 && shape(t, 1, dim)) || is_type(name, t, dt_f32)) return -1;
    if (n > 1 || (n == 1 && dim[0] != 1)) {
        PyErr_Format(PyExc_ValueError, "%s: one value", name);
        return -1;
    }
    return here(name, t, device) || address(t, p) ? -1 : 0;
}
/* grad_clip(table's address, tensors, max_norm (None: the norm alone), eps, norm, coef, workspace, stream, device) */
static PyObject* py_grad_clip(PyObject* self, PyObject* const* a, Py_ssize_t n) {
    (void)self;
    int64_t table, tensors, stream, dev;
    float max_norm = 0.f, eps = 0.f;
    void *norm, *coef, *ws;
    size_t ws_bytes;
    if (arguments(n, 9, f_grad_clip) || integer(a[0], &table) || integer(a[1], &tensors) || (a[2] != Py_None && (real(a[2], &max_norm) || real(a[3], &eps))) ||
        integer(a[7], &stream) || integer(a[8], &dev) || one_value("norm", a[4], dev, &norm) || one_value("coef", a[5], dev, &coef) ||
        workspace_of(a[6], dev, &ws, &ws_bytes))
        return NULL;
    hq_status r;
    Py_BEGIN_ALLOW_THREADS
    const hq_grad_tensor* t = (const hq_grad_tensor*)(intptr_t)table;
    r = a[2] == Py_None ? f_grad_norm(t, tensors, norm, ws, ws_bytes, (void*)(intptr_t)stream)
                        : f_grad_clip(t, tensors, max_norm, eps, norm, coef, ws, ws_bytes, (void*)(intptr_t)stream);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(r);
}

/* bind_block(int64, gate_norm, gate_norm_bwd, embedding, embedding_bwd, grad_norm, grad_clip), behind bind_attention */
static PyObject* py_bind_block(PyObject* self, PyObject* args) {
    (void)self;
    PyObject* d;
    unsigned long long p[6];
    if (!PyArg_ParseTuple(args, "OKKKKKK", &d, &p[0], &p[1], &p[2], &p[3], &p[4], &p[5])) return NULL;
    Py_INCREF(d);
    Py_XSETREF(dt_i64, d);
    f_grad_norm = (grad_norm_fn)(uintptr_t)p[4];
    f_grad_clip = (grad_clip_fn)(uintptr_t)p[5];
    f_gate_norm = (gate_norm_fn)(uintptr_t)p[0];
    f_gate_norm_bwd = (gate_norm_bwd_fn)(uintptr_t)p[1];
    f_embedding = (embedding_fn)(uintptr_t)p[2];
    f_embedding_bwd = (embedding_bwd_fn)(uintptr_t)p[3];
    Py_RETURN_NONE;
}

/* bind_attention(float32, bfloat16, int32, qk_rope, qk_rope_bwd, attention_fwd, attention_bwd): torch's types and the entry points' addresses */
static PyObject* py_bind_attention(PyObject* self, PyObject* args) {
    (void)self;
    PyObject* d[3];
    unsigned long long p[4];
    if (!PyArg_ParseTuple(args, "OOOKKKK", &d[0], &d[1], &d[2], &p[0], &p[1], &p[2], &p[3])) return NULL;
    for (int i = 0; i < 3; ++i) Py_INCREF(d[i]);
    Py_XSETREF(dt_f32, d[0]);
    Py_XSETREF(dt_bf16, d[1]);
    Py_XSETREF(dt_i32, d[2]);
    f_rope = (rope_fn)(uintptr_t)p[0];
    f_rope_bwd = (rope_bwd_fn)(uintptr_t)p[1];
    f_attn_fwd = (attn_fwd_fn)(uintptr_t)p[2];
    f_attn_bwd = (attn_bwd_fn)(uintptr_t)p[3];
    Py_RETURN_NONE;
}

static PyMethodDef methods[] = {
    {"bind_attention", py_bind_attention, METH_VARARGS, NULL},
    {"qk_rope", (PyCFunction)(void (*)(void))py_rope, METH_FASTCALL, NULL},
    {"qk_rope_bwd", (PyCFunction)(void (*)(void))py_rope_bwd, METH_FASTCALL, NULL},
    {"attention_fwd", (PyCFunction)(void (*)(void))py_attn_fwd, METH_FASTCALL, NULL},
    {"attention_bwd", (PyCFunction)(void (*)(void))py_attn_bwd, METH_FASTCALL, NULL},
    {"bind_block", py_bind_block, METH_VARARGS, NULL},
    {"gate_norm", (PyCFunction)(void (*)(void))py_gate_norm, METH_FASTCALL, NULL},
    {"gate_norm_bwd", (PyCFunction)(void (*)(void))py_gate_norm_bwd, METH_FASTCALL, NULL},
    {"grad_clip", (PyCFunction)(void (*)(void))py_grad_clip, METH_FASTCALL, NULL},
    {"embedding", (PyCFunction)(void (*)(void))py_embedding, METH_FASTCALL, NULL},
    {"embedding_bwd", (PyCFunction)(void (*)(void))py_embedding_bwd, METH_FASTCALL, NULL},
    {"bind", py_bind, METH_VARARGS, NULL},
    {"qlinear", (PyCFunction)(void (*)(void))py_qlinear, METH_FASTCALL, NULL},
    {"qconv", (PyCFunction)(void (*)(void))py_qconv, METH_FASTCALL, NULL},
    {"ln_qlinear", (PyCFunction)(void (*)(void))py_ln_qlinear, METH_FASTCALL, NULL},
    {"hadamard_quant", (PyCFunction)(void (*)(void))py_quant, METH_FASTCALL, NULL},
    {NULL, NULL, 0, NULL}};
static struct PyModuleDef module = {PyModuleDef_HEAD_INIT, "_hqcall", NULL, -1, methods, NULL, NULL, NULL, NULL};

PyMODINIT_FUNC PyInit__hqcall(void) {
    s_data_ptr = PyUnicode_InternFromString("data_ptr");
    s_shape = PyUnicode_InternFromString("shape");
    s_stride = PyUnicode_InternFromString("stride");
    s_dtype = PyUnicode_InternFromString("dtype");
    s_nbytes = PyUnicode_InternFromString("nbytes");
    s_desc = PyUnicode_InternFromString("desc");
    s_blob_dev = PyUnicode_InternFromString("blob_dev");
    s_s_w_dev = PyUnicode_InternFromString("s_w_dev");
    s_get_device = PyUnicode_InternFromString("get_device");
    s_is_contiguous = PyUnicode_InternFromString("is_contiguous");
    zero = PyLong_FromLong(0);
    return PyModule_Create(&module);
}
