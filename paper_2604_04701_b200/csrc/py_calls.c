/* The binding's calls on the hot path as CPython functions: tensor pointers, shapes and parameters are taken from the
 * Python objects here and passed to libmuxq's entry points (whose addresses binding.py hands over once).
 *
 * Why: at decode shapes a layer takes the GPU less time than ctypes and torch's stream lookup take the host.  Per
 * muxq_linear call, host side, 16 x 768 -> 768: 20 us with ctypes (3.5 us of it the lookup of the current stream, 4 us
 * argument conversion). */
#define PY_SSIZE_T_CLEAN
#include <Python.h>
#include <stdint.h>
#include <string.h>

#include "../../include/muxq.h"
#include "py_tensor.h"

typedef int (*linear_fn)(const void *, int, int, int, const int8_t *, int, const float *, int, const muxq_params *, void *,
                         int, int, void *, size_t, int32_t *, void *);
typedef int (*linear_bias_fn)(const void *, int, int, int, const int8_t *, int, const float *, const float *, int,
                              const muxq_params *, void *, int, int, void *, size_t, int32_t *, void *);
typedef int (*quantize_fn)(const void *, int, int, int, const muxq_params *, int, const float *, const int32_t *,
                           const int32_t *, int8_t *, int, int8_t *, int, float *, void *, size_t, void *);

typedef int (*residual_norm_fn)(const void *, int, int, const void *, int, int, const muxq_norm *, const void *, int, int, int, float,
                                const muxq_norm *, int, int, void *, int, void *, int, void *);

typedef int (*adapters_fn)(const void *, int, int, int, const muxq_adapter_set *, const int32_t *, int, const void *, int, void *, int, int,
                           int32_t *, void *);
typedef int (*adapters_check_fn)(const void *, int, int, int, const muxq_adapter_set *, const int32_t *, int, const void *, int, const void *, int,
                                 int, const int32_t *);

static linear_fn f_linear;
static linear_bias_fn f_linear_bias;
static quantize_fn f_quantize;
static residual_norm_fn f_residual_norm;
static adapters_fn f_adapters;
static adapters_check_fn f_adapters_check;
static PyObject *get_device, *raw_stream, *dt_f16, *dt_f32, *dt_i32;
static PyObject *n_data_ptr, *n_shape, *n_stride, *n_dtype, *n_is_cuda, *n_numel, *n_is_contiguous, *n_get_device;
static PyObject *n_threshold, *n_exp_factor, *n_act_bits, *n_w_bits, *n_gran, *n_aux_scale, *n_max_outliers;

static int tensor_ptr(PyObject *t, void **out) {
    PyObject *v = PyObject_CallMethodNoArgs(t, n_data_ptr);
    if (!v) return -1;
    *out = PyLong_AsVoidPtr(v);
    Py_DECREF(v);
    return PyErr_Occurred() ? -1 : 0;
}

static int as_int(PyObject *v, int *out) { /* takes the reference */
    if (!v) return -1;
    const long x = PyLong_AsLong(v);
    Py_DECREF(v);
    if (x == -1 && PyErr_Occurred()) return -1;
    if (x < INT32_MIN || x > INT32_MAX) {
        PyErr_SetString(PyExc_OverflowError, "value does not fit a C int");
        return -1;
    }
    *out = (int)x;
    return 0;
}

/* the first two entries of a tensor's shape / stride (*b: 0 where there is only one); *dim: number of dimensions */
static int pair_of(PyObject *tuple, int *a, int *b, int *dim) { /* takes the reference */
    if (!tuple) return -1;
    int rc = 0;
    *a = *b = 0;
    *dim = PyTuple_Check(tuple) ? (int)PyTuple_GET_SIZE(tuple) : 0;
    if (*dim >= 1) rc = as_int(Py_NewRef(PyTuple_GET_ITEM(tuple, 0)), a);
    else rc = (PyErr_SetString(PyExc_IndexError, "a tensor with at least one dimension is wanted"), -1);
    if (!rc && *dim >= 2) rc = as_int(Py_NewRef(PyTuple_GET_ITEM(tuple, 1)), b);
    Py_DECREF(tuple);
    return rc;
}
static int shape_of(PyObject *t, int *a, int *b, int *dim) { return pair_of(PyObject_GetAttr(t, n_shape), a, b, dim); }
static int stride_of(PyObject *t, int *a, int *b) {
    int dim;
    return pair_of(PyObject_CallMethodNoArgs(t, n_stride), a, b, &dim);
}
static int is_true(PyObject *t, PyObject *name) { /* 1, 0 or -1 */
    PyObject *v = PyObject_GetAttr(t, name);
    if (!v) return -1;
    const int r = PyObject_IsTrue(v);
    Py_DECREF(v);
    return r;
}
static int has_dtype(PyObject *t, PyObject *dt) {
    PyObject *v = PyObject_GetAttr(t, n_dtype);
    if (!v) return -1;
    const int r = v == dt;
    Py_DECREF(v);
    return r;
}
static int numel_of(PyObject *t, Py_ssize_t *out) {
    PyObject *v = PyObject_CallMethodNoArgs(t, n_numel);
    if (!v) return -1;
    *out = PyLong_AsSsize_t(v);
    Py_DECREF(v);
    return *out == -1 && PyErr_Occurred() ? -1 : 0;
}

static int params_of(PyObject *p, muxq_params *c) {
    PyObject *v = PyObject_GetAttr(p, n_threshold);
    if (!v) return -1;
    c->threshold = (float)PyFloat_AsDouble(v);
    Py_DECREF(v);
    if (PyErr_Occurred()) return -1;
    return as_int(PyObject_GetAttr(p, n_exp_factor), &c->exp_factor) || as_int(PyObject_GetAttr(p, n_act_bits), &c->act_bits) ||
                   as_int(PyObject_GetAttr(p, n_w_bits), &c->w_bits) || as_int(PyObject_GetAttr(p, n_gran), &c->gran) ||
                   as_int(PyObject_GetAttr(p, n_aux_scale), &c->aux_scale) ||
                   as_int(PyObject_GetAttr(p, n_max_outliers), &c->max_outliers)
               ? -1
               : 0;
}

/* the current device, and the stream that is current for the calling thread on it */
static int current_place(int *device, void **out) {
    PyObject *dev = PyObject_CallNoArgs(get_device);
    if (!dev) return -1;
    PyObject *s = PyObject_CallOneArg(raw_stream, dev);
    if (as_int(dev, device)) {
        Py_XDECREF(s);
        return -1;
    }
    if (!s) return -1;
    *out = PyLong_AsVoidPtr(s);
    Py_DECREF(s);
    return PyErr_Occurred() ? -1 : 0;
}

static int current_stream(void **out) {
    int device;
    return current_place(&device, out);
}

static PyObject *stream(PyObject *self, PyObject *unused) {
    void *s;
    if (current_stream(&s)) return NULL;
    return PyLong_FromVoidPtr(s);
}

/* X [M, K] fp16 on the device with unit column stride, as the entry points want it */
static int matrix_f16(PyObject *t, void **ptr, int *rows, int *cols, int *ld) {
    int dim, cs = 0, ok = is_true(t, n_is_cuda);
    if (ok > 0) ok = has_dtype(t, dt_f16);
    if (ok < 0 || (ok && (shape_of(t, rows, cols, &dim) || stride_of(t, ld, &cs)))) return -1;
    if (!ok || dim != 2 || cs != 1) { /* (dim is set where ok) */
        PyErr_SetString(PyExc_AssertionError, "a 2-D fp16 CUDA tensor with unit column stride is wanted");
        return -1;
    }
    return tensor_ptr(t, ptr);
}

/* linear(X, w_q, s_w, params, workspace, status, out_kind, Y, bias or None) -> status code */
static PyObject *linear(PyObject *self, PyObject *const *a, Py_ssize_t n) {
    if (n != 9) return PyErr_Format(PyExc_TypeError, "linear takes 9 arguments");
    muxq_params p;
    void *x, *w, *sw, *ws, *st, *y, *bias = NULL, *s;
    int M, K, ldx, N, wk, dim, ldw, ldy, unused, out_kind;
    Py_ssize_t ws_bytes;
    if (matrix_f16(a[0], &x, &M, &K, &ldx) || shape_of(a[1], &N, &wk, &dim) || stride_of(a[1], &ldw, &unused) ||
        stride_of(a[7], &ldy, &unused) || params_of(a[3], &p) || as_int(Py_NewRef(a[6]), &out_kind))
        return NULL;
    if (a[8] != Py_None) {
        int ok = is_true(a[8], n_is_cuda);
        Py_ssize_t len = 0;
        if (ok > 0) ok = has_dtype(a[8], dt_f32);
        if (ok > 0) {
            PyObject *v = PyObject_CallMethodNoArgs(a[8], n_is_contiguous);
            ok = v ? PyObject_IsTrue(v) : -1;
            Py_XDECREF(v);
        }
        if (ok < 0 || numel_of(a[8], &len)) return NULL;
        if (!ok || len != N) {
            PyErr_SetString(PyExc_AssertionError, "the bias is a contiguous fp32 CUDA tensor of N entries");
            return NULL;
        }
        if (tensor_ptr(a[8], &bias)) return NULL;
    }
    if (tensor_ptr(a[1], &w) || tensor_ptr(a[2], &sw) || tensor_ptr(a[4], &ws) || numel_of(a[4], &ws_bytes) ||
        tensor_ptr(a[5], &st) || tensor_ptr(a[7], &y) || current_stream(&s))
        return NULL;
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = a[8] != Py_None ? f_linear_bias(x, M, K, ldx, w, ldw, sw, bias, N, &p, y, ldy, out_kind, ws, (size_t)ws_bytes, st, s)
                         : f_linear(x, M, K, ldx, w, ldw, sw, N, &p, y, ldy, out_kind, ws, (size_t)ws_bytes, st, s);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(rc);
}

/* quantize_weight(W, params, W_q, scales, workspace) -> status code */
static PyObject *quantize_weight(PyObject *self, PyObject *const *a, Py_ssize_t n) {
    if (n != 5) return PyErr_Format(PyExc_TypeError, "quantize_weight takes 5 arguments");
    muxq_params p;
    void *w, *q, *sc, *ws, *s;
    int K, N, ld;
    Py_ssize_t ws_bytes;
    if (matrix_f16(a[0], &w, &K, &N, &ld) || params_of(a[1], &p) || tensor_ptr(a[2], &q) || tensor_ptr(a[3], &sc) ||
        tensor_ptr(a[4], &ws) || numel_of(a[4], &ws_bytes) || current_stream(&s))
        return NULL;
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = f_quantize(w, K, N, ld, &p, 1, NULL, NULL, NULL, q, K, NULL, 0, sc, ws, (size_t)ws_bytes, s);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(rc);
}

/* A tensor as an operand, with what is wanted of it checked.  `what` stands in the message. */
static int refuse(const char *what, const char *why) {
    PyErr_Format(PyExc_ValueError, "%s: %s", what, why);
    return -1;
}
/* the same of an object that only behaves like a tensor */
static int info_by_attributes(PyObject *t, tensor_info *o) {
    if (as_int(PyObject_CallMethodNoArgs(t, n_get_device), &o->device)) return -1;
    PyObject *dt = PyObject_GetAttr(t, n_dtype), *shape = dt ? PyObject_GetAttr(t, n_shape) : NULL, *st = shape ? PyObject_CallMethodNoArgs(t, n_stride) : NULL;
    int rc = st ? 0 : -1;
    if (!rc) {
        o->dtype = dt == dt_f16 ? TENSOR_F16 : dt == dt_f32 ? TENSOR_F32 : dt == dt_i32 ? TENSOR_I32 : TENSOR_OTHER;
        o->dim = -1;
        if (PyTuple_Check(shape) && PyTuple_Check(st) && PyTuple_GET_SIZE(shape) == PyTuple_GET_SIZE(st)) o->dim = (int)PyTuple_GET_SIZE(shape);
        for (int i = 0; i < o->dim && i < 3 && !rc; ++i) {
            o->size[i] = PyLong_AsLongLong(PyTuple_GET_ITEM(shape, i));
            o->stride[i] = PyLong_AsLongLong(PyTuple_GET_ITEM(st, i));
            rc = PyErr_Occurred() ? -1 : 0;
        }
    }
    Py_XDECREF(dt);
    Py_XDECREF(shape);
    Py_XDECREF(st);
    return rc ? -1 : tensor_ptr(t, &o->ptr);
}
/* a CUDA tensor on the current device with unit stride along its last dimension */
static int cuda_info(PyObject *t, const char *what, int device, int dims, tensor_info *o) { /* dims: bit d for d dimensions */
    const int rc = tensor_info_of(t, o);
    if (rc < 0 || (!rc && info_by_attributes(t, o))) return -1;
    if (o->device < 0) return refuse(what, "a CUDA tensor is wanted");
    if (o->device != device) return refuse(what, "the tensor is on another device than the current one");
    if (o->dim < 1 || o->dim > 3 || !(dims >> o->dim & 1)) return refuse(what, "the number of dimensions is not what is wanted");
    for (int i = 0; i < o->dim; ++i)
        if (o->size[i] > INT32_MAX) return refuse(what, "a dimension does not fit a C int");
    if (o->size[o->dim - 1] > 1 && o->stride[o->dim - 1] != 1) return refuse(what, "unit stride along the last dimension is wanted");
    return 0;
}
static int pitch_of(const tensor_info *o, int dim, const char *what, int *ld) { /* (the stride of a dimension of one says nothing) */
    const int64_t v = o->size[dim] == 1 ? o->size[dim + 1] : o->stride[dim];
    if (v > INT32_MAX || v < 0) return refuse(what, "a pitch does not fit a C int");
    *ld = (int)v;
    return 0;
}
typedef struct {
    void *ptr;
    int kind, rows, cols, ld, dim; /* kind: MUXQ_OUT_F16 or MUXQ_OUT_F32; one dimension: rows = 1 */
} operand;
static int operand_of(PyObject *t, const char *what, int device, int dims, operand *o) {
    tensor_info v = {0};
    if (cuda_info(t, what, device, dims, &v)) return -1;
    if (v.dtype != TENSOR_F16 && v.dtype != TENSOR_F32) return refuse(what, "fp16 or fp32 is wanted");
    o->ptr = v.ptr;
    o->kind = v.dtype == TENSOR_F16 ? MUXQ_OUT_F16 : MUXQ_OUT_F32;
    o->dim = v.dim;
    o->rows = v.dim == 1 ? 1 : (int)v.size[0];
    o->cols = o->ld = (int)v.size[v.dim - 1];
    return v.dim == 1 ? 0 : pitch_of(&v, 0, what, &o->ld);
}
static int matrix_of(PyObject *t, const char *what, int device, int rows, int cols, operand *o) {
    if (operand_of(t, what, device, 1 << 2, o)) return -1;
    return o->rows == rows && o->cols == cols ? 0 : refuse(what, "the shape does not fit the other operands");
}
static int vector_f32(PyObject *t, const char *what, int device, int len, const float **out) {
    operand o;
    *out = NULL;
    if (t == Py_None) return 0;
    if (operand_of(t, what, device, 1 << 1, &o)) return -1;
    if (o.kind != MUXQ_OUT_F32 || o.cols != len) return refuse(what, "an fp32 vector of the rows' length is wanted");
    *out = o.ptr;
    return 0;
}
static int norm_of(PyObject *t, const char *what, int device, int len, muxq_norm *n) { /* (kind, weight, bias, eps) or None */
    memset(n, 0, sizeof *n);
    if (t == Py_None) return 0;
    if (!PyTuple_Check(t) || PyTuple_GET_SIZE(t) != 4) return refuse(what, "a Norm is wanted");
    if (as_int(Py_NewRef(PyTuple_GET_ITEM(t, 0)), &n->kind)) return -1;
    n->eps = (float)PyFloat_AsDouble(PyTuple_GET_ITEM(t, 3));
    if (PyErr_Occurred()) return -1;
    return vector_f32(PyTuple_GET_ITEM(t, 1), what, device, len, &n->weight) || vector_f32(PyTuple_GET_ITEM(t, 2), what, device, len, &n->bias) ? -1 : 0;
}

/* residual_norm(R or None, Y or None, pre or None, post or None, gate or None, gate_group, scale, H or None, X or None) -> status code */
static PyObject *residual_norm(PyObject *self, PyObject *const *a, Py_ssize_t n) {
    if (n != 9) return PyErr_Format(PyExc_TypeError, "residual_norm takes 9 arguments");
    operand r = {0}, y = {0}, g = {0}, h = {0}, x = {0};
    muxq_norm pre, post;
    void *s;
    int device, group;
    if (current_place(&device, &s)) return NULL;
    if (a[0] == Py_None && a[1] == Py_None) return refuse("R", "R or Y is wanted"), NULL;
    if (operand_of(a[0] != Py_None ? a[0] : a[1], "R", device, 1 << 2, &r)) return NULL;
    const int M = r.rows, D = r.cols;
    if (a[0] == Py_None) r.ptr = NULL;
    if ((a[1] != Py_None && matrix_of(a[1], "Y", device, M, D, &y)) || (a[7] != Py_None && matrix_of(a[7], "H", device, M, D, &h)) ||
        (a[8] != Py_None && matrix_of(a[8], "X", device, M, D, &x)) || norm_of(a[2], "pre", device, D, &pre) ||
        norm_of(a[3], "post", device, D, &post) || as_int(Py_NewRef(a[5]), &group))
        return NULL;
    if (a[7] != Py_None && a[0] != Py_None && h.kind != r.kind) return refuse("H", "the type of R is wanted"), NULL;
    if (a[8] != Py_None && x.kind != MUXQ_OUT_F16) return refuse("X", "fp16 is wanted"), NULL;
    if (a[4] != Py_None) {
        if (operand_of(a[4], "gate", device, 1 << 1 | 1 << 2, &g)) return NULL;
        if (group < 1) return refuse("gate_group", "at least 1 is wanted"), NULL;
        if (g.dim == 1) group = 0;
        if (g.cols != D || (g.dim == 2 && g.rows != (int)(((long long)M + group - 1) / group)))
            return refuse("gate", "the shape does not fit the other operands"), NULL;
    }
    const double scale = PyFloat_AsDouble(a[6]);
    if (PyErr_Occurred()) return NULL;
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = f_residual_norm(r.ptr, r.ld, r.ptr ? r.kind : h.kind, y.ptr, y.ld, y.kind, &post, g.ptr, g.ld, g.kind, group, (float)scale, &pre, M, D,
                         h.ptr, h.ld, x.ptr, x.ld, s);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(rc);
}

/* a 3-D fp16 tensor: [n][rows, cols] */
static int stack_of(PyObject *t, const char *what, int device, const void **ptr, int *n, int *rows, int *cols, int *ld, int64_t *stride) {
    tensor_info v = {0};
    if (cuda_info(t, what, device, 1 << 3, &v)) return -1;
    if (v.dtype != TENSOR_F16) return refuse(what, "fp16 is wanted");
    *ptr = v.ptr;
    *n = (int)v.size[0];
    *rows = (int)v.size[1];
    *cols = (int)v.size[2];
    *stride = v.stride[0];
    return pitch_of(&v, 1, what, ld);
}
static int vector_i32(PyObject *t, const char *what, int device, int len, const int32_t **out) { /* len < 0: at least one entry */
    tensor_info v = {0};
    *out = NULL;
    if (t == Py_None) return 0;
    if (cuda_info(t, what, device, 1 << 1, &v)) return -1;
    if (v.dtype != TENSOR_I32 || (len < 0 ? v.size[0] < 1 : v.size[0] != len)) return refuse(what, "an int32 vector is wanted, one entry for each row or slot");
    *out = v.ptr;
    return 0;
}

typedef struct {
    operand x, base, y;
    muxq_adapter_set set;
    const int32_t *row_slot, *status;
    int K, N;
    void *stream;
} adapter_operands;
/* X, A, B, row_slot, scale or None, rank or None, base or None, Y, status */
static int adapter_operands_of(PyObject *const *a, Py_ssize_t n, adapter_operands *o) {
    int device, slots, rank;
    if (n != 9) return PyErr_Format(PyExc_TypeError, "the adapters' calls take 9 arguments"), -1;
    memset(o, 0, sizeof *o);
    if (current_place(&device, &o->stream) || operand_of(a[0], "X", device, 1 << 2, &o->x) ||
        stack_of(a[1], "A", device, &o->set.A_f16, &o->set.slots, &o->set.max_rank, &o->K, &o->set.lda, &o->set.stride_a) ||
        stack_of(a[2], "B", device, &o->set.B_f16, &slots, &o->N, &rank, &o->set.ldb, &o->set.stride_b))
        return -1;
    if (o->x.kind != MUXQ_OUT_F16) return refuse("X", "fp16 is wanted");
    if (o->x.cols != o->K) return refuse("A", "the shape does not fit X");
    if (slots != o->set.slots || rank != o->set.max_rank) return refuse("B", "the shape does not fit A");
    if (matrix_of(a[7], "Y", device, o->x.rows, o->N, &o->y) || (a[6] != Py_None && matrix_of(a[6], "base", device, o->x.rows, o->N, &o->base)) ||
        vector_i32(a[3], "row_slot", device, o->x.rows, &o->row_slot) || vector_f32(a[4], "scale", device, slots, &o->set.scale) ||
        vector_i32(a[5], "rank", device, slots, &o->set.rank) || vector_i32(a[8], "status", device, -1, &o->status))
        return -1;
    return a[6] != Py_None && o->base.kind != o->y.kind ? refuse("base", "the type of Y is wanted") : 0;
}
/* adapters(the operands) -> status code */
static PyObject *adapters(PyObject *self, PyObject *const *a, Py_ssize_t n) {
    adapter_operands o;
    if (adapter_operands_of(a, n, &o)) return NULL;
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = f_adapters(o.x.ptr, o.x.rows, o.K, o.x.ld, &o.set, o.row_slot, o.N, o.base.ptr, o.base.ld, o.y.ptr, o.y.ld, o.y.kind, (int32_t *)o.status, o.stream);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(rc);
}
/* adapters_check(the operands) -> the status code that adapters would give for them; nothing is launched */
static PyObject *adapters_check(PyObject *self, PyObject *const *a, Py_ssize_t n) {
    adapter_operands o;
    if (adapter_operands_of(a, n, &o)) return NULL;
    return PyLong_FromLong(f_adapters_check(o.x.ptr, o.x.rows, o.K, o.x.ld, &o.set, o.row_slot, o.N, o.base.ptr, o.base.ld, o.y.ptr, o.y.ld, o.y.kind, o.status));
}

/* bind(muxq_linear, muxq_linear_bias, muxq_quantize, get_device, raw_stream, float16, float32[, muxq_residual_norm[,
 * muxq_adapters, int32[, muxq_adapters_check]]]) */
static PyObject *bind(PyObject *self, PyObject *const *a, Py_ssize_t n) {
    if (n != 7 && n != 8 && n != 10 && n != 11) return PyErr_Format(PyExc_TypeError, "bind takes 7, 8, 10 or 11 arguments");
    f_linear = (linear_fn)PyLong_AsVoidPtr(a[0]);
    f_linear_bias = (linear_bias_fn)PyLong_AsVoidPtr(a[1]);
    f_quantize = (quantize_fn)PyLong_AsVoidPtr(a[2]);
    if (n > 7) f_residual_norm = (residual_norm_fn)PyLong_AsVoidPtr(a[7]);
    if (n > 8) f_adapters = (adapters_fn)PyLong_AsVoidPtr(a[8]);
    if (n > 10) f_adapters_check = (adapters_check_fn)PyLong_AsVoidPtr(a[10]);
    if (PyErr_Occurred()) return NULL;
    Py_XSETREF(get_device, Py_NewRef(a[3]));
    Py_XSETREF(raw_stream, Py_NewRef(a[4]));
    Py_XSETREF(dt_f16, Py_NewRef(a[5]));
    Py_XSETREF(dt_f32, Py_NewRef(a[6]));
    if (n > 9) Py_XSETREF(dt_i32, Py_NewRef(a[9]));
    Py_RETURN_NONE;
}

static PyMethodDef methods[] = {
    {"bind", (PyCFunction)(void (*)(void))bind, METH_FASTCALL, "addresses of the entry points, torch's stream lookup and dtypes"},
    {"linear", (PyCFunction)(void (*)(void))linear, METH_FASTCALL, "muxq_linear / muxq_linear_bias"},
    {"quantize_weight", (PyCFunction)(void (*)(void))quantize_weight, METH_FASTCALL, "muxq_quantize(is_weight = 1)"},
    {"adapters", (PyCFunction)(void (*)(void))adapters, METH_FASTCALL, "muxq_adapters"},
    {"adapters_check", (PyCFunction)(void (*)(void))adapters_check, METH_FASTCALL, "muxq_adapters_check"},
    {"residual_norm", (PyCFunction)(void (*)(void))residual_norm, METH_FASTCALL, "muxq_residual_norm"},
    {"stream", stream, METH_NOARGS, "handle of the current stream"},
    {NULL, NULL, 0, NULL}};
static struct PyModuleDef module = {PyModuleDef_HEAD_INIT, "_calls", NULL, -1, methods, NULL, NULL, NULL, NULL};

PyMODINIT_FUNC PyInit__calls(void) {
    struct { PyObject **to; const char *name; } names[] = {
        {&n_data_ptr, "data_ptr"}, {&n_shape, "shape"}, {&n_stride, "stride"}, {&n_dtype, "dtype"}, {&n_is_cuda, "is_cuda"},
        {&n_numel, "numel"}, {&n_is_contiguous, "is_contiguous"}, {&n_get_device, "get_device"}, {&n_threshold, "threshold"}, {&n_exp_factor, "exp_factor"}, {&n_act_bits, "act_bits"},
        {&n_w_bits, "w_bits"}, {&n_gran, "gran"}, {&n_aux_scale, "aux_scale"}, {&n_max_outliers, "max_outliers"}};
    for (size_t i = 0; i < sizeof names / sizeof *names; ++i)
        if (!*names[i].to && !(*names[i].to = PyUnicode_InternFromString(names[i].name))) return NULL;
    PyObject *m = PyModule_Create(&module);
    if (m && PyModule_AddStringConstant(m, "built_for", CALLS_BUILT_FOR)) { /* by the build: Python and torch that this was compiled against */
        Py_DECREF(m);
        return NULL;
    }
    return m;
}
