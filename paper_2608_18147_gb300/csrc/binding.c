/* binding.c -- the Python side of the operators on 4-bit codes (CPython API, no torch headers).
 *
 * The other entry points synchronise, and their binding is ctypes.  These are launches of a few microseconds, so what is
 * in front of them has to be short too: here a call's tensors are looked at once (type, shape, strides, device, address), and the
 * C entry point is called.  (A ctypes binding with the same checks took 14, 22 and 9 us for a product, an attention and a cache
 * write; this takes 7 to 13, 11 to 15, with a join 14 to 20, and 5, by process and machine: equal programs differ that
 * much.)  A call returns its result; None where the arguments are not what the entry point takes, or where a gradient is asked
 * for (the caller says why); or the entry point's status.
 */
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include "../../include/ecasq.h"

typedef int (*matvec_fn)(const void *, int64_t, int32_t, int64_t, const uint8_t *, int64_t, const void *, int32_t, const void *, int64_t,
                         int32_t, int64_t, int64_t, int32_t, void *, int64_t, int32_t *, ecasq_stream_t);
typedef int (*write_fn)(const void *, int32_t, int64_t, int64_t, int64_t, const float *, int32_t, const int32_t *, const int64_t *,
                        const ecasq_cache_t *, uint64_t, int32_t *, ecasq_stream_t);
typedef int (*attend_fn)(const void *, int64_t, int64_t, int64_t, int32_t, const ecasq_cache_t *, const ecasq_cache_t *, const int32_t *,
                         int64_t, const int32_t *, const int32_t *, int64_t, float, void *, int64_t, int64_t, float *, void *, size_t,
                         int32_t *, ecasq_stream_t);

typedef int (*project_fn)(const void *, int64_t, int32_t, int64_t, const uint8_t *, int64_t, const void *, int32_t, const void *, int64_t, int32_t,
                          int64_t, int64_t, int32_t, const void *, int32_t, const void *, int64_t, void *, int64_t, void *, size_t, int32_t *,
                          ecasq_stream_t);
typedef int (*gated_fn)(const void *, int64_t, int32_t, int64_t, const uint8_t *, int64_t, const void *, int32_t, const void *, int64_t, int32_t,
                        int64_t, int64_t, int32_t, int32_t, void *, int64_t, void *, size_t, int32_t *, ecasq_stream_t);
typedef size_t (*room_fn)(int64_t, int64_t, int64_t, int32_t);
typedef int (*norm_fn)(const void *, int64_t, int32_t, int64_t, int64_t, const void *, int64_t, const void *, int32_t, float, int64_t, void *,
                       int64_t, void *, int64_t, float *, int64_t, ecasq_stream_t);

static matvec_fn call_matvec;
static project_fn call_project;
static gated_fn call_gated;
static room_fn call_room;
static norm_fn call_norm;
static write_fn call_write;
static attend_fn call_attend;
static PyObject *tensor_type, *empty, *current_device, *raw_stream, *make_workspace, *grad_enabled, *forward_ad;
/* torch's dtypes, in the order of the names below; the first three are ECASQ_F32, ECASQ_F16, ECASQ_BF16 */
enum { U8 = 3, I32 = 4, I64 = 5, E4M3 = 6, DTYPES = 7 };
static PyObject *dtypes[DTYPES];
static PyObject *s_dtype, *s_device, *s_shape, *s_stride, *s_data_ptr, *s_get_device, *s_numel, *s_requires_grad, *s_level, *s_unpack, *empty_kw;

typedef struct {
    PyObject *o;
    int type, nd;          /* index in dtypes, -1: another */
    int64_t n[4], step[4]; /* shape and strides */
    int64_t count;         /* elements */
    void *at;
    long device;
} Tensor;

static int numbers(PyObject *tuple, int64_t *to, int nd) {
    for (int i = 0; i < nd; i++) {
        to[i] = PyLong_AsLongLong(PyTuple_GET_ITEM(tuple, i));
        if (to[i] == -1 && PyErr_Occurred()) return 0;
    }
    return 1;
}

/* What a CUDA tensor of one to four dimensions is; 0 (and no exception) for anything else. */
static int look(PyObject *o, Tensor *t) {
    PyObject *dtype = NULL, *shape = NULL, *stride = NULL, *at = NULL, *device = NULL;
    int ok = 0;
    if (!tensor_type || !PyObject_TypeCheck(o, (PyTypeObject *)tensor_type)) return 0;
    t->o = o;
    if (!(dtype = PyObject_GetAttr(o, s_dtype)) || !(shape = PyObject_GetAttr(o, s_shape)) || !PyTuple_Check(shape)) goto done;
    if (!(stride = PyObject_CallMethodNoArgs(o, s_stride)) || !PyTuple_Check(stride)) goto done;
    t->nd = (int)PyTuple_GET_SIZE(shape);
    if (t->nd < 1 || t->nd > 4 || PyTuple_GET_SIZE(stride) != t->nd) goto done;
    if (!numbers(shape, t->n, t->nd) || !numbers(stride, t->step, t->nd)) goto done;
    if (!(device = PyObject_CallMethodNoArgs(o, s_get_device)) || !(at = PyObject_CallMethodNoArgs(o, s_data_ptr))) goto done;
    t->device = PyLong_AsLong(device);
    t->at = PyLong_AsVoidPtr(at);
    if (PyErr_Occurred()) goto done;
    t->type = -1;
    for (int i = 0; i < DTYPES; i++)
        if (dtype == dtypes[i]) t->type = i;
    t->count = 1;
    for (int i = 0; i < t->nd; i++) t->count *= t->n[i];
    ok = t->device >= 0;
done:
    if (!ok) PyErr_Clear();
    Py_XDECREF(dtype);
    Py_XDECREF(shape);
    Py_XDECREF(stride);
    Py_XDECREF(at);
    Py_XDECREF(device);
    return ok;
}

static int contiguous(const Tensor *t) {
    int64_t step = 1;
    for (int i = t->nd - 1; i >= 0; i--) {
        if (t->n[i] != 1 && t->step[i] != step) return 0;
        step *= t->n[i];
    }
    return 1;
}

/* The current stream of the device, which has to be the current one. */
static int stream_of(long device, ecasq_stream_t *to) {
    PyObject *now = PyObject_CallNoArgs(current_device), *index = NULL, *raw = NULL;
    int ok = 0;
    if (now && PyLong_AsLong(now) == device && (index = PyLong_FromLong(device)) && (raw = PyObject_CallOneArg(raw_stream, index))) {
        *to = (ecasq_stream_t)PyLong_AsVoidPtr(raw);
        ok = !PyErr_Occurred();
    }
    if (!ok) PyErr_Clear();
    Py_XDECREF(now);
    Py_XDECREF(index);
    Py_XDECREF(raw);
    return ok;
}

/* torch.empty(shape, dtype=..., device=that of `like`) */
static PyObject *new_tensor(int nd, const int64_t *n, int type, const Tensor *like) {
    PyObject *shape = PyTuple_New(nd), *device = PyObject_GetAttr(like->o, s_device), *made = NULL;
    for (int i = 0; shape && i < nd; i++) {
        PyObject *v = PyLong_FromLongLong(n[i]);
        if (!v) Py_CLEAR(shape);
        else PyTuple_SET_ITEM(shape, i, v);
    }
    if (shape && device) {
        PyObject *args[3] = {shape, dtypes[type], device};
        made = PyObject_Vectorcall(empty, args, 1, empty_kw);
    }
    Py_XDECREF(shape);
    Py_XDECREF(device);
    return made;
}

/* A status word: None, or the first element of an int32 tensor of any shape on the device. */
static int status_of(PyObject *o, long device, int32_t **to) {
    PyObject *dtype, *count = NULL, *at = NULL, *where = NULL;
    int ok = 0;
    *to = NULL;
    if (o == Py_None) return 1;
    if (!PyObject_TypeCheck(o, (PyTypeObject *)tensor_type)) return 0;
    if ((dtype = PyObject_GetAttr(o, s_dtype)) == dtypes[I32] && (count = PyObject_CallMethodNoArgs(o, s_numel)) &&
        (where = PyObject_CallMethodNoArgs(o, s_get_device)) && (at = PyObject_CallMethodNoArgs(o, s_data_ptr))) {
        ok = PyLong_AsLongLong(count) > 0 && PyLong_AsLong(where) == device;
        *to = (int32_t *)PyLong_AsVoidPtr(at);
        ok = ok && !PyErr_Occurred();
    }
    if (!ok) PyErr_Clear();
    Py_XDECREF(dtype);
    Py_XDECREF(count);
    Py_XDECREF(where);
    Py_XDECREF(at);
    return ok;
}

/* Whether a gradient or a tangent of one of the given tensors (NULL and None allowed) is asked for, which these calls do not give. */
static int tracked(PyObject *const *o, int n) {
    PyObject *on = PyObject_CallNoArgs(grad_enabled), *level = PyObject_GetAttr(forward_ad, s_level);
    int found = !on;
    const int dual = level && PyLong_AsLong(level) >= 0;
    PyErr_Clear();
    for (int i = 0; i < n && !found; i++) {
        if (!o[i] || o[i] == Py_None) continue;
        if (on == Py_True) {
            PyObject *wants = PyObject_GetAttr(o[i], s_requires_grad);
            found = wants != Py_False;
            Py_XDECREF(wants);
        }
        if (dual && !found) {
            PyObject *pair = PyObject_CallMethodOneArg(forward_ad, s_unpack, o[i]);
            found = !pair || !PyTuple_Check(pair) || PyTuple_GET_SIZE(pair) != 2 || PyTuple_GET_ITEM(pair, 1) != Py_None;
            Py_XDECREF(pair);
        }
    }
    Py_XDECREF(on);
    Py_XDECREF(level);
    PyErr_Clear();
    return found;
}

#define NO Py_RETURN_NONE

/* The operands of a product with a coded matrix: x [b, k] or [k], codes, levels, scales, group; `rows` of the matrix. */
typedef struct {
    Tensor x, codes, levels, scales;
    int64_t k, rows, b;
    int32_t group;
} Product;

static int product_of(PyObject *const *v, Product *p) {
    if (!look(v[0], &p->x) || !look(v[1], &p->codes) || !look(v[2], &p->levels) || !look(v[3], &p->scales)) return 0;
    const Tensor *x = &p->x, *codes = &p->codes, *levels = &p->levels, *scales = &p->scales;
    const long long group = PyLong_AsLongLong(v[4]);
    if (group == -1 && PyErr_Occurred()) {
        PyErr_Clear();
        return 0;
    }
    if (x->type < 0 || x->type > 2 || x->nd > 2 || codes->type != U8 || codes->nd != 2 || levels->type != x->type || levels->nd != 1 ||
        scales->nd != 2 || (scales->type != x->type && scales->type != ECASQ_F32) || group < 32 || group % 32 || group > INT32_MAX / 2)
        return 0;
    p->k = x->n[x->nd - 1];
    p->rows = codes->n[0];
    p->b = x->nd == 2 ? x->n[0] : 1;
    p->group = (int32_t)group;
    if ((p->k > 1 && x->step[x->nd - 1] != 1) || codes->step[1] != 1 || codes->n[1] < (p->k + 127) / 128 * 64 || levels->n[0] < 1 || levels->n[0] > 16 ||
        !contiguous(levels) || scales->n[0] != p->rows || scales->n[1] < (p->k + group - 1) / group || (scales->n[1] > 1 && scales->step[1] != 1))
        return 0;
    return codes->device == x->device && levels->device == x->device && scales->device == x->device;
}
static int64_t x_row(const Product *p) { return p->x.nd == 2 ? p->x.step[0] : p->k; }
static int64_t code_row(const Product *p) { return p->rows > 1 ? p->codes.step[0] : p->codes.n[1]; }
static int64_t scale_row(const Product *p) { return p->rows > 1 ? p->scales.step[0] : p->scales.n[1]; }

/* A tensor [b, n], or [n] where x has one dimension, of type `type` with contiguous rows, on x's device. */
static int rows_like(const Tensor *t, const Tensor *x, int64_t b, int64_t n, int type) {
    return t->type == type && t->nd == x->nd && t->device == x->device && t->n[t->nd - 1] == n && (t->nd == 1 || t->n[0] == b) && (n < 2 || t->step[t->nd - 1] == 1);
}
/* What new_tensor made: all but its address is known. */
static int look_at_made(PyObject *o, int nd, const int64_t *n, int type, const Tensor *like, Tensor *t) {
    PyObject *at = PyObject_CallMethodNoArgs(o, s_data_ptr);
    if (!at) return 0;
    t->o = o;
    t->type = type;
    t->nd = nd;
    t->device = like->device;
    t->at = PyLong_AsVoidPtr(at);
    t->count = 1;
    for (int i = nd - 1; i >= 0; i--) {
        t->n[i] = n[i];
        t->step[i] = t->count;
        t->count *= n[i];
    }
    Py_DECREF(at);
    return !PyErr_Occurred();
}
/* `given`, or such a tensor made where that is None; NULL with an exception, or None, where it is not one. */
static PyObject *output_of(PyObject *given, const Tensor *x, int64_t b, int64_t n, int type, Tensor *y) {
    if (given == Py_None) {
        const int64_t shape[2] = {x->nd == 2 ? b : n, n};
        PyObject *made = new_tensor(x->nd, shape, type, x);
        if (made && !look_at_made(made, x->nd, shape, type, x, y)) Py_CLEAR(made);
        return made;
    }
    if (look(given, y) && rows_like(y, x, b, n, type)) return Py_NewRef(given);
    NO;
}
static int64_t row_step(const Tensor *t, int64_t n) { return t->nd == 2 ? t->step[0] : n; }

/* matvec(x, codes, levels, scales, group, out, status) */
static PyObject *py_matvec(PyObject *self, PyObject *const *v, Py_ssize_t n_args) {
    Product p;
    Tensor y;
    int32_t *status;
    ecasq_stream_t stream;
    PyObject *made;
    if (n_args != 7 || !product_of(v, &p)) NO;
    PyObject *const floats[] = {v[0], v[2], v[3], v[5]};
    if (tracked(floats, 4)) NO;
    if (!status_of(v[6], p.x.device, &status) || !stream_of(p.x.device, &stream)) NO;
    if (!(made = output_of(v[5], &p.x, p.b, p.rows, p.x.type, &y)) || made == Py_None) return made;
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = call_matvec(p.x.at, x_row(&p), p.x.type, p.b, p.codes.at, code_row(&p), p.levels.at, (int32_t)p.levels.n[0], p.scales.at, scale_row(&p), p.scales.type,
                     p.rows, p.k, p.group, y.at, row_step(&y, p.rows), status, stream);
    Py_END_ALLOW_THREADS
    if (!rc) return made;
    Py_DECREF(made);
    return PyLong_FromLong(rc);
}

/* A product with an epilogue: project(x, codes, levels, scales, group, bias, activation, residual, out, ws, status), and gated(x, codes,
 * levels, scales, group, activation, out, ws, status) with `gated`. */
static PyObject *layer_product(PyObject *const *v, int gated) {
    Product p;
    Tensor bias, residual, y, ws;
    int32_t *status;
    ecasq_stream_t stream;
    PyObject *made, *space = NULL;
    PyObject *const *w = v + (gated ? 6 : 8); /* out, ws, status */
    if (!product_of(v, &p) || (gated && p.rows % 2)) NO;
    const int64_t n = gated ? p.rows / 2 : p.rows;
    const long act = PyLong_AsLong(v[gated ? 5 : 6]);
    if (act == -1 && PyErr_Occurred()) {
        PyErr_Clear();
        NO;
    }
    bias.at = residual.at = ws.at = NULL;
    ws.count = 0;
    if (!gated && v[5] != Py_None && (!look(v[5], &bias) || bias.type != p.x.type || bias.nd != 1 || bias.n[0] != n || !contiguous(&bias) || bias.device != p.x.device)) NO;
    if (!gated && v[7] != Py_None && (!look(v[7], &residual) || !rows_like(&residual, &p.x, p.b, n, p.x.type))) NO;
    PyObject *const floats[] = {v[0], v[2], v[3], w[0], gated ? Py_None : v[5], gated ? Py_None : v[7]};
    if (tracked(floats, 6)) NO;
    if (!status_of(w[2], p.x.device, &status) || !stream_of(p.x.device, &stream)) NO;
    if (w[1] != Py_None && (!look(w[1], &ws) || ws.type != U8 || ws.device != p.x.device || !contiguous(&ws))) NO;
    if (!(made = output_of(w[0], &p.x, p.b, n, p.x.type, &y)) || made == Py_None) return made;
    if (w[1] == Py_None) {
        /* (16-bit rows of x on 16-byte boundaries need none) */
        const int plain = p.x.type != ECASQ_F32 && ((uintptr_t)p.x.at & 15) == 0 && (p.b == 1 || x_row(&p) % 8 == 0);
        const int64_t room = plain ? 0 : (int64_t)call_room(p.b, p.rows, p.k, p.x.type);
        if (room && (!(space = new_tensor(1, &room, U8, &p.x)) || !look(space, &ws))) {
            Py_XDECREF(space);
            Py_DECREF(made);
            return PyErr_Occurred() ? NULL : Py_NewRef(Py_None);
        }
    }
    int rc;
    Py_BEGIN_ALLOW_THREADS
    if (gated)
        rc = call_gated(p.x.at, x_row(&p), p.x.type, p.b, p.codes.at, code_row(&p), p.levels.at, (int32_t)p.levels.n[0], p.scales.at, scale_row(&p), p.scales.type, n, p.k,
                        p.group, (int32_t)act, y.at, row_step(&y, n), ws.at, (size_t)ws.count, status, stream);
    else
        rc = call_project(p.x.at, x_row(&p), p.x.type, p.b, p.codes.at, code_row(&p), p.levels.at, (int32_t)p.levels.n[0], p.scales.at, scale_row(&p), p.scales.type, n,
                          p.k, p.group, bias.at, (int32_t)act, residual.at, residual.at ? row_step(&residual, n) : 0, y.at, row_step(&y, n), ws.at, (size_t)ws.count,
                          status, stream);
    Py_END_ALLOW_THREADS
    Py_XDECREF(space);
    if (!rc) return made;
    Py_DECREF(made);
    return PyLong_FromLong(rc);
}
static PyObject *py_project(PyObject *self, PyObject *const *v, Py_ssize_t n_args) {
    if (n_args != 11) NO;
    return layer_product(v, 0);
}
static PyObject *py_gated(PyObject *self, PyObject *const *v, Py_ssize_t n_args) {
    if (n_args != 9) NO;
    return layer_product(v, 1);
}

/* norm(x, weight, eps, residual, group, out, out_sum, out_scales): y; (y, scales); with a residual the sum behind them */
static PyObject *py_norm(PyObject *self, PyObject *const *v, Py_ssize_t n_args) {
    Tensor x, weight, residual, y, sum, scales;
    ecasq_stream_t stream;
    PyObject *made[3] = {NULL, NULL, NULL}, *all = NULL;
    if (n_args != 8 || !look(v[0], &x) || !look(v[1], &weight)) NO;
    const double eps = PyFloat_AsDouble(v[2]);
    const long long group = v[4] == Py_None ? 0 : PyLong_AsLongLong(v[4]);
    if (PyErr_Occurred()) {
        PyErr_Clear();
        NO;
    }
    if (x.type < 0 || x.type > 2 || x.nd > 2) NO;
    const int64_t k = x.n[x.nd - 1], b = x.nd == 2 ? x.n[0] : 1;
    if ((k > 1 && x.step[x.nd - 1] != 1) || weight.nd != 1 || weight.n[0] != k || !contiguous(&weight) || (weight.type != x.type && weight.type != ECASQ_F32) ||
        weight.device != x.device || k < 1 || (v[4] != Py_None && group < 1))
        NO;
    residual.at = sum.at = scales.at = NULL;
    if (v[3] != Py_None && (!look(v[3], &residual) || !rows_like(&residual, &x, b, k, x.type))) NO;
    if ((v[3] == Py_None && v[6] != Py_None) || (!group && v[7] != Py_None)) NO;
    PyObject *const floats[] = {v[0], v[1], v[3], v[5], v[6], v[7]};
    if (tracked(floats, 6)) NO;
    if (!stream_of(x.device, &stream)) NO;
    const int64_t groups = !group ? 0 : group >= k ? 1 : (k + group - 1) / group;
    if (!(made[0] = output_of(v[5], &x, b, k, group ? E4M3 : x.type, &y)) || made[0] == Py_None) return made[0];
    if (group && (!(made[1] = output_of(v[7], &x, b, groups, ECASQ_F32, &scales)) || made[1] == Py_None)) goto done;
    if (v[3] != Py_None && (!(made[2] = output_of(v[6], &x, b, k, x.type, &sum)) || made[2] == Py_None)) goto done;
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = call_norm(x.at, row_step(&x, k), x.type, b, k, residual.at, v[3] != Py_None ? row_step(&residual, k) : 0, weight.at, weight.type, (float)eps, group, y.at,
                   row_step(&y, k), sum.at, v[3] != Py_None ? row_step(&sum, k) : 0, scales.at, group ? row_step(&scales, groups) : 0, stream);
    Py_END_ALLOW_THREADS
    if (rc) all = PyLong_FromLong(rc);
    else if (made[1] && made[2]) all = PyTuple_Pack(3, made[0], made[1], made[2]);
    else if (made[1] || made[2]) all = PyTuple_Pack(2, made[0], made[1] ? made[1] : made[2]);
    else all = Py_NewRef(made[0]);
done:
    if (!all && !PyErr_Occurred()) all = Py_NewRef(Py_None);
    for (int i = 0; i < 3; i++) Py_XDECREF(made[i]);
    return all;
}

/* One side of a paged cache: rows and, for coded ones, levels (else None). */
static int cache_of(PyObject *rows, PyObject *levels, ecasq_cache_t *c, long *device) {
    Tensor r, l;
    if (!look(rows, &r) || r.nd != 4 || r.step[3] != 1) return 0;
    for (int i = 0; i < 4; i++)
        if (r.n[i] > INT32_MAX && i) return 0;
    *c = (ecasq_cache_t){r.at, NULL, r.step[0], r.step[1], r.step[2], 0, 0, 0, r.n[0], (int32_t)r.n[1], (int32_t)r.n[2], (int32_t)r.n[3], r.type, 0, 0};
    *device = r.device;
    if (levels == Py_None) return r.type >= 0 && r.type <= 2;
    if (r.type != U8 || !look(levels, &l) || l.nd != 4 || l.step[3] != 1 || (l.type != ECASQ_F16 && l.type != ECASQ_BF16) || l.device != r.device ||
        l.n[0] != r.n[0] || l.n[1] != r.n[1] || l.n[2] != r.n[2] || (l.n[3] != 8 && l.n[3] != 16) || r.n[3] > 1 << 20)
        return 0;
    c->levels = l.at;
    c->level_page = l.step[0];
    c->level_slot = l.step[1];
    c->level_head = l.step[2];
    c->d = (int32_t)(2 * r.n[3]);
    c->type = l.type;
    c->levels_n = (int32_t)l.n[3];
    return 1;
}

/* cache_write(x, Q, m, slots, codes, levels, seed, status): None where it is refused, else the status */
static PyObject *py_write(PyObject *self, PyObject *const *v, Py_ssize_t n_args) {
    Tensor x, q, m, slots;
    ecasq_cache_t c;
    int32_t *status;
    ecasq_stream_t stream;
    long device;
    if (n_args != 8 || v[5] == Py_None || !look(v[0], &x) || !look(v[1], &q) || !look(v[3], &slots) || !cache_of(v[4], v[5], &c, &device)) NO;
    const uint64_t seed = PyLong_AsUnsignedLongLongMask(v[6]);
    if (PyErr_Occurred()) {
        PyErr_Clear();
        NO;
    }
    const int64_t n = slots.count, rows = n * c.heads, s = q.n[q.nd - 1];
    if (x.nd != 3 || (x.type != ECASQ_F32 && x.type != c.type) || x.n[0] != n || x.n[1] != c.heads || x.n[2] != c.d || x.step[2] != 1 || slots.type != I64 ||
        !contiguous(&slots) || q.type != ECASQ_F32 || !contiguous(&q) || s < 1 || s > c.levels_n || q.count != rows * s || q.device != x.device ||
        slots.device != x.device || device != x.device)
        NO;
    m.at = NULL;
    if (v[2] != Py_None && (!look(v[2], &m) || m.type != I32 || m.count != rows || !contiguous(&m) || m.device != x.device)) NO;
    PyObject *const floats[] = {v[0], v[1], v[5]};
    if (tracked(floats, 3)) NO;
    if (!status_of(v[7], x.device, &status) || !stream_of(x.device, &stream)) NO;
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = call_write(x.at, x.type, n, x.step[0], x.step[1], q.at, (int32_t)s, m.at, slots.at, &c, seed, status, stream);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(rc);
}

/* attend(q, k, v, table, lengths, scale, starts, k_levels, v_levels, max_len, out, ws, status) */
static PyObject *py_attend(PyObject *self, PyObject *const *v, Py_ssize_t n_args) {
    Tensor q, table, lengths, starts, out, ws, lse;
    ecasq_cache_t ck, cv;
    int32_t *status;
    ecasq_stream_t stream;
    long dk, dv;
    PyObject *made = NULL, *space = NULL, *sums = NULL, *both = NULL;
    if (n_args != 13 || !look(v[0], &q) || !cache_of(v[1], v[7], &ck, &dk) || !cache_of(v[2], v[8], &cv, &dv) || !look(v[3], &table) || !look(v[4], &lengths)) NO;
    if (q.nd != 3 || q.step[2] != 1 || q.type != ck.type || q.type != cv.type || ck.levels_n != cv.levels_n || ck.d != cv.d || q.n[2] != ck.d || q.n[1] > INT32_MAX ||
        dk != q.device || dv != q.device || table.type != I32 || table.nd != 2 || table.n[0] != q.n[0] || (table.n[1] > 1 && table.step[1] != 1) ||
        table.device != q.device || lengths.type != I32 || lengths.nd != 1 || lengths.n[0] != q.n[0] || !contiguous(&lengths) || lengths.device != q.device)
        NO;
    starts.at = NULL;
    if (v[6] != Py_None && (!look(v[6], &starts) || starts.type != I32 || starts.nd != 1 || starts.n[0] != q.n[0] || !contiguous(&starts) || starts.device != q.device)) NO;
    const int64_t b = q.n[0], heads = q.n[1], most = table.n[1] * ck.page_size, max_len = v[9] == Py_None ? most : PyLong_AsLongLong(v[9]);
    const double scale = v[5] == Py_None ? 0.0 : PyFloat_AsDouble(v[5]);
    if (PyErr_Occurred()) {
        PyErr_Clear();
        NO;
    }
    PyObject *const floats[] = {v[0], v[1], v[2], v[7], v[8], v[10]};
    if (tracked(floats, 6)) NO;
    if (max_len < 0 || max_len > most || !status_of(v[12], q.device, &status) || !stream_of(q.device, &stream)) NO;
    if (!(made = v[10] == Py_None ? new_tensor(3, q.n, q.type, &q) : Py_NewRef(v[10]))) goto done;
    if (!look(made, &out) || out.type != q.type || out.nd != 3 || out.n[0] != b || out.n[1] != heads || out.n[2] != q.n[2] || out.step[2] != 1 || out.device != q.device) {
        both = Py_NewRef(Py_None);
        goto done;
    }
    space = v[11] == Py_None ? PyObject_CallFunction(make_workspace, "LLiiL", (long long)b, (long long)heads, ck.heads, ck.d, (long long)max_len) : Py_NewRef(v[11]);
    if (!space) goto done;
    if (!look(space, &ws) || ws.type != U8 || ws.device != q.device || !contiguous(&ws)) {
        both = Py_NewRef(Py_None);
        goto done;
    }
    const int64_t shape[2] = {b, heads};
    if (!(sums = new_tensor(2, shape, ECASQ_F32, &q))) goto done;
    if (!look(sums, &lse)) {
        both = Py_NewRef(Py_None);
        goto done;
    }
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = call_attend(q.at, q.step[0], q.step[1], b, (int32_t)heads, &ck, &cv, table.at, b > 1 ? table.step[0] : table.n[1], lengths.at, starts.at, max_len,
                     v[5] == Py_None ? (float)(1.0 / __builtin_sqrt((double)q.n[2])) : (float)scale, out.at, out.step[0], out.step[1], lse.at, ws.at,
                     (size_t)ws.count, status, stream);
    Py_END_ALLOW_THREADS
    both = rc ? PyLong_FromLong(rc) : PyTuple_Pack(2, made, sums);
done:
    Py_XDECREF(made);
    Py_XDECREF(space);
    Py_XDECREF(sums);
    return both;
}

/* setup(addresses of matvec, cache_write, attend, project, gated, workspace_size_project, norm, torch.Tensor, torch.empty, current
 * device, raw stream, workspace, torch.is_grad_enabled, torch.autograd.forward_ad, dtypes) */
static PyObject *py_setup(PyObject *self, PyObject *args) {
    unsigned long long a[7];
    PyObject *o[7], *types;
    if (!PyArg_ParseTuple(args, "KKKKKKKOOOOOOOO!", &a[0], &a[1], &a[2], &a[3], &a[4], &a[5], &a[6], &o[0], &o[1], &o[2], &o[3], &o[4], &o[5], &o[6], &PyTuple_Type,
                          &types))
        return NULL;
    if (PyTuple_GET_SIZE(types) != DTYPES || !PyType_Check(o[0])) {
        PyErr_SetString(PyExc_TypeError, "setup: seven dtypes and a tensor type");
        return NULL;
    }
    call_matvec = (matvec_fn)(uintptr_t)a[0];
    call_write = (write_fn)(uintptr_t)a[1];
    call_attend = (attend_fn)(uintptr_t)a[2];
    call_project = (project_fn)(uintptr_t)a[3];
    call_gated = (gated_fn)(uintptr_t)a[4];
    call_room = (room_fn)(uintptr_t)a[5];
    call_norm = (norm_fn)(uintptr_t)a[6];
    PyObject **to[7] = {&tensor_type, &empty, &current_device, &raw_stream, &make_workspace, &grad_enabled, &forward_ad};
    for (int i = 0; i < 7; i++) Py_XSETREF(*to[i], Py_NewRef(o[i]));
    for (int i = 0; i < DTYPES; i++) Py_XSETREF(dtypes[i], Py_NewRef(PyTuple_GET_ITEM(types, i)));
    Py_RETURN_NONE;
}

static PyMethodDef methods[] = {{"setup", py_setup, METH_VARARGS, NULL},
                                {"matvec", (PyCFunction)(void (*)(void))py_matvec, METH_FASTCALL, NULL},
                                {"project", (PyCFunction)(void (*)(void))py_project, METH_FASTCALL, NULL},
                                {"gated", (PyCFunction)(void (*)(void))py_gated, METH_FASTCALL, NULL},
                                {"norm", (PyCFunction)(void (*)(void))py_norm, METH_FASTCALL, NULL},
                                {"cache_write", (PyCFunction)(void (*)(void))py_write, METH_FASTCALL, NULL},
                                {"attend", (PyCFunction)(void (*)(void))py_attend, METH_FASTCALL, NULL},
                                {NULL, NULL, 0, NULL}};
static struct PyModuleDef module = {PyModuleDef_HEAD_INIT, "_codes", NULL, -1, methods, NULL, NULL, NULL, NULL};

PyMODINIT_FUNC PyInit__codes(void) {
    PyObject **names[] = {&s_dtype, &s_device, &s_shape, &s_stride, &s_data_ptr, &s_get_device, &s_numel, &s_requires_grad, &s_level, &s_unpack};
    const char *text[] = {"dtype", "device", "shape", "stride", "data_ptr", "get_device", "numel", "requires_grad", "_current_level", "unpack_dual"};
    for (int i = 0; i < 10; i++)
        if (!(*names[i] = PyUnicode_InternFromString(text[i]))) return NULL;
    if (!(empty_kw = PyTuple_Pack(2, s_dtype, s_device))) return NULL;
    return PyModule_Create(&module);
}
