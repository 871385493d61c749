/* CPython entry points of the paged cache's calls: argument marshalling of one launch, in C.
 *
 * A decoding step's kernels last a few microseconds each; describing a cache, a batch and a call through ctypes and checking
 * eight tensors in Python took 20 us.  Here the same takes 4 to 5 (one token through attention, with its descriptions and
 * the result's allocation: 25 -> 12 us of the host, the kernel takes 8).
 *
 * What is as it should be goes straight to the library; whatever is not (keywords, another type, a view, a wrong size) is handed
 * to the function of the same name in cache_binding.py, which makes the call or says what is wrong.  Descriptions made here hold
 * the C struct (buffer protocol) and references to the tensors that it points to.
 */
#define PY_SSIZE_T_CLEAN
#include <Python.h>
#include <string.h>

#include "spmm_cache.h"

enum { CACHE, BATCH, APPEND, ATTEND, SELECT, WEIGH, EVICT, KINDS };
static const Py_ssize_t sizes[KINDS] = {sizeof(spmm_cache_t), sizeof(spmm_batch_t), sizeof(spmm_append_t), sizeof(spmm_attend_t),
                                        sizeof(spmm_select_t), sizeof(spmm_weigh_t), sizeof(spmm_evict_t)};

typedef struct {
    PyObject_HEAD
    int kind;
    PyObject *keep;
    union {
        spmm_cache_t cache;
        spmm_batch_t batch;
        spmm_append_t append;
        spmm_attend_t attend;
        spmm_select_t select;
        spmm_weigh_t weigh;
        spmm_evict_t evict;
    } u;
} Record;

static int record_buffer(PyObject *self, Py_buffer *view, int flags)
{
    return PyBuffer_FillInfo(view, self, &((Record *)self)->u, sizes[((Record *)self)->kind], 0, flags);
}
static void record_free(PyObject *self)
{
    Py_XDECREF(((Record *)self)->keep);
    PyObject_Free(self);
}
/* the tensors, as cache_binding.py keeps them: of a call to append (q_weight, k_weight, rope, positions) */
static PyObject *record_keep(PyObject *self, void *unused)
{
    const Record *const r = (Record *)self;
    (void)unused;
    if (r->kind != APPEND) return Py_NewRef(r->keep);
    return PyTuple_Pack(4, PyTuple_GET_ITEM(r->keep, 4), PyTuple_GET_ITEM(r->keep, 5), PyTuple_GET_ITEM(r->keep, 7), Py_None);
}
static PyGetSetDef record_attributes[] = {{"_keepalive", record_keep, NULL, NULL, NULL}, {NULL, NULL, NULL, NULL, NULL}};
static PyBufferProcs record_as_buffer = {record_buffer, NULL};
static PyTypeObject RecordType = {
    PyVarObject_HEAD_INIT(NULL, 0).tp_name = "spmm_cache_record", .tp_basicsize = sizeof(Record), .tp_dealloc = record_free,
    .tp_as_buffer = &record_as_buffer, .tp_getset = record_attributes, .tp_flags = Py_TPFLAGS_DEFAULT,
    .tp_doc = "A cache, a batch or a call of include/spmm_cache.h, described"};

enum { F_APPEND, F_ATTEND, F_ATTEND_WORK, F_FORK, F_COMPACT, F_CACHE_WORK, F_BOUNDS, F_SCORE, F_SELECT, F_SELECTED_WORK, F_SELECTED, F_WEIGH_WORK, F_WEIGH, F_EVICT,
       FUNCTIONS };
static void *functions[FUNCTIONS];
enum { S_MAKE_CACHE, S_MAKE_BATCH, S_MAKE_APPEND, S_MAKE_ATTEND, S_APPEND, S_ATTEND, S_ATTEND_WORK, S_FORK, S_COMPACT, S_CACHE_WORK,
       S_MAKE_SELECT, S_MAKE_WEIGH, S_MAKE_EVICT, S_BOUNDS, S_SCORE, S_SELECT, S_SELECTED_WORK, S_SELECTED, S_WEIGH_WORK, S_WEIGH, S_EVICT, SLOW };
static PyObject *slow[SLOW], *py_check;
static PyObject *s_data_ptr, *s_nbytes, *s_is_contiguous, *s_dtype, *s_is_cuda, *s_shape;

enum { BF16, F32, S8, U8, S32, TYPES };
static const char *const type_names[TYPES] = {"torch.bfloat16", "torch.float32", "torch.int8", "torch.uint8", "torch.int32"};
static PyObject *types[TYPES];      /* the dtype objects, once they have been seen */

/* a tensor's type, -1: another */
static int type_of(PyObject *t)
{
    PyObject *d = PyObject_GetAttr(t, s_dtype);
    int k = -1;
    if (!d) return -1;
    for (int i = 0; i < TYPES && k < 0; ++i)
        if (d == types[i]) k = i;
    if (k < 0) {
        PyObject *name = PyObject_Str(d);
        for (int i = 0; name && i < TYPES; ++i)
            if (!types[i] && PyUnicode_CompareWithASCIIString(name, type_names[i]) == 0) {
                types[i] = Py_NewRef(d);    /* (a dtype lives as long as torch does) */
                k = i;
            }
        Py_XDECREF(name);
    }
    Py_DECREF(d);
    return k;
}

static int is_true(PyObject *v)     /* steals v */
{
    const int yes = v == Py_True;
    Py_XDECREF(v);
    return yes;
}

/* The address of a contiguous device tensor of this type with at least `need` bytes, of a raw integer, or NULL for None; 0: not so. */
static int operand(PyObject *t, int type, int64_t need, void **out)
{
    *out = NULL;
    if (t == Py_None) return 1;
    PyObject *v = t;
    if (PyLong_CheckExact(t)) {
        Py_INCREF(v);
    } else {
        if (type >= 0 && type_of(t) != type) return 0;
        if (!is_true(PyObject_CallMethodNoArgs(t, s_is_contiguous)) || !is_true(PyObject_GetAttr(t, s_is_cuda))) return 0;
        if (need > 0) {
            PyObject *n = PyObject_GetAttr(t, s_nbytes);
            const long long have = n && PyLong_CheckExact(n) ? PyLong_AsLongLong(n) : -1;
            Py_XDECREF(n);
            if (have < need) return 0;
        }
        v = PyObject_CallMethodNoArgs(t, s_data_ptr);
        if (!v || !PyLong_CheckExact(v)) {
            Py_XDECREF(v);
            return 0;
        }
    }
    *out = (void *)(uintptr_t)PyLong_AsUnsignedLongLongMask(v);
    Py_DECREF(v);
    return !PyErr_Occurred();
}

static int shape_of(PyObject *t, int dims, int64_t *out)
{
    PyObject *s = PyObject_GetAttr(t, s_shape);
    int ok = s && PyTuple_Check(s) && PyTuple_GET_SIZE(s) == dims;
    for (int i = 0; ok && i < dims; ++i) {
        out[i] = PyLong_AsLongLong(PyTuple_GET_ITEM(s, i));
        ok = out[i] >= 0;
    }
    Py_XDECREF(s);
    return ok;
}

static int number(PyObject *v, int64_t *out)
{
    if (!PyLong_Check(v)) return 0;     /* (truth values are) */
    *out = PyLong_AsLongLong(v);
    return !PyErr_Occurred();
}
static int real(PyObject *v, float *out)
{
    if (!PyFloat_Check(v) && !PyLong_Check(v)) return 0;
    *out = (float)PyFloat_AsDouble(v);
    return !PyErr_Occurred();
}
static int name_in(PyObject *v, const char *const *names, const int *values, int n, int *out)
{
    if (!PyUnicode_Check(v)) return 0;
    for (int i = 0; i < n; ++i)
        if (PyUnicode_CompareWithASCIIString(v, names[i]) == 0) {
            *out = values[i];
            return 1;
        }
    return 0;
}

/* a record's struct, or that of another object with a buffer of this size (ctypes structures): NULL if neither */
static const void *description(PyObject *v, int kind, Py_buffer *b)
{
    b->obj = NULL;
    if (Py_TYPE(v) == &RecordType) return ((Record *)v)->kind == kind ? &((Record *)v)->u : NULL;
    if (!PyObject_CheckBuffer(v) || PyObject_GetBuffer(v, b, PyBUF_SIMPLE) < 0) return NULL;
    if (b->len == sizes[kind]) return b->buf;
    PyBuffer_Release(b);
    b->obj = NULL;
    return NULL;
}
static void release(Py_buffer *b)
{
    if (b->obj) PyBuffer_Release(b);
}

static PyObject *instead(int k, PyObject *const *args, Py_ssize_t nargs, PyObject *kwnames)
{
    PyErr_Clear();
    return PyObject_Vectorcall(slow[k], args, nargs, kwnames);
}

static Record *record(int kind, PyObject *const *args, Py_ssize_t nargs)
{
    Record *r = PyObject_New(Record, &RecordType);
    if (!r) return NULL;
    r->kind = kind;
    memset(&r->u, 0, sizeof(r->u));
    r->keep = PyTuple_New(nargs);
    if (!r->keep) {
        Py_DECREF(r);
        return NULL;
    }
    for (Py_ssize_t i = 0; i < nargs; ++i) PyTuple_SET_ITEM(r->keep, i, Py_NewRef(args[i]));
    return r;
}

static PyObject *make_cache(PyObject *self, PyObject *const *args, Py_ssize_t nargs, PyObject *kwnames)
{
    int64_t ks[5], vs[5], ss[4];
    (void)self;
    if (kwnames || nargs < 2 || nargs > 6 || !shape_of(args[0], 5, ks) || !shape_of(args[1], 5, vs)) return instead(S_MAKE_CACHE, args, nargs, kwnames);
    const int type = type_of(args[0]);
    PyObject *const scale[2] = {nargs > 2 ? args[2] : Py_None, nargs > 3 ? args[3] : Py_None};
    int ok = (type == BF16 || type == S8) && ks[0] == vs[0] && ks[1] == vs[1] && ks[2] == vs[2] && ks[3] == vs[4] && ks[4] == vs[3] &&
             ks[0] <= INT32_MAX && ks[2] <= INT32_MAX && ks[3] <= INT32_MAX && ks[4] <= INT32_MAX;
    void *p[6] = {0};
    ok = ok && operand(args[0], type, 0, p) && operand(args[1], type, 0, p + 1);
    if (ok && nargs > 4 && args[4] != Py_None)
        ok = shape_of(args[4], 5, vs) && vs[0] == ks[0] && vs[1] == ks[1] && vs[2] == ks[2] && vs[3] == 2 && vs[4] == ks[4] && operand(args[4], BF16, 0, p + 4);
    if (ok && nargs > 5 && args[5] != Py_None)
        ok = shape_of(args[5], 4, ss) && ss[0] == ks[0] && ss[1] == ks[1] && ss[2] == ks[2] && ss[3] == ks[3] && operand(args[5], F32, 0, p + 5);
    for (int i = 0; i < 2 && ok; ++i) {
        if (type == S8)
            ok = scale[i] != Py_None && shape_of(scale[i], 4, ss) && ss[0] == ks[0] && ss[1] == ks[1] && ss[2] == ks[2] && ss[3] == ks[3] &&
                 operand(scale[i], F32, 0, p + 2 + i);
        else
            ok = scale[i] == Py_None;
    }
    if (!ok) return instead(S_MAKE_CACHE, args, nargs, kwnames);
    Record *r = record(CACHE, args, nargs);
    if (r) r->u.cache = (spmm_cache_t){p[0], p[1], p[2], p[3], type == S8 ? SPMM_CACHE_S8 : SPMM_CACHE_BF16, (int32_t)ks[0], (int32_t)ks[2],
                                       (int32_t)ks[4], (int32_t)ks[3], ks[1], p[4], p[5]};
    return (PyObject *)r;
}

static PyObject *make_batch(PyObject *self, PyObject *const *args, Py_ssize_t nargs, PyObject *kwnames)
{
    int64_t a, b, t[2];
    void *p[3];
    (void)self;
    if (kwnames || nargs != 3 || !shape_of(args[0], 1, &a) || !shape_of(args[1], 1, &b) || !shape_of(args[2], 2, t) || a != t[0] + 1 || b != t[0] ||
        !operand(args[0], S32, 0, p) || !operand(args[1], S32, 0, p + 1) || !operand(args[2], S32, 0, p + 2))
        return instead(S_MAKE_BATCH, args, nargs, kwnames);
    Record *r = record(BATCH, args, nargs);
    if (r) r->u.batch = (spmm_batch_t){t[0], p[0], p[1], p[2], t[1]};
    return (PyObject *)r;
}

static const char *const out_names[] = {"f32", "s8", "u8", "bf16"};
static const int out_values[] = {SPMM_OUT_F32, SPMM_OUT_S8, SPMM_OUT_U8, SPMM_OUT_BF16};

/* make_append(q_heads, x_type, x_scale, x_zero_point, q_weight, k_weight, eps, rope, interleaved): all nine (positions: the slow way) */
static PyObject *make_append(PyObject *self, PyObject *const *args, Py_ssize_t nargs, PyObject *kwnames)
{
    int64_t heads, zero, inter, shape[3] = {0, 0, 2};
    int type;
    float scale, eps;
    void *p[3];
    (void)self;
    if (kwnames || nargs != 9 || !number(args[0], &heads) || !name_in(args[1], out_names, out_values, 3, &type) || !real(args[2], &scale) || !number(args[3], &zero) ||
        !operand(args[4], F32, 0, p) || !operand(args[5], F32, 0, p + 1) || !real(args[6], &eps) || (args[7] != Py_None && !shape_of(args[7], 3, shape)) || shape[2] != 2 ||
        !operand(args[7], F32, 0, p + 2) || !number(args[8], &inter) || heads > INT32_MAX || heads < INT32_MIN || zero > INT32_MAX || zero < INT32_MIN || shape[1] > INT32_MAX / 2)
        return instead(S_MAKE_APPEND, args, nargs, kwnames);
    Record *r = record(APPEND, args, nargs);
    if (r) r->u.append = (spmm_append_t){(int32_t)heads, (spmm_out_t)type, scale, (int32_t)zero, p[0], p[1], eps, p[2], shape[0], (int32_t)(2 * shape[1]), inter != 0, NULL};
    return (PyObject *)r;
}

/* make_attend(q_heads, max_new, scale, causal, window, out_type, out_scale, out_zero_point), at least the first six */
static PyObject *make_attend(PyObject *self, PyObject *const *args, Py_ssize_t nargs, PyObject *kwnames)
{
    int64_t heads, most, causal, window, zero = 0;
    float scale, out_scale = 1.0f;
    int type;
    (void)self;
    if (kwnames || nargs < 6 || nargs > 8 || !number(args[0], &heads) || !number(args[1], &most) || !real(args[2], &scale) || !number(args[3], &causal) ||
        !number(args[4], &window) || !name_in(args[5], out_names, out_values, 4, &type) || (nargs > 6 && !real(args[6], &out_scale)) ||
        (nargs > 7 && !number(args[7], &zero)) || heads > INT32_MAX || heads < INT32_MIN || window > INT32_MAX || window < INT32_MIN || zero > INT32_MAX || zero < INT32_MIN)
        return instead(S_MAKE_ATTEND, args, nargs, kwnames);
    Record *r = record(ATTEND, args, nargs);
    if (r) r->u.attend = (spmm_attend_t){(int32_t)heads, most, scale, causal != 0, (int32_t)window, type, out_scale, (int32_t)zero};
    return (PyObject *)r;
}

static PyObject *done(int status, const char *name)
{
    if (status != SPMM_OK) return PyObject_CallFunction(py_check, "is", status, name);      /* raises SpmmError */
    Py_RETURN_NONE;
}

/* bytes from one row's first element to the last row's last one */
static int64_t covered(__int128 rows, int64_t cols, int64_t ld, int64_t each)
{
    if (rows < 1 || cols < 1 || ld < 0) return 0;        /* (the library refuses it) */
    const __int128 n = ((rows - 1) * ld + cols) * each;
    return n > INT64_MAX ? INT64_MAX : (int64_t)n;
}

/* spmm_cache_append(cache, layer, batch, x, T, ldx, how, q, stream) */
static PyObject *cache_append(PyObject *self, PyObject *const *args, Py_ssize_t nargs, PyObject *kwnames)
{
    Py_buffer cb = {0}, bb = {0};
    int64_t layer, T, ldx, stream = 0;
    void *x, *q, *ignored;
    (void)self;
    if (kwnames || nargs < 8 || nargs > 9 || !functions[F_APPEND] || Py_TYPE(args[6]) != &RecordType || ((Record *)args[6])->kind != APPEND) return instead(S_APPEND, args, nargs, kwnames);
    const Record *const how = (Record *)args[6];
    const spmm_cache_t *const c = description(args[0], CACHE, &cb);
    const spmm_batch_t *const b = c ? description(args[2], BATCH, &bb) : NULL;
    int ok = c && b && number(args[1], &layer) && layer >= INT32_MIN && layer <= INT32_MAX && number(args[4], &T) && number(args[5], &ldx) &&
             (nargs < 9 || args[8] == Py_None || number(args[8], &stream));
    if (ok) {
        const spmm_append_t *const a = &how->u.append;
        const __int128 rows = ((__int128)a->q_heads + 2 * (__int128)c->n_heads) * c->head_dim;
        ok = operand(args[3], a->x_type == SPMM_OUT_F32 ? F32 : a->x_type == SPMM_OUT_S8 ? S8 : U8, covered(rows, T, ldx, a->x_type == SPMM_OUT_F32 ? 4 : 1), &x) &&
             operand(args[7], BF16, covered(1, T, 0, 2 * (int64_t)a->q_heads * c->head_dim), &q);
        for (int i = 4; i < 6 && ok; ++i) ok = operand(PyTuple_GET_ITEM(how->keep, i), F32, 4 * (int64_t)c->head_dim, &ignored);
    }
    int st = 0;
    if (ok) {
        Py_BEGIN_ALLOW_THREADS
        st = ((spmm_status_t (*)(const spmm_cache_t *, int32_t, const spmm_batch_t *, const void *, int64_t, int64_t, const spmm_append_t *, void *, void *))functions[F_APPEND])(
            c, (int32_t)layer, b, x, T, ldx, &how->u.append, q, (void *)(uintptr_t)stream);
        Py_END_ALLOW_THREADS
    }
    release(&cb);
    release(&bb);
    return ok ? done(st, "spmm_cache_append") : instead(S_APPEND, args, nargs, kwnames);
}

typedef spmm_status_t (*work_fn)(const spmm_cache_t *, int64_t, int64_t, const spmm_attend_t *, int64_t *);

/* spmm_attend_work_bytes(cache, n_seqs, T, how) */
static PyObject *attend_work(PyObject *self, PyObject *const *args, Py_ssize_t nargs, PyObject *kwnames)
{
    Py_buffer cb = {0}, hb = {0};
    int64_t n, T, bytes = 0;
    (void)self;
    if (kwnames || nargs != 4 || !functions[F_ATTEND_WORK] || !number(args[1], &n) || !number(args[2], &T)) return instead(S_ATTEND_WORK, args, nargs, kwnames);
    const spmm_cache_t *const c = description(args[0], CACHE, &cb);
    const spmm_attend_t *const a = c ? description(args[3], ATTEND, &hb) : NULL;
    const int st = a ? (int)((work_fn)functions[F_ATTEND_WORK])(c, n, T, a, &bytes) : -1;
    release(&cb);
    release(&hb);
    return st == SPMM_OK ? PyLong_FromLongLong(bytes) : instead(S_ATTEND_WORK, args, nargs, kwnames);
}

/* spmm_cache_attend(cache, layer, batch, q, T, how, out, ldo, work, stream) */
static PyObject *cache_attend(PyObject *self, PyObject *const *args, Py_ssize_t nargs, PyObject *kwnames)
{
    Py_buffer cb = {0}, bb = {0}, hb = {0};
    int64_t layer, T, ldo, stream = 0, need = 0;
    void *q, *out, *work;
    (void)self;
    if (kwnames || nargs < 9 || nargs > 10 || !functions[F_ATTEND]) return instead(S_ATTEND, args, nargs, kwnames);
    const spmm_cache_t *const c = description(args[0], CACHE, &cb);
    const spmm_batch_t *const b = c ? description(args[2], BATCH, &bb) : NULL;
    const spmm_attend_t *const a = b ? description(args[5], ATTEND, &hb) : NULL;
    int ok = a && number(args[1], &layer) && layer >= INT32_MIN && layer <= INT32_MAX && number(args[4], &T) && number(args[7], &ldo) &&
             (nargs < 10 || args[9] == Py_None || number(args[9], &stream));
    if (ok) {
        static const int of[] = {-1, F32, S8, U8, BF16};
        const int known = a->out_type >= 1 && a->out_type <= 4;
        const int64_t each = a->out_type == SPMM_OUT_F32 ? 4 : a->out_type == SPMM_OUT_BF16 ? 2 : 1;
        const __int128 rows = (__int128)a->q_heads * c->head_dim;
        ok = known && ((work_fn)functions[F_ATTEND_WORK])(c, b->n_seqs, T, a, &need) == SPMM_OK &&
             operand(args[3], BF16, covered(1, T, 0, 2 * (int64_t)a->q_heads * c->head_dim), &q) && operand(args[6], of[known ? a->out_type : 0], covered(rows, T, ldo, each), &out) &&
             operand(args[8], -1, need, &work);
    }
    int st = 0;
    if (ok) {
        Py_BEGIN_ALLOW_THREADS
        st = ((spmm_status_t (*)(const spmm_cache_t *, int32_t, const spmm_batch_t *, const void *, int64_t, const spmm_attend_t *, void *, int64_t, void *, void *))functions[F_ATTEND])(
            c, (int32_t)layer, b, q, T, a, out, ldo, work, (void *)(uintptr_t)stream);
        Py_END_ALLOW_THREADS
    }
    release(&cb);
    release(&bb);
    release(&hb);
    return ok ? done(st, "spmm_cache_attend") : instead(S_ATTEND, args, nargs, kwnames);
}

/* spmm_cache_work_bytes(cache, n_rows) */
static PyObject *cache_work(PyObject *self, PyObject *const *args, Py_ssize_t nargs, PyObject *kwnames)
{
    Py_buffer cb = {0};
    int64_t n, bytes = 0;
    (void)self;
    if (kwnames || nargs != 2 || !functions[F_CACHE_WORK] || !number(args[1], &n)) return instead(S_CACHE_WORK, args, nargs, kwnames);
    const spmm_cache_t *const c = description(args[0], CACHE, &cb);
    const int st = c ? (int)((spmm_status_t (*)(const spmm_cache_t *, int64_t, int64_t *))functions[F_CACHE_WORK])(c, n, &bytes) : -1;
    release(&cb);
    return st == SPMM_OK ? PyLong_FromLongLong(bytes) : instead(S_CACHE_WORK, args, nargs, kwnames);
}

/* a [rows][width] int32 tensor */
static int table_of(PyObject *t, int64_t shape[2], void **p) { return shape_of(t, 2, shape) && operand(t, S32, 0, p); }
static int row_of(PyObject *t, int64_t n, void **p)
{
    int64_t m;
    return shape_of(t, 1, &m) && m == n && operand(t, S32, 0, p);
}
static int64_t page_work(const spmm_cache_t *c, int64_t rows)
{
    int64_t bytes = 0;
    return ((spmm_status_t (*)(const spmm_cache_t *, int64_t, int64_t *))functions[F_CACHE_WORK])(c, rows, &bytes) == SPMM_OK ? bytes : -1;
}

/* spmm_cache_fork(cache, table, kv_len, parent, keep, want, table_out, kv_len_out, info, work, stream) */
static PyObject *cache_fork(PyObject *self, PyObject *const *args, Py_ssize_t nargs, PyObject *kwnames)
{
    Py_buffer cb = {0};
    int64_t in[2], out[2], need, stream = 0;
    void *p[9];
    (void)self;
    if (kwnames || nargs < 10 || nargs > 11 || !functions[F_FORK]) return instead(S_FORK, args, nargs, kwnames);
    const spmm_cache_t *const c = description(args[0], CACHE, &cb);
    const int ok = c && table_of(args[1], in, p) && table_of(args[6], out, p + 5) && in[1] == out[1] && row_of(args[2], in[0], p + 1) && row_of(args[3], out[0], p + 2) &&
                   row_of(args[4], out[0], p + 3) && row_of(args[5], out[0], p + 4) && row_of(args[7], out[0], p + 6) && operand(args[8], S32, 16, p + 7) &&
                   (need = page_work(c, out[0])) >= 0 && operand(args[9], -1, need, p + 8) && (nargs < 11 || args[10] == Py_None || number(args[10], &stream));
    int st = 0;
    if (ok) {
        Py_BEGIN_ALLOW_THREADS
        st = ((spmm_status_t (*)(const spmm_cache_t *, const int32_t *, int64_t, const int32_t *, int64_t, const int32_t *, const int32_t *, const int32_t *, int64_t, int32_t *, int32_t *,
                                 int32_t *, void *, void *))functions[F_FORK])(c, p[0], in[1], p[1], in[0], p[2], p[3], p[4], out[0], p[5], p[6], p[7], p[8], (void *)(uintptr_t)stream);
        Py_END_ALLOW_THREADS
    }
    release(&cb);
    return ok ? done(st, "spmm_cache_fork") : instead(S_FORK, args, nargs, kwnames);
}

/* spmm_cache_compact(cache, table, table_out, info, work, stream) */
static PyObject *cache_compact(PyObject *self, PyObject *const *args, Py_ssize_t nargs, PyObject *kwnames)
{
    Py_buffer cb = {0};
    int64_t in[2], out[2], need, stream = 0;
    void *p[4];
    (void)self;
    if (kwnames || nargs < 5 || nargs > 6 || !functions[F_COMPACT]) return instead(S_COMPACT, args, nargs, kwnames);
    const spmm_cache_t *const c = description(args[0], CACHE, &cb);
    const int ok = c && table_of(args[1], in, p) && table_of(args[2], out, p + 1) && in[0] == out[0] && in[1] == out[1] && operand(args[3], S32, 16, p + 2) &&
                   (need = page_work(c, in[0])) >= 0 && operand(args[4], -1, need, p + 3) && (nargs < 6 || args[5] == Py_None || number(args[5], &stream));
    int st = 0;
    if (ok) {
        Py_BEGIN_ALLOW_THREADS
        st = ((spmm_status_t (*)(const spmm_cache_t *, const int32_t *, int64_t, int64_t, int32_t *, int32_t *, void *, void *))functions[F_COMPACT])(
            c, p[0], in[1], in[0], p[1], p[2], p[3], (void *)(uintptr_t)stream);
        Py_END_ALLOW_THREADS
    }
    release(&cb);
    return ok ? done(st, "spmm_cache_compact") : instead(S_COMPACT, args, nargs, kwnames);
}

static int narrow(PyObject *v, int64_t *out) { return number(v, out) && *out >= INT32_MIN && *out <= INT32_MAX; }
static int narrow_all(PyObject *const *args, int n, int64_t *out)
{
    for (int i = 0; i < n; ++i)
        if (!narrow(args[i], out + i)) return 0;
    return 1;
}
static int stream_of(PyObject *const *args, Py_ssize_t nargs, Py_ssize_t at, int64_t *out)
{
    *out = 0;
    return nargs <= at || args[at] == Py_None || number(args[at], out);
}

/* make_select(q_heads, pages, first, last, causal, window): all six */
static PyObject *make_select(PyObject *self, PyObject *const *args, Py_ssize_t nargs, PyObject *kwnames)
{
    int64_t v[6];
    (void)self;
    if (kwnames || nargs != 6 || !narrow_all(args, 6, v)) return instead(S_MAKE_SELECT, args, nargs, kwnames);
    Record *r = record(SELECT, args, nargs);
    if (r) r->u.select = (spmm_select_t){(int32_t)v[0], (int32_t)v[1], (int32_t)v[2], (int32_t)v[3], v[4] != 0, (int32_t)v[5]};
    return (PyObject *)r;
}

/* make_weigh(q_heads, max_new, scale, causal, window, decay): all six */
static PyObject *make_weigh(PyObject *self, PyObject *const *args, Py_ssize_t nargs, PyObject *kwnames)
{
    int64_t heads, most, causal, window;
    float scale, decay;
    (void)self;
    if (kwnames || nargs != 6 || !narrow(args[0], &heads) || !number(args[1], &most) || !real(args[2], &scale) || !number(args[3], &causal) || !narrow(args[4], &window) ||
        !real(args[5], &decay))
        return instead(S_MAKE_WEIGH, args, nargs, kwnames);
    Record *r = record(WEIGH, args, nargs);
    if (r) r->u.weigh = (spmm_weigh_t){(int32_t)heads, most, scale, causal != 0, (int32_t)window, decay};
    return (PyObject *)r;
}

/* make_evict(first, recent, most) */
static PyObject *make_evict(PyObject *self, PyObject *const *args, Py_ssize_t nargs, PyObject *kwnames)
{
    int64_t v[2], most;
    (void)self;
    if (kwnames || nargs != 3 || !narrow_all(args, 2, v) || !number(args[2], &most)) return instead(S_MAKE_EVICT, args, nargs, kwnames);
    Record *r = record(EVICT, args, nargs);
    if (r) r->u.evict = (spmm_evict_t){(int32_t)v[0], (int32_t)v[1], most};
    return (PyObject *)r;
}

/* spmm_cache_bounds(cache, layer, batch, T, stream) */
static PyObject *cache_bounds(PyObject *self, PyObject *const *args, Py_ssize_t nargs, PyObject *kwnames)
{
    Py_buffer cb = {0}, bb = {0};
    int64_t layer, T, stream;
    (void)self;
    if (kwnames || nargs < 4 || nargs > 5 || !functions[F_BOUNDS] || !narrow(args[1], &layer) || !number(args[3], &T) || !stream_of(args, nargs, 4, &stream))
        return instead(S_BOUNDS, args, nargs, kwnames);
    const spmm_cache_t *const c = description(args[0], CACHE, &cb);
    const spmm_batch_t *const b = c ? description(args[2], BATCH, &bb) : NULL;
    int st = 0;
    if (b) {
        Py_BEGIN_ALLOW_THREADS
        st = ((spmm_status_t (*)(const spmm_cache_t *, int32_t, const spmm_batch_t *, int64_t, void *))functions[F_BOUNDS])(c, (int32_t)layer, b, T, (void *)(uintptr_t)stream);
        Py_END_ALLOW_THREADS
    }
    const int ok = b != NULL;
    release(&cb);
    release(&bb);
    return ok ? done(st, "spmm_cache_bounds") : instead(S_BOUNDS, args, nargs, kwnames);
}

/* spmm_cache_score(cache, layer, batch, q, T, how, scores, lds, stream) */
static PyObject *cache_score(PyObject *self, PyObject *const *args, Py_ssize_t nargs, PyObject *kwnames)
{
    Py_buffer cb = {0}, bb = {0}, hb = {0};
    int64_t layer, T, lds, stream;
    void *q, *scores;
    (void)self;
    if (kwnames || nargs < 8 || nargs > 9 || !functions[F_SCORE] || !narrow(args[1], &layer) || !number(args[4], &T) || !number(args[7], &lds) || !stream_of(args, nargs, 8, &stream))
        return instead(S_SCORE, args, nargs, kwnames);
    const spmm_cache_t *const c = description(args[0], CACHE, &cb);
    const spmm_batch_t *const b = c ? description(args[2], BATCH, &bb) : NULL;
    const spmm_select_t *const a = b ? description(args[5], SELECT, &hb) : NULL;
    const int ok = a && operand(args[3], BF16, covered(T, (int64_t)a->q_heads * c->head_dim, (int64_t)a->q_heads * c->head_dim, 2), &q) &&
                   operand(args[6], F32, covered((__int128)T * c->n_heads, lds, lds, 4), &scores);
    int st = 0;
    if (ok) {
        Py_BEGIN_ALLOW_THREADS
        st = ((spmm_status_t (*)(const spmm_cache_t *, int32_t, const spmm_batch_t *, const void *, int64_t, const spmm_select_t *, void *, int64_t, void *))functions[F_SCORE])(
            c, (int32_t)layer, b, q, T, a, scores, lds, (void *)(uintptr_t)stream);
        Py_END_ALLOW_THREADS
    }
    release(&cb);
    release(&bb);
    release(&hb);
    return ok ? done(st, "spmm_cache_score") : instead(S_SCORE, args, nargs, kwnames);
}

/* spmm_cache_select(cache, batch, scores, T, lds, how, lists, stream) */
static PyObject *cache_select(PyObject *self, PyObject *const *args, Py_ssize_t nargs, PyObject *kwnames)
{
    Py_buffer cb = {0}, bb = {0}, hb = {0};
    int64_t T, lds, stream;
    void *scores, *lists;
    (void)self;
    if (kwnames || nargs < 7 || nargs > 8 || !functions[F_SELECT] || !number(args[3], &T) || !number(args[4], &lds) || !stream_of(args, nargs, 7, &stream))
        return instead(S_SELECT, args, nargs, kwnames);
    const spmm_cache_t *const c = description(args[0], CACHE, &cb);
    const spmm_batch_t *const b = c ? description(args[1], BATCH, &bb) : NULL;
    const spmm_select_t *const a = b ? description(args[5], SELECT, &hb) : NULL;
    const int ok = a && operand(args[2], F32, covered((__int128)T * c->n_heads, lds, lds, 4), &scores) &&
                   operand(args[6], S32, covered((__int128)T * c->n_heads, a->pages, a->pages, 4), &lists);
    int st = 0;
    if (ok) {
        Py_BEGIN_ALLOW_THREADS
        st = ((spmm_status_t (*)(const spmm_cache_t *, const spmm_batch_t *, const void *, int64_t, int64_t, const spmm_select_t *, void *, void *))functions[F_SELECT])(
            c, b, scores, T, lds, a, lists, (void *)(uintptr_t)stream);
        Py_END_ALLOW_THREADS
    }
    release(&cb);
    release(&bb);
    release(&hb);
    return ok ? done(st, "spmm_cache_select") : instead(S_SELECT, args, nargs, kwnames);
}

typedef spmm_status_t (*selected_work_fn)(const spmm_cache_t *, int64_t, const spmm_attend_t *, int64_t, int64_t *);

/* spmm_selected_work_bytes(cache, T, how, pages) */
static PyObject *selected_work(PyObject *self, PyObject *const *args, Py_ssize_t nargs, PyObject *kwnames)
{
    Py_buffer cb = {0}, hb = {0};
    int64_t T, pages, bytes = 0;
    (void)self;
    if (kwnames || nargs != 4 || !functions[F_SELECTED_WORK] || !number(args[1], &T) || !number(args[3], &pages)) return instead(S_SELECTED_WORK, args, nargs, kwnames);
    const spmm_cache_t *const c = description(args[0], CACHE, &cb);
    const spmm_attend_t *const a = c ? description(args[2], ATTEND, &hb) : NULL;
    const int st = a ? (int)((selected_work_fn)functions[F_SELECTED_WORK])(c, T, a, pages, &bytes) : -1;
    release(&cb);
    release(&hb);
    return st == SPMM_OK ? PyLong_FromLongLong(bytes) : instead(S_SELECTED_WORK, args, nargs, kwnames);
}

/* spmm_cache_attend_selected(cache, layer, batch, q, T, how, lists, pages, out, ldo, work, stream) */
static PyObject *cache_selected(PyObject *self, PyObject *const *args, Py_ssize_t nargs, PyObject *kwnames)
{
    Py_buffer cb = {0}, bb = {0}, hb = {0};
    int64_t layer, T, pages, ldo, stream, need = 0;
    void *q, *lists, *out, *work;
    (void)self;
    if (kwnames || nargs < 11 || nargs > 12 || !functions[F_SELECTED] || !narrow(args[1], &layer) || !number(args[4], &T) || !number(args[7], &pages) || !number(args[9], &ldo) ||
        !stream_of(args, nargs, 11, &stream))
        return instead(S_SELECTED, args, nargs, kwnames);
    const spmm_cache_t *const c = description(args[0], CACHE, &cb);
    const spmm_batch_t *const b = c ? description(args[2], BATCH, &bb) : NULL;
    const spmm_attend_t *const a = b ? description(args[5], ATTEND, &hb) : NULL;
    int ok = a != NULL;
    if (ok) {
        static const int of[] = {-1, F32, S8, U8, BF16};
        const int known = a->out_type >= 1 && a->out_type <= 4;
        const int64_t each = a->out_type == SPMM_OUT_F32 ? 4 : a->out_type == SPMM_OUT_BF16 ? 2 : 1, values = (int64_t)a->q_heads * c->head_dim;
        ok = known && ((selected_work_fn)functions[F_SELECTED_WORK])(c, T, a, pages, &need) == SPMM_OK && operand(args[3], BF16, covered(T, values, values, 2), &q) &&
             operand(args[6], S32, covered((__int128)T * c->n_heads, pages, pages, 4), &lists) && operand(args[8], of[known ? a->out_type : 0], covered(values, T, ldo, each), &out) &&
             operand(args[10], -1, need, &work);
    }
    int st = 0;
    if (ok) {
        Py_BEGIN_ALLOW_THREADS
        st = ((spmm_status_t (*)(const spmm_cache_t *, int32_t, const spmm_batch_t *, const void *, int64_t, const spmm_attend_t *, const void *, int64_t, void *, int64_t, void *,
                                 void *))functions[F_SELECTED])(c, (int32_t)layer, b, q, T, a, lists, pages, out, ldo, work, (void *)(uintptr_t)stream);
        Py_END_ALLOW_THREADS
    }
    release(&cb);
    release(&bb);
    release(&hb);
    return ok ? done(st, "spmm_cache_attend_selected") : instead(S_SELECTED, args, nargs, kwnames);
}

typedef spmm_status_t (*weigh_work_fn)(const spmm_cache_t *, const spmm_batch_t *, int64_t, const spmm_weigh_t *, int64_t *);

/* spmm_weigh_work_bytes(cache, batch, T, how) */
static PyObject *weigh_work(PyObject *self, PyObject *const *args, Py_ssize_t nargs, PyObject *kwnames)
{
    Py_buffer cb = {0}, bb = {0}, hb = {0};
    int64_t T, bytes = 0;
    (void)self;
    if (kwnames || nargs != 4 || !functions[F_WEIGH_WORK] || !number(args[2], &T)) return instead(S_WEIGH_WORK, args, nargs, kwnames);
    const spmm_cache_t *const c = description(args[0], CACHE, &cb);
    const spmm_batch_t *const b = c ? description(args[1], BATCH, &bb) : NULL;
    const spmm_weigh_t *const a = b ? description(args[3], WEIGH, &hb) : NULL;
    const int st = a ? (int)((weigh_work_fn)functions[F_WEIGH_WORK])(c, b, T, a, &bytes) : -1;
    release(&cb);
    release(&bb);
    release(&hb);
    return st == SPMM_OK ? PyLong_FromLongLong(bytes) : instead(S_WEIGH_WORK, args, nargs, kwnames);
}

/* spmm_cache_weigh(cache, layer, batch, q, T, how, work, stream) */
static PyObject *cache_weigh(PyObject *self, PyObject *const *args, Py_ssize_t nargs, PyObject *kwnames)
{
    Py_buffer cb = {0}, bb = {0}, hb = {0};
    int64_t layer, T, stream, need = 0;
    void *q, *work;
    (void)self;
    if (kwnames || nargs < 7 || nargs > 8 || !functions[F_WEIGH] || !narrow(args[1], &layer) || !number(args[4], &T) || !stream_of(args, nargs, 7, &stream))
        return instead(S_WEIGH, args, nargs, kwnames);
    const spmm_cache_t *const c = description(args[0], CACHE, &cb);
    const spmm_batch_t *const b = c ? description(args[2], BATCH, &bb) : NULL;
    const spmm_weigh_t *const a = b ? description(args[5], WEIGH, &hb) : NULL;
    const int ok = a && ((weigh_work_fn)functions[F_WEIGH_WORK])(c, b, T, a, &need) == SPMM_OK &&
                   operand(args[3], BF16, covered(T, (int64_t)a->q_heads * c->head_dim, (int64_t)a->q_heads * c->head_dim, 2), &q) && operand(args[6], -1, need, &work);
    int st = 0;
    if (ok) {
        Py_BEGIN_ALLOW_THREADS
        st = ((spmm_status_t (*)(const spmm_cache_t *, int32_t, const spmm_batch_t *, const void *, int64_t, const spmm_weigh_t *, void *, void *))functions[F_WEIGH])(
            c, (int32_t)layer, b, q, T, a, work, (void *)(uintptr_t)stream);
        Py_END_ALLOW_THREADS
    }
    release(&cb);
    release(&bb);
    release(&hb);
    return ok ? done(st, "spmm_cache_weigh") : instead(S_WEIGH, args, nargs, kwnames);
}

/* spmm_cache_evict(cache, table, kv_len, keep, how, table_to, kv_len_out, kept, stream) */
static PyObject *cache_evict(PyObject *self, PyObject *const *args, Py_ssize_t nargs, PyObject *kwnames)
{
    Py_buffer cb = {0}, hb = {0};
    int64_t in[2], to[2], stream;
    void *p[6];
    (void)self;
    if (kwnames || nargs < 8 || nargs > 9 || !functions[F_EVICT] || !stream_of(args, nargs, 8, &stream)) return instead(S_EVICT, args, nargs, kwnames);
    const spmm_cache_t *const c = description(args[0], CACHE, &cb);
    const spmm_evict_t *const a = c ? description(args[4], EVICT, &hb) : NULL;
    const int ok = a && table_of(args[1], in, p) && table_of(args[5], to, p + 3) && in[0] == to[0] && in[1] == to[1] && row_of(args[2], in[0], p + 1) && row_of(args[3], in[0], p + 2) &&
                   row_of(args[6], in[0], p + 4) && a->most >= 0 && operand(args[7], S32, covered((__int128)c->n_layers * c->n_heads * in[0], a->most, a->most, 4), p + 5);
    int st = 0;
    if (ok) {
        Py_BEGIN_ALLOW_THREADS
        st = ((spmm_status_t (*)(const spmm_cache_t *, const void *, int64_t, const void *, int64_t, const void *, const spmm_evict_t *, const void *, void *, void *, void *))functions[F_EVICT])(
            c, p[0], in[1], p[1], in[0], p[2], a, p[3], p[4], p[5], (void *)(uintptr_t)stream);
        Py_END_ALLOW_THREADS
    }
    release(&cb);
    release(&hb);
    return ok ? done(st, "spmm_cache_evict") : instead(S_EVICT, args, nargs, kwnames);
}

/* hooks(_check, the slow functions) */
static PyObject *native_hooks(PyObject *self, PyObject *args)
{
    (void)self;
    if (PyTuple_GET_SIZE(args) != 1 + SLOW) return PyErr_Format(PyExc_TypeError, "hooks() takes %d functions", 1 + SLOW);
    Py_XSETREF(py_check, Py_NewRef(PyTuple_GET_ITEM(args, 0)));
    for (int i = 0; i < SLOW; ++i) Py_XSETREF(slow[i], Py_NewRef(PyTuple_GET_ITEM(args, 1 + i)));
    Py_RETURN_NONE;
}

/* bind(addresses of the functions) */
static PyObject *native_bind(PyObject *self, PyObject *args)
{
    (void)self;
    if (PyTuple_GET_SIZE(args) != FUNCTIONS) return PyErr_Format(PyExc_TypeError, "bind() takes %d addresses", FUNCTIONS);
    for (int i = 0; i < FUNCTIONS; ++i) {
        const unsigned long long p = PyLong_AsUnsignedLongLong(PyTuple_GET_ITEM(args, i));
        if (PyErr_Occurred()) return NULL;
        functions[i] = (void *)(uintptr_t)p;
    }
    Py_RETURN_NONE;
}

#define FAST(name, f) {name, (PyCFunction)(void (*)(void))f, METH_FASTCALL | METH_KEYWORDS, "See cache_binding.py."}
static PyMethodDef methods[] = {
    FAST("make_cache", make_cache), FAST("make_batch", make_batch), FAST("make_append", make_append), FAST("make_attend", make_attend),
    FAST("spmm_cache_append", cache_append), FAST("spmm_cache_attend", cache_attend), FAST("spmm_attend_work_bytes", attend_work),
    FAST("spmm_cache_fork", cache_fork), FAST("spmm_cache_compact", cache_compact), FAST("spmm_cache_work_bytes", cache_work),
    FAST("make_select", make_select), FAST("make_weigh", make_weigh), FAST("make_evict", make_evict), FAST("spmm_cache_bounds", cache_bounds),
    FAST("spmm_cache_score", cache_score), FAST("spmm_cache_select", cache_select), FAST("spmm_selected_work_bytes", selected_work),
    FAST("spmm_cache_attend_selected", cache_selected), FAST("spmm_weigh_work_bytes", weigh_work), FAST("spmm_cache_weigh", cache_weigh),
    FAST("spmm_cache_evict", cache_evict),
    {"hooks", native_hooks, METH_VARARGS, NULL}, {"bind", native_bind, METH_VARARGS, NULL}, {NULL, NULL, 0, NULL}};
static struct PyModuleDef module = {PyModuleDef_HEAD_INIT, "_native_cache", NULL, -1, methods, NULL, NULL, NULL, NULL};

PyMODINIT_FUNC PyInit__native_cache(void)
{
    if (PyType_Ready(&RecordType) < 0) return NULL;
    s_data_ptr = PyUnicode_InternFromString("data_ptr");
    s_nbytes = PyUnicode_InternFromString("nbytes");
    s_is_contiguous = PyUnicode_InternFromString("is_contiguous");
    s_dtype = PyUnicode_InternFromString("dtype");
    s_is_cuda = PyUnicode_InternFromString("is_cuda");
    s_shape = PyUnicode_InternFromString("shape");
    if (!s_data_ptr || !s_nbytes || !s_is_contiguous || !s_dtype || !s_is_cuda || !s_shape) return NULL;
    return PyModule_Create(&module);
}
