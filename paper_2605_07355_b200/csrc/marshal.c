/* Argument marshalling of the Python binding in C: the entry points of include/ttf.h that a program calls per clip or
 * per batch.  A call through ctypes converts its 12 to 17 arguments one by one in about 4 us, which is more than the
 * driver takes to launch a kernel; here it is about 0.3 us.  No CUDA and no torch headers: pointers and streams arrive as integers
 * (0 = NULL), or tensors are asked for their attributes as Python would; the addresses of the library's functions are handed
 * in once by bind().  The GIL is released around every
 * call. */
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include "ttf.h"

#define NFN 14
static struct {
    int (*compress)(const void*, int, int, int, int, int, float, int, void*, int*, int*, ttf_stream_t);
    int (*compress_ws)(const void*, int, int, int, int, int, float, int, void*, int*, int*, void*, size_t, ttf_stream_t);
    int (*compress_ex)(const void*, int, int, int, int, int, float, int, const ttf_options*, void*, int*, int*, ttf_stream_t);
    int (*compress_segment)(const void*, int, int, int, int, int, float, int, int, void*, int*, int*, ttf_stream_t);
    int (*compress_batch)(const void* const*, int, int, int, int, int, int, float, int, void* const*, int* const*,
                          int* const*, ttf_stream_t);
    int (*compress_batch_ex)(const void* const*, int, int, int, int, int, int, float, int, const ttf_options*, void* const*,
                             int* const*, int* const*, ttf_stream_t);
    int (*query)(const void*, int, int, int, int, int, float, int, int*, unsigned char*, int*, float*, int*, ttf_stream_t);
    int (*query_ws)(const void*, int, int, int, int, int, float, int, int*, unsigned char*, int*, float*, int*, void*, size_t,
                    ttf_stream_t);
    int (*query_ex)(const void*, int, int, int, int, int, float, int, const ttf_options*, int*, unsigned char*, int*, float*,
                    int*, ttf_stream_t);
    int (*restore)(const void*, size_t, int, int, int, const int*, const unsigned char*, const int*, void*, int*,
                   ttf_stream_t);
    int (*stats)(const float*, const unsigned char*, const int*, int, int, int, float, float, long long*, ttf_stream_t);
    int (*rotate)(const ttf_heads*, const ttf_heads*, int, int, int, const int*, const int*, const ttf_rotation*,
                  const ttf_heads*, const ttf_heads*, ttf_stream_t);
    int (*cache_append)(const ttf_heads*, const ttf_heads*, const ttf_heads*, const int*, const ttf_rotation*,
                        const ttf_sequences*, const ttf_cache*, const ttf_heads*, ttf_stream_t);
    int (*attend)(const ttf_heads*, const ttf_sequences*, const ttf_cache*, float, int, int, const ttf_heads*, ttf_stream_t);
} fn;

/* the arguments of one call, taken in order; the first conversion that fails leaves a Python error set */
typedef struct { PyObject* const* a; Py_ssize_t n, at; int bad; } Args;

static PyObject* next_arg(Args* s) {
    if (s->bad) return NULL;
    if (s->at >= s->n) { s->bad = 1; PyErr_SetString(PyExc_TypeError, "too few arguments"); return NULL; }
    return s->a[s->at++];
}
static void* ptr(Args* s) {
    PyObject* o = next_arg(s);
    if (!o) return NULL;
    void* p = PyLong_AsVoidPtr(o);
    if (!p && PyErr_Occurred()) s->bad = 1;
    return p;
}
static int num(Args* s) {
    PyObject* o = next_arg(s);
    if (!o) return 0;
    long v = PyLong_AsLong(o);
    if (v == -1 && PyErr_Occurred()) s->bad = 1;
    else if (v != (int)v) { s->bad = 1; PyErr_SetString(PyExc_OverflowError, "argument does not fit an int"); }
    return (int)v;
}
static size_t size(Args* s) {
    PyObject* o = next_arg(s);
    if (!o) return 0;
    size_t v = PyLong_AsSize_t(o);
    if (v == (size_t)-1 && PyErr_Occurred()) s->bad = 1;
    return v;
}
static long long wide(Args* s) {
    PyObject* o = next_arg(s);
    if (!o) return 0;
    long long v = PyLong_AsLongLong(o);
    if (v == -1 && PyErr_Occurred()) s->bad = 1;
    return v;
}
static float real(Args* s) {
    PyObject* o = next_arg(s);
    if (!o) return 0.f;
    double v = PyFloat_AsDouble(o);
    if (v == -1.0 && PyErr_Occurred()) s->bad = 1;
    return (float)v;
}
static int done(Args* s) {
    if (!s->bad && s->at != s->n) { s->bad = 1; PyErr_SetString(PyExc_TypeError, "too many arguments"); }
    return !s->bad;
}

/* the leading arguments that most entry points share */
typedef struct { const void* x; int F, H, W, C, r, dtype; float t; } Clip;
static Clip clip(Args* s) {
    Clip c;
    c.x = ptr(s); c.F = num(s); c.H = num(s); c.W = num(s); c.C = num(s); c.r = num(s); c.t = real(s); c.dtype = num(s);
    return c;
}
static ttf_options options(Args* s) {
    ttf_options o;
    o.anchor_mode = num(s); o.anchor_frame = num(s); o.order = num(s); o.pos_base = num(s);
    return o;
}
static int plain(const ttf_options* o) { return !(o->anchor_mode || o->anchor_frame || o->order || o->pos_base); }

#define CALL(expr)                      \
    if (!done(&s)) return NULL;         \
    int rc;                             \
    Py_BEGIN_ALLOW_THREADS rc = (expr); \
    Py_END_ALLOW_THREADS return PyLong_FromLong(rc)

static PyObject* m_bind(PyObject* self, PyObject* const* a, Py_ssize_t n) {
    if (n != NFN) { PyErr_SetString(PyExc_TypeError, "bind() takes the address of every function"); return NULL; }
    void* p[NFN];
    for (int i = 0; i < NFN; ++i) {
        p[i] = PyLong_AsVoidPtr(a[i]);
        if (!p[i]) { if (!PyErr_Occurred()) PyErr_SetString(PyExc_ValueError, "NULL function"); return NULL; }
    }
    *(void**)&fn.compress = p[0]; *(void**)&fn.compress_ws = p[1]; *(void**)&fn.compress_ex = p[2];
    *(void**)&fn.compress_segment = p[3]; *(void**)&fn.compress_batch = p[4]; *(void**)&fn.compress_batch_ex = p[5];
    *(void**)&fn.query = p[6]; *(void**)&fn.query_ws = p[7]; *(void**)&fn.query_ex = p[8];
    *(void**)&fn.restore = p[9]; *(void**)&fn.stats = p[10];
    *(void**)&fn.rotate = p[11]; *(void**)&fn.cache_append = p[12]; *(void**)&fn.attend = p[13];
    Py_RETURN_NONE;
}

/* clip, 4 options, tokens, count, positions, stream */
static PyObject* m_compress(PyObject* self, PyObject* const* a, Py_ssize_t n) {
    Args s = {a, n, 0, 0};
    Clip c = clip(&s);
    ttf_options o = options(&s);
    void* tok = ptr(&s); int* cnt = ptr(&s); int* pos = ptr(&s); ttf_stream_t st = ptr(&s);
    CALL(plain(&o) ? fn.compress(c.x, c.F, c.H, c.W, c.C, c.r, c.t, c.dtype, tok, cnt, pos, st)
                   : fn.compress_ex(c.x, c.F, c.H, c.W, c.C, c.r, c.t, c.dtype, &o, tok, cnt, pos, st));
}
/* clip, tokens, count, positions, workspace, bytes, stream */
static PyObject* m_compress_ws(PyObject* self, PyObject* const* a, Py_ssize_t n) {
    Args s = {a, n, 0, 0};
    Clip c = clip(&s);
    void* tok = ptr(&s); int* cnt = ptr(&s); int* pos = ptr(&s); void* ws = ptr(&s); size_t b = size(&s);
    ttf_stream_t st = ptr(&s);
    CALL(fn.compress_ws(c.x, c.F, c.H, c.W, c.C, c.r, c.t, c.dtype, tok, cnt, pos, ws, b, st));
}
/* clip, frame base, tokens, count, positions, stream */
static PyObject* m_compress_segment(PyObject* self, PyObject* const* a, Py_ssize_t n) {
    Args s = {a, n, 0, 0};
    Clip c = clip(&s);
    int base = num(&s); void* tok = ptr(&s); int* cnt = ptr(&s); int* pos = ptr(&s); ttf_stream_t st = ptr(&s);
    CALL(fn.compress_segment(c.x, c.F, c.H, c.W, c.C, c.r, c.t, c.dtype, base, tok, cnt, pos, st));
}
/* clip, 4 options, anchor, keep, dst, best_sim, fuse_cnt, stream */
static PyObject* m_query(PyObject* self, PyObject* const* a, Py_ssize_t n) {
    Args s = {a, n, 0, 0};
    Clip c = clip(&s);
    ttf_options o = options(&s);
    int* an = ptr(&s); unsigned char* keep = ptr(&s); int* dst = ptr(&s); float* sim = ptr(&s); int* fuse = ptr(&s);
    ttf_stream_t st = ptr(&s);
    CALL(plain(&o) ? fn.query(c.x, c.F, c.H, c.W, c.C, c.r, c.t, c.dtype, an, keep, dst, sim, fuse, st)
                   : fn.query_ex(c.x, c.F, c.H, c.W, c.C, c.r, c.t, c.dtype, &o, an, keep, dst, sim, fuse, st));
}
/* clip, anchor, keep, dst, best_sim, fuse_cnt, workspace, bytes, stream */
static PyObject* m_query_ws(PyObject* self, PyObject* const* a, Py_ssize_t n) {
    Args s = {a, n, 0, 0};
    Clip c = clip(&s);
    int* an = ptr(&s); unsigned char* keep = ptr(&s); int* dst = ptr(&s); float* sim = ptr(&s); int* fuse = ptr(&s);
    void* ws = ptr(&s); size_t b = size(&s); ttf_stream_t st = ptr(&s);
    CALL(fn.query_ws(c.x, c.F, c.H, c.W, c.C, c.r, c.t, c.dtype, an, keep, dst, sim, fuse, ws, b, st));
}
/* compressed, row bytes, F, H, W, anchor, keep, dst, out, row index, stream */
static PyObject* m_restore(PyObject* self, PyObject* const* a, Py_ssize_t n) {
    Args s = {a, n, 0, 0};
    const void* x = ptr(&s); size_t b = size(&s); int F = num(&s), H = num(&s), W = num(&s);
    const int* an = ptr(&s); const unsigned char* keep = ptr(&s); const int* dst = ptr(&s);
    void* out = ptr(&s); int* idx = ptr(&s); ttf_stream_t st = ptr(&s);
    CALL(fn.restore(x, b, F, H, W, an, keep, dst, out, idx, st));
}
/* best_sim, keep, anchor, F, H, W, t, band, out, stream */
static PyObject* m_stats(PyObject* self, PyObject* const* a, Py_ssize_t n) {
    Args s = {a, n, 0, 0};
    const float* sim = ptr(&s); const unsigned char* keep = ptr(&s); const int* an = ptr(&s);
    int F = num(&s), H = num(&s), W = num(&s); float t = real(&s), band = real(&s);
    long long* out = ptr(&s); ttf_stream_t st = ptr(&s);
    CALL(fn.stats(sim, keep, an, F, H, W, t, band, out, st));
}
/* list of clip addresses, F, H, W, C, r, t, dtype, 4 options, lists of token, count and position addresses, stream */
static PyObject* m_compress_batch(PyObject* self, PyObject* const* a, Py_ssize_t n) {
    Args s = {a, n, 0, 0};
    PyObject* lists[4];
    lists[0] = next_arg(&s);
    int F = num(&s), H = num(&s), W = num(&s), C = num(&s), r = num(&s); float t = real(&s); int dtype = num(&s);
    ttf_options o = options(&s);
    for (int q = 1; q < 4; ++q) lists[q] = next_arg(&s);
    ttf_stream_t st = ptr(&s);
    if (!done(&s)) return NULL;
    Py_ssize_t B = PyList_Check(lists[0]) ? PyList_GET_SIZE(lists[0]) : -1;
    for (int q = 0; q < 4; ++q)
        if (!PyList_Check(lists[q]) || PyList_GET_SIZE(lists[q]) != B || B < 1 || B > 0x7fffffff) {
            PyErr_SetString(PyExc_ValueError, "four lists of one length");
            return NULL;
        }
    void** p = PyMem_Malloc(sizeof(void*) * 4 * (size_t)B);
    if (!p) return PyErr_NoMemory();
    for (int q = 0; q < 4; ++q)
        for (Py_ssize_t i = 0; i < B; ++i) {
            p[q * B + i] = PyLong_AsVoidPtr(PyList_GET_ITEM(lists[q], i));
            if (!p[q * B + i] && PyErr_Occurred()) { PyMem_Free(p); return NULL; }
        }
    int rc;
    Py_BEGIN_ALLOW_THREADS
    const void* const* x = (const void* const*)p;
    int* const* cnt = (int* const*)(p + 2 * B);
    int* const* pos = (int* const*)(p + 3 * B);
    rc = plain(&o) ? fn.compress_batch(x, (int)B, F, H, W, C, r, t, dtype, p + B, cnt, pos, st)
                   : fn.compress_batch_ex(x, (int)B, F, H, W, C, r, t, dtype, &o, p + B, cnt, pos, st);
    Py_END_ALLOW_THREADS
    PyMem_Free(p);
    return PyLong_FromLong(rc);
}

/* what the calls over the cache share: heads (address, strides, number), rotation, sequences, cache */
static ttf_heads heads(Args* s) {
    ttf_heads h;
    h.data = ptr(s); h.row_stride = wide(s); h.head_stride = wide(s); h.heads = num(s);
    return h;
}
static const ttf_heads* given(const ttf_heads* h) { return h->data ? h : NULL; }
static ttf_rotation rotation(Args* s) {
    ttf_rotation r;
    r.freq = ptr(s); r.rot_dim = num(s); r.interleaved = num(s); r.axes = num(s);
    for (int i = 0; i < 3; ++i) r.section[i] = num(s);
    r.cyclic = num(s); r.factor = real(s); r.q_weight = ptr(s); r.k_weight = ptr(s); r.eps = real(s);
    return r;
}
static ttf_sequences sequences(Args* s) {
    ttf_sequences q;
    q.start = ptr(s); q.length = ptr(s); q.table = ptr(s); q.table_stride = wide(s); q.table_pages = num(s); q.seqs = num(s);
    q.rows = num(s);
    return q;
}
static ttf_cache cache(Args* s) {
    ttf_cache c;
    c.k = ptr(s); c.k_page = wide(s); c.k_row = wide(s); c.k_head = wide(s);
    c.v = ptr(s); c.v_page = wide(s); c.v_row = wide(s); c.v_head = wide(s);
    c.pages = num(s); c.page_size = num(s); c.heads = num(s); c.head_dim = num(s); c.dtype = num(s);
    return c;
}
/* q, k, head dim, dtype, rows, count, positions, rotation, out_q, out_k, stream */
static PyObject* m_rotate(PyObject* self, PyObject* const* a, Py_ssize_t n) {
    Args s = {a, n, 0, 0};
    ttf_heads q = heads(&s), k = heads(&s);
    int dim = num(&s), dtype = num(&s), rows = num(&s);
    const int* cnt = ptr(&s); const int* pos = ptr(&s);
    ttf_rotation r = rotation(&s);
    ttf_heads oq = heads(&s), ok = heads(&s);
    ttf_stream_t st = ptr(&s);
    CALL(fn.rotate(given(&q), given(&k), dim, dtype, rows, cnt, pos, &r, given(&oq), given(&ok), st));
}
/* k, v, q, positions, rotated (0: as they come), rotation, sequences, cache, out_q, stream */
static PyObject* m_cache_append(PyObject* self, PyObject* const* a, Py_ssize_t n) {
    Args s = {a, n, 0, 0};
    ttf_heads k = heads(&s), v = heads(&s), q = heads(&s);
    const int* pos = ptr(&s);
    int rotated = num(&s);
    ttf_rotation r = rotation(&s);
    ttf_sequences sq = sequences(&s);
    ttf_cache c = cache(&s);
    ttf_heads oq = heads(&s);
    ttf_stream_t st = ptr(&s);
    CALL(fn.cache_append(given(&k), given(&v), given(&q), pos, rotated ? &r : NULL, &sq, &c, given(&oq), st));
}
/* q, sequences, cache, scale, causal, window, out, stream */
static PyObject* m_attend(PyObject* self, PyObject* const* a, Py_ssize_t n) {
    Args s = {a, n, 0, 0};
    ttf_heads q = heads(&s);
    ttf_sequences sq = sequences(&s);
    ttf_cache c = cache(&s);
    float scale = real(&s); int causal = num(&s), window = num(&s);
    ttf_heads o = heads(&s);
    ttf_stream_t st = ptr(&s);
    CALL(fn.attend(given(&q), &sq, &c, scale, causal, window, given(&o), st));
}

/* ---- tensors as they are -------------------------------------------------------------------------------------------
 * ttf_rotate, ttf_cache_append and ttf_attend take seven to twelve tensors each; asking every one for its shape, strides,
 * address, type and device from Python costs more than the kernels of a small call take.  These functions ask here (about
 * 0.3 us per tensor), and answer -1 where anything is not exactly as the plain case has it: the Python code then looks at
 * the arguments one by one, raises what is to be raised, or makes the call itself.  Nothing is kept between calls. */
static PyObject *t_f32, *t_bf16, *t_i32;                   /* the torch.dtype objects */
static PyObject *f_device, *f_stream;                      /* current device; current raw stream of a device */
static PyObject *s_shape, *s_dtype, *s_stride, *s_ptr, *s_dev;

typedef struct { long long n[4], s[4]; int dims, dev, type; void* p; } Facts;      /* type: 0 fp32, 1 bf16, 2 int32 */

static int longs(PyObject* t, long long* to) {             /* a tuple of up to four ints; its length, or -1 */
    if (!t || !PyTuple_Check(t) || PyTuple_GET_SIZE(t) > 4) { Py_XDECREF(t); return -1; }
    int n = (int)PyTuple_GET_SIZE(t);
    for (int i = 0; i < n; ++i) to[i] = PyLong_AsLongLong(PyTuple_GET_ITEM(t, i));
    Py_DECREF(t);
    return n;
}
static int facts(PyObject* x, Facts* f) {
    PyObject* o;
    f->dims = longs(PyObject_GetAttr(x, s_shape), f->n);
    if (f->dims < 0) return 0;
    if (longs(PyObject_CallMethodNoArgs(x, s_stride), f->s) != f->dims) return 0;
    if (!(o = PyObject_GetAttr(x, s_dtype))) return 0;
    f->type = o == t_f32 ? 0 : (o == t_bf16 ? 1 : (o == t_i32 ? 2 : -1));
    Py_DECREF(o);
    if (!(o = PyObject_CallMethodNoArgs(x, s_dev))) return 0;
    f->dev = (int)PyLong_AsLong(o);
    Py_DECREF(o);
    if (!(o = PyObject_CallMethodNoArgs(x, s_ptr))) return 0;
    f->p = PyLong_AsVoidPtr(o);
    Py_DECREF(o);
    return f->type >= 0 && !PyErr_Occurred();
}
/* [rows, heads, channels] of the type and device of `like` (rows and channels of it too) */
static int heads_of(PyObject* x, const Facts* like, ttf_heads* h) {
    Facts f;
    h->data = NULL; h->heads = 0; h->row_stride = h->head_stride = 0;
    if (x == Py_None) return 1;
    if (!facts(x, &f) || f.dims != 3 || f.type != like->type || f.dev != like->dev || f.n[0] != like->n[0] || f.n[2] != like->n[2] ||
        (f.s[2] != 1 && f.n[2] > 1) || f.n[1] < 1 || f.n[1] > 0x7fffffff || !f.p) return 0;
    h->data = f.p; h->row_stride = f.s[0]; h->head_stride = f.s[1]; h->heads = (int)f.n[1];
    return 1;
}
/* one contiguous axis of `n` elements (n < 0: any number) */
static int line_of(PyObject* x, int type, int dev, long long n, const void** p, long long* got) {
    Facts f;
    if (!facts(x, &f) || f.dims != 1 || f.type != type || f.dev != dev || (n >= 0 && f.n[0] != n) || (f.n[0] > 1 && f.s[0] != 1)) return 0;
    *p = f.p;
    if (got) *got = f.n[0];
    return 1;
}
static int cache_of(PyObject* k, PyObject* v, const Facts* like, ttf_cache* c) {
    Facts a, b;
    if (!facts(k, &a) || !facts(v, &b) || a.dims != 4 || b.dims != 4 || a.type != like->type || b.type != like->type ||
        a.dev != like->dev || b.dev != like->dev || a.n[3] != like->n[2]) return 0;
    for (int i = 0; i < 4; ++i) if (a.n[i] != b.n[i] || a.n[i] < 1 || a.n[i] > 0x7fffffff) return 0;
    if ((a.s[3] != 1 || b.s[3] != 1) && a.n[3] > 1) return 0;
    c->k = a.p; c->k_page = a.s[0]; c->k_row = a.s[1]; c->k_head = a.s[2];
    c->v = b.p; c->v_page = b.s[0]; c->v_row = b.s[1]; c->v_head = b.s[2];
    c->pages = (int)a.n[0]; c->page_size = (int)a.n[1]; c->heads = (int)a.n[2]; c->head_dim = (int)a.n[3]; c->dtype = a.type;
    return 1;
}
static int sequences_of(PyObject* start, PyObject* length, PyObject* table, const Facts* like, ttf_sequences* q) {
    Facts t;
    if (!facts(table, &t) || t.dims != 2 || t.type != 2 || t.dev != like->dev || t.n[0] < 1 || t.n[1] < 1 || t.n[0] > 0x7ffffffe ||
        t.n[1] > 0x7fffffff || (t.n[1] > 1 && t.s[1] != 1)) return 0;
    if (!line_of(start, 2, like->dev, t.n[0] + 1, (const void**)&q->start, NULL) ||
        !line_of(length, 2, like->dev, t.n[0], (const void**)&q->length, NULL)) return 0;
    q->table = t.p; q->table_stride = t.n[0] > 1 ? t.s[0] : t.n[1]; q->table_pages = (int)t.n[1]; q->seqs = (int)t.n[0];
    q->rows = (int)like->n[0];
    return 1;
}
/* positions, freq, q_weight, k_weight, rot_dim, interleaved, sections, cyclic, factor, eps from a[0] on */
static int rotation_of(PyObject* const* a, const Facts* like, ttf_rotation* r, const int** pos) {
    Facts f;
    if (!facts(a[0], &f) || f.type != 2 || f.dev != like->dev || f.dims < 1 || f.dims > 2 || f.n[0] != like->n[0]) return 0;
    if (f.dims == 1) { f.n[1] = 1; f.s[1] = 1; }
    if (f.n[1] < 1 || f.n[1] > 3 || (f.n[1] > 1 && f.s[1] != 1) || (f.n[0] > 1 && f.s[0] != f.n[1])) return 0;
    *pos = f.p;
    r->axes = (int)f.n[1];
    long long rot = a[4] == Py_None ? like->n[2] : PyLong_AsLongLong(a[4]);
    if (rot < 0 || rot > 0x7fffffff || !line_of(a[1], 0, like->dev, rot / 2, (const void**)&r->freq, NULL)) return 0;
    r->rot_dim = (int)rot;
    r->q_weight = r->k_weight = NULL;
    if (a[2] != Py_None && !line_of(a[2], like->type, like->dev, like->n[2], &r->q_weight, NULL)) return 0;
    if (a[3] != Py_None && !line_of(a[3], like->type, like->dev, like->n[2], &r->k_weight, NULL)) return 0;
    r->interleaved = PyObject_IsTrue(a[5]);
    r->section[0] = r->section[1] = r->section[2] = 0;
    if (a[6] == Py_None) {
        if (r->axes != 1) return 0;
    } else {
        if (!PyTuple_Check(a[6]) || PyTuple_GET_SIZE(a[6]) != r->axes) return 0;
        for (int i = 0; i < r->axes; ++i) {
            const long section = PyLong_AsLong(PyTuple_GET_ITEM(a[6], i));
            if (section != (int)section) return 0;
            r->section[i] = (int)section;
        }
    }
    r->cyclic = PyObject_IsTrue(a[7]);
    r->factor = (float)PyFloat_AsDouble(a[8]);
    r->eps = (float)PyFloat_AsDouble(a[9]);
    return !PyErr_Occurred();
}
/* the first tensor decides type and device; that device has to be the current one.  Its current stream, or the one given */
static int lead(PyObject* x, PyObject* stream, Facts* f, ttf_stream_t* st) {
    if (!facts(x, f) || f->dims != 3 || f->type > 1 || f->dev < 0 || f->n[0] < 1 || f->n[0] > 0x7fffffff || f->n[2] < 1 || f->n[2] > 0x7fffffff) return 0;
    PyObject* o = PyObject_CallNoArgs(f_device);
    if (!o) return 0;
    const long dev = PyLong_AsLong(o);
    if (dev != f->dev) { Py_DECREF(o); return 0; }
    if (stream == Py_None) {
        PyObject* p = PyObject_CallOneArg(f_stream, o);
        Py_DECREF(o);
        if (!p) return 0;
        *st = PyLong_AsVoidPtr(p);
        Py_DECREF(p);
    } else {
        Py_DECREF(o);
        if (!PyLong_Check(stream)) return 0;
        *st = PyLong_AsVoidPtr(stream);
    }
    return !PyErr_Occurred();
}
#define UNUSUAL() do { PyErr_Clear(); return PyLong_FromLong(-1); } while (0)
#define MADE(expr) do { int rc; Py_BEGIN_ALLOW_THREADS rc = (expr); Py_END_ALLOW_THREADS return PyLong_FromLong(rc); } while (0)

/* f32, bf16, int32 (torch.dtype objects), current device, current raw stream */
static PyObject* m_bind_torch(PyObject* self, PyObject* const* a, Py_ssize_t n) {
    if (n != 5) { PyErr_SetString(PyExc_TypeError, "bind_torch() takes three types and two functions"); return NULL; }
    for (int i = 0; i < 5; ++i) Py_INCREF(a[i]);
    t_f32 = a[0]; t_bf16 = a[1]; t_i32 = a[2]; f_device = a[3]; f_stream = a[4];
    s_shape = PyUnicode_InternFromString("shape"); s_dtype = PyUnicode_InternFromString("dtype");
    s_stride = PyUnicode_InternFromString("stride"); s_ptr = PyUnicode_InternFromString("data_ptr");
    s_dev = PyUnicode_InternFromString("get_device");
    Py_RETURN_NONE;
}
/* q, k, the ten of rotation_of, count, out_q, out_k, stream */
static PyObject* m_rotate_tensors(PyObject* self, PyObject* const* a, Py_ssize_t n) {
    Facts like;
    ttf_heads q, k, oq, ok;
    ttf_rotation r;
    ttf_stream_t st;
    const int* pos;
    const void* cnt = NULL;
    if (n != 16 || !t_f32 || !lead(a[0] != Py_None ? a[0] : a[1], a[15], &like, &st) || !heads_of(a[0], &like, &q) ||
        !heads_of(a[1], &like, &k) || !heads_of(a[13], &like, &oq) || !heads_of(a[14], &like, &ok) || q.heads != oq.heads ||
        k.heads != ok.heads || !rotation_of(a + 2, &like, &r, &pos) ||
        (a[12] != Py_None && !line_of(a[12], 2, like.dev, 1, &cnt, NULL))) UNUSUAL();
    MADE(fn.rotate(given(&q), given(&k), (int)like.n[2], like.type, (int)like.n[0], cnt, pos, &r, given(&oq), given(&ok), st));
}
/* k, v, k_cache, v_cache, start, length, table, the ten of rotation_of, q, out_q, stream */
static PyObject* m_cache_append_tensors(PyObject* self, PyObject* const* a, Py_ssize_t n) {
    Facts like;
    ttf_heads k, v, q, oq;
    ttf_cache c;
    ttf_sequences sq;
    ttf_rotation r;
    ttf_stream_t st;
    const int* pos;
    if (n != 20 || !t_f32 || !lead(a[0], a[19], &like, &st) || !heads_of(a[0], &like, &k) || !heads_of(a[1], &like, &v) ||
        !heads_of(a[17], &like, &q) || !heads_of(a[18], &like, &oq) || q.heads != oq.heads || a[7] == Py_None ||
        !cache_of(a[2], a[3], &like, &c) || !sequences_of(a[4], a[5], a[6], &like, &sq) || !rotation_of(a + 7, &like, &r, &pos)) UNUSUAL();
    MADE(fn.cache_append(given(&k), given(&v), given(&q), pos, &r, &sq, &c, given(&oq), st));
}
/* q, k_cache, v_cache, start, length, table, scale, causal, window, out, stream */
static PyObject* m_attend_tensors(PyObject* self, PyObject* const* a, Py_ssize_t n) {
    Facts like;
    ttf_heads q, o;
    ttf_cache c;
    ttf_sequences sq;
    ttf_stream_t st;
    if (n != 11 || !t_f32 || !lead(a[0], a[10], &like, &st) || !heads_of(a[0], &like, &q) || !heads_of(a[9], &like, &o) ||
        q.heads != o.heads || !cache_of(a[1], a[2], &like, &c) || !sequences_of(a[3], a[4], a[5], &like, &sq)) UNUSUAL();
    const double scale = PyFloat_AsDouble(a[6]);
    const int causal = PyObject_IsTrue(a[7]);
    const long window = PyLong_AsLong(a[8]);
    if (PyErr_Occurred() || window != (int)window) UNUSUAL();
    MADE(fn.attend(&q, &sq, &c, (float)scale, causal, (int)window, &o, st));
}

#define METHOD(name) {#name, (PyCFunction)(void (*)(void))m_##name, METH_FASTCALL, NULL}
static PyMethodDef methods[] = {METHOD(bind), METHOD(compress), METHOD(compress_ws), METHOD(compress_segment),
                                METHOD(compress_batch), METHOD(query), METHOD(query_ws), METHOD(restore), METHOD(stats),
                                METHOD(rotate), METHOD(cache_append), METHOD(attend),
                                METHOD(bind_torch), METHOD(rotate_tensors), METHOD(cache_append_tensors), METHOD(attend_tensors),
                                {NULL, NULL, 0, NULL}};
static struct PyModuleDef module = {PyModuleDef_HEAD_INIT, "_marshal", NULL, -1, methods, NULL, NULL, NULL, NULL};
PyMODINIT_FUNC PyInit__marshal(void) { return PyModule_Create(&module); }
