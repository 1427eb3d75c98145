// Native side of the Python binding: takes the binding's Segment / Cache objects and tensors apart and calls the C ABI.
//
// The calls of a frame step are short on the GPU for small frames, so the time that the host takes to issue them decides:
// building the same structs through ctypes took 51 us of host time for a frame step (6.4 us per cache, 9.6 us for the plan,
// 2.3 us per array pointer), more than the launches of the step.  Host time of a
// pass, ctypes against this file: frame step 51 -> 27 us (fp32 62 -> 24, with a shorter launch list), attention over a cache
// 19.8 -> 10.6, mask, score, pack and attend 82 -> 36; the small bf16 step 53.8 -> 37.5 us a pass.
// Tensors are read through their Python methods (data_ptr, is_contiguous, shape) or the C table of their type, so nothing here depends on torch's C++ ABI.
// Each function returns the pc_status; the Python wrapper raises.  The interpreter lock is released around the library calls.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <algorithm>
#include <cstdarg>
#include <cstdint>
#include <vector>

#include <ATen/dlpack.h>

#include "packcache.h"

namespace {

PyObject *s_data_ptr, *s_is_contiguous, *s_shape, *s_k, *s_v, *s_pos, *s_n_tokens, *s_anchors, *s_history, *s_frame_count, *s_value, *s_rows, *s_weight, *s_t_shift;
PyObject *g_f32, *g_tensor, *g_refusal;          // torch.float32, torch.Tensor; the binding's error, made of a status and a text
const DLPackExchangeAPI *g_exchange;              // through which a tensor describes itself in one call
PyObject *g_as_i32;       // numpy.ascontiguousarray(x, dtype=int32), for anything that is not an int32 array already

bool failed() { return PyErr_Occurred() != nullptr; }

// Address of a tensor (None: null).  Sets an error if it is not contiguous.
void *tensor_ptr(PyObject *t) {
    if (t == Py_None) return nullptr;
    PyObject *c = PyObject_CallMethodNoArgs(t, s_is_contiguous);
    if (!c) return nullptr;
    const int ok = PyObject_IsTrue(c);
    Py_DECREF(c);
    if (ok <= 0) {
        if (ok == 0) PyErr_SetString(PyExc_AssertionError, "tensors passed to the library must be contiguous");
        return nullptr;
    }
    PyObject *p = PyObject_CallMethodNoArgs(t, s_data_ptr);
    if (!p) return nullptr;
    void *r = PyLong_AsVoidPtr(p);
    Py_DECREF(p);
    return r;
}

int32_t int_of(PyObject *o) { return (int32_t)PyLong_AsLong(o); }

int32_t int_attr(PyObject *o, PyObject *name) {
    PyObject *v = PyObject_GetAttr(o, name);
    if (!v) return 0;
    PyObject *i = PyNumber_Index(v);                  // numpy integers as well
    Py_DECREF(v);
    if (!i) return 0;
    const int32_t r = int_of(i);
    Py_DECREF(i);
    return r;
}

// first extent of a tensor
int32_t rows_of(PyObject *t) {
    PyObject *s = PyObject_GetAttr(t, s_shape);
    if (!s) return 0;
    PyObject *n = PySequence_GetItem(s, 0);
    Py_DECREF(s);
    if (!n) return 0;
    const int32_t r = int_of(n);
    Py_DECREF(n);
    return r;
}

void *handle_of(PyObject *h) {                        // a ctypes c_void_p, or None after close()
    if (h == Py_None) return nullptr;
    PyObject *v = PyObject_GetAttr(h, s_value);
    if (!v) return nullptr;
    void *p = v == Py_None ? nullptr : PyLong_AsVoidPtr(v);
    Py_DECREF(v);
    return p;
}

void *stream_of(PyObject *s) { return PyLong_AsVoidPtr(s); }

// A host array of int32 with any number of dimensions, held for the duration of a call.
struct Ints {
    Py_buffer view{};
    const int32_t *p = nullptr;
    int32_t n = 0;            // its length (first extent)
    int64_t size = 0;         // elements in all
    bool take(PyObject *o) {
        if (!as_is(o)) {
            PyObject *a = PyObject_CallOneArg(g_as_i32, o);
            if (!a) return false;
            const bool ok = as_is(a);                 // the buffer holds the array from here on
            Py_DECREF(a);
            if (!ok) {
                if (!failed()) PyErr_SetString(PyExc_TypeError, "an array of integers is expected");
                return false;
            }
        }
        return true;
    }
    bool as_is(PyObject *o) {
        if (!PyObject_CheckBuffer(o)) return false;
        if (PyObject_GetBuffer(o, &view, PyBUF_FORMAT | PyBUF_C_CONTIGUOUS) != 0) {
            PyErr_Clear();
            return false;
        }
        const char *f = view.format ? view.format : "B";
        if (view.itemsize != 4 || view.ndim < 1 || f[1] != '\0' || (f[0] != 'i' && f[0] != 'l')) {
            PyBuffer_Release(&view);
            view = Py_buffer{};
            return false;
        }
        p = static_cast<const int32_t *>(view.buf);
        n = (int32_t)view.shape[0];
        size = view.len / 4;
        return true;
    }
    // the library reads (or writes) this many entries: a shorter array is an error
    bool holds(int32_t want, const char *what) const {
        if (size >= want) return true;
        PyErr_Format(PyExc_ValueError, "%s has %lld entries, %d are needed", what, (long long)size, (int)want);
        return false;
    }
    ~Ints() {
        if (view.obj) PyBuffer_Release(&view);
    }
};

bool segment_of(PyObject *o, pc_segment *out) {
    *out = pc_segment{};
    PyObject *k = PyObject_GetAttr(o, s_k), *v = PyObject_GetAttr(o, s_v), *pos = PyObject_GetAttr(o, s_pos);
    if (k && v && pos) {
        out->k = tensor_ptr(k);
        if (!failed()) out->v = tensor_ptr(v);
        if (!failed()) out->pos = static_cast<int32_t *>(tensor_ptr(pos));
        if (!failed()) out->n_tokens = int_attr(o, s_n_tokens);
        if (!failed() && k != Py_None) out->capacity = rows_of(k);
    }
    Py_XDECREF(k);
    Py_XDECREF(v);
    Py_XDECREF(pos);
    return !failed();
}

// ---- Calls of the 4-bit cache and of eviction look at the types and lengths of what they are given (the kernels would read and write past it): what does not
// fit is refused as PC_ERR_INVALID_ARG, with the tensor's name.
void refuse(const char *format, ...) {
    va_list args;
    va_start(args, format);
    PyObject *text = PyUnicode_FromFormatV(format, args);
    va_end(args);
    if (!text) return;
    PyObject *e = PyObject_CallFunction(g_refusal, "iO", (int)PC_ERR_INVALID_ARG, text);
    Py_DECREF(text);
    if (!e) return;
    PyErr_SetObject(g_refusal, e);
    Py_DECREF(e);
}

enum Type { I32, F32, BF16, U8, BYTE /* any of one byte */ };

// Where a tensor lies and what it holds.  Asked for through the table that the tensor's type publishes (DLPack's C exchange table): address, contiguity, shape,
// type and bytes one attribute after the other are five calls of 0.05 to 0.1 us a tensor, of which a call has six to eleven.
struct Tensor {
    void *p = nullptr;                                // null for None
    int64_t rows = 0, n = 0;                          // first extent, elements
    DLDataType type{};
    bool none = true;

    bool take(PyObject *t) {
        if (t == Py_None) return true;
        if (!PyObject_TypeCheck(t, reinterpret_cast<PyTypeObject *>(g_tensor))) {
            PyErr_Format(PyExc_TypeError, "a tensor is expected, not %s", Py_TYPE(t)->tp_name);
            return false;
        }
        DLTensor d;
        if (g_exchange->dltensor_from_py_object_no_sync(t, &d) != 0) return false;
        n = 1;
        bool dense = true;
        for (int i = d.ndim - 1; i >= 0; --i) {       // strides of extents of one may be anything
            if (d.strides && d.shape[i] != 1 && d.strides[i] != n) dense = false;
            n *= d.shape[i];
        }
        if (!dense && n > 0) {
            PyErr_SetString(PyExc_AssertionError, "tensors passed to the library must be contiguous");
            return false;
        }
        p = static_cast<char *>(d.data) + d.byte_offset;
        rows = d.ndim > 0 ? d.shape[0] : 1;
        type = d.dtype;
        none = false;
        return true;
    }
    bool is(Type t) const {
        if (type.lanes != 1) return false;
        switch (t) {
        case I32: return type.code == kDLInt && type.bits == 32;
        case F32: return type.code == kDLFloat && type.bits == 32;
        case BF16: return type.code == kDLBfloat && type.bits == 16;
        case U8: return type.code == kDLUInt && type.bits == 8;
        case BYTE: return type.bits == 8;
        }
        return false;
    }
    enum How { AT_LEAST, EXACTLY };
    // It has elements of this type, and so many of them; None is left to the library
    bool fits(Type t, int64_t want, How how, const char *what) const {
        static const char *const names[] = {"torch.int32", "torch.float32", "torch.bfloat16", "torch.uint8", "of one byte an element"};
        if (none) return true;
        if (!is(t)) {
            refuse("%s has to be %s", what, names[t]);
            return false;
        }
        if (how == EXACTLY ? n == want : n >= want) return true;
        refuse("%s has %lld elements, %lld are needed", what, (long long)n, (long long)want);
        return false;
    }
};

// heads, head dimension and element type of a context (Context.sizes)
struct Sizes {
    long long hq, hkv, d;
    Type type;
    bool take(PyObject *t) {
        PyObject *dtype;
        if (!PyArg_ParseTuple(t, "LLLO", &hq, &hkv, &d, &dtype)) return false;
        type = dtype == g_f32 ? F32 : BF16;
        return true;
    }
    int64_t q_row() const { return hq * d; }
    int64_t kv_row() const { return hkv * d; }
};

bool tensor_attr(PyObject *o, PyObject *name, Tensor *out) {
    PyObject *t = PyObject_GetAttr(o, name);
    if (!t) return false;
    const bool ok = out->take(t);
    Py_DECREF(t);
    return ok;
}

bool fitting_segment_of(PyObject *o, const Sizes &z, pc_segment *out) {
    Tensor k, v, pos;
    if (!tensor_attr(o, s_k, &k) || !tensor_attr(o, s_v, &v) || !tensor_attr(o, s_pos, &pos)) return false;
    const int64_t n = k.rows;
    *out = pc_segment{k.p, v.p, static_cast<int32_t *>(pos.p), int_attr(o, s_n_tokens), (int32_t)n};
    return !failed() && k.fits(z.type, n * z.kv_row(), Tensor::EXACTLY, "k") && v.fits(z.type, n * z.kv_row(), Tensor::AT_LEAST, "v") &&
           pos.fits(I32, 4 * n, Tensor::AT_LEAST, "pos");
}

bool q4_segment_of(PyObject *o, const Sizes &z, pc_q4_segment *out) {
    Tensor rows, pos, weight;
    if (!tensor_attr(o, s_rows, &rows) || !tensor_attr(o, s_pos, &pos) || !tensor_attr(o, s_weight, &weight)) return false;
    const int64_t n = rows.rows;
    *out = pc_q4_segment{rows.p, static_cast<int32_t *>(pos.p), static_cast<float *>(weight.p), int_attr(o, s_n_tokens), (int32_t)n, int_attr(o, s_t_shift)};
    return !failed() && rows.fits(U8, n * z.kv_row() * 5 / 4, Tensor::EXACTLY, "rows") && pos.fits(I32, 4 * n, Tensor::AT_LEAST, "pos") &&
           weight.fits(F32, n, Tensor::AT_LEAST, "weight");
}

struct CacheArg {
    pc_cache c{};
    Ints counts;
    bool take(PyObject *o) {
        PyObject *a = PyObject_GetAttr(o, s_anchors);
        if (!a) return false;
        const bool ok_a = segment_of(a, &c.anchors);
        Py_DECREF(a);
        if (!ok_a) return false;
        PyObject *h = PyObject_GetAttr(o, s_history);
        if (!h) return false;
        const bool ok_h = segment_of(h, &c.history);
        Py_DECREF(h);
        if (!ok_h) return false;
        PyObject *f = PyObject_GetAttr(o, s_frame_count);
        if (!f) return false;
        const bool ok_f = counts.take(f);
        Py_DECREF(f);
        c.n_frames = counts.n;
        c.frame_count = counts.p;
        return ok_f;
    }
};

template <typename F> PyObject *call(F f) {
    pc_status st;
    Py_BEGIN_ALLOW_THREADS
    st = f();
    Py_END_ALLOW_THREADS
    return PyLong_FromLong((long)st);
}

bool arity(Py_ssize_t got, Py_ssize_t want) {
    if (got == want) return true;
    PyErr_Format(PyExc_TypeError, "%zd arguments expected, got %zd", want, got);
    return false;
}

// Tensors of a call, in order; null for None.
template <int N> struct Tensors {
    void *p[N];
    bool take(PyObject *const *a) {
        for (int i = 0; i < N; ++i) {
            p[i] = tensor_ptr(a[i]);
            if (failed()) return false;
        }
        return true;
    }
};

PyObject *plan_budget(PyObject *, PyObject *const *a, Py_ssize_t n) {       // kind, param, total, keep_full, min_quota, avail, out
    if (!arity(n, 7)) return nullptr;
    pc_budget_params p{};
    p.kind = int_of(a[0]);
    p.param = PyFloat_AsDouble(a[1]);
    p.total = PyLong_AsLongLong(a[2]);
    p.keep_full = int_of(a[3]);
    p.min_quota = int_of(a[4]);
    Ints avail, out;
    if (failed() || !avail.take(a[5]) || !out.take(a[6]) || !out.holds(avail.n, "the budget array")) return nullptr;
    return PyLong_FromLong((long)pc_plan_budget(&p, avail.n, avail.p, const_cast<int32_t *>(out.p)));
}

PyObject *total(PyObject *, PyObject *const *a, Py_ssize_t n) {             // sum of an int32 array
    if (!arity(n, 1)) return nullptr;
    Ints v;
    if (!v.take(a[0])) return nullptr;
    int64_t s = 0;
    for (int64_t i = 0; i < v.size; ++i) s += v.p[i];
    return PyLong_FromLongLong(s);
}

PyObject *score(PyObject *, PyObject *const *a, Py_ssize_t n) {             // ctx, src, q, q_pos, budget, valid, override, scores, sel, stream
    if (!arity(n, 10)) return nullptr;
    CacheArg src;
    Ints budget;
    Tensors<2> q;
    Tensors<4> t;
    void *ctx = handle_of(a[0]), *stream = stream_of(a[9]);
    if (failed() || !src.take(a[1]) || !q.take(a + 2) || !budget.take(a[4]) || !budget.holds(src.c.n_frames, "budget") || !t.take(a + 5)) return nullptr;
    const int32_t n_q = a[2] == Py_None ? 0 : rows_of(a[2]);
    if (failed()) return nullptr;
    return call([&] {
        return pc_score(static_cast<pc_ctx *>(ctx), &src.c, q.p[0], static_cast<int32_t *>(q.p[1]), n_q, budget.p,
                        static_cast<uint8_t *>(t.p[0]), static_cast<float *>(t.p[1]), static_cast<float *>(t.p[2]),
                        static_cast<int32_t *>(t.p[3]), stream);
    });
}

PyObject *compact(PyObject *, PyObject *const *a, Py_ssize_t n) {           // ctx, src, sel, budget, delta_t, dst, stream
    if (!arity(n, 7)) return nullptr;
    CacheArg src, dst;
    Ints budget;
    Tensors<1> sel;
    void *ctx = handle_of(a[0]), *stream = stream_of(a[6]);
    const int32_t delta_t = int_of(a[4]);
    if (failed() || !src.take(a[1]) || !sel.take(a + 2) || !budget.take(a[3]) || !budget.holds(src.c.n_frames, "budget") || !dst.take(a[5])) return nullptr;
    return call([&] { return pc_compact(static_cast<pc_ctx *>(ctx), &src.c, static_cast<int32_t *>(sel.p[0]), budget.p, delta_t, &dst.c, stream); });
}

PyObject *attend_frame(PyObject *, PyObject *const *a, Py_ssize_t n) {      // ctx, cache, current, q, q_pos, out, lse, stream
    if (!arity(n, 8)) return nullptr;
    CacheArg cache;
    pc_segment cur{};
    Tensors<4> t;
    void *ctx = handle_of(a[0]), *stream = stream_of(a[7]);
    if (failed() || !cache.take(a[1]) || (a[2] != Py_None && !segment_of(a[2], &cur)) || !t.take(a + 3)) return nullptr;
    const int32_t n_q = rows_of(a[3]);
    if (failed()) return nullptr;
    return call([&] {
        return pc_attend_frame(static_cast<pc_ctx *>(ctx), &cache.c, a[2] != Py_None ? &cur : nullptr, t.p[0], static_cast<int32_t *>(t.p[1]),
                               n_q, t.p[2], static_cast<float *>(t.p[3]), stream);
    });
}

PyObject *attend_prepare(PyObject *, PyObject *const *a, Py_ssize_t n) {    // ctx, cache, current, stream
    if (!arity(n, 4)) return nullptr;
    CacheArg cache;
    pc_segment cur{};
    void *ctx = handle_of(a[0]), *stream = stream_of(a[3]);
    if (failed() || !cache.take(a[1]) || (a[2] != Py_None && !segment_of(a[2], &cur))) return nullptr;
    return call([&] { return pc_attend_prepare(static_cast<pc_ctx *>(ctx), &cache.c, a[2] != Py_None ? &cur : nullptr, stream); });
}

PyObject *attend_prepared(PyObject *, PyObject *const *a, Py_ssize_t n) {   // ctx, q, q_pos, out, lse, stream
    if (!arity(n, 6)) return nullptr;
    Tensors<4> t;
    void *ctx = handle_of(a[0]), *stream = stream_of(a[5]);
    if (failed() || !t.take(a + 1)) return nullptr;
    const int32_t n_q = rows_of(a[1]);
    if (failed()) return nullptr;
    return call([&] {
        return pc_attend_prepared(static_cast<pc_ctx *>(ctx), t.p[0], static_cast<int32_t *>(t.p[1]), n_q, t.p[2], static_cast<float *>(t.p[3]), stream);
    });
}

PyObject *attend_mass(PyObject *, PyObject *const *a, Py_ssize_t n) {       // ctx, lse, mass, n_keys, stream
    if (!arity(n, 5)) return nullptr;
    Tensors<2> t;
    void *ctx = handle_of(a[0]), *stream = stream_of(a[4]);
    const int32_t n_keys = int_of(a[3]);
    if (failed() || !t.take(a + 1)) return nullptr;
    return call([&] { return pc_attend_mass(static_cast<pc_ctx *>(ctx), static_cast<float *>(t.p[0]), static_cast<float *>(t.p[1]), n_keys, stream); });
}

PyObject *frame_step(PyObject *, PyObject *const *a, Py_ssize_t n) {        // ctx, src, budget, delta_t, dst, q, q_pos, scores, sel, out, lse, stream
    if (!arity(n, 12)) return nullptr;
    CacheArg src, dst;
    Ints budget;
    Tensors<6> t;
    void *ctx = handle_of(a[0]), *stream = stream_of(a[11]);
    const int32_t delta_t = int_of(a[3]);
    if (failed() || !src.take(a[1]) || !budget.take(a[2]) || !budget.holds(src.c.n_frames, "budget") || !dst.take(a[4]) || !t.take(a + 5)) return nullptr;
    const int32_t n_q = rows_of(a[5]);
    if (failed()) return nullptr;
    return call([&] {
        return pc_frame_step(static_cast<pc_ctx *>(ctx), &src.c, budget.p, delta_t, &dst.c, t.p[0], static_cast<int32_t *>(t.p[1]), n_q,
                             static_cast<float *>(t.p[2]), static_cast<int32_t *>(t.p[3]), t.p[4], static_cast<float *>(t.p[5]), stream);
    });
}

PyObject *window_append(PyObject *, PyObject *const *a, Py_ssize_t n) {     // window, frame, stream
    if (!arity(n, 3)) return nullptr;
    pc_segment frame{};
    void *w = handle_of(a[0]), *stream = stream_of(a[2]);
    if (failed() || !segment_of(a[1], &frame)) return nullptr;
    return call([&] { return pc_window_append(static_cast<pc_window *>(w), &frame, stream); });
}

PyObject *window_step(PyObject *, PyObject *const *a, Py_ssize_t n) {       // window, q, q_pos, out, lse, stream -> (status, regime)
    if (!arity(n, 6)) return nullptr;
    Tensors<4> t;
    void *w = handle_of(a[0]), *stream = stream_of(a[5]);
    if (failed() || !t.take(a + 1)) return nullptr;
    const int32_t n_q = rows_of(a[1]);
    if (failed()) return nullptr;
    int32_t regime = -1;
    pc_status st;
    Py_BEGIN_ALLOW_THREADS
    st = pc_window_step(static_cast<pc_window *>(w), t.p[0], static_cast<int32_t *>(t.p[1]), n_q, t.p[2], static_cast<float *>(t.p[3]), &regime, stream);
    Py_END_ALLOW_THREADS
    return Py_BuildValue("ii", (int)st, (int)regime);
}

PyObject *q4_store(PyObject *, PyObject *const *a, Py_ssize_t n) {          // ctx, sizes, src, dst, at, stream
    if (!arity(n, 6)) return nullptr;
    Sizes z;
    pc_segment src{};
    pc_q4_segment dst{};
    void *ctx = handle_of(a[0]), *stream = stream_of(a[5]);
    const int32_t at = int_of(a[4]);
    if (failed() || !z.take(a[1]) || !fitting_segment_of(a[2], z, &src) || !q4_segment_of(a[3], z, &dst)) return nullptr;
    return call([&] { return pc_q4_store(static_cast<pc_ctx *>(ctx), &src, &dst, at, stream); });
}

PyObject *q4_load(PyObject *, PyObject *const *a, Py_ssize_t n) {           // ctx, sizes, src, first, n, dst, stream
    if (!arity(n, 7)) return nullptr;
    Sizes z;
    pc_q4_segment src{};
    pc_segment dst{};
    void *ctx = handle_of(a[0]), *stream = stream_of(a[6]);
    const int32_t first = int_of(a[3]), count = int_of(a[4]);
    if (failed() || !z.take(a[1]) || !q4_segment_of(a[2], z, &src) || !fitting_segment_of(a[5], z, &dst)) return nullptr;
    return call([&] { return pc_q4_load(static_cast<pc_ctx *>(ctx), &src, first, count, &dst, stream); });
}

PyObject *q4_attend(PyObject *, PyObject *const *a, Py_ssize_t n) {         // work, sizes, cache, valid, q, q_pos, out, lse, decay, gain (None: no weights), stream
    if (!arity(n, 11)) return nullptr;
    Sizes z;
    pc_q4_cache cache{};
    Tensor valid, q, q_pos, out, lse;
    pc_q4_weigh weigh{};
    void *work = handle_of(a[0]), *stream = stream_of(a[10]);
    const bool weighs = a[8] != Py_None;
    if (weighs) {
        weigh.decay = (float)PyFloat_AsDouble(a[8]);
        weigh.gain = (float)PyFloat_AsDouble(a[9]);
    }
    if (failed() || !z.take(a[1])) return nullptr;
    PyObject *anchors = PyObject_GetAttr(a[2], s_anchors), *history = PyObject_GetAttr(a[2], s_history);
    const bool ok = anchors && history && q4_segment_of(anchors, z, &cache.anchors) && q4_segment_of(history, z, &cache.history);
    Py_XDECREF(anchors);
    Py_XDECREF(history);
    if (!ok || !valid.take(a[3]) || !q.take(a[4]) || !q_pos.take(a[5]) || !out.take(a[6]) || !lse.take(a[7])) return nullptr;
    const int64_t n_q = q.rows;
    if (!valid.fits(BYTE, cache.history.n_tokens, Tensor::AT_LEAST, "valid") || !q.fits(z.type, n_q * z.q_row(), Tensor::EXACTLY, "q") ||
        !q_pos.fits(I32, 4 * n_q, Tensor::AT_LEAST, "q_pos") || !out.fits(z.type, n_q * z.q_row(), Tensor::AT_LEAST, "out") ||
        !lse.fits(F32, n_q * z.hq, Tensor::AT_LEAST, "lse")) return nullptr;
    return call([&] {
        return pc_q4_attend(static_cast<pc_q4 *>(work), &cache, static_cast<uint8_t *>(valid.p), q.p, static_cast<int32_t *>(q_pos.p), (int32_t)n_q, out.p,
                            static_cast<float *>(lse.p), weighs ? &weigh : nullptr, stream);
    });
}

PyObject *q4_evict(PyObject *, PyObject *const *a, Py_ssize_t n) {          // ctx, sizes, src, keep, recent, delta_t, valid, dst, sel, stream
    if (!arity(n, 10)) return nullptr;
    Sizes z;
    pc_q4_segment src{}, dst{};
    Tensor valid, sel;
    void *ctx = handle_of(a[0]), *stream = stream_of(a[9]);
    const pc_evict_params p{int_of(a[3]), int_of(a[4]), int_of(a[5])};
    if (failed() || !z.take(a[1]) || !q4_segment_of(a[2], z, &src) || !valid.take(a[6]) || !q4_segment_of(a[7], z, &dst) || !sel.take(a[8]) ||
        !valid.fits(BYTE, src.n_tokens, Tensor::AT_LEAST, "valid") || !sel.fits(I32, std::min(p.keep, src.n_tokens), Tensor::AT_LEAST, "sel_idx")) return nullptr;
    return call([&] {
        return pc_q4_evict(static_cast<pc_ctx *>(ctx), &src, &p, static_cast<uint8_t *>(valid.p), &dst, static_cast<int32_t *>(sel.p), stream);
    });
}

PyObject *evict(PyObject *, PyObject *const *a, Py_ssize_t n) {             // ctx, sizes, src, weight, keep, recent, delta_t, valid, dst, dst_weight, sel, stream
    if (!arity(n, 12)) return nullptr;
    Sizes z;
    pc_segment src{}, dst{};
    Tensor weight, valid, to_weight, sel;
    void *ctx = handle_of(a[0]), *stream = stream_of(a[11]);
    const pc_evict_params p{int_of(a[4]), int_of(a[5]), int_of(a[6])};
    if (failed() || !z.take(a[1]) || !fitting_segment_of(a[2], z, &src) || !weight.take(a[3]) || !valid.take(a[7]) || !fitting_segment_of(a[8], z, &dst) ||
        !to_weight.take(a[9]) || !sel.take(a[10])) return nullptr;
    const int64_t kept = std::min(p.keep, src.n_tokens);
    if (!weight.fits(F32, src.n_tokens, Tensor::AT_LEAST, "weight") || !valid.fits(BYTE, src.n_tokens, Tensor::AT_LEAST, "valid") ||
        !to_weight.fits(F32, kept, Tensor::AT_LEAST, "dst_weight") || !sel.fits(I32, kept, Tensor::AT_LEAST, "sel_idx")) return nullptr;
    return call([&] {
        return pc_evict(static_cast<pc_ctx *>(ctx), &src, static_cast<float *>(weight.p), &p, static_cast<uint8_t *>(valid.p), &dst,
                        static_cast<float *>(to_weight.p), static_cast<int32_t *>(sel.p), stream);
    });
}

PyObject *set_i32_converter(PyObject *, PyObject *f) {
    Py_INCREF(f);
    Py_XSETREF(g_as_i32, f);
    Py_RETURN_NONE;
}

PyObject *set_types(PyObject *, PyObject *const *a, Py_ssize_t n) {        // torch.float32, torch.Tensor, its exchange table, the error
    if (!arity(n, 4)) return nullptr;
    const auto *table = static_cast<const DLPackExchangeAPI *>(PyCapsule_GetPointer(a[2], "dlpack_exchange_api"));
    if (!table) return nullptr;
    if (table->header.version.major != DLPACK_MAJOR_VERSION || !table->dltensor_from_py_object_no_sync) {
        PyErr_SetString(PyExc_RuntimeError, "tensors do not describe themselves in a form that is known here");
        return nullptr;
    }
    g_exchange = table;
    PyObject **to[] = {&g_f32, &g_tensor, &g_refusal}, *from[] = {a[0], a[1], a[3]};
    for (int i = 0; i < 3; ++i) {
        Py_INCREF(from[i]);
        Py_XSETREF(*to[i], from[i]);
    }
    Py_RETURN_NONE;
}

#define FAST(name) {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)(void)>(name)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {FAST(plan_budget), FAST(total), FAST(score), FAST(compact), FAST(attend_frame), FAST(attend_prepare), FAST(attend_prepared),
                         FAST(attend_mass), FAST(frame_step), FAST(window_append), FAST(window_step),
                         FAST(q4_store), FAST(q4_load), FAST(q4_attend), FAST(q4_evict), FAST(evict), FAST(set_types),
                         {"set_i32_converter", set_i32_converter, METH_O, nullptr}, {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_packcache_py", "Calls of libpackcache.so on the binding's objects.", -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__packcache_py(void) {
    struct { PyObject **at; const char *name; } names[] = {{&s_data_ptr, "data_ptr"}, {&s_is_contiguous, "is_contiguous"}, {&s_shape, "shape"},
        {&s_k, "k"}, {&s_v, "v"}, {&s_pos, "pos"}, {&s_n_tokens, "n_tokens"}, {&s_anchors, "anchors"}, {&s_history, "history"},
        {&s_frame_count, "frame_count"}, {&s_value, "value"}, {&s_rows, "rows"}, {&s_weight, "weight"}, {&s_t_shift, "t_shift"}};
    for (auto &x : names)
        if (!(*x.at = PyUnicode_InternFromString(x.name))) return nullptr;
    return PyModule_Create(&module);
}
