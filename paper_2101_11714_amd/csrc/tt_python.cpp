// Argument marshalling of the calls that a training or serving step makes, as a CPython extension: tensors are unpacked,
// checked and handed to the C ABI of libtt_emb.so here, where the same work in Python (ctypes objects, a dozen tensor
// attributes and the current stream, per call) took 6-9 us, more than most of the kernels of a step.  Host time of a pass:
// a forward of 64 lookups 8.7 -> 3.4 us, the two calls of the Kaggle-shaped step 20 -> 7 us, of which the launches are 2-3 us each.
// Every function takes its arguments by position, returns the library's return code, and raises AssertionError for a
// tensor of the wrong device, type, layout or size.  binding.py documents and wraps them.  What torch throws on the way
// (a tensor without storage, as tracing and vmap make them) becomes a RuntimeError.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <c10/hip/HIPStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include "../../include/tt_emb.h"

namespace {

// What a call has collected; `ok` turns false, with the Python error set, at the first argument that does not fit.
struct Args {
    PyObject *const *a;
    bool ok = true;

    explicit Args(PyObject *const *args, Py_ssize_t n, Py_ssize_t want) : a(args)
    {
        if (n != want) {
            PyErr_Format(PyExc_TypeError, "%zd arguments expected, %zd given", want, n);
            ok = false;
        }
    }

    bool fail(const char *what)
    {
        if (ok) PyErr_SetString(PyExc_AssertionError, what);
        return ok = false;
    }

    const at::Tensor *tensor(PyObject *o)
    {
        if (!ok) return nullptr;
        if (!THPVariable_Check(o)) {
            PyErr_SetString(PyExc_TypeError, "a tensor is expected");
            ok = false;
            return nullptr;
        }
        return &THPVariable_Unpack(o);
    }

    // a contiguous device tensor of the given type: its address, and the number of its elements in *n
    void *dev(PyObject *o, at::ScalarType type, int64_t *n = nullptr)
    {
        const at::Tensor *t = tensor(o);
        if (!t) return nullptr;
        if (!t->is_cuda() || t->scalar_type() != type || !t->is_contiguous()) {
            fail("a contiguous device tensor of the right type is expected");
            return nullptr;
        }
        if (n) *n = t->numel();
        return t->data_ptr();
    }
    float *f32(int i, int64_t *n = nullptr) { return (float *)dev(a[i], at::kFloat, n); }
    int64_t *i64(int i, int64_t *n = nullptr) { return (int64_t *)dev(a[i], at::kLong, n); }
    uint8_t *u8(int i, int64_t *n = nullptr) { return (uint8_t *)dev(a[i], at::kByte, n); }
    float *f32_or_null(int i, int64_t *n = nullptr) { return ok && a[i] != Py_None ? f32(i, n) : nullptr; }

    // a contiguous array of the device, of whatever type (or pinned host memory, which the device reads and writes as well)
    void *bytes_or_null(int i, size_t *n)
    {
        *n = 0;
        if (!ok || a[i] == Py_None) return nullptr;
        const at::Tensor *t = tensor(a[i]);
        if (!t) return nullptr;
        if (!t->is_contiguous() || !(t->is_cuda() || t->is_pinned())) {
            fail("a contiguous workspace on the device is expected");
            return nullptr;
        }
        *n = (size_t)t->numel() * t->element_size();
        return t->data_ptr();
    }

    // a device tensor seen as rows: its last dimension is dense, the others are one dimension of evenly spaced rows (a row stride
    // of 0, as expand() makes it, is one)
    bool rows(int i, tt_rows_t *r, int64_t *n, int64_t *N)
    {
        *r = tt_rows_t{nullptr, 0, -1};
        *n = *N = 0;
        const at::Tensor *t = ok ? tensor(a[i]) : nullptr;
        if (!t) return false;
        if (!t->is_cuda()) return fail("a device tensor is expected");
        switch (t->scalar_type()) {
        case at::kFloat: r->type = TT_F32; break;
        case at::kBFloat16: r->type = TT_BF16; break;
        case at::kHalf: r->type = TT_F16; break;
        case at::kFloat8_e4m3fn: r->type = TT_E4M3; break;
        default: return fail("a tensor of 32- or 16-bit floating values (or float8_e4m3fn) is expected");
        }
        const int64_t d = t->dim();
        if (d < 1) return fail("a tensor of rows is expected");
        *N = t->size(d - 1);
        if (*N > 1 && t->stride(d - 1) != 1) return fail("rows must be dense");
        int64_t n_rows = 1, step = 0, next = 0;              // next: the stride that an outer dimension must have
        bool any = false;
        for (int64_t k = d - 2; k >= 0; --k) {
            const int64_t size = t->size(k);
            n_rows *= size;
            if (size <= 1) continue;
            if (!any) step = t->stride(k);
            else if (t->stride(k) != next) return fail("rows must be evenly spaced");
            next = t->stride(k) * size;
            any = true;
        }
        *n = n_rows;
        r->ld = any ? step : *N;
        r->data = n_rows && *N ? t->data_ptr() : nullptr;
        return true;
    }
    // the same, of n rows of N columns, or None: null
    const tt_rows_t *rows_or_null(int i, tt_rows_t *r, int64_t n, int64_t N)
    {
        int64_t rn, rN;
        if (!ok || a[i] == Py_None || !rows(i, r, &rn, &rN)) return nullptr;
        if (rn != n || rN != N) fail("an array has other sizes than the others");
        return r;
    }
    // tokens: contiguous, of 32 or 64 bits
    tt_tokens_t tokens(int i)
    {
        const at::Tensor *t = ok ? tensor(a[i]) : nullptr;
        if (!t) return {};
        const bool wide = t->scalar_type() == at::kLong;
        if (!t->is_cuda() || !(wide || t->scalar_type() == at::kInt) || !t->is_contiguous()) {
            fail("a contiguous device tensor of int64 or int32 tokens is expected");
            return {};
        }
        return {t->numel() ? t->data_ptr() : nullptr, t->numel(), wide ? 64 : 32};
    }
    // None, or (p, state, site)
    const tt_dropout_t *dropout(int i, tt_dropout_t *d)
    {
        if (!ok || a[i] == Py_None) return nullptr;
        if (!PyTuple_Check(a[i]) || PyTuple_GET_SIZE(a[i]) != 3) {
            fail("dropout is (p, state, site)");
            return nullptr;
        }
        int64_t n = 0;
        d->state = (const int64_t *)dev(PyTuple_GET_ITEM(a[i], 1), at::kLong, &n);
        if (!ok) return nullptr;
        if (n < 2) {
            fail("dropout's state is two 64-bit words");
            return nullptr;
        }
        const double p = PyFloat_AsDouble(PyTuple_GET_ITEM(a[i], 0));
        const long long site = PyLong_AsLongLong(PyTuple_GET_ITEM(a[i], 2));
        if (PyErr_Occurred()) {
            ok = false;
            return nullptr;
        }
        if (site < 0 || site > 0xffffffffll) {
            fail("dropout's site has 32 bits");
            return nullptr;
        }
        d->p = (float)p;
        d->site = (uint32_t)site;
        return d;
    }
    // a dense vector of N values of any floating type, or None
    void *vector_or_null(int i, int64_t N, int32_t *type)
    {
        *type = TT_F32;
        if (!ok || a[i] == Py_None) return nullptr;
        tt_rows_t r;
        int64_t n, rN;
        if (!rows(i, &r, &n, &rN)) return nullptr;
        if (n != 1 || rN != N) fail("a vector has another size than the rows");
        *type = r.type;
        return r.data;
    }

    // The arrays of a call live where it is enqueued: a tensor on another device than the current one is refused.
    void here(int i)
    {
        if (!ok || a[i] == Py_None || !THPVariable_Check(a[i])) return;
        const at::Tensor &t = THPVariable_Unpack(a[i]);
        if (t.is_cuda() && t.get_device() != c10::hip::current_device()) fail("a tensor is on another device than the current one");
    }
    // a tensor [..., H, D], its last dimension dense: n rows of H heads of D columns
    const tt_heads_t *heads(int i, tt_heads_t *h, int64_t *n, int64_t *D)
    {
        if (!ok || a[i] == Py_None) return nullptr;
        const at::Tensor *t = tensor(a[i]);
        if (!t) return nullptr;
        *h = tt_heads_t{nullptr, 0, 0, 0, -1};
        if (!t->is_cuda()) return fail("a device tensor is expected"), nullptr;
        switch (t->scalar_type()) {
        case at::kFloat: h->type = TT_F32; break;
        case at::kBFloat16: h->type = TT_BF16; break;
        case at::kHalf: h->type = TT_F16; break;
        default: return fail("a tensor of 32- or 16-bit floating values is expected"), nullptr;
        }
        const int64_t d = t->dim();
        if (d < 2) return fail("a tensor of heads, [..., heads, columns], is expected"), nullptr;
        const int64_t H = t->size(d - 2), cols = t->size(d - 1);
        if (H > INT32_MAX) return fail("too many heads"), nullptr;
        if (cols > 1 && t->stride(d - 1) != 1) return fail("heads must be dense"), nullptr;
        int64_t rows = 1, step = 0, next = 0;
        bool any = false;
        for (int64_t k = d - 3; k >= 0; --k) {
            const int64_t size = t->size(k);
            rows *= size;
            if (size <= 1) continue;
            if (!any) step = t->stride(k);
            else if (t->stride(k) != next) return fail("rows must be evenly spaced"), nullptr;
            next = t->stride(k) * size;
            any = true;
        }
        if (*n >= 0 && (rows != *n || cols != *D)) return fail("an array has other sizes than the others"), nullptr;
        *n = rows;
        *D = cols;
        h->heads = (int32_t)H;
        h->ld = any ? step : H * cols;
        h->ld_head = H > 1 ? t->stride(d - 2) : cols;
        h->data = rows && H && cols ? t->data_ptr() : nullptr;
        return h;
    }
    // None, or (positions, freqs, sections, neighbours)
    const tt_rotation_t *rotation(int i, tt_rotation_t *r, int64_t n)
    {
        if (!ok || a[i] == Py_None) return nullptr;
        if (!PyTuple_Check(a[i]) || PyTuple_GET_SIZE(a[i]) != 4) return fail("rotation is (positions, freqs, sections, neighbours)"), nullptr;
        *r = tt_rotation_t{};
        const at::Tensor *p = tensor(PyTuple_GET_ITEM(a[i], 0)), *f = tensor(PyTuple_GET_ITEM(a[i], 1));
        if (!ok) return nullptr;
        const bool wide = p->scalar_type() == at::kLong;
        if (!p->is_cuda() || !(wide || p->scalar_type() == at::kInt) || p->dim() < 1) return fail("positions are a device tensor of int64 or int32"), nullptr;
        if (!f->is_cuda() || f->scalar_type() != at::kFloat || !f->is_contiguous()) return fail("freqs is a contiguous device tensor of float32"), nullptr;
        if (p->get_device() != c10::hip::current_device() || f->get_device() != c10::hip::current_device()) return fail("a tensor is on another device than the current one"), nullptr;
        // [axes, rows...] or, of one axis, [rows...]; the rows in their order, dense
        PyObject *seq = PySequence_Fast(PyTuple_GET_ITEM(a[i], 2), "sections are whole numbers");
        if (!seq) {
            ok = false;
            return nullptr;
        }
        const Py_ssize_t axes = PySequence_Fast_GET_SIZE(seq);
        if (axes < 1 || axes > 4) fail("rotation has one to four sections");
        for (Py_ssize_t k = 0; ok && k < axes; ++k) {
            const long long v = PyLong_AsLongLong(PySequence_Fast_GET_ITEM(seq, k));
            if (v == -1 && PyErr_Occurred()) ok = false;
            else if (v < 0 || v > INT32_MAX) fail("a section is out of range");
            else r->sections[k] = (int32_t)v;
        }
        Py_DECREF(seq);
        const int neighbours = ok ? PyObject_IsTrue(PyTuple_GET_ITEM(a[i], 3)) : 0;
        if (neighbours < 0) ok = false;
        if (!ok) return nullptr;
        r->axes = (int32_t)axes;
        r->neighbours = neighbours;
        if (f->numel() > INT32_MAX) return fail("too many frequencies"), nullptr;
        r->pairs = (int32_t)f->numel();
        r->bits = wide ? 64 : 32;
        if (p->numel() != axes * n) return fail("positions are [axes, rows]"), nullptr;
        if (axes > 1 && p->size(0) != axes) return fail("positions are [axes, rows]"), nullptr;
        if (p->numel() && (axes > 1 || p->size(0) == 1) && p->dim() > 1) {
            if (!p->select(0, 0).is_contiguous()) return fail("the rows' positions must be dense"), nullptr;
            r->ld_positions = axes > 1 ? p->stride(0) : 0;
        } else if (!p->is_contiguous()) {
            return fail("the rows' positions must be dense"), nullptr;
        } else {
            r->ld_positions = axes > 1 ? n : 0;
        }
        r->positions = p->numel() ? p->data_ptr() : nullptr;
        r->freqs = r->pairs ? (const float *)f->data_ptr() : nullptr;
        return r;
    }

    int64_t integer(int i)
    {
        if (!ok) return 0;
        const long long v = PyLong_AsLongLong(a[i]);
        if (v == -1 && PyErr_Occurred()) ok = false;
        return v;
    }
    float real(int i)
    {
        if (!ok) return 0.f;
        const double v = PyFloat_AsDouble(a[i]);
        if (v == -1.0 && PyErr_Occurred()) ok = false;
        return (float)v;
    }
    bool truth(int i)
    {
        const int v = ok ? PyObject_IsTrue(a[i]) : 0;
        if (v < 0) ok = false;
        return v > 0;
    }

    // offsets[n_bags + 1] or None; longer: a call that takes an array with more entries as well
    const int64_t *offsets(int i, int64_t n_bags, bool longer = false)
    {
        if (!ok || a[i] == Py_None) return nullptr;
        int64_t n = 0;
        const int64_t *p = i64(i, &n);
        if (ok && (longer ? n < n_bags + 1 : n != n_bags + 1)) fail("offsets must have n_bags + 1 entries");
        return p;
    }

    // the struct behind a ctypes structure (which outlives the call)
    const void *structure(PyObject *o, size_t size)
    {
        Py_buffer v;
        if (!ok) return nullptr;
        if (PyObject_GetBuffer(o, &v, PyBUF_SIMPLE) != 0) {
            ok = false;
            return nullptr;
        }
        const void *p = v.buf;
        const bool fits = (size_t)v.len == size;
        PyBuffer_Release(&v);
        if (!fits) {
            PyErr_SetString(PyExc_TypeError, "a structure of another size is expected");
            ok = false;
        }
        return p;
    }
    const tt_shape_t *shape(int i) { return (const tt_shape_t *)structure(a[i], sizeof(tt_shape_t)); }
    const void *member(int i, const char *name, size_t size)
    {
        if (!ok || a[i] == Py_None) return nullptr;
        PyObject *c = PyObject_GetAttrString(a[i], name);
        if (!c) {
            ok = false;
            return nullptr;
        }
        const void *p = structure(c, size);
        Py_DECREF(c);                                        // (its owner still holds it)
        return p;
    }
    const tt_cache_t *cache(int i) { return (const tt_cache_t *)member(i, "c", sizeof(tt_cache_t)); }
    const tt_freq_t *freq(int i) { return (const tt_freq_t *)member(i, "_c", sizeof(tt_freq_t)); }

    // three fp32 tensors; like: the sizes they must have, or null; n: their sizes, or null
    void cores(int i, float *p[3], const int64_t *like = nullptr, int64_t *n = nullptr)
    {
        if (!ok) return;
        PyObject *seq = PySequence_Fast(a[i], "three tensors are expected");
        if (!seq) {
            ok = false;
            return;
        }
        if (PySequence_Fast_GET_SIZE(seq) < 3) fail("three tensors are expected");
        for (int k = 0; ok && k < 3; ++k) {
            int64_t m = 0;
            p[k] = (float *)dev(PySequence_Fast_GET_ITEM(seq, k), at::kFloat, &m);
            if (ok && like && m != like[k]) fail("an array has another size than its core");
            if (n) n[k] = m;
        }
        Py_DECREF(seq);
    }
};

int64_t dim(const tt_shape_t *s) { return (int64_t)s->n[0] * s->n[1] * s->n[2]; }
int64_t t0_floats(const tt_shape_t *s) { return (int64_t)s->n[0] * s->n[1] * s->r[2]; }
void *stream() { return (void *)c10::hip::getCurrentHIPStream().stream(); }

template <typename F>
PyObject *call(F f)
{
    void *st = stream();
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = f(st);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(rc);
}

// shape, cores, indices, offsets, n_bags: the first five arguments of the lookup calls
struct Lookup {
    const tt_shape_t *shape;
    float *cores[3] = {};
    int64_t sizes[3] = {};
    const int64_t *indices, *offsets;
    int64_t L = 0, n_bags;

    explicit Lookup(Args &g, bool longer_offsets = false)
    {
        shape = g.shape(0);
        g.cores(1, cores, nullptr, sizes);
        indices = g.i64(2, &L);
        n_bags = g.integer(4);
        offsets = g.offsets(3, n_bags, longer_offsets);
    }
};

#define TT_FUNCTION(name) PyObject *name(PyObject *, PyObject *const *args, Py_ssize_t nargs)

// no C++ exception may leave a function that Python calls
template <PyObject *(*F)(PyObject *, PyObject *const *, Py_ssize_t)>
TT_FUNCTION(guarded)
{
    try {
        return F(nullptr, args, nargs);
    } catch (const c10::Error &e) {
        PyErr_SetString(PyExc_RuntimeError, e.what_without_backtrace());
    } catch (const std::exception &e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
    }
    return nullptr;
}

// The calling thread may allocate although a stream is captured somewhere: what is enqueued on a stream that is not captured is no
// part of the graph, and by default an allocation of any thread would end the capture.
struct CaptureElsewhere {
    hipStreamCaptureMode mode = hipStreamCaptureModeRelaxed;
    const bool on = hipThreadExchangeStreamCaptureMode(&mode) == hipSuccess;
    ~CaptureElsewhere()
    {
        if (on) (void)hipThreadExchangeStreamCaptureMode(&mode);
    }
};

// Scratch memory of torch's allocator for the current stream (the kernels that use it are enqueued there before it is given
// back), or nothing: while the stream is captured, since a graph's scratch memory has to live as long as the graph, and where
// there is no room for it.
at::DataPtr scratch(size_t bytes, void *st)
{
    const CaptureElsewhere guard;
    hipStreamCaptureStatus status = hipStreamCaptureStatusNone;
    if (!bytes || hipStreamIsCapturing((hipStream_t)st, &status) != hipSuccess || status != hipStreamCaptureStatusNone) return {};
    try {
        return c10::GetAllocator(c10::DeviceType::CUDA)->allocate(bytes);
    } catch (const c10::OutOfMemoryError &) {
        return {};
    }
}

// shape cores indices offsets n_bags output alpha cache workspace
TT_FUNCTION(emb_fwd)
{
    Args g(args, nargs, 9);
    if (!g.ok) return nullptr;
    Lookup q(g);
    int64_t no = 0;
    size_t wsb;
    float *out = g.f32(5, &no);
    const float *alpha = g.f32_or_null(6);
    const tt_cache_t *cache = g.cache(7);
    void *ws = g.bytes_or_null(8, &wsb);
    if (g.ok && no != q.n_bags * dim(q.shape)) g.fail("output has another size");
    if (!g.ok) return nullptr;
    const int64_t cached = cache ? cache->K : 0;
    if (tt_emb_fwd_rows_pays(q.shape, q.L, q.n_bags, cached)) {
        const size_t bytes = tt_emb_fwd_rows_workspace_bytes(q.shape, q.L, q.n_bags);
        const at::DataPtr mem = scratch(bytes, stream());
        if (mem)
            return call([&](void *st) { return tt_emb_fwd_rows(q.shape, q.cores, q.indices, q.L, q.offsets, q.n_bags, alpha, out, mem.get(), bytes, st); });
    }
    return call([&](void *st) { return tt_emb_fwd(q.shape, q.cores, q.indices, q.L, q.offsets, q.n_bags, alpha, cache, out, ws, wsb, st); });
}

// shape cores indices offsets n_bags output alpha workspace
TT_FUNCTION(emb_fwd_rows)
{
    Args g(args, nargs, 8);
    if (!g.ok) return nullptr;
    Lookup q(g);
    int64_t no = 0;
    size_t wsb;
    float *out = g.f32(5, &no);
    const float *alpha = g.f32_or_null(6);
    void *ws = g.bytes_or_null(7, &wsb);
    if (g.ok && no != q.n_bags * dim(q.shape)) g.fail("output has another size");
    if (!g.ok) return nullptr;
    return call([&](void *st) { return tt_emb_fwd_rows(q.shape, q.cores, q.indices, q.L, q.offsets, q.n_bags, alpha, out, ws, wsb, st); });
}

// shape cores indices offsets n_bags output t0 alpha cache
TT_FUNCTION(emb_fwd_keep_t0)
{
    Args g(args, nargs, 9);
    if (!g.ok) return nullptr;
    Lookup q(g);
    int64_t nt = 0;
    float *out = g.f32(5), *t0 = g.f32(6, &nt);
    const float *alpha = g.f32_or_null(7);
    const tt_cache_t *cache = g.cache(8);
    if (g.ok && nt < q.L * t0_floats(q.shape)) g.fail("t0 is too small");
    if (!g.ok) return nullptr;
    return call([&](void *st) { return tt_emb_fwd_keep_t0(q.shape, q.cores, q.indices, q.L, q.offsets, q.n_bags, alpha, cache, out, t0, st); });
}

// shape cores indices offsets n_bags output workspace t0 alpha cache
TT_FUNCTION(emb_fwd_prepared)
{
    Args g(args, nargs, 10);
    if (!g.ok) return nullptr;
    Lookup q(g);
    int64_t no = 0, nt = 0, wsb = 0;
    float *out = g.f32(5, &no);
    uint8_t *ws = g.u8(6, &wsb);
    float *t0 = g.f32_or_null(7, &nt);
    const float *alpha = g.f32_or_null(8);
    const tt_cache_t *cache = g.cache(9);
    if (g.ok && t0 && nt < q.L * t0_floats(q.shape)) g.fail("t0 is too small");
    if (g.ok && no != q.n_bags * dim(q.shape)) g.fail("output has another size");
    if (!g.ok) return nullptr;
    return call([&](void *st) {
        return tt_emb_fwd_prepared(q.shape, q.cores, q.indices, q.L, q.offsets, q.n_bags, alpha, cache, out, t0, ws, (size_t)wsb, st);
    });
}

// shape cores indices offsets n_bags grad_output grad_cores alpha cache grad_cache workspace t0
TT_FUNCTION(emb_bwd)
{
    Args g(args, nargs, 12);
    if (!g.ok) return nullptr;
    Lookup q(g);
    size_t wsb;
    float *grads[3] = {};
    const float *go = g.f32(5);
    g.cores(6, grads, q.sizes);
    const float *alpha = g.f32_or_null(7);
    const tt_cache_t *cache = g.cache(8);
    float *gc = g.f32_or_null(9);
    void *ws = g.bytes_or_null(10, &wsb);
    const float *t0 = g.f32_or_null(11);
    const bool with_t0 = args[11] != Py_None;
    if (!g.ok) return nullptr;
    return call([&](void *st) {
        return with_t0 ? tt_emb_bwd_t0(q.shape, q.cores, q.indices, q.L, q.offsets, q.n_bags, alpha, cache, go, t0, grads, gc, ws, wsb, st)
                       : tt_emb_bwd(q.shape, q.cores, q.indices, q.L, q.offsets, q.n_bags, alpha, cache, go, grads, gc, ws, wsb, st);
    });
}

// shape indices offsets n_bags cache workspace kept_t0
TT_FUNCTION(emb_bwd_prepare)
{
    Args g(args, nargs, 7);
    if (!g.ok) return nullptr;
    int64_t L = 0;
    size_t wsb;
    const tt_shape_t *shape = g.shape(0);
    const int64_t *indices = g.i64(1, &L);
    const int64_t n_bags = g.integer(3);
    const int64_t *offsets = g.offsets(2, n_bags, true);
    const tt_cache_t *cache = g.cache(4);
    void *ws = g.bytes_or_null(5, &wsb);
    const bool kept = g.truth(6);
    if (!g.ok) return nullptr;
    return call([&](void *st) { return tt_emb_bwd_prepare(shape, indices, L, offsets, n_bags, cache, kept ? 1 : 0, ws, wsb, st); });
}

// shape cores cores_out indices offsets n_bags grad_output lr alpha cache workspace t0 prepared
TT_FUNCTION(emb_bwd_sgd)
{
    Args g(args, nargs, 13);
    if (!g.ok) return nullptr;
    int64_t L = 0, sizes[3];
    size_t wsb;
    float *cores[3] = {}, *outs[3] = {};
    const tt_shape_t *shape = g.shape(0);
    g.cores(1, cores, nullptr, sizes);
    g.cores(2, outs, sizes);
    const int64_t *indices = g.i64(3, &L);
    const int64_t n_bags = g.integer(5);
    const int64_t *offsets = g.offsets(4, n_bags);
    const float *go = g.f32(6);
    const float lr = g.real(7);
    const float *alpha = g.f32_or_null(8);
    const tt_cache_t *cache = g.cache(9);
    void *ws = g.bytes_or_null(10, &wsb);
    const float *t0 = g.f32_or_null(11);
    const bool with_t0 = args[11] != Py_None, prepared = g.truth(12);
    if (!g.ok) return nullptr;
    return call([&](void *st) {
        if (prepared) return tt_emb_bwd_sgd_prepared(shape, cores, outs, indices, L, offsets, n_bags, alpha, cache, go, t0, lr, ws, wsb, st);
        if (with_t0) return tt_emb_bwd_sgd_t0(shape, cores, outs, indices, L, offsets, n_bags, alpha, cache, go, t0, lr, ws, wsb, st);
        return tt_emb_bwd_sgd(shape, cores, outs, indices, L, offsets, n_bags, alpha, cache, go, lr, ws, wsb, st);
    });
}

// shape indices kept cache
TT_FUNCTION(emb_kept_prepare)
{
    Args g(args, nargs, 4);
    if (!g.ok) return nullptr;
    int64_t L = 0, kb = 0;
    const tt_shape_t *shape = g.shape(0);
    const int64_t *indices = g.i64(1, &L);
    uint8_t *kept = g.u8(2, &kb);
    const tt_cache_t *cache = g.cache(3);
    if (!g.ok) return nullptr;
    return call([&](void *st) { return tt_emb_kept_prepare(shape, indices, L, cache, kept, (size_t)kb, st); });
}

// shape cores indices offsets n_bags output kept alpha cache lists_ready
TT_FUNCTION(emb_fwd_keep)
{
    Args g(args, nargs, 10);
    if (!g.ok) return nullptr;
    Lookup q(g);
    int64_t kb = 0;
    float *out = g.f32(5);
    uint8_t *kept = g.u8(6, &kb);
    const float *alpha = g.f32_or_null(7);
    const tt_cache_t *cache = g.cache(8);
    const bool ready = g.truth(9);
    if (!g.ok) return nullptr;
    return call([&](void *st) {
        return tt_emb_fwd_keep(q.shape, q.cores, q.indices, q.L, q.offsets, q.n_bags, alpha, cache, out, kept, (size_t)kb, ready ? 1 : 0, st);
    });
}

// the (indices, kept) pair of the next batch, or None
const tt_next_batch_t *next_batch(Args &g, int i, tt_next_batch_t *nb)
{
    if (!g.ok || g.a[i] == Py_None) return nullptr;
    PyObject *seq = PySequence_Fast(g.a[i], "next_batch is a pair (indices, kept)");
    if (!seq) {
        g.ok = false;
        return nullptr;
    }
    if (PySequence_Fast_GET_SIZE(seq) != 2) {
        g.fail("next_batch is a pair (indices, kept)");
    } else {
        int64_t kb = 0;
        nb->indices = (const int64_t *)g.dev(PySequence_Fast_GET_ITEM(seq, 0), at::kLong, &nb->L);
        nb->kept = g.dev(PySequence_Fast_GET_ITEM(seq, 1), at::kByte, &kb);
        nb->kept_bytes = (size_t)kb;
    }
    Py_DECREF(seq);
    return g.ok ? nb : nullptr;
}

// shape cores indices offsets n_bags grad_output kept grad_cores alpha cache grad_cache workspace next_batch
TT_FUNCTION(emb_bwd_kept)
{
    Args g(args, nargs, 13);
    if (!g.ok) return nullptr;
    Lookup q(g, true);
    int64_t kb = 0;
    size_t wsb;
    float *grads[3] = {};
    tt_next_batch_t nb{};
    const float *go = g.f32(5);
    const uint8_t *kept = g.u8(6, &kb);
    g.cores(7, grads);
    const float *alpha = g.f32_or_null(8);
    const tt_cache_t *cache = g.cache(9);
    float *gc = g.f32_or_null(10);
    void *ws = g.bytes_or_null(11, &wsb);
    const tt_next_batch_t *next = next_batch(g, 12, &nb);
    if (!g.ok) return nullptr;
    return call([&](void *st) {
        return tt_emb_bwd_kept(q.shape, q.cores, q.indices, q.L, q.offsets, q.n_bags, alpha, cache, go, kept, (size_t)kb, grads, gc, next, ws, wsb, st);
    });
}

// shape cores cores_out indices offsets n_bags grad_output kept lr alpha cache workspace next_batch
TT_FUNCTION(emb_bwd_sgd_kept)
{
    Args g(args, nargs, 13);
    if (!g.ok) return nullptr;
    int64_t L = 0, kb = 0, sizes[3];
    size_t wsb;
    float *cores[3] = {}, *outs[3] = {};
    tt_next_batch_t nb{};
    const tt_shape_t *shape = g.shape(0);
    g.cores(1, cores, nullptr, sizes);
    g.cores(2, outs, sizes);
    const int64_t *indices = g.i64(3, &L);
    const int64_t n_bags = g.integer(5);
    const int64_t *offsets = g.offsets(4, n_bags, true);
    const float *go = g.f32(6);
    const uint8_t *kept = g.u8(7, &kb);
    const float lr = g.real(8);
    const float *alpha = g.f32_or_null(9);
    const tt_cache_t *cache = g.cache(10);
    void *ws = g.bytes_or_null(11, &wsb);
    const tt_next_batch_t *next = next_batch(g, 12, &nb);
    if (!g.ok) return nullptr;
    return call([&](void *st) {
        return tt_emb_bwd_sgd_kept(shape, cores, outs, indices, L, offsets, n_bags, alpha, cache, go, kept, (size_t)kb, lr, next, ws, wsb, st);
    });
}

// shape cores cores_out indices offsets n_bags grad_output lr alpha cache
TT_FUNCTION(emb_bwd_sgd_static)
{
    Args g(args, nargs, 10);
    if (!g.ok) return nullptr;
    int64_t L = 0, sizes[3];
    float *cores[3] = {}, *outs[3] = {};
    const tt_shape_t *shape = g.shape(0);
    g.cores(1, cores, nullptr, sizes);
    g.cores(2, outs, sizes);
    const int64_t *indices = g.i64(3, &L);
    const int64_t n_bags = g.integer(5);
    const int64_t *offsets = g.offsets(4, n_bags);
    const float *go = g.f32(6);
    const float lr = g.real(7);
    const float *alpha = g.f32_or_null(8);
    const tt_cache_t *cache = g.cache(9);
    if (!g.ok) return nullptr;
    return call([&](void *st) { return tt_emb_bwd_sgd_static(shape, cores, outs, indices, L, offsets, n_bags, alpha, cache, go, lr, st); });
}

// shape cores grad_cores lr cache grad_cache zero_grad
TT_FUNCTION(emb_sgd_update)
{
    Args g(args, nargs, 7);
    if (!g.ok) return nullptr;
    float *cores[3] = {}, *grads[3] = {};
    const tt_shape_t *shape = g.shape(0);
    g.cores(1, cores);
    g.cores(2, grads);
    const float lr = g.real(3);
    const tt_cache_t *cache = g.cache(4);
    float *gc = g.f32_or_null(5);
    const bool zero = g.truth(6);
    if (!g.ok) return nullptr;
    return call([&](void *st) { return tt_emb_sgd_update(shape, cores, grads, lr, cache, gc, zero ? 1 : 0, st); });
}

// shape cores cand_rows cand_counts cache workspace
template <int (*F)(const tt_shape_t *, const float *const *, const int64_t *, const int64_t *, int64_t, const tt_cache_t *, void *, size_t, void *)>
TT_FUNCTION(cache_fill)
{
    Args g(args, nargs, 6);
    if (!g.ok) return nullptr;
    float *cores[3] = {};
    int64_t n = 0, m = 0;
    size_t wsb;
    const tt_shape_t *shape = g.shape(0);
    g.cores(1, cores);
    const int64_t *rows = g.i64(2, &n), *counts = g.i64(3, &m);
    const tt_cache_t *cache = g.cache(4);
    void *ws = g.bytes_or_null(5, &wsb);
    if (g.ok && n != m) g.fail("as many counts as rows are expected");
    if (!g.ok) return nullptr;
    return call([&](void *st) { return F(shape, cores, rows, counts, n, cache, ws, wsb, st); });
}

// tracker indices
TT_FUNCTION(freq_update)
{
    Args g(args, nargs, 2);
    if (!g.ok) return nullptr;
    int64_t L = 0;
    const tt_freq_t *f = g.freq(0);
    const int64_t *indices = g.i64(1, &L);
    if (!g.ok) return nullptr;
    return call([&](void *st) { return tt_freq_update(f, indices, L, st); });
}

// tracker rows counts n_out
TT_FUNCTION(freq_export)
{
    Args g(args, nargs, 4);
    if (!g.ok) return nullptr;
    int64_t nr = 0, nc = 0;
    const tt_freq_t *f = g.freq(0);
    int64_t *rows = g.i64(1, &nr), *counts = g.i64(2, &nc), *n_out = g.i64(3);
    if (g.ok && (nr < f->capacity || nc < f->capacity)) g.fail("rows and counts need room for the whole table");
    if (!g.ok) return nullptr;
    return call([&](void *st) { return tt_freq_export(f, rows, counts, n_out, st); });
}

// table tokens output scale dropout
TT_FUNCTION(token_fwd)
{
    Args g(args, nargs, 5);
    if (!g.ok) return nullptr;
    tt_rows_t table, out;
    tt_dropout_t d;
    int64_t num_rows, N, L, M;
    g.rows(0, &table, &num_rows, &N);
    const tt_tokens_t tokens = g.tokens(1);
    g.rows(2, &out, &L, &M);
    const float scale = g.real(3);
    const tt_dropout_t *drop = g.dropout(4, &d);
    if (g.ok && (L != tokens.L || M != N)) g.fail("output has another size");
    if (!g.ok) return nullptr;
    return call([&](void *st) { return tt_token_fwd(&table, num_rows, N, &tokens, scale, drop, &out, st); });
}

// tokens grad_output table scale dropout workspace f(...)
template <typename F>
PyObject *token_grad(Args &g, F f)
{
    tt_rows_t go, table;
    tt_dropout_t d;
    int64_t L, M, num_rows, N;
    size_t wsb;
    const tt_tokens_t tokens = g.tokens(0);
    g.rows(1, &go, &L, &M);
    g.rows(2, &table, &num_rows, &N);
    const float scale = g.real(3);
    const tt_dropout_t *drop = g.dropout(4, &d);
    void *ws = g.bytes_or_null(5, &wsb);
    if (g.ok && (L != tokens.L || M != N)) g.fail("grad_output has another size");
    if (!g.ok) return nullptr;
    at::DataPtr mem;
    if (!ws) {
        wsb = tt_token_bwd_workspace_bytes(L, num_rows, N);
        mem = scratch(wsb, stream());
        if (!mem) wsb = 0;
        ws = mem.get();
    }
    return call([&](void *st) { return f(&tokens, &go, scale, drop, &table, num_rows, N, ws, wsb, st); });
}

// tokens grad_output grad_table scale dropout workspace accumulate
TT_FUNCTION(token_bwd)
{
    Args g(args, nargs, 7);
    if (!g.ok) return nullptr;
    const bool add = g.truth(6);
    if (!g.ok) return nullptr;
    return token_grad(g, [&](auto t, auto go, float scale, auto drop, auto table, int64_t rows, int64_t N, void *ws, size_t wsb, void *st) {
        return tt_token_bwd(t, go, scale, drop, table, rows, N, add ? 1 : 0, ws, wsb, st);
    });
}

// tokens grad_output table scale dropout workspace lr
TT_FUNCTION(token_bwd_sgd)
{
    Args g(args, nargs, 7);
    if (!g.ok) return nullptr;
    const float lr = g.real(6);
    if (!g.ok) return nullptr;
    return token_grad(g, [&](auto t, auto go, float scale, auto drop, auto table, int64_t rows, int64_t N, void *ws, size_t wsb, void *st) {
        return tt_token_bwd_sgd(t, go, scale, drop, table, rows, N, lr, ws, wsb, st);
    });
}

// x output dropout residual
TT_FUNCTION(dropout_fwd)
{
    Args g(args, nargs, 4);
    if (!g.ok) return nullptr;
    tt_rows_t x, out, r;
    tt_dropout_t d;
    int64_t n, N;
    g.rows(0, &x, &n, &N);
    const tt_rows_t *o = g.rows_or_null(1, &out, n, N);
    const tt_dropout_t *drop = g.dropout(2, &d);
    const tt_rows_t *res = g.rows_or_null(3, &r, n, N);
    if (!g.ok) return nullptr;
    return call([&](void *st) { return tt_dropout_fwd(&x, res, drop, o, n, N, st); });
}

// grad_output grad_x dropout
TT_FUNCTION(dropout_bwd)
{
    Args g(args, nargs, 3);
    if (!g.ok) return nullptr;
    tt_rows_t go, gx;
    tt_dropout_t d;
    int64_t n, N;
    g.rows(0, &go, &n, &N);
    const tt_rows_t *x = g.rows_or_null(1, &gx, n, N);
    const tt_dropout_t *drop = g.dropout(2, &d);
    if (!g.ok) return nullptr;
    return call([&](void *st) { return tt_dropout_bwd(&go, drop, x, n, N, st); });
}

// x weight output residual sum rstd scales group eps dropout
TT_FUNCTION(add_rms_norm_fwd)
{
    Args g(args, nargs, 10);
    if (!g.ok) return nullptr;
    tt_rows_t x, out, res, sum, sc;
    tt_dropout_t d;
    int64_t n, N, nr = 0;
    int32_t wt;
    g.rows(0, &x, &n, &N);
    const void *w = g.vector_or_null(1, N, &wt);
    const tt_rows_t *o = g.rows_or_null(2, &out, n, N), *r = g.rows_or_null(3, &res, n, N), *s = g.rows_or_null(4, &sum, n, N);
    float *rstd = g.f32_or_null(5, &nr);
    const int64_t group = g.integer(7);
    const tt_rows_t *scales = g.rows_or_null(6, &sc, n, group > 0 ? (N + group - 1) / group : 1);
    const float eps = g.real(8);
    const tt_dropout_t *drop = g.dropout(9, &d);
    if (g.ok && args[5] != Py_None && nr != n) g.fail("rstd has another size");
    if (g.ok && (group < 0 || group > 128)) g.fail("group is 0, 32, 64 or 128");
    if (!g.ok) return nullptr;
    return call([&](void *st) { return tt_add_rms_norm_fwd(&x, r, drop, w, wt, eps, s, o, rstd, scales, (int32_t)group, n, N, st); });
}

// grad_output h rstd weight grad_x grad_weight grad_sum grad_residual dropout accumulate workspace
TT_FUNCTION(add_rms_norm_bwd)
{
    Args g(args, nargs, 11);
    if (!g.ok) return nullptr;
    tt_rows_t go, h, gx, gs, gr;
    tt_dropout_t d;
    int64_t n, N, nr = 0;
    int32_t wt, gwt;
    size_t wsb;
    g.rows(0, &go, &n, &N);
    const tt_rows_t *hp = g.rows_or_null(1, &h, n, N);
    const float *rstd = g.f32(2, &nr);
    const void *w = g.vector_or_null(3, N, &wt);
    const tt_rows_t *x = g.rows_or_null(4, &gx, n, N);
    void *gw = g.vector_or_null(5, N, &gwt);
    const tt_rows_t *s = g.rows_or_null(6, &gs, n, N), *r = g.rows_or_null(7, &gr, n, N);
    const tt_dropout_t *drop = g.dropout(8, &d);
    const bool add = g.truth(9);
    void *ws = g.bytes_or_null(10, &wsb);
    if (g.ok && nr != n) g.fail("rstd has another size");
    if (!g.ok) return nullptr;
    at::DataPtr mem;
    if (!ws && gw) {
        wsb = tt_add_rms_norm_bwd_workspace_bytes(n, N);
        mem = scratch(wsb, stream());
        if (!mem) wsb = 0;
        ws = mem.get();
    }
    return call([&](void *st) { return tt_add_rms_norm_bwd(&go, hp, rstd, w, wt, s, drop, x, r, gw, gwt, add ? 1 : 0, n, N, ws, wsb, st); });
}

// the workspace that is given, or scratch memory
struct Room {
    at::DataPtr mem;
    void *data;
    size_t bytes;

    Room(void *ws, size_t given, size_t need) : data(ws), bytes(given)
    {
        if (ws) return;
        mem = scratch(need, stream());
        bytes = mem ? need : 0;
        data = mem.get();
    }
};

// what the products load as it lies
static int whole_chunks(int64_t columns, std::initializer_list<const tt_rows_t *> arrays)
{
    int64_t odd = columns;
    for (const tt_rows_t *r : arrays)
        if (r) odd |= r->ld | (int64_t)((uintptr_t)r->data / 2) | (r->ld > (1 << 22));
    return odd % 8 == 0;
}

// x weight output bias activation residual pre workspace
TT_FUNCTION(linear_fwd)
{
    Args g(args, nargs, 8);
    if (!g.ok) return nullptr;
    tt_rows_t x, w, out, res, pre;
    int64_t n, K, N, Kw;
    int32_t bt;
    size_t wsb;
    g.rows(0, &x, &n, &K);
    g.rows(1, &w, &N, &Kw);
    if (g.ok && Kw != K) g.fail("weight has another number of columns than x");
    const tt_rows_t *o = g.rows_or_null(2, &out, n, N), *r = g.rows_or_null(5, &res, n, N), *p = g.rows_or_null(6, &pre, n, N);
    const void *b = g.vector_or_null(3, N, &bt);
    const int64_t act = g.integer(4);
    void *ws = g.bytes_or_null(7, &wsb);
    for (int i : {0, 1, 2, 3, 5, 6, 7}) g.here(i);
    if (!g.ok) return nullptr;
    const Room room(ws, wsb, tt_linear_fwd_workspace_bytes(n, K, N, x.type, whole_chunks(K, {&x, &w})));
    return call([&](void *st) { return tt_linear_fwd(&x, &w, b, bt, (int32_t)act, r, p, o, n, K, N, room.data, room.bytes, st); });
}

// grad_output x weight pre activation grad_x grad_weight grad_bias accumulate workspace
TT_FUNCTION(linear_bwd)
{
    Args g(args, nargs, 10);
    if (!g.ok) return nullptr;
    tt_rows_t go, xs, ws_, pre, gxs, gws;
    int64_t n, N, K = -1;
    int32_t bt;
    size_t wsb;
    g.rows(0, &go, &n, &N);
    // K is the columns of whichever array of rows is there
    auto matrix = [&](int i, tt_rows_t *r, int64_t rows) -> const tt_rows_t * {
        int64_t m, cols;
        if (!g.ok || args[i] == Py_None || !g.rows(i, r, &m, &cols)) return nullptr;
        if (m != rows || (K >= 0 && cols != K)) g.fail("an array has other sizes than the others");
        K = cols;
        return r;
    };
    const tt_rows_t *x = matrix(1, &xs, n), *w = matrix(2, &ws_, N), *gx = matrix(5, &gxs, n), *gw = matrix(6, &gws, N);
    const tt_rows_t *p = g.rows_or_null(3, &pre, n, N);
    const int64_t act = g.integer(4);
    void *gb = g.vector_or_null(7, N, &bt);
    const bool add = g.truth(8);
    void *ws = g.bytes_or_null(9, &wsb);
    for (int i : {0, 1, 2, 3, 5, 6, 7, 9}) g.here(i);
    if (!g.ok) return nullptr;
    if (K < 0) K = 0;
    const Room room(ws, wsb, tt_linear_bwd_workspace_bytes(n, K, N, go.type, (int32_t)act, whole_chunks(K | N, {&go, x, w})));
    return call([&](void *st) { return tt_linear_bwd(&go, x, w, p, (int32_t)act, gx, gw, gb, bt, add ? 1 : 0, n, K, N, room.data, room.bytes, st); });
}

// q k q_output k_output rotation norm q_weight k_weight eps
TT_FUNCTION(qk_norm_rotate_fwd)
{
    Args g(args, nargs, 9);
    if (!g.ok) return nullptr;
    tt_heads_t q, k, qo, ko;
    tt_rotation_t rot;
    int64_t n = -1, D = -1;
    int32_t qt, kt;
    const tt_heads_t *pq = g.heads(0, &q, &n, &D), *pk = g.heads(1, &k, &n, &D), *pqo = g.heads(2, &qo, &n, &D), *pko = g.heads(3, &ko, &n, &D);
    const tt_rotation_t *r = g.rotation(4, &rot, n);
    const bool norm = g.truth(5);
    const void *qw = g.vector_or_null(6, D, &qt), *kw = g.vector_or_null(7, D, &kt);
    const float eps = g.real(8);
    for (int i : {0, 1, 2, 3, 6, 7}) g.here(i);
    if (!g.ok) return nullptr;
    return call([&](void *st) { return tt_qk_norm_rotate_fwd(pq, pk, r, norm ? 1 : 0, eps, qw, qt, kw, kt, pqo, pko, n, D, st); });
}

// grad_q_output grad_k_output q k grad_q grad_k rotation norm q_weight k_weight grad_q_weight grad_k_weight eps accumulate workspace
TT_FUNCTION(qk_norm_rotate_bwd)
{
    Args g(args, nargs, 15);
    if (!g.ok) return nullptr;
    tt_heads_t gqo, gko, q, k, gq, gk;
    tt_rotation_t rot;
    int64_t n = -1, D = -1;
    int32_t qt, kt, gqt, gkt;
    size_t wsb;
    const tt_heads_t *pgqo = g.heads(0, &gqo, &n, &D), *pgko = g.heads(1, &gko, &n, &D), *pq = g.heads(2, &q, &n, &D), *pk = g.heads(3, &k, &n, &D), *pgq = g.heads(4, &gq, &n, &D),
                     *pgk = g.heads(5, &gk, &n, &D);
    const tt_rotation_t *r = g.rotation(6, &rot, n);
    const bool norm = g.truth(7);
    const void *qw = g.vector_or_null(8, D, &qt), *kw = g.vector_or_null(9, D, &kt);
    void *gqw = g.vector_or_null(10, D, &gqt), *gkw = g.vector_or_null(11, D, &gkt);
    const float eps = g.real(12);
    const bool add = g.truth(13);
    void *ws = g.bytes_or_null(14, &wsb);
    for (int i : {0, 1, 2, 3, 4, 5, 8, 9, 10, 11, 14}) g.here(i);
    if (!g.ok) return nullptr;
    const Room room(ws, wsb, gqw || gkw ? tt_qk_norm_rotate_bwd_workspace_bytes(n, pgqo ? gqo.heads : 0, pgko ? gko.heads : 0, D) : 0);
    return call([&](void *st) {
        return tt_qk_norm_rotate_bwd(pgqo, pgko, pq, pk, r, norm ? 1 : 0, eps, qw, qt, kw, kt, pgq, pgk, gqw, gqt, gkw, gkt, add ? 1 : 0, n, D, room.data, room.bytes, st);
    });
}

// logits tokens logprob lse entropy top_ids top_logprobs scale workspace
TT_FUNCTION(token_logprob_fwd)
{
    Args g(args, nargs, 9);
    if (!g.ok) return nullptr;
    tt_rows_t logits;
    int64_t n, V, nl = 0, ns = 0, ne = 0, ni = 0, nt = 0, k = 0;
    size_t wsb;
    g.rows(0, &logits, &n, &V);
    tt_tokens_t t{};
    if (args[1] != Py_None) t = g.tokens(1);
    float *logprob = g.f32_or_null(2, &nl), *lse = g.f32_or_null(3, &ns), *entropy = g.f32_or_null(4, &ne);
    tt_tokens_t ids{};
    if (args[5] != Py_None) {
        ids = g.tokens(5);
        if (g.ok) {
            const at::Tensor &x = THPVariable_Unpack(args[5]);
            k = x.dim() ? x.size(x.dim() - 1) : 0;
            ni = ids.L;
        }
    }
    float *top = g.f32_or_null(6, &nt);
    const float scale = g.real(7);
    void *ws = g.bytes_or_null(8, &wsb);
    for (int i : {0, 1, 2, 3, 4, 5, 6, 8}) g.here(i);
    if (g.ok && ((args[2] != Py_None && nl != n) || (args[3] != Py_None && ns != n) || (args[4] != Py_None && ne != n))) g.fail("logprob, lse and entropy have one value per row");
    if (g.ok && (k > 64 || ni != n * k || (args[6] != Py_None && nt != ni))) g.fail("top_ids and top_logprobs are [rows, k], k up to 64");
    if (!g.ok) return nullptr;
    const Room room(ws, wsb, tt_token_logprob_fwd_workspace_bytes(n, V, (int32_t)k));
    return call([&](void *st) {
        return tt_token_logprob_fwd(&logits, args[1] != Py_None ? &t : nullptr, scale, logprob, lse, entropy, (int32_t)k, const_cast<void *>(ids.data), ids.bits, top, n, V, room.data, room.bytes, st);
    });
}

// logits tokens lse entropy grad_logprob grad_entropy grad_logits scale
TT_FUNCTION(token_logprob_bwd)
{
    Args g(args, nargs, 8);
    if (!g.ok) return nullptr;
    tt_rows_t logits, out;
    int64_t n, V, nl = 0, ne = 0, ng = 0, nh = 0;
    g.rows(0, &logits, &n, &V);
    tt_tokens_t t{};
    if (args[1] != Py_None) t = g.tokens(1);
    const float *lse = g.f32(2, &nl), *entropy = g.f32_or_null(3, &ne), *gl = g.f32_or_null(4, &ng), *ge = g.f32_or_null(5, &nh);
    const tt_rows_t *o = g.rows_or_null(6, &out, n, V);
    const float scale = g.real(7);
    for (int i = 0; i < 7; ++i) g.here(i);
    if (g.ok && (nl != n || (args[3] != Py_None && ne != n) || (args[4] != Py_None && ng != n) || (args[5] != Py_None && nh != n))) g.fail("lse, entropy and their gradients have one value per row");
    if (!g.ok) return nullptr;
    return call([&](void *st) { return tt_token_logprob_bwd(&logits, args[1] != Py_None ? &t : nullptr, scale, lse, entropy, gl, ge, o, n, V, st); });
}

#define TT_METHOD(name, function) {name, (PyCFunction)(void (*)(void))guarded<function>, METH_FASTCALL, nullptr}

PyMethodDef methods[] = {
    TT_METHOD("emb_fwd", emb_fwd),
    TT_METHOD("emb_fwd_rows", emb_fwd_rows),
    TT_METHOD("emb_fwd_keep_t0", emb_fwd_keep_t0),
    TT_METHOD("emb_fwd_prepared", emb_fwd_prepared),
    TT_METHOD("emb_bwd", emb_bwd),
    TT_METHOD("emb_bwd_prepare", emb_bwd_prepare),
    TT_METHOD("emb_bwd_sgd", emb_bwd_sgd),
    TT_METHOD("emb_kept_prepare", emb_kept_prepare),
    TT_METHOD("emb_fwd_keep", emb_fwd_keep),
    TT_METHOD("emb_bwd_kept", emb_bwd_kept),
    TT_METHOD("emb_bwd_sgd_kept", emb_bwd_sgd_kept),
    TT_METHOD("emb_bwd_sgd_static", emb_bwd_sgd_static),
    TT_METHOD("emb_sgd_update", emb_sgd_update),
    TT_METHOD("freq_update", freq_update),
    TT_METHOD("freq_export", freq_export),
    TT_METHOD("token_fwd", token_fwd),
    TT_METHOD("token_bwd", token_bwd),
    TT_METHOD("token_bwd_sgd", token_bwd_sgd),
    TT_METHOD("dropout_fwd", dropout_fwd),
    TT_METHOD("dropout_bwd", dropout_bwd),
    TT_METHOD("add_rms_norm_fwd", add_rms_norm_fwd),
    TT_METHOD("add_rms_norm_bwd", add_rms_norm_bwd),
    TT_METHOD("linear_fwd", linear_fwd),
    TT_METHOD("linear_bwd", linear_bwd),
    TT_METHOD("qk_norm_rotate_fwd", qk_norm_rotate_fwd),
    TT_METHOD("qk_norm_rotate_bwd", qk_norm_rotate_bwd),
    TT_METHOD("token_logprob_fwd", token_logprob_fwd),
    TT_METHOD("token_logprob_bwd", token_logprob_bwd),
    TT_METHOD("cache_build", cache_fill<tt_cache_build>),
    TT_METHOD("cache_refill", cache_fill<tt_cache_refill>),
    {nullptr, nullptr, 0, nullptr}};

PyModuleDef module = {PyModuleDef_HEAD_INIT, "_tt_call", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__tt_call(void) { return PyModule_Create(&module); }
