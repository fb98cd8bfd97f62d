// The calls that a training step makes, as functions of a Python extension: tensors in, the C ABI's status out.
//
// A small layer's call takes less time on the GPU than its arguments took on their way through Python and ctypes
// (checks, addresses and conversions of up to 18 arguments: 4 to 5 us of a call); here they take 0.5 us.
// Argument checks are those of the binding: every tensor contiguous and on the GPU, None stands for NULL.  The
// interpreter lock is given back while the library launches, as ctypes does.
#include <exception>
#include <initializer_list>
#include <sstream>

#include <torch/csrc/autograd/python_variable.h>

#include "falqon.h"

namespace {

// Arguments of one call, read in order.  After a failed read (Python error set) the others return nothing.
class Args {
public:
    Args(PyObject* const* args, Py_ssize_t count, Py_ssize_t want) : args_(args)
    {
        if (count != want) {
            PyErr_Format(PyExc_TypeError, "%zd arguments, %zd expected", count, want);
            failed_ = true;
        }
    }
    bool failed() const { return failed_; }

    const at::Tensor* tensor()                                       // null for None
    {
        if (failed_) return nullptr;
        PyObject* const o = args_[next_++];
        if (o == Py_None) return nullptr;
        if (!THPVariable_Check(o)) return fail(PyExc_TypeError, "a tensor or None expected");
        const at::Tensor& t = THPVariable_Unpack(o);
        if (!t.is_cuda() || !t.is_contiguous()) return fail(PyExc_ValueError, "tensors must be contiguous GPU tensors");
        return &t;
    }
    const at::Tensor* matrix(bool longer = false)                    // its shape is asked for; longer: the first two dimensions of it
    {
        const at::Tensor* const t = tensor();
        if (failed_) return nullptr;
        if (!t) return fail(PyExc_AttributeError, "'NoneType' object has no attribute 'shape'");
        if (longer ? t->dim() < 2 : t->dim() != 2) return fail(PyExc_ValueError, "a tensor of two dimensions expected");
        return t;
    }
    const at::Tensor* rows()                                         // a matrix whose rows may lie apart (a view of a wider one)
    {
        if (failed_) return nullptr;
        PyObject* const o = args_[next_++];
        if (o == Py_None) return nullptr;
        if (!THPVariable_Check(o)) return fail(PyExc_TypeError, "a tensor or None expected");
        const at::Tensor& t = THPVariable_Unpack(o);
        if (!t.is_cuda() || t.dim() != 2 || (t.size(1) > 1 && t.stride(1) != 1)) return fail(PyExc_ValueError, "a GPU tensor of two dimensions with unit stride along its rows expected");
        return &t;
    }
    // t, where it is given, has this type and shape
    void expect(const at::Tensor* t, at::ScalarType type, std::initializer_list<int64_t> shape, const char* name)
    {
        if (failed_ || !t) return;
        if (t->scalar_type() == type && t->sizes() == at::IntArrayRef(shape)) return;
        std::ostringstream want;
        want << name << ": " << c10::toString(type) << " " << at::IntArrayRef(shape) << " expected, got " << c10::toString(t->scalar_type()) << " " << t->sizes();
        fail(PyExc_ValueError, want.str().c_str());
    }
    void need(const at::Tensor* t, const char* name)
    {
        if (!failed_ && !t) {
            PyErr_Format(PyExc_ValueError, "%s is needed", name);
            failed_ = true;
        }
    }
    int64_t integer()
    {
        if (failed_) return 0;
        const long long v = PyLong_AsLongLong(args_[next_++]);
        if (v == -1 && PyErr_Occurred()) failed_ = true;
        return v;
    }
    double real()
    {
        if (failed_) return 0.0;
        const double v = PyFloat_AsDouble(args_[next_++]);
        if (v == -1.0 && PyErr_Occurred()) failed_ = true;
        return v;
    }
    void* address() { return reinterpret_cast<void*>(static_cast<uintptr_t>(unsigned_integer())); }
    // of an output whose type the caller chooses; `absent` for None
    falqon_dtype dtype(const at::Tensor* t, falqon_dtype absent)
    {
        if (failed_ || !t) return absent;
        if (t->scalar_type() == at::kBFloat16) return FALQON_BF16;
        if (t->scalar_type() == at::kFloat) return FALQON_F32;
        PyErr_Format(PyExc_TypeError, "unsupported dtype %s", c10::toString(t->scalar_type()));
        failed_ = true;
        return absent;
    }
    const at::Tensor* fail(PyObject* type, const char* what)
    {
        PyErr_SetString(type, what);
        failed_ = true;
        return nullptr;
    }

private:
    uint64_t unsigned_integer()
    {
        if (failed_) return 0;
        const unsigned long long v = PyLong_AsUnsignedLongLong(args_[next_++]);
        if (v == static_cast<unsigned long long>(-1) && PyErr_Occurred()) failed_ = true;
        return v;
    }
    PyObject* const* args_;
    Py_ssize_t next_ = 0;
    bool failed_ = false;
};

template <typename T = void>
T* data(const at::Tensor* t) { return t ? static_cast<T*>(t->data_ptr()) : nullptr; }
size_t bytes(const at::Tensor* t) { return t ? t->nbytes() : 0; }
int64_t stride(const at::Tensor* t) { return !t ? 0 : t->size(0) > 1 ? t->stride(0) : t->size(1); }

// f() without the interpreter lock; its status as a Python integer
template <typename F>
PyObject* status_of(F f)
{
    falqon_status status;
    Py_BEGIN_ALLOW_THREADS
    status = f();
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(status);
}

// No C++ exception leaves a call.
template <typename F>
PyObject* guarded(F f)
{
    try {
        return f();
    } catch (const std::exception& e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
    } catch (...) {
        PyErr_SetString(PyExc_RuntimeError, "unknown C++ exception");
    }
    return nullptr;
}

PyObject* melded_fwd(PyObject*, PyObject* const* args, Py_ssize_t count)
{
    return guarded([&]() -> PyObject* {
        Args a(args, count, 12);
        const at::Tensor *x = a.tensor(), *wq = a.tensor(), *s_w = a.tensor();
        const int64_t m = a.integer(), r = a.integer();
        const at::Tensor *xq = a.matrix(), *s_x = a.tensor(), *y = a.tensor(), *o_a = a.tensor(), *amax = a.tensor(), *ws = a.tensor();
        if (!a.failed() && !y) a.fail(PyExc_AttributeError, "'NoneType' object has no attribute 'dtype'");
        const falqon_dtype yt = a.dtype(y, FALQON_BF16);
        void* const stream = a.address();
        if (a.failed()) return nullptr;
        const int64_t T = xq->size(0), n = xq->size(1);
        void *const px = data(x), *const py = data(y), *const po = data(o_a), *const pw = data(ws);
        uint8_t *const pwq = data<uint8_t>(wq), *const pxq = data<uint8_t>(xq);
        float *const psw = data<float>(s_w), *const psx = data<float>(s_x), *const pam = data<float>(amax);
        const size_t size = bytes(ws);
        return status_of([=] { return falqon_melded_fwd(px, pwq, psw, T, n, m, r, pxq, psx, py, yt, po, pam, pw, size, stream); });
    });
}

template <bool ADDS>
PyObject* melded_bwd(PyObject*, PyObject* const* args, Py_ssize_t count)
{
    return guarded([&]() -> PyObject* {
        Args a(args, count, 16);
        const at::Tensor *dy = a.matrix(), *wq = a.tensor(), *s_w = a.tensor(), *o_a = a.tensor(), *amax = a.tensor();
        const int64_t n = a.integer(), r = a.integer();
        const at::Tensor *dyq = a.tensor(), *s_dy = a.tensor(), *dx = a.tensor(), *d_b = a.tensor(), *buf = a.tensor();
        const float lr = static_cast<float>(a.real());
        const at::Tensor *ws = a.tensor(), *scores = a.tensor();
        const falqon_dtype dxt = a.dtype(dx, FALQON_BF16);
        void* const stream = a.address();
        if (a.failed()) return nullptr;
        const int64_t T = dy->size(0), m = dy->size(1);
        void *const pdy = data(dy), *const po = data(o_a), *const pdx = data(dx), *const pw = data(ws);
        uint8_t *const pwq = data<uint8_t>(wq), *const pq = data<uint8_t>(dyq);
        float *const psw = data<float>(s_w), *const pam = data<float>(amax), *const ps = data<float>(s_dy), *const pdb = data<float>(d_b), *const pb = data<float>(buf);
        double* const psc = data<double>(scores);
        const size_t size = bytes(ws);
        return status_of([=] {
            return ADDS ? falqon_melded_bwd_add(pdy, pwq, psw, po, pam, T, n, m, r, pq, ps, pdx, pdb, pb, lr, psc, pw, size, stream)
                        : falqon_melded_bwd(pdy, pwq, psw, po, pam, T, n, m, r, pq, ps, pdx, dxt, pdb, pb, lr, psc, pw, size, stream);
        });
    });
}

PyObject* proxy_update(PyObject*, PyObject* const* args, Py_ssize_t count)
{
    return guarded([&]() -> PyObject* {
        Args a(args, count, 10);
        const at::Tensor *buf = a.tensor(), *wq = a.matrix(true);
        const int64_t m = a.integer(), r = a.integer(), k = a.integer();
        const at::Tensor *idx = a.tensor(), *ws = a.tensor();
        const int clear = a.integer() != 0;
        const at::Tensor* scores = a.tensor();
        void* const stream = a.address();
        if (a.failed()) return nullptr;
        const int64_t n = wq->size(1);
        float* const pb = data<float>(buf);
        uint8_t* const pwq = data<uint8_t>(wq);
        int32_t* const pi = data<int32_t>(idx);
        double* const psc = data<double>(scores);
        void* const pw = data(ws);
        const size_t size = bytes(ws);
        return status_of([=] { return falqon_proxy_update(pb, pwq, n, m, r, k, pi, clear, psc, pw, size, stream); });
    });
}

PyObject* grad_sqnorm(PyObject*, PyObject* const* args, Py_ssize_t count)
{
    return guarded([&]() -> PyObject* {
        Args a(args, count, 4);
        const at::Tensor *g = a.tensor(), *sum = a.tensor(), *ws = a.tensor();
        if (!a.failed() && !g) a.fail(PyExc_AttributeError, "'NoneType' object has no attribute 'numel'");
        void* const stream = a.address();
        if (a.failed()) return nullptr;
        float* const pg = data<float>(g);
        double* const ps = data<double>(sum);
        void* const pw = data(ws);
        const int64_t elements = g->numel();
        const size_t size = bytes(ws);
        return status_of([=] { return falqon_grad_sqnorm(pg, elements, ps, pw, size, stream); });
    });
}

PyObject* adamw_delta(PyObject*, PyObject* const* args, Py_ssize_t count)
{
    return guarded([&]() -> PyObject* {
        Args a(args, count, 12);
        const at::Tensor *d_b = a.matrix(), *avg = a.tensor(), *avg_sq = a.tensor(), *buf = a.tensor();
        const int64_t step = a.integer();
        const double lr = a.real(), beta1 = a.real(), beta2 = a.real(), eps = a.real();
        const at::Tensor* sum = a.tensor();
        const double max_norm = a.real();
        void* const stream = a.address();
        if (a.failed()) return nullptr;
        const int64_t m = d_b->size(0), r = d_b->size(1);
        float *const pd = data<float>(d_b), *const pa = data<float>(avg), *const pq = data<float>(avg_sq), *const pb = data<float>(buf);
        double* const ps = data<double>(sum);
        return status_of([=] { return falqon_adamw_delta(pd, pa, pq, pb, m, r, step, lr, beta1, beta2, eps, ps, max_norm, stream); });
    });
}

PyObject* workspace_bytes(PyObject*, PyObject* const* args, Py_ssize_t count)
{
    Args a(args, count, 4);
    const int64_t T = a.integer(), n = a.integer(), m = a.integer(), r = a.integer();
    if (a.failed()) return nullptr;
    return PyLong_FromSize_t(falqon_workspace_bytes(T, n, m, r));
}

// ---- operators around the layer: every shape and type is checked here, as their kernels go by the first tensor's --------------------

PyObject* norm_fwd(PyObject*, PyObject* const* args, Py_ssize_t count)
{
    return guarded([&]() -> PyObject* {
        Args a(args, count, 16);
        const at::Tensor *x = a.rows(), *w = a.tensor(), *h = a.tensor(), *rstd = a.tensor(), *b = a.rows(), *s = a.tensor();
        const double scale = a.real();
        const at::Tensor *gate = a.tensor(), *w_post = a.tensor(), *rstd_b = a.tensor(), *sq = a.tensor(), *s_exp = a.tensor(), *bq = a.tensor(), *b_exp = a.tensor();
        const double eps = a.real();
                void* const stream = a.address();
        a.need(x, "x");
        if (a.failed()) return nullptr;
        const int64_t T = x->size(0), d = x->size(1), blocks = (d + 31) / 32;
        const at::ScalarType type = x->scalar_type();
        const falqon_dtype xt = a.dtype(x, FALQON_BF16);
        a.expect(w, type, {d}, "w"); a.expect(h, type, {T, d}, "h"); a.expect(b, type, {T, d}, "b"); a.expect(s, type, {T, d}, "s");
        a.expect(gate, type, {d}, "gate"); a.expect(w_post, type, {d}, "w_post");
        a.expect(rstd, at::kFloat, {T}, "rstd"); a.expect(rstd_b, at::kFloat, {T}, "rstd_b");
        a.expect(sq, at::kByte, {T, d}, "sq"); a.expect(s_exp, at::kByte, {T, blocks}, "s_exp"); a.expect(bq, at::kByte, {T, d}, "bq"); a.expect(b_exp, at::kByte, {T, blocks}, "b_exp");
        if (a.failed()) return nullptr;
        const falqon_norm_fwd_args call{data(x), data(b), data(w), data(w_post), data(gate), scale, eps, xt, T, d, stride(x), stride(b), data(s), data(h),
                                        data<float>(rstd), data<float>(rstd_b), data<uint8_t>(sq), data<uint8_t>(s_exp), data<uint8_t>(bq), data<uint8_t>(b_exp)};
        return status_of([=] { return falqon_norm_fwd(&call, stream); });
    });
}

PyObject* norm_bwd(PyObject*, PyObject* const* args, Py_ssize_t count)
{
    return guarded([&]() -> PyObject* {
        Args a(args, count, 19);
        const at::Tensor *dh = a.rows(), *s = a.rows(), *w = a.tensor(), *rstd = a.tensor(), *dx = a.tensor(), *ds = a.rows(), *b = a.rows(), *db = a.tensor();
        const double scale = a.real();
        const at::Tensor *gate = a.tensor(), *w_post = a.tensor(), *rstd_b = a.tensor(), *s_exp = a.tensor(), *b_exp = a.tensor();
        const at::Tensor *dw = a.tensor(), *dw_post = a.tensor(), *dgate = a.tensor(), *ws = a.tensor();
                void* const stream = a.address();
        a.need(dh, "dh");
        if (a.failed()) return nullptr;
        const int64_t T = dh->size(0), d = dh->size(1), blocks = (d + 31) / 32;
        const at::ScalarType type = dh->scalar_type(), saved = s_exp ? at::kByte : type;
        const falqon_dtype xt = a.dtype(dh, FALQON_BF16);
        a.expect(s, saved, {T, d}, "s"); a.expect(b, saved, {T, d}, "b"); a.expect(w, type, {d}, "w"); a.expect(gate, type, {d}, "gate"); a.expect(w_post, type, {d}, "w_post");
        a.expect(dx, type, {T, d}, "dx"); a.expect(ds, type, {T, d}, "ds"); a.expect(db, type, {T, d}, "db");
        a.expect(rstd, at::kFloat, {T}, "rstd"); a.expect(rstd_b, at::kFloat, {T}, "rstd_b");
        a.expect(s_exp, at::kByte, {T, blocks}, "s_exp"); a.expect(b_exp, at::kByte, {T, blocks}, "b_exp");
        a.expect(dw, at::kFloat, {d}, "dw"); a.expect(dw_post, at::kFloat, {d}, "dw_post"); a.expect(dgate, at::kFloat, {d}, "dgate");
        if (!a.failed() && s_exp && ((s && !s->is_contiguous()) || (b && !b->is_contiguous()))) a.fail(PyExc_ValueError, "codes are contiguous");
        if (a.failed()) return nullptr;
        const falqon_norm_bwd_args call{data(dh), data(ds), data(s), data(b), data(w), data(w_post), data(gate), data<uint8_t>(s_exp), data<uint8_t>(b_exp),
                                        data<float>(rstd), data<float>(rstd_b), scale, xt, T, d, stride(dh), stride(ds), stride(s), stride(b), data(dx), data(db),
                                        data<float>(dw), data<float>(dw_post), data<float>(dgate), data(ws), bytes(ws)};
        return status_of([=] { return falqon_norm_bwd(&call, stream); });
    });
}

PyObject* swiglu_fwd(PyObject*, PyObject* const* args, Py_ssize_t count)
{
    return guarded([&]() -> PyObject* {
        Args a(args, count, 8);
        const at::Tensor *g = a.rows(), *u = a.rows(), *h = a.tensor(), *gq = a.tensor(), *g_exp = a.tensor(), *uq = a.tensor(), *u_exp = a.tensor();
                void* const stream = a.address();
        a.need(g, "g");
        if (a.failed()) return nullptr;
        const int64_t T = g->size(0), m = g->size(1), blocks = (m + 31) / 32;
        const falqon_dtype xt = a.dtype(g, FALQON_BF16);
        a.expect(u, g->scalar_type(), {T, m}, "u"); a.expect(h, g->scalar_type(), {T, m}, "h");
        a.expect(gq, at::kByte, {T, m}, "gq"); a.expect(g_exp, at::kByte, {T, blocks}, "g_exp"); a.expect(uq, at::kByte, {T, m}, "uq"); a.expect(u_exp, at::kByte, {T, blocks}, "u_exp");
        if (a.failed()) return nullptr;
        const int64_t lg = stride(g), lu = stride(u);
        void *const pg = data(g), *const pu = data(u), *const ph = data(h);
        uint8_t *const q1 = data<uint8_t>(gq), *const e1 = data<uint8_t>(g_exp), *const q2 = data<uint8_t>(uq), *const e2 = data<uint8_t>(u_exp);
        return status_of([=] { return falqon_swiglu_fwd(pg, pu, xt, T, m, lg, lu, ph, q1, e1, q2, e2, stream); });
    });
}

PyObject* swiglu_bwd(PyObject*, PyObject* const* args, Py_ssize_t count)
{
    return guarded([&]() -> PyObject* {
        Args a(args, count, 8);
        const at::Tensor *dh = a.rows(), *g = a.rows(), *u = a.rows(), *dg = a.tensor(), *du = a.tensor(), *g_exp = a.tensor(), *u_exp = a.tensor();
                void* const stream = a.address();
        a.need(dh, "dh");
        if (a.failed()) return nullptr;
        const int64_t T = dh->size(0), m = dh->size(1), blocks = (m + 31) / 32;
        const at::ScalarType type = dh->scalar_type(), saved = g_exp ? at::kByte : type;
        const falqon_dtype xt = a.dtype(dh, FALQON_BF16);
        a.expect(g, saved, {T, m}, "g"); a.expect(u, saved, {T, m}, "u"); a.expect(dg, type, {T, m}, "dg"); a.expect(du, type, {T, m}, "du");
        a.expect(g_exp, at::kByte, {T, blocks}, "g_exp"); a.expect(u_exp, at::kByte, {T, blocks}, "u_exp");
        if (!a.failed() && g_exp && ((g && !g->is_contiguous()) || (u && !u->is_contiguous()))) a.fail(PyExc_ValueError, "codes are contiguous");
        if (a.failed()) return nullptr;
        const int64_t ld = stride(dh), lg = stride(g), lu = stride(u);
        void *const pd = data(dh), *const pg = data(g), *const pu = data(u), *const og = data(dg), *const ou = data(du);
        uint8_t *const e1 = data<uint8_t>(g_exp), *const e2 = data<uint8_t>(u_exp);
        return status_of([=] { return falqon_swiglu_bwd(pd, ld, pg, pu, e1, e2, lg, lu, xt, T, m, og, ou, stream); });
    });
}

PyObject* mx4_linear(PyObject*, PyObject* const* args, Py_ssize_t count)
{
    return guarded([&]() -> PyObject* {
        Args a(args, count, 7);
        const at::Tensor *x = a.tensor(), *wq = a.matrix(), *w_exp = a.tensor(), *xq = a.matrix(), *x_exp = a.tensor(), *y = a.matrix();
        const falqon_dtype yt = a.dtype(y, FALQON_BF16);
        void* const stream = a.address();
        if (a.failed()) return nullptr;
        const int64_t T = y->size(0), m = y->size(1), n = wq->size(1) * 2, pitch = falqon_mx4_exp_pitch(n);
        a.expect(x, at::kBFloat16, {T, n}, "x"); a.expect(wq, at::kByte, {m, n / 2}, "wq"); a.expect(w_exp, at::kByte, {m, pitch}, "w_exp");
        a.expect(xq, at::kByte, {T, n / 2}, "xq"); a.expect(x_exp, at::kByte, {T, pitch}, "x_exp");
        if (a.failed()) return nullptr;
        void *const px = data(x), *const py = data(y);
        uint8_t *const pw = data<uint8_t>(wq), *const ew = data<uint8_t>(w_exp), *const pq = data<uint8_t>(xq), *const eq = data<uint8_t>(x_exp);
        return status_of([=] { return falqon_mx4_linear(px, pw, ew, T, n, m, pq, eq, py, yt, stream); });
    });
}

PyObject* token_logprob(PyObject*, PyObject* const* args, Py_ssize_t count)
{
    return guarded([&]() -> PyObject* {
        Args a(args, count, 7);
        const at::Tensor *x = a.rows(), *labels = a.tensor(), *logp = a.tensor(), *lse = a.tensor(), *ws = a.tensor(), *low = a.tensor();
        void* const stream = a.address();
        a.need(x, "logits");
        if (a.failed()) return nullptr;
        const int64_t T = x->size(0), V = x->size(1), ld = stride(x);
        const falqon_dtype lt = a.dtype(x, FALQON_BF16);
        a.expect(labels, at::kLong, {T}, "labels"); a.expect(logp, at::kFloat, {T}, "logp"); a.expect(lse, at::kFloat, {T}, "lse"); a.expect(low, at::kFloat, {T}, "lse_low");
        if (a.failed()) return nullptr;
        void *const px = data(x), *const pw = data(ws);
        const int64_t* const pl = data<int64_t>(labels);
        float *const pp = data<float>(logp), *const ps = data<float>(lse), *const plow = data<float>(low);
        const size_t size = bytes(ws);
        return status_of([=] { return falqon_token_logprob_low(px, lt, T, V, ld, pl, pp, ps, plow, pw, size, stream); });
    });
}

PyObject* token_logprob_bwd(PyObject*, PyObject* const* args, Py_ssize_t count)
{
    return guarded([&]() -> PyObject* {
        Args a(args, count, 7);
        const at::Tensor *d = a.tensor(), *x = a.rows(), *labels = a.tensor(), *lse = a.tensor(), *out = a.rows(), *low = a.tensor();
        void* const stream = a.address();
        a.need(x, "logits");
        if (a.failed()) return nullptr;
        const int64_t T = x->size(0), V = x->size(1), ld = stride(x), ld_d = stride(out);
        const falqon_dtype lt = a.dtype(x, FALQON_BF16);
        a.expect(d, at::kFloat, {T}, "d_logp"); a.expect(labels, at::kLong, {T}, "labels"); a.expect(lse, at::kFloat, {T}, "lse"); a.expect(out, x->scalar_type(), {T, V}, "dlogits");
        a.expect(low, at::kFloat, {T}, "lse_low");
        if (a.failed()) return nullptr;
        void *const px = data(x), *const po = data(out);
        const int64_t* const pl = data<int64_t>(labels);
        float *const pd = data<float>(d), *const ps = data<float>(lse), *const plow = data<float>(low);
        return status_of([=] { return falqon_token_logprob_bwd_low(pd, px, lt, T, V, ld, pl, ps, plow, po, ld_d, stream); });
    });
}

PyObject* preference_loss(PyObject*, PyObject* const* args, Py_ssize_t count)
{
    return guarded([&]() -> PyObject* {
        Args a(args, count, 10);
        const at::Tensor *logp = a.tensor(), *ref = a.tensor(), *offsets = a.tensor(), *loss = a.tensor(), *rewards = a.matrix(), *d = a.tensor(), *ws = a.tensor();
        const double beta = a.real(), smoothing = a.real();
        void* const stream = a.address();
        a.need(logp, "logp");
        if (a.failed()) return nullptr;
        const int64_t T = logp->numel(), P = rewards->size(1);
        a.expect(logp, at::kFloat, {T}, "logp"); a.expect(ref, at::kFloat, {T}, "ref_logp"); a.expect(offsets, at::kLong, {2 * P + 1}, "offsets");
        a.expect(loss, at::kFloat, {1}, "loss"); a.expect(rewards, at::kFloat, {2, P}, "rewards"); a.expect(d, at::kFloat, {T}, "d_logp");
        if (a.failed()) return nullptr;
        const int64_t* const po = data<int64_t>(offsets);
        float *const pl = data<float>(logp), *const pr = data<float>(ref), *const ps = data<float>(loss), *const pw = data<float>(rewards), *const pd = data<float>(d);
        void* const pws = data(ws);
        const size_t size = bytes(ws);
        return status_of([=] { return falqon_preference_loss(pl, pr, po, T, P, beta, smoothing, ps, pw, pd, pws, size, stream); });
    });
}

PyCFunction fast(PyObject* (*f)(PyObject*, PyObject* const*, Py_ssize_t))
{
    return reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(f));
}

PyMethodDef methods[] = {
    {"melded_fwd", fast(melded_fwd), METH_FASTCALL, nullptr},
    {"melded_bwd", fast(melded_bwd<false>), METH_FASTCALL, nullptr},
    {"melded_bwd_add", fast(melded_bwd<true>), METH_FASTCALL, nullptr},
    {"proxy_update", fast(proxy_update), METH_FASTCALL, nullptr},
    {"grad_sqnorm", fast(grad_sqnorm), METH_FASTCALL, nullptr},
    {"adamw_delta", fast(adamw_delta), METH_FASTCALL, nullptr},
    {"workspace_bytes", fast(workspace_bytes), METH_FASTCALL, nullptr},
    {"norm_fwd", fast(norm_fwd), METH_FASTCALL, nullptr},
    {"norm_bwd", fast(norm_bwd), METH_FASTCALL, nullptr},
    {"swiglu_fwd", fast(swiglu_fwd), METH_FASTCALL, nullptr},
    {"swiglu_bwd", fast(swiglu_bwd), METH_FASTCALL, nullptr},
    {"mx4_linear", fast(mx4_linear), METH_FASTCALL, nullptr},
    {"token_logprob", fast(token_logprob), METH_FASTCALL, nullptr},
    {"token_logprob_bwd", fast(token_logprob_bwd), METH_FASTCALL, nullptr},
    {"preference_loss", fast(preference_loss), METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_calls", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__calls() { return PyModule_Create(&module); }
