// Native argument marshalling of the Python binding (mbscan.py).
//
// A Python-level call spends 12-20 us on checking ten tensors (type, dtype,
// shape, strides, device) and filling the argument struct, several times what
// the small calls take on the GPU. These functions make the same checks on the
// tensors' C++ objects and call the C ABI. Each returns the mb_status, or -1 if
// anything is not as the plain path wants it (a tensor subclass, a wrong dtype,
// shape, stride or device, no storage, no CUDA device, ...): the caller then
// takes the plain path, which raises the error or handles the rest. Nothing is
// kept from one call for the next.
#include <Python.h>

#include <ATen/core/Tensor.h>
#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cstring>

#include "mbscan.h"

namespace {

// The C ABI's entry points, from the library that mbscan.py has loaded (init).
struct Api {
    decltype(&mb_scan_prefill) prefill;
    decltype(&mb_scan_verify) verify;
    decltype(&mb_scan_verify_resume) verify_resume;
    decltype(&mb_scan_prefill_ckpt) prefill_ckpt;
    decltype(&mb_step) step;
    decltype(&mb_step_resume) step_resume;
    decltype(&mb_rollback) rollback;
    decltype(&mb_accept_topk) accept_topk;
    decltype(&mb_rmsnorm) rmsnorm;
    decltype(&mb_conv1d_step) conv1d_step;
    decltype(&mb_conv_xproj) conv_xproj;
    decltype(&mb_conv1d) conv1d;
    decltype(&mb_conv1d_backward) conv1d_backward;
    decltype(&mb_embed) embed;
    decltype(&mb_embed_backward) embed_backward;
    decltype(&mb_cross_entropy) cross_entropy;
    decltype(&mb_grad_norm) grad_norm;
    decltype(&mb_grad_clip) grad_clip;
    decltype(&mb_rmsnorm_q8) rmsnorm_q8;
    decltype(&mb_quantize_q8) quantize_q8;
    decltype(&mb_dequantize_q8) dequantize_q8;
    decltype(&mb_matmul_q8) matmul_q8;
    decltype(&mb_sample) sample;
} api;

// One call's tensors and whether all of them are as they should be.
struct Call {
    PyObject *const *v;
    bool ok = true;
    c10::Device dev{c10::kCPU};
    bool have_dev = false;

    const at::Tensor *get(int i) {   // null for None
        if (v[i] == Py_None) return nullptr;
        if (!THPVariable_CheckExact(v[i])) {
            ok = false;
            return nullptr;
        }
        return &THPVariable_Unpack(v[i]);
    }
    void *ptr(const at::Tensor *t) { return t && ok ? t->data_ptr() : nullptr; }
    // contiguous, of this dtype and shape, on the call's device (that of its first tensor, a CUDA device)
    void *need(int i, at::ScalarType ty, c10::IntArrayRef dims, bool any_shape = false) {
        const at::Tensor *t = get(i);
        if (!t || !ok) return nullptr;
        if (t->scalar_type() != ty || (!any_shape && t->sizes() != dims) || !t->is_contiguous() || !on(*t)) ok = false;
        return ptr(t);
    }
    // the same, and not None
    void *must(int i, at::ScalarType ty, c10::IntArrayRef dims, bool any_shape = false) {
        if (v[i] == Py_None) ok = false;
        return need(i, ty, dims, any_shape);
    }
    bool on(const at::Tensor &t) {
        if (!have_dev) {
            dev = t.device();
            have_dev = true;
        }
        return t.device() == dev && dev.is_cuda();
    }
    // row stride of a [batch, L, width] tensor: contiguous, or a column block of wider rows
    int64_t row_stride(const at::Tensor *t, int64_t batch, int64_t L, int64_t width, at::ScalarType ty) {
        if (!t || t->scalar_type() != ty || t->sizes() != c10::IntArrayRef({batch, L, width}) || !on(*t)) {
            ok = false;
            return 0;
        }
        if (t->is_contiguous()) return width;
        const auto st = t->strides();
        if (st[2] != 1 || (L > 1 && st[0] != L * st[1]) || st[1] < width) {
            ok = false;
            return 0;
        }
        return L > 1 || batch == 1 ? st[1] : st[0];
    }
};

constexpr at::ScalarType kF32 = at::kFloat;

bool dtype_of(const at::Tensor *t, int32_t &dt) {
    if (!t) return false;
    if (t->scalar_type() == at::kFloat) dt = MB_F32;
    else if (t->scalar_type() == at::kBFloat16) dt = MB_BF16;
    else return false;
    return true;
}

// v[0..9]: x, dt, B, C, A, y, z, D, dt_bias, h0
bool fill(Call &c, mb_scan_args &a) {
    a = mb_scan_args{};
    const at::Tensor *x = c.get(0), *A = c.get(4), *B = c.get(2), *C = c.get(3);
    if (!c.ok || !x || !A || !B || !C || x->dim() != 3 || A->dim() != 2 || !dtype_of(x, a.dtype)) return false;
    c.on(*x);
    const at::ScalarType ty = x->scalar_type();
    const int64_t b = x->size(0), L = x->size(1), D = x->size(2), N = A->size(1);
    a.batch = b; a.seqlen = L; a.d_inner = D; a.d_state = N;
    const int64_t tok[3] = {b, L, D};
    a.x = c.must(0, ty, tok);
    a.dt = c.must(1, ty, tok);
    a.y = c.must(5, ty, tok);
    a.z = c.need(6, ty, tok);
    const int64_t S = c.row_stride(B, b, L, N, ty), S2 = c.row_stride(C, b, L, N, ty);
    if (S != S2 || S > INT32_MAX) c.ok = false;
    a.bc_stride = S == N ? 0 : (int32_t)S;
    a.B = c.ptr(B);
    a.C = c.ptr(C);
    a.A = static_cast<const float *>(c.must(4, kF32, {D, N}));
    a.D = static_cast<const float *>(c.need(7, kF32, {D}));
    a.dt_bias = static_cast<const float *>(c.need(8, kF32, {D}));
    a.h0 = static_cast<const float *>(c.need(9, kF32, {b, D, N}));
    return c.ok;
}

// A workspace tensor: uint8, contiguous; bytes in `n`
void *workspace(Call &c, int i, size_t &n, bool may_be_none) {
    n = 0;
    if (c.v[i] == Py_None) {
        if (!may_be_none) c.ok = false;
        return nullptr;
    }
    void *p = c.need(i, at::kByte, {}, true);
    if (c.ok) n = (size_t)c.get(i)->numel();
    return p;
}

void *stream() { return c10::cuda::getCurrentCUDAStream().stream(); }

template <typename F>
PyObject *guarded(Py_ssize_t have, Py_ssize_t want, F &&f) {
    if (have != want) {
        PyErr_Format(PyExc_TypeError, "expected %zd arguments, got %zd", want, have);
        return nullptr;
    }
    long rc = -1;
    try {
        rc = f();
    } catch (...) {   // e.g. a tensor without storage: the plain path reports it
        rc = -1;
    }
    return PyLong_FromLong(rc);
}

// Run a C ABI call without the interpreter lock (as ctypes does).
template <typename F>
long call(F &&f) {
    void *s = stream();
    long rc;
    Py_BEGIN_ALLOW_THREADS
    rc = (long)f(s);
    Py_END_ALLOW_THREADS
    return rc;
}

#define ARGS PyObject *, PyObject *const *v, Py_ssize_t n

// x, dt, B, C, A, y, z, D, dt_bias, None, state, ws
PyObject *step(ARGS) {
    return guarded(n, 12, [&]() -> long {
        Call c{v};
        mb_scan_args a;
        if (!fill(c, a)) return -1;
        float *state = static_cast<float *>(c.must(10, kF32, {a.batch, a.d_inner, a.d_state}));
        size_t wb;
        void *ws = workspace(c, 11, wb, true);
        if (!c.ok) return -1;
        return call([&](void *s) { return api.step(&a, state, ws, wb, s); });
    });
}

// x, dt, B, C, A, y, z, D, dt_bias, h0, h_all, accept, state, ws
PyObject *step_resume(ARGS) {
    return guarded(n, 14, [&]() -> long {
        Call c{v};
        mb_scan_args a;
        if (!fill(c, a)) return -1;
        const at::Tensor *h = c.get(10);
        if (!h || h->dim() != 4) return -1;
        const int64_t k = h->size(1);
        const float *h_all = static_cast<const float *>(c.must(10, kF32, {a.batch, k, a.d_inner, a.d_state}));
        const int32_t *acc = static_cast<const int32_t *>(c.must(11, at::kInt, {a.batch}));
        float *state = static_cast<float *>(c.must(12, kF32, {a.batch, a.d_inner, a.d_state}));
        size_t wb;
        void *ws = workspace(c, 13, wb, true);
        if (!c.ok) return -1;
        return call([&](void *s) { return api.step_resume(&a, h_all, acc, k, state, ws, wb, s); });
    });
}

// x, dt, B, C, A, y, z, D, dt_bias, h0, h_last, ws
PyObject *prefill(ARGS) {
    return guarded(n, 12, [&]() -> long {
        Call c{v};
        mb_scan_args a;
        if (!fill(c, a)) return -1;
        float *h_last = static_cast<float *>(c.need(10, kF32, {a.batch, a.d_inner, a.d_state}));
        size_t wb;
        void *ws = workspace(c, 11, wb, false);
        if (!c.ok) return -1;
        return call([&](void *s) { return api.prefill(&a, h_last, ws, wb, s); });
    });
}

// x, dt, B, C, A, y, z, D, dt_bias, h0, h_last, h_ckpt, ws
PyObject *prefill_ckpt(ARGS) {
    return guarded(n, 13, [&]() -> long {
        Call c{v};
        mb_scan_args a;
        if (!fill(c, a)) return -1;
        float *h_last = static_cast<float *>(c.need(10, kF32, {a.batch, a.d_inner, a.d_state}));
        const int64_t nch = (a.seqlen + MB_CKPT_STEPS - 1) / MB_CKPT_STEPS;
        float *ck = static_cast<float *>(c.must(11, kF32, {a.batch, nch, a.d_inner, a.d_state}));
        size_t wb;
        void *ws = workspace(c, 12, wb, false);
        if (!c.ok) return -1;
        return call([&](void *s) { return api.prefill_ckpt(&a, h_last, ck, ws, wb, s); });
    });
}

// x, dt, B, C, A, y, z, D, dt_bias, h0, h_all, ws
PyObject *verify(ARGS) {
    return guarded(n, 12, [&]() -> long {
        Call c{v};
        mb_scan_args a;
        if (!fill(c, a)) return -1;
        float *h_all = static_cast<float *>(c.must(10, kF32, {a.batch, a.seqlen, a.d_inner, a.d_state}));
        size_t wb;
        void *ws = workspace(c, 11, wb, false);
        if (!c.ok) return -1;
        return call([&](void *s) { return api.verify(&a, h_all, ws, wb, s); });
    });
}

// x, dt, B, C, A, y, z, D, dt_bias, h0, h_all, h_all_prev, accept, ws
PyObject *verify_resume(ARGS) {
    return guarded(n, 14, [&]() -> long {
        Call c{v};
        mb_scan_args a;
        if (!fill(c, a)) return -1;
        float *h_all = static_cast<float *>(c.must(10, kF32, {a.batch, a.seqlen, a.d_inner, a.d_state}));
        const at::Tensor *h = c.get(11);
        if (!h || h->dim() != 4) return -1;
        const int64_t k = h->size(1);
        const float *prev = static_cast<const float *>(c.must(11, kF32, {a.batch, k, a.d_inner, a.d_state}));
        const int32_t *acc = static_cast<const int32_t *>(c.must(12, at::kInt, {a.batch}));
        size_t wb;
        void *ws = workspace(c, 13, wb, false);
        if (!c.ok) return -1;
        return call([&](void *s) { return api.verify_resume(&a, prev, acc, k, h_all, ws, wb, s); });
    });
}

// h0, h_all, accept, h_out, ws
PyObject *rollback(ARGS) {
    return guarded(n, 5, [&]() -> long {
        Call c{v};
        const at::Tensor *h = c.get(1);
        if (!h || h->dim() != 4) return -1;
        c.on(*h);
        const int64_t b = h->size(0), k = h->size(1), D = h->size(2), N = h->size(3);
        const float *h_all = static_cast<const float *>(c.must(1, kF32, {b, k, D, N}));
        const float *h0 = static_cast<const float *>(c.need(0, kF32, {b, D, N}));
        const int32_t *acc = static_cast<const int32_t *>(c.must(2, at::kInt, {b}));
        float *out = static_cast<float *>(c.must(3, kF32, {b, D, N}));
        size_t wb;
        void *ws = workspace(c, 4, wb, true);
        if (!c.ok) return -1;
        return call([&](void *s) { return api.rollback(h0, h_all, acc, out, b, k, D, N, ws, s); });
    });
}

// logits, drafted, accept, beta
PyObject *accept_topk(ARGS) {
    return guarded(n, 4, [&]() -> long {
        Call c{v};
        const at::Tensor *t = c.get(0);
        int32_t dt;
        if (!t || t->dim() != 3 || t->size(2) != 256 || !dtype_of(t, dt) || !PyLong_CheckExact(v[3])) return -1;
        int over = 0;
        const long beta = PyLong_AsLongAndOverflow(v[3], &over);
        if (over || beta < INT32_MIN || beta > INT32_MAX) return -1;
        const int64_t b = t->size(0), k = t->size(1);
        const void *logits = c.must(0, t->scalar_type(), {b, k, 256});
        const uint8_t *drafted = static_cast<const uint8_t *>(c.must(1, at::kByte, {b, k}));
        int32_t *acc = static_cast<int32_t *>(c.must(2, at::kInt, {b}));
        if (!c.ok) return -1;
        return call([&](void *s) { return api.accept_topk(logits, dt, drafted, b, k, (int32_t)beta, acc, s); });
    });
}

// residual, w, out, add, eps
PyObject *rmsnorm(ARGS) {
    return guarded(n, 5, [&]() -> long {
        Call c{v};
        const at::Tensor *r = c.get(0), *o = c.get(2);
        int32_t dt;
        if (!r || r->dim() != 2 || !dtype_of(o, dt) || !PyFloat_CheckExact(v[4])) return -1;
        c.on(*r);
        const int64_t b = r->size(0), w = r->size(1);
        float *res = static_cast<float *>(c.must(0, kF32, {b, w}));
        const float *wt = static_cast<const float *>(c.must(1, kF32, {w}));
        void *out = c.must(2, o->scalar_type(), {b, w});
        const void *add = c.need(3, o->scalar_type(), {b, w});
        if (!c.ok) return -1;
        const float eps = (float)PyFloat_AS_DOUBLE(v[4]);
        return call([&](void *s) { return api.rmsnorm(add, res, wt, eps, out, b, w, dt, s); });
    });
}

// x, state, w, out, bias
PyObject *conv1d_step(ARGS) {
    return guarded(n, 5, [&]() -> long {
        Call c{v};
        const at::Tensor *x = c.get(0);
        int32_t dt;
        if (!x || x->dim() != 2 || !dtype_of(x, dt)) return -1;
        c.on(*x);
        const at::ScalarType ty = x->scalar_type();
        const int64_t b = x->size(0), w = x->size(1);
        const void *xp = c.must(0, ty, {b, w});
        void *st = c.must(1, ty, {b, 3, w});
        const float *wt = static_cast<const float *>(c.must(2, kF32, {w, 4}));
        void *out = c.must(3, ty, {b, w});
        const float *bias = static_cast<const float *>(c.need(4, kF32, {w}));
        if (!c.ok) return -1;
        return call([&](void *s) { return api.conv1d_step(xp, st, wt, bias, out, b, w, dt, s); });
    });
}

// x, state, w, W, xc, out, ws, bias
PyObject *conv_xproj(ARGS) {
    return guarded(n, 8, [&]() -> long {
        Call c{v};
        const at::Tensor *x = c.get(0), *W = c.get(3);
        if (!x || x->dim() != 2 || !W || W->dim() != 2 || W->size(0) > INT32_MAX) return -1;
        c.on(*x);
        constexpr at::ScalarType bf = at::kBFloat16;
        const int64_t b = x->size(0), w = x->size(1), no = W->size(0);
        const void *xp = c.must(0, bf, {b, w});
        void *st = c.must(1, bf, {b, 3, w});
        const float *wt = static_cast<const float *>(c.must(2, kF32, {w, 4}));
        const void *Wp = c.must(3, bf, {no, w});
        void *xc = c.must(4, bf, {b, w}), *out = c.must(5, bf, {b, no});
        size_t wb;
        void *ws = workspace(c, 6, wb, false);
        const float *bias = static_cast<const float *>(c.need(7, kF32, {w}));
        if (!c.ok) return -1;
        return call([&](void *s) {
            return api.conv_xproj(xp, st, wt, bias, Wp, xc, out, b, w, (int32_t)no, MB_BF16, ws, wb, s);
        });
    });
}

// The arguments of a convolution over a span.
bool fill_conv(Call &c, mb_conv1d_args &a, int x_at, int w_at, int bias_at, int state_at) {
    a = mb_conv1d_args{};
    const at::Tensor *x = c.get(x_at);
    if (!x || x->dim() != 3 || !dtype_of(x, a.dtype)) return false;
    c.on(*x);
    const at::ScalarType ty = x->scalar_type();
    a.batch = x->size(0); a.seqlen = x->size(1); a.width = x->size(2);
    const int64_t S = c.row_stride(x, a.batch, a.seqlen, a.width, ty);
    if (S > INT32_MAX) c.ok = false;
    a.x_stride = S == a.width ? 0 : (int32_t)S;
    a.x = c.ptr(x);
    a.w = static_cast<const float *>(c.must(w_at, kF32, {a.width, 4}));
    a.bias = static_cast<const float *>(c.need(bias_at, kF32, {a.width}));
    a.state = c.need(state_at, ty, {a.batch, 3, a.width});
    return c.ok;
}

// x, w, out, bias, state, state_out
PyObject *conv1d(ARGS) {
    return guarded(n, 6, [&]() -> long {
        Call c{v};
        mb_conv1d_args a;
        if (!fill_conv(c, a, 0, 1, 3, 4)) return -1;
        const at::ScalarType ty = c.get(0)->scalar_type();
        void *out = c.must(2, ty, {a.batch, a.seqlen, a.width});
        void *so = c.need(5, ty, {a.batch, 3, a.width});
        if (!c.ok) return -1;
        return call([&](void *s) { return api.conv1d(&a, out, so, s); });
    });
}

// x, w, dout, bias, state, dstate_out, dx, dw, dbias, dstate, ws
PyObject *conv1d_backward(ARGS) {
    return guarded(n, 11, [&]() -> long {
        Call c{v};
        mb_conv1d_args a;
        if (!fill_conv(c, a, 0, 1, 3, 4)) return -1;
        const at::ScalarType ty = c.get(0)->scalar_type();
        const void *dout = c.must(2, ty, {a.batch, a.seqlen, a.width});
        const void *dso = c.need(5, ty, {a.batch, 3, a.width});
        const at::Tensor *dx = c.get(6);
        const int64_t S = c.row_stride(dx, a.batch, a.seqlen, a.width, ty);
        mb_conv1d_grads g{};
        g.dx = c.ptr(dx);
        g.dx_stride = S == a.width ? 0 : S;
        g.dw = static_cast<float *>(c.must(7, kF32, {a.width, 4}));
        g.dbias = static_cast<float *>(c.need(8, kF32, {a.width}));
        g.dstate = c.need(9, ty, {a.batch, 3, a.width});
        size_t wb;
        void *ws = workspace(c, 10, wb, false);
        if (!c.ok) return -1;
        return call([&](void *s) { return api.conv1d_backward(&a, dout, dso, &g, ws, wb, s); });
    });
}

bool token_type(const at::Tensor *t, int32_t &ty) {
    if (!t) return false;
    if (t->scalar_type() == at::kByte) ty = MB_TOKEN_U8;
    else if (t->scalar_type() == at::kInt) ty = MB_TOKEN_I32;
    else if (t->scalar_type() == at::kLong) ty = MB_TOKEN_I64;
    else return false;
    return true;
}

// Whether t's shape is that of `rows` with one more dimension of this size.
bool rows_of(const at::Tensor *t, const at::Tensor *rows, int64_t last) {
    return t && t->dim() == rows->dim() + 1 && t->size(-1) == last && t->sizes().slice(0, rows->dim()) == rows->sizes();
}

// tokens, table, out, scale
PyObject *embed(ARGS) {
    return guarded(n, 4, [&]() -> long {
        Call c{v};
        const at::Tensor *tok = c.get(0), *table = c.get(1), *o = c.get(2);
        int32_t tt, dt, od;
        if (!token_type(tok, tt) || !dtype_of(table, dt) || !dtype_of(o, od) || table->dim() != 2 ||
            !PyFloat_CheckExact(v[3]) || !rows_of(o, tok, table->size(1)))
            return -1;
        const void *tp = c.must(0, tok->scalar_type(), {}, true), *wp = c.must(1, table->scalar_type(), {}, true);
        void *op = c.must(2, o->scalar_type(), {}, true);
        if (!c.ok) return -1;
        const float scale = (float)PyFloat_AS_DOUBLE(v[3]);
        const int64_t count = tok->numel(), vocab = table->size(0), width = table->size(1);
        return call([&](void *s) { return api.embed(tp, tt, wp, dt, scale, op, od, count, vocab, width, s); });
    });
}

// tokens, dout, dtable, scale, accumulate, ws
PyObject *embed_backward(ARGS) {
    return guarded(n, 6, [&]() -> long {
        Call c{v};
        const at::Tensor *tok = c.get(0), *d = c.get(1), *table = c.get(2);
        int32_t tt, dt;
        if (!token_type(tok, tt) || !dtype_of(d, dt) || !table || table->dim() != 2 || !PyFloat_CheckExact(v[3]) ||
            !PyBool_Check(v[4]) || !rows_of(d, tok, table->size(1)))
            return -1;
        const void *tp = c.must(0, tok->scalar_type(), {}, true), *dp = c.must(1, d->scalar_type(), {}, true);
        float *op = static_cast<float *>(c.must(2, kF32, {}, true));
        size_t wb;
        void *ws = workspace(c, 5, wb, false);
        if (!c.ok) return -1;
        const float scale = (float)PyFloat_AS_DOUBLE(v[3]);
        const int32_t acc = v[4] == Py_True;
        const int64_t count = tok->numel(), vocab = table->size(0), width = table->size(1);
        return call([&](void *s) {
            return api.embed_backward(tp, tt, dp, dt, scale, acc, op, count, vocab, width, ws, wb, s);
        });
    });
}

// logits, targets, loss, dlogits, weight, scale
PyObject *cross_entropy(ARGS) {
    return guarded(n, 6, [&]() -> long {
        Call c{v};
        const at::Tensor *l = c.get(0), *tgt = c.get(1);
        int32_t tt, dt;
        if (!token_type(tgt, tt) || !dtype_of(l, dt) || l->dim() < 1 || !PyFloat_CheckExact(v[5]) ||
            !rows_of(l, tgt, l->size(-1)))
            return -1;
        const at::ScalarType ty = l->scalar_type();
        const void *lp = c.must(0, ty, {}, true), *tp = c.must(1, tgt->scalar_type(), {}, true);
        float *loss = static_cast<float *>(c.must(2, kF32, tgt->sizes()));
        void *dl = c.need(3, ty, l->sizes());
        const float *w = static_cast<const float *>(c.need(4, kF32, tgt->sizes()));
        if (!c.ok) return -1;
        const float scale = (float)PyFloat_AS_DOUBLE(v[5]);
        const int64_t count = tgt->numel(), vocab = l->size(-1);
        return call([&](void *s) { return api.cross_entropy(lp, dt, tp, tt, w, scale, loss, dl, count, vocab, s); });
    });
}

// The array of a tensor list (mbscan.py's TensorList, which has checked its tensors) and its length.
bool tensor_list(Call &c, int at, int count_at, const mb_tensor *&list, int64_t &count) {
    if (!PyLong_CheckExact(c.v[at]) || !PyLong_CheckExact(c.v[count_at])) return false;
    list = static_cast<const mb_tensor *>(PyLong_AsVoidPtr(c.v[at]));
    count = PyLong_AsLongLong(c.v[count_at]);
    if (PyErr_Occurred()) {
        PyErr_Clear();
        return false;
    }
    return true;
}

// address, count, the list's first tensor, norm, ws
PyObject *grad_norm(ARGS) {
    return guarded(n, 5, [&]() -> long {
        Call c{v};
        const mb_tensor *list;
        int64_t count;
        const at::Tensor *first = c.get(2);
        if (!tensor_list(c, 0, 1, list, count) || !first || !c.on(*first)) return -1;
        float *norm = static_cast<float *>(c.must(3, kF32, {1}));
        size_t wb;
        void *ws = workspace(c, 4, wb, false);
        if (!c.ok) return -1;
        return call([&](void *s) { return api.grad_norm(list, count, norm, ws, wb, s); });
    });
}

// address, count, the list's first tensor, norm, max_norm, the outputs' address (0: in place), their first tensor or None
PyObject *grad_clip(ARGS) {
    return guarded(n, 7, [&]() -> long {
        Call c{v};
        const mb_tensor *list, *out;
        int64_t count;
        const at::Tensor *first = c.get(2), *first_out = c.get(6);
        if (!tensor_list(c, 0, 1, list, count) || !tensor_list(c, 5, 1, out, count) || !first || !c.on(*first) ||
            (first_out && !c.on(*first_out)) || !PyFloat_CheckExact(v[4]))
            return -1;
        const float *norm = static_cast<const float *>(c.must(3, kF32, {1}));
        if (!c.ok) return -1;
        const float most = (float)PyFloat_AS_DOUBLE(v[4]);
        return call([&](void *s) { return api.grad_clip(list, out, count, norm, most, s); });
    });
}

// An 8-bit matrix [rows, width] at i and its scales at `scales_at`.
struct Q8 {
    uint8_t *q = nullptr, *scales = nullptr;
    int64_t rows = 0, width = 0;
};
bool fill_q8(Call &c, Q8 &m, int i, int scales_at, int64_t block_rows) {
    const at::Tensor *t = c.get(i);
    if (!t || t->dim() != 2 || (t->scalar_type() != at::kFloat8_e4m3fn && t->scalar_type() != at::kByte)) return false;
    m.rows = t->size(0);
    m.width = t->size(1);
    m.q = static_cast<uint8_t *>(c.must(i, t->scalar_type(), {}, true));
    const int64_t words = (m.width + 511) / 512;
    m.scales = static_cast<uint8_t *>(c.must(scales_at, at::kByte, {(m.rows + block_rows - 1) / block_rows, 4 * words}));
    return c.ok;
}
// The call's tensors are on the current device, whose stream it takes.
bool here(const Call &c) { return c.dev.index() == c10::cuda::current_device(); }

bool block_rows_of(PyObject *o, int32_t &block_rows) {
    if (!PyLong_CheckExact(o)) return false;
    int over = 0;
    const long n = PyLong_AsLongAndOverflow(o, &over);
    block_rows = (int32_t)n;
    return !over && (n == 1 || n == 128);
}

// residual, w, q, scales, add, eps
PyObject *rmsnorm_q8(ARGS) {
    return guarded(n, 6, [&]() -> long {
        Call c{v};
        Q8 m;
        if (!fill_q8(c, m, 2, 3, 1) || !PyFloat_CheckExact(v[5])) return -1;
        float *res = static_cast<float *>(c.must(0, kF32, {m.rows, m.width}));
        const float *w = static_cast<const float *>(c.must(1, kF32, {m.width}));
        const at::Tensor *add = c.get(4);
        int32_t dt = MB_BF16;
        if (add && !dtype_of(add, dt)) return -1;
        const void *ap = add ? c.must(4, add->scalar_type(), {m.rows, m.width}) : nullptr;
        if (!c.ok || !here(c)) return -1;
        const float eps = (float)PyFloat_AS_DOUBLE(v[5]);
        return call([&](void *s) { return api.rmsnorm_q8(ap, dt, res, w, eps, m.q, m.scales, m.rows, m.width, s); });
    });
}

// x, q, scales, block_rows
PyObject *quantize_q8(ARGS) {
    return guarded(n, 4, [&]() -> long {
        Call c{v};
        Q8 m;
        int32_t br, dt;
        const at::Tensor *x = c.get(0);
        if (!block_rows_of(v[3], br) || !fill_q8(c, m, 1, 2, br) || !dtype_of(x, dt)) return -1;
        if (x->dim() != 2 || x->size(0) != m.rows || x->size(1) != m.width || !c.on(*x) || !here(c)) return -1;
        if (!x->is_contiguous() && (x->stride(1) != 1 || x->stride(0) < m.width)) return -1;
        const int64_t S = x->is_contiguous() || m.rows == 1 ? m.width : x->stride(0);
        const void *xp = c.ptr(x);
        if (!c.ok) return -1;
        return call([&](void *s) { return api.quantize_q8(xp, dt, S, br, m.q, m.scales, m.rows, m.width, s); });
    });
}

// q, scales, out, block_rows
PyObject *dequantize_q8(ARGS) {
    return guarded(n, 4, [&]() -> long {
        Call c{v};
        Q8 m;
        int32_t br, dt;
        const at::Tensor *o = c.get(2);
        if (!block_rows_of(v[3], br) || !fill_q8(c, m, 0, 1, br) || !dtype_of(o, dt)) return -1;
        void *op = c.must(2, o->scalar_type(), {m.rows, m.width});
        if (!c.ok || !here(c)) return -1;
        return call([&](void *s) { return api.dequantize_q8(m.q, m.scales, br, op, dt, m.rows, m.width, s); });
    });
}

// a, a_scales, w, w_scales, out, ws
PyObject *matmul_q8(ARGS) {
    return guarded(n, 6, [&]() -> long {
        Call c{v};
        Q8 a, w;
        int32_t dt;
        const at::Tensor *o = c.get(4);
        if (!fill_q8(c, a, 0, 1, 1) || !fill_q8(c, w, 2, 3, 128) || !dtype_of(o, dt) || a.width != w.width) return -1;
        void *op;
        int64_t part = w.rows;
        if (o->dim() == 2) op = c.must(4, o->scalar_type(), {a.rows, w.rows});
        else if (o->dim() == 3) {
            part = o->size(2);
            if (o->size(0) * part != w.rows) return -1;
            op = c.must(4, o->scalar_type(), {o->size(0), a.rows, part});
        } else return -1;
        size_t wb;
        void *ws = workspace(c, 5, wb, true);
        if (!c.ok || !here(c)) return -1;
        return call([&](void *s) {
            return api.matmul_q8(a.q, a.scales, w.q, w.scales, op, dt, a.rows, w.rows, a.width, part, ws, wb, s);
        });
    });
}

// logits, u, tokens, temperature, top_k, top_p, min_p, prob
PyObject *sample(ARGS) {
    return guarded(n, 8, [&]() -> long {
        Call c{v};
        const at::Tensor *l = c.get(0), *tok = c.get(2);
        int32_t dt, tt;
        if (!dtype_of(l, dt) || l->dim() != 2 || !token_type(tok, tt) || tt == MB_TOKEN_U8) return -1;
        const int64_t rows = l->size(0), vocab = l->size(1);
        const void *lp = c.must(0, l->scalar_type(), {rows, vocab});
        const float *u = static_cast<const float *>(c.must(1, kF32, {rows}));
        void *tp = c.must(2, tok->scalar_type(), {rows});
        const float *temperature = static_cast<const float *>(c.need(3, kF32, {rows}));
        const int32_t *top_k = static_cast<const int32_t *>(c.need(4, at::kInt, {rows}));
        const float *top_p = static_cast<const float *>(c.need(5, kF32, {rows}));
        const float *min_p = static_cast<const float *>(c.need(6, kF32, {rows}));
        float *prob = static_cast<float *>(c.need(7, kF32, {rows}));
        if (!c.ok || !here(c)) return -1;
        return call([&](void *s) {
            return api.sample(lp, dt, u, temperature, top_k, top_p, min_p, tp, tt, prob, rows, vocab, s);
        });
    });
}

// init(addresses of the entry points, in Api's order)
PyObject *init(ARGS) {
    constexpr Py_ssize_t kN = sizeof(Api) / sizeof(void *);
    if (n != kN) {
        PyErr_Format(PyExc_TypeError, "expected %zd addresses, got %zd", kN, n);
        return nullptr;
    }
    void *p[kN];
    for (Py_ssize_t i = 0; i < kN; ++i) {
        p[i] = PyLong_AsVoidPtr(v[i]);
        if (PyErr_Occurred()) return nullptr;
    }
    static_assert(sizeof(p) == sizeof(api), "one address per entry point");
    std::memcpy(&api, p, sizeof(api));
    Py_RETURN_NONE;
}

#define DEF(f) {#f, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(f)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {DEF(init),     DEF(step),          DEF(step_resume), DEF(prefill), DEF(prefill_ckpt),
                         DEF(verify),   DEF(verify_resume), DEF(rollback),    DEF(accept_topk), DEF(rmsnorm),
                         DEF(conv1d_step), DEF(conv_xproj), DEF(conv1d), DEF(conv1d_backward),
                         DEF(embed), DEF(embed_backward), DEF(cross_entropy), DEF(grad_norm), DEF(grad_clip),
                         DEF(rmsnorm_q8), DEF(quantize_q8), DEF(dequantize_q8), DEF(matmul_q8), DEF(sample),
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_mbcall", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__mbcall(void) { return PyModule_Create(&module); }
