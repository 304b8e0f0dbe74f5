// The marshalling of positnn_lm.h's calls, as binding_native.cpp does for those of a training step: what lm.py does for one of them (checks,
// outputs, workspace, the call through ctypes) takes 12 to 19 us of host time where a single token's kernels take 5 to 15.
// As there, a function returns None for whatever it does not take, and the Python code decides.
// Included by binding_native.cpp only.
#pragma once

#include "../../include/positnn_lm.h"

namespace {

enum LmFn { LM_NORM_FWD, LM_NORM_BWD, LM_NORM_WS, LM_SCALE, LM_ATTN_FWD, LM_ATTN_BWD, LM_ATTN_WS, LM_LOGPROB_FWD, LM_LOGPROB_WS, LM_LOGPROB_BWD, LM_COUNT };
void* g_lm[LM_COUNT];

// An element format's tensor: any strides but for elements in a row
bool lm_fits(const at::Tensor& t, long f) {
    if (f == PNN_BF16) return t.scalar_type() == at::kBFloat16 || t.scalar_type() == at::kShort || t.scalar_type() == at::kUInt16;
    return f >= 0 && f < FORMATS && dtype_fits(t.scalar_type(), f);
}
bool lm_format(long f) { return f == PNN_BF16 || (f >= 0 && f < FORMATS && elem_size(f) != 0); }
at::ScalarType lm_dtype(long f) { return f == PNN_BF16 ? at::kBFloat16 : dtype_of(f); }

const at::Tensor* lm_tensor(PyObject* o, long f, int dims) {
    if (!THPVariable_CheckExact(o)) return nullptr;
    const at::Tensor& t = THPVariable_Unpack(o);
    if (!t.is_cuda() || t.dim() != dims || !lm_fits(t, f) || (t.size(dims - 1) > 1 && t.stride(dims - 1) != 1)) return nullptr;
    return &t;
}
// A dense vector of n values, or none where that is allowed
bool lm_vector(PyObject* o, at::ScalarType type, int64_t n, bool optional, const at::Tensor** out) {
    *out = nullptr;
    if (o == Py_None) return optional;
    if (!THPVariable_CheckExact(o)) return false;
    const at::Tensor& t = THPVariable_Unpack(o);
    if (!t.is_cuda() || t.scalar_type() != type || t.numel() != n || !t.is_contiguous()) return false;
    *out = &t;
    return true;
}
bool lm_weight(PyObject* o, long f, int64_t n, const at::Tensor** out) {
    if (!THPVariable_CheckExact(o)) return false;
    const at::Tensor& t = THPVariable_Unpack(o);
    if (!t.is_cuda() || !lm_fits(t, f) || t.numel() != n || !t.is_contiguous()) return false;
    *out = &t;
    return true;
}
int64_t lm_pitch(const at::Tensor& t) { return t.size(0) > 1 ? t.stride(0) : t.size(1); }
const void* lm_in(const at::Tensor* t) { return t ? t->data_ptr() : nullptr; }
void* lm_out(const at::Tensor& t) { return t.defined() ? t.data_ptr() : nullptr; }

PyObject* lm_result(int status, std::initializer_list<const at::Tensor*> out) {
    if (status) return PyLong_FromLong(status);
    PyObject* r = PyTuple_New((Py_ssize_t)out.size());
    Py_ssize_t i = 0;
    for (const at::Tensor* t : out) {
        PyObject* o = t->defined() ? THPVariable_Wrap(*t) : none();
        if (!o || !r) {
            Py_XDECREF(o);
            Py_XDECREF(r);
            return nullptr;
        }
        PyTuple_SET_ITEM(r, i++, o);
    }
    return r;
}
bool lm_real(PyObject* o, float* v) {
    if (!PyFloat_CheckExact(o)) return false;
    *v = (float)PyFloat_AS_DOUBLE(o);
    return true;
}
template <class F>
F lm_fn(LmFn which) { return reinterpret_cast<F>(g_lm[which]); }

// rmsnorm_fwd(stream, fx, fw, fy, fres, scaled, eps, x, w, res)
PyObject* rmsnorm_fwd(PyObject*, PyObject* const* args, Py_ssize_t n) {
    Args a;
    if (!g_lm[0] || !parse(args, n, 6, 4, &a)) return none();
    return guarded([&]() -> PyObject* {
        const long fx = a.i[1], fw = a.i[2], fy = a.i[3], fres = a.i[4];
        const bool scaled = a.i[5] != 0;
        float eps;
        const at::Tensor *x = lm_tensor(a.o[1], fx, 2), *w, *res = nullptr;
        if (!x || x->size(1) == 0 || !lm_format(fy) || !lm_real(a.o[0], &eps) || !lm_weight(a.o[2], fw, x->size(1), &w)) return none();
        if (a.o[3] != Py_None && (!(res = lm_tensor(a.o[3], fres, 2)) || res->sizes() != x->sizes())) return none();
        const int64_t rows = x->size(0), cols = x->size(1);
        at::Tensor y, scale, out, rstd;
        int status;
        {
            Unlocked here;
            y = empty({rows, cols}, lm_dtype(fy), *x);
            rstd = empty({rows}, at::kFloat, *x);
            if (scaled) scale = empty({rows}, at::kFloat, *x);
            if (res) out = empty({rows, cols}, lm_dtype(fres), *x);
            status = lm_fn<decltype(&posit_rmsnorm_fwd)>(LM_NORM_FWD)(a.stream, (int)fx, (int)fres, (int)fw, (int)fy, rows, cols, lm_in(x), lm_pitch(*x), lm_in(res),
                                                                       res ? lm_pitch(*res) : 0, lm_in(w), eps, lm_out(out), cols, lm_out(y), cols, (float*)lm_out(scale),
                                                                       (float*)lm_out(rstd));
        }
        return lm_result(status, {&y, &scale, &out, &rstd});
    });
}

// rmsnorm_bwd(stream, fd, fh, fw, fdx, fdw, fdres, want_dw, dy, h, w, rstd, dres)
PyObject* rmsnorm_bwd(PyObject*, PyObject* const* args, Py_ssize_t n) {
    Args a;
    if (!g_lm[0] || !parse(args, n, 8, 5, &a)) return none();
    return guarded([&]() -> PyObject* {
        const long fd = a.i[1], fh = a.i[2], fw = a.i[3], fdx = a.i[4], fdw = a.i[5], fdres = a.i[6];
        const bool want = a.i[7] != 0;
        const at::Tensor *dy = lm_tensor(a.o[0], fd, 2), *h = lm_tensor(a.o[1], fh, 2), *w, *rstd, *dres = nullptr;
        if (!dy || !h || h->sizes() != dy->sizes() || dy->size(0) == 0 || !lm_format(fdx) || !lm_format(fdw)) return none();
        const int64_t rows = dy->size(0), cols = dy->size(1);
        if (!lm_weight(a.o[2], fw, cols, &w) || !lm_vector(a.o[3], at::kFloat, rows, false, &rstd)) return none();
        if (a.o[4] != Py_None && (!(dres = lm_tensor(a.o[4], fdres, 2)) || dres->sizes() != dy->sizes())) return none();
        at::Tensor dx, dw, ws;
        int status;
        {
            Unlocked here;
            dx = empty({rows, cols}, lm_dtype(fdx), *dy);
            size_t bytes = 0;
            if (want) {
                dw = empty({cols}, lm_dtype(fdw), *dy);
                bytes = lm_fn<decltype(&posit_rmsnorm_bwd_workspace)>(LM_NORM_WS)(rows, cols);
                if (bytes) ws = empty({(int64_t)bytes}, at::kByte, *dy);
            }
            status = lm_fn<decltype(&posit_rmsnorm_bwd)>(LM_NORM_BWD)(a.stream, (int)fd, (int)fh, (int)fw, (int)fdres, (int)fdx, (int)fdw, rows, cols, lm_in(dy), lm_pitch(*dy),
                                                                       lm_in(h), lm_pitch(*h), lm_in(w), (const float*)lm_in(rstd), lm_in(dres), dres ? lm_pitch(*dres) : 0,
                                                                       lm_out(dx), cols, lm_out(dw), lm_out(ws), bytes);
        }
        return lm_result(status, {&dx, &dw});
    });
}

// scale_rows(stream, fin, fout, x, scale)
PyObject* scale_rows(PyObject*, PyObject* const* args, Py_ssize_t n) {
    Args a;
    if (!g_lm[0] || !parse(args, n, 3, 2, &a)) return none();
    return guarded([&]() -> PyObject* {
        const long fin = a.i[1], fout = a.i[2];
        const at::Tensor *x = lm_tensor(a.o[0], fin, 2), *s;
        if (!x || !lm_format(fout) || !lm_vector(a.o[1], at::kFloat, x->size(0), false, &s)) return none();
        at::Tensor y;
        int status;
        {
            Unlocked here;
            y = empty(x->sizes(), lm_dtype(fout), *x);
            status = lm_fn<decltype(&posit_scale_rows)>(LM_SCALE)(a.stream, (int)fin, (int)fout, x->size(0), x->size(1), lm_in(x), lm_pitch(*x), (const float*)lm_in(s), lm_out(y),
                                                                   x->size(1));
        }
        return result(status, y);
    });
}

bool lm_attention(long fq, long fkv, PyObject* oq, PyObject* ok, PyObject* ov, PyObject* ol, PyObject* oscale, long window, long sinks, const at::Tensor* (&t)[4],
                  pnn_attention_desc* d) {
    t[0] = lm_tensor(oq, fq, 4);
    t[1] = lm_tensor(ok, fkv, 4);
    t[2] = lm_tensor(ov, fkv, 4);
    if (!t[0] || !t[1] || !t[2] || t[1]->sizes() != t[2]->sizes() || t[1]->size(0) != t[0]->size(0) || t[1]->size(3) != t[0]->size(3)) return false;
    if (!lm_real(oscale, &d->scale) || !lm_vector(ol, at::kInt, t[0]->size(0), true, &t[3])) return false;
    d->B = t[0]->size(0);
    d->LQ = t[0]->size(1);
    d->HQ = t[0]->size(2);
    d->D = t[0]->size(3);
    d->LK = t[1]->size(1);
    d->HKV = t[1]->size(2);
    d->window = window;
    d->sinks = sinks;
    d->qb = t[0]->stride(0); d->ql = t[0]->stride(1); d->qh = t[0]->stride(2);
    d->kb = t[1]->stride(0); d->kl = t[1]->stride(1); d->kh = t[1]->stride(2);
    d->vb = t[2]->stride(0); d->vl = t[2]->stride(1); d->vh = t[2]->stride(2);
    return true;
}

// attention_fwd(stream, fq, fkv, fout, window, sinks, fcopy, scale, q, k, v, lens): fcopy -1 for no copy
PyObject* attention_fwd(PyObject*, PyObject* const* args, Py_ssize_t n) {
    Args a;
    if (!g_lm[0] || !parse(args, n, 7, 5, &a)) return none();
    return guarded([&]() -> PyObject* {
        const long fq = a.i[1], fkv = a.i[2], fout = a.i[3], fcopy = a.i[6];
        const at::Tensor* t[4];
        pnn_attention_desc d;
        if (!lm_format(fout) || (fcopy != -1 && !lm_format(fcopy)) || !lm_attention(fq, fkv, a.o[1], a.o[2], a.o[3], a.o[4], a.o[0], a.i[4], a.i[5], t, &d)) return none();
        if (d.D == 0) return none();
        at::Tensor o, lse, copy, ws;
        int status;
        {
            Unlocked here;
            o = empty({d.B, d.LQ, d.HQ, d.D}, lm_dtype(fout), *t[0]);
            lse = empty({d.B, d.HQ, d.LQ}, at::kFloat, *t[0]);
            if (fcopy != -1) copy = empty({d.B, d.LQ, d.HQ, d.D}, lm_dtype(fcopy), *t[0]);
            const size_t bytes = lm_fn<decltype(&posit_attention_workspace)>(LM_ATTN_WS)(0, (int)fkv, &d);
            if (bytes) ws = empty({(int64_t)bytes}, at::kByte, *t[0]);
            status = lm_fn<decltype(&posit_attention_fwd)>(LM_ATTN_FWD)(a.stream, (int)fq, (int)fkv, (int)fout, &d, lm_in(t[0]), lm_in(t[1]), lm_in(t[2]), (const int32_t*)lm_in(t[3]),
                                                                         lm_out(o), (float*)lm_out(lse), fcopy == -1 ? 0 : (int)fcopy, lm_out(copy), lm_out(ws), bytes);
        }
        return lm_result(status, {&o, &lse, &copy});
    });
}

// attention_bwd(stream, fd, fq, fkv, fo, fout, window, sinks, scale, do, q, k, v, o, lse, lens)
PyObject* attention_bwd(PyObject*, PyObject* const* args, Py_ssize_t n) {
    Args a;
    if (!g_lm[0] || !parse(args, n, 8, 8, &a)) return none();
    return guarded([&]() -> PyObject* {
        const long fd = a.i[1], fq = a.i[2], fkv = a.i[3], fo = a.i[4], fout = a.i[5];
        const at::Tensor* t[4];
        pnn_attention_desc d;
        if (!lm_format(fout) || !lm_attention(fq, fkv, a.o[2], a.o[3], a.o[4], a.o[7], a.o[0], a.i[6], a.i[7], t, &d)) return none();
        const at::Tensor *g = lm_tensor(a.o[1], fd, 4), *o = lm_tensor(a.o[5], fo, 4), *lse;
        if (!g || !o || g->sizes() != t[0]->sizes() || g->strides() != t[0]->strides() || o->sizes() != t[0]->sizes() || !o->is_contiguous()) return none();
        if (!lm_vector(a.o[6], at::kFloat, d.B * d.HQ * d.LQ, false, &lse)) return none();
        at::Tensor dq, dk, dv, ws;
        int status;
        {
            Unlocked here;
            dq = empty({d.B, d.LQ, d.HQ, d.D}, lm_dtype(fout), *t[0]);
            dk = empty({d.B, d.LK, d.HKV, d.D}, lm_dtype(fout), *t[0]);
            dv = empty({d.B, d.LK, d.HKV, d.D}, lm_dtype(fout), *t[0]);
            const size_t bytes = lm_fn<decltype(&posit_attention_workspace)>(LM_ATTN_WS)(1, (int)fkv, &d);
            if (bytes) ws = empty({(int64_t)bytes}, at::kByte, *t[0]);
            status = lm_fn<decltype(&posit_attention_bwd)>(LM_ATTN_BWD)(a.stream, (int)fd, (int)fq, (int)fkv, (int)fo, (int)fout, &d, lm_in(g), lm_in(t[0]), lm_in(t[1]), lm_in(t[2]),
                                                                         (const int32_t*)lm_in(t[3]), lm_in(o), (const float*)lm_in(lse), lm_out(dq), lm_out(dk), lm_out(dv), lm_out(ws),
                                                                         bytes);
        }
        return lm_result(status, {&dq, &dk, &dv});
    });
}

// logprob_fwd(stream, fz, top, inv_temperature, logits, targets)
PyObject* logprob_fwd(PyObject*, PyObject* const* args, Py_ssize_t n) {
    Args a;
    if (!g_lm[0] || !parse(args, n, 3, 3, &a)) return none();
    return guarded([&]() -> PyObject* {
        const long fz = a.i[1], top = a.i[2];
        float tau;
        const at::Tensor *z = lm_tensor(a.o[1], fz, 2), *y;
        if (!z || z->size(1) == 0 || top < 0 || top > 64 || !lm_real(a.o[0], &tau) || !lm_vector(a.o[2], at::kInt, z->size(0), true, &y)) return none();
        const int64_t rows = z->size(0), vocab = z->size(1);
        at::Tensor lp, lse, ent, tl, ti, ws;
        int status;
        {
            Unlocked here;
            if (y) lp = empty({rows}, at::kFloat, *z);
            lse = empty({rows}, at::kFloat, *z);
            ent = empty({rows}, at::kFloat, *z);
            if (top) {
                tl = empty({rows, top}, at::kFloat, *z);
                ti = empty({rows, top}, at::kInt, *z);
            }
            const size_t bytes = lm_fn<decltype(&posit_token_logprob_workspace)>(LM_LOGPROB_WS)((int)fz, rows, vocab, (int)top);
            if (bytes) ws = empty({(int64_t)bytes}, at::kByte, *z);
            status = lm_fn<decltype(&posit_token_logprob_fwd)>(LM_LOGPROB_FWD)(a.stream, (int)fz, rows, vocab, lm_in(z), lm_pitch(*z), (const int32_t*)lm_in(y), tau, (int)top,
                                                                                (float*)lm_out(lp), (float*)lm_out(lse), (float*)lm_out(ent), (float*)lm_out(tl), (int32_t*)lm_out(ti),
                                                                                lm_out(ws), bytes);
        }
        return lm_result(status, {&lp, &lse, &ent, &tl, &ti});
    });
}

// logprob_bwd(stream, fz, fg, inv_temperature, logits, targets, lse, entropy, g_logprob, g_entropy)
PyObject* logprob_bwd(PyObject*, PyObject* const* args, Py_ssize_t n) {
    Args a;
    if (!g_lm[0] || !parse(args, n, 3, 7, &a)) return none();
    return guarded([&]() -> PyObject* {
        const long fz = a.i[1], fg = a.i[2];
        float tau;
        const at::Tensor *z = lm_tensor(a.o[1], fz, 2), *y, *lse, *ent, *g1, *g2;
        if (!z || !lm_format(fg) || !lm_real(a.o[0], &tau)) return none();
        const int64_t rows = z->size(0), vocab = z->size(1);
        if (!lm_vector(a.o[2], at::kInt, rows, true, &y) || !lm_vector(a.o[3], at::kFloat, rows, false, &lse) || !lm_vector(a.o[4], at::kFloat, rows, true, &ent) ||
            !lm_vector(a.o[5], at::kFloat, rows, true, &g1) || !lm_vector(a.o[6], at::kFloat, rows, true, &g2))
            return none();
        at::Tensor dz;
        int status;
        {
            Unlocked here;
            dz = empty({rows, vocab}, lm_dtype(fg), *z);
            status = lm_fn<decltype(&posit_token_logprob_bwd)>(LM_LOGPROB_BWD)(a.stream, (int)fz, (int)fg, rows, vocab, lm_in(z), lm_pitch(*z), (const int32_t*)lm_in(y), tau,
                                                                                (const float*)lm_in(lse), (const float*)lm_in(ent), (const float*)lm_in(g1), (const float*)lm_in(g2),
                                                                                lm_out(dz), vocab);
        }
        return result(status, dz);
    });
}

// init_lm(address ...): the library's functions in the order of LmFn; after init, which brings the formats
PyObject* init_lm(PyObject*, PyObject* const* args, Py_ssize_t n) {
    if (n != LM_COUNT) {
        PyErr_SetString(PyExc_TypeError, "one address per function");
        return nullptr;
    }
    void* fn[LM_COUNT];
    for (int k = 0; k < LM_COUNT; ++k) {
        fn[k] = PyLong_AsVoidPtr(args[k]);
        if (!fn[k]) {
            if (!PyErr_Occurred()) PyErr_SetString(PyExc_ValueError, "null address");
            return nullptr;
        }
    }
    for (int k = 0; k < LM_COUNT; ++k) g_lm[k] = fn[k];
    Py_RETURN_NONE;
}

}  // namespace
