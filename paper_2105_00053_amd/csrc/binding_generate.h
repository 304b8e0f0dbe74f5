// The marshalling of positnn_generate.h's calls, as binding_lm.h does for those of positnn_lm.h: a step of single tokens makes four of them, whose kernels take 5 to 15 us and
// whose marshalling by generate.py 12 to 20 each.
// As there, a function returns None for whatever it does not take, and the Python code decides.
// Included by binding_native.cpp only.
#pragma once

#include "../../include/positnn_generate.h"

namespace {

enum GenFn { GEN_HEADS_FWD, GEN_HEADS_BWD, GEN_HEADS_WS, GEN_APPEND, GEN_READ, GEN_PAGED, GEN_PAGED_WS, GEN_SAMPLE, GEN_SAMPLE_WS, GEN_COUNT };
void* g_gen[GEN_COUNT];
template <class F>
F gen_fn(GenFn which) { return reinterpret_cast<F>(g_gen[which]); }

bool gen_on(const at::Tensor* t, long device) { return !t || t->get_device() == device; }

// [rows][heads][elements]
bool gen_heads(PyObject* o, long f, long device, const at::Tensor** out) {
    *out = lm_tensor(o, f, 3);
    return *out && gen_on(*out, device);
}
bool gen_weight(PyObject* o, long f, int64_t n, long device, const at::Tensor** out) {
    *out = nullptr;
    return o == Py_None || (lm_weight(o, f, n, out) && gen_on(*out, device));
}
bool gen_vector(PyObject* o, at::ScalarType type, int64_t n, long device, const at::Tensor** out) { return lm_vector(o, type, n, true, out) && gen_on(*out, device); }
// the pairs' frequencies, of any number that a head has room for
bool gen_freq(PyObject* o, int64_t d, long device, const at::Tensor** out) {
    *out = nullptr;
    if (o == Py_None) return true;
    if (!THPVariable_CheckExact(o)) return false;
    const at::Tensor& t = THPVariable_Unpack(o);
    if (!t.is_cuda() || t.scalar_type() != at::kDouble || !t.is_contiguous() || 2 * t.numel() > d) return false;
    *out = &t;
    return gen_on(*out, device);
}

// q, k (may be None), wq, wk, positions, inv_freq
struct GenHeads {
    const at::Tensor *q, *k, *wq, *wk, *pos, *freq;
    pnn_heads_desc d;
};
bool gen_heads_args(PyObject* const* o, long fx, long fw, long device, GenHeads* g) {
    g->k = nullptr;
    if (!gen_heads(o[0], fx, device, &g->q)) return false;
    const int64_t T = g->q->size(0), D = g->q->size(2);
    if (o[1] != Py_None && (!gen_heads(o[1], fx, device, &g->k) || g->k->size(0) != T || g->k->size(2) != D)) return false;
    if (!gen_weight(o[2], fw, D, device, &g->wq) || !gen_weight(o[3], fw, D, device, &g->wk)) return false;
    if (g->k ? !g->wq != !g->wk : g->wk && !g->wq) return false;
    if (!gen_vector(o[4], at::kInt, T, device, &g->pos) || !gen_freq(o[5], D, device, &g->freq) || !g->pos != !g->freq) return false;
    g->d = {};
    g->d.T = T;
    g->d.HQ = g->q->size(1);
    g->d.HKV = g->k ? g->k->size(1) : 0;
    g->d.D = D;
    g->d.R = g->freq ? 2 * g->freq->numel() : 0;
    g->d.ql = g->q->stride(0);
    g->d.qh = g->q->stride(1);
    if (g->k) {
        g->d.kl = g->k->stride(0);
        g->d.kh = g->k->stride(1);
    }
    return true;
}

// heads_fwd(stream, device, fx, fw, fy, neighbours, eps, q, k, wq, wk, positions, inv_freq)
PyObject* heads_fwd(PyObject*, PyObject* const* args, Py_ssize_t n) {
    Args a;
    if (!g_gen[0] || !parse(args, n, 6, 7, &a)) return none();
    return guarded([&]() -> PyObject* {
        const long dev = a.i[1], fx = a.i[2], fw = a.i[3], fy = a.i[4];
        GenHeads g;
        float eps;
        if (!lm_format(fy) || !lm_real(a.o[0], &eps) || !gen_heads_args(a.o + 1, fx, fw, dev, &g)) return none();
        g.d.neighbours = a.i[5] != 0;
        g.d.eps = eps;
        at::Tensor yq, yk, rstd;
        int status;
        {
            Unlocked here;
            yq = empty(g.q->sizes(), lm_dtype(fy), *g.q);
            if (g.k) yk = empty(g.k->sizes(), lm_dtype(fy), *g.q);
            if (g.wq) rstd = empty({g.d.T, g.d.HQ + g.d.HKV}, at::kFloat, *g.q);
            status = gen_fn<decltype(&posit_qk_norm_rope_fwd)>(GEN_HEADS_FWD)(a.stream, (int)fx, (int)fw, (int)fy, &g.d, lm_in(g.q), lm_in(g.k), lm_in(g.wq), lm_in(g.wk),
                                                                               (const int32_t*)lm_in(g.pos), (const double*)lm_in(g.freq), lm_out(yq), lm_out(yk), (float*)lm_out(rstd));
        }
        return lm_result(status, {&yq, &yk, &rstd});
    });
}

// heads_bwd(stream, device, fd, fx, fw, fdx, fdw, flags, dyq, dyk, q, k, wq, wk, positions, inv_freq, rstd): flags 1: neighbours, 2: gradients of the weights
PyObject* heads_bwd(PyObject*, PyObject* const* args, Py_ssize_t n) {
    Args a;
    if (!g_gen[0] || !parse(args, n, 8, 9, &a)) return none();
    return guarded([&]() -> PyObject* {
        const long dev = a.i[1], fd = a.i[2], fx = a.i[3], fw = a.i[4], fdx = a.i[5], fdw = a.i[6];
        GenHeads g;
        const at::Tensor *gq, *gk = nullptr, *rstd;
        if (!lm_format(fdx) || !lm_format(fdw) || !gen_heads_args(a.o + 2, fx, fw, dev, &g) || g.d.T == 0 || g.d.HQ + g.d.HKV == 0) return none();
        if (!gen_heads(a.o[0], fd, dev, &gq) || gq->sizes() != g.q->sizes()) return none();
        if (g.k && (!gen_heads(a.o[1], fd, dev, &gk) || gk->sizes() != g.k->sizes())) return none();
        if (!gen_vector(a.o[8], at::kFloat, g.d.T * (g.d.HQ + g.d.HKV), dev, &rstd) || !rstd != !g.wq) return none();
        g.d.neighbours = a.i[7] & 1;
        g.d.gql = gq->stride(0);
        g.d.gqh = gq->stride(1);
        if (gk) {
            g.d.gkl = gk->stride(0);
            g.d.gkh = gk->stride(1);
        }
        const bool want = (a.i[7] & 2) && g.wq;
        at::Tensor dq, dk, dwq, dwk, ws;
        int status;
        {
            Unlocked here;
            dq = empty(g.q->sizes(), lm_dtype(fdx), *g.q);
            if (g.k) dk = empty(g.k->sizes(), lm_dtype(fdx), *g.q);
            size_t bytes = 0;
            if (want) {
                dwq = empty({g.d.D}, lm_dtype(fdw), *g.q);
                if (g.k) dwk = empty({g.d.D}, lm_dtype(fdw), *g.q);
                bytes = gen_fn<decltype(&posit_qk_norm_rope_bwd_workspace)>(GEN_HEADS_WS)(&g.d);
                if (bytes) ws = empty({(int64_t)bytes}, at::kByte, *g.q);
            }
            status = gen_fn<decltype(&posit_qk_norm_rope_bwd)>(GEN_HEADS_BWD)(a.stream, (int)fd, (int)fx, (int)fw, (int)fdx, (int)fdw, &g.d, lm_in(gq), lm_in(gk), lm_in(g.q), lm_in(g.k),
                                                                               lm_in(g.wq), lm_in(g.wk), (const float*)lm_in(rstd), (const int32_t*)lm_in(g.pos), (const double*)lm_in(g.freq),
                                                                               lm_out(dq), lm_out(dk), lm_out(dwq), lm_out(dwk), lm_out(ws), bytes);
        }
        return lm_result(status, {&dq, &dk, &dwq, &dwk});
    });
}

// pages_k, pages_v, table, lens, starts (may be None)
struct GenCache {
    const at::Tensor *k, *v, *table, *lens, *starts;
};
bool gen_cache(PyObject* const* o, long fc, int64_t hkv, int64_t d, int64_t rows, long device, GenCache* c, pnn_paged_desc* p) {
    const long f = fc == PNN_F4 ? 0 : fc;  // bytes, as 8-bit posits are
    if (!gen_heads(o[0], f, device, &c->k) || !gen_heads(o[1], f, device, &c->v) || c->k->sizes() != c->v->sizes() || !c->k->is_contiguous() || !c->v->is_contiguous()) return false;
    if (hkv < 0) hkv = c->k->size(1);
    const int64_t per = fc == PNN_F4 ? d / 2 + (d + 31) / 32 : d;
    if (c->k->size(1) != hkv || per <= 0 || c->k->size(2) == 0 || c->k->size(2) % per != 0) return false;
    if (!THPVariable_CheckExact(o[2])) return false;
    c->table = &THPVariable_Unpack(o[2]);
    if (!c->table->is_cuda() || c->table->dim() != 2 || c->table->scalar_type() != at::kInt || (c->table->size(1) > 1 && c->table->stride(1) != 1) || !gen_on(c->table, device)) return false;
    const int64_t b = c->table->size(0);
    if (!gen_vector(o[3], at::kInt, b, device, &c->lens) || !c->lens || !gen_vector(o[4], at::kInt, b + 1, device, &c->starts) || (rows >= 0 && !c->starts && rows != b)) return false;
    *p = {};
    p->T = rows < 0 ? 0 : rows;
    p->B = b;
    p->HKV = hkv;
    p->D = d;
    p->page = c->k->size(2) / per;
    p->pages = c->k->size(0);
    p->columns = c->table->size(1);
    p->pitch = b > 1 ? c->table->stride(0) : c->table->size(1);
    return true;
}
bool gen_cache_format(long f) { return f == PNN_F4 || lm_format(f); }

// cache_append(stream, device, fx, fw, fq, fcache, neighbours, eps, k, v, pages_k, pages_v, table, lens, starts, q, inv_freq, wq, wk)
PyObject* cache_append(PyObject*, PyObject* const* args, Py_ssize_t n) {
    Args a;
    if (!g_gen[0] || !parse(args, n, 7, 12, &a)) return none();
    return guarded([&]() -> PyObject* {
        const long dev = a.i[1], fx = a.i[2], fw = a.i[3], fq = a.i[4], fc = a.i[5];
        const at::Tensor *k, *v, *q = nullptr, *freq, *wq, *wk;
        GenCache c;
        pnn_paged_desc p;
        float eps;
        if (!gen_cache_format(fc) || !lm_format(fq) || !lm_real(a.o[0], &eps) || !gen_heads(a.o[1], fx, dev, &k) || !gen_heads(a.o[2], fx, dev, &v) || v->sizes() != k->sizes()) return none();
        const int64_t rows = k->size(0), d = k->size(2);
        if (!gen_cache(a.o + 3, fc, k->size(1), d, rows, dev, &c, &p)) return none();
        if (a.o[8] != Py_None && (!gen_heads(a.o[8], fx, dev, &q) || q->size(0) != rows || q->size(2) != d)) return none();
        if (!gen_freq(a.o[9], d, dev, &freq) || !gen_weight(a.o[10], fw, d, dev, &wq) || !gen_weight(a.o[11], fw, d, dev, &wk)) return none();
        if ((wq && !wk) || (q && wk && !wq)) return none();
        p.R = freq ? 2 * freq->numel() : 0;
        p.neighbours = a.i[6] != 0;
        p.eps = eps;
        p.kl = k->stride(0);
        p.kh = k->stride(1);
        p.vl = v->stride(0);
        p.vh = v->stride(1);
        if (q) {
            p.HQ = q->size(1);
            p.ql = q->stride(0);
            p.qh = q->stride(1);
        }
        at::Tensor yq;
        int status;
        {
            Unlocked here;
            if (q) yq = empty(q->sizes(), lm_dtype(fq), *k);
            status = gen_fn<decltype(&posit_cache_append)>(GEN_APPEND)(a.stream, (int)fx, (int)fw, (int)fq, (int)fc, &p, lm_in(q), lm_in(k), lm_in(v), lm_in(wq), lm_in(wk),
                                                                        (const double*)lm_in(freq), (const int32_t*)lm_in(c.starts), (const int32_t*)lm_in(c.lens),
                                                                        (const int32_t*)lm_in(c.table), c.k->data_ptr(), c.v->data_ptr(), lm_out(yq));
        }
        return lm_result(status, {&yq});
    });
}

// cache_read(stream, device, longest, d, fcache, fout, pages_k, pages_v, table, lens, None)
PyObject* cache_read(PyObject*, PyObject* const* args, Py_ssize_t n) {
    Args a;
    if (!g_gen[0] || !parse(args, n, 6, 5, &a)) return none();
    return guarded([&]() -> PyObject* {
        const long dev = a.i[1], longest = a.i[2], d = a.i[3], fc = a.i[4], fout = a.i[5];
        GenCache c;
        pnn_paged_desc p;
        if (longest < 0 || d < 0 || !gen_cache_format(fc) || !lm_format(fout) || !gen_cache(a.o, fc, -1, d, -1, dev, &c, &p)) return none();
        p.longest = longest;
        at::Tensor k, v;
        int status;
        {
            Unlocked here;
            k = empty({p.B, longest, p.HKV, d}, lm_dtype(fout), *c.table);
            v = empty({p.B, longest, p.HKV, d}, lm_dtype(fout), *c.table);
            status = gen_fn<decltype(&posit_cache_read)>(GEN_READ)(a.stream, (int)fc, (int)fout, &p, (const int32_t*)lm_in(c.lens), (const int32_t*)lm_in(c.table), lm_in(c.k), lm_in(c.v),
                                                                    lm_out(k), lm_out(v));
        }
        return lm_result(status, {&k, &v});
    });
}

// attention_paged(stream, device, fq, fcache, fout, most, window, sinks, scale, q, pages_k, pages_v, table, lens, starts, longest): longest None for what the table holds
PyObject* attention_paged(PyObject*, PyObject* const* args, Py_ssize_t n) {
    Args a;
    if (!g_gen[0] || !parse(args, n, 8, 8, &a)) return none();
    return guarded([&]() -> PyObject* {
        const long dev = a.i[1], fq = a.i[2], fc = a.i[3], fout = a.i[4];
        const at::Tensor* q;
        GenCache c;
        pnn_paged_desc p;
        float scale;
        long longest = 0;
        if (!gen_cache_format(fc) || !lm_format(fout) || !lm_real(a.o[0], &scale) || !gen_heads(a.o[1], fq, dev, &q) || !gen_cache(a.o + 2, fc, -1, q->size(2), q->size(0), dev, &c, &p)) return none();
        if (a.o[7] != Py_None && !integer(a.o[7], &longest)) return none();
        p.HQ = q->size(1);
        p.ql = q->stride(0);
        p.qh = q->stride(1);
        p.most = a.i[5];
        p.window = a.i[6];
        p.sinks = a.i[7];
        p.longest = a.o[7] == Py_None ? p.columns * p.page : longest;
        p.scale = scale;
        at::Tensor o, lse, ws;
        int status;
        {
            Unlocked here;
            o = empty(q->sizes(), lm_dtype(fout), *q);
            lse = empty({p.T, p.HQ}, at::kFloat, *q);
            const size_t bytes = gen_fn<decltype(&posit_attention_paged_workspace)>(GEN_PAGED_WS)(&p);
            if (bytes) ws = empty({(int64_t)bytes}, at::kByte, *q);
            status = gen_fn<decltype(&posit_attention_paged)>(GEN_PAGED)(a.stream, (int)fq, (int)fc, (int)fout, &p, lm_in(q), (const int32_t*)lm_in(c.starts), (const int32_t*)lm_in(c.lens),
                                                                          (const int32_t*)lm_in(c.table), lm_in(c.k), lm_in(c.v), lm_out(o), (float*)lm_out(lse), lm_out(ws), bytes);
        }
        return lm_result(status, {&o, &lse});
    });
}

// sample(stream, device, fz, logits, u, temperature, top_k, top_p, min_p)
PyObject* sample(PyObject*, PyObject* const* args, Py_ssize_t n) {
    Args a;
    if (!g_gen[0] || !parse(args, n, 3, 6, &a)) return none();
    return guarded([&]() -> PyObject* {
        const long dev = a.i[1], fz = a.i[2];
        const at::Tensor *z = lm_tensor(a.o[0], fz, 2), *u, *temperature, *k, *p, *m;
        if (!z || z->size(1) == 0 || !gen_on(z, dev)) return none();
        const int64_t rows = z->size(0), vocab = z->size(1);
        if (!gen_vector(a.o[1], at::kFloat, rows, dev, &u) || !u || !gen_vector(a.o[2], at::kFloat, rows, dev, &temperature) || !gen_vector(a.o[3], at::kInt, rows, dev, &k) ||
            !gen_vector(a.o[4], at::kFloat, rows, dev, &p) || !gen_vector(a.o[5], at::kFloat, rows, dev, &m))
            return none();
        at::Tensor token, lp, kept, ws;
        int status;
        {
            Unlocked here;
            token = empty({rows}, at::kInt, *z);
            lp = empty({rows}, at::kFloat, *z);
            kept = empty({rows}, at::kInt, *z);
            const size_t bytes = gen_fn<decltype(&posit_sample_workspace)>(GEN_SAMPLE_WS)((int)fz, rows, vocab);
            if (bytes) ws = empty({(int64_t)bytes}, at::kByte, *z);
            status = gen_fn<decltype(&posit_sample)>(GEN_SAMPLE)(a.stream, (int)fz, rows, vocab, lm_in(z), lm_pitch(*z), (const float*)lm_in(u), (const float*)lm_in(temperature),
                                                                  (const int32_t*)lm_in(k), (const float*)lm_in(p), (const float*)lm_in(m), (int32_t*)lm_out(token), (float*)lm_out(lp),
                                                                  (int32_t*)lm_out(kept), lm_out(ws), bytes);
        }
        return lm_result(status, {&token, &lp, &kept});
    });
}

// init_generate(address ...): the library's functions in the order of GenFn; after init, which brings the formats
PyObject* init_generate(PyObject*, PyObject* const* args, Py_ssize_t n) {
    if (n != GEN_COUNT) {
        PyErr_SetString(PyExc_TypeError, "one address per function");
        return nullptr;
    }
    void* fn[GEN_COUNT];
    for (int k = 0; k < GEN_COUNT; ++k) {
        fn[k] = PyLong_AsVoidPtr(args[k]);
        if (!fn[k]) {
            if (!PyErr_Occurred()) PyErr_SetString(PyExc_ValueError, "null address");
            return nullptr;
        }
    }
    for (int k = 0; k < GEN_COUNT; ++k) g_gen[k] = fn[k];
    Py_RETURN_NONE;
}

}  // namespace
