"""Binding of include/positnn_generate.h: norms of queries and keys with the rotation by their positions, a cache of keys and values in pages with the
attention that reads it, and the draw of the next token.

Argument marshalling only, as in lm.py, whose formats these are; "f4" is a cache's format of 4 bits.  Tensors may be views: rows and heads with any strides, elements
contiguous.  All tensors of a call are on the current device.
"""
import ctypes
import math

import torch

from . import binding
from .binding import PositError, _check, _stream, load
from .lm import _code as _lm_code, _dtype, _ptr, _returned, _vector, _work

F4 = 103


class HeadsDesc(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int64) for n in ("T", "HQ", "HKV", "D", "R", "ql", "qh", "kl", "kh", "gql", "gqh", "gkl", "gkh")] + [
        ("neighbours", ctypes.c_int32), ("eps", ctypes.c_float)]


class PagedDesc(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int64) for n in ("T", "B", "HQ", "HKV", "D", "R", "page", "pages", "columns", "pitch", "ql", "qh", "kl", "kh", "vl", "vh", "window", "sinks",
                                              "most", "longest")] + [("scale", ctypes.c_float), ("eps", ctypes.c_float), ("neighbours", ctypes.c_int32)]


_lib = None


def _load():
    """The shared library with the signatures of this header's functions."""
    global _lib
    if _lib is None:
        L = load()
        vp, i64, ci, sz = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int, ctypes.c_size_t
        hp, pp = ctypes.POINTER(HeadsDesc), ctypes.POINTER(PagedDesc)
        L.posit_qk_norm_rope_fwd.argtypes = [vp, ci, ci, ci, hp] + [vp] * 9
        L.posit_qk_norm_rope_bwd.argtypes = [vp, ci, ci, ci, ci, ci, hp] + [vp] * 14 + [sz]
        L.posit_qk_norm_rope_bwd_workspace.argtypes = [hp]
        L.posit_cache_append.argtypes = [vp, ci, ci, ci, ci, pp] + [vp] * 12
        L.posit_cache_read.argtypes = [vp, ci, ci, pp] + [vp] * 6
        L.posit_attention_paged.argtypes = [vp, ci, ci, ci, pp] + [vp] * 9 + [sz]
        L.posit_attention_paged_workspace.argtypes = [pp]
        L.posit_sample.argtypes = [vp, ci, i64, i64, vp, i64] + [vp] * 9 + [sz]
        L.posit_sample_workspace.argtypes = [ci, i64, i64]
        for name in ("posit_qk_norm_rope_fwd", "posit_qk_norm_rope_bwd", "posit_cache_append", "posit_cache_read", "posit_attention_paged", "posit_sample"):
            getattr(L, name).restype = ci
        for name in ("posit_qk_norm_rope_bwd_workspace", "posit_attention_paged_workspace", "posit_sample_workspace"):
            getattr(L, name).restype = sz
        if binding._native is not None:
            binding._native.init_generate(*(ctypes.cast(getattr(L, name), vp).value for name in _NATIVE_ORDER))
        _lib = L
    return _lib


# As in lm.py, a call goes to the extension module first, which returns None for whatever it does not take.
_NATIVE_ORDER = ("posit_qk_norm_rope_fwd", "posit_qk_norm_rope_bwd", "posit_qk_norm_rope_bwd_workspace", "posit_cache_append", "posit_cache_read", "posit_attention_paged",
                 "posit_attention_paged_workspace", "posit_sample", "posit_sample_workspace")


def _ready():
    """(the extension module, the current stream, the current device), or three times None where the Python code takes the call."""
    if _lib is None:
        _load()
    stream = binding._ready()
    return (None, None, None) if stream is None else (binding._native, stream, binding._current_device())


def _code(f):
    return F4 if f == "f4" else _lm_code(f)


def _here(*tensors):
    """Every tensor is on the current device, whose stream the call goes to."""
    device = torch.cuda.current_device()
    for t in tensors:
        if t is not None and t.get_device() != device:
            raise PositError("a tensor is on device %s, the current one is %d" % (t.device, device))


def _rows_of_heads(t, fmt, name, shape=None):
    """(pointer, stride of rows, stride of heads) of [rows][heads][elements]."""
    if not isinstance(t, torch.Tensor) or t.dim() != 3 or (shape is not None and tuple(t.shape) != tuple(shape)):
        raise PositError("%s must be [rows][heads][elements]%s" % (name, "" if shape is None else " of %s" % (tuple(shape),)))
    return _ptr(t, fmt, name), t.stride(0), t.stride(1)


def _head_weight(w, fmt, d, name):
    if w is None:
        return None
    if not isinstance(w, torch.Tensor) or w.numel() != d or not w.is_contiguous():
        raise PositError("%s must be a dense device tensor of %d values" % (name, d))
    return _ptr(w, fmt, name)


def _frequencies(inv_freq, d):
    """(pointer, rotated elements)."""
    if inv_freq is None:
        return None, 0
    if not isinstance(inv_freq, torch.Tensor) or 2 * inv_freq.numel() > d:
        raise PositError("inv_freq must hold a value for each of at most %d pairs" % (d // 2))
    return _vector(inv_freq, torch.float64, inv_freq.numel(), "inv_freq"), 2 * inv_freq.numel()


def rope_frequencies(rotated, base=10000.0, device="cuda"):
    """base^(-2i / rotated) for the pairs 0 <= i < rotated / 2, in binary64: what the rotations take as inv_freq."""
    return float(base) ** (torch.arange(rotated // 2, dtype=torch.float64, device=device) * (-2.0 / rotated))


def _heads(q, k, fx, positions, inv_freq, wq, wk, fw, neighbours, eps):
    """(description, pointers of q, k, wq, wk, positions, inv_freq)."""
    qp, ql, qh = _rows_of_heads(q, fx, "q")
    t, hq, d = q.shape
    kp, kl, kh, hkv = None, 0, 0, 0
    if k is not None:
        kp, kl, kh = _rows_of_heads(k, fx, "k", (t, k.shape[1] if isinstance(k, torch.Tensor) and k.dim() == 3 else 0, d))
        hkv = k.shape[1]
    if (positions is None) != (inv_freq is None):
        raise PositError("positions and inv_freq go together")
    if (wq is None) != (wk is None) and k is not None:
        raise PositError("wq and wk go together")
    fp, rotated = _frequencies(inv_freq, d)
    _here(q, k, positions, inv_freq, wq, wk)
    desc = HeadsDesc(t, hq, hkv, d, rotated, ql, qh, kl, kh, 0, 0, 0, 0, 1 if neighbours else 0, eps)
    return desc, qp, kp, _head_weight(wq, fw, d, "wq"), _head_weight(wk, fw, d, "wk"), _vector(positions, torch.int32, t, "positions"), fp


def posit_qk_norm_rope_fwd(q, k, fx, fy, positions=None, inv_freq=None, wq=None, wk=None, fw=None, eps=1e-6, neighbours=False):
    """(yq, yk, rstd) for q [rows][heads][elements] and k (may be None): each head normalised (with wq and wk) and its first elements rotated by the row's position
    (with positions and inv_freq).  rstd [rows][heads of q, then of k] is None without norm."""
    fx, fy = _code(fx), _code(fy)
    fw = fx if fw is None else _code(fw)
    native, st, dev = _ready()
    if native is not None:
        r = native.heads_fwd(st, dev, fx, fw, fy, 1 if neighbours else 0, float(eps), q, k, wq, wk, positions, inv_freq)
        if r is not None:
            return _returned(r)
    desc, qp, kp, wqp, wkp, pp, fp = _heads(q, k, fx, positions, inv_freq, wq, wk, fw, neighbours, eps)
    yq = torch.empty(q.shape, dtype=_dtype(fy), device=q.device)
    yk = None if k is None else torch.empty(k.shape, dtype=_dtype(fy), device=q.device)
    rstd = None if wq is None else torch.empty((desc.T, desc.HQ + desc.HKV), dtype=torch.float32, device=q.device)
    _check(_load().posit_qk_norm_rope_fwd(_stream(), fx, fw, fy, ctypes.byref(desc), qp, kp, wqp, wkp, pp, fp, yq.data_ptr(), None if yk is None else yk.data_ptr(),
                                          None if rstd is None else rstd.data_ptr()))
    return yq, yk, rstd


def posit_qk_norm_rope_bwd(dyq, dyk, q, k, rstd, fd, fx, fdx, positions=None, inv_freq=None, wq=None, wk=None, fw=None, fdw="f32", neighbours=False, want_dw=True, workspace=None):
    """(dq, dk, dwq, dwk) for the gradients dyq and dyk of the outputs; q, k and rstd as the forward call took and returned them.  dwq and dwk are None without norm."""
    fd, fx, fdx, fdw = _code(fd), _code(fx), _code(fdx), _code(fdw)
    fw = fx if fw is None else _code(fw)
    native, st, dev = _ready()
    if native is not None and workspace is None:
        r = native.heads_bwd(st, dev, fd, fx, fw, fdx, fdw, (1 if neighbours else 0) | (2 if want_dw else 0), dyq, dyk, q, k, wq, wk, positions, inv_freq, rstd)
        if r is not None:
            return _returned(r)
    desc, qp, kp, wqp, wkp, pp, fp = _heads(q, k, fx, positions, inv_freq, wq, wk, fw, neighbours, 0.0)
    gqp, desc.gql, desc.gqh = _rows_of_heads(dyq, fd, "dyq", q.shape)
    gkp = None
    if k is not None:
        gkp, desc.gkl, desc.gkh = _rows_of_heads(dyk, fd, "dyk", k.shape)
    _here(dyq, dyk if k is not None else None, rstd)
    dev, want = q.device, want_dw and wq is not None
    dq = torch.empty(q.shape, dtype=_dtype(fdx), device=dev)
    dk = None if k is None else torch.empty(k.shape, dtype=_dtype(fdx), device=dev)
    make = torch.zeros if desc.T == 0 or desc.HQ + desc.HKV == 0 else torch.empty  # sums over nothing
    dwq = make((desc.D,), dtype=_dtype(fdw), device=dev) if want else None
    dwk = make((desc.D,), dtype=_dtype(fdw), device=dev) if want and k is not None else None
    L = _load()
    wp, wbytes, _keep = _work(L.posit_qk_norm_rope_bwd_workspace(ctypes.byref(desc)) if want else 0, dev, workspace)
    _check(L.posit_qk_norm_rope_bwd(_stream(), fd, fx, fw, fdx, fdw, ctypes.byref(desc), gqp, gkp, qp, kp, wqp, wkp,
                                    _vector(rstd, torch.float32, desc.T * (desc.HQ + desc.HKV), "rstd") if wq is not None else None, pp, fp, dq.data_ptr(),
                                    None if dk is None else dk.data_ptr(), None if dwq is None else dwq.data_ptr(), None if dwk is None else dwk.data_ptr(), wp, wbytes))
    return dq, dk, dwq, dwk


# ---- the cache in pages ----

def _per_token(fcache, d):
    """Elements (bytes of "f4") that a token of one head takes in a page."""
    return d // 2 + (d + 31) // 32 if fcache == F4 else d


def _cache_dtype(fcache):
    return torch.uint8 if fcache == F4 else _dtype(fcache)


def posit_cache_pages(pages, heads, page, d, fcache, device="cuda"):
    """(keys, values): two tensors of `pages` pages of `page` tokens in fcache, zeros."""
    fcache = _code(fcache)
    shape = (pages, heads, page * _per_token(fcache, d))
    return tuple(torch.zeros(shape, dtype=_cache_dtype(fcache), device=device) for _ in range(2))


def _cache(pages_k, pages_v, table, lens, starts, fcache, hkv, d, rows):
    """(description with the cache's part filled in, pointers of k_pages, v_pages, table, lens, starts)."""
    if not isinstance(table, torch.Tensor) or table.dim() != 2 or table.dtype != torch.int32 or not table.is_cuda or (table.shape[1] > 1 and table.stride(1) != 1):
        raise PositError("table must be a device tensor [sequences][pages] of int32")
    b, per = table.shape[0], _per_token(fcache, d)
    shape = None
    for t, name in ((pages_k, "pages_k"), (pages_v, "pages_v")):
        if not isinstance(t, torch.Tensor) or t.dim() != 3 or not t.is_contiguous() or t.shape[1] != hkv or per == 0 or t.shape[2] == 0 or t.shape[2] % per:
            raise PositError("%s must be a dense tensor [pages][%d heads][elements of a page]" % (name, hkv))
        _ptr(t, fcache if fcache != F4 else binding.P8, name)
        if shape is not None and t.shape != shape:
            raise PositError("pages_k and pages_v have shapes %s and %s" % (tuple(shape), tuple(t.shape)))
        shape = t.shape
    if starts is None and rows is not None and rows != b:
        raise PositError("%d rows for %d sequences: starts says whose they are" % (rows, b))
    _here(pages_k, pages_v, table, lens, starts)
    desc = PagedDesc(T=rows or 0, B=b, HKV=hkv, D=d, page=shape[2] // per, pages=shape[0], columns=table.shape[1], pitch=table.stride(0) if b > 1 else table.shape[1])
    return desc, pages_k.data_ptr(), pages_v.data_ptr(), table.data_ptr(), _vector(lens, torch.int32, b, "lens"), _vector(starts, torch.int32, b + 1, "starts")


def posit_cache_append(k, v, pages_k, pages_v, table, lens, fx, fcache, starts=None, q=None, fq=None, inv_freq=None, wq=None, wk=None, fw=None, eps=1e-6, neighbours=False):
    """Puts the rows k and v [rows][heads][elements] into the pages as the last of their sequences' lens tokens, k normalised and rotated; returns q likewise (in fq), or
    None without one.  starts [sequences + 1]: first row of each; None for one row each."""
    fx, fcache = _code(fx), _code(fcache)
    fw, fq = fx if fw is None else _code(fw), fx if fq is None else _code(fq)
    native, st, dev = _ready()
    if native is not None:
        r = native.cache_append(st, dev, fx, fw, fq, fcache, 1 if neighbours else 0, float(eps), k, v, pages_k, pages_v, table, lens, starts, q, inv_freq, wq, wk)
        if r is not None:
            return _returned(r)[0]
    kp, kl, kh = _rows_of_heads(k, fx, "k")
    rows, hkv, d = k.shape
    vp, vl, vh = _rows_of_heads(v, fx, "v", k.shape)
    desc, kc, vc, tp, lp, sp = _cache(pages_k, pages_v, table, lens, starts, fcache, hkv, d, rows)
    if lp is None:
        raise PositError("lens must be given")
    desc.kl, desc.kh, desc.vl, desc.vh, desc.eps, desc.neighbours = kl, kh, vl, vh, eps, 1 if neighbours else 0
    fp, desc.R = _frequencies(inv_freq, d)
    qp = yq = None
    if q is not None:
        qp, desc.ql, desc.qh = _rows_of_heads(q, fx, "q", (rows, q.shape[1] if isinstance(q, torch.Tensor) and q.dim() == 3 else 0, d))
        desc.HQ = q.shape[1]
        yq = torch.empty(q.shape, dtype=_dtype(fq), device=k.device)
    if wk is None and wq is not None or q is not None and wk is not None and wq is None:
        raise PositError("wq and wk go together")
    _here(k, v, q, inv_freq, wq, wk)
    _check(_load().posit_cache_append(_stream(), fx, fw, fq, fcache, ctypes.byref(desc), qp, kp, vp, _head_weight(wq, fw, d, "wq"), _head_weight(wk, fw, d, "wk"), fp, sp, lp, tp,
                                      kc, vc, None if yq is None else yq.data_ptr()))
    return yq


def posit_cache_read(pages_k, pages_v, table, lens, longest, d, fcache, fout):
    """(k, v) [sequences][longest][heads][d] in fout of what the pages hold; zeros behind a sequence's end."""
    fcache, fout = _code(fcache), _code(fout)
    native, st, dev = _ready()
    if native is not None:
        r = native.cache_read(st, dev, longest, d, fcache, fout, pages_k, pages_v, table, lens, None)
        if r is not None:
            return _returned(r)
    if not isinstance(pages_k, torch.Tensor) or pages_k.dim() != 3:
        raise PositError("pages_k must be [pages][heads][elements of a page]")
    hkv = pages_k.shape[1]
    desc, kc, vc, tp, lp, _ = _cache(pages_k, pages_v, table, lens, None, fcache, hkv, d, None)
    if lp is None:
        raise PositError("lens must be given")
    desc.longest = longest
    k, v = (torch.empty((desc.B, max(longest, 0), hkv, d), dtype=_dtype(fout), device=table.device) for _ in range(2))
    _check(_load().posit_cache_read(_stream(), fcache, fout, ctypes.byref(desc), lp, tp, kc, vc, k.data_ptr(), v.data_ptr()))
    return k, v


def posit_attention_paged_workspace(desc):
    return int(_load().posit_attention_paged_workspace(ctypes.byref(desc)))


def posit_attention_paged(q, pages_k, pages_v, table, lens, fq, fcache, fout, longest=None, starts=None, most=1, scale=None, window=0, sinks=0, workspace=None):
    """(o [rows][heads][elements], lse [rows][heads]) of the rows q over their sequences' pages.  starts [sequences + 1]: first row of each; None for one row each.  `longest`
    bounds lens (None: what the table holds), `most` the rows of a sequence; scale: 1 / sqrt(elements) by default."""
    fq, fcache, fout = _code(fq), _code(fcache), _code(fout)
    native, st, dev = _ready()
    if native is not None and workspace is None and isinstance(q, torch.Tensor) and q.dim() == 3:
        r = native.attention_paged(st, dev, fq, fcache, fout, most, window, sinks, 1.0 / math.sqrt(max(q.shape[2], 1)) if scale is None else float(scale), q, pages_k, pages_v, table, lens,
                                   starts, longest)
        if r is not None:
            return _returned(r)
    qp, ql, qh = _rows_of_heads(q, fq, "q")
    rows, hq, d = q.shape
    if not isinstance(pages_k, torch.Tensor) or pages_k.dim() != 3:
        raise PositError("pages_k must be [pages][heads][elements of a page]")
    desc, kc, vc, tp, lp, sp = _cache(pages_k, pages_v, table, lens, starts, fcache, pages_k.shape[1], d, rows)
    if lp is None:
        raise PositError("lens must be given")
    desc.HQ, desc.ql, desc.qh, desc.window, desc.sinks, desc.most = hq, ql, qh, window, sinks, most
    desc.longest = desc.columns * desc.page if longest is None else longest
    desc.scale = 1.0 / math.sqrt(max(d, 1)) if scale is None else float(scale)
    _here(q)
    o = torch.empty((rows, hq, d), dtype=_dtype(fout), device=q.device)
    lse = torch.empty((rows, hq), dtype=torch.float32, device=q.device)
    L = _load()
    wp, wbytes, _keep = _work(L.posit_attention_paged_workspace(ctypes.byref(desc)), q.device, workspace)
    _check(L.posit_attention_paged(_stream(), fq, fcache, fout, ctypes.byref(desc), qp, sp, lp, tp, kc, vc, o.data_ptr(), lse.data_ptr(), wp, wbytes))
    return o, lse


# ---- the draw ----

def posit_sample(logits, u, fz, temperature=None, top_k=None, top_p=None, min_p=None, workspace=None):
    """(token, logprob, kept) for each row of logits from u, one number from 0 to 1 each; the limits are a value per row, or None."""
    fz = _code(fz)
    native, st, dev = _ready()
    if native is not None and workspace is None:
        r = native.sample(st, dev, fz, logits, u, temperature, top_k, top_p, min_p)
        if r is not None:
            return _returned(r)
    if not isinstance(logits, torch.Tensor) or logits.dim() != 2:
        raise PositError("logits must be a 2-D tensor")
    zp = _ptr(logits, fz, "logits")
    rows, vocab = logits.shape
    if vocab == 0 and rows > 0:
        raise PositError("logits have no columns")
    if u is None:
        raise PositError("u must be given")
    _here(logits, u, temperature, top_k, top_p, min_p)
    f32 = torch.float32
    token, kept = (torch.empty((rows,), dtype=torch.int32, device=logits.device) for _ in range(2))
    logprob = torch.empty((rows,), dtype=f32, device=logits.device)
    L = _load()
    wp, wbytes, _keep = _work(L.posit_sample_workspace(fz, rows, vocab), logits.device, workspace)
    _check(L.posit_sample(_stream(), fz, rows, vocab, zp, logits.stride(0) if rows > 1 else vocab, _vector(u, f32, rows, "u"), _vector(temperature, f32, rows, "temperature"),
                          _vector(top_k, torch.int32, rows, "top_k"), _vector(top_p, f32, rows, "top_p"), _vector(min_p, f32, rows, "min_p"), token.data_ptr(), logprob.data_ptr(),
                          kept.data_ptr(), wp, wbytes))
    return token, logprob, kept
