"""Binding of include/positnn_lm.h: the RMS norm with the residual's addition, attention with a sliding window and
sinks, and the log probabilities of given tokens.

Argument marshalling only, as in binding.py; formats are its names or codes for posits of at most 16 bits, "f32" and, here
only, "bf16".  Tensors may be views: rows with a pitch, heads and positions with any strides, elements contiguous.
"""
import ctypes
import math

import torch

from . import binding
from .binding import ELEM_SIZE, FORMAT_CODES, PositError, TORCH_DTYPE, _SAME_SIZE, _check, _stream, load

BF16 = 102
_CODES = dict(FORMAT_CODES, bf16=BF16)
_DTYPES = dict(TORCH_DTYPE)
_DTYPES[BF16] = torch.bfloat16


class AttentionDesc(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int64) for n in ("B", "HQ", "HKV", "LQ", "LK", "D", "window", "sinks")] + [("scale", ctypes.c_float)] + [
        (n, ctypes.c_int64) for n in ("qb", "ql", "qh", "kb", "kl", "kh", "vb", "vl", "vh")]


_lib = None


def _load():
    """The shared library with the signatures of this header's functions."""
    global _lib
    if _lib is None:
        L = load()
        vp, i64, ci, sz, cf = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int, ctypes.c_size_t, ctypes.c_float
        dp = ctypes.POINTER(AttentionDesc)
        L.posit_rmsnorm_fwd.argtypes = [vp, ci, ci, ci, ci, i64, i64, vp, i64, vp, i64, vp, cf, vp, i64, vp, i64, vp, vp]
        L.posit_rmsnorm_bwd.argtypes = [vp, ci, ci, ci, ci, ci, ci, i64, i64, vp, i64, vp, i64, vp, vp, vp, i64, vp, i64, vp, vp, sz]
        L.posit_rmsnorm_bwd_workspace.argtypes = [i64, i64]
        L.posit_scale_rows.argtypes = [vp, ci, ci, i64, i64, vp, i64, vp, vp, i64]
        L.posit_attention_fwd.argtypes = [vp, ci, ci, ci, dp, vp, vp, vp, vp, vp, vp, ci, vp, vp, sz]
        L.posit_attention_bwd.argtypes = [vp, ci, ci, ci, ci, ci, dp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, sz]
        L.posit_attention_workspace.argtypes = [ci, ci, dp]
        L.posit_token_logprob_fwd.argtypes = [vp, ci, i64, i64, vp, i64, vp, cf, ci, vp, vp, vp, vp, vp, vp, sz]
        L.posit_token_logprob_workspace.argtypes = [ci, i64, i64, ci]
        L.posit_token_logprob_bwd.argtypes = [vp, ci, ci, i64, i64, vp, i64, vp, cf, vp, vp, vp, vp, vp, i64]
        for name in ("posit_rmsnorm_fwd", "posit_rmsnorm_bwd", "posit_scale_rows", "posit_attention_fwd", "posit_attention_bwd",
                     "posit_token_logprob_fwd", "posit_token_logprob_bwd"):
            getattr(L, name).restype = ci
        for name in ("posit_rmsnorm_bwd_workspace", "posit_attention_workspace", "posit_token_logprob_workspace"):
            getattr(L, name).restype = sz
        if binding._native is not None:
            binding._native.init_lm(*(ctypes.cast(getattr(L, name), vp).value for name in _NATIVE_ORDER))
        _lib = L
    return _lib


# As in binding.py, a call goes to the extension module first, which returns None for whatever it does not take.
_NATIVE_ORDER = ("posit_rmsnorm_fwd", "posit_rmsnorm_bwd", "posit_rmsnorm_bwd_workspace", "posit_scale_rows", "posit_attention_fwd", "posit_attention_bwd",
                 "posit_attention_workspace", "posit_token_logprob_fwd", "posit_token_logprob_workspace", "posit_token_logprob_bwd")


def _ready():
    """(the extension module, the current stream), or (None, None) where the Python code takes the call."""
    if _lib is None:
        _load()
    stream = binding._ready()
    return (None, None) if stream is None else (binding._native, stream)


def _returned(r):
    if r.__class__ is int:
        _check(r)
    return r


def _code(f):
    return _CODES[f] if isinstance(f, str) else int(f)


def _ptr(t, fmt, name):
    """Pointer of a device tensor whose last dimension is contiguous."""
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise PositError("%s must be a device tensor" % name)
    if fmt == BF16:
        if t.dtype not in (torch.bfloat16, torch.int16, torch.uint16):
            raise PositError("%s has dtype %s, expected bfloat16" % (name, t.dtype))
    elif fmt not in ELEM_SIZE or t.dtype not in _SAME_SIZE[ELEM_SIZE[fmt]]:
        raise PositError("%s has dtype %s, not that of format %d" % (name, t.dtype, fmt))
    if t.dim() and t.shape[-1] > 1 and t.stride(-1) != 1:
        raise PositError("%s must be contiguous along its last dimension" % name)
    return t.data_ptr()


def _vector(t, dtype, n, name):
    """Pointer of a dense device vector of n values, None for None."""
    if t is None:
        return None
    if not isinstance(t, torch.Tensor) or not t.is_cuda or t.dtype != dtype or t.numel() != n or not t.is_contiguous():
        raise PositError("%s must be a dense device tensor of %d values of %s" % (name, n, dtype))
    return t.data_ptr()


def _matrix(t, fmt, name, shape=None):
    """(pointer, pitch) of a 2-D tensor."""
    if not isinstance(t, torch.Tensor) or t.dim() != 2 or (shape is not None and tuple(t.shape) != tuple(shape)):
        raise PositError("%s must be a 2-D tensor%s" % (name, "" if shape is None else " of %d x %d" % tuple(shape)))
    return _ptr(t, fmt, name), (t.stride(0) if t.shape[0] > 1 else t.shape[1])


def _weight(w, fmt, n):
    if not isinstance(w, torch.Tensor) or w.numel() != n or not w.is_contiguous():
        raise PositError("w must be a dense device tensor of %d values" % n)
    return _ptr(w, fmt, "w")


def _work(nbytes, device, workspace):
    """(pointer, bytes, tensor to keep until the call is issued)."""
    if workspace is None:
        if nbytes == 0:
            return None, 0, None
        workspace = torch.empty(nbytes, dtype=torch.uint8, device=device)
    if not isinstance(workspace, torch.Tensor) or not workspace.is_cuda or not workspace.is_contiguous():
        raise PositError("workspace must be a dense device tensor")
    return workspace.data_ptr(), workspace.numel() * workspace.element_size(), workspace


def _dtype(fmt):
    if fmt not in _DTYPES:
        raise PositError("unknown format %r" % (fmt,))
    return _DTYPES[fmt]


def posit_rmsnorm_fwd(x, w, fx, fw, fy, eps=1e-6, res=None, fres=None, scaled=False):
    """(y, scale, res_out, rstd) of the RMS norm of x (+ res): scale is None unless `scaled`, res_out None without res."""
    fx, fw, fy = _code(fx), _code(fw), _code(fy)
    fres = fx if fres is None else _code(fres)
    native, st = _ready()
    if native is not None:
        r = native.rmsnorm_fwd(st, fx, fw, fy, fres, 1 if scaled else 0, float(eps), x, w, res)
        if r is not None:
            return _returned(r)
    xp, ldx = _matrix(x, fx, "x")
    rows, cols = x.shape
    if cols == 0 and rows > 0:
        raise PositError("x has no columns")
    res_out, rp, ldr, op, ldo = None, None, 0, None, 0
    if res is not None:
        rp, ldr = _matrix(res, fres, "res", x.shape)
        res_out = torch.empty((rows, cols), dtype=_dtype(fres), device=x.device)
        op, ldo = res_out.data_ptr(), cols
    y = torch.empty((rows, cols), dtype=_dtype(fy), device=x.device)
    stats = torch.empty((2 if scaled else 1, rows), dtype=torch.float32, device=x.device)
    _check(_load().posit_rmsnorm_fwd(_stream(), fx, fres, fw, fy, rows, cols, xp, ldx, rp, ldr, _weight(w, fw, cols), eps, op, ldo, y.data_ptr(), cols,
                                     stats[1].data_ptr() if scaled else None, stats.data_ptr()))
    return y, stats[1] if scaled else None, res_out, stats[0]


def posit_rmsnorm_bwd(dy, h, w, rstd, fd, fh, fw, fdx, fdw, dres=None, fdres=None, want_dw=True, workspace=None):
    """(dx, dw) for the gradient dy of the unscaled output; h is the normalised stream (res_out, or x), dres the gradient past the norm."""
    fd, fh, fw, fdx, fdw = _code(fd), _code(fh), _code(fw), _code(fdx), _code(fdw)
    fdres = fd if fdres is None else _code(fdres)
    native, st = _ready()
    if native is not None and workspace is None:
        r = native.rmsnorm_bwd(st, fd, fh, fw, fdx, fdw, fdres, 1 if want_dw else 0, dy, h, w, rstd, dres)
        if r is not None:
            return _returned(r)
    dp, lddy = _matrix(dy, fd, "dy")
    rows, cols = dy.shape
    hp, ldh = _matrix(h, fh, "h", dy.shape)
    rp, lddr = (None, 0) if dres is None else _matrix(dres, fdres, "dres", dy.shape)
    dx = torch.empty((rows, cols), dtype=_dtype(fdx), device=dy.device)
    dw = None
    if want_dw:
        dw = (torch.zeros if rows == 0 else torch.empty)((cols,), dtype=_dtype(fdw), device=dy.device)
    L = _load()
    wp, wbytes, _keep = _work(L.posit_rmsnorm_bwd_workspace(rows, cols) if want_dw else 0, dy.device, workspace)
    _check(L.posit_rmsnorm_bwd(_stream(), fd, fh, fw, fdres, fdx, fdw, rows, cols, dp, lddy, hp, ldh, _weight(w, fw, cols), _vector(rstd, torch.float32, rows, "rstd"),
                               rp, lddr, dx.data_ptr(), cols, dw.data_ptr() if want_dw else None, wp, wbytes))
    return dx, dw


def posit_scale_rows(x, scale, fin, fout):
    """scale[r] * x[r], rounded to fout."""
    fin, fout = _code(fin), _code(fout)
    native, st = _ready()
    if native is not None:
        r = native.scale_rows(st, fin, fout, x, scale)
        if r is not None:
            return _returned(r)
    xp, ldx = _matrix(x, fin, "x")
    rows, cols = x.shape
    y = torch.empty((rows, cols), dtype=_dtype(fout), device=x.device)
    _check(_load().posit_scale_rows(_stream(), fin, fout, rows, cols, xp, ldx, _vector(scale, torch.float32, rows, "scale"), y.data_ptr(), cols))
    return y


def _scale(scale, q):
    return 1.0 / math.sqrt(max(q.shape[3], 1)) if scale is None else float(scale)


def _attention(q, k, v, fq, fkv, scale, window, sinks, lens):
    for t, f, name in ((q, fq, "q"), (k, fkv, "k"), (v, fkv, "v")):
        if not isinstance(t, torch.Tensor) or t.dim() != 4:
            raise PositError("%s must be [batch][positions][heads][elements]" % name)
        _ptr(t, f, name)
    b, lq, hq, d = q.shape
    lk, hkv = k.shape[1:3]
    if tuple(k.shape) != (b, lk, hkv, d) or tuple(v.shape) != (b, lk, hkv, d):
        raise PositError("q, k and v have shapes %s, %s, %s" % (tuple(q.shape), tuple(k.shape), tuple(v.shape)))
    desc = AttentionDesc(b, hq, hkv, lq, lk, d, window, sinks, _scale(scale, q),
                         *q.stride()[:3], *k.stride()[:3], *v.stride()[:3])
    return desc, _vector(lens, torch.int32, b, "lens")


def posit_attention_workspace(which, fkv, desc):
    return int(_load().posit_attention_workspace(int(which), _code(fkv), ctypes.byref(desc)))


def posit_attention_fwd(q, k, v, fq, fkv, fout, scale=None, window=0, sinks=0, lens=None, fcopy=None, workspace=None):
    """(o, lse, o_copy) for q [b][i][h][d], k and v [b][j][h'][d]; o_copy is o rounded to fcopy, None without it.  scale: 1 / sqrt(d) by default."""
    fq, fkv, fout = _code(fq), _code(fkv), _code(fout)
    native, st = _ready()
    if native is not None and workspace is None and isinstance(q, torch.Tensor) and q.dim() == 4:
        r = native.attention_fwd(st, fq, fkv, fout, window, sinks, -1 if fcopy is None else _code(fcopy), _scale(scale, q), q, k, v, lens)
        if r is not None:
            return _returned(r)
    desc, lp = _attention(q, k, v, fq, fkv, scale, window, sinks, lens)
    b, lq, hq, d = q.shape
    if d == 0 and b * lq * hq > 0:
        raise PositError("heads have no elements")
    o = torch.empty((b, lq, hq, d), dtype=_dtype(fout), device=q.device)
    lse = torch.empty((b, hq, lq), dtype=torch.float32, device=q.device)
    copy = None if fcopy is None else torch.empty((b, lq, hq, d), dtype=_dtype(_code(fcopy)), device=q.device)
    L = _load()
    wp, wbytes, _keep = _work(L.posit_attention_workspace(0, fkv, ctypes.byref(desc)), q.device, workspace)
    _check(L.posit_attention_fwd(_stream(), fq, fkv, fout, ctypes.byref(desc), q.data_ptr(), k.data_ptr(), v.data_ptr(), lp, o.data_ptr(), lse.data_ptr(),
                                 0 if copy is None else _code(fcopy), None if copy is None else copy.data_ptr(), wp, wbytes))
    return o, lse, copy


def posit_attention_bwd(do, q, k, v, o, lse, fd, fq, fkv, fo, fout, scale=None, window=0, sinks=0, lens=None, workspace=None):
    """(dq, dk, dv) for the gradient do of the output; o (dense, in fo) and lse come from the forward call."""
    fd, fq, fkv, fo, fout = _code(fd), _code(fq), _code(fkv), _code(fo), _code(fout)
    native, st = _ready()
    if native is not None and workspace is None and isinstance(q, torch.Tensor) and q.dim() == 4:
        r = native.attention_bwd(st, fd, fq, fkv, fo, fout, window, sinks, _scale(scale, q), do, q, k, v, o, lse, lens)
        if r is not None:
            return _returned(r)
    desc, lp = _attention(q, k, v, fq, fkv, scale, window, sinks, lens)
    b, lq, hq, d = q.shape
    lk, hkv = k.shape[1:3]
    for t, f, name in ((do, fd, "do"), (o, fo, "o")):
        if not isinstance(t, torch.Tensor) or tuple(t.shape) != (b, lq, hq, d):
            raise PositError("%s must have the shape of q" % name)
        _ptr(t, f, name)
    if not o.is_contiguous():
        raise PositError("o must be contiguous")
    if tuple(do.stride()[:3]) != tuple(q.stride()[:3]):
        do = do.contiguous()
        if not q.is_contiguous():
            q = q.contiguous()
            desc.qb, desc.ql, desc.qh = q.stride()[:3]
    dq = torch.empty((b, lq, hq, d), dtype=_dtype(fout), device=q.device)
    dk, dv = (torch.empty((b, lk, hkv, d), dtype=_dtype(fout), device=q.device) for _ in range(2))
    L = _load()
    wp, wbytes, _keep = _work(L.posit_attention_workspace(1, fkv, ctypes.byref(desc)), q.device, workspace)
    _check(L.posit_attention_bwd(_stream(), fd, fq, fkv, fo, fout, ctypes.byref(desc), do.data_ptr(), q.data_ptr(), k.data_ptr(), v.data_ptr(), lp, o.data_ptr(),
                                 _vector(lse, torch.float32, b * hq * lq, "lse"), dq.data_ptr(), dk.data_ptr(), dv.data_ptr(), wp, wbytes))
    return dq, dk, dv


def posit_token_logprob_fwd(logits, targets, fz, inv_temperature=1.0, top=0, workspace=None):
    """(logprob, lse, entropy, top_logprob, top_index) of each row; logprob is None without targets, the last two without `top`."""
    fz = _code(fz)
    native, st = _ready()
    if native is not None and workspace is None:
        r = native.logprob_fwd(st, fz, top, float(inv_temperature), logits, targets)
        if r is not None:
            return _returned(r)
    zp, ldz = _matrix(logits, fz, "logits")
    rows, vocab = logits.shape
    if vocab == 0 and rows > 0:
        raise PositError("logits have no columns")
    tp = _vector(targets, torch.int32, rows, "targets")
    stats = torch.empty((3, rows), dtype=torch.float32, device=logits.device)
    top_lp = torch.empty((rows, top), dtype=torch.float32, device=logits.device) if top else None
    top_ix = torch.empty((rows, top), dtype=torch.int32, device=logits.device) if top else None
    L = _load()
    wp, wbytes, _keep = _work(L.posit_token_logprob_workspace(fz, rows, vocab, top), logits.device, workspace)
    at, step = stats.data_ptr(), 4 * rows
    _check(L.posit_token_logprob_fwd(_stream(), fz, rows, vocab, zp, ldz, tp, inv_temperature, top, at if tp is not None else None, at + step, at + 2 * step,
                                     top_lp.data_ptr() if top else None, top_ix.data_ptr() if top else None, wp, wbytes))
    return stats[0] if tp is not None else None, stats[1], stats[2], top_lp, top_ix


def posit_token_logprob_bwd(logits, targets, lse, entropy, g_logprob, g_entropy, fz, fg, inv_temperature=1.0):
    """Gradient with respect to the logits, for those of logprob and entropy (each may be None)."""
    fz, fg = _code(fz), _code(fg)
    native, st = _ready()
    if native is not None:
        r = native.logprob_bwd(st, fz, fg, float(inv_temperature), logits, targets, lse, entropy, g_logprob, g_entropy)
        if r is not None:
            return _returned(r)
    zp, ldz = _matrix(logits, fz, "logits")
    rows, vocab = logits.shape
    f32 = torch.float32
    dz = torch.empty((rows, vocab), dtype=_dtype(fg), device=logits.device)
    _check(_load().posit_token_logprob_bwd(_stream(), fz, fg, rows, vocab, zp, ldz, _vector(targets, torch.int32, rows, "targets"), inv_temperature,
                                           _vector(lse, f32, rows, "lse"), _vector(entropy, f32, rows, "entropy"), _vector(g_logprob, f32, rows, "g_logprob"),
                                           _vector(g_entropy, f32, rows, "g_entropy"), dz.data_ptr(), vocab))
    return dz
