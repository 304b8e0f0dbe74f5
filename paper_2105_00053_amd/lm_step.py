"""Device-resident step of a one-layer token model: training over sequences, and decoding with a cache.

Chains the operators of lm.py with the products of the library: tokens -> rows of a fixed table -> RMS norm -> q, k, v in one product ->
attention with a sliding window and sinks -> product -> residual's addition and RMS norm -> logits -> log probabilities of the next tokens; and
back.  Pure orchestration, as train_step.py: every number is produced by a kernel of libpositnn_hip.so; torch moves data (rows of the
table, a token's keys and values into their cache, dq, dk and dv side by side).

Formats: activations, weight copies, the cache and back-propagated errors in `compute`; the residual, the norms' weights, the master weights and
their gradients in `master`; logits in `loss`.  Errors of single tokens lie far below one where 8-bit posits are coarse, so the loss is scaled by a
power of two that the update divides by.  The table is not trained: the library has no addition of rows by index.
"""
import torch

from . import binding as pn
from . import lm


def _movable(t):
    """The same patterns in a type that torch indexes by: it has no such kernels for unsigned 16 bits."""
    return t.view(torch.int16) if t.dtype == torch.uint16 else t


class TokenNet:
    """Weights from float tensors: table [vocab][dim], qkv [(heads + 2 kv_heads) * d][dim], out [dim][heads * d], head [vocab][dim]; norm weights start at one."""

    def __init__(self, table, qkv, out, head, heads, kv_heads, window=0, sinks=0, compute="p8_2", master="p16", loss="p16", eps=1e-6):
        self.heads, self.kv_heads, self.d = heads, kv_heads, out.shape[1] // heads
        self.window, self.sinks, self.eps = window, sinks, eps
        self.compute, self.master, self.loss = compute, master, loss
        self.table = _movable(pn.posit_round(table.contiguous(), master))
        self.w = [pn.posit_round(t.contiguous(), master) for t in (qkv, out, head)]
        self.copies = [pn.posit_convert(t, master, compute) for t in self.w]
        self.norms = [pn.posit_round(torch.ones(table.shape[1], device=table.device), master) for _ in range(2)]

    def pattern(self, value):
        """Pattern of a number in the master format, rounded by the library."""
        raw = pn.posit_round(torch.tensor([value], dtype=torch.float32, device=self.table.device), self.master)
        return int.from_bytes(raw.cpu().contiguous().view(torch.uint8).numpy().tobytes(), "little")

    def split(self, qkv, batch, length):
        """Views of q [b][i][h][d], k and v [b][j][h'][d] in the rows of their product."""
        x = qkv.view(batch, length, self.heads + 2 * self.kv_heads, self.d)
        return x[:, :, :self.heads], x[:, :, self.heads:self.heads + self.kv_heads], x[:, :, self.heads + self.kv_heads:]


def _project(net, tokens):
    """(rows of the table, normalised rows, 1 / rms, their q, k and v side by side)."""
    fc, fm = net.compute, net.master
    x = net.table[tokens.reshape(-1).long()]
    y, _, _, rstd = lm.posit_rmsnorm_fwd(x, net.norms[0], fm, fm, fc, net.eps)
    return x, y, rstd, pn.posit_gemm(y, net.copies[0], fc, fc, trans_b=True)


def _read_out(net, x, o):
    """(residual, normalised rows, 1 / rms, logits) behind the attention's output o [rows][heads * d]."""
    fc, fm = net.compute, net.master
    z = pn.posit_gemm(o, net.copies[1], fc, fc, trans_b=True)
    y, _, h, rstd = lm.posit_rmsnorm_fwd(z, net.norms[1], fc, fm, fc, net.eps, res=x, fres=fm)
    return h, y, rstd, pn.posit_gemm(y, net.copies[2], fc, net.loss, trans_b=True)


def gradients(net, tokens, targets, loss_scale=64.0):
    """(log probabilities [b][l], gradients of the three matrices and the two norm weights in the master format, of minus their sum times loss_scale).
    tokens, targets: [b][l] int32; a negative target counts nothing."""
    fc, fm, fl = net.compute, net.master, net.loss
    b, l = tokens.shape
    x, y1, rstd1, qkv = _project(net, tokens)
    q, k, v = net.split(qkv, b, l)
    how = dict(window=net.window, sinks=net.sinks)
    # the products read o as it is; the backward pass takes rowsum(dO * o) from a copy in binary32, since all score gradients of a row share its error
    o, lse, o_copy = lm.posit_attention_fwd(q, k, v, fc, fc, fc, fcopy="f32", **how)
    h, y2, rstd2, logits = _read_out(net, x, o.view(b * l, -1))
    targets = targets.reshape(-1)
    logprob, z_lse, entropy, _, _ = lm.posit_token_logprob_fwd(logits, targets, fl)

    g = torch.full((b * l,), -loss_scale, dtype=torch.float32, device=tokens.device)
    dz = lm.posit_token_logprob_bwd(logits, targets, z_lse, entropy, g, None, fl, fc)
    dhead = pn.posit_gemm(dz, y2, fc, fm, trans_a=True)
    dh, dnorm2 = lm.posit_rmsnorm_bwd(pn.posit_gemm(dz, net.copies[2], fc, fc), h, net.norms[1], rstd2, fc, fm, fm, fc, fm)
    dout = pn.posit_gemm(dh, o.view(b * l, -1), fc, fm, trans_a=True)
    do = pn.posit_gemm(dh, net.copies[1], fc, fc).view(o.shape)
    dqkv = torch.cat([_movable(t) for t in lm.posit_attention_bwd(do, q, k, v, o_copy, lse, fc, fc, fc, "f32", fc, **how)], dim=2).view(b * l, -1)
    dw = pn.posit_gemm(dqkv, y1, fc, fm, trans_a=True)
    _, dnorm1 = lm.posit_rmsnorm_bwd(pn.posit_gemm(dqkv, net.copies[0], fc, fc), x, net.norms[0], rstd1, fc, fm, fm, fc, fm)
    return logprob.view(b, l), [dw, dout, dhead], [dnorm1, dnorm2]


def training_step(net, tokens, targets, rate, loss_scale=64.0):
    """One step of gradient descent on minus the log probabilities' sum; returns them."""
    logprob, dws, dnorms = gradients(net, tokens, targets, loss_scale)
    alpha = net.pattern(-rate / loss_scale)
    pn.posit_axpy_multi(alpha, dws + dnorms, net.w + net.norms, net.master, net.master, fcopy=net.compute, y_copies=net.copies + [None, None])
    return logprob


class Decoder:
    """A cache of keys and values in the compute format, and the step that appends a token to each sequence."""

    def __init__(self, net, batch, most):
        self.net = net
        self.k = torch.zeros((batch, most, net.kv_heads, net.d), dtype=_movable(net.copies[0]).dtype, device=net.table.device)
        self.v = torch.zeros_like(self.k)
        self.lens = torch.zeros(batch, dtype=torch.int32, device=net.table.device)
        self.most, self.count = most, 0
        self.rows = torch.arange(batch, device=net.table.device)

    def step(self, tokens, top=1):
        """(log probabilities, indices) of the `top` likeliest next tokens behind tokens [b] int32."""
        if self.count >= self.most:
            raise pn.PositError("the cache holds %d tokens" % self.most)
        net, fc = self.net, self.net.compute
        x, _, _, qkv = _project(net, tokens)
        q, k, v = net.split(qkv, len(self.rows), 1)
        at = self.lens.long()
        self.k[self.rows, at], self.v[self.rows, at] = _movable(k)[:, 0], _movable(v)[:, 0]
        self.lens += 1
        self.count += 1
        o, _, _ = lm.posit_attention_fwd(q, self.k, self.v, fc, fc, fc, window=net.window, sinks=net.sinks, lens=self.lens)
        _, _, _, logits = _read_out(net, x, o.view(len(self.rows), -1))
        _, _, _, logprob, index = lm.posit_token_logprob_fwd(logits, None, net.loss, top=top)
        return logprob, index
