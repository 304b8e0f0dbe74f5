"""Device-resident step of a one-layer token model: training over sequences, decoding with a cache, and generating with a cache in pages.

Chains the operators of lm.py and generate.py with the products of the library: tokens -> rows of a fixed table -> RMS norm -> q, k, v in one product ->
(norms of their heads and rotation by positions, where the net has them) -> attention with a sliding window and sinks -> product -> residual's addition and RMS norm -> logits -> log probabilities of the next tokens; and
back.  Pure orchestration, as train_step.py: every number is produced by a kernel of libpositnn_hip.so; torch moves data (rows of the
table, a token's keys and values into their cache, dq, dk and dv side by side).

Formats: activations, weight copies, the cache and back-propagated errors in `compute`; the residual, the norms' weights, the master weights and
their gradients in `master`; logits in `loss`.  Errors of single tokens lie far below one where 8-bit posits are coarse, so the loss is scaled by a
power of two that the update divides by.  The table is not trained: the library has no addition of rows by index.
"""
import torch

from . import binding as pn
from . import generate, lm


def _movable(t):
    """The same patterns in a type that torch indexes by: it has no such kernels for unsigned 16 bits."""
    return t.view(torch.int16) if t.dtype == torch.uint16 else t


class TokenNet:
    """Weights from float tensors: table [vocab][dim], qkv [(heads + 2 kv_heads) * d][dim], out [dim][heads * d], head [vocab][dim]; norm weights start at one.
    rotated: the first elements of each query and key head that are rotated by the token's position (0: none); head_norms: whether these heads are normalised."""

    def __init__(self, table, qkv, out, head, heads, kv_heads, window=0, sinks=0, compute="p8_2", master="p16", loss="p16", eps=1e-6, rotated=0, head_norms=False, base=10000.0):
        self.heads, self.kv_heads, self.d = heads, kv_heads, out.shape[1] // heads
        self.window, self.sinks, self.eps = window, sinks, eps
        self.compute, self.master, self.loss = compute, master, loss
        self.table = _movable(pn.posit_round(table.contiguous(), master))
        self.w = [pn.posit_round(t.contiguous(), master) for t in (qkv, out, head)]
        self.copies = [pn.posit_convert(t, master, compute) for t in self.w]
        self.norms = [pn.posit_round(torch.ones(table.shape[1], device=table.device), master) for _ in range(2)]
        self.inv_freq = generate.rope_frequencies(rotated, base, table.device) if rotated else None
        self.head_norms = [pn.posit_round(torch.ones(self.d, device=table.device), master) if head_norms else None for _ in range(2)]

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


def _turned(net, qkv, batch, length):
    """q, k, v of whole sequences as attention takes them, what the norms' gradients need (None where the net has neither norms nor rotation), and how the heads were turned."""
    q, k, v = net.split(qkv, batch, length)
    if net.inv_freq is None and net.head_norms[0] is None:
        return q, k, v, None, None
    fc, rows = net.compute, batch * length
    how = dict(inv_freq=net.inv_freq, wq=net.head_norms[0], wk=net.head_norms[1], fw=net.master)
    if net.inv_freq is not None:
        how["positions"] = torch.arange(length, dtype=torch.int32, device=qkv.device).repeat(batch)
    heads = qkv.view(rows, net.heads + 2 * net.kv_heads, net.d)
    given = heads[:, :net.heads], heads[:, net.heads:net.heads + net.kv_heads]
    yq, yk, rstd = generate.posit_qk_norm_rope_fwd(*given, fc, fc, eps=net.eps, **how)
    return yq.view(q.shape), yk.view(k.shape), v, (*given, rstd), how


def _read_out(net, x, o):
    """(residual, normalised rows, 1 / rms, logits) behind the attention's output o [rows][heads * d]."""
    fc, fm = net.compute, net.master
    z = pn.posit_gemm(o, net.copies[1], fc, fc, trans_b=True)
    y, _, h, rstd = lm.posit_rmsnorm_fwd(z, net.norms[1], fc, fm, fc, net.eps, res=x, fres=fm)
    return h, y, rstd, pn.posit_gemm(y, net.copies[2], fc, net.loss, trans_b=True)


def gradients(net, tokens, targets, loss_scale=64.0):
    """(log probabilities [b][l], gradients of the three matrices and of the norm weights (two, then those of the heads' norms, where the net has them) in the master format, of minus
    their sum times loss_scale).  tokens, targets: [b][l] int32; a negative target counts nothing."""
    fc, fm, fl = net.compute, net.master, net.loss
    b, l = tokens.shape
    x, y1, rstd1, qkv = _project(net, tokens)
    q, k, v, given, turned = _turned(net, qkv, b, l)
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
    dq, dk, dv = lm.posit_attention_bwd(do, q, k, v, o_copy, lse, fc, fc, fc, "f32", fc, **how)
    dheads = []
    if given is not None:
        dq, dk, *dheads = generate.posit_qk_norm_rope_bwd(dq.view(b * l, net.heads, net.d), dk.view(b * l, net.kv_heads, net.d), *given, fc, fc, fc, fdw=fm, **turned)
        dq, dk = dq.view(q.shape), dk.view(k.shape)
    dqkv = torch.cat([_movable(t) for t in (dq, dk, dv)], dim=2).view(b * l, -1)
    dw = pn.posit_gemm(dqkv, y1, fc, fm, trans_a=True)
    _, dnorm1 = lm.posit_rmsnorm_bwd(pn.posit_gemm(dqkv, net.copies[0], fc, fc), x, net.norms[0], rstd1, fc, fm, fm, fc, fm)
    return logprob.view(b, l), [dw, dout, dhead], [dnorm1, dnorm2] + [t for t in dheads if t is not None]


def training_step(net, tokens, targets, rate, loss_scale=64.0):
    """One step of gradient descent on minus the log probabilities' sum; returns them."""
    logprob, dws, dnorms = gradients(net, tokens, targets, loss_scale)
    alpha = net.pattern(-rate / loss_scale)
    norms = net.norms + [w for w in net.head_norms if w is not None]
    pn.posit_axpy_multi(alpha, dws + dnorms, net.w + norms, net.master, net.master, fcopy=net.compute, y_copies=net.copies + [None] * len(norms))
    return logprob


class Decoder:
    """A cache of keys and values in the compute format, and the step that appends a token to each sequence."""

    def __init__(self, net, batch, most):
        if net.inv_freq is not None or net.head_norms[0] is not None:
            raise pn.PositError("a net whose heads are rotated or normalised decodes with PagedDecoder")
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


class PagedDecoder:
    """A cache in pages for sequences that come and go, and the step that takes packed tokens of any of them: the next ones of running sequences and whole prompts of new ones in
    one call.  Queries and keys are rotated and normalised as in the training step, where the net says so.  cache: a format of generate.py's; by default the compute format, or bfloat16 where
    that has more than 8 bits."""

    def __init__(self, net, pages, page=64, cache=None):
        self.net, self.page = net, page
        self.cache = (net.compute if pn.FORMAT_BITS[net.compute] == 8 else "bf16") if cache is None else cache
        self.k, self.v = generate.posit_cache_pages(pages, net.kv_heads, page, net.d, self.cache, device=net.table.device)
        self.free = list(range(pages - 1, -1, -1))
        self.held = {}   # pages and tokens of each sequence, by the name that its caller gave

    def length(self, name):
        return self.held[name][1] if name in self.held else 0

    def drop(self, name):
        """Forgets a sequence; its pages are free again."""
        self.free.extend(reversed(self.held.pop(name)[0]))

    def step(self, new, most_rows=64):
        """Logits behind the last new token of each sequence, in the order of new = {name: its tokens, a list of one or more}; sequences that are not known begin.  Rows that share a key head with
        at most `most_rows` others of their sequence read the pages themselves; where there are more, as for prompts, the pages are read back and go through posit_attention_fwd.  A step that is
        refused leaves the sequences and the free pages as they were."""
        logits, *after = self._run(new, most_rows)
        self._take(*after)
        return logits

    def _take(self, held, left):
        """What a step leaves: its sequences' pages and tokens, and how many of the free pages."""
        self.held.update(held)
        del self.free[left:]

    def _run(self, new, most_rows=64):
        """(logits, and what _take makes of the state behind them); the state stays."""
        net, fc, dev = self.net, self.net.compute, self.net.table.device
        if not new or not all(len(tokens) for tokens in new.values()):
            raise pn.PositError("a step takes one token or more of each of its sequences")
        # an index beyond the table would end the process on the device, and -1, which a draw without candidates gives, would be its last row
        vocab = net.table.shape[0]
        if any(min(tokens) < 0 or max(tokens) >= vocab for tokens in new.values()):
            raise pn.PositError("a token is none of the table's %d" % vocab)
        need = {name: -(-(self.length(name) + len(tokens)) // self.page) - len(self.held.get(name, ((), 0))[0]) for name, tokens in new.items()}
        if sum(need.values()) > len(self.free):
            raise pn.PositError("%d pages are free, the step takes %d" % (len(self.free), sum(need.values())))
        held, left = {}, len(self.free)
        for name, tokens in new.items():
            pages, n = self.held.get(name, ([], 0))
            held[name] = (pages + self.free[left - need[name]:left][::-1], n + len(tokens))
            left -= need[name]
        names, counts = list(new), [len(tokens) for tokens in new.values()]
        columns, longest, most = max(len(held[name][0]) for name in names), max(held[name][1] for name in names), max(counts)
        # one copy to the device: the table, lengths, first rows and tokens side by side
        flat = [p for name in names for p in held[name][0] + [-1] * (columns - len(held[name][0]))] + [held[name][1] for name in names]
        starts = [0]
        for c in counts:
            starts.append(starts[-1] + c)
        flat = torch.tensor(flat + starts + [t for tokens in new.values() for t in tokens], dtype=torch.int32).to(dev)
        b = len(names)
        table, lens = flat[:b * columns].view(b, columns), flat[b * columns:b * (columns + 1)]
        starts, tokens = flat[b * (columns + 1):b * (columns + 2) + 1], flat[b * (columns + 2) + 1:]
        x, _, _, qkv = _project(net, tokens)
        q, k, v = (t[0] for t in net.split(qkv, 1, len(tokens)))
        how = dict(inv_freq=net.inv_freq, wq=net.head_norms[0], wk=net.head_norms[1], fw=net.master, eps=net.eps)
        q = generate.posit_cache_append(k, v, self.k, self.v, table, lens, fc, self.cache, starts=starts, q=q, fq=fc, **how)
        if most * (net.heads // net.kv_heads) <= most_rows:
            o, _ = generate.posit_attention_paged(q, self.k, self.v, table, lens, fc, self.cache, fc, longest=longest, starts=starts, most=most, window=net.window, sinks=net.sinks)
        else:
            fkv = "bf16" if self.cache == "f4" else self.cache
            dense_k, dense_v = generate.posit_cache_read(self.k, self.v, table, lens, longest, net.d, self.cache, fkv)
            # the new rows of a sequence are its last ones: padded in front
            at = torch.cat([torch.arange(i * most + most - c, (i + 1) * most, device=dev) for i, c in enumerate(counts)])
            rows = torch.zeros((b * most, net.heads, net.d), dtype=_movable(q).dtype, device=dev)
            rows[at] = _movable(q)
            o, _, _ = lm.posit_attention_fwd(rows.view(b, most, net.heads, net.d), dense_k, dense_v, fc, fkv, fc, window=net.window, sinks=net.sinks, lens=lens)
            o = _movable(o).view(b * most, net.heads, net.d)[at]
        last = (starts[1:] - 1).long()
        _, _, _, logits = _read_out(net, x[last], _movable(o.reshape(len(tokens), -1))[last])
        return logits, held, left

    def sample(self, new, u, **limits):
        """(token, logprob, kept) of the draw behind each sequence's new tokens, in the order of `new`: u and the limits as posit_sample takes them."""
        logits, *after = self._run(new)
        drawn = generate.posit_sample(logits, u, self.net.loss, **limits)
        self._take(*after)
        return drawn
