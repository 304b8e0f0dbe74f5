"""Cases of the operators that a language model needs around its products: the RMS norm with the residual's addition, attention with
a sliding window and sinks, and the log probabilities of given tokens.

listed() holds the fixed cases, draw(rng) gives more of the same ranges.  A case is a dict of plain values:

  op "norm"      rows x cols; "pass" "fwd": res <- res + x, y <- norm(res) in 8-bit posits with a scale for each row, read back as
                 values; "train": forward and backward with a gradient that comes down the residual stream
  op "attn"      b sequences, hq query heads that share hkv key heads of size d; "pass" "token": lq = 1 query for each sequence on a
                 cache of lk keys, filled to lengths that fall from lk by the share `ragged`; "prompt": forward, lq = lk;
                 "train": forward and backward.  window 0 is none; `sinks` first tokens stay visible
  op "logprob"   rows x vocab logits; "pass" "fwd": log probability of each row's token, entropy, `top` alternatives; "train":
                 forward and the gradient with respect to the logits

Where `own` is false, run() computes the same in elementary operations on binary32.  Formats are named as in the binding ("p8_1" is
posit<8,1>); "bf16" is bfloat16 and "f32" binary32.  8- and 16-bit posits are given as their patterns.
"""
import math
import random

import numpy as np
import torch

own = False

EPS = 1e-6
POSITS = {"p8": (8, 0), "p8_1": (8, 1), "p8_2": (8, 2), "p10_1": (10, 1), "p10_2": (10, 2), "p12_1": (12, 1), "p12_2": (12, 2), "p16": (16, 1)}
BYTES = {"p8": 1, "p8_1": 1, "p8_2": 1, "p10_1": 2, "p10_2": 2, "p12_1": 2, "p12_2": 2, "p16": 2, "bf16": 2, "f32": 4}


def listed():
    return [
        # one new token for each of four sequences, between two products of a decoder layer: latency
        {"name": "norm_token_4x2048", "op": "norm", "pass": "fwd", "rows": 4, "cols": 2048, "fx": "p8_1", "fres": "p16", "fw": "p16", "fy": "p8_1"},
        # a prompt, odd on both sides, with the residual stream in bfloat16
        {"name": "norm_prompt_4099x5119", "op": "norm", "pass": "fwd", "rows": 4099, "cols": 5119, "fx": "p8_2", "fres": "bf16", "fw": "p12_2", "fy": "p8"},
        # a small training step
        {"name": "norm_train_500x1000", "op": "norm", "pass": "train", "rows": 500, "cols": 1000, "fx": "p8_2", "fres": "p16", "fw": "p16", "fy": "bf16"},
        # a training step of a wide model
        {"name": "norm_train_16384x4096", "op": "norm", "pass": "train", "rows": 16384, "cols": 4096, "fx": "p8_2", "fres": "p16", "fw": "p16", "fy": "bf16"},
        # single tokens of a small model on a short cache: latency
        {"name": "attn_token_3x300", "op": "attn", "pass": "token", "b": 3, "lq": 1, "lk": 300, "hq": 8, "hkv": 2, "d": 64, "window": 0, "sinks": 0,
         "ragged": 0.5, "fq": "bf16", "fkv": "p8_1", "fout": "bf16"},
        # single tokens of a batch in serving, on long caches of 8-bit posits of every length
        {"name": "attn_token_48x8192", "op": "attn", "pass": "token", "b": 48, "lq": 1, "lk": 8192, "hq": 32, "hkv": 8, "d": 128, "window": 4096, "sinks": 4,
         "ragged": 0.9, "fq": "bf16", "fkv": "p8_1", "fout": "bf16"},
        # a prompt with a window and sinks, no multiple of a tile
        {"name": "attn_prompt_2x4001", "op": "attn", "pass": "prompt", "b": 2, "lq": 4001, "lk": 4001, "hq": 16, "hkv": 4, "d": 128, "window": 1024, "sinks": 4,
         "ragged": 0.0, "fq": "p8_1", "fkv": "p8_1", "fout": "p8_1"},
        # a training step over whole sequences
        {"name": "attn_train_4x2048", "op": "attn", "pass": "train", "b": 4, "lq": 2048, "lk": 2048, "hq": 16, "hkv": 4, "d": 64, "window": 0, "sinks": 0,
         "ragged": 0.0, "fq": "p8_2", "fkv": "p8_2", "fout": "bf16"},
        # the token that was just sampled, with its alternatives: one row
        {"name": "logprob_token_1x100003", "op": "logprob", "pass": "fwd", "rows": 1, "vocab": 100003, "fz": "p16", "top": 20, "masked": 0.0},
        # a small batch whose decoder forbids most tokens
        {"name": "logprob_masked_32x5003", "op": "logprob", "pass": "fwd", "rows": 32, "vocab": 5003, "fz": "f32", "top": 5, "masked": 0.7},
        # scoring of a long text with 8-bit logits, which tie all the time
        {"name": "logprob_score_2048x50021", "op": "logprob", "pass": "fwd", "rows": 2048, "vocab": 50021, "fz": "p8_2", "top": 8, "masked": 0.0},
        # the end of a training step: loss and gradient
        {"name": "logprob_train_4096x32000", "op": "logprob", "pass": "train", "rows": 4096, "vocab": 32000, "fz": "p16", "top": 0, "masked": 0.0},
    ]


def _log(rng, lo, hi):
    """An integer spread over the logarithm of lo..hi, half of them as they fall, the others a multiple of 8 where they are long."""
    v = int(round(lo * (hi / lo) ** rng.random()))
    if rng.random() < 0.5 and v >= 64:
        v -= v % 8
    return max(lo, min(hi, v))


def draw(rng):
    op = rng.choice(["norm", "attn", "attn", "logprob"])
    if op == "norm":
        case = {"op": op, "pass": rng.choice(["fwd", "train"]), "rows": _log(rng, 1, 16384), "cols": _log(rng, 64, 8192),
                "fx": rng.choice(["p8", "p8_1", "p8_2", "bf16"]), "fres": rng.choice(["p16", "p16", "bf16", "f32"]), "fw": rng.choice(["p16", "p12_2", "f32"])}
        case["fy"] = rng.choice(["p8", "p8_1", "p8_2"]) if case["pass"] == "fwd" else "bf16"
        while case["rows"] * case["cols"] > 16384 * 4096:
            case["rows"] //= 2
        return case
    if op == "attn":
        which = rng.choice(["token", "prompt", "train"])
        hkv = rng.choice([1, 2, 4, 8])
        case = {"op": op, "pass": which, "b": _log(rng, 1, 48 if which == "token" else 8), "lq": 1, "lk": _log(rng, 16, 8192 if which == "token" else 4096),
                "hq": hkv * rng.choice([1, 2, 4, 5]), "hkv": hkv, "d": rng.choice([40, 64, 80, 96, 128]), "window": 0, "sinks": 0,
                "ragged": rng.choice([0.0, 0.5, 0.9]), "fq": rng.choice(["bf16", "p8_1", "p8_2"]), "fkv": rng.choice(["p8", "p8_1", "p8_2", "bf16"]),
                "fout": "bf16"}
        if rng.random() < 0.6:
            case["window"], case["sinks"] = _log(rng, 16, 2048), rng.choice([0, 1, 4, 16])
        if which != "token":
            case["fq"] = case["fkv"]
            if which == "prompt":
                case["fout"] = rng.choice(["bf16", "p8_1"])
            # at most the scores of the largest listed case of the same kind, and its operations
            most, d = (2 * 16 * 4001 * 4001, 128) if which == "prompt" else (4 * 16 * 2048 * 2048, 64)
            while case["b"] * case["hq"] * case["lk"] * case["lk"] * max(case["d"], d) > most * d:
                if case["b"] > 1:
                    case["b"] //= 2
                else:
                    case["lk"] = case["lk"] * 3 // 4
            case["lq"] = case["lk"]
        return case
    which = rng.choice(["fwd", "train"])
    case = {"op": op, "pass": which, "rows": _log(rng, 1, 4096), "vocab": _log(rng, 500, 131072), "fz": rng.choice(["p16", "p8_2", "p12_2", "bf16", "f32"]),
            "top": rng.choice([0, 1, 5, 20]) if which == "fwd" else 0, "masked": 0.0}
    if case["fz"] in ("bf16", "f32"):
        case["masked"] = rng.choice([0.0, 0.5])
    while case["rows"] * case["vocab"] > 2048 * 50021:
        case["rows"] //= 2
    return case


# ---- posits in elementary operations ----

_tables = {}


def _values(n, es):
    """The values of the patterns 0 .. 2^(n-1)-1 of posit<n,es>, in 64 bits: sign 0, then regime, exponent and fraction."""
    p = np.arange(1, 1 << (n - 1), dtype=np.int64)
    ones = p >> (n - 2) == 1                                     # the regime's bits are ones
    other = np.where(ones, (1 << (n - 1)) - 1 - p, p)            # its first bit of the other kind is the highest one here
    top = np.where(other > 0, np.frexp(other.astype(np.float64))[1] - 1, -1)
    run = n - 2 - top
    k = np.where(ones, run - 1, -run)
    left = np.maximum(top, 0)                                     # bits after the one that ended the run
    rest = p & ((1 << left) - 1)
    short = np.maximum(es - left, 0)                              # exponent bits that are cut off are zeros
    rest, left = rest << short, left + short
    e, f = rest >> (left - es), rest & ((1 << (left - es)) - 1)
    return np.concatenate([[0.0], np.ldexp(1.0 + f / np.exp2(left - es), k * (1 << es) + e)])


def _table(fmt):
    """(value of each pattern in binary32, bounds: a magnitude above the i-th bound and not above the next rounds to pattern i + 2)."""
    if fmt not in _tables:
        n, es = POSITS[fmt]
        v = _values(n, es)
        whole = np.concatenate([v, [np.nan], -v[:0:-1]]).astype(np.float32)
        # between neighbours u and u + 1 lies the pattern 2u + 1 of one bit more; ties go to the even pattern; nothing rounds to zero
        mid = _values(n + 1, es)[3:-1:2].astype(np.float32)
        odd = np.arange(1, len(mid) + 1) % 2 == 1
        bounds = np.where(odd, np.nextafter(mid, np.float32(0)), mid).astype(np.float32)
        _tables[fmt] = (torch.from_numpy(whole).cuda(), torch.from_numpy(bounds).cuda())
    return _tables[fmt]


def decode(t, fmt):
    """Values of a tensor of `fmt` in binary32."""
    if fmt not in POSITS:
        return t.to(torch.float32)
    n, _ = POSITS[fmt]
    return _table(fmt)[0][t.to(torch.int32) & ((1 << n) - 1)]


def encode(x, fmt):
    """The tensor of `fmt` nearest to x, ties to the even pattern, never to zero; NaN and infinities give NaR."""
    if fmt not in POSITS:
        return x.to(torch.bfloat16 if fmt == "bf16" else torch.float32)
    n, _ = POSITS[fmt]
    i = torch.bucketize(x.abs(), _table(fmt)[1], out_int32=True) + 1
    p = torch.where(x == 0, 0, torch.where(x < 0, -i, i))
    p = torch.where(torch.isfinite(x), p, 1 << (n - 1)) & ((1 << n) - 1)
    return p.to(torch.uint8) if n == 8 else p.to(torch.int16)


def rounded(x, fmt):
    """x rounded to `fmt`, as the values that stand there: in bfloat16 where that holds them exactly."""
    return decode(encode(x, fmt), fmt).to(torch.float32 if fmt in ("f32", "p16", "p12_1") else torch.bfloat16)


# ---- inputs ----

def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(1000003 * (seed + 1))
    return g


def _normal(g, shape, sigma=1.0):
    return torch.randn(shape, generator=g, device="cuda", dtype=torch.float32) * sigma


def _lengths(case):
    """Keys of each sequence: from lk down by the share `ragged`, at least lq where lq is 1."""
    return [max(1, case["lk"] - int(case["lk"] * case["ragged"] * i / case["b"])) for i in range(case["b"])]


def prepare(case, seed):
    g = _gen(seed)
    s = {"case": case}
    if case["op"] == "norm":
        r, c = case["rows"], case["cols"]
        # a residual stream has a few columns that are larger than the others
        big = torch.where(torch.rand((1, c), generator=g, device="cuda") < 0.01, 4.0, 1.0)
        s["x"] = encode(_normal(g, (r, c), 0.5), case["fx"])
        s["res"] = encode(_normal(g, (r, c)) * big, case["fres"])
        s["w"] = encode(1.0 + _normal(g, (c,), 0.1), case["fw"])
        if case["pass"] == "train":
            s["dy"] = _normal(g, (r, c)).to(torch.bfloat16)
            s["dres"] = _normal(g, (r, c)).to(torch.bfloat16)
    elif case["op"] == "attn":
        b, lq, lk, d = case["b"], case["lq"], case["lk"], case["d"]
        s["q"] = encode(_normal(g, (b, lq, case["hq"], d), 1.5), case["fq"])
        s["k"] = encode(_normal(g, (b, lk, case["hkv"], d)), case["fkv"])
        s["v"] = encode(_normal(g, (b, lk, case["hkv"], d)), case["fkv"])
        s["lens"] = torch.tensor(_lengths(case), dtype=torch.int32, device="cuda")
        if case["pass"] == "train":
            s["do"] = encode(_normal(g, (b, lq, case["hq"], d)), case["fq"])
    else:
        r, v = case["rows"], case["vocab"]
        z = _normal(g, (r, v), 2.0)
        s["targets"] = torch.randint(0, v, (r,), generator=g, device="cuda", dtype=torch.int32)
        at = s["targets"].long()[:, None]
        z.scatter_add_(1, at, _normal(g, (r, 1), 3.0) + 6.0)  # a trained model prefers the right token
        if case["masked"]:
            hide = torch.rand((r, v), generator=g, device="cuda") < case["masked"]
            hide.scatter_(1, at, False)
            z.masked_fill_(hide, -math.inf)
        s["logits"] = encode(z, case["fz"])
        if case["pass"] == "train":
            s["g_lp"] = torch.where(torch.rand((r,), generator=g, device="cuda") < 0.1, 0.0, -1.0)  # a tenth is padding or prompt
            s["g_ent"] = _normal(g, (r,), 0.01)
    if case["op"] != "logprob":
        s["fmts"] = [_table(case[f]) for f in ("fx", "fres", "fw", "fy", "fq", "fkv", "fout") if case.get(f) in POSITS]
    return s


# ---- plain forms ----

def _power(k):
    """2^k in binary32, exactly."""
    return ((k + 127) << 23).view(torch.float32)


def _norm_fwd_plain(case, s):
    h_bits = encode(decode(s["x"], case["fx"]) + decode(s["res"], case["fres"]), case["fres"])
    h = decode(h_bits, case["fres"])
    rstd = 1.0 / torch.sqrt((h * h).mean(dim=1) + EPS)
    return h_bits, h, rstd, h * decode(s["w"], case["fw"])


def _norm_plain(case, s):
    h_bits, h, rstd, t = _norm_fwd_plain(case, s)
    if case["pass"] == "fwd":
        # each row's power of two brings its largest magnitude into [4, 8); the rest of the scale is the row's 1 / rms
        a = t.abs().amax(dim=1)
        e = torch.where(a > 0, torch.frexp(a)[1] - 1, 2)
        p = rounded(t * _power(2 - e)[:, None], case["fy"]).float()
        scale = rstd * _power(e - 2)
        return {"res": h_bits, "values": p * scale[:, None], "scale": scale}
    w, dy = decode(s["w"], case["fw"]), s["dy"].float()
    g = dy * w
    c = (g * h).mean(dim=1)
    dx = rstd[:, None] * g - (rstd ** 3 * c)[:, None] * h + s["dres"].float()
    return {"res": h_bits, "y": rounded(t * rstd[:, None], case["fy"]), "dx": dx.to(torch.bfloat16), "dw": (dy * h * rstd[:, None]).sum(dim=0)}


def _visible(case, lens, dev):
    """[b, 1, 1, lq, lk]: which key each query sees."""
    i = torch.arange(case["lq"], device=dev, dtype=torch.int32)
    j = torch.arange(case["lk"], device=dev, dtype=torch.int32)
    p = (lens[:, None] - case["lq"] + i)[:, :, None]
    see = (j <= p) & (p >= 0)
    if case["window"]:
        see = see & ((j > p - case["window"]) | (j < case["sinks"]))
    return see[:, None, None]


def _heads(t, hkv):
    """[b, l, h, d] to [b, hkv, h / hkv * l, d]."""
    b, l, h, d = t.shape
    return t.permute(0, 2, 1, 3).reshape(b, hkv, h // hkv * l, d).contiguous()


def _back(t, b, l, h, d):
    return t.reshape(b, h, l, d).permute(0, 2, 1, 3).contiguous()


def _attn_plain(case, s):
    b, lq, lk, hq, hkv, d = (case[n] for n in ("b", "lq", "lk", "hq", "hkv", "d"))
    q, k, v = _heads(decode(s["q"], case["fq"]), hkv), _heads(decode(s["k"], case["fkv"]), hkv), _heads(decode(s["v"], case["fkv"]), hkv)
    see = _visible(case, s["lens"], q.device)
    scale = 1.0 / math.sqrt(d)
    z = (torch.matmul(q, k.transpose(2, 3).contiguous()) * scale).reshape(b, hkv, hq // hkv, lq, lk)
    z = torch.where(see, z, -math.inf)
    m = z.amax(dim=4, keepdim=True)
    m = torch.where(m == -math.inf, 0.0, m)
    e = torch.exp(z - m)
    total = e.sum(dim=4, keepdim=True)
    lse = (m + torch.log(total)).reshape(b, hq, lq)
    p = (e / torch.where(total == 0, 1.0, total)).reshape(b, hkv, hq // hkv * lq, lk)
    o = torch.matmul(p, v)
    out = {"o": rounded(_back(o, b, lq, hq, d), case["fout"]), "lse": lse}
    if case["pass"] == "train":
        do = _heads(decode(s["do"], case["fq"]), hkv)
        dp = torch.matmul(do, v.transpose(2, 3).contiguous())
        ds = p * (dp - (do * o).sum(dim=3, keepdim=True)) * scale
        back = lambda t, l, h: rounded(_back(t, b, l, h, d), case["fout"])  # noqa: E731
        out["dq"] = back(torch.matmul(ds, k), lq, hq)
        out["dk"] = back(torch.matmul(ds.transpose(2, 3).contiguous(), q), lk, hkv)
        out["dv"] = back(torch.matmul(p.transpose(2, 3).contiguous(), do), lk, hkv)
    return out


def _logprob_plain(case, s):
    z = decode(s["logits"], case["fz"])
    at = s["targets"].long()[:, None]
    m = z.amax(dim=1, keepdim=True)
    lse = m + torch.log(torch.exp(z - m).sum(dim=1, keepdim=True))
    lp = z - lse
    p = torch.exp(lp)
    ent = -torch.where(p > 0, p * lp, 0.0).sum(dim=1)
    out = {"logprob": lp.gather(1, at)[:, 0], "lse": lse[:, 0], "entropy": ent}
    if case["top"]:
        # the order of the values first, then the lowest index: one integer for both
        bits = (z + 0.0).view(torch.int32)
        order = torch.where(bits < 0, bits ^ 0x7FFFFFFF, bits).long()
        key = order * (1 << 32) + (case["vocab"] - 1 - torch.arange(case["vocab"], device=z.device))
        best = torch.topk(key, case["top"], dim=1)[0]
        index = case["vocab"] - 1 - (best & 0xFFFFFFFF)
        out["top_index"], out["top_logprob"] = index.int(), lp.gather(1, index)
    if case["pass"] == "train":
        hit = torch.zeros_like(p).scatter_(1, at, 1.0)
        dz = s["g_lp"][:, None] * (hit - p) - s["g_ent"][:, None] * torch.where(p > 0, p * (lp + ent[:, None]), 0.0)
        out["dlogits"] = dz.to(torch.bfloat16)
    return out


# ---- the framework's calls ----

def _norm_own(case, s):
    import paper_2105_00053_amd as pn
    if case["pass"] == "fwd":
        y, scale, res, _ = pn.posit_rmsnorm_fwd(s["x"], s["w"], case["fx"], case["fw"], case["fy"], eps=EPS, res=s["res"], fres=case["fres"], scaled=True)
        return {"res": _as_given(res, s["res"]), "values": pn.posit_scale_rows(y, scale, case["fy"], "f32"), "scale": scale}
    y, _, res, rstd = pn.posit_rmsnorm_fwd(s["x"], s["w"], case["fx"], case["fw"], case["fy"], eps=EPS, res=s["res"], fres=case["fres"])
    dx, dw = pn.posit_rmsnorm_bwd(s["dy"], res, s["w"], rstd, "bf16", case["fres"], case["fw"], "bf16", "f32", dres=s["dres"], fdres="bf16")
    return {"res": _as_given(res, s["res"]), "y": y, "dx": dx, "dw": dw}


def _as_given(t, like):
    """16-bit patterns in the signed type that the inputs have."""
    return t.view(like.dtype)


def _attn_own(case, s):
    import paper_2105_00053_amd as pn
    mask = {"scale": 1.0 / math.sqrt(case["d"]), "window": case["window"], "sinks": case["sinks"], "lens": s["lens"]}
    if case["pass"] != "train":
        o, lse, _ = pn.posit_attention_fwd(s["q"], s["k"], s["v"], case["fq"], case["fkv"], case["fout"], **mask)
        if case["fout"] != "bf16":
            o = pn.posit_convert(o, case["fout"], "f32").to(torch.bfloat16)
        return {"o": o, "lse": lse}
    o, lse, o32 = pn.posit_attention_fwd(s["q"], s["k"], s["v"], case["fq"], case["fkv"], case["fout"], fcopy="f32", **mask)
    dq, dk, dv = pn.posit_attention_bwd(s["do"], s["q"], s["k"], s["v"], o32, lse, case["fq"], case["fq"], case["fkv"], "f32", case["fout"], **mask)
    return {"o": o, "lse": lse, "dq": dq, "dk": dk, "dv": dv}


def _logprob_own(case, s):
    import paper_2105_00053_amd as pn
    lp, lse, ent, top_lp, top_index = pn.posit_token_logprob_fwd(s["logits"], s["targets"], case["fz"], top=case["top"])
    out = {"logprob": lp, "lse": lse, "entropy": ent}
    if case["top"]:
        out["top_index"], out["top_logprob"] = top_index, top_lp
    if case["pass"] == "train":
        out["dlogits"] = pn.posit_token_logprob_bwd(s["logits"], s["targets"], lse, ent, s["g_lp"], s["g_ent"], case["fz"], "bf16")
    return out


def run(state):
    case = state["case"]
    if own:
        return {"norm": _norm_own, "attn": _attn_own, "logprob": _logprob_own}[case["op"]](case, state)
    return {"norm": _norm_plain, "attn": _attn_plain, "logprob": _logprob_plain}[case["op"]](case, state)


# ---- what a pass cannot do without ----

def work(case):
    def seen():
        """Pairs of a query and a key that it sees, over the sequences, for one head; and the keys that any query sees."""
        pairs = keys = 0
        for n in _lengths(case):
            first = max(n - case["lq"], 0)
            w = case["window"] or n
            p = np.arange(first, n, dtype=np.int64)
            inside = np.minimum(p + 1, w)
            pairs += int((inside + np.minimum(case["sinks"], p + 1 - inside)).sum())
            low = max(0, first - w + 1)  # the first query's window reaches furthest back
            keys += (n - low) + min(case["sinks"], low)
        return pairs, keys

    if case["op"] == "norm":
        n = case["rows"] * case["cols"]
        b = BYTES[case["fx"]] + 2 * BYTES[case["fres"]]
        if case["pass"] == "fwd":
            return {"bytes": n * (b + 4) + case["cols"] * BYTES[case["fw"]] + 4 * case["rows"], "flops": 8 * n}
        return {"bytes": n * (b + 2 + 2 + 2 + 2) + case["cols"] * (BYTES[case["fw"]] + 4), "flops": 20 * n}
    if case["op"] == "attn":
        pairs, keys = seen()
        nq = case["b"] * case["lq"] * case["hq"] * case["d"]
        kv = keys * case["hkv"] * case["d"] * BYTES[case["fkv"]]
        given = nq * BYTES[case["fq"]] + 2 * kv
        back = 2 * nq + 4 * case["b"] * case["lq"] * case["hq"]
        if case["pass"] != "train":
            return {"bytes": given + back, "flops": 4 * pairs * case["hq"] * case["d"]}
        nk = case["b"] * case["lk"] * case["hkv"] * case["d"]
        return {"bytes": given + nq * BYTES[case["fq"]] + back + 2 * nq + 4 * nk, "flops": 14 * pairs * case["hq"] * case["d"]}
    n = case["rows"] * case["vocab"]
    if case["pass"] == "fwd":
        return {"bytes": n * BYTES[case["fz"]] + case["rows"] * (16 + 8 * case["top"]), "flops": 6 * n}
    return {"bytes": n * (BYTES[case["fz"]] + 2) + 24 * case["rows"], "flops": 14 * n}


# ---- the definitions in 64 bits ----

_wide = {}


def exact(case, seed):
    """What run() returns, from the definitions in 64 bits; what is rounded at the end to be stored stands here before that."""
    s = prepare(case, seed)
    wide = _wide

    def wide_values(t, fmt):
        if fmt not in POSITS:
            return t.to(torch.float64)
        n, es = POSITS[fmt]
        if fmt not in wide:
            v = _values(n, es)
            wide[fmt] = torch.from_numpy(np.concatenate([v, [np.nan], -v[:0:-1]])).cuda()
        return wide[fmt][t.long() % (1 << n)]

    def near(x, fmt):
        """x rounded to `fmt`: by comparison with the midpoints of neighbouring patterns."""
        if fmt not in POSITS:
            return x.to(torch.bfloat16 if fmt == "bf16" else torch.float32).double()
        n, es = POSITS[fmt]
        key = (fmt, "mid")
        if key not in wide:
            wide[key] = (torch.from_numpy(_values(n, es)).cuda(), torch.from_numpy(_values(n + 1, es)[3:-1:2].copy()).cuda())
        v, mid = wide[key]
        a = x.abs()
        low = torch.searchsorted(mid, a, right=False) + 1      # the lower of the two patterns of a tie
        high = torch.searchsorted(mid, a, right=True) + 1
        at = torch.where(low % 2 == 0, low, high)
        return torch.where(x == 0, 0.0, torch.sign(x) * v[at])

    def norm():
        # the stream is kept in its format, so the sum is rounded before anything else; its patterns are whole numbers
        h = near((wide_values(s["x"], case["fx"]) + wide_values(s["res"], case["fres"])), case["fres"])
        w = wide_values(s["w"], case["fw"])
        inv = (h.pow(2).sum(1) / case["cols"] + EPS).rsqrt()
        stream = h if case["fres"] in ("bf16", "f32") else None
        if case["pass"] == "fwd":
            t = h * w
            e = torch.floor(torch.log2(t.abs().amax(1))) - 2
            scale = inv * 2.0 ** e
            return {"res": stream, "values": near(t / (2.0 ** e)[:, None], case["fy"]) * scale[:, None], "scale": scale}
        dy = s["dy"].double()
        xhat = h * inv[:, None]
        gx = dy * w
        dx = (gx - xhat * (gx * xhat).sum(1, keepdim=True) / case["cols"]) * inv[:, None] + s["dres"].double()
        return {"res": stream, "y": xhat * w, "dx": dx, "dw": (dy * xhat).sum(0)}

    def attn():
        b, lq, lk, hq, hkv, d = (case[n] for n in ("b", "lq", "lk", "hq", "hkv", "d"))
        q, k, v = wide_values(s["q"], case["fq"]), wide_values(s["k"], case["fkv"]), wide_values(s["v"], case["fkv"])
        train = case["pass"] == "train"
        do = wide_values(s["do"], case["fq"]) if train else None
        o = torch.zeros_like(q)
        lse = torch.full((b, hq, lq), -math.inf, dtype=torch.float64, device=q.device)
        dq, dk, dv = torch.zeros_like(q), torch.zeros_like(k), torch.zeros_like(v)
        for i, n in enumerate(_lengths(case)):
            at = torch.arange(n - lq, n, device=q.device)[:, None]
            key = torch.arange(n, device=q.device)[None, :]
            hidden = key > at
            if case["window"]:
                hidden = hidden | ((key <= at - case["window"]) & (key >= case["sinks"]))
            some = ~hidden.all(dim=1)
            for h in range(hq):
                j = h // (hq // hkv)
                kk, vv = k[i, :n, j].contiguous(), v[i, :n, j].contiguous()
                z = (q[i, :, h] @ kk.T.contiguous() / math.sqrt(d)).masked_fill(hidden, -math.inf)
                lse[i, h] = torch.logsumexp(z, 1)
                p = torch.exp(z - torch.where(some, lse[i, h], 0.0)[:, None])
                o[i, :, h] = p @ vv
                if train:
                    g = do[i, :, h].contiguous()
                    dv[i, :n, j] += p.T.contiguous() @ g
                    dp = g @ vv.T.contiguous()
                    dz = p * (dp - (dp * p).sum(1, keepdim=True)) / math.sqrt(d)
                    dq[i, :, h] = dz @ kk
                    dk[i, :n, j] += dz.T.contiguous() @ q[i, :, h].contiguous()
        out = {"o": o, "lse": lse}
        return dict(out, dq=dq, dk=dk, dv=dv) if train else out

    def logprob():
        out = {"logprob": [], "lse": [], "entropy": [], "top_logprob": [], "dlogits": []}
        for rows in torch.arange(case["rows"], device="cuda").split(512):
            z = wide_values(s["logits"][rows], case["fz"])
            at = s["targets"][rows].long()[:, None]
            lse = torch.logsumexp(z, 1, keepdim=True)
            p = (z - lse).exp()
            ent = -torch.xlogy(p, p).sum(1)
            out["logprob"].append((z.gather(1, at) - lse)[:, 0])
            out["lse"].append(lse[:, 0])
            out["entropy"].append(ent)
            if case["top"]:
                out["top_logprob"].append(torch.topk(z, case["top"], dim=1)[0] - lse)
            if case["pass"] == "train":
                dz = -s["g_lp"][rows].double()[:, None] * p - s["g_ent"][rows].double()[:, None] * (torch.xlogy(p, p) + p * ent[:, None])
                out["dlogits"].append(dz.scatter_add(1, at, s["g_lp"][rows].double()[:, None]))
        return {k: torch.cat(t) for k, t in out.items() if t}

    return {"norm": norm, "attn": attn, "logprob": logprob}[case["op"]]()


if __name__ == "__main__":
    r = random.Random(0)
    for c in listed() + [draw(r) for _ in range(8)]:
        print(c, work(c))
