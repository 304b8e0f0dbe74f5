"""Cases of the operators with which a language model generates text: norms of queries and keys with the rotation by their positions, a cache of keys
and values in pages with the attention that reads it, and the draw of the next token.

listed() holds the fixed cases, draw(rng) gives more of the same ranges.  A case is a dict of plain values:

  op "heads"     `tokens` rows of hq query and hkv key heads of d elements, each normalised, its first `rot` elements rotated by the row's position;
                 "pass" "fwd", or "train": forward and backward
  op "append"    b sequences with up to `had` tokens in a cache of pages of `page` tokens get up to `new` more: queries and keys normalised and rotated,
                 keys and values rounded into the pages; then each sequence's keys and values read back as rows of bfloat16, what attention of a prompt on
                 a filled cache takes
  op "paged"     b sequences of up to `keys` tokens in pages; the last `new` of each are queries; window 0 is none, `sinks` first tokens stay visible
  op "sample"    one token for each of rows x vocab logits from a given random number; "how" says what limits the choice

Numbers of tokens fall from sequence to sequence by the share `ragged`.  Where `own` is false, run() computes the same in elementary operations.  Formats are
named as in the binding ("p8_1" is posit<8,1>, "bf16" bfloat16, "f32" binary32); "f4" is a cache's format of 4 bits: magnitudes 0 1/2 1 3/2 2 3 4 6 in blocks of 32
elements, each with a power of two.  8- and 16-bit posits are given as their patterns.

A cache's tensor is [pages][heads][bytes or elements of a page].  Keys lie as [token][d]; values as [token / 4][d / 8][token % 4][d % 8].  For "f4" that is the order of
half bytes, low one first (bit 3 the sign), and behind them lie a block's exponents plus 127: [token][block] of keys, [token / 4][block][token % 4] of values.
"""
import math
import random

import numpy as np
import torch

own = False

EPS = 1e-6
BASE = 10000.0
POSITS = {"p8": (8, 0), "p8_1": (8, 1), "p8_2": (8, 2), "p12_2": (12, 2), "p16": (16, 1)}
BYTES = {"p8": 1, "p8_1": 1, "p8_2": 1, "p12_2": 2, "p16": 2, "bf16": 2, "f32": 4, "f4": 0.53125}


def listed():
    return [
        # a prompt of a few tokens: latency
        {"name": "heads_prompt_7", "op": "heads", "pass": "fwd", "tokens": 7, "hq": 16, "hkv": 4, "d": 64, "rot": 64, "neighbours": False, "far": 0,
         "fx": "p8_1", "fw": "p16", "fy": "p8_1"},
        # a training step over whole sequences
        {"name": "heads_train_16384", "op": "heads", "pass": "train", "tokens": 16384, "hq": 32, "hkv": 8, "d": 128, "rot": 128, "neighbours": False, "far": 0,
         "fx": "p8_2", "fw": "p16", "fy": "bf16"},
        # single tokens of four sequences that have just begun: latency
        {"name": "append_token_4", "op": "append", "b": 4, "had": 40, "new": 1, "ragged": 0.5, "hq": 16, "hkv": 4, "d": 64, "rot": 64, "neighbours": False, "norm": False, "page": 16,
         "fx": "p8_1", "fw": "p16", "fq": "bf16", "fc": "p8_1"},
        # parts of prompts of every length behind short beginnings, heads that are rotated in part, neighbouring elements in pairs
        {"name": "append_mixed_21x100", "op": "append", "b": 21, "had": 65, "new": 100, "ragged": 0.99, "hq": 20, "hkv": 4, "d": 80, "rot": 32, "neighbours": True, "norm": True,
         "page": 16, "fx": "bf16", "fw": "f32", "fq": "p8_2", "fc": "p8"},
        # a batch of prompts into a cache of 4 bits
        {"name": "append_prompts_9x2048", "op": "append", "b": 9, "had": 0, "new": 2048, "ragged": 0.7, "hq": 32, "hkv": 8, "d": 128, "rot": 128, "neighbours": False, "norm": True,
         "page": 64, "fx": "p8_2", "fw": "p16", "fq": "bf16", "fc": "f4"},
        # single tokens of a small model on short caches: latency
        {"name": "paged_token_3x300", "op": "paged", "b": 3, "keys": 300, "new": 1, "ragged": 0.5, "hq": 8, "hkv": 2, "d": 64, "page": 16, "window": 0, "sinks": 0,
         "fq": "bf16", "fc": "p8_1", "fout": "bf16"},
        # one long text in 4 bits
        {"name": "paged_token_1x60000", "op": "paged", "b": 1, "keys": 60000, "new": 1, "ragged": 0.0, "hq": 32, "hkv": 8, "d": 128, "page": 64, "window": 0, "sinks": 0,
         "fq": "bf16", "fc": "f4", "fout": "bf16"},
        # five guessed tokens of each sequence at once, with a window and sinks
        {"name": "paged_guess_16x4001", "op": "paged", "b": 16, "keys": 4001, "new": 5, "ragged": 0.8, "hq": 16, "hkv": 4, "d": 96, "page": 32, "window": 2000, "sinks": 4,
         "fq": "p8_1", "fc": "p8_2", "fout": "bf16"},
        # a batch in serving, on long caches of 4 bits of every length
        {"name": "paged_token_64x8192", "op": "paged", "b": 64, "keys": 8192, "new": 1, "ragged": 0.9, "hq": 32, "hkv": 8, "d": 128, "page": 64, "window": 0, "sinks": 0,
         "fq": "bf16", "fc": "f4", "fout": "bf16"},
        # one row, everything at once
        {"name": "sample_1x100003", "op": "sample", "rows": 1, "vocab": 100003, "fz": "p16", "how": "mixed", "masked": 0.0},
        # a small batch whose decoder forbids most tokens
        {"name": "sample_masked_32x5003", "op": "sample", "rows": 32, "vocab": 5003, "fz": "f32", "how": "min", "masked": 0.7},
        # a large batch, each row with its own temperature and limits
        {"name": "sample_256x50021", "op": "sample", "rows": 256, "vocab": 50021, "fz": "p16", "how": "mixed", "masked": 0.0},
    ]


def _log(rng, lo, hi):
    """An integer spread over the logarithm of lo..hi, half of them as they fall, the others a multiple of 8 where they are long."""
    v = int(round(lo * (hi / lo) ** rng.random()))
    if rng.random() < 0.5 and v >= 64:
        v -= v % 8
    return max(lo, min(hi, v))


def draw(rng):
    op = rng.choice(["heads", "append", "paged", "paged", "sample"])
    hkv = rng.choice([1, 2, 4, 8])
    heads = {"hq": hkv * rng.choice([1, 2, 4, 5]), "hkv": hkv, "d": rng.choice([32, 64, 80, 96, 128])}
    if op == "heads":
        case = {"op": op, "pass": rng.choice(["fwd", "train"]), "tokens": _log(rng, 1, 16384), **heads, "far": rng.choice([0, 0, 100000]),
                "neighbours": rng.choice([False, True]), "fx": rng.choice(["p8", "p8_1", "p8_2", "bf16"]), "fw": rng.choice(["p16", "p12_2", "f32"])}
        case["rot"] = rng.choice([case["d"], case["d"], case["d"] // 2])
        # 8-bit outputs of few rows: among many values some lie next to a border, and 32 bits do not say on which side
        case["fy"] = case["fx"] if case["pass"] == "fwd" and case["tokens"] <= 256 else "bf16"
        return case
    if op == "append":
        case = {"op": op, "b": _log(rng, 1, 48), "had": rng.choice([0, 17, 100]), "new": rng.choice([1, _log(rng, 2, 2048)]), "ragged": rng.choice([0.0, 0.5, 0.9]), **heads,
                "neighbours": rng.choice([False, True]), "norm": rng.choice([False, True]), "page": rng.choice([16, 32, 64, 256]),
                "fx": rng.choice(["p8", "p8_1", "p8_2", "bf16"]), "fw": rng.choice(["p16", "f32"])}
        case["rot"] = rng.choice([case["d"], case["d"] // 2])
        case["fq"], case["fc"] = rng.choice(["bf16", case["fx"]]), rng.choice(["f4", "f4", "p8", "p8_1", "p8_2", "bf16"])
        while case["b"] > 1 and case["b"] * (case["had"] + case["new"]) > 8192:
            case["b"] //= 2
        return case
    if op == "paged":
        case = {"op": op, "b": _log(rng, 1, 64), "keys": _log(rng, 16, 8192), "new": rng.choice([1, 1, 2, 5]), "ragged": rng.choice([0.0, 0.5, 0.9]), **heads,
                "page": rng.choice([16, 32, 64, 256]), "window": 0, "sinks": 0, "fq": rng.choice(["bf16", "p8_1"]), "fc": rng.choice(["f4", "f4", "p8", "p8_1", "p8_2", "bf16"]), "fout": "bf16"}
        if rng.random() < 0.4:
            case["window"], case["sinks"] = _log(rng, 16, 2048), rng.choice([0, 1, 4, 16])
        while work(case)["bytes"] > 260e6:
            case["b"] //= 2
        return case
    case = {"op": op, "rows": _log(rng, 1, 256), "vocab": _log(rng, 500, 131072), "fz": rng.choice(["p16", "p8_2", "p12_2", "bf16", "f32"]),
            "how": rng.choice(["all", "k", "p", "min", "mixed"]), "masked": 0.0}
    if case["fz"] in ("bf16", "f32"):
        case["masked"] = rng.choice([0.0, 0.5])
    while case["rows"] * case["vocab"] > 256 * 50021:
        case["rows"] //= 2
    return case


# ---- formats in elementary operations ----

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
    """(value of each pattern in 64 bits, bounds: a magnitude above the i-th bound and not above the next rounds to pattern i + 2)."""
    if fmt not in _tables:
        n, es = POSITS[fmt]
        v = _values(n, es)
        # between neighbours u and u + 1 lies the pattern 2u + 1 of one bit more; ties go to the even pattern; nothing rounds to zero
        mid = _values(n + 1, es)[3:-1:2]
        odd = np.arange(1, len(mid) + 1) % 2 == 1
        _tables[fmt] = (torch.from_numpy(np.concatenate([v, [np.nan], -v[:0:-1]])).cuda(), torch.from_numpy(np.where(odd, np.nextafter(mid, 0), mid)).cuda())
    return _tables[fmt]


def decode(t, fmt, dtype=torch.float32):
    """Values of a tensor of `fmt`."""
    if fmt not in POSITS:
        return t.to(dtype)
    n, _ = POSITS[fmt]
    return _table(fmt)[0].to(dtype)[t.to(torch.int32) & ((1 << n) - 1)]


def encode(x, fmt):
    """The tensor of `fmt` nearest to x, ties to the even pattern, never to zero; NaN and infinities give NaR."""
    if fmt not in POSITS:
        return x.to(torch.bfloat16 if fmt == "bf16" else torch.float32)
    n, _ = POSITS[fmt]
    i = torch.bucketize(x.abs().double(), _table(fmt)[1], out_int32=True) + 1
    p = torch.where(x == 0, 0, torch.where(x < 0, -i, i))
    p = torch.where(torch.isfinite(x), p, 1 << (n - 1)) & ((1 << n) - 1)
    return p.to(torch.uint8) if n == 8 else p.to(torch.int16)


def rounded(x, fmt):
    """x rounded to `fmt`, as the values that stand there, in bfloat16, which holds them exactly."""
    return decode(encode(x, fmt), fmt).to(torch.bfloat16)


def _f4_encode(x):
    """(codes 0 .. 15, exponents plus 127 of the blocks of 32) of x [..., d] in 64 bits.  A block's power of two is the smallest that leaves its largest element
    at 7 or below: no element is then off by more than half a step of its own binade."""
    d = x.shape[-1]
    blocks = -(-d // 32)
    y = torch.nn.functional.pad(x, (0, 32 * blocks - d)).reshape(*x.shape[:-1], blocks, 32)
    most = y.abs().amax(-1)
    m, e = torch.frexp(most)                                       # most = m 2^e, m in [1/2, 1)
    e = torch.where(m > 0.875, e - 2, e - 3)
    e = torch.where(most > 0, e.clamp(-124, 125), -124)
    step = torch.ldexp(y.abs(), -e[..., None])
    grid = torch.where(step < 2, 0.5, torch.where(step < 4, 1.0, 2.0)).to(step.dtype)
    v = (torch.round(step / grid) * grid).clamp(max=6)             # ties to even: the codes alternate as the multiples do
    code = torch.where(v < 2, 2 * v, torch.where(v < 4, v + 2, v / 2 + 4)).to(torch.int32)
    code = code + 8 * torch.signbit(y)
    return code.reshape(*x.shape[:-1], 32 * blocks)[..., :d], (e + 127).to(torch.int32)


def _f4_decode(code, e):
    mag = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], device=code.device)
    v = mag[code & 7] * torch.where(code >= 8, -1.0, 1.0)
    e = e.to(torch.int32).repeat_interleave(32, dim=-1)[..., :code.shape[-1]]
    return torch.ldexp(v, e - 127)


def _page_views(t, fc, page, d):
    """Views of a cache's tensors of keys or values: (keys' elements [p][h][token][.], their exponents or None), and the same of values [p][h][token / 4][d / 8][token % 4][.]."""
    p, h = t.shape[:2]
    if fc != "f4":
        return (t.view(p, h, page, d), None), (t.view(p, h, page // 4, d // 8, 4, 8), None)
    n = page * d // 2
    codes, e = t[:, :, :n], t[:, :, n:]
    return (codes.unflatten(2, (page, d // 2)), e.unflatten(2, (page, -1))), (codes.unflatten(2, (page // 4, d // 8, 4, 4)), e.unflatten(2, (page // 4, -1, 4)))


def _put(t, fc, page, d, values, x, pg, at):
    """x [n][h][d] in 64 bits into a cache's tensor, at tokens `at` of pages `pg`."""
    n, h = x.shape[:2]
    keys_of, values_of = _page_views(t, fc, page, d)
    to, scales = values_of if values else keys_of
    if fc == "f4":
        code, e = _f4_encode(x)
        raw = (code[..., ::2] | code[..., 1::2] << 4).to(torch.uint8)
        if values:
            scales[pg, :, at // 4, :, at % 4] = e.to(torch.uint8)
        else:
            scales[pg, :, at] = e.to(torch.uint8)
    else:
        raw = encode(x, fc)
    if values:
        to[pg, :, at // 4, :, at % 4] = raw.unflatten(2, (d // 8, 4 if fc == "f4" else 8))
    else:
        to[pg, :, at] = raw


def _take(t, fc, page, d, values, table, longest):
    """Values [b][longest][h][d] in binary32 of a cache's tensor: whatever lies there behind a sequence's end, too."""
    j = torch.arange(longest, device=t.device)
    pg, at = table[:, j // page].long(), (j % page)[None, :].expand(table.shape[0], -1)
    keys_of, values_of = _page_views(t, fc, page, d)
    to, scales = values_of if values else keys_of
    raw = (to[pg, :, at // 4, :, at % 4] if values else to[pg, :, at]).flatten(3)
    if fc != "f4":
        return decode(raw, fc)
    e = scales[pg, :, at // 4, :, at % 4] if values else scales[pg, :, at]
    return _f4_decode(torch.stack([raw & 15, raw >> 4], dim=-1).flatten(3).to(torch.int32), e)


# ---- inputs ----

def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(1000003 * (seed + 1))
    return g


def _normal(g, shape, sigma=1.0):
    return torch.randn(shape, generator=g, device="cuda", dtype=torch.float32) * sigma


def _falling(most, case):
    """most, and down from it by the share `ragged`; one at least unless there is none."""
    return [max(min(most, 1), most - int(most * case["ragged"] * i / case["b"])) for i in range(case["b"])]


def _counts(case):
    """(new tokens, tokens in all) of each sequence."""
    if case["op"] == "append":
        new = _falling(case["new"], case)
        return new, [n + h for n, h in zip(new, _falling(case["had"], case))]
    every = _falling(case["keys"], case)
    return [min(case["new"], n) for n in every], every


def _ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def _frequencies(rot):
    return BASE ** (torch.arange(rot // 2, dtype=torch.float64, device="cuda") * (-2.0 / rot))


def _cache(case, every, g, new):
    """(tensors of keys and values, page table) for sequences of `every` tokens, in pages in no order, a few of them nobody's.  Filled but for the `new` last tokens: with
    what the format rounds normal values to."""
    page, d, h, fc = case["page"], case["d"], case["hkv"], case["fc"]
    need = [-(-n // page) for n in every]
    order = torch.randperm(sum(need) + 3, generator=g, device="cuda")
    table = torch.full((case["b"], max(need)), -1, dtype=torch.int32, device="cuda")
    first = 0
    for i, n in enumerate(need):
        table[i, :n] = order[first:first + n]
        first += n
    size = page * d if fc != "f4" else page * d // 2 + page * -(-d // 32)
    both = []
    for values in (False, True):
        t = torch.zeros((len(order), h, size), dtype=torch.bfloat16 if fc == "bf16" else torch.uint8, device="cuda")
        for i, n in enumerate(every):
            for at in torch.arange(n - new[i], device="cuda").split(16384):
                _put(t, fc, page, d, values, _normal(g, (len(at), h, d)).double(), table[i, at // page].long(), at % page)
        both.append(t)
    return both, table


def prepare(case, seed):
    g = _gen(seed)
    s = {"case": case}
    if case["op"] == "heads":
        n, hq, h, d = case["tokens"], case["hq"], case["hq"] + case["hkv"], case["d"]
        # the rows of one product: queries, keys and values side by side
        qkv = encode(_normal(g, (n, h + case["hkv"], d), 1.5), case["fx"])
        s["q"], s["k"] = qkv[:, :hq], qkv[:, hq:h]
        s["wq"], s["wk"] = (encode(1.0 + _normal(g, (d,), 0.1), case["fw"]) for _ in range(2))
        s["freq"] = _frequencies(case["rot"])
        s["pos"] = case["far"] + torch.arange(n, dtype=torch.int32, device="cuda") % 2048
        if case["pass"] == "train":
            s["dq"], s["dk"] = (encode(_normal(g, t.shape), case["fx"]) for t in (s["q"], s["k"]))
    elif case["op"] == "append":
        new, every = _counts(case)
        n, hq, h, d = sum(new), case["hq"], case["hq"] + case["hkv"], case["d"]
        qkv = encode(_normal(g, (n, h + case["hkv"], d), 1.5), case["fx"])
        s["q"], s["k"], s["v"] = qkv[:, :hq], qkv[:, hq:h], qkv[:, h:]
        s["wq"], s["wk"] = (encode(1.0 + _normal(g, (d,), 0.1), case["fw"]) for _ in range(2)) if case["norm"] else (None, None)
        s["freq"] = _frequencies(case["rot"])
        (s["pages_k"], s["pages_v"]), s["table"] = _cache(case, every, g, new)
        s["lens"], s["starts"] = _ints(every), _ints([0] + np.cumsum(new).tolist())
        s["longest"] = max(every)
        s["seq"] = torch.repeat_interleave(torch.arange(case["b"], device="cuda"), _ints(new))
        s["pos"] = torch.cat([torch.arange(t - m, t, device="cuda") for m, t in zip(new, every)])
    elif case["op"] == "paged":
        new, every = _counts(case)
        s["q"] = encode(_normal(g, (sum(new), case["hq"], case["d"]), 1.5), case["fq"])
        (s["pages_k"], s["pages_v"]), s["table"] = _cache(case, every, g, [0] * case["b"])
        s["lens"], s["starts"] = _ints(every), _ints([0] + np.cumsum(new).tolist())
        s["longest"] = max(every)
        s["seq"] = torch.repeat_interleave(torch.arange(case["b"], device="cuda"), _ints(new))
        s["pos"] = torch.cat([torch.arange(t - m, t, device="cuda") for m, t in zip(new, every)])
        if case["new"] == 1:
            s["starts"] = None
    else:
        r, v = case["rows"], case["vocab"]
        z = _normal(g, (r, v), 2.0)
        z.scatter_add_(1, torch.randint(0, v, (r, 8), generator=g, device="cuda"), _normal(g, (r, 8), 2.0) + 5.0)  # a few tokens that the text asks for
        if case["masked"]:
            z.masked_fill_(torch.rand((r, v), generator=g, device="cuda") < case["masked"], -math.inf)
        s["logits"] = encode(z, case["fz"])
        s["u"] = torch.rand((r,), generator=g, device="cuda")
        how, some = case["how"], lambda: torch.rand((r,), generator=g, device="cuda")  # noqa: E731
        s["temperature"] = 0.6 + 0.6 * some() if how in ("mixed", "min") else None
        s["top_k"] = torch.exp(some() * math.log(v)).int() if how in ("k", "mixed") else None
        s["top_p"] = 0.8 + 0.199 * some() if how in ("p", "mixed") else None
        s["min_p"] = torch.exp(-some() * 7.0 - 1.0) if how in ("min", "mixed") else None
        if how == "mixed" and r > 4:
            # some requests take the likeliest token, some set no limits
            off = some()
            s["temperature"] = torch.where(off < 0.1, 0.0, s["temperature"])
            s["top_k"] = torch.where(off > 0.6, 0, s["top_k"])
            s["top_p"] = torch.where(off > 0.7, 1.0, s["top_p"])
            s["min_p"] = torch.where(off > 0.8, 0.0, s["min_p"])
    s["fmts"] = [_table(case[f]) for f in ("fx", "fw", "fy", "fq", "fc", "fz") if case.get(f) in POSITS]
    return s


# ---- plain forms ----

def _turned(t, cos, sin, case):
    """The first `rot` elements of t [n][h][d] rotated: cos, sin [n][1][rot / 2]."""
    r = case["rot"]
    if case["neighbours"]:
        a, b = t[..., 0:r:2], t[..., 1:r:2]
        y = torch.stack([a * cos - b * sin, b * cos + a * sin], dim=-1).flatten(2)
    else:
        a, b = t[..., :r // 2], t[..., r // 2:r]
        y = torch.cat([a * cos - b * sin, b * cos + a * sin], dim=2)
    return torch.cat([y, t[..., r:]], dim=2)


def _angles(s, dtype):
    """cos and sin of the rows' positions; the angles themselves in 64 bits."""
    a = (s["pos"].double()[:, None] * s["freq"][None, :])[:, None]
    return torch.cos(a).to(dtype), torch.sin(a).to(dtype)


def _normed(x, w, fw):
    """(x w rstd, x rstd, rstd); without w x itself."""
    if w is None:
        return x, x, None
    rstd = 1.0 / torch.sqrt((x * x).mean(dim=2, keepdim=True) + EPS)
    return x * rstd * decode(w, fw, x.dtype), x * rstd, rstd


def _heads_plain(case, s):
    cos, sin = _angles(s, torch.float32)
    out, rstds = {}, []
    for n in ("q", "k"):
        x, w = decode(s[n], case["fx"]), decode(s["w" + n], case["fw"])
        t, hat, rstd = _normed(x, s["w" + n], case["fw"])
        out["y" + n] = rounded(_turned(t, cos, sin, case), case["fy"])
        rstds.append(rstd[..., 0])
        if case["pass"] == "train":
            g = _turned(decode(s["d" + n], case["fx"]), cos, -sin, case)
            gw = g * w
            out["dx" + n] = (rstd * (gw - hat * (gw * hat).mean(dim=2, keepdim=True))).to(torch.bfloat16)
            out["dw" + n] = (g * hat).double().sum(dim=(0, 1)).float()
    return dict(out, rstd=torch.cat(rstds, dim=1))


def _append_plain(case, s):
    # in 64 bits: a value next to the border of two patterns may go to either in 32
    cos, sin = _angles(s, torch.float64)
    page, d, fc = case["page"], case["d"], case["fc"]
    q, k = (_turned(_normed(decode(s[n], case["fx"], torch.float64), s["w" + n], case["fw"])[0], cos, sin, case) for n in ("q", "k"))
    pg, at = s["table"][s["seq"], s["pos"] // page].long(), s["pos"] % page
    _put(s["pages_k"], fc, page, d, False, k, pg, at)
    _put(s["pages_v"], fc, page, d, True, decode(s["v"], case["fx"], torch.float64), pg, at)
    there = (torch.arange(s["longest"], device=pg.device)[None, :] < s["lens"][:, None])[:, :, None, None]
    k, v = (torch.where(there, _take(s["pages_" + n], fc, page, d, n == "v", s["table"], s["longest"]), 0.0).to(torch.bfloat16) for n in ("k", "v"))
    return {"q": rounded(q, case["fq"]), "k": k, "v": v}


def _paged_plain(case, s):
    hq, hkv, d, page, fc, b = (case[n] for n in ("hq", "hkv", "d", "page", "fc", "b"))
    k, v = (_take(s["pages_" + n], fc, page, d, n == "v", s["table"], s["longest"]) for n in ("k", "v"))
    j = torch.arange(s["longest"], device=k.device)
    v = torch.where((j[None, :] < s["lens"][:, None])[:, :, None, None], v, 0.0)
    # packed rows to a row of `new` places for each sequence, the last ones filled
    place = case["new"] - (s["lens"][s["seq"]] - s["pos"])
    q = torch.zeros((b, case["new"], hq, d), device=k.device)
    q[s["seq"], place] = decode(s["q"], case["fq"])
    p = s["lens"][:, None] - case["new"] + torch.arange(case["new"], device=k.device)[None, :]
    see = (j <= p[..., None]) & (p[..., None] >= 0)
    if case["window"]:
        see = see & ((j > p[..., None] - case["window"]) | (j < case["sinks"]))
    q = q.reshape(b, case["new"], hkv, hq // hkv, d).permute(0, 2, 3, 1, 4).reshape(b, hkv, -1, d)
    z = torch.matmul(q, k.permute(0, 2, 3, 1).contiguous()) * (1.0 / math.sqrt(d))
    z = torch.where(see[:, None, None], z.reshape(b, hkv, hq // hkv, case["new"], -1), -math.inf)
    m = z.amax(dim=4, keepdim=True)
    m = torch.where(m == -math.inf, 0.0, m)
    e = torch.exp(z - m)
    total = e.sum(dim=4, keepdim=True)
    lse = (m + torch.log(total))[..., 0]
    w = (e / torch.where(total == 0, 1.0, total)).reshape(b, hkv, -1, s["longest"])
    o = torch.matmul(w, v.permute(0, 2, 1, 3).contiguous()).reshape(b, hq, case["new"], d)
    return {"o": o[s["seq"], :, place].to(torch.bfloat16), "lse": lse.reshape(b, hq, -1)[s["seq"], :, place]}


def _sample_plain(case, s):
    z = decode(s["logits"], case["fz"], torch.float64)
    v = case["vocab"]
    z, index = torch.sort(z, dim=1, descending=True, stable=True)
    rank = torch.arange(v, device=z.device)[None, :]
    keep = torch.isfinite(z)
    if s["temperature"] is not None:
        t = s["temperature"].double()[:, None]
        keep = keep & ((rank == 0) | (t > 0))
        w = torch.exp((z - z[:, :1]) / torch.where(t > 0, t, 1.0))
    else:
        w = torch.exp(z - z[:, :1])
    if s["top_k"] is not None:
        k = s["top_k"][:, None]
        keep = keep & ((rank < k) | (k <= 0))
    w = torch.where(keep, w, 0.0)
    if s["top_p"] is not None:
        p = s["top_p"].double()[:, None]
        before = torch.cumsum(w, dim=1) - w
        keep = keep & ((before < p * w.sum(dim=1, keepdim=True)) | (p >= 1))
    if s["min_p"] is not None:
        keep = keep & (w >= s["min_p"].double()[:, None])
    w = torch.where(keep, w, 0.0)
    up, kept = torch.cumsum(w, dim=1), keep.sum(dim=1, keepdim=True)
    total = up[:, -1:]
    n = torch.minimum((up <= s["u"].double()[:, None] * total).sum(dim=1, keepdim=True), kept - 1)
    return {"token": index.gather(1, n)[:, 0].int(), "logprob": torch.log(w.gather(1, n) / total)[:, 0].float(), "kept": kept[:, 0].int()}


# ---- the framework's calls ----

def _as_bf16(t, fmt):
    import paper_2105_00053_amd as pn
    return t if fmt == "bf16" else pn.posit_convert(t, fmt, "f32").to(torch.bfloat16)


def _heads_own(case, s):
    import paper_2105_00053_amd as pn
    how = {"positions": s["pos"], "inv_freq": s["freq"], "wq": s["wq"], "wk": s["wk"], "fw": case["fw"], "neighbours": case["neighbours"]}
    yq, yk, rstd = pn.posit_qk_norm_rope_fwd(s["q"], s["k"], case["fx"], case["fy"], eps=EPS, **how)
    out = {"yq": _as_bf16(yq, case["fy"]), "yk": _as_bf16(yk, case["fy"]), "rstd": rstd}
    if case["pass"] == "train":
        dxq, dxk, dwq, dwk = pn.posit_qk_norm_rope_bwd(s["dq"], s["dk"], s["q"], s["k"], rstd, case["fx"], case["fx"], "bf16", fdw="f32", **how)
        out.update(dxq=dxq, dxk=dxk, dwq=dwq, dwk=dwk)
    return out


def _append_own(case, s):
    import paper_2105_00053_amd as pn
    q = pn.posit_cache_append(s["k"], s["v"], s["pages_k"], s["pages_v"], s["table"], s["lens"], case["fx"], case["fc"], starts=s["starts"], q=s["q"], fq=case["fq"],
                              inv_freq=s["freq"], wq=s["wq"], wk=s["wk"], fw=case["fw"], eps=EPS, neighbours=case["neighbours"])
    k, v = pn.posit_cache_read(s["pages_k"], s["pages_v"], s["table"], s["lens"], s["longest"], case["d"], case["fc"], "bf16")
    return {"q": _as_bf16(q, case["fq"]), "k": k, "v": v}


def _paged_own(case, s):
    import paper_2105_00053_amd as pn
    o, lse = pn.posit_attention_paged(s["q"], s["pages_k"], s["pages_v"], s["table"], s["lens"], case["fq"], case["fc"], case["fout"], longest=s["longest"], starts=s["starts"],
                                      most=case["new"], scale=1.0 / math.sqrt(case["d"]), window=case["window"], sinks=case["sinks"])
    return {"o": o, "lse": lse}


def _sample_own(case, s):
    import paper_2105_00053_amd as pn
    token, logprob, kept = pn.posit_sample(s["logits"], s["u"], case["fz"], temperature=s["temperature"], top_k=s["top_k"], top_p=s["top_p"], min_p=s["min_p"])
    return {"token": token, "logprob": logprob, "kept": kept}


def run(state):
    case = state["case"]
    if own:
        return {"heads": _heads_own, "append": _append_own, "paged": _paged_own, "sample": _sample_own}[case["op"]](case, state)
    return {"heads": _heads_plain, "append": _append_plain, "paged": _paged_plain, "sample": _sample_plain}[case["op"]](case, state)


# ---- what a pass cannot do without ----

def work(case):
    if case["op"] == "sample":
        n = case["rows"] * case["vocab"]
        return {"bytes": n * BYTES[case["fz"]] + 32 * case["rows"], "flops": 8 * n}
    d = case["d"]
    if case["op"] == "heads":
        n = case["tokens"] * (case["hq"] + case["hkv"]) * d
        once = n * (BYTES[case["fx"]] + 2) + 4 * case["tokens"] * (case["hq"] + case["hkv"] + 1)
        if case["pass"] == "fwd":
            return {"bytes": once, "flops": 9 * n}
        return {"bytes": once + n * (BYTES[case["fx"]] + 2), "flops": 27 * n}
    new, every = _counts(case)
    if case["op"] == "append":
        rows, kv = case["hkv"] * d, 2 * case["hkv"] * d
        given = sum(new) * ((case["hq"] * d + kv) * BYTES[case["fx"]] + case["hq"] * d * 2 + kv * BYTES[case["fc"]])
        return {"bytes": given + sum(every) * kv * BYTES[case["fc"]] + case["b"] * max(every) * kv * 2, "flops": sum(new) * (9 * case["hq"] * d + 12 * rows)}
    pairs = keys = 0
    for m, n in zip(new, every):
        w = case["window"] or n
        p = np.arange(n - m, n, dtype=np.int64)
        inside = np.minimum(p + 1, w)
        pairs += int((inside + np.minimum(case["sinks"], p + 1 - inside)).sum())
        low = max(0, n - m - w + 1)  # the first query's window reaches furthest back
        keys += (n - low) + min(case["sinks"], low)
    q = sum(new) * case["hq"]
    return {"bytes": keys * 2 * case["hkv"] * d * BYTES[case["fc"]] + q * (d * (BYTES[case["fq"]] + 2) + 4), "flops": 4 * pairs * case["hq"] * d}


# ---- the definitions in 64 bits ----

def exact(case, seed):
    """What run() returns, from the definitions in 64 bits; what is rounded to bfloat16 at the end to be stored stands here before that, what is rounded to 8 or 4 bits
    behind it."""
    s = prepare(case, seed)
    dev = "cuda"

    def wide(t, fmt):
        if fmt not in POSITS:
            return t.double()
        n, es = POSITS[fmt]
        v = _values(n, es)
        return torch.from_numpy(np.concatenate([v, [np.nan], -v[:0:-1]])).to(dev)[t.long() % (1 << n)]

    def near(x, fmt):
        """x rounded to `fmt` (not bfloat16): by comparison with the midpoints of neighbouring patterns."""
        if fmt not in POSITS:
            return x
        n, es = POSITS[fmt]
        v, mid = (torch.from_numpy(t).to(dev) for t in (_values(n, es), _values(n + 1, es)[3:-1:2].copy()))
        a = x.abs().contiguous()
        low = torch.searchsorted(mid, a, right=False) + 1      # the lower of the two patterns of a tie
        high = torch.searchsorted(mid, a, right=True) + 1
        return torch.where(x == 0, 0.0, torch.sign(x) * v[torch.where(low % 2 == 0, low, high)])

    def rotation():
        """The rows' rotations as complex numbers, reduced as fractions of a turn."""
        turns = s["pos"].double()[:, None] * s["freq"][None, :] / (2 * math.pi)
        turns = turns - torch.round(turns)
        return torch.polar(torch.ones_like(turns), 2 * math.pi * turns)[:, None]

    def spin(t, z):
        r = case["rot"]
        out = t.clone()
        first, second = (slice(0, r, 2), slice(1, r, 2)) if case["neighbours"] else (slice(0, r // 2), slice(r // 2, r))
        y = torch.complex(t[..., first].contiguous(), t[..., second].contiguous()) * z
        out[..., first], out[..., second] = y.real, y.imag
        return out

    def normalise(x, w):
        inv = (x.square().sum(2, keepdim=True) / case["d"] + EPS).rsqrt()
        return x * inv * w, inv

    def heads():
        z = rotation()
        out, invs = {}, []
        for n in ("q", "k"):
            x, w = wide(s[n], case["fx"]), wide(s["w" + n], case["fw"])
            t, inv = normalise(x, w)
            out["y" + n] = near(spin(t, z), case["fy"])
            invs.append(inv[..., 0])
            if case["pass"] == "train":
                g = spin(wide(s["d" + n], case["fx"]), z.conj())
                # d (x w / |x|) by the quotient's rule
                out["dx" + n] = g * w * inv - x * inv ** 3 * (g * w * x).sum(2, keepdim=True) / case["d"]
                out["dw" + n] = (g * x * inv).sum((0, 1))
        return dict(out, rstd=torch.cat(invs, 1))

    def near4(x):
        """The nearest values of 4 bits, block by block: by distance, the even code of two that are as near."""
        d = x.shape[-1]
        mags = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6], dtype=torch.float64, device=dev)
        out = torch.zeros_like(x)
        for first in range(0, d, 32):
            y = x[..., first:first + 32]
            top = y.abs().amax(-1, keepdim=True)
            e = torch.ceil(torch.log2(torch.where(top > 0, top, 1.0) / 7))
            e = torch.where(top > 7 * 2.0 ** e, e + 1, torch.where(top <= 3.5 * 2.0 ** e, e - 1, e))
            a = y.abs() / 2.0 ** e
            low = (torch.searchsorted(mags, a.contiguous(), right=True) - 1).clamp(0, 6)
            up, down = mags[low + 1] - a, a - mags[low]
            code = torch.where((up < down) | ((up == down) & (low % 2 == 1)), low + 1, low)
            out[..., first:first + 32] = torch.sign(y) * mags[code] * 2.0 ** e
        return out

    def append():
        z = rotation()
        turned = {}
        for n in ("q", "k"):
            x = wide(s[n], case["fx"])
            turned[n] = spin(normalise(x, wide(s["w" + n], case["fw"]))[0] if case["norm"] else x, z)
        new = {"k": turned["k"], "v": wide(s["v"], case["fx"])}
        out = {"q": near(turned["q"], case["fq"])}
        for n in ("k", "v"):
            t = _take(s["pages_" + n], case["fc"], case["page"], case["d"], n == "v", s["table"], s["longest"]).double()
            for i, length in enumerate(s["lens"].tolist()):
                t[i, length:] = 0
            t[s["seq"], s["pos"]] = near4(new[n]) if case["fc"] == "f4" else near(new[n], case["fc"])
            out[n] = t
        return out

    def paged():
        hq, hkv, d = case["hq"], case["hkv"], case["d"]
        q = wide(s["q"], case["fq"])
        o, lse = torch.zeros_like(q), torch.zeros(q.shape[:2], dtype=torch.float64, device=dev)
        first = 0
        for i, (m, n) in enumerate(zip(*_counts(case))):
            k, v = (_take(s["pages_" + x], case["fc"], case["page"], d, x == "v", s["table"][i:i + 1], n)[0].double() for x in ("k", "v"))
            at = torch.arange(n - m, n, device=dev)[:, None]
            key = torch.arange(n, device=dev)[None, :]
            hidden = key > at
            if case["window"]:
                hidden = hidden | ((key <= at - case["window"]) & (key >= case["sinks"]))
            for h in range(hq):
                g = h // (hq // hkv)
                z = (q[first:first + m, h] @ k[:, g].T.contiguous() / math.sqrt(d)).masked_fill(hidden, -math.inf)
                lse[first:first + m, h] = torch.logsumexp(z, 1)
                o[first:first + m, h] = torch.softmax(z, 1) @ v[:, g].contiguous()
            first += m
        return {"o": o, "lse": lse}

    def sample():
        z = wide(s["logits"], case["fz"])
        token, logprob, kept = [], [], []
        for r in range(case["rows"]):
            t = 1.0 if s["temperature"] is None else s["temperature"][r].item()
            value, index = z[r].sort(descending=True, stable=True)
            k = 0 if s["top_k"] is None else s["top_k"][r].item()
            lp = torch.log_softmax(value[: 1 if t == 0 else (k if k > 0 else None)] / (t or 1.0), 0)
            p = lp.exp()
            n = int((lp > -math.inf).sum())
            if s["top_p"] is not None and s["top_p"][r] < 1:
                n = min(n, int((p.cumsum(0) - p < s["top_p"][r].double()).sum()))
            if s["min_p"] is not None and s["min_p"][r] > 0:
                n = min(n, int((lp - lp[0] >= math.log(s["min_p"][r].item())).sum()))
            p = p[:n] / p[:n].sum()
            at = min(n - 1, int((p.cumsum(0) <= s["u"][r].double()).sum()))
            token.append(index[at])
            logprob.append(p[at].log())
            kept.append(n)
        return {"token": torch.stack(token).int(), "logprob": torch.stack(logprob), "kept": _ints(kept)}

    return {"heads": heads, "append": append, "paged": paged, "sample": sample}[case["op"]]()


if __name__ == "__main__":
    r = random.Random(0)
    for c in listed() + [draw(r) for _ in range(8)]:
        print(c, work(c))
