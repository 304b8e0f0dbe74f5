"""The one-layer token model with rotated and normalised heads: its gradients against those of the same model in 64-bit floats, and generating with a cache in pages, prompts and
single tokens of several sequences at once, against whole sequences."""
import numpy as np
import pytest
import torch

import generate_util as gu
import lm_util as lu
import paper_2105_00053_amd as pn
from paper_2105_00053_amd import lm_step
from test_gpu_lm_step import make, tokens_of

pytestmark = pytest.mark.gpu


def in_doubles(net, tokens, targets, loss_scale):
    """The same gradients by torch in 64 bits, from the weights that the products read."""
    b, l = tokens.shape
    fc, fm = net.compute, net.master
    x = torch.from_numpy(lu.values(net.table, fm))[tokens.cpu().reshape(-1).long()]
    ws = [torch.from_numpy(lu.values(w, fc)).requires_grad_() for w in net.copies]
    ns = [torch.from_numpy(lu.values(w, fm)).requires_grad_() for w in net.norms + net.head_norms]
    norm = lambda t, w: t * torch.rsqrt(t.square().mean(-1, keepdim=True) + net.eps) * w  # noqa: E731
    q, k, v = (norm(x, ns[0]) @ ws[0].T).view(b, l, -1, net.d).split([net.heads, net.kv_heads, net.kv_heads], dim=2)
    angle = torch.arange(l, dtype=torch.float64)[:, None] * net.inv_freq.cpu()
    half = len(net.inv_freq)

    def turned(t, w):
        t = norm(t, w)
        c, s = torch.cos(angle)[None, :, None], torch.sin(angle)[None, :, None]
        a, e = t[..., :half], t[..., half:2 * half]
        return torch.cat([a * c - e * s, e * c + a * s, t[..., 2 * half:]], dim=-1)

    q, k = turned(q, ns[2]), turned(k, ns[3])
    k, v = (t.repeat_interleave(net.heads // net.kv_heads, dim=2) for t in (k, v))
    s = torch.einsum("bihd,bjhd->bhij", q, k) / net.d ** 0.5
    s = s.masked_fill(torch.arange(l)[None, :] > torch.arange(l)[:, None], -float("inf"))
    o = torch.einsum("bhij,bjhd->bihd", torch.softmax(s, -1), v).reshape(b * l, -1)
    logprob = torch.log_softmax(norm(x + o @ ws[1].T, ns[1]) @ ws[2].T, 1).gather(1, targets.cpu().reshape(-1, 1).long())
    (-loss_scale * logprob.sum()).backward()
    return logprob.detach().view(b, l).numpy(), [w.grad.numpy() for w in ws + ns]


@pytest.mark.parametrize("how", [dict(rotated=16), dict(rotated=8, compute="p8_1")])
def test_gradients_follow_the_model(how):
    """As for the net without rotation: some ten roundings to 8 bits in a row, with signs of their own, leave a cosine well above 0.9."""
    net, g = make(3, head_norms=True, **how)
    tokens, targets = tokens_of(g, 3, 37)
    logprob, dws, dns = lm_step.gradients(net, tokens, targets)
    want_lp, want = in_doubles(net, tokens, targets, 64.0)
    assert len(dns) == 4
    assert np.corrcoef(logprob.cpu().numpy().reshape(-1), want_lp.reshape(-1))[0, 1] > 0.95
    for got, w in zip(dws + dns, want):
        a, c = lu.values(got, net.master).reshape(-1), w.reshape(-1)
        assert np.dot(a, c) / (np.linalg.norm(a) * np.linalg.norm(c)) > 0.9


def test_a_training_step_moves_the_heads_norms():
    net, g = make(5, rotated=16, head_norms=True)
    before = [w.clone() for w in net.head_norms]
    logprob = lm_step.training_step(net, *tokens_of(g, 4, 32), 1.0 / 64)
    assert torch.isfinite(logprob).all()
    assert all(not torch.equal(lm_step._movable(a), lm_step._movable(b)) for a, b in zip(before, net.head_norms))


def whole(net, tokens):
    """Log probabilities [l][vocab] behind each token of one sequence, all at once."""
    t = torch.tensor([tokens], dtype=torch.int32, device="cuda")
    x, _, _, qkv = lm_step._project(net, t)
    q, k, v, _, _ = lm_step._turned(net, qkv, 1, len(tokens))
    o, _, _ = pn.posit_attention_fwd(q, k, v, net.compute, net.compute, net.compute, window=net.window, sinks=net.sinks)
    logits = lm_step._read_out(net, x, o.view(len(tokens), -1))[3]
    return torch.log_softmax(torch.from_numpy(lu.values(logits, net.loss)), 1)


@pytest.mark.parametrize("how,cache,atol", [(dict(rotated=16, head_norms=True), None, 0.1), (dict(), None, 0.1), (dict(rotated=8, window=9, sinks=2), "p8_2", 0.1),
                                            (dict(rotated=16, head_norms=True, compute="p12_2"), None, 0.1), (dict(rotated=16, head_norms=True), "f4", 1.0)])
def test_generating_is_the_model_over_whole_sequences(how, cache, atol):
    """The same operators on the same rows; what differs is the order of the attention's sums, which moves a result of 8 bits to the neighbouring pattern now and then, and in 4 bits the
    cache's rounding (11 % of a key, less than that of a log probability of a handful)."""
    net, g = make(7, **how)
    text = torch.randint(0, 67, (3, 60), generator=g).tolist()
    want = {n: whole(net, t) for n, t in zip("abc", text)}
    text = dict(zip("abc", text))
    cache = lm_step.PagedDecoder(net, pages=16, page=16, cache=cache)
    # prompts of several lengths at once, one more while others go on, a part of a prompt behind a beginning, single tokens
    steps = [{"a": 5, "b": 1}, {"a": 1, "b": 30, "c": 20}, {"b": 1, "c": 1}, {"a": 1, "b": 1, "c": 1}, {"c": 25}, {"c": 1, "a": 2}]
    at = dict.fromkeys("abc", 0)
    for step in steps:
        new = {n: text[n][at[n]:at[n] + c] for n, c in step.items()}
        logits = cache.step(new)
        for n, c in step.items():
            at[n] += c
        assert [cache.length(n) for n in "abc"] == [at[n] for n in "abc"]
        got = torch.log_softmax(torch.from_numpy(lu.values(logits, net.loss)), 1)
        torch.testing.assert_close(got, torch.stack([want[n][at[n] - 1] for n in step]), rtol=0, atol=atol)


def test_sequences_come_and_go():
    net, g = make(9, rotated=16, head_norms=True)
    cache = lm_step.PagedDecoder(net, pages=4, page=16)
    u = torch.full((2,), 0.5, device="cuda")
    text = torch.randint(0, 67, (40,), generator=g).tolist()
    token, logprob, kept = cache.sample({1: text[:20], 2: text[20:25]}, u, top_k=torch.tensor([5, 1], dtype=torch.int32, device="cuda"))
    assert kept.tolist() == [5, 1] and (token >= 0).all() and (token < 67).all() and logprob[1] == 0 and logprob[0] < 0
    with pytest.raises(pn.PositError):
        cache.step({3: text[:17]})              # one page is free
    with pytest.raises(pn.PositError):
        cache.step({1: []})
    want = cache.step({2: token[1:].tolist()})
    cache.drop(1)
    again = cache.step({3: text[20:25]})        # in the pages that were the first sequence's
    again = cache.step({3: token[1:].tolist()})
    assert torch.equal(lm_step._movable(want), lm_step._movable(again))
    with pytest.raises(pn.PositError):
        lm_step.Decoder(net, 1, 4)
