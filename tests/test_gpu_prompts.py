"""Prompts in large chunks, other rotary positions and rules on tokens together, as a beam search uses them: against a model in 64 bits without a cache."""
import numpy as np
import pytest
import torch

from paper_2402_13720_b200 import build, synth
from paper_2402_13720_b200.beams import BeamDecoder
from paper_2402_13720_b200.rotary import Rotary, frequencies
from paper_2402_13720_b200.scores import allowed_words

gpu = pytest.mark.gpu
DEV = "cuda:0"
M = synth.ModelDesc(2, 128, 4, 2, 32, 256, 300, 64, "f32")
# what is turned, in which pairs, how far the context is stretched
FORMS = [dict(), dict(rotary_dim=16, interleaved=True), dict(interleaved=True, scaling="yarn", factor=4.0, original=32), dict(scaling="linear", factor=2.0)]


def weights():
    w = synth.model_weights(M, 5, device=DEV)
    w["lm_head"] = w["lm_head"] * 4
    return w


def logits64(w, tokens, form):
    """Logits behind every token of a text, in 64 bits."""
    def d(t):
        return t.double()

    kw = dict(form)
    rd, inter = kw.pop("rotary_dim", M.head_dim), kw.pop("interleaved", False)
    inv, mag = frequencies(rd, 10000.0, **kw)
    n = len(tokens)
    angle = torch.arange(n, dtype=torch.float64, device=DEV)[:, None] * inv.to(DEV)
    c, s = mag * torch.cos(angle)[:, None], mag * torch.sin(angle)[:, None]

    def turn(x):
        y = x.clone()
        a, b = (x[..., 0:rd:2], x[..., 1:rd:2]) if inter else (x[..., : rd // 2], x[..., rd // 2: rd])
        ya, yb = a * c - b * s, b * c + a * s
        if inter:
            y[..., 0:rd:2], y[..., 1:rd:2] = ya, yb
        else:
            y[..., : rd // 2], y[..., rd // 2: rd] = ya, yb
        return y

    def norm(x, g):
        return x * torch.rsqrt((x * x).mean(-1, keepdim=True) + M.rms_eps) * d(g)

    x = d(w["embed"])[torch.as_tensor(np.asarray(tokens), device=DEV).long()]
    hidden = torch.ones((n, n), dtype=torch.bool, device=DEV).triu(1)
    for lw in w["layers"]:
        y = norm(x, lw["attn_norm"])
        q, k, v = (y @ d(lw[m]).T for m in ("wq", "wk", "wv"))
        q, k, v = turn(q.view(n, M.n_heads, -1)), turn(k.view(n, M.n_kv_heads, -1)), v.view(n, M.n_kv_heads, -1)
        k, v = (t.repeat_interleave(M.n_heads // M.n_kv_heads, 1) for t in (k, v))
        p = torch.einsum("ihd,jhd->hij", q, k) / M.head_dim ** 0.5
        p = torch.softmax(p.masked_fill(hidden, -float("inf")), -1)
        x = x + torch.einsum("hij,jhd->ihd", p, v).reshape(n, -1) @ d(lw["wo"]).T
        y = norm(x, lw["ffn_norm"])
        x = x + (torch.nn.functional.silu(y @ d(lw["w_gate"]).T) * (y @ d(lw["w_up"]).T)) @ d(lw["w_down"]).T
    return norm(x, w["final_norm"]) @ d(w["lm_head"]).T


def decoder(w, form, beams, max_len, page, chunk):
    rotary = Rotary(M.head_dim, M.rope_theta, device=DEV, **form) if form else None
    return BeamDecoder(M, w, beams, max_len, page, rotary=rotary, chunk=chunk)


@gpu
@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("chunk,page", [(16, 8), (17, 5), (40, 16), (1000, 7)])
def test_prompts_in_chunks_give_the_same_scores(form, chunk, page):
    build.build()
    w = weights()
    prompt = synth.prompt(3, M.vocab, 90, 0.4, 3, 6)
    conts = [synth.prompt(10 + i, M.vocab, n, 0.4, 3, 6)[:n] for i, n in enumerate((1, 25, 9, 40))]
    d = decoder(w, form, 4, 140, page, chunk)
    got = d.score_all(prompt, conts)
    for c, lp in zip(conts, got):
        want = torch.log_softmax(logits64(w, np.concatenate([prompt, c])[:-1], form)[prompt.size - 1:], -1)
        want = want[torch.arange(c.size), torch.as_tensor(c, device=DEV).long()]
        # (as for the same model's other logits in 32 bits)
        assert float((lp.double() - want).abs().max()) < 1e-4
        one, _ = d.score(prompt, c)
        assert float((one - lp).abs().max()) < 2e-4
    # a prompt of one token
    lp = d.score_all(prompt[:1], conts[1:2])[0]
    assert float((lp - d.score(prompt[:1], conts[1])[0]).abs().max()) < 2e-4


@gpu
@pytest.mark.parametrize("form", FORMS[:2])
def test_search_under_rules(form):
    """Penalties, a bias and a grammar that depends on the text, against the same search on the logits in 64 bits."""
    build.build()
    w = weights()
    beams, new = 4, 6
    prompt = synth.prompt(8, M.vocab, 50, 0.4, 3, 6)
    bias = torch.randn(M.vocab, device=DEV, generator=torch.Generator(device=DEV).manual_seed(2))

    def grammar(texts):                                             # a token's successor is of another class modulo 3
        return (torch.arange(M.vocab, device=texts.device)[None] % 3) != (texts[:, -1:] % 3)

    d = decoder(w, form, beams, prompt.size + new, 8, 64)
    text, score = d.search(prompt, new, repetition=1.3, presence=0.2, frequency=0.1, bias=bias, allowed=lambda t: allowed_words(grammar(t)))

    def ruled(tokens):
        x = logits64(w, tokens, form)[-1]
        ids, c = torch.as_tensor(np.asarray(tokens), device=DEV).long().unique(return_counts=True)
        y = x[ids]
        x[ids] = torch.where(y > 0, y / 1.3, y * 1.3) - (0.1 * c + 0.2)
        x = x + bias.double()
        ok = grammar(torch.as_tensor(np.asarray(tokens), device=DEV)[None])[0]
        return torch.log_softmax(torch.where(ok, x, -float("inf")), -1).cpu().numpy()

    texts = [([], 0.0)]
    for _ in range(new):
        found = []
        for tail, s in texts:
            lp = ruled(list(prompt) + tail)
            found += [(tail + [int(t)], s + lp[t]) for t in np.argsort(-lp, kind="stable")[:beams]]
        texts = sorted(found, key=lambda f: -f[1])[:beams]
    assert np.abs(score.cpu().numpy() - np.array([s for _, s in texts])).max() < 1e-3
    gaps = -np.diff([s for _, s in texts])
    for i, (tokens, _) in enumerate(texts):                         # beams that no other is level with
        if (i == 0 or gaps[i - 1] > 2e-3) and (i == len(gaps) or gaps[i] > 2e-3):
            assert text[i].tolist() == tokens, i
    a = np.concatenate([[prompt[-1]], text[0].cpu().numpy()]) % 3
    assert bool((a[1:] != a[:-1]).all())


@gpu
def test_rules_may_be_given_one_by_one():
    build.build()
    w = weights()
    prompt = synth.prompt(8, M.vocab, 30, 0.4, 3, 6)
    d = decoder(w, {}, 3, 40, 8, 16)
    free, s0 = d.search(prompt, 5)
    mask = torch.ones(M.vocab, dtype=torch.bool, device=DEV)
    same, s1 = d.search(prompt, 5, allowed=allowed_words(mask))
    assert torch.equal(free, same) and torch.equal(s0, s1)
    mask[free.unique().long()] = False                              # none of what came before
    other, _ = d.search(prompt, 5, allowed=allowed_words(mask))
    assert bool(mask[other.long()].all())
    told = torch.zeros(M.vocab, dtype=torch.bool, device=DEV)
    told[torch.as_tensor(prompt, device=DEV).long()] = True
    new, _ = d.search(prompt, 3, presence=1e4)                      # nothing twice
    assert not bool(told[new.long()].any()) and all(len(set(row)) == 3 for row in new.tolist())
    up, _ = d.search(prompt, 2, bias=torch.nn.functional.one_hot(torch.tensor(17), M.vocab).float().to(DEV) * 1e4)
    assert up[0].tolist() == [17, 17]


@gpu
def test_bf16_prompt_chunks_agree():
    """The same model with its prompt in steps of 16 and in one chunk: logits differ by the roundings of 16 bits only."""
    build.build()
    m = synth.ModelDesc(2, 512, 8, 2, 64, 512, 1024, 256, "bf16")
    w = synth.model_weights(m, 9, device=DEV)
    prompt = synth.prompt(1, m.vocab, 200, 0.4, 4, 8)
    cont = synth.prompt(2, m.vocab, 30, 0.4, 4, 8)
    a, _ = BeamDecoder(m, w, 2, 240, chunk=16).score(prompt, cont)
    b, _ = BeamDecoder(m, w, 2, 240, chunk=4096).score(prompt, cont)
    # (a few 2^-8 of logits up to 2)
    assert float((a - b).abs().max()) < 0.05


def bare():
    d = object.__new__(BeamDecoder)                                 # without a cache: nothing here gets that far
    d.m, d.beams, d.max_len = M, 2, 20
    return d


@pytest.mark.parametrize("prompt,conts", [([1], []), ([1], [[1], [2], [3]]), ([1], [[]]), ([], [[1]]), ([1], [[1], [300]]), ([1] * 15, [[1], [1] * 6])])
def test_score_all_refuses(prompt, conts):
    with pytest.raises(ValueError):
        bare().score_all(prompt, conts)


def test_decoder_refuses():
    with pytest.raises(ValueError):
        BeamDecoder(M, {}, 2, 20, chunk=0)
    with pytest.raises(ValueError):
        BeamDecoder(M, {}, 2, 20, rotary=Rotary(64, device="cpu"))
