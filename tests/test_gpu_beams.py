"""Beam search over the paged cache, its attention and the token scores together, against the same search on the oracle's logits in 64 bits."""
import numpy as np
import pytest
import torch

from oracle import transformer as tf
from paper_2402_13720_b200 import build, synth
from paper_2402_13720_b200.beams import BeamDecoder

pytestmark = pytest.mark.gpu


def oracle_logprobs(W, desc, tokens):
    """Log probabilities behind every token of a text, in 64 bits, without a cache."""
    n = len(tokens)
    x = tf.forward(W, tf.KVCache(desc), list(tokens), list(range(n)), np.tril(np.ones((n, n), dtype=bool)))
    x = x - x.max(axis=1, keepdims=True)
    return x - np.log(np.exp(x).sum(axis=1, keepdims=True))


def oracle_search(W, desc, prompt, beams, new):
    texts = [([], 0.0)]
    for _ in range(new):
        found = []
        for text, score in texts:
            lp = oracle_logprobs(W, desc, list(prompt) + text)[-1]
            found += [(text + [int(t)], score + lp[t]) for t in np.argsort(-lp, kind="stable")[:beams]]
        texts = sorted(found, key=lambda f: -f[1])[:beams]
    return texts


def spread(desc, seed):
    """Weights whose logits tell tokens apart: the head's rows four times as large."""
    w = synth.model_weights(desc, seed)
    w["lm_head"] = w["lm_head"] * 4
    return w


def on_gpu(w):
    return {k: [{n: t.cuda() for n, t in lw.items()} for lw in v] if k == "layers" else v.cuda() for k, v in w.items()}


@pytest.mark.parametrize("beams,prompt_len,new,page", [(1, 5, 6, 4), (4, 19, 7, 8), (7, 33, 6, 5)])
def test_beam_search_finds_what_the_oracle_finds(beams, prompt_len, new, page):
    build.build()
    desc = synth.ModelDesc(2, 128, 4, 2, 32, 256, 300, 64, "f32")
    w = spread(desc, 5)
    prompt = synth.prompt(beams, desc.vocab, prompt_len, 0.4, 3, 6)
    d = BeamDecoder(desc, on_gpu(w), beams, prompt_len + new, page)
    text, score = d.search(prompt, new)
    W = tf.Weights(desc, w)
    want = oracle_search(W, desc, prompt, beams, new)
    # (sums of six log probabilities, each off by less than the f32 logits' 1e-4)
    assert np.abs(score.cpu().numpy() - np.array([s for _, s in want])).max() < 1e-3
    gaps = -np.diff([s for _, s in want])
    for i, (tokens, _) in enumerate(want):                 # beams that no other is level with
        if (i == 0 or gaps[i - 1] > 2e-3) and (i == len(gaps) or gaps[i] > 2e-3):
            assert text[i].tolist() == tokens, i
    # a given text, scored through the same cache
    logprob, entropy = d.score(prompt, text[0].cpu())
    lp = oracle_logprobs(W, desc, list(prompt) + text[0].tolist()[:-1])[prompt_len - 1:]
    assert np.abs(logprob.cpu().numpy() - lp[np.arange(new), text[0].cpu().numpy()]).max() < 1e-4
    assert np.abs(entropy.cpu().numpy() + (np.exp(lp) * lp).sum(axis=1)).max() < 1e-3
    # the counts are those of the table
    assert int((d.cache.table >= 0).sum()) == int(d.cache.refs.sum()) and int(d.cache.lens.max()) <= prompt_len + new


def test_beam_search_in_bf16_shares_pages_and_scores_its_own_text():
    build.build()
    desc = synth.ModelDesc(2, 512, 8, 2, 64, 512, 1024, 256, "bf16")
    w = synth.model_weights(desc, 9, device="cuda:0")
    w["lm_head"] = w["lm_head"] * 4
    prompt = synth.prompt(1, desc.vocab, 100, 0.4, 4, 8)
    d = BeamDecoder(desc, w, 6, 140)
    text, score = d.search(prompt, 30)
    assert text.shape == (6, 30) and bool((score[:-1] >= score[1:]).all()) and len({tuple(t) for t in text.tolist()}) == 6
    assert int((d.cache.refs > 1).sum()) >= 100 // 16      # the prompt's whole pages at least
    logprob, _ = d.score(prompt, text[0].cpu())
    # the same sums but for the rounding of other block sizes in 16 bits: 30 tokens, each off by a few 2^-8 of logits up to 8
    assert abs(float(logprob.sum()) - float(score[0])) < 30 * 0.05
    with pytest.raises(ValueError):
        d.search(prompt, 41)
