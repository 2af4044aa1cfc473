"""What a beam decoder works out and keeps of a text that it reads: logits behind the tokens that are asked about, not of a whole prompt."""
import numpy as np
import pytest
import torch

from paper_2402_13720_b200 import beams, build, synth
from paper_2402_13720_b200.beams import BeamDecoder

gpu = pytest.mark.gpu


class Stop(Exception):
    pass


class Room:
    """A cache that has room for everything and keeps nothing."""

    def reset(self):
        self.tokens = 0

    def extend(self, seqs, new, width):
        self.tokens += int(new.sum())
        return torch.zeros((2, seqs.numel(), width), dtype=torch.int32).unbind()

    def fork(self, src, dst):
        pass


@pytest.fixture
def decoder(monkeypatch):
    """A decoder without layers, on the CPU, up to where scores are asked for; rows: how many went through the output matrix at a time."""
    def make(chunk):
        d = object.__new__(BeamDecoder)
        d.m = synth.ModelDesc(0, 16, 2, 2, 32, 16, 50, 400, "f32")
        d.w = {"embed": torch.randn((50, 16)), "layers": [], "final_norm": torch.ones(16), "lm_head": torch.randn((50, 16))}
        d.beams, d.max_len, d.chunk, d.cache, d.device = 3, 400, chunk, Room(), torch.device("cpu")
        d.all = torch.arange(3, dtype=torch.int32)
        d.rows = []
        norm = d._norm

        def spy(x, gain):
            d.rows.append(x.shape[0])
            return norm(x, gain)

        d._norm = spy
        return d

    def stop(logits, *_):
        raise Stop(logits)

    monkeypatch.setattr(beams, "token_logprobs", stop)
    return make


def plain(d, text):
    x = d.w["embed"][torch.as_tensor(np.asarray(text)).long()]
    return (x * torch.rsqrt((x * x).mean(-1, keepdim=True) + d.m.rms_eps)) @ d.w["lm_head"].T


@pytest.mark.parametrize("chunk", [1, 5, 16, 17, 64, 1000])
@pytest.mark.parametrize("n", [1, 15, 16, 17, 200])
def test_search_works_out_the_last_rows_only(decoder, chunk, n):
    d = decoder(chunk)
    prompt = np.random.default_rng(n).integers(0, 50, n)
    with pytest.raises(Stop) as e:
        d.search(prompt, 4)
    logits = e.value.args[0]
    assert d.cache.tokens == n and len(d.rows) == 1 and d.rows[0] <= 16
    assert logits.shape == (1, 50) and torch.allclose(logits, plain(d, prompt)[-1:], atol=1e-5)


@pytest.mark.parametrize("chunk", [1, 5, 16, 17, 64, 1000])
@pytest.mark.parametrize("n,new", [(1, 1), (1, 40), (33, 1), (150, 70), (160, 16)])
def test_score_works_out_what_is_asked_about(decoder, chunk, n, new):
    d = decoder(chunk)
    text = np.random.default_rng(n).integers(0, 50, n + new)
    with pytest.raises(Stop) as e:
        d.score(text[:n], text[n:])
    logits = e.value.args[0]
    assert d.cache.tokens == n + new - 1 and sum(d.rows) < new + 16
    assert logits.shape == (new, 50) and torch.allclose(logits, plain(d, text[:-1])[n - 1:], atol=1e-5)


@pytest.mark.parametrize("chunk", [1, 5, 16, 17, 64, 1000])
@pytest.mark.parametrize("n", [1, 2, 100])
def test_score_all_works_out_nothing_of_the_prompt(decoder, chunk, n):
    d = decoder(chunk)
    r = np.random.default_rng(n)
    prompt, conts = r.integers(0, 50, n), [r.integers(0, 50, k) for k in (1, 20, 7)]
    with pytest.raises(Stop) as e:
        d.score_all(prompt, conts)
    logits = e.value.args[0]
    assert d.rows == [28] and d.cache.tokens == n - 1 + 28
    want = torch.cat([plain(d, np.concatenate([prompt[-1:], c[:-1]])) for c in conts])
    assert torch.allclose(logits, want, atol=1e-5)


@gpu
@pytest.mark.parametrize("chunk", [16, 300])
def test_memory_does_not_grow_with_the_prompt(chunk):
    build.build()
    m = synth.ModelDesc(1, 64, 2, 2, 32, 64, 60000, 2100, "f32")
    w = synth.model_weights(m, 1, device="cuda:0")
    d = BeamDecoder(m, w, 2, 2100, chunk=chunk)
    prompt = synth.prompt(1, m.vocab, 2000, 0.4, 4, 8)
    cont = synth.prompt(2, m.vocab, 20, 0.4, 4, 8)
    for call in (lambda: d.search(prompt, 2), lambda: d.score(prompt, cont), lambda: d.score_all(prompt, [cont, cont[:3]])):
        call()
        torch.cuda.synchronize()
        before = torch.cuda.memory_allocated()
        torch.cuda.reset_peak_memory_stats()
        call()
        torch.cuda.synchronize()
        # (the prompt's logits are 480 MB; 36 rows of them are 8.6, and a few copies)
        assert torch.cuda.max_memory_allocated() - before < 64 << 20
