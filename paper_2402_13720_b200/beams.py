"""Several continuations of one prompt at once: beam search over a paged cache.

    python -m paper_2402_13720_b200.beams [--config C1] [--beams 4] [--new 32] [--layers N]

One step of the search: the scores of every beam's best tokens (``token_logprobs``), the best beams among them, the pages of their parents
(``PagedCache.fork``), room for a token (``extend``, which copies an unfinished page that several beams share), and a forward pass whose layers
write the new keys and values to their pages (``append``) and attend to them (``attend``).  The prompt is cached once and shared by all beams;
it goes through the same forward, sixteen tokens at a time.  Projections and FFN are torch's matrix products: this is the cache, its attention and
the scores at work, not the decoding path of this library (``Engine``).
"""
from __future__ import annotations

import argparse
import time

import numpy as np
import torch

from . import build, synth
from .binding import OURO_MAX_NEW, OURO_MAX_TOP
from .paged import PagedCache, rotary_tables
from .scores import token_logprobs


class BeamDecoder:
    """A Llama-style model (``synth.ModelDesc`` and its weights) with a paged cache for ``beams`` continuations of up to ``max_len`` tokens."""

    def __init__(self, m: synth.ModelDesc, w: dict, beams: int, max_len: int, page_size: int = 16, device="cuda:0"):
        if not 1 <= beams <= OURO_MAX_TOP:
            raise ValueError(f"1 to {OURO_MAX_TOP} beams")
        self.m, self.w, self.beams, self.max_len = m, w, beams, max_len
        self.device = torch.device(device)
        # weights laid out once: one product for q, k and v, one for gate and up
        self.qkv = [torch.cat([lw["wq"], lw["wk"], lw["wv"]]) for lw in w["layers"][: m.n_layers]]
        self.gate_up = [torch.cat([lw["w_gate"], lw["w_up"]]) for lw in w["layers"][: m.n_layers]]
        pages = -(-max_len // page_size)
        # every beam on pages of its own in the worst case, and a page each that is given up only after the copy
        self.cache = PagedCache(m.n_layers, beams * (pages + 1), page_size, m.n_kv_heads, m.head_dim, m.dtype, max_seqs=beams, max_pages=pages, device=device)
        self.cos, self.sin = rotary_tables(max_len, m.head_dim, m.rope_theta, device)
        self.all = torch.arange(beams, dtype=torch.int32, device=device)

    def _norm(self, x, gain):
        y = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + self.m.rms_eps)
        return (gain.float() * y).to(self.m.torch_dtype)

    def forward(self, tokens: torch.Tensor, seqs: torch.Tensor) -> torch.Tensor:
        """tokens [n, t]: the t newest of each of the sequences.  Extends the cache by them; logits [n * t, vocab]."""
        m, c = self.m, self.cache
        n, t = tokens.shape
        slots, positions = c.extend(seqs, torch.full((n,), t, dtype=torch.int32, device=self.device), t)
        slots, positions = slots.view(-1), positions.view(-1)
        heads, kv = m.n_heads, m.n_kv_heads
        x = self.w["embed"][tokens.reshape(-1).long()].float()
        for l in range(m.n_layers):
            lw = self.w["layers"][l]
            p = (self._norm(x, lw["attn_norm"]) @ self.qkv[l].T).view(n * t, heads + 2 * kv, m.head_dim)
            q = c.append(l, p[:, :heads], p[:, heads: heads + kv], p[:, heads + kv:], slots, positions, self.cos, self.sin)
            a = c.attend(l, q.view(n, t, heads, m.head_dim), seqs)
            x = x + (a.reshape(n * t, -1) @ lw["wo"].T).float()
            g, u = (self._norm(x, lw["ffn_norm"]) @ self.gate_up[l].T).float().chunk(2, -1)
            x = x + ((torch.nn.functional.silu(g) * u).to(m.torch_dtype) @ lw["w_down"].T).float()
        return self._norm(x, self.w["final_norm"]) @ self.w["lm_head"].T

    def _text(self, prompt, more=(), new: int = 0):
        """A prompt, and what follows it (`more`, or `new` tokens to come), as int32 arrays of tokens that the model has: the embedding is indexed with them."""
        prompt, more = np.asarray(prompt, dtype=np.int32).reshape(-1), np.asarray(more, dtype=np.int32).reshape(-1)
        if prompt.size < 1 or more.size + new < 1 or prompt.size + more.size + new > self.max_len:
            raise ValueError("the prompt or what is to follow is empty, or the two are longer than max_len")
        both = np.concatenate([prompt, more])
        if both.min() < 0 or both.max() >= self.m.vocab:
            raise ValueError(f"a token is not one of the model's {self.m.vocab}")
        return prompt, more

    def search(self, prompt, max_new: int):
        """The ``beams`` best continuations of max_new tokens that a beam search finds: tokens [beams, max_new], sums of log probabilities
        [beams], best first."""
        prompt, _ = self._text(prompt, new=max_new)
        m, B, c = self.m, self.beams, self.cache
        c.reset()
        ids = torch.as_tensor(prompt, device=self.device)
        for a in range(0, prompt.size, OURO_MAX_NEW):               # the prompt, once
            logits = self.forward(ids[None, a: a + OURO_MAX_NEW], self.all[:1])
        c.fork(torch.zeros_like(self.all), self.all)                # all beams begin there
        n_top = min(B, m.vocab)
        first = token_logprobs(logits[-1:], None, n_top)
        score = torch.full((B,), -float("inf"), device=self.device)
        score[:n_top] = first.top_logprobs[0]
        token = torch.zeros(B, dtype=torch.int32, device=self.device)
        token[:n_top] = first.top_ids[0]
        text = token[:, None]
        for _ in range(max_new - 1):
            s = token_logprobs(self.forward(token[:, None], self.all), None, n_top)
            score, pick = (score[:, None] + s.top_logprobs).view(-1).topk(B)
            parents = (pick // n_top).int()
            token = s.top_ids.view(-1)[pick]
            c.fork(parents, self.all)
            text = torch.cat([text[parents.long()], token[:, None]], 1)
        c.check()
        return text, score

    def score(self, prompt, continuation):
        """Log probability and entropy of every token of a given continuation."""
        prompt, cont = self._text(prompt, continuation)
        self.cache.reset()
        ids = torch.as_tensor(np.concatenate([prompt, cont])[:-1], device=self.device)
        logits = torch.cat([self.forward(ids[None, a: a + OURO_MAX_NEW], self.all[:1]) for a in range(0, ids.numel(), OURO_MAX_NEW)])
        s = token_logprobs(logits[prompt.size - 1:], torch.as_tensor(cont, device=self.device))
        self.cache.check()
        return s.logprob, s.entropy


def main():
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--config", default="C1", help="target model and prompt of synth.config")
    ap.add_argument("--beams", type=int, default=4)
    ap.add_argument("--new", type=int, default=32)
    ap.add_argument("--layers", type=int, default=0, help="use the first N layers only")
    a = ap.parse_args()
    build.build()
    m, _, _, r = synth.config(a.config)
    if a.layers:
        m = m.early_exit(a.layers)
    prompt = synth.prompt(0, m.vocab, r["n"], r["copy_frac"], *r["span"])
    d = BeamDecoder(m, synth.model_weights(m, 0, device="cuda:0"), a.beams, len(prompt) + a.new)
    text, score = d.search(prompt, a.new)                           # (and warm)
    torch.cuda.synchronize()
    t = time.perf_counter()
    text, score = d.search(prompt, a.new)
    torch.cuda.synchronize()
    t = time.perf_counter() - t
    used = int((d.cache.refs > 0).sum())
    alone = a.beams * -(-(len(prompt) + a.new - 1) // d.cache.page_size)
    print(f"{a.beams} beams of {a.new} tokens behind {len(prompt)}: {t * 1e3:.1f} ms, {a.beams * a.new / t:.0f} tokens/s; "
          f"{used} pages in use, {alone} if nothing were shared")
    for row, s in zip(text.tolist(), score.tolist()):
        print(f"{s:9.3f}  {row[:16]}{' ..' if len(row) > 16 else ''}")
    logprob, entropy = d.score(prompt, text[0].cpu())
    print(f"the best, scored again: {float(logprob.sum()):.3f}, mean entropy {float(entropy.mean()):.3f}")


if __name__ == "__main__":
    main()
