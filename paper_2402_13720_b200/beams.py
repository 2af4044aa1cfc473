"""Several continuations of one prompt at once: beam search over a paged cache.

    python -m paper_2402_13720_b200.beams [--config C1] [--beams 4] [--new 32] [--layers N] [--chunk 16] [--repetition 1.0]

One step of the search: the scores of every beam's best tokens (``token_logprobs``), the best beams among them, the pages of their parents
(``PagedCache.fork``), room for a token (``extend``, which copies an unfinished page that several beams share), and a forward pass whose layers
write the new keys and values to their pages (``append``, or ``append_rotary`` for models with other rotary positions) and attend to them (``attend``).
The prompt is cached once and shared by all beams; it goes through the same forward, ``chunk`` tokens at a time, as do texts to be scored
(``attend_chunk`` where that is more than sixteen, or differs from text to text).  Penalties, biases and grammars are put on the logits before they are
scored (``constrain_logits``).  Projections and FFN are torch's matrix products: this is the cache, its attention and the scores at work, not the decoding path
of this library (``Engine``).
"""
from __future__ import annotations

import argparse
import time

import numpy as np
import torch

from . import build, synth
from .binding import OURO_MAX_NEW, OURO_MAX_TOP
from .paged import PagedCache, rotary_tables
from .rotary import Rotary
from .scores import constrain_logits, token_logprobs


class BeamDecoder:
    """A Llama-style model (``synth.ModelDesc`` and its weights) with a paged cache for ``beams`` continuations of up to ``max_len`` tokens.
    ``rotary``: its positions, where they are not whole heads of half-split pairs; ``chunk``: tokens of a prompt that one forward takes."""

    def __init__(self, m: synth.ModelDesc, w: dict, beams: int, max_len: int, page_size: int = 16, device="cuda:0", rotary: Rotary | None = None,
                 chunk: int = OURO_MAX_NEW):
        if not 1 <= beams <= OURO_MAX_TOP:
            raise ValueError(f"1 to {OURO_MAX_TOP} beams")
        if chunk < 1:
            raise ValueError("a chunk has a token at least")
        if rotary is not None and rotary.head_dim != m.head_dim:
            raise ValueError(f"rotary: positions for heads of {m.head_dim} are needed")
        self.m, self.w, self.beams, self.max_len = m, w, beams, max_len
        self.device = torch.device(device)
        # weights laid out once: one product for q, k and v, one for gate and up
        self.qkv = [torch.cat([lw["wq"], lw["wk"], lw["wv"]]) for lw in w["layers"][: m.n_layers]]
        self.gate_up = [torch.cat([lw["w_gate"], lw["w_up"]]) for lw in w["layers"][: m.n_layers]]
        pages = -(-max_len // page_size)
        # every beam on pages of its own in the worst case, and a page each that is given up only after the copy
        self.cache = PagedCache(m.n_layers, beams * (pages + 1), page_size, m.n_kv_heads, m.head_dim, m.dtype, max_seqs=beams, max_pages=pages, device=device)
        self.rotary, self.chunk = rotary, chunk
        if rotary is None:
            self.cos, self.sin = rotary_tables(max_len, m.head_dim, m.rope_theta, device)
        self.all = torch.arange(beams, dtype=torch.int32, device=device)

    def _norm(self, x, gain):
        y = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + self.m.rms_eps)
        return (gain.float() * y).to(self.m.torch_dtype)

    def _layers(self, tokens, slots, positions, attend, first):
        """Rows of tokens through the model; attend(layer, q): attention of the rotated queries [rows, heads, head_dim].  Logits of the rows from `first` on, None where
        that is none of them."""
        m, c = self.m, self.cache
        heads, kv = m.n_heads, m.n_kv_heads
        x = self.w["embed"][tokens.long()].float()
        for l in range(m.n_layers):
            lw = self.w["layers"][l]
            p = (self._norm(x, lw["attn_norm"]) @ self.qkv[l].T).view(-1, heads + 2 * kv, m.head_dim)
            new = p[:, :heads], p[:, heads: heads + kv], p[:, heads + kv:]
            if self.rotary is None:
                q = c.append(l, *new, slots, positions, self.cos, self.sin)
            else:
                q = c.append_rotary(l, *new, slots, positions, self.rotary)
            x = x + (attend(l, q).reshape(x.shape[0], -1) @ lw["wo"].T).float()
            g, u = (self._norm(x, lw["ffn_norm"]) @ self.gate_up[l].T).float().chunk(2, -1)
            x = x + ((torch.nn.functional.silu(g) * u).to(m.torch_dtype) @ lw["w_down"].T).float()
        return self._norm(x[first:], self.w["final_norm"]) @ self.w["lm_head"].T if first < x.shape[0] else None

    def forward(self, tokens: torch.Tensor, seqs: torch.Tensor, first: int = 0) -> torch.Tensor | None:
        """tokens [n, t], t <= 16: the t newest of each of the sequences.  Extends the cache by them; logits [n * t, vocab], those in front of row `first` left out."""
        n, t = tokens.shape
        slots, positions = self.cache.extend(seqs, torch.full((n,), t, dtype=torch.int32, device=self.device), t)
        shape = (n, t, self.m.n_heads, self.m.head_dim)
        return self._layers(tokens.reshape(-1), slots.view(-1), positions.view(-1), lambda l, q: self.cache.attend(l, q.view(shape), seqs), first)

    def forward_chunks(self, tokens: torch.Tensor, lens, seqs: torch.Tensor, first: int = 0) -> torch.Tensor | None:
        """The same with lens[i] >= 1 new tokens of sequence seqs[i], one sequence's after the other's in tokens [sum of lens]; logits [sum of lens, vocab]."""
        lens = np.asarray(lens, dtype=np.int32)
        ends = np.cumsum(lens, dtype=np.int32)
        starts = torch.as_tensor(np.concatenate([[0], ends]).astype(np.int32), device=self.device)
        width = int(lens.max())
        slots, positions = self.cache.extend(seqs, torch.as_tensor(lens, device=self.device), width)
        if width * lens.size > int(ends[-1]):                       # rows of different lengths: the padding goes
            rows = torch.as_tensor(np.concatenate([i * width + np.arange(k) for i, k in enumerate(lens)]), device=self.device)
            slots, positions = slots.view(-1)[rows], positions.view(-1)[rows]
        return self._layers(tokens, slots.view(-1), positions.view(-1), lambda l, q: self.cache.attend_chunk(l, q, starts, seqs), first)

    def _read(self, ids: torch.Tensor, first: int):
        """Caches a text as sequence 0, a chunk at a time.  Logits behind its tokens from the first-th on; None where it has none.  Of what lies in front of them
        nothing is kept, and the output matrix is not asked (but for what shares its sixteen rows of a chunk with the first)."""
        out = []
        for a in range(0, ids.numel(), self.chunk):
            piece = ids[a: a + self.chunk]
            skip = max(first - a, 0)
            whole = skip // OURO_MAX_NEW * OURO_MAX_NEW if skip < piece.numel() else skip
            if self.chunk <= OURO_MAX_NEW:
                logits = self.forward(piece[None], self.all[:1], whole)
            else:
                logits = self.forward_chunks(piece, [piece.numel()], self.all[:1], whole)
            if logits is not None:
                out.append(logits[skip - whole:])
        return torch.cat(out) if out else None

    def _text(self, prompt, more=(), new: int = 0):
        """A prompt, and what follows it (`more`, or `new` tokens to come), as int32 arrays of tokens that the model has: the embedding is indexed with them."""
        prompt, more = np.asarray(prompt, dtype=np.int32).reshape(-1), np.asarray(more, dtype=np.int32).reshape(-1)
        if prompt.size < 1 or more.size + new < 1 or prompt.size + more.size + new > self.max_len:
            raise ValueError("the prompt or what is to follow is empty, or the two are longer than max_len")
        both = np.concatenate([prompt, more])
        if both.min() < 0 or both.max() >= self.m.vocab:
            raise ValueError(f"a token is not one of the model's {self.m.vocab}")
        return prompt, more

    def _constrain(self, logits, told, rules):
        """Rules on rows of logits whose texts are told [rows, length], in place."""
        rows = logits.shape[0]
        penalties = {k: torch.full((rows,), float(rules[k]), device=self.device) for k in ("repetition", "presence", "frequency") if rules[k] is not None}
        allowed = rules["allowed"](told) if callable(rules["allowed"]) else rules["allowed"]
        return constrain_logits(logits, tokens=told if penalties else None, **penalties, bias=rules["bias"], allowed=allowed, out=logits)

    def search(self, prompt, max_new: int, *, repetition: float | None = None, presence: float | None = None, frequency: float | None = None,
               bias: torch.Tensor | None = None, allowed=None):
        """The ``beams`` best continuations of max_new tokens that a beam search finds: tokens [beams, max_new], sums of log probabilities
        [beams], best first.  Rules as in ``constrain_logits``, penalties for what the prompt and the continuation have, ``bias`` [vocab]; ``allowed``: the words of
        one mask for all, or a function of the texts [rows, length] int32 (prompt first) that gives the words [rows, ceil(vocab / 32)] of theirs."""
        prompt, _ = self._text(prompt, new=max_new)
        m, B, c = self.m, self.beams, self.cache
        rules = dict(repetition=repetition, presence=presence, frequency=frequency, bias=bias, allowed=allowed)
        ruled = any(x is not None for x in rules.values())
        c.reset()
        ids = torch.as_tensor(prompt, device=self.device)
        logits = self._read(ids, prompt.size - 1)                   # the prompt, once
        c.fork(torch.zeros_like(self.all), self.all)                # all beams begin there
        n_top = min(B, m.vocab)
        first = token_logprobs(self._constrain(logits, ids[None], rules) if ruled else logits, None, n_top)
        score = torch.full((B,), -float("inf"), device=self.device)
        score[:n_top] = first.top_logprobs[0]
        token = torch.zeros(B, dtype=torch.int32, device=self.device)
        token[:n_top] = first.top_ids[0]
        text = token[:, None]
        for _ in range(max_new - 1):
            logits = self.forward(token[:, None], self.all)
            if ruled:
                logits = self._constrain(logits, torch.cat([ids.expand(B, -1), text], 1), rules)
            s = token_logprobs(logits, None, n_top)
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
        s = token_logprobs(self._read(ids, prompt.size - 1), torch.as_tensor(cont, device=self.device))
        self.cache.check()
        return s.logprob, s.entropy

    def score_all(self, prompt, continuations):
        """Log probabilities of every token of several continuations of a prompt, each of a length of its own, at most ``beams`` of them: the prompt is
        cached once, all continuations go through one forward.  A list of tensors."""
        if not 1 <= len(continuations) <= self.beams:
            raise ValueError(f"1 to {self.beams} continuations")
        texts = [self._text(prompt, c) for c in continuations]
        prompt, conts = texts[0][0], [c for _, c in texts]
        self.cache.reset()
        self._read(torch.as_tensor(prompt[:-1], device=self.device), prompt.size)
        seqs = self.all[: len(conts)]
        self.cache.fork(torch.zeros_like(seqs), seqs)
        rows = np.concatenate([np.concatenate([prompt[-1:], c[:-1]]) for c in conts])
        logits = self.forward_chunks(torch.as_tensor(rows, device=self.device), [c.size for c in conts], seqs)
        s = token_logprobs(logits, torch.as_tensor(np.concatenate(conts), device=self.device))
        self.cache.check()
        return list(s.logprob.split([c.size for c in conts]))


def main():
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--config", default="C1", help="target model and prompt of synth.config")
    ap.add_argument("--beams", type=int, default=4)
    ap.add_argument("--new", type=int, default=32)
    ap.add_argument("--layers", type=int, default=0, help="use the first N layers only")
    ap.add_argument("--chunk", type=int, default=OURO_MAX_NEW, help="tokens of the prompt in one forward")
    ap.add_argument("--repetition", type=float, default=None, help="penalty for tokens that the text has already")
    a = ap.parse_args()
    build.build()
    m, _, _, r = synth.config(a.config)
    if a.layers:
        m = m.early_exit(a.layers)
    prompt = synth.prompt(0, m.vocab, r["n"], r["copy_frac"], *r["span"])
    d = BeamDecoder(m, synth.model_weights(m, 0, device="cuda:0"), a.beams, len(prompt) + a.new, chunk=a.chunk)
    text, score = d.search(prompt, a.new, repetition=a.repetition)  # (and warm)
    torch.cuda.synchronize()
    t = time.perf_counter()
    text, score = d.search(prompt, a.new, repetition=a.repetition)
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
    again = d.score_all(prompt, list(text.cpu()))
    print("all, in one forward: " + " ".join(f"{float(x.sum()):.3f}" for x in again))


if __name__ == "__main__":
    main()
