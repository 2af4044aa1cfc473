"""Performance cases of the operators that several continuations of a text need: a paged key-value cache, attention over
it, the step that writes it, and the scores by which continuations are chosen.

  attend   attention of the newest tokens of n sequences over their pages
  append   rotary positions for new queries and keys; keys and values to their pages
  pages    fork and extend (a step of a beam search), or truncate and compact (sequences end, the pool is tidied up)
  score    log probabilities of given tokens with entropy and the best alternatives

Head layouts, layers and vocabularies are those of this repository's configurations (``synth.config``).  Lengths, batch and
page sizes are generic.  ``run`` computes the plain form out of elementary torch operations in 32 bits; with ``own`` set it
calls the framework.
"""
from __future__ import annotations

import math
import random

import numpy as np
import torch

own = False

# layers, query heads, kv heads, head dim, vocabulary
SHAPES = {
    "tiny": (2, 4, 4, 32, 512),
    "small": (2, 4, 2, 128, 1024),
    "1b": (22, 32, 4, 64, 32000),
    "7b": (32, 32, 32, 128, 32000),
    "34b": (60, 56, 8, 128, 64000),
    "70b": (80, 64, 8, 128, 32000),
}
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
DEVICE = "cuda:0"


def listed():
    return [
        # The smallest use: one token of one short text, the fp32 model of the tests.
        dict(name="attend_tiny_f32", kind="attend", shape="tiny", dtype="f32", seqs=1, new=1, longest=67, ragged=False, page=16, layout=1),
        # A beam search with the 1.1B-shaped model: short ragged sequences, head dim 64, eight query heads to a kv head.
        dict(name="attend_1b_beams", kind="attend", shape="1b", dtype="bf16", seqs=24, new=1, longest=700, ragged=True, page=16, layout=2),
        # Plain decoding of a batch with the 7B shape, which has a kv head for every query head, at the benchmark's cache length.
        dict(name="attend_7b", kind="attend", shape="7b", dtype="bf16", seqs=8, new=1, longest=4096, ragged=True, page=32, layout=3),
        # Verification of four drafted tokens behind the pending one, seven query heads to a kv head.
        dict(name="attend_34b_drafts", kind="attend", shape="34b", dtype="bf16", seqs=5, new=5, longest=1777, ragged=True, page=64, layout=4),
        # A full batch with long contexts, the largest call.
        dict(name="attend_70b_long", kind="attend", shape="70b", dtype="bf16", seqs=48, new=1, longest=12345, ragged=True, page=128, layout=5),
        # One new token of one text, where only latency counts.
        dict(name="append_1b_token", kind="append", shape="1b", dtype="bf16", rows=1, padding=0, page=16, layout=6),
        # A prompt's rows enter the cache, among them the padding of shorter prompts.
        dict(name="append_70b_prompts", kind="append", shape="70b", dtype="bf16", rows=4100, padding=300, page=64, layout=7),
        # Between two steps of a beam search: beams continue their parents and get room for a token; shared partial pages are copied.
        dict(name="pages_beam_step", kind="pages", op="step", shape="1b", layers=22, dtype="bf16", seqs=12, new=1, longest=389, page=16, pool=400, layout=8),
        # Sequences end and the pool is tidied up, so that its end can be given back: whole pages of all layers move.
        dict(name="pages_compact_7b", kind="pages", op="compact", shape="7b", layers=32, dtype="bf16", seqs=16, longest=411, page=16, pool=300,
             moves=70, layout=9),
        # One generated token with its five best alternatives, as an API answers them.
        dict(name="score_token", kind="score", rows=1, vocab=32000, dtype="f32", top=5, banned=0.0, layout=10),
        # Expanding the beams of a constrained search: a part of the vocabulary is masked out.
        dict(name="score_beams", kind="score", rows=24, vocab=64000, dtype="bf16", top=24, banned=0.3, layout=11),
        # Scoring whole texts (perplexity, reranking), the largest call.
        dict(name="score_texts", kind="score", rows=2048, vocab=64000, dtype="f32", top=20, banned=0.0, layout=12),
    ]


def _between(rng, lo, hi):
    """Whole number spread over the logarithm of [lo, hi]."""
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["attend", "attend", "attend", "append", "step", "compact", "score", "score"])
    layout = rng.randrange(1 << 30)
    page = rng.choice([8, 16, 16, 24, 32, 64, 128])
    if kind == "attend":
        shape = rng.choice(["tiny", "small", "1b", "7b", "34b", "70b"])
        _, _, hkv, d, _ = SHAPES[shape]
        dtype = "f32" if shape == "tiny" or rng.random() < 0.15 else "bf16"
        longest = _between(rng, 1, 30000)
        room = 48 * 12345 * 8 * 128 * 2 // 2                      # about what the largest listed case reads
        most = max(1, min(96, room // (longest * hkv * d * (2 if dtype == "f32" else 1))))
        return dict(kind="attend", shape=shape, dtype=dtype, seqs=_between(rng, 1, most), new=rng.choice([1, 1, 1, 2, 5, 8]), longest=longest,
                    ragged=rng.random() < 0.75, page=page, layout=layout)
    if kind == "append":
        rows = _between(rng, 1, 4100)
        return dict(kind="append", shape=rng.choice(["tiny", "small", "1b", "7b", "34b", "70b"]), dtype=rng.choice(["bf16", "bf16", "f32"]) if rows < 2000 else "bf16",
                    rows=rows, padding=rng.randrange(rows // 4 + 1), page=page, layout=layout)
    if kind == "step":
        shape = rng.choice(["tiny", "small", "1b"])
        seqs = _between(rng, 2, 24)
        longest = _between(rng, 1, 1200)
        return dict(kind="pages", op="step", shape=shape, layers=SHAPES[shape][0], dtype="f32" if shape == "tiny" else "bf16", seqs=seqs, new=rng.choice([1, 1, 5, 37]),
                    longest=longest, page=page, pool=seqs * (-(-longest // page) + 37 // page + 3) + rng.randrange(40), layout=layout)
    if kind == "compact":
        shape = rng.choice(["tiny", "small", "1b", "7b"])
        layers = rng.randrange(1, SHAPES[shape][0] // (4 if shape == "7b" else 1) + 1)
        seqs = _between(rng, 2, 16)
        longest = _between(rng, 20, 700)
        live = seqs // 2 * -(-longest // page)                    # at most
        return dict(kind="pages", op="compact", shape=shape, layers=layers, dtype="bf16" if rng.random() < 0.7 else "f32", seqs=seqs, longest=longest, page=page,
                    pool=seqs * -(-longest // page) + live + 40, moves=rng.randrange(live + 1), layout=layout)
    vocab = rng.choice([512, 1024, 32000, 32000, 64000, _between(rng, 500, 130000)])
    rows = _between(rng, 1, max(2, min(2048, 2048 * 64000 // vocab)))
    return dict(kind="score", rows=rows, vocab=vocab, dtype=rng.choice(["f32", "f32", "bf16"]), top=rng.choice([0, 1, 5, 20, 32]),
                banned=rng.choice([0.0, 0.0, 0.3, 0.95]), layout=layout)


# ---- what a case fixes beside its sizes ---------------------------------------------------------------------------------
def _lens(case):
    """Lengths of the sequences of a case: equal, or ragged with one of the longest and one of a single token."""
    if not case.get("ragged", True):
        return [case["longest"]] * case["seqs"]
    r = random.Random(case["layout"])
    lens = [r.randint(1, case["longest"]) for _ in range(case["seqs"])]
    lens[r.randrange(len(lens))] = case["longest"]
    if len(lens) > 4:
        lens[r.randrange(len(lens))] = 1
    return lens


def _pages(n, page):
    return -(-n // page)


def _parents(case):
    """A step of a beam search: which beam each beam continues."""
    r = random.Random(case["layout"] + 1)
    return [r.randrange(case["seqs"]) if r.random() < 0.6 else i for i in range(case["seqs"])]


def _step_copies(case):
    """Pages that a step copies, and their rows: all but one of the beams that share an unfinished page."""
    lens, parents = _lens(case), _parents(case)
    shared = [p for p in parents if lens[p] % case["page"]]
    rows = sum((shared.count(p) - 1) * (lens[p] % case["page"]) for p in set(shared))
    return rows


def _staying(case):
    """Pages of the sequences that go on when the others have ended."""
    lens = _lens(case)
    return sum(_pages(n, case["page"]) for n in lens[: len(lens) // 2])


def _moves(case):
    stay = _staying(case)
    return min(case["moves"], stay, case["pool"] - stay)


def work(case):
    if case["kind"] == "score":
        e = 4 if case["dtype"] == "f32" else 2
        n = case["rows"] * case["vocab"]
        return {"bytes": n * e + case["rows"] * (12 + 8 * case["top"]), "flops": 6 * n}
    _, h, hkv, d, _ = SHAPES[case["shape"]]
    e = 4 if case["dtype"] == "f32" else 2
    if case["kind"] == "attend":
        lens = _lens(case)
        seen = [sum(max(0, n - case["new"] + 1 + i) for i in range(case["new"])) for n in lens]
        return {"bytes": sum(lens) * hkv * d * 2 * e + 2 * case["seqs"] * case["new"] * h * d * e + 4 * sum(_pages(n, case["page"]) + 1 for n in lens),
                "flops": 4 * d * h * sum(seen)}
    if case["kind"] == "append":
        live = case["rows"] - case["padding"]
        return {"bytes": 2 * case["rows"] * h * d * e + live * 4 * hkv * d * e + case["rows"] * (8 + 4 * d), "flops": 3 * d * (case["rows"] * h + live * hkv)}
    row = case["layers"] * 2 * hkv * d * e
    if case["op"] == "step":
        entries = sum(_pages(n, case["page"]) for n in _lens(case))
        return {"bytes": 2 * row * _step_copies(case) + 4 * (case["pool"] + 4 * entries), "flops": 0}
    return {"bytes": 2 * row * case["page"] * _moves(case) + 4 * 3 * case["pool"], "flops": 0}


# ---- inputs -------------------------------------------------------------------------------------------------------------
def _generator(seed):
    g = torch.Generator(device=DEVICE)
    g.manual_seed(seed)
    return g


def _randn(shape, dtype, g, scale=1.0):
    x = torch.randn(shape, dtype=dtype, device=DEVICE, generator=g)
    return x if scale == 1.0 else x.mul_(scale)


def _i32(values):
    return torch.tensor(np.asarray(values, dtype=np.int32), device=DEVICE)


def _rotary(positions, d):
    inv = 10000.0 ** (-2.0 * torch.arange(d // 2, dtype=torch.float64, device=DEVICE) / d)
    a = torch.arange(positions, dtype=torch.float64, device=DEVICE)[:, None] * inv
    return torch.cos(a).float(), torch.sin(a).float()


def _cache(st, max_seqs, max_pages):
    """The framework's handle of the pools and tables of a state."""
    from paper_2402_13720_b200.paged import PagedCache
    return PagedCache(k=st["k"], v=st["v"], max_seqs=max_seqs, max_pages=max_pages)


def prepare(case, seed):
    g = _generator(seed)
    r = random.Random(seed)
    dtype = DTYPES[case["dtype"]]
    if case["kind"] == "score":
        return _prepare_score(case, g, dtype)
    _, h, hkv, d, _ = SHAPES[case["shape"]]
    page = case["page"]
    st = dict(case=case)
    if case["kind"] == "append":
        # new rows of a few sequences, each at its own place in the pool; padding has no slot
        rows, live = case["rows"], case["rows"] - case["padding"]
        n_pages = 2 * _pages(rows, page) + 8
        ids = r.sample(range(n_pages), _pages(rows, page) + 1)
        slots = [ids[i // page] * page + i % page for i in range(live)] + [-1] * case["padding"]
        start = r.randrange(500)
        st.update(k=_randn((1, n_pages, page, hkv, d), dtype, g), v=_randn((1, n_pages, page, hkv, d), dtype, g),
                  q=_randn((rows, h, d), dtype, g), k_new=_randn((rows, hkv, d), dtype, g), v_new=_randn((rows, hkv, d), dtype, g),
                  slots=_i32(slots), positions=_i32([start + i for i in range(live)] + [0] * case["padding"]))
        st["cos"], st["sin"] = _rotary(start + rows, d)
        if own:
            st["cache"] = _cache(st, 1, 1)
        return st
    lens = _lens(case)
    n = len(lens)
    if case["kind"] == "attend":
        used = sum(_pages(x, page) for x in lens)
        n_pages = used + used // 8 + 3
        width = max(_pages(x, page) for x in lens) + 1
        ids = r.sample(range(n_pages), used)
        table = np.full((n, width), -1, dtype=np.int32)
        at = 0
        for i, x in enumerate(lens):
            m = _pages(x, page)
            table[i, :m] = ids[at: at + m]
            at += m
        # queries twice as wide as keys: attention that favours some keys, as trained models' does
        st.update(k=_randn((1, n_pages, page, hkv, d), dtype, g), v=_randn((1, n_pages, page, hkv, d), dtype, g),
                  q=_randn((n, case["new"], h, d), dtype, g, 2.0), table=_i32(table), lens=_i32(lens), longest=max(lens))
        if own:
            st["cache"] = _cache(st, n, width)
            st["cache"].table.copy_(st["table"])
            st["cache"].lens.copy_(st["lens"])
        return st
    pool, layers = case["pool"], case["layers"]
    table, refs = None, np.zeros(pool, dtype=np.int32)
    if case["op"] == "step":
        # beams that have run apart from a common beginning: the whole pages of it are shared
        width = _pages(case["longest"] + case["new"], page) + 2
        table = np.full((n, width), -1, dtype=np.int32)
        common = min(lens) // (2 * page)
        ids = r.sample(range(pool), common + sum(_pages(x, page) - common for x in lens))
        at = common
        for i, x in enumerate(lens):
            m = _pages(x, page)
            table[i, :common] = ids[:common]
            table[i, common:m] = ids[at: at + m - common]
            at += m - common
        st.update(parents=_i32(_parents(case)), beams=_i32(range(n)), new=_i32([case["new"]] * n))
    else:
        # the second half of the sequences ends; of the others' pages `moves` lie beyond the first ones
        width = _pages(case["longest"], page)
        table = np.full((n, width), -1, dtype=np.int32)
        stay, moves = _staying(case), _moves(case)
        ids = r.sample(range(stay), stay - moves) + r.sample(range(stay, pool), moves)
        r.shuffle(ids)
        rest = [p for p in range(pool) if p not in set(ids)]
        r.shuffle(rest)
        at = 0
        for i, x in enumerate(lens):
            m = _pages(x, page)
            if i == n // 2:
                ids, at = rest, 0
            table[i, :m] = ids[at: at + m]
            at += m
        st.update(ended=_i32(range(n // 2, n)), keep=_i32([0] * (n - n // 2)))
    for p in table[table >= 0]:
        refs[p] += 1
    st.update(k=_randn((layers, pool, page, hkv, d), dtype, g), v=_randn((layers, pool, page, hkv, d), dtype, g),
              start=torch.cat([_i32(table).view(-1), _i32(lens), _i32(refs)]), n=n, width=width)
    if own:
        st["cache"] = _cache(st, n, width)
    return st


def _prepare_score(case, g, dtype):
    rows, vocab = case["rows"], case["vocab"]
    x = _randn((rows, vocab), torch.float32, g, 2.0)
    # a few tokens stand out, less and less, as in a trained model's output
    few = 40
    at = torch.arange(few, device=DEVICE) * (vocab // few) + torch.randint(vocab // few, (rows, few), device=DEVICE, generator=g)
    at = (at + torch.randint(vocab, (rows, 1), device=DEVICE, generator=g)) % vocab
    x.scatter_(1, at, x.gather(1, at) + 12.0 * 0.85 ** torch.arange(few, device=DEVICE, dtype=torch.float32))
    if case["banned"]:
        ban = torch.rand((1, vocab), device=DEVICE, generator=g) < case["banned"]
        ban[0, 0] = False
        x.masked_fill_(ban, float("-inf"))
    tokens = torch.where(torch.rand(rows, device=DEVICE, generator=g) < 0.7, at[:, 0], torch.randint(vocab, (rows,), device=DEVICE, generator=g))
    return dict(case=case, logits=x.to(dtype), tokens=tokens.int())


# ---- one pass -----------------------------------------------------------------------------------------------------------
def run(st):
    case = st["case"]
    if case["kind"] == "pages":
        return _run_step(st) if case["op"] == "step" else _run_compact(st)
    return {"attend": _run_attend, "append": _run_append, "score": _run_score}[case["kind"]](st)


def _run_attend(st):
    if own:
        return st["cache"].attend(0, st["q"])
    k, v, q, lens = st["k"][0], st["v"][0], st["q"], st["lens"]
    n, t, h, d = q.shape
    page, hkv = k.shape[1], k.shape[2]
    m = _pages(st["longest"], page)
    ids = st["table"][:, :m].clamp(min=0).long()
    keys = k[ids].view(n, m * page, hkv, d).float()
    values = v[ids].view(n, m * page, hkv, d).float()
    s = torch.einsum("ntgrd,nkgd->ngtrk", q.float().view(n, t, hkv, h // hkv, d), keys) / math.sqrt(d)
    seen = lens.view(n, 1) - t + 1 + torch.arange(t, device=q.device)
    hidden = torch.arange(m * page, device=q.device).view(1, 1, 1, 1, -1) >= seen.view(n, 1, t, 1, 1)
    s = s.masked_fill(hidden, float("-inf"))
    top = s.amax(-1, keepdim=True).clamp(min=-3e38)
    p = torch.exp(s - top)
    p = p / p.sum(-1, keepdim=True).clamp(min=1e-30)
    return torch.einsum("ngtrk,nkgd->ntgrd", p, values).reshape(n, t, h, d).to(q.dtype)


def _rotate(x, c, s):
    half = x.shape[-1] // 2
    a, b = x[..., :half].float(), x[..., half:].float()
    return torch.cat([a * c - b * s, b * c + a * s], -1).to(x.dtype)


def _run_append(st):
    if own:
        q = st["cache"].append(0, st["q"], st["k_new"], st["v_new"], st["slots"], st["positions"], st["cos"], st["sin"])
        return {"q": q, "k": st["k"], "v": st["v"]}
    at = st["positions"].long()
    c, s = st["cos"][at][:, None], st["sin"][at][:, None]
    keep = (st["slots"] >= 0).nonzero()[:, 0]
    slots = st["slots"][keep].long()
    hkv, d = st["k"].shape[-2:]
    st["k"].view(-1, hkv, d)[slots] = _rotate(st["k_new"], c, s)[keep]
    st["v"].view(-1, hkv, d)[slots] = st["v_new"][keep]
    return {"q": _rotate(st["q"], c, s), "k": st["k"], "v": st["v"]}


def _tables(st):
    n, w = st["n"], st["width"]
    s = st["start"]
    return s[: n * w].view(n, w).clone(), s[n * w: n * w + n].clone(), s[n * w + n:].clone()


def _run_step(st):
    page = st["case"]["page"]
    if own:
        c = st["cache"]
        c.state.copy_(st["start"])
        c.fork(st["parents"], st["beams"])
        slots, positions = c.extend(st["beams"], st["new"], st["case"]["new"])
        return {"table": c.table, "lens": c.lens, "refs": c.refs, "slots": slots, "positions": positions, "k": st["k"], "v": st["v"]}
    _, lens, refs = _tables(st)
    n, w, new, most = st["n"], st["width"], st["new"].long(), st["case"]["new"]
    parents = st["parents"].long()
    dev = lens.device
    # fork
    table = st["start"][: n * w].view(n, w)[parents]
    lens = lens.long()[parents]
    live = table >= 0
    refs = torch.zeros_like(refs).index_add_(0, table.clamp(min=0).long().view(-1), live.int().view(-1))
    # extend: who needs a page of its own for the unfinished last page
    rows = lens % page
    order = torch.arange(n, device=dev)
    last = table.gather(1, ((lens - 1).clamp(min=0) // page)[:, None])[:, 0].long()
    partial = (rows > 0) & (new > 0)
    same = (last[:, None] == last[None, :]) & partial[:, None] & partial[None, :]
    before = (same & (order[None, :] < order[:, None])).sum(1)
    copy = partial & (refs[last.clamp(min=0)] - before > 1)
    more = (lens + new + page - 1) // page - (lens + page - 1) // page
    need = more + copy
    ends = need.cumsum(0)
    free = (refs == 0).nonzero()[:, 0]
    j = torch.arange(_pages(most, page) + 2, device=dev)
    place = (lens // page)[:, None] + j                            # the unfinished page's entry, or the first new one
    place = torch.where((partial & ~copy)[:, None], place + 1, place)
    mine = j[None, :] < need[:, None]
    ids = free[((ends - need)[:, None] + j).clamp(max=max(0, free.numel() - 1))]
    r, c = mine.nonzero(as_tuple=True)
    table = table.clone()
    table[r, place[r, c]] = ids[r, c].int()
    refs = refs.index_add(0, ids[r, c], torch.ones_like(r, dtype=torch.int32))
    who = copy.nonzero()[:, 0]
    refs = refs.index_add(0, last[who], -torch.ones_like(who, dtype=torch.int32))
    at = torch.arange(page, device=dev)
    w_, a_ = (copy[:, None] & (at[None, :] < rows[:, None])).nonzero(as_tuple=True)
    st["k"][:, ids[w_, 0], a_] = st["k"][:, last[w_], a_]
    st["v"][:, ids[w_, 0], a_] = st["v"][:, last[w_], a_]
    i = torch.arange(most, device=dev)
    positions = lens[:, None] + i
    slots = table.gather(1, positions // page).long() * page + positions % page
    positions, slots = (torch.where(i < new[:, None], x, -1).int() for x in (positions, slots))
    return {"table": table, "lens": (lens + new).int(), "refs": refs, "slots": slots, "positions": positions, "k": st["k"], "v": st["v"]}


def _run_compact(st):
    if own:
        c = st["cache"]
        c.state.copy_(st["start"])
        c.truncate(st["ended"], st["keep"])
        live = c.compact()
        return {"table": c.table, "lens": c.lens, "refs": c.refs, "live": live, "k": st["k"], "v": st["v"]}
    table, lens, refs = _tables(st)
    page, w, pool = st["case"]["page"], st["width"], refs.numel()
    ended, keep = st["ended"].long(), st["keep"]
    # truncate
    lens[ended] = torch.minimum(lens[ended], keep)
    gone = (torch.arange(w, device=lens.device)[None, :] >= ((lens + page - 1) // page)[:, None]) & (table >= 0)
    refs.index_add_(0, table.clamp(min=0).long().view(-1), -gone.int().view(-1))
    table = torch.where(gone, -1, table)
    # compact
    used = refs > 0
    live = used.sum()
    ids = torch.arange(pool, device=lens.device)
    src, dst = (used & (ids >= live)).nonzero()[:, 0], (~used & (ids < live)).nonzero()[:, 0]
    st["k"][:, dst] = st["k"][:, src]
    st["v"][:, dst] = st["v"][:, src]
    to = ids.clone()
    to[src] = dst
    refs[dst] = refs[src]
    refs[src] = 0
    table = torch.where(table >= 0, to[table.clamp(min=0).long()].int(), table)
    return {"table": table, "lens": lens, "refs": refs, "live": live.int().view(1), "k": st["k"], "v": st["v"]}


def _run_score(st):
    top = st["case"]["top"]
    if own:
        from paper_2402_13720_b200.scores import token_logprobs
        s = token_logprobs(st["logits"], st["tokens"], top)
        out = {"logprob": s.logprob, "entropy": s.entropy}
        return dict(out, top_ids=s.top_ids, top_logprobs=s.top_logprobs) if top else out
    x = st["logits"].float()
    m = x.amax(-1, keepdim=True)
    e = torch.exp(x - m)
    z = e.sum(-1, keepdim=True)
    lse = m + torch.log(z)
    logp = x - lse
    out = {"logprob": logp.gather(1, st["tokens"].long()[:, None])[:, 0],
           "entropy": -torch.where(e > 0, e * logp, 0.0).sum(-1) / z[:, 0]}
    if top:
        # by value, then by the lowest id: a 64-bit key that no two tokens share
        bits = (x + 0.0).view(torch.int32).long()
        key = (torch.where(bits < 0, (-1 << 31) - 1 - bits, bits) << 32) + (x.shape[1] - torch.arange(x.shape[1], device=x.device))
        ids = key.topk(top, dim=1).indices
        out.update(top_ids=ids.int(), top_logprobs=logp.gather(1, ids))
    return out


# ---- the definitions in 64 bits -----------------------------------------------------------------------------------------
def exact(case, seed):
    if case["kind"] == "pages":
        return None                                               # whole numbers and moved values: nothing is computed
    st = prepare(case, seed)
    return {"attend": _exact_attend, "append": _exact_append, "score": _exact_score}[case["kind"]](st)


def _exact_attend(st):
    q = st["q"].double()
    n, t, h, d = q.shape
    page, hkv = st["k"].shape[2:4]
    out = torch.zeros_like(q)
    table, lens = st["table"].cpu().numpy(), st["lens"].cpu().numpy()
    for s in range(n):
        slots = torch.tensor([int(table[s, j // page]) * page + j % page for j in range(int(lens[s]))], device=DEVICE)
        keys = st["k"][0].view(-1, hkv, d)[slots].double()
        values = st["v"][0].view(-1, hkv, d)[slots].double()
        for i in range(t):
            m = int(lens[s]) - t + 1 + i
            if m <= 0:
                continue
            for head in range(hkv):
                rows = slice(head * (h // hkv), (head + 1) * (h // hkv))
                p = torch.softmax(q[s, i, rows] @ keys[:m, head].T / d ** 0.5, dim=-1)
                out[s, i, rows] = p @ values[:m, head]
    return out


def _exact_append(st):
    d = st["q"].shape[-1]
    at = st["positions"].long()

    def turned(x):
        z = torch.complex(x[..., : d // 2].double(), x[..., d // 2:].double())
        z = z * torch.complex(st["cos"][at].double(), st["sin"][at].double())[:, None]
        return torch.cat([z.real, z.imag], -1)

    q, k_new = turned(st["q"]), turned(st["k_new"])
    k, v = st["k"].double(), st["v"].double()
    page = k.shape[2]
    for row, slot in enumerate(st["slots"].tolist()):
        if slot >= 0:
            k[0, slot // page, slot % page] = k_new[row]
            v[0, slot // page, slot % page] = st["v_new"][row].double()
    return {"q": q, "k": k, "v": v}


def _exact_score(st):
    top, rows = st["case"]["top"], st["logits"].shape[0]
    logprob, entropy, best = [], [], []
    for a in range(0, rows, 128):
        x = st["logits"][a: a + 128].double()
        lp = torch.log_softmax(x, dim=-1)
        logprob.append(lp[torch.arange(x.shape[0]), st["tokens"][a: a + 128].long()])
        entropy.append(torch.special.entr(lp.exp()).sum(-1))
        if top:
            best.append(lp.sort(dim=-1, descending=True).values[:, :top])
    out = {"logprob": torch.cat(logprob), "entropy": torch.cat(entropy)}
    return dict(out, top_ids=None, top_logprobs=torch.cat(best)) if top else out
