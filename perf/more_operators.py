"""Performance cases of what a text needs on its way into and out of a paged key-value cache, beside the step by step decoding that
``operators.py`` measures: prompts in large pieces, positions of models with long contexts, and the rules under which tokens are chosen.

  chunk      attention of a chunk of new tokens for each of several sequences over their pages; every sequence has its own number of them
  rotary     rotary positions (pairs interleaved or in halves, part of the head, scaled for long contexts) for new queries and keys, computed
             from frequencies, and keys and values to their pages
  constrain  penalties for repeated tokens, biases and grammar masks on rows of logits

Head layouts and vocabularies are those of this repository's configurations (``synth.config``).  Lengths, batch and page sizes are generic.
``run`` computes the plain form out of elementary torch operations in 32 bits; with ``own`` set it calls the framework.
"""
from __future__ import annotations

import math
import random

import numpy as np
import torch

own = False

# query heads, kv heads, head dim, vocabulary
SHAPES = {
    "tiny": (4, 4, 32, 512),
    "small": (4, 2, 128, 1024),
    "1b": (32, 4, 64, 32000),
    "7b": (32, 32, 128, 32000),
    "34b": (56, 8, 128, 64000),
    "70b": (64, 8, 128, 32000),
}
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
DEVICE = "cuda:0"
MOST_FLOPS = 0.9e12                                               # of a drawn chunk: the largest listed one's
SLOW_F32 = 16                                                     # f32 operations count as so many of these


def listed():
    return [
        # The smallest use: a short prompt of the fp32 model of the tests behind what is cached already.
        dict(name="chunk_tiny_f32", kind="chunk", shape="tiny", dtype="f32", seqs=1, new=23, cached=44, ragged=False, page=16, layout=1),
        # A batch of the 1.1B-shaped model in which some sequences decode one token and others bring a piece of a prompt.
        dict(name="chunk_1b_mixed", kind="chunk", shape="1b", dtype="bf16", seqs=14, new=150, cached=700, ragged=True, page=16, layout=2),
        # One whole prompt with the 7B shape, which has a kv head for every query head.
        dict(name="chunk_7b_prompt", kind="chunk", shape="7b", dtype="bf16", seqs=1, new=2048, cached=0, ragged=False, page=32, layout=3),
        # A short piece of a prompt behind a long context that is cached already, seven query heads to a kv head: the keys have to be split up.
        dict(name="chunk_34b_behind", kind="chunk", shape="34b", dtype="bf16", seqs=1, new=61, cached=24000, ragged=False, page=64, layout=4),
        # Prompts of the fp32 model with heads of 128, in the middle of the range.
        dict(name="chunk_small_f32", kind="chunk", shape="small", dtype="f32", seqs=5, new=411, cached=200, ragged=True, page=24, layout=5),
        # Long prompts of several users at once, the largest call.
        dict(name="chunk_70b_prompts", kind="chunk", shape="70b", dtype="bf16", seqs=5, new=4096, cached=1500, ragged=True, page=128, layout=6),
        # One new token of one text, where only latency counts; a quarter of the head is rotated, interleaved.
        dict(name="rotary_1b_token", kind="rotary", shape="1b", dtype="bf16", rows=1, padding=0, page=16, part=4, interleaved=True, scaling="none", factor=1.0,
             first=250, layout=7),
        # A batch of texts far out in a stretched context, fp32.
        dict(name="rotary_small_f32", kind="rotary", shape="small", dtype="f32", rows=333, padding=40, page=24, part=1, interleaved=True, scaling="linear",
             factor=8.0, first=90000, layout=8),
        # A prompt's rows enter the cache of a model stretched to sixteen times its context, among them the padding of shorter prompts.
        dict(name="rotary_70b_prompts", kind="rotary", shape="70b", dtype="bf16", rows=4100, padding=300, page=64, part=1, interleaved=False, scaling="yarn",
             factor=16.0, first=30000, layout=9),
        # One generated token of a chat, with the usual penalties for what it has said.
        dict(name="constrain_token", kind="constrain", rows=1, vocab=32000, dtype="f32", history=411, penalties=True, bias="none", mask="none", allowed=1.0,
             layout=10),
        # The beams of a search under a grammar, each in a state of its own: most tokens cannot come.
        dict(name="constrain_beams", kind="constrain", rows=24, vocab=64000, dtype="bf16", history=700, penalties=True, bias="none", mask="rows", allowed=0.1,
             layout=11),
        # A large batch with everything: penalties, one bias for all, a grammar for each; the largest call.
        dict(name="constrain_batch", kind="constrain", rows=1000, vocab=64000, dtype="f32", history=2500, penalties=True, bias="shared", mask="rows", allowed=0.8,
             layout=12),
    ]


def _between(rng, lo, hi):
    """Whole number spread over the logarithm of [lo, hi]."""
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["chunk", "chunk", "chunk", "rotary", "constrain", "constrain"])
    layout = rng.randrange(1 << 30)
    page = rng.choice([8, 16, 16, 24, 32, 64, 128])
    if kind == "chunk":
        shape = rng.choice(["tiny", "small", "1b", "7b", "34b", "70b"])
        dtype = "f32" if shape == "tiny" or rng.random() < 0.15 else "bf16"
        new = _between(rng, 1, 6000)
        cached = 0 if rng.random() < 0.3 else _between(rng, 1, 24000)
        seqs = _between(rng, 1, 24)
        case = dict(kind="chunk", shape=shape, dtype=dtype, seqs=seqs, new=new, cached=cached, ragged=rng.random() < 0.75, page=page, layout=layout)
        while work(case)["flops"] * (SLOW_F32 if dtype == "f32" else 1) > MOST_FLOPS or case["seqs"] * (case["cached"] + case["new"]) > 100000:
            for key, low in (("seqs", 1), ("cached", 0), ("new", 1)):
                case[key] = max(low, case[key] * 3 // 4)
        return case
    if kind == "rotary":
        rows = _between(rng, 1, 4100)
        return dict(kind="rotary", shape=rng.choice(["tiny", "small", "1b", "7b", "34b", "70b"]), dtype=rng.choice(["bf16", "bf16", "f32"]) if rows < 2000 else "bf16",
                    rows=rows, padding=rng.randrange(rows // 4 + 1), page=page, part=rng.choice([1, 1, 2]), interleaved=rng.random() < 0.5,
                    scaling=rng.choice(["none", "linear", "ntk", "yarn"]), factor=rng.choice([1.5, 4.0, 16.0]), first=_between(rng, 1, 1000000), layout=layout)
    vocab = rng.choice([512, 1024, 32000, 32000, 64000, _between(rng, 500, 130000)])
    rows = _between(rng, 1, max(2, min(1000, 1000 * 64000 // vocab)))
    bias, mask = rng.choice(["none", "shared", "rows"]), rng.choice(["none", "shared", "rows", "rows"])
    return dict(kind="constrain", rows=rows, vocab=vocab, dtype=rng.choice(["f32", "f32", "bf16"]), history=_between(rng, 1, 4000),
                penalties=bias == mask == "none" or rng.random() < 0.8, bias=bias, mask=mask, allowed=rng.choice([0.001, 0.1, 0.8, 1.0]),
                layout=layout)


# ---- what a case fixes beside its sizes ---------------------------------------------------------------------------------
def _chunks(case):
    """(tokens cached before, new tokens) of every sequence of a case: equal, or ragged with one of the largest and one single token."""
    if not case["ragged"]:
        return [(case["cached"], case["new"])] * case["seqs"]
    r = random.Random(case["layout"])
    c = [(r.randint(0, case["cached"]), r.randint(1, case["new"])) for _ in range(case["seqs"])]
    i = r.randrange(len(c))
    c[i] = (case["cached"], case["new"])
    if len(c) > 2:
        c[i - 1] = (c[i - 1][0], 1)
    return c


def _lens(case):
    """Tokens of the history of every row."""
    r = random.Random(case["layout"])
    lens = [r.randint(0, case["history"]) for _ in range(case["rows"])]
    lens[r.randrange(len(lens))] = case["history"]
    return lens


def _pages(n, page):
    return -(-n // page)


def work(case):
    e = 4 if case["dtype"] == "f32" else 2
    if case["kind"] == "constrain":
        rows, words = case["rows"], _pages(case["vocab"], 32)
        n = rows * case["vocab"]
        nbytes = 2 * n * e + {"none": 0, "shared": 1, "rows": rows}[case["bias"]] * case["vocab"] * 4 + {"none": 0, "shared": 1, "rows": rows}[case["mask"]] * words * 4
        if case["penalties"]:
            nbytes += 4 * sum(_lens(case)) + 16 * rows
        return {"bytes": nbytes, "flops": 2 * n}
    h, hkv, d, _ = SHAPES[case["shape"]]
    if case["kind"] == "chunk":
        c = _chunks(case)
        new = sum(m for _, m in c)
        return {"bytes": sum(a + m for a, m in c) * hkv * d * 2 * e + 2 * new * h * d * e + 4 * sum(_pages(a + m, case["page"]) + 2 for a, m in c),
                "flops": 4 * d * h * sum(a * m + m * (m + 1) // 2 for a, m in c)}
    live = case["rows"] - case["padding"]
    rd = d // case["part"]
    return {"bytes": 2 * case["rows"] * h * d * e + live * 4 * hkv * d * e + case["rows"] * 8 + 4 * rd, "flops": 3 * rd * (case["rows"] * h + live * hkv)}


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


def _cache(st, max_seqs, max_pages):
    """The framework's handle of the pools and tables of a state."""
    from paper_2402_13720_b200.paged import PagedCache
    return PagedCache(k=st["k"], v=st["v"], max_seqs=max_seqs, max_pages=max_pages)


def prepare(case, seed):
    return {"chunk": _prepare_chunk, "rotary": _prepare_rotary, "constrain": _prepare_constrain}[case["kind"]](case, _generator(seed), random.Random(seed))


def _prepare_chunk(case, g, r):
    h, hkv, d, _ = SHAPES[case["shape"]]
    dtype, page = DTYPES[case["dtype"]], case["page"]
    chunks = _chunks(case)
    lens = [a + m for a, m in chunks]
    starts = np.concatenate([[0], np.cumsum([m for _, m in chunks])])
    used = sum(_pages(x, page) for x in lens)
    n_pages = used + used // 8 + 3
    width = max(_pages(x, page) for x in lens) + 1
    ids = r.sample(range(n_pages), used)
    table = np.full((len(lens), width), -1, dtype=np.int32)
    at = 0
    for i, x in enumerate(lens):
        m = _pages(x, page)
        table[i, :m] = ids[at: at + m]
        at += m
    # queries twice as wide as keys: attention that favours some keys, as trained models' does
    st = dict(case=case, k=_randn((1, n_pages, page, hkv, d), dtype, g), v=_randn((1, n_pages, page, hkv, d), dtype, g),
              q=_randn((int(starts[-1]), h, d), dtype, g, 2.0), table=_i32(table), lens=_i32(lens), starts=_i32(starts), chunks=chunks)
    if own:
        st["cache"] = _cache(st, len(lens), width)
        st["cache"].table.copy_(st["table"])
        st["cache"].lens.copy_(st["lens"])
    return st


def _prepare_rotary(case, g, r):
    # new rows of a few sequences, each at its own place in the pool; padding has no slot
    h, hkv, d, _ = SHAPES[case["shape"]]
    dtype, page = DTYPES[case["dtype"]], case["page"]
    rows, live = case["rows"], case["rows"] - case["padding"]
    n_pages = 2 * _pages(rows, page) + 8
    ids = r.sample(range(n_pages), _pages(rows, page) + 1)
    slots = [ids[i // page] * page + i % page for i in range(live)] + [-1] * case["padding"]
    first = case["first"] + r.randrange(500)
    st = dict(case=case, k=_randn((1, n_pages, page, hkv, d), dtype, g), v=_randn((1, n_pages, page, hkv, d), dtype, g),
              q=_randn((rows, h, d), dtype, g), k_new=_randn((rows, hkv, d), dtype, g), v_new=_randn((rows, hkv, d), dtype, g),
              slots=_i32(slots), positions=_i32([first + i for i in range(live)] + [0] * case["padding"]))
    st["inv"], st["magnitude"] = _frequencies(case)
    if own:
        from paper_2402_13720_b200.rotary import Rotary
        st["cache"] = _cache(st, 1, 1)
        st["rotary"] = Rotary(d, rotary_dim=d // case["part"], interleaved=case["interleaved"], scaling=case["scaling"], factor=case["factor"],
                              original=4096, device=DEVICE)
    return st


def _frequencies(case):
    """Radians a position for every pair, in 64 bits, and what rotated vectors are multiplied with."""
    rd, theta, f = SHAPES[case["shape"]][2] // case["part"], 10000.0, case["factor"]
    if case["scaling"] == "ntk":
        theta *= f ** (rd / (rd - 2))
    pair = torch.arange(rd // 2, dtype=torch.float64, device=DEVICE)
    inv = theta ** (-2.0 * pair / rd)
    if case["scaling"] == "linear":
        return inv / f, 1.0
    if case["scaling"] == "yarn":
        # pairs that turn more than 32 times within the 4096 tokens of training stay, those of less than one turn are stretched
        def at(turns):
            return rd * math.log(4096 / (turns * 2 * math.pi)) / (2 * math.log(theta))
        lo, hi = max(math.floor(at(32.0)), 0), min(math.ceil(at(1.0)), rd - 1)
        ramp = ((pair - lo) / max(hi - lo, 0.001)).clamp(0, 1)
        return inv / f * ramp + inv * (1 - ramp), 0.1 * math.log(f) + 1.0
    return inv, 1.0


def _prepare_constrain(case, g, r):
    rows, vocab = case["rows"], case["vocab"]
    x = _randn((rows, vocab), torch.float32, g, 2.0)
    # a few tokens stand out, less and less, as in a trained model's output
    few = 40
    at = torch.arange(few, device=DEVICE) * (vocab // few) + torch.randint(vocab // few, (rows, few), device=DEVICE, generator=g)
    at = (at + torch.randint(vocab, (rows, 1), device=DEVICE, generator=g)) % vocab
    x.scatter_(1, at, x.gather(1, at) + 12.0 * 0.85 ** torch.arange(few, device=DEVICE, dtype=torch.float32))
    st = dict(case=case, logits=x.to(DTYPES[case["dtype"]]), tokens=None, lens=None, repetition=None, presence=None, frequency=None, bias=None, allowed=None)
    if case["penalties"]:
        # some tokens come again and again; behind a row's history lies whatever was there
        u = torch.rand((rows, case["history"]), device=DEVICE, generator=g)
        tokens = (vocab * u ** 4).int().clamp(max=vocab - 1)
        lens = _i32(_lens(case))
        st.update(tokens=torch.where(torch.arange(case["history"], device=DEVICE) < lens[:, None], tokens, -1), lens=lens,
                  repetition=1.0 + 0.3 * torch.rand(rows, device=DEVICE, generator=g), presence=0.6 * torch.rand(rows, device=DEVICE, generator=g),
                  frequency=0.5 * torch.rand(rows, device=DEVICE, generator=g))
    if case["bias"] != "none":
        b = _randn((rows if case["bias"] == "rows" else 1, vocab), torch.float32, g)
        st["bias"] = b if case["bias"] == "rows" else b[0]
    if case["mask"] != "none":
        n = rows if case["mask"] == "rows" else 1
        bits = torch.rand((n, _pages(vocab, 32), 32), device=DEVICE, generator=g) < case["allowed"]
        words = (bits.long() << torch.arange(32, device=DEVICE)).sum(-1)
        words = torch.where(words >= 1 << 31, words - (1 << 32), words).int()
        st["allowed"] = words if case["mask"] == "rows" else words[0]
    return st


# ---- one pass -----------------------------------------------------------------------------------------------------------
def run(st):
    return {"chunk": _run_chunk, "rotary": _run_rotary, "constrain": _run_constrain}[st["case"]["kind"]](st)


def _run_chunk(st):
    if own:
        return st["cache"].attend_chunk(0, st["q"], st["starts"])
    k, v, q = st["k"][0], st["v"][0], st["q"]
    _, h, d = q.shape
    page, hkv = k.shape[1], k.shape[2]
    out = torch.empty_like(q)
    at = 0
    for i, (cached, new) in enumerate(st["chunks"]):
        n = cached + new
        ids = st["table"][i, : _pages(n, page)].long()
        keys = k[ids].view(-1, hkv, d)[:n].float().permute(1, 2, 0)
        values = v[ids].view(-1, hkv, d)[:n].float().transpose(0, 1)
        x = q[at: at + new].float().view(new, hkv, h // hkv, d).transpose(0, 1).reshape(hkv, -1, d)
        s = (x @ keys).view(hkv, new, h // hkv, n) * d ** -0.5
        hidden = torch.arange(n, device=q.device) > cached + torch.arange(new, device=q.device)[:, None]
        s = s.masked_fill(hidden[:, None], float("-inf"))
        p = torch.exp(s - s.amax(-1, keepdim=True))
        p = (p / p.sum(-1, keepdim=True)).view(hkv, -1, n)
        out[at: at + new] = (p @ values).view(hkv, new, h // hkv, d).transpose(0, 1).reshape(new, h, d).to(q.dtype)
        at += new
    return out


def _turned(x, c, s, rd, interleaved):
    y = x.float()
    pairs = y[..., :rd].unflatten(-1, (rd // 2, 2) if interleaved else (2, rd // 2))
    a, b = pairs.unbind(-1 if interleaved else -2)
    pairs = torch.stack([a * c - b * s, b * c + a * s], -1 if interleaved else -2)
    return torch.cat([pairs.flatten(-2), y[..., rd:]], -1).to(x.dtype)


def _run_rotary(st):
    if own:
        q = st["cache"].append_rotary(0, st["q"], st["k_new"], st["v_new"], st["slots"], st["positions"], st["rotary"])
        return {"q": q, "k": st["k"], "v": st["v"]}
    case = st["case"]
    angle = st["positions"].double()[:, None] * st["inv"]
    c, s = ((f(angle) * st["magnitude"]).float()[:, None] for f in (torch.cos, torch.sin))
    hkv, d = st["k"].shape[-2:]
    rd = d // case["part"]
    keep = (st["slots"] >= 0).nonzero()[:, 0]
    slots = st["slots"][keep].long()
    st["k"].view(-1, hkv, d)[slots] = _turned(st["k_new"], c, s, rd, case["interleaved"])[keep]
    st["v"].view(-1, hkv, d)[slots] = st["v_new"][keep]
    return {"q": _turned(st["q"], c, s, rd, case["interleaved"]), "k": st["k"], "v": st["v"]}


def _run_constrain(st):
    if own:
        from paper_2402_13720_b200.scores import constrain_logits
        return constrain_logits(st["logits"], tokens=st["tokens"], lens=st["lens"], repetition=st["repetition"], presence=st["presence"],
                                frequency=st["frequency"], bias=st["bias"], allowed=st["allowed"])
    x = st["logits"].float()
    rows, vocab = x.shape
    if st["tokens"] is not None:
        told = (torch.arange(st["tokens"].shape[1], device=x.device) < st["lens"][:, None]).float()
        count = torch.zeros_like(x).scatter_add_(1, st["tokens"].clamp(min=0).long(), told)
        rep = st["repetition"][:, None]
        seen = count > 0
        x = torch.where(seen, torch.where(x > 0, x / rep, x * rep), x)
        x = x - (st["frequency"][:, None] * count + torch.where(seen, st["presence"][:, None], 0.0))
    if st["bias"] is not None:
        x = x + st["bias"]
    if st["allowed"] is not None:
        bits = (st["allowed"][..., None] >> torch.arange(32, device=x.device, dtype=torch.int32)) & 1
        x = x.masked_fill(bits.flatten(-2)[..., :vocab] == 0, float("-inf"))
    return x.to(st["logits"].dtype)


# ---- the definitions in 64 bits -----------------------------------------------------------------------------------------
def exact(case, seed):
    st = prepare(case, seed)
    return {"chunk": _exact_chunk, "rotary": _exact_rotary, "constrain": _exact_constrain}[case["kind"]](st)


def _exact_chunk(st):
    q = st["q"].double()
    _, h, d = q.shape
    page, hkv = st["k"].shape[2:4]
    group = h // hkv
    out = torch.zeros_like(q)
    table, lens, starts = (st[x].cpu().numpy() for x in ("table", "lens", "starts"))
    for s, n in enumerate(lens):
        j = np.arange(n)
        slots = torch.tensor(table[s, j // page].astype(np.int64) * page + j % page, device=DEVICE)
        first = int(starts[s + 1]) - int(n)                       # the row that position 0 would have
        for head in range(hkv):
            keys = st["k"][0].view(-1, hkv, d)[slots, head].double()
            values = st["v"][0].view(-1, hkv, d)[slots, head].double()
            for a in range(int(starts[s]), int(starts[s + 1]), 512):
                b = min(a + 512, int(starts[s + 1]))
                m = b - first                                     # keys that the last of these rows sees
                scores = torch.einsum("tgd,kd->gtk", q[a:b, head * group: (head + 1) * group], keys[:m]) / math.sqrt(d)
                scores += torch.full((b - a, m), float("-inf"), dtype=torch.float64, device=DEVICE).triu(a - first + 1)
                out[a:b, head * group: (head + 1) * group] = torch.einsum("gtk,kd->tgd", torch.softmax(scores, -1), values[:m])
    return out


def _exact_rotary(st):
    case = st["case"]
    d = st["q"].shape[-1]
    rd = d // case["part"]
    angle = torch.outer(st["positions"].double(), st["inv"])
    turn = torch.polar(torch.full_like(angle, st["magnitude"]), angle)[:, None]

    def turned(x):
        y = x.double().clone()
        re, im = (slice(0, rd, 2), slice(1, rd, 2)) if case["interleaved"] else (slice(0, rd // 2), slice(rd // 2, rd))
        z = torch.complex(y[..., re].clone(), y[..., im].clone()) * turn
        y[..., re], y[..., im] = z.real, z.imag
        return y

    q, k_new = turned(st["q"]), turned(st["k_new"])
    k, v = st["k"].double(), st["v"].double()
    page = k.shape[2]
    slots = st["slots"].cpu().numpy()
    rows = np.nonzero(slots >= 0)[0]
    at = [torch.tensor(x, device=DEVICE) for x in (rows, slots[rows] // page, slots[rows] % page)]
    k[0, at[1], at[2]] = k_new[at[0]]
    v[0, at[1], at[2]] = st["v_new"][at[0]].double()
    return {"q": q, "k": k, "v": v}


def _exact_constrain(st):
    out = torch.empty_like(st["logits"], dtype=torch.float64)
    vocab = out.shape[1]
    for row in range(out.shape[0]):
        x = st["logits"][row].double()
        if st["tokens"] is not None:
            ids, count = st["tokens"][row, : int(st["lens"][row])].long().unique(return_counts=True)
            y, rep = x[ids], st["repetition"][row].double()
            y = torch.where(y > 0, y / rep, y * rep)
            x[ids] = y - count * st["frequency"][row].double() - st["presence"][row].double()
        if st["bias"] is not None:
            x = x + (st["bias"] if st["bias"].dim() == 1 else st["bias"][row]).double()
        if st["allowed"] is not None:
            words = st["allowed"] if st["allowed"].dim() == 1 else st["allowed"][row]
            bits = np.unpackbits(words.cpu().numpy().view(np.uint8), bitorder="little")[:vocab]
            x = x.masked_fill(torch.tensor(bits == 0, device=DEVICE), float("-inf"))
        out[row] = x
    return out
