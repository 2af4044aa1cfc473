"""The paged cache, its attention and the token scores against plain implementations: pages against a sequential simulation of the header's
words, everything computed against 64 bits.

Tolerances, from the arithmetic (fixed before the first run):
 * bf16 attention: the output is rounded once, to 8 bits of significand: 2^-8 relative.  Scores are exact products added up in 32 bits and
   probabilities go in as two bf16 parts (2^-17): below 2^-13 of the largest |value|.
 * f32 attention: a score of 128 products, each |q k| scale adding up to about 25, in a chain of 34 roundings: 34 x 2^-24 x 25 = 5e-5 relative in
   a probability, twice that in the quotient: 1e-4 of the largest |value|.
 * log probabilities and entropy: a thread adds up at most 300 terms, 300 x 2^-24 = 2e-5 relative in Z and T, where T is at most
   12 Z here; the difference x - m and the logarithm are rounded to 2^-24 of themselves: 3e-5 and 12 x 2e-5 + 2e-5 = 3e-4, + 2^-22 relative.
 * rotation: the products and their sum in 32 bits, then one rounding: 2^-8 relative + 2^-22 of the pair (bf16), 2^-22 of the pair (f32).
"""
import math
import ctypes as C

import numpy as np
import pytest
import torch

from paper_2402_13720_b200 import binding, build, paged, scores

gpu = pytest.mark.gpu
DEV = "cuda:0"


def i32(x):
    return torch.tensor(np.asarray(x, dtype=np.int32), device=DEV)


# ---------------------------------------------------------------------------------------------- pages
class Sim:
    """The header's words, one sequence and one page after the other."""

    def __init__(self, n_pages, page, max_seqs, max_pages):
        self.page, self.max_pages, self.max_seqs = page, max_pages, max_seqs
        self.rows = [[] for _ in range(max_seqs)]
        self.lens = [0] * max_seqs
        self.refs = [0] * n_pages
        self.copies = []

    def _drop(self, rows):
        for p in rows:
            self.refs[p] -= 1

    def fork(self, src, dst, keep=None):
        if any(not 0 <= s < self.max_seqs for s in list(src) + list(dst)) or len(set(dst)) < len(dst) or (keep is not None and min(keep) < 0):
            return binding.OURO_EINVAL
        new = []
        for i, s in enumerate(src):
            n = self.lens[s] if keep is None else min(self.lens[s], keep[i])
            new.append((list(self.rows[s][: -(-n // self.page)]), n))
        for (row, _) in new:
            for p in row:
                self.refs[p] += 1
        for (row, n), d in zip(new, dst):
            self._drop(self.rows[d])
            self.rows[d], self.lens[d] = row, n
        return 0

    def truncate(self, seqs, keep):
        return self.fork(seqs, seqs, keep)

    def extend(self, seqs, new, width):
        if len(set(seqs)) < len(seqs) or any(not 0 <= s < self.max_seqs for s in seqs) or any(not 0 <= a <= width for a in new):
            return binding.OURO_EINVAL, None, None
        if any(self.lens[s] + a > self.max_pages * self.page for s, a in zip(seqs, new)):
            return binding.OURO_ECAPACITY, None, None
        free = [p for p, r in enumerate(self.refs) if r == 0]
        refs, rows, copies, lens = list(self.refs), [list(r) for r in self.rows], [], list(self.lens)
        slots, pos = np.full((len(seqs), width), -1), np.full((len(seqs), width), -1)
        for i, (s, a) in enumerate(zip(seqs, new)):
            if a and lens[s] % self.page and refs[rows[s][-1]] > 1:
                if not free:
                    return binding.OURO_ECAPACITY, None, None
                p = free.pop(0)
                copies.append((rows[s][-1], p, lens[s] % self.page))
                refs[rows[s][-1]] -= 1
                refs[p] = 1
                rows[s][-1] = p
            for j in range(a):
                if lens[s] % self.page == 0:
                    if not free:
                        return binding.OURO_ECAPACITY, None, None
                    rows[s].append(free.pop(0))
                    refs[rows[s][-1]] = 1
                slots[i, j], pos[i, j] = rows[s][-1] * self.page + lens[s] % self.page, lens[s]
                lens[s] += 1
        self.refs, self.rows, self.lens = refs, rows, lens
        self.copies = copies
        return 0, slots, pos

    def compact(self):
        live = [p for p, r in enumerate(self.refs) if r > 0]
        n = len(live)
        holes = [p for p in range(n) if self.refs[p] == 0]
        to = dict(zip([p for p in live if p >= n], holes))
        self.copies = [(a, b, self.page) for a, b in to.items()]
        for a, b in to.items():
            self.refs[b], self.refs[a] = self.refs[a], 0
        self.rows = [[to.get(p, p) for p in row] for row in self.rows]
        return n

    def table(self):
        t = np.full((self.max_seqs, self.max_pages), -1)
        for s, row in enumerate(self.rows):
            t[s, : len(row)] = row
        return t


def layouts(kind, L, n_pages, page, H, D, dtype):
    """Pools whose elements lie in different orders, filled with values that tell them apart."""
    if kind == "rows":
        k, v = (torch.zeros((L, n_pages, page, H, D), dtype=dtype, device=DEV) for _ in range(2))
    elif kind == "heads":                                 # heads outside of rows
        k, v = (torch.zeros((L, n_pages, H, page, D), dtype=dtype, device=DEV).transpose(2, 3) for _ in range(2))
    elif kind == "padded":                                # rows 16 bytes further apart than they are long
        k, v = (torch.zeros((L, n_pages, page, H, D + 16), dtype=dtype, device=DEV)[..., :D] for _ in range(2))
    else:                                                 # pages hold all layers, keys beside values
        both = torch.zeros((n_pages, L, 2, page, H, D), dtype=dtype, device=DEV).transpose(0, 1)
        k, v = both[:, :, 0], both[:, :, 1]
    g = torch.Generator(device=DEV).manual_seed(5)
    for t in (k, v):
        t.copy_(torch.randn(t.shape, device=DEV, generator=g).to(dtype))
    return k, v


def same(cache, sim, k, v, want_k, want_v):
    assert np.array_equal(cache.table.cpu().numpy(), sim.table())
    assert cache.lens.tolist() == sim.lens and cache.refs.tolist() == sim.refs
    assert torch.equal(k, want_k) and torch.equal(v, want_v)


def copy_in(sim, *pools):
    for t in pools:
        was = t.clone()
        for a, b, rows in sim.copies:
            t[:, b, :rows] = was[:, a, :rows]
    sim.copies = []


@gpu
@pytest.mark.parametrize("layout,page,H,D,dtype,n_pages,max_seqs,max_pages", [
    ("rows", 16, 2, 64, torch.bfloat16, 70, 9, 12),
    ("heads", 5, 3, 32, torch.float32, 101, 13, 17),
    ("both", 1, 1, 96, torch.bfloat16, 333, 7, 60),
    ("padded", 24, 2, 128, torch.bfloat16, 40, 40, 6),
])
def test_pages_follow_a_sequential_simulation(layout, page, H, D, dtype, n_pages, max_seqs, max_pages):
    build.build()
    k, v = layouts(layout, 3, n_pages, page, H, D, dtype)
    wk, wv = k.clone(), v.clone()
    cache = paged.PagedCache(max_seqs=max_seqs, max_pages=max_pages, k=k, v=v)
    sim = Sim(n_pages, page, max_seqs, max_pages)
    rng = np.random.default_rng(n_pages)
    refused = copies = moved = 0
    for step in range(120):
        n = int(rng.integers(1, max_seqs + 1))
        seqs = rng.permutation(max_seqs)[:n].tolist()
        op = rng.choice(["fork", "extend", "extend", "extend", "truncate", "compact"])
        rc = 0
        if op == "fork":
            src = rng.integers(0, max_seqs, n).tolist()
            if step % 11 == 0 and n > 1:
                seqs[1] = seqs[0]                          # refused
            rc = sim.fork(src, seqs)
            cache.fork(i32(src), i32(seqs))
        elif op == "truncate":
            keep = [int(rng.integers(0, page * max_pages)) if rng.random() < 0.7 else 0 for _ in seqs]
            rc = sim.truncate(seqs, keep)
            cache.truncate(i32(seqs), i32(keep))
        elif op == "extend":
            width = int(rng.choice([1, 2, page + 3, 3 * page]))
            new = rng.integers(0, width + 1, n).tolist()
            rc, slots, pos = sim.extend(seqs, new, width)
            got_slots, got_pos = cache.extend(i32(seqs), i32(new), width)
            if rc:
                assert bool((got_slots == -1).all()) and bool((got_pos == -1).all())
            else:
                assert np.array_equal(got_slots.cpu().numpy(), slots) and np.array_equal(got_pos.cpu().numpy(), pos)
                copies += len(sim.copies)
        else:
            n_live = sim.compact()
            moved += len(sim.copies)
            assert int(cache.compact()) == n_live
        copy_in(sim, wk, wv)
        same(cache, sim, k, v, wk, wv)
        if rc:
            refused += 1
            with pytest.raises(binding.OuroError) as e:
                cache.check()
            assert e.value.status == rc
        cache.check()
    assert refused and moved and (copies or page == 1)     # the walk met what it is for


@gpu
def test_many_long_rows_and_the_last_sharer():
    """The cluster's fork (more entries than one CTA takes), pages beyond one round of the scan, and that the last to ask keeps a shared page."""
    build.build()
    n_pages, page, seqs, width = 40000, 2, 64, 701
    cache = paged.PagedCache(1, n_pages, page, 1, 32, "bf16", max_seqs=seqs, max_pages=width)
    sim = Sim(n_pages, page, seqs, width)
    every = list(range(seqs))
    for src, new in ((None, [1399 - 13 * i for i in every]), ([0] * 32 + [63] * 32, [1] * 64), ([(7 * i) % 64 for i in every], [0, 1] * 32)):
        if src is not None:
            sim.fork(src, every)
            cache.fork(i32(src), i32(every))
        w = max(new)
        _, slots, pos = sim.extend(every, new, w)
        got = cache.extend(i32(every), i32(new), w)
        assert np.array_equal(got[0].cpu().numpy(), slots) and np.array_equal(got[1].cpu().numpy(), pos)
        assert np.array_equal(cache.table.cpu().numpy(), sim.table()) and cache.refs.tolist() == sim.refs
    order = every[::-1]                                    # the order of the list, not of the sequences, decides
    sim.fork([5] * 64, every)
    cache.fork(i32([5] * 64), i32(every))
    sim.extend(order, [1] * 64, 1)
    cache.extend(i32(order), i32([1] * 64), 1)
    assert np.array_equal(cache.table.cpu().numpy(), sim.table()) and cache.refs.tolist() == sim.refs
    cut = [3 * i for i in every]
    sim.truncate(every, cut)
    cache.truncate(i32(every), i32(cut))
    assert int(cache.compact()) == sim.compact()
    assert np.array_equal(cache.table.cpu().numpy(), sim.table()) and cache.refs.tolist() == sim.refs and cache.lens.tolist() == sim.lens
    cache.check()


@gpu
def test_extending_by_more_than_31_bits_of_pages_is_refused():
    """Two sequences that together ask for 2^31 pages of one token."""
    build.build()
    cache = paged.PagedCache(1, 8, 1, 1, 32, "bf16", max_seqs=2, max_pages=2 ** 30)
    seqs, new = i32([0, 1]), i32([2 ** 30, 2 ** 30])
    binding._check(cache._L.ouro_paged_extend(cache._p, seqs.data_ptr(), new.data_ptr(), 2, 2 ** 30, None, None, cache._stream()))
    with pytest.raises(binding.OuroError) as e:
        cache.check()
    assert e.value.status == binding.OURO_ECAPACITY and cache.lens.tolist() == [0, 0] and not bool(cache.refs.any())
    slots, _ = cache.extend(seqs, i32([3, 4]), 4)          # and the pages are there for who asks for less
    assert slots.tolist() == [[0, 1, 2, -1], [3, 4, 5, 6]]
    cache.check()


@gpu
def test_pages_of_half_a_thousand_million_tokens():
    """A sequence's tokens and a page's together are more than 31 bits hold: the pages of a sequence are counted all the same."""
    build.build()
    page = 500_000_000
    one = torch.zeros((1, 1, 1, 1, 32), dtype=torch.bfloat16, device=DEV).expand(1, 4, page, 1, 32)     # (nobody reads it)
    cache = paged.PagedCache(max_seqs=2, max_pages=4, k=one, v=one)

    def extend(seq, n):
        seqs, new = i32([seq]), i32([n])
        binding._check(cache._L.ouro_paged_extend(cache._p, seqs.data_ptr(), new.data_ptr(), 1, n, None, None, cache._stream()))

    extend(0, 1_200_000_000)
    assert cache.lens.tolist() == [1_200_000_000, 0] and cache.refs.tolist() == [1, 1, 1, 0] and cache.table[0].tolist() == [0, 1, 2, -1]
    extend(0, 800_000_000)
    assert cache.refs.tolist() == [1, 1, 1, 1]
    cache.fork(i32([0]), i32([1]))
    assert cache.refs.tolist() == [2, 2, 2, 2]
    cache.truncate(i32([0, 1]), i32([1_700_000_000, 0]))
    assert cache.lens.tolist() == [1_700_000_000, 0] and cache.refs.tolist() == [1, 1, 1, 1]
    cache.truncate(i32([0]), i32([0]))
    assert not bool(cache.refs.any()) and bool((cache.table == -1).all())
    cache.check()


def test_sizes_near_31_bits_are_refused_on_the_host():
    build.build()
    L, top = binding.lib(), 2 ** 31 - 65536

    def desc(**change):
        c = binding.PagedCacheC()
        for name, value in dict(dict(n_layers=1, n_pages=4, page_size=16, n_kv_heads=1, head_dim=32, dtype=1, max_seqs=1, max_pages=3, layer_stride=8192, page_stride=2048,
                                     slot_stride=128, head_stride=64, k=256, v=256, table=256, lens=256, refs=256, status=256, workspace=256, workspace_bytes=1 << 50),
                                **change).items():
            setattr(c, name, value)
        return C.byref(c)

    for n in ("n_pages", "max_pages"):
        assert L.ouro_paged_workspace_bytes(desc(page_size=1, **{n: top})) > 0
        assert L.ouro_paged_workspace_bytes(desc(page_size=1, **{n: top + 1})) == 0
        assert L.ouro_paged_workspace_bytes(desc(page_size=1, **{n: 2 ** 31 - 1})) == 0
    assert L.ouro_paged_workspace_bytes(desc(n_pages=1, max_pages=1, page_size=top // 4)) > 0
    assert L.ouro_paged_workspace_bytes(desc(n_pages=1, max_pages=1, page_size=top // 4 + 1)) == 0
    assert L.ouro_paged_workspace_bytes(desc(n_kv_heads=2 ** 31 - 1)) == 0
    # more units of work than 31 bits hold: refused, not rounded over
    d = desc(page_size=1, max_pages=top, n_kv_heads=128)
    assert L.ouro_paged_attention(d, 0, None, 1, 1, 256, 128 * 32, 128, 1.0, 256, None, None) == binding.OURO_EINVAL
    assert b"2^31 units" in L.ouro_last_error(None)


@gpu
@pytest.mark.parametrize("h,d", [(1, 32), (4, 32), (20, 64)])
def test_a_sequence_of_nearly_all_tokens_that_there_can_be(h, d):
    """134 million entries that name one page over and over: units, their costs and page ids at the end of the range.  The last key is looked for twice,
    once among equals, where the output is the mean of the values, and once alone.

    2^31 keys on some 150 CTAs of 4 warps: a sum takes at most 250000 times 64 keys in a row, each rounded to 2^-24 of the sum, in l and in the output."""
    build.build()
    page, n = 16, 2 ** 27 - 4096
    k, v = torch.zeros((2, 1, 2, page, 1, d), dtype=torch.bfloat16, device=DEV)
    v[0, 0] = torch.randn((page, 1, d), device=DEV).to(torch.bfloat16)
    v[0, 1] = 3.0
    k[0, 1, -1, 0, 0] = 1.0                                # the last page's last key, in the first dim
    cache = paged.PagedCache(max_seqs=1, max_pages=n, k=k, v=v)
    cache.table.zero_()
    cache.table[0, -1] = 1
    cache.lens.fill_(n * page - 3)
    q = torch.zeros((1, 1, h, d), dtype=torch.bfloat16, device=DEV)
    mean = v[0, 0].double().mean(0)[0]
    got = cache.attend(0, q, scale=1.0).double()
    assert bool(((got - mean).abs() <= 2 ** -8 * mean.abs() + 2 * 250000 * 2 ** -24 * float(v[0, 0].abs().max())).all())
    k[0, 1, -4, 0, 0] = 1.0                                # the last key of the sequence, and one behind its end
    q[..., 0] = 64.0
    v[0, 1, -4] = 7.0
    assert bool((cache.attend(0, q, scale=1.0) == 7.0).all())      # e^64 for 2^31 others: 3e-19 of it is theirs
    cache.check()


# ---------------------------------------------------------------------------------------------- attention
def reference(k, v, table, lens, seqs, q, scale):
    n, t, h, d = q.shape
    page, hkv = k.shape[1], k.shape[2]
    out = torch.zeros((n, t, h, d), dtype=torch.float64, device=DEV)
    lse = torch.full((n, t, h), -float("inf"), dtype=torch.float64, device=DEV)
    for i, s in enumerate(seqs):
        if not 0 <= s < len(lens):
            continue
        at = [(int(table[s][j // page]), j % page, j) for j in range(lens[s])]
        for tok in range(t):
            seen = [(p, r) for p, r, j in at if j < lens[s] - t + 1 + tok and 0 <= p < k.shape[0]]
            if not seen:
                continue
            p, r = torch.tensor(seen, device=DEV).T
            kk, vv = k[p, r].double(), v[p, r].double()
            x = torch.einsum("grd,jgd->grj", q[i, tok].double().view(hkv, h // hkv, d), kk) * scale
            lse[i, tok] = torch.logsumexp(x, -1).view(h)
            out[i, tok] = torch.einsum("grj,jgd->grd", torch.softmax(x, -1), vv).reshape(h, d)
    return out, lse


def filled(layout, page, hkv, d, dtype, lens, spare=3, seed=0, garbage=True):
    """A cache whose sequences have these lengths, on pages in no order; what no sequence names holds NaN and infinities."""
    used = sum(-(-x // page) for x in lens)
    n_pages, width = used + spare, max(1, max(-(-x // page) for x in lens)) + 1
    k, v = layouts(layout, 2, n_pages, page, hkv, d, dtype)
    cache = paged.PagedCache(max_seqs=len(lens), max_pages=width, k=k, v=v)
    ids = np.random.default_rng(seed).permutation(n_pages)
    table, at = np.full((len(lens), width), -1), 0
    named = torch.zeros((n_pages, page), dtype=torch.bool)
    for s, x in enumerate(lens):
        m = -(-x // page)
        table[s, :m] = ids[at: at + m]
        at += m
        for j in range(x):
            named[int(table[s, j // page]), j % page] = True
    if garbage:
        junk = torch.tensor([float("nan"), float("inf"), -float("inf"), 1e30], device=DEV, dtype=dtype).repeat(d // 4)
        for t in (k, v):
            t[:, ~named.to(DEV)] = junk
    cache.table.copy_(i32(table))
    cache.lens.copy_(i32(lens))
    return cache, table


def close(got, want, vmax, dtype):
    bound = (2 ** -8 * want.abs() + 2 ** -13 * vmax) if dtype == torch.bfloat16 else torch.full_like(want, 1e-4 * vmax)
    bad = (got.double() - want).abs() > bound
    assert torch.isfinite(got).all() and not bool(bad.any()), float(((got.double() - want).abs() / bound).max())


CASES = [  # layout, page, query heads, kv heads, head dim, type, new, lengths
    ("rows", 16, 4, 4, 32, "f32", 1, [0, 1, 2, 7, 8, 9, 31, 32, 33, 67]),
    ("rows", 16, 32, 4, 64, "bf16", 1, [0, 1, 15, 16, 17, 63, 64, 65, 129, 700]),
    ("heads", 24, 32, 32, 128, "bf16", 1, [1, 130, 1025, 0]),
    ("rows", 64, 56, 8, 128, "bf16", 5, [0, 1, 3, 4, 5, 6, 64, 68, 69, 777]),
    ("both", 1, 8, 1, 96, "bf16", 3, [2, 3, 40, 199]),
    ("padded", 7, 71, 1, 64, "bf16", 1, [5, 400, 0, 64]),
    ("rows", 128, 64, 8, 128, "bf16", 16, [15, 16, 17, 300, 2000]),
    ("heads", 40, 6, 2, 96, "f32", 4, [0, 2, 5, 33, 250]),
    ("rows", 8, 12, 1, 128, "f32", 2, [1, 90, 1000]),
    ("rows", 32, 2, 1, 32, "bf16", 1, [6000]),
    ("rows", 256, 8, 8, 64, "f32", 1, [3000, 2]),
]


@gpu
@pytest.mark.parametrize("layout,page,h,hkv,d,dtype,new,lens", CASES)
def test_attention_equals_the_definition(layout, page, h, hkv, d, dtype, new, lens):
    build.build()
    dt = torch.float32 if dtype == "f32" else torch.bfloat16
    cache, table = filled(layout, page, hkv, d, dt, lens)
    n = len(lens)
    g = torch.Generator(device=DEV).manual_seed(1)
    q = (2 * torch.randn((n, new, h, d), device=DEV, generator=g)).to(dt)
    scale = d ** -0.5
    vmax = 5.5
    for layer in (0, 1):
        out, lse = cache.attend(layer, q, want_lse=True)
        want, want_lse = reference(cache.k[layer], cache.v[layer], table, lens, range(n), q, scale)
        close(out, want, vmax, dt)
        some = torch.isfinite(want_lse)
        assert torch.equal(some, torch.isfinite(lse)) and bool((lse[~some] == -float("inf")).all())
        assert bool(((lse - want_lse)[some].abs() <= 1e-4).all())
    again = cache.attend(1, q)
    assert torch.equal(again, out)                         # whoever joins the pieces
    # other sequences, in another order, one of them twice, one outside the table; queries that are part of a wider projection
    seqs = ([n - 1, 0, -1, n - 1, n] + list(range(n)))[: 6]
    wide = torch.zeros((len(seqs), new, h + 2, d), dtype=dt, device=DEV)
    part = wide[:, :, 1: h + 1]
    part.copy_(q[[s if 0 <= s < n else 0 for s in seqs]])
    got = cache.attend(1, part, i32(seqs), scale=0.3)
    want, _ = reference(cache.k[1], cache.v[1], table, lens, seqs, part, 0.3)
    close(got, want, vmax, dt)


@gpu
@pytest.mark.parametrize("page,h,hkv,d", [(16, 4, 4, 128), (32, 32, 4, 64), (64, 16, 1, 128), (128, 12, 1, 64), (16, 6, 3, 96)])
def test_whole_units_to_the_last(page, h, hkv, d):
    """Lengths of whole units with one new token: nothing at a sequence's end is looked at apart, the contractions come right behind the wait."""
    build.build()
    for lens in ([64], [128, 64, 192], [64 * k for k in range(1, 30)], [64 * 200, 64], [4096] * 9):
        lens = [-(-x // page) * page for x in lens]
        cache, table = filled("rows", page, hkv, d, torch.bfloat16, lens)
        q = torch.randn((len(lens), 1, h, d), device=DEV).to(torch.bfloat16)
        want, _ = reference(cache.k[0], cache.v[0], table, lens, range(len(lens)), q, d ** -0.5)
        first = cache.attend(0, q)
        close(first, want, 5.5, torch.bfloat16)
        for _ in range(20):
            assert torch.equal(cache.attend(0, q), first)
        cache.check()


@gpu
def test_one_token_and_three_dimensions():
    build.build()
    cache, table = filled("rows", 16, 2, 128, torch.bfloat16, [33, 5])
    q = torch.randn((2, 4, 128), device=DEV).to(torch.bfloat16)
    a, b = cache.attend(0, q), cache.attend(0, q.view(2, 1, 4, 128))
    assert a.shape == q.shape and torch.equal(a, b[:, 0])
    out = torch.empty_like(q)
    assert cache.attend(0, q, out=out) is out and torch.equal(out, a)


@gpu
@pytest.mark.parametrize("layout,page,h,hkv,d,new,lens", [
    ("rows", 16, 24, 1, 128, 1, [0, 1, 63, 64, 65, 1000]), ("heads", 48, 40, 8, 128, 5, [0, 1, 4, 5, 6, 64, 65, 700, 63, 129]), ("rows", 64, 64, 8, 128, 16, [3, 16, 17, 300, 2000]),
    ("both", 32, 32, 4, 64, 8, [8, 7, 63, 64, 65, 500, 1, 0]), ("padded", 16, 71, 1, 64, 16, [15, 16, 200]), ("rows", 128, 32, 1, 128, 4, [5000]), ("rows", 16, 8, 1, 64, 9, [1, 9, 300, 10000]),
    ("rows", 80, 18, 1, 128, 1, [4000, 1, 1, 64]), ("heads", 256, 56, 8, 128, 16, [777, 20])])
def test_attention_of_many_query_rows(layout, page, h, hkv, d, new, lens):
    """More than 16 query rows to a kv head: up to 128, with rows of several row tiles, and several boxes a page."""
    build.build()
    cache, table = filled(layout, page, hkv, d, torch.bfloat16, lens)
    g = torch.Generator(device=DEV).manual_seed(2)
    q = (2 * torch.randn((len(lens), new, h, d), device=DEV, generator=g)).to(torch.bfloat16)
    for layer in (0, 1):
        out, lse = cache.attend(layer, q, want_lse=True)
        want, want_lse = reference(cache.k[layer], cache.v[layer], table, lens, range(len(lens)), q, d ** -0.5)
        close(out, want, 5.5, torch.bfloat16)
        some = torch.isfinite(want_lse)
        assert torch.equal(some, torch.isfinite(lse)) and bool(((lse - want_lse)[some].abs() <= 1e-4).all())
    assert torch.equal(cache.attend(1, q), out)
    # scores that grow along the text, so that maxima do: every key's score larger than the last one's
    n = max(lens)
    ramp = torch.linspace(0, 40, n, device=DEV)
    for s, x in enumerate(lens):
        for j in range(0, x, max(1, x // 50)):
            cache.k[0, int(table[s, j // page]), j % page] = (ramp[j] * torch.ones((hkv, d), device=DEV) / d ** 0.5).to(torch.bfloat16)
    q = torch.ones_like(q)
    want, _ = reference(cache.k[0], cache.v[0], table, lens, range(len(lens)), q, d ** -0.5)
    close(cache.attend(0, q), want, 5.5, torch.bfloat16)
    cache.check()


@gpu
@pytest.mark.parametrize("dtype,heads,d", [("f32", 8, 64), ("bf16", 8, 64), ("bf16", 20, 64), ("bf16", 64, 128)])
def test_later_tokens_do_not_reach_earlier_ones(dtype, heads, d):
    """Keys and values of a later token that are not numbers are masked places for the earlier ones."""
    build.build()
    dt = torch.float32 if dtype == "f32" else torch.bfloat16
    lens, new = [37, 64, 3, 66, 400], 4
    cache, table = filled("rows", 16, 2, d, dt, lens)
    q = torch.randn((len(lens), new, heads, d), device=DEV).to(dt)
    want = cache.attend(0, q)
    at = [(int(table[s, (x - 1) // 16]), (x - 1) % 16) for s, x in enumerate(lens)]
    keep = cache.v[0].clone()
    for p, r in at:                                        # a single value: its column alone, for the last token alone
        cache.v[0, p, r, :, 5] = float("inf")
    got = cache.attend(0, q)
    assert bool((got[:, -1, :, 5] == float("inf")).all())
    got[:, -1, :, 5] = want[:, -1, :, 5]
    assert torch.isfinite(got).all() and bool(((got - want).abs() <= 2 ** -7 * want.abs() + 2 ** -12).all())
    cache.v[0].copy_(keep)
    for p, r in at:
        cache.k[0, p, r] = float("nan")
        cache.v[0, p, r] = float("inf")
    got = cache.attend(0, q)
    assert torch.equal(got[:, :-1], want[:, :-1]) if dtype == "f32" else bool(((got - want)[:, :-1].abs() <= 2 ** -7 * want[:, :-1].abs() + 2 ** -12).all())
    assert not torch.isfinite(got[:, -1]).any()


@gpu
@pytest.mark.parametrize("h,hkv,d,new,page,lens", [
    (8, 2, 128, 1, 16, [0, 1, 700, 64, 4000]), (32, 4, 64, 2, 32, [33, 900]), (16, 2, 96, 1, 16, [300, 300]), (4, 4, 32, 1, 16, [90]),      # mma.sync
    (64, 8, 128, 5, 64, [0, 3, 700, 64, 4000]), (32, 1, 64, 1, 16, [5000, 17]), (64, 4, 64, 16, 32, [40] * 30), (24, 1, 128, 1, 128, [9])])  # tcgen05
def test_a_wait_that_runs_out_is_reported_and_leaves_nothing_behind(h, hkv, d, new, page, lens):
    """The kernels return normally, the status says so, and the calls that follow give the bits they gave before."""
    build.build()
    cache, _ = filled("rows", page, hkv, d, torch.bfloat16, lens)
    q = torch.randn((len(lens), new, h, d), device=DEV).to(torch.bfloat16)
    want, lse = cache.attend(1, q, want_lse=True)
    cache.check()
    try:
        for limit in (0, 0, 1, 2, 5, 20):
            paged.set_wait_limit(limit)
            for _ in range(3):
                cache.attend(1, q)
            if limit == 0:
                with pytest.raises(binding.OuroError) as e:
                    cache.check()
                assert e.value.status == binding.OURO_ETIMEOUT
            paged.set_wait_limit(-1)
            got, got_lse = cache.attend(1, q, want_lse=True)
            if limit == 0:
                cache.check()
            else:                                          # (so few polls may or may not do)
                try:
                    cache.check()
                except binding.OuroError as err:
                    assert err.status == binding.OURO_ETIMEOUT
            assert torch.equal(got, want) and torch.equal(got_lse, lse)
    finally:
        paged.set_wait_limit(-1)
    cache.check()


@gpu
def test_missing_and_foreign_pages_are_left_out():
    build.build()
    cache, table = filled("rows", 16, 2, 128, torch.bfloat16, [100, 40], garbage=False)
    table[0, 2], table[1, 0] = -1, cache.k.shape[1]        # the latter one beyond the pool
    cache.table.copy_(i32(table))
    q = torch.randn((2, 1, 4, 128), device=DEV).to(torch.bfloat16)
    want, _ = reference(cache.k[0], cache.v[0], table, [100, 40], [0, 1], q, 128 ** -0.5)
    close(cache.attend(0, q), want, 5.5, torch.bfloat16)
    cache.lens.copy_(i32([10 ** 6, -5]))                   # lengths beyond the table's row, and below nothing
    want, _ = reference(cache.k[0], cache.v[0], table, [cache.max_pages * 16, 0], [0, 1], q, 128 ** -0.5)
    close(cache.attend(0, q), want, 5.5, torch.bfloat16)


@gpu
def test_a_batch_of_more_sequences_than_threads():
    build.build()
    rng = np.random.default_rng(3)
    lens = rng.integers(0, 40, 1024).tolist()
    cache, table = filled("rows", 8, 1, 32, torch.bfloat16, lens, garbage=False)
    q = torch.randn((1024, 1, 2, 32), device=DEV).to(torch.bfloat16)
    want, _ = reference(cache.k[0], cache.v[0], table, lens, range(1024), q, 32 ** -0.5)
    close(cache.attend(0, q), want, 5.5, torch.bfloat16)


@gpu
def test_offsets_beyond_32_bits():
    """A pool of more than 2^31 elements: the pages at its end."""
    build.build()
    page, hkv, d = 64, 8, 128
    n_pages = 2 ** 31 // (page * hkv * d) + 40
    k = torch.empty((1, n_pages, page, hkv, d), dtype=torch.bfloat16, device=DEV)
    v = torch.empty_like(k)
    cache = paged.PagedCache(max_seqs=1, max_pages=8, k=k, v=v)
    ids = [n_pages - 1, 0, n_pages - 7, n_pages - 2]
    for p in ids:
        k[0, p] = torch.randn((page, hkv, d), device=DEV).to(torch.bfloat16)
        v[0, p] = torch.randn((page, hkv, d), device=DEV).to(torch.bfloat16)
    cache.table[0, :4] = i32(ids)
    cache.lens.fill_(250)
    q = torch.randn((1, 1, 16, d), device=DEV).to(torch.bfloat16)
    want, _ = reference(k[0], v[0], [ids], [250], [0], q, d ** -0.5)
    close(cache.attend(0, q), want, 5.5, torch.bfloat16)
    cos, sin = paged.rotary_tables(4, d)
    slots = i32([(n_pages - 3) * page + 5, -1])
    kv = torch.randn((2, hkv, d), device=DEV).to(torch.bfloat16)
    cache.append(0, torch.zeros((2, 16, d), dtype=torch.bfloat16, device=DEV), kv, kv, slots, i32([0, 1]), cos, sin)
    assert torch.equal(k[0, n_pages - 3, 5], kv[0]) and torch.equal(v[0, n_pages - 3, 5], kv[0])


# ---------------------------------------------------------------------------------------------- append
@gpu
@pytest.mark.parametrize("layout,page,h,hkv,d,dtype,rows", [("rows", 16, 32, 4, 64, "bf16", 1), ("heads", 5, 6, 3, 96, "bf16", 37), ("both", 64, 64, 8, 128, "bf16", 130),
                                                            ("padded", 16, 4, 4, 32, "f32", 20), ("rows", 1, 5, 5, 128, "f32", 9), ("rows", 24, 3, 1, 32, "bf16", 64)])
def test_append_rotates_and_writes(layout, page, h, hkv, d, dtype, rows):
    build.build()
    dt = torch.float32 if dtype == "f32" else torch.bfloat16
    n_pages = 2 * rows // page + 4
    k, v = layouts(layout, 2, n_pages, page, hkv, d, dt)
    wk, wv = k.clone(), v.clone()
    cache = paged.PagedCache(max_seqs=1, max_pages=1, k=k, v=v)
    qkv = torch.randn((rows, h + 2 * hkv, d), device=DEV).to(dt)             # one projection
    q, kn, vn = qkv[:, :h], qkv[:, h: h + hkv], qkv[:, h + hkv:]
    rng = np.random.default_rng(0)
    slots = rng.permutation(n_pages * page)[:rows]
    pos = rng.integers(0, 50, rows)
    if rows > 8:
        slots[[2, 5]] = -1, n_pages * page                                   # padding, and beyond the pool
        pos[7], pos[8] = -1, 50                                              # positions without angles
    cos, sin = paged.rotary_tables(50, d)
    out = cache.append(1, q, kn, vn, i32(slots), i32(pos), cos, sin)
    known = torch.tensor((pos >= 0) & (pos < 50), device=DEV)
    there = known & torch.tensor((slots >= 0) & (slots < n_pages * page), device=DEV)
    a = torch.outer(torch.tensor(np.clip(pos, 0, 49), device=DEV, dtype=torch.float64), 10000.0 ** (-2.0 * torch.arange(d // 2, dtype=torch.float64, device=DEV) / d))

    def turned(x):
        z = torch.complex(x[..., : d // 2].double(), x[..., d // 2:].double()) * torch.polar(torch.ones_like(a), a)[:, None]
        return torch.cat([z.real, z.imag], -1), torch.cat([z.abs(), z.abs()], -1)

    def check(got, x, rows_):
        want, size = turned(x)
        bound = (2 ** -8 * want.abs() if dt == torch.bfloat16 else 0) + 2 ** -22 * size
        assert bool(((got.double() - want).abs() <= bound)[rows_].all())

    check(out, q, known)
    assert bool((out[~known] == 0).all())
    at = torch.tensor(slots, device=DEV)[there]
    got_k = k[1, at // page, at % page]
    want, size = turned(kn)
    bound = (2 ** -8 * want.abs() if dt == torch.bfloat16 else 0) + 2 ** -22 * size
    assert bool(((got_k.double() - want[there]).abs() <= bound[there]).all())
    wk[1, at // page, at % page] = got_k                                     # nothing else was touched
    wv[1, at // page, at % page] = vn[there]
    assert torch.equal(k, wk) and torch.equal(v, wv)
    own = q.contiguous()
    assert cache.append(1, own, kn, vn, i32(slots), i32(pos), cos, sin, out=own) is own and torch.equal(own, out)


# ---------------------------------------------------------------------------------------------- scores
def score_reference(x, tokens, n):
    x = x.double()
    lp = torch.log_softmax(x, -1)
    lp = torch.where((x == -float("inf")).all(-1, keepdim=True), torch.full_like(lp, -float("inf")), lp)
    order = np.lexsort((np.arange(x.shape[1])[None].repeat(x.shape[0], 0), -x.cpu().numpy()))[:, :n]
    ids = torch.tensor(order, device=DEV)
    h = torch.special.entr(lp.exp()).sum(-1)
    ok = (tokens >= 0) & (tokens < x.shape[1])
    got = torch.where(ok, lp.gather(1, tokens.clamp(0, x.shape[1] - 1).long()[:, None])[:, 0], -float("inf"))
    return got, h, ids, lp.gather(1, ids)


def score_check(s, want, n):
    for got, ref, bound in ((s.logprob, want[0], 3e-5), (s.entropy, want[1], 3e-4)) + (((s.top_logprobs, want[3], 3e-5),) if n else ()):
        f = torch.isfinite(ref)
        assert torch.equal(f, torch.isfinite(got)) and torch.equal(got[~f].double(), ref[~f])
        assert bool(((got.double() - ref)[f].abs() <= bound + 2 ** -22 * ref[f].abs()).all()), float((got.double() - ref)[f].abs().max())
    if n:
        assert torch.equal(s.top_ids.long(), want[2])


@gpu
@pytest.mark.parametrize("rows,vocab,dtype,n", [(1, 1, "f32", 1), (1, 7, "bf16", 5), (3, 31, "f32", 31), (2, 33, "f32", 32), (1, 32000, "f32", 5), (1, 4096, "bf16", 0),
                                                (5, 16385, "bf16", 32), (40, 64001, "f32", 20), (300, 1000, "f32", 8), (17, 32000, "bf16", 1), (2, 130001, "f32", 32)])
@pytest.mark.parametrize("kind", ["peaked", "flat", "rising", "falling", "ties", "banned", "few"])
def test_scores_equal_the_definition(rows, vocab, dtype, n, kind):
    build.build()
    dt = torch.float32 if dtype == "f32" else torch.bfloat16
    g = torch.Generator(device=DEV).manual_seed(vocab + n)
    x = torch.randn((rows, vocab), device=DEV, generator=g)
    if kind == "peaked":
        x = 4 * x
    elif kind == "rising":
        x = torch.linspace(-9, 9, vocab, device=DEV).expand(rows, vocab).clone()
    elif kind == "falling":
        x = torch.linspace(9, -9, vocab, device=DEV).expand(rows, vocab).clone()
    elif kind == "ties":
        x = x.round()
        x[0] = 0.0
        x[0, ::2] = -0.0
    elif kind == "banned":
        x[torch.rand((rows, vocab), device=DEV, generator=g) < 0.9] = -float("inf")
        x[-1, vocab // 2:] = torch.finfo(dt).min            # masks of the type's lowest value
    elif kind == "few":
        x[:] = -float("inf")
        if rows > 1:
            x[1:, vocab - 1] = 3.0
            x[1:, 0] = 2.0
    # rows at an odd distance, so that they begin at every alignment
    wide = torch.full((rows, vocab + 3), float("nan"), dtype=dt, device=DEV)
    part = wide[:, 1: vocab + 1]
    part.copy_(x.clamp(min=torch.finfo(dt).min) if kind not in ("banned", "few") else x)
    tokens = torch.randint(0, vocab, (rows,), device=DEV, generator=g, dtype=torch.int32)
    tokens[0] = 0
    if rows > 2:
        tokens[1], tokens[2] = vocab, -1                    # outside the vocabulary
    want = score_reference(part, tokens, n)
    score_check(scores.token_logprobs(part, tokens, n), want, n)
    dense = part.contiguous()
    score_check(scores.token_logprobs(dense, tokens, n), want, n)
    only = scores.token_logprobs(dense, None, n)
    assert only.logprob is None and torch.equal(only.entropy, scores.token_logprobs(dense, tokens, n).entropy)


@gpu
@pytest.mark.parametrize("rows,vocab,dtype,n", [(1, 32000, "f32", 20), (5, 32001, "bf16", 32), (600, 16000, "f32", 20), (700, 9001, "bf16", 5), (3, 3000, "f32", 32)])
@pytest.mark.parametrize("left", [0.003, 0.02, 0.0005])
def test_scores_of_rows_where_little_is_left(rows, vocab, dtype, n, left):
    """Constrained decoding: nearly everything is masked; the masked tokens with the lowest ids stand behind what is left, where that is less than n."""
    build.build()
    dt = torch.float32 if dtype == "f32" else torch.bfloat16
    g = torch.Generator(device=DEV).manual_seed(vocab + n)
    x = 3 * torch.randn((rows, vocab), device=DEV, generator=g)
    x[torch.rand((rows, vocab), device=DEV, generator=g) >= left] = -float("inf")
    x[:, vocab // 2] = 0.25                                # (something is)
    x[-1, :200] = 1.0                                      # ties in the first warp's share
    x = x.to(dt)
    tokens = torch.full((rows,), vocab // 2, device=DEV, dtype=torch.int32)
    score_check(scores.token_logprobs(x, tokens, n), score_reference(x, tokens, n), n)


@gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_scores_of_many_rows_that_go_on_rising(dtype):
    """Whole rows in one CTA, whose every batch brings more candidates than the last; and rows of which all logits are equal."""
    build.build()
    dt = torch.float32 if dtype == "f32" else torch.bfloat16
    x = torch.linspace(-20, 20, 100000, device=DEV).expand(300, 100000).clone()
    x[1::3] = x[1::3].flip(1)
    x[2::3] = 0.5
    x = x.to(dt)
    tokens = torch.arange(300, device=DEV, dtype=torch.int32) * 300
    for n in (1, 32):
        score_check(scores.token_logprobs(x, tokens, n), score_reference(x, tokens, n), n)


@gpu
@pytest.mark.parametrize("rows,vocab,dtype,n", [(9, 5, "f32", 1), (7, 700, "bf16", 1), (2, 1024, "f32", 0), (12, 32001, "f32", 20), (700, 4001, "f32", 5), (40, 64000, "bf16", 0)])
@pytest.mark.parametrize("gap", [4.0, 12.0, 20.0])
def test_scores_of_a_token_that_has_nearly_everything(rows, vocab, dtype, n, gap):
    """Its log probability and the entropy are as small as what the others leave, and are known to as many digits.

    A term e^d is off by |d| 2^-23 (the difference and the product with log2 e, rounded), e^x itself by 2^-22, some thirty sums in a row by 2^-24 each;
    where the others have an eighth, what is rounded beside 1 (eight times 2^-24) by 2^-18 of them."""
    build.build()
    dt = torch.float32 if dtype == "f32" else torch.bfloat16
    g = torch.Generator(device=DEV).manual_seed(vocab + int(gap))
    x = torch.randn((rows, vocab + 1), device=DEV, generator=g).clamp(-4, 4).to(dt)[:, :vocab]
    top = (torch.arange(rows, device=DEV) * max(1, (vocab - 1) // max(1, rows - 1))).clamp(max=vocab - 1)
    top[-1] = vocab - 1
    x.scatter_(1, top[:, None], (math.log(vocab) + gap))
    d = x.double() - x.double().gather(1, top[:, None])
    e = d.exp().scatter(1, top[:, None], 0.0)
    left = e.sum(1).log1p()
    h = left - (d * e).sum(1) / (1 + e.sum(1))
    s = scores.token_logprobs(x, top.int(), n)
    bound = float(-d.min()) * 2 ** -23 + 2 ** -22 + 30 * 2 ** -24 + 2 ** -18
    for got, want in ((s.logprob, -left), (s.entropy, h)) + (((s.top_logprobs[:, 0], -left),) if n else ()):
        assert bool(((got.double() - want).abs() <= bound * want.abs()).all()), float(((got.double() - want) / want).abs().max())


@gpu
def test_scores_where_there_is_no_distribution():
    build.build()
    x = torch.randn((4, 5000), device=DEV)
    x[1, 4321] = float("nan")
    x[2, [17, 4000]] = float("inf")
    tokens = i32([3, 3, 3, 3])
    s = scores.token_logprobs(x, tokens, 3)
    for r in (1, 2):
        assert bool(torch.isnan(s.logprob[r])) and bool(torch.isnan(s.entropy[r])) and bool(torch.isnan(s.top_logprobs[r]).all())
    assert s.top_ids[1].tolist()[0] == 4321 and s.top_ids[2].tolist()[:2] == [17, 4000]
    for r in (0, 3):
        want = score_reference(x[r: r + 1], tokens[:1], 3)
        score_check(scores.TokenScores(*(t[r: r + 1] for t in s)), want, 3)


# ---------------------------------------------------------------------------------------------- refusals and streams
def test_refusals_that_need_no_gpu():
    build.build()
    L = binding.lib()
    ok = dict(n_layers=1, n_pages=4, page_size=16, n_kv_heads=2, head_dim=64, dtype=1, max_seqs=2, max_pages=3, layer_stride=8192, page_stride=2048, slot_stride=128,
              head_stride=64, k=256, v=256, table=256, lens=256, refs=256, status=256, workspace=256, workspace_bytes=1 << 30)

    def desc(**change):
        c = binding.PagedCacheC()
        for name, value in dict(ok, **change).items():
            setattr(c, name, value)
        return C.byref(c)

    assert L.ouro_paged_workspace_bytes(desc()) > 0
    for bad in (dict(head_dim=48), dict(head_dim=160), dict(dtype=2), dict(page_size=0), dict(n_pages=0), dict(max_seqs=65537), dict(n_pages=1 << 30), dict(max_pages=1 << 28)):
        assert L.ouro_paged_workspace_bytes(desc(**bad)) == 0, bad
        assert L.ouro_paged_reset(desc(**bad), None) == binding.OURO_EINVAL
    assert L.ouro_paged_workspace_bytes(None) == 0
    for bad in (dict(k=0), dict(v=264), dict(table=0), dict(workspace=128), dict(workspace_bytes=100), dict(head_stride=60), dict(slot_stride=-128), dict(refs=258), dict(status=0)):
        for call in (lambda d: L.ouro_paged_reset(d, None), lambda d: L.ouro_paged_fork(d, 256, 256, 1, None), lambda d: L.ouro_paged_compact(d, None, None),
                     lambda d: L.ouro_paged_attention(d, 0, None, 1, 1, 256, 128, 2, 1.0, 256, None, None), lambda d: L.ouro_paged_status(d, None)):
            assert call(desc(**bad)) == binding.OURO_EINVAL and L.ouro_last_error(None).startswith(b"ouro_paged_"), bad
    d = desc()
    att = lambda layer=0, n=1, new=1, q=256, stride=128, heads=2, out=256, scale=1.0: L.ouro_paged_attention(
        d, layer, None, n, new, q, stride, heads, scale, out, None, None)
    for bad in (dict(layer=1), dict(layer=-1), dict(n=-1), dict(n=1025), dict(new=0), dict(new=17), dict(heads=3), dict(heads=0), dict(q=0), dict(out=0), dict(q=8), dict(stride=124),
                dict(stride=64), dict(n=3), dict(scale=0.0), dict(scale=-1.0), dict(scale=float("nan")), dict(scale=float("inf"))):
        assert att(**bad) == binding.OURO_EINVAL, bad
    assert att(n=0) == binding.OURO_OK
    app = lambda layer=0, q=256, qs=128, k=256, kvs=128, rows=1, heads=2, slots=256, cos=256, np_=4, out=512: L.ouro_paged_append(
        d, layer, q, qs, k, 256, kvs, rows, heads, slots, 256, cos, 256, np_, out, None)
    for bad in (dict(layer=2), dict(q=0), dict(qs=64), dict(kvs=120), dict(rows=-1), dict(heads=0), dict(slots=0), dict(cos=4), dict(np_=0), dict(out=0), dict(q=512, qs=256), dict(k=264)):
        assert app(**bad) == binding.OURO_EINVAL, bad
    assert app(rows=0) == binding.OURO_OK
    for rc in (L.ouro_paged_fork(d, None, 256, 1, None), L.ouro_paged_fork(d, 256, 256, 1025, None), L.ouro_paged_truncate(d, 256, None, 1, None), L.ouro_paged_truncate(d, 256, 256, -1, None),
               L.ouro_paged_extend(d, 256, 256, 1, -1, None, None, None), L.ouro_paged_extend(d, 256, None, 1, 1, None, None, None)):
        assert rc == binding.OURO_EINVAL
    assert L.ouro_paged_fork(d, None, None, 0, None) == binding.OURO_OK
    sc = lambda x=256, dt=0, stride=100, rows=2, vocab=100, tok=256, n=1, lp=256, ids=256, top=256: L.ouro_token_logprobs(x, dt, stride, rows, vocab, tok, n, lp, 256, ids, top, None)
    for bad in (dict(x=0), dict(x=258), dict(dt=2), dict(stride=99), dict(rows=-1), dict(vocab=0), dict(tok=0), dict(lp=0), dict(n=33), dict(n=-1), dict(n=0), dict(ids=0), dict(top=0),
                dict(vocab=5, n=6)):
        assert sc(**bad) == binding.OURO_EINVAL and L.ouro_last_error(None).startswith(b"ouro_token_logprobs"), bad
    assert sc(rows=0) == binding.OURO_OK


def test_arrays_of_words_have_to_be_aligned():
    build.build()
    L, W = binding.lib(), 256
    d = binding.PagedCacheC(n_layers=1, n_pages=4, page_size=16, n_kv_heads=2, head_dim=64, dtype=1, max_seqs=2, max_pages=3, layer_stride=8192, page_stride=2048, slot_stride=128,
                            head_stride=64, k=W, v=W, table=W, lens=W, refs=W, status=W, workspace=W, workspace_bytes=1 << 30)
    d = C.byref(d)
    fork = lambda src=W, dst=W: L.ouro_paged_fork(d, src, dst, 1, None)
    cut = lambda seqs=W, keep=W: L.ouro_paged_truncate(d, seqs, keep, 1, None)
    extend = lambda seqs=W, new=W, slots=W, pos=W: L.ouro_paged_extend(d, seqs, new, 1, 1, slots, pos, None)
    compact = lambda live=W: L.ouro_paged_compact(d, live, None)
    append = lambda slots=W, pos=W: L.ouro_paged_append(d, 0, W, 128, W, W, 128, 1, 2, slots, pos, W, W, 4, 512, None)
    attend = lambda seqs=W, lse=W: L.ouro_paged_attention(d, 0, seqs, 1, 1, W, 128, 2, 1.0, W, lse, None)
    score = lambda tokens=W, lp=W, h=W, ids=W, top=W: L.ouro_token_logprobs(W, 0, 100, 2, 100, tokens, 1, lp, h, ids, top, None)
    for call, names in ((fork, "src dst"), (cut, "seqs keep"), (extend, "seqs new slots pos"), (compact, "live"), (append, "slots pos"), (attend, "seqs lse"),
                        (score, "tokens lp h ids top")):
        for name in names.split():
            for off in (1, 2, 3):
                assert call(**{name: W + off}) == binding.OURO_EINVAL, (name, off)
                assert b"4-byte" in L.ouro_last_error(None)


@pytest.mark.parametrize("dtype", ["fp32", "float32", "f16", "fp8", torch.float16, torch.int32, None])
def test_pages_of_a_type_that_there_is_not(dtype):
    """(Refused before anything is allocated: no GPU is needed.)"""
    with pytest.raises(ValueError, match="dtype"):
        paged.PagedCache(1, 8, 16, 2, 64, dtype, max_seqs=1, max_pages=1)


def test_python_handles_need_a_gpu():
    if torch.cuda.is_available():
        pytest.skip("GPU present")
    with pytest.raises(ValueError):
        paged.PagedCache(max_seqs=1, max_pages=1, k=torch.zeros(1, 1, 1, 1, 32), v=torch.zeros(1, 1, 1, 1, 32))
    with pytest.raises(ValueError):
        scores.token_logprobs(torch.zeros(1, 4))


@gpu
def test_pages_are_of_the_type_asked_for():
    build.build()
    for dtype, want in (("f32", torch.float32), ("bf16", torch.bfloat16), (torch.float32, torch.float32), (torch.bfloat16, torch.bfloat16)):
        cache = paged.PagedCache(1, 8, 16, 2, 64, dtype, max_seqs=1, max_pages=1)
        assert cache.k.dtype is want and cache.v.dtype is want


@gpu
@pytest.mark.parametrize("shape", [(), (64,), (4, 64), (1, 1, 1, 4, 64)])
def test_attend_takes_three_or_four_dimensions(shape):
    build.build()
    cache = paged.PagedCache(1, 8, 16, 2, 64, "bf16", max_seqs=4, max_pages=4)
    with pytest.raises(ValueError):
        cache.attend(0, torch.zeros(shape, dtype=torch.bfloat16, device=DEV))


@gpu
def test_python_refuses_what_does_not_fit():
    build.build()
    cache = paged.PagedCache(1, 8, 16, 2, 64, "bf16", max_seqs=4, max_pages=4)
    q = torch.zeros((1, 4, 64), dtype=torch.bfloat16, device=DEV)
    for bad in (lambda: cache.attend(0, q.float()), lambda: cache.attend(0, q[..., :32]), lambda: cache.attend(0, q, seqs=torch.zeros(1, dtype=torch.int64, device=DEV)),
                lambda: cache.attend(0, q, out=q[:, :2]), lambda: cache.attend(0, q.transpose(1, 2).contiguous().transpose(1, 2)), lambda: cache.fork(i32([0]), i32([1, 2])),
                lambda: cache.extend(torch.zeros(1, dtype=torch.int32), i32([1]), 1), lambda: scores.token_logprobs(q[0].half()), lambda: scores.token_logprobs(q[0], i32([1, 2])),
                lambda: scores.token_logprobs(q[0].T), lambda: paged.PagedCache(max_seqs=1, max_pages=1, k=cache.k, v=cache.v.float())):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: cache.attend(1, q), lambda: cache.attend(0, q[:, :3].contiguous()), lambda: scores.token_logprobs(q[0], None, 33),
                lambda: cache.attend(0, q.expand(5, 4, 64).contiguous())):
        with pytest.raises(binding.OuroError) as e:
            bad()
        assert e.value.status == binding.OURO_EINVAL
    # lists that only the device can see wrong
    for call, status in ((lambda: cache.fork(i32([0, 9]), i32([1, 2])), binding.OURO_EINVAL), (lambda: cache.fork(i32([0, 0]), i32([1, 1])), binding.OURO_EINVAL),
                         (lambda: cache.truncate(i32([0]), i32([-1])), binding.OURO_EINVAL), (lambda: cache.extend(i32([-1]), i32([1]), 1), binding.OURO_EINVAL),
                         (lambda: cache.extend(i32([0]), i32([2]), 1), binding.OURO_EINVAL), (lambda: cache.extend(i32([0, 0]), i32([1, 1]), 1), binding.OURO_EINVAL),
                         (lambda: cache.extend(i32([0]), i32([65]), 65), binding.OURO_ECAPACITY), (lambda: cache.extend(i32([0, 1, 2]), i32([64, 64, 64]), 64), binding.OURO_ECAPACITY)):
        before = cache.state.clone()
        call()
        with pytest.raises(binding.OuroError) as e:
            cache.check()
        assert e.value.status == status and torch.equal(cache.state, before)
        cache.check()


@gpu
@pytest.mark.parametrize("q,k,v", [((5, 1, 4, 64), (5, 1, 2, 64), (5, 1, 2, 64)), ((5, 4, 64), (5, 2, 2, 64), (5, 2, 2, 64)), ((5, 4, 64), (5, 2, 64), (5, 1, 2, 64)),
                                   ((1, 5, 4, 64), (1, 5, 2, 64), (1, 5, 2, 64)), ((5 * 4, 64), (5, 2, 64), (5, 2, 64)), ((64,), (64,), (64,))])
def test_append_takes_rows_of_heads_only(q, k, v):
    """Tensors as `attend` takes them, with a dimension for the new tokens, would be read as other numbers of rows and heads."""
    build.build()
    cache = paged.PagedCache(1, 8, 16, 2, 64, "bf16", max_seqs=4, max_pages=4)
    cos, sin = paged.rotary_tables(16, 64)
    q, k, v = (torch.ones(s, dtype=torch.bfloat16, device=DEV) for s in (q, k, v))
    rows = i32(range(q.shape[0]))
    with pytest.raises(ValueError):
        cache.append(0, q, k, v, rows, rows, cos, sin)
    assert not bool(cache.k.any()) and not bool(cache.v.any())


@gpu
@pytest.mark.parametrize("shape", [(32,), (1, 16, 32), (16, 1, 32), (16, 31), (0, 32), (16, 64)])
def test_append_takes_tables_of_positions_only(shape):
    """A single row of angles would be read as head_dim / 2 positions, beyond its end; a table with another dimension as one position."""
    build.build()
    cache = paged.PagedCache(1, 8, 16, 2, 64, "bf16", max_seqs=4, max_pages=4)
    q, kv = torch.ones((3, 4, 64), dtype=torch.bfloat16, device=DEV), torch.ones((3, 2, 64), dtype=torch.bfloat16, device=DEV)
    t = torch.ones(shape, device=DEV)
    with pytest.raises((ValueError, binding.OuroError)):
        cache.append(0, q, kv, kv, i32(range(3)), i32(range(3)), t, t)
    assert not bool(cache.k.any())


@gpu
def test_calls_run_on_the_current_stream():
    build.build()
    cache, table = filled("rows", 16, 2, 64, torch.bfloat16, [500, 30])
    q = torch.randn((2, 1, 8, 64), device=DEV).to(torch.bfloat16)
    x = torch.randn((64, 32000), device=DEV)
    want, s = cache.attend(0, q), scores.token_logprobs(x, None, 4)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    late = torch.zeros_like(q), torch.zeros_like(x)
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(20_000_000)                      # the inputs arrive late on this stream
        late[0].copy_(q)
        late[1].copy_(x)
        got, t = cache.attend(0, late[0]), scores.token_logprobs(late[1], None, 4)
    side.synchronize()
    assert torch.equal(got, want) and torch.equal(t.entropy, s.entropy) and torch.equal(t.top_ids, s.top_ids)
