"""Attention of chunks of new tokens over the paged cache, and rotary positions from frequencies, against plain implementations in 64 bits.

Tolerances, from the arithmetic (fixed before the first run):
 * bf16 attention: the output is rounded once and every probability at most once, each by half a step, 2^-8: 2^-8 (|o| + sum p |v|).  Scores are exact
   products added up in 32 bits: below 2^-13 of the largest |value|.
 * f32 attention: a score of 128 products, each |q k| scale adding up to about 25, in a chain of 128 roundings at worst: 128 x 2^-24 x 25 = 2e-4 relative in
   a probability, twice that in the quotient: 4e-4 of the largest |value|.
 * the logarithm of the sum: the same relative error of a probability plus 2^-22 of itself (bf16 scores: 25 x 128 x 2^-24 as well).
 * rotation: the angle is good to 2^-24 of a radian and its cosine to 2^-23, products and their sum are in 32 bits: 2^-21 of the pair; bf16 then rounds once, 2^-8 relative.
"""
import ctypes as C
import math

import numpy as np
import pytest
import torch

from paper_2402_13720_b200 import binding, build, paged
from paper_2402_13720_b200.rotary import SCALINGS, Rotary, frequencies

gpu = pytest.mark.gpu
DEV = "cuda:0"
F32, BF16 = torch.float32, torch.bfloat16


def i32(x):
    return torch.tensor(np.asarray(x, dtype=np.int32), device=DEV)


def pools(kind, layers, n_pages, page, H, D, dtype, seed):
    """Pools whose elements lie in different orders."""
    if kind == "rows":
        k, v = (torch.zeros((layers, n_pages, page, H, D), dtype=dtype, device=DEV) for _ in range(2))
    elif kind == "heads":                                 # heads outside of rows
        k, v = (torch.zeros((layers, n_pages, H, page, D), dtype=dtype, device=DEV).transpose(2, 3) for _ in range(2))
    elif kind == "padded":                                # rows 32 bytes further apart than they are long
        k, v = (torch.zeros((layers, n_pages, page, H, D + 16), dtype=dtype, device=DEV)[..., :D] for _ in range(2))
    else:                                                 # pages hold all layers, keys beside values
        both = torch.zeros((n_pages, layers, 2, page, H, D), dtype=dtype, device=DEV).transpose(0, 1)
        k, v = both[:, :, 0], both[:, :, 1]
    g = torch.Generator(device=DEV).manual_seed(seed)
    for t in (k, v):
        t.copy_(torch.randn(t.shape, device=DEV, generator=g).to(dtype))
    return k, v


class Call:
    """A cache whose sequences have (len, new) tokens on pages in random order, and queries for the new ones."""

    def __init__(self, chunks, H, Hkv, D, page, dtype, layout="rows", layers=1, seed=0, first=0, more=0, spare=3, max_pages=None):
        build.build()
        r = np.random.default_rng(seed)
        self.chunks, self.H, self.Hkv, self.D, self.page, self.dtype = chunks, H, Hkv, D, page, dtype
        need = [-(-n // page) for n, _ in chunks]
        n_pages = sum(need) + spare
        self.k, self.v = pools(layout, layers, n_pages, page, Hkv, D, dtype, seed)
        self.cache = paged.PagedCache(max_seqs=len(chunks), max_pages=max_pages or max(need + [1]) + 1, k=self.k, v=self.v)
        ids = r.permutation(n_pages)
        self.table = np.full((len(chunks), self.cache.max_pages), -1, dtype=np.int32)
        at = 0
        for i, m in enumerate(need):
            self.table[i, :m] = ids[at: at + m]
            at += m
        self.starts = first + np.concatenate([[0], np.cumsum([m for _, m in chunks])])
        self.set()
        g = torch.Generator(device=DEV).manual_seed(seed + 1)
        self.q = (2 * torch.randn((int(self.starts[-1]) + more, H, D), device=DEV, generator=g)).to(dtype)

    def set(self):
        self.cache.table.copy_(i32(self.table))
        self.cache.lens.copy_(i32([n for n, _ in self.chunks]))

    def slots(self, s):
        """Where the keys of sequence s are that lie on pages: positions and slots."""
        n = self.chunks[s][0]
        j = np.arange(n)
        page = self.table[s, j // self.page].astype(np.int64)
        on = (page >= 0) & (page < self.k.shape[1])
        return j[on], page[on], (j % self.page)[on]

    def expected(self, layer=0, scale=None, seqs=None):
        """out, sum of p |v|, lse in 64 bits; rows of no sequence NaN."""
        scale = self.D ** -0.5 if scale is None else scale
        q = self.q.double()
        out = torch.full_like(q, float("nan"))
        mag = torch.zeros_like(q)
        lse = torch.full(q.shape[:2], float("nan"), dtype=torch.float64, device=DEV)
        g = self.H // self.Hkv
        for i, s in enumerate(range(len(self.chunks)) if seqs is None else seqs):
            a, b = int(self.starts[i]), int(self.starts[i + 1])
            m, n = b - a, self.chunks[s][0] if 0 <= s < len(self.chunks) else 0
            if m == 0:
                continue
            out[a:b], lse[a:b] = 0.0, -float("inf")
            if n == 0:
                continue
            j, pg, row = (torch.tensor(x, device=DEV) for x in self.slots(s))
            keys, values = (t[layer, pg, row].double() for t in (self.k, self.v))
            pos = n - m + torch.arange(m, device=DEV)
            hidden = j[None, :] > pos[:, None]
            for h in range(self.H):
                sc = (q[a:b, h] @ keys[:, h // g].T) * scale
                sc = torch.where(hidden, -float("inf"), sc)
                top = sc.amax(-1, keepdim=True) if sc.shape[1] else torch.full((m, 1), -float("inf"), device=DEV, dtype=torch.float64)
                e = torch.where(hidden, 0.0, torch.exp(sc - torch.where(top == -float("inf"), 0.0, top)))
                z = e.sum(-1, keepdim=True)
                p = torch.where(z > 0, e / z, 0.0)
                v = values[:, h // g]
                clean = torch.where(torch.isfinite(v), v, 0.0)
                o = p @ clean
                odd = (~torch.isfinite(v)).any(1)
                if odd.any():                              # only rows that see them get them
                    for x in odd.nonzero()[:, 0].tolist():
                        seen = ~hidden[:, x]
                        o[seen] = o[seen] + p[seen, x][:, None] * torch.where(torch.isfinite(v[x]), 0.0, v[x])
                out[a:b, h], mag[a:b, h] = o, p @ clean.abs()
                lse[a:b, h] = (top + torch.log(z))[:, 0]
        return out, mag, lse

    def check(self, out, lse, want, untouched=None, most=None):
        o, mag, l = want
        rows = ~torch.isnan(l[:, 0])
        most = most or float(self.v.float().nan_to_num(0, 0, 0).abs().max())
        a, b = out[rows].double(), o[rows]
        tol = 2.0 ** -8 * (b.abs() + mag[rows]) + 2.0 ** -13 * most if self.dtype is BF16 else torch.full_like(b, 4e-4 * most)
        fine = torch.isfinite(b)
        assert bool(((a - b).abs() <= tol)[fine].all()), float(((a - b).abs() - tol)[fine].max())
        assert bool((~torch.isfinite(a) == ~fine).all())
        if lse is not None:
            x, y = lse[rows].double(), l[rows]
            assert bool((torch.isinf(x) == torch.isinf(y)).all())
            ok = torch.isfinite(y)
            assert bool(((x - y).abs()[ok] <= 2e-4 + 2.0 ** -22 * y.abs()[ok]).all()), float((x - y).abs()[ok].max())
        if untouched is not None:
            assert torch.equal(out[~rows], untouched[~rows])

    def run(self, **kw):
        return self.cache.attend_chunk(0, self.q, i32(self.starts), **kw)


SHAPES = [
    # chunks (len, new), heads, kv heads, head dim, page, layout
    ([(1, 1)], 1, 1, 32, 1, "rows"),
    ([(67, 23)], 4, 4, 32, 16, "rows"),
    ([(5, 5), (64, 1), (65, 64), (129, 128), (200, 3)], 4, 2, 64, 16, "heads"),
    ([(300, 257), (1, 1), (0, 0), (256, 256)], 8, 1, 128, 32, "padded"),
    ([(700, 37), (33, 33), (128, 127)], 14, 2, 128, 64, "layers"),
    ([(90, 90), (17, 2)], 6, 2, 96, 8, "rows"),
    ([(200, 130), (10, 10)], 3, 3, 96, 24, "heads"),
    ([(77, 40), (12, 5)], 5, 1, 64, 7, "rows"),
    ([(400, 300)], 2, 2, 128, 20, "rows"),
    ([(513, 385), (640, 128), (384, 384)], 4, 4, 128, 128, "rows"),
    ([(1000, 150)], 64, 8, 128, 48, "rows"),
    ([(50, 3)] * 40, 32, 4, 64, 16, "rows"),
    ([(3 + i, 1 + i % 5) for i in range(300)], 2, 1, 64, 16, "rows"),
    ([(6000, 5)], 4, 2, 64, 16, "rows"),
    ([(20, 30), (0, 4), (1, 2), (64, 65)], 4, 2, 128, 16, "rows"),
]


@gpu
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("chunks,H,Hkv,D,page,layout", SHAPES)
def test_chunk_against_64_bits(chunks, H, Hkv, D, page, layout, dtype):
    c = Call(chunks, H, Hkv, D, page, dtype, layout)
    out, lse = c.run(want_lse=True)
    c.check(out, lse, c.expected())
    again, lse2 = c.run(want_lse=True)
    assert torch.equal(out, again) and torch.equal(lse, lse2)       # the same bits
    c.cache.check()


@gpu
@pytest.mark.parametrize("dtype,page", [(F32, 16), (BF16, 16), (BF16, 8), (BF16, 12)])
def test_chunk_few_rows_behind_long_contexts_are_split_and_joined(dtype, page):
    c = Call([(20011, 9), (4500, 1), (1, 1), (8000, 20)], 8, 2, 128, page, dtype)
    out, lse = c.run(want_lse=True)
    c.check(out, lse, c.expected())


@gpu
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_chunk_lists_strides_and_rows_of_no_sequence(dtype):
    c = Call([(300, 40), (90, 7), (500, 120), (64, 64)], 8, 4, 64, 16, dtype, layers=2, first=3, more=9)
    seqs = [2, 0, 3, 2, -1, 99]                            # twice the same, and two outside the table
    c.starts = np.array([3, 43, 50, 50, 170, 180, 231])
    c.q = c.q[:232].clone()
    wide = torch.randn((232, 3, 8, 64), device=DEV).to(dtype)   # queries that lie among other things
    wide[:, 1] = c.q
    q = wide[:, 1]
    before = torch.randn((232, 8, 64), device=DEV).to(dtype)
    out, lse = c.cache.attend_chunk(1, q, i32(c.starts), i32(seqs), scale=0.3, out=before.clone(), want_lse=True)
    c.check(out, lse, c.expected(layer=1, scale=0.3, seqs=seqs), before)


@gpu
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("page", [16, 8, 20])
def test_chunk_what_is_masked_may_be_anything(dtype, page):
    """Rows of pages behind a sequence's end, missing pages, and keys and values of tokens that come later: infinities and NaN there change nothing."""
    c = Call([(333, 200), (77, 77), (500, 1)], 4, 2, 128, page, dtype)
    clean = c.run()
    rest = torch.ones(c.k.shape[1:3], dtype=torch.bool, device=DEV)
    for s in range(3):
        _, pg, row = c.slots(s)
        rest[torch.tensor(pg, device=DEV), torch.tensor(row, device=DEV)] = False
    c.k[0][rest], c.v[0][rest] = float("nan"), float("inf")
    assert torch.equal(c.run(), clean)
    # the values of some new tokens are no numbers: earlier rows stay what they were
    j, pg, row = c.slots(0)
    for at, x in ((250, float("inf")), (251, float("nan")), (332, -float("inf"))):
        c.v[0, pg[at], row[at], :, 5] = x
    c.k[0, pg[332], row[332]] = float("nan")
    out = c.run()
    first = 333 - 200                                       # position of row 0
    assert torch.equal(out[: 250 - first], clean[: 250 - first])
    assert torch.equal(out[200:], clean[200:])
    assert not bool(torch.isfinite(out[250 - first: 200, :, 5]).any())
    fine = [d for d in range(128) if d != 5]
    assert torch.equal(out[250 - first: 199][:, :, fine], clean[250 - first: 199][:, :, fine])


@gpu
@pytest.mark.parametrize("D", [32, 64, 96, 128])
def test_chunk_products_of_f32_lose_nothing(D):
    """A product made of parts is good to 2^-20 and sums of a few in the contractions to 2^-21, of |q| |k| scale at most in a score; that is 3 x 2^-21 relative in a
    probability, twice in the quotient: 2^-18 with what sums in 32 bits add.  Products with values, the exponentials and the other sums: 2^-17."""
    c = Call([(300, 150), (700, 40), (64, 64)], 4, 2, D, 16, F32)
    out, _ = c.run(want_lse=True)
    want, _, lse = c.expected()
    rows = ~torch.isnan(lse[:, 0])
    size = float(c.q.norm(dim=-1).max() * c.k.norm(dim=-1).max()) / math.sqrt(D)
    most = float(c.v.abs().max())
    assert float((out[rows].double() - want[rows]).abs().max()) <= most * (2.0 ** -18 * size + 2.0 ** -17)


@gpu
@pytest.mark.parametrize("dtype,page", [(F32, 16), (BF16, 16), (BF16, 20)])
def test_chunk_missing_pages_are_left_out(dtype, page):
    c = Call([(333, 50), (200, 200)], 4, 2, 64, page, dtype)
    c.table[0, 3] = -1
    c.table[0, 7] = c.k.shape[1]
    c.table[1, 0] = -5                                      # its first tokens see nothing
    c.set()
    out, lse = c.run(want_lse=True)
    want = c.expected()
    c.check(out, lse, want)
    assert bool((out[50: 50 + page] == 0).all()) and bool(torch.isneginf(lse[50: 50 + page]).all())


@gpu
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_chunk_large_scores(dtype):
    """Scores that grow along the text, so that every unit has a new maximum, and scores of hundreds."""
    c = Call([(700, 300)], 2, 1, 128, 16, dtype)
    j, pg, row = c.slots(0)
    ramp = torch.linspace(0.01, 4.0, 700, device=DEV)
    c.k[0, torch.tensor(pg, device=DEV), torch.tensor(row, device=DEV)] = (ramp[:, None, None] * torch.ones(128, device=DEV)).to(dtype)
    c.q.copy_((torch.rand(c.q.shape, device=DEV) + 0.5).to(dtype))
    out, lse = c.run(want_lse=True)
    o, mag, l = c.expected()
    # (scores up to 4 x 1.5 x 128 / sqrt(128) = 68 of 128 products: 128 x 2^-24 x 68 = 5.2e-4 in a probability)
    most = float(c.v.float().abs().max())
    tol = 2.0 ** -8 * (o.abs() + mag) + 1.1e-3 * most if dtype is BF16 else torch.full_like(o, 1.1e-3 * most)
    assert bool(((out.double() - o).abs() <= tol).all())
    assert bool(((lse.double() - l).abs() <= 6e-4 + 2.0 ** -22 * l.abs()).all())


@gpu
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_chunk_agrees_with_attend(dtype):
    c = Call([(300, 4), (90, 4), (17, 4)], 8, 2, 64, 16, dtype)
    a = c.run()
    b = c.cache.attend(0, c.q.view(3, 4, 8, 64)).view(12, 8, 64)
    _, mag, _ = c.expected()
    most = float(c.v.float().abs().max())
    # both are within their bounds of the same values
    tol = 2.0 ** -8 * (2 * a.double().abs() + mag) * 1.01 + 2.0 ** -12 * most if dtype is BF16 else 8e-4 * most
    assert bool(((a.double() - b.double()).abs() <= tol).all())


@gpu
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("starts", [[-1, 5, 9], [0, 7, 5], [0, 5, 11], [3, 2, 2], [0, 2 ** 31 - 1, 9], [-(2 ** 31), 0, 9]])
def test_chunk_wrong_starts_do_nothing_and_show(starts, dtype):
    c = Call([(30, 5), (20, 5)], 2, 2, 64, 16, dtype)
    out = torch.full_like(c.q, 7.0)
    c.cache.attend_chunk(0, c.q, i32(starts), out=out)
    with pytest.raises(binding.OuroError) as e:
        c.cache.check()
    assert e.value.status == binding.OURO_EINVAL and bool((out == 7.0).all())
    c.cache.check()
    o, lse = c.run(want_lse=True)
    c.check(o, lse, c.expected())


@gpu
def test_chunk_nothing_to_do():
    c = Call([(30, 0), (20, 0)], 2, 2, 64, 16, BF16, more=4)
    out = torch.full_like(c.q, 7.0)
    c.run(out=out)
    assert bool((out == 7.0).all())
    c.cache.attend_chunk(0, c.q, i32([0]), out=out)          # no sequences
    c.cache.attend_chunk(0, c.q[:0], i32([0, 0, 0]))         # no rows
    c.cache.check()
    assert bool((out == 7.0).all())


@gpu
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_chunk_captured_and_on_another_stream(dtype):
    c = Call([(300, 100), (800, 30)], 8, 2, 128, 16, dtype)
    starts, out = i32(c.starts), torch.empty_like(c.q)
    c.cache.attend_chunk(0, c.q, starts, out=out)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        c.cache.attend_chunk(0, c.q, starts, out=out)
    for seed in (3, 4):                                     # other queries, lengths and chunks of the same total
        c.q.copy_(torch.randn(c.q.shape, device=DEV).to(dtype))
        c.chunks = [(300 - seed, 90 + seed), (800, 40 - seed)]
        c.starts = np.array([0, 90 + seed, 130])
        starts.copy_(i32(c.starts))
        c.set()
        out.fill_(0)
        g.replay()
        torch.cuda.synchronize()
        c.check(out, None, c.expected())
    with torch.cuda.stream(s):
        s.wait_stream(torch.cuda.default_stream())
        other = c.run()
    s.synchronize()
    assert torch.equal(other, out)


@gpu
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_chunk_pages_beyond_32_bit_offsets(dtype):
    """A pool of 2^31 elements and more, whose last pages are used."""
    H, D, page = 8, 128, 64
    n_pages = (1 << 31) // (H * D * page) + 70
    build.build()
    k = torch.zeros((1, n_pages, page, H, D), dtype=dtype, device=DEV)
    v = torch.zeros_like(k)
    k[:, -70:].normal_()
    v[:, -70:].normal_()
    c = object.__new__(Call)
    c.chunks, c.H, c.Hkv, c.D, c.page, c.dtype, c.k, c.v = [(4000, 50)], 16, H, D, page, dtype, k, v
    c.cache = paged.PagedCache(max_seqs=1, max_pages=64, k=k, v=v)
    c.table = np.full((1, 64), -1, dtype=np.int32)
    c.table[0, :63] = n_pages - 1 - np.arange(63)
    c.starts = np.array([0, 50])
    c.set()
    c.q = torch.randn((50, 16, D), device=DEV).to(dtype)
    out, lse = c.run(want_lse=True)
    c.check(out, lse, c.expected(), most=float(v[:, -70:].float().abs().max()))


@gpu
@pytest.mark.parametrize("page", [16, 8])
def test_chunk_waits_that_run_out(page):
    """Waits of no or few polls give up: the call returns, the status says so, and the next call is right again."""
    c = Call([(900, 700), (3000, 20), (5, 5)], 8, 2, 128, page, BF16)
    want, lse = c.run(want_lse=True)
    c.cache.check()
    try:
        for limit in (0, 0, 1, 2, 5, 20):
            paged.set_wait_limit(limit)
            for _ in range(3):
                c.run()
            if limit == 0:
                with pytest.raises(binding.OuroError) as e:
                    c.cache.check()
                assert e.value.status == binding.OURO_ETIMEOUT
            paged.set_wait_limit(-1)
            got, got_lse = c.run(want_lse=True)
            if limit == 0:
                c.cache.check()
            else:                                          # (so few polls may or may not do)
                try:
                    c.cache.check()
                except binding.OuroError as err:
                    assert err.status == binding.OURO_ETIMEOUT
            assert torch.equal(got, want) and torch.equal(got_lse, lse)
    finally:
        paged.set_wait_limit(-1)
    c.cache.check()


@gpu
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("page", [16, 20])
def test_chunk_hidden_values_as_large_as_they_get(dtype, page):
    """0 times the type's largest value is 0: tokens that come later, and rows of a page behind the end."""
    c = Call([(300, 150)], 4, 2, 64, page, dtype)
    clean = c.run()
    j, pg, row = c.slots(0)
    big = torch.finfo(dtype).max
    for at in range(200, 300):
        c.v[0, pg[at], row[at]] = big if at % 2 else -big
    out = c.run()
    assert torch.equal(out[:50], clean[:50])


@gpu
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_chunk_keys_that_are_no_numbers_show_where_they_are_seen(dtype):
    """Every place of a unit: a NaN among the keys that a token sees leaves it no distribution, and no other token notices."""
    c = Call([(260, 130)], 2, 1, 64, 16, dtype)
    clean = c.run()
    j, pg, row = c.slots(0)
    starts = i32(c.starts)
    for at in list(range(60, 130)) + [131, 200, 259]:
        keep = c.k[0, pg[at], row[at]].clone()
        c.k[0, pg[at], row[at], :, 3] = float("nan")
        out = c.cache.attend_chunk(0, c.q, starts)
        first = max(0, at - 130)
        assert bool(torch.isnan(out[first:]).all()) and torch.equal(out[:first], clean[:first]), at
        c.k[0, pg[at], row[at]] = keep
    assert torch.equal(c.run(), clean)


@gpu
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("H,Hkv,D", [(160, 1, 64), (256, 2, 32), (66, 3, 128)])
def test_chunk_more_heads_than_a_tile_has_rows(H, Hkv, D, dtype):
    c = Call([(70, 33), (200, 1), (12, 12)], H, Hkv, D, 16, dtype)
    out, lse = c.run(want_lse=True)
    c.check(out, lse, c.expected())


@gpu
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_chunk_as_many_sequences_as_there_may_be(dtype):
    r = np.random.default_rng(5)
    chunks = [(int(a + b), int(b)) for a, b in zip(r.integers(0, 60, 1024), r.integers(0, 4, 1024))]
    c = Call(chunks, 2, 1, 32, 8, dtype)
    out, lse = c.run(want_lse=True)
    c.check(out, lse, c.expected())


@gpu
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_chunk_lengths_outside_the_table(dtype):
    c = Call([(64, 10), (64, 10), (30, 10)], 2, 2, 64, 16, dtype, max_pages=4)
    c.cache.lens.copy_(i32([10 ** 6, -5, 30]))
    out, lse = c.run(want_lse=True)
    c.chunks = [(64, 10), (0, 10), (30, 10)]
    c.check(out, lse, c.expected())


@gpu
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_chunk_two_caches_at_once(dtype):
    """Calls on two caches, which have a workspace each, on two streams; and two graphs of one cache, one after the other."""
    a, b = (Call([(700, 400), (900, 30)], 8, 2, 128, 16, dtype, seed=s) for s in (1, 2))
    want = [x.run() for x in (a, b)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = [[], []]
    for _ in range(10):
        for k, x in enumerate((a, b)):
            with torch.cuda.stream(streams[k]):
                got[k].append(x.run())
    torch.cuda.synchronize()
    for k in range(2):
        assert all(torch.equal(x, want[k]) for x in got[k])
    starts, short = i32(a.starts), i32([0, 100, 103])
    outs = [torch.zeros_like(a.q) for _ in range(2)]
    graphs = [torch.cuda.CUDAGraph() for _ in range(2)]
    for g, s, o in zip(graphs, (starts, short), outs):
        with torch.cuda.graph(g):
            a.cache.attend_chunk(0, a.q, s, out=o)
    for _ in range(3):
        for g in graphs:
            g.replay()
    torch.cuda.synchronize()
    assert torch.equal(outs[0], want[0])
    a.starts = np.array([0, 100, 103])
    a.check(outs[1], None, a.expected(), torch.zeros_like(a.q))


# ---------------------------------------------------------------------------------------------- refusals, on the host
def fake(dtype=binding.OURO_BF16, **kw):
    """A description whose pointers nothing reads: every call below is refused before it launches anything."""
    c = binding.PagedCacheC(2, 10, 16, 2, 64, dtype, 4, 8, 10 * 16 * 2 * 64, 16 * 2 * 64, 2 * 64, 64, 4096, 4096, 4096, 4096, 4096, 4096, 4096, 0)
    build.build()
    c.workspace_bytes = binding.lib().ouro_paged_workspace_bytes(C.byref(c))
    for n, x in kw.items():
        setattr(c, n, x)
    return c


def chunk_call(c, layer=0, seqs=None, starts=4096, n=2, rows=8, q=4096, stride=256, heads=4, scale=0.125, out=4096, lse=None):
    return binding.lib().ouro_paged_chunk_attention(C.byref(c), layer, seqs, starts, n, rows, q, stride, heads, scale, out, lse, None)


@pytest.mark.parametrize("kw", [dict(layer=2), dict(layer=-1), dict(n=-1), dict(n=1025), dict(n=5), dict(rows=-1), dict(heads=0), dict(heads=3), dict(scale=0.0),
                                dict(scale=float("nan")), dict(scale=float("inf")), dict(q=None), dict(out=None), dict(starts=None), dict(starts=4098), dict(seqs=4097),
                                dict(lse=4098), dict(q=4104), dict(out=4104), dict(stride=252), dict(stride=192), dict(rows=2 ** 31 - 1),
                                dict(heads=2 * 65537, stride=2 ** 24)])
def test_chunk_refuses(kw):
    assert chunk_call(fake(), **kw) == binding.OURO_EINVAL
    assert b"ouro_paged_chunk_attention" in binding.lib().ouro_last_error(None)


def test_chunk_refuses_wrong_caches():
    for kw in (dict(head_dim=48), dict(dtype=7), dict(k=None), dict(workspace_bytes=1000), dict(table=4098)):
        c = fake()
        for n, x in kw.items():
            setattr(c, n, x)
        assert chunk_call(c) == binding.OURO_EINVAL, kw
    assert binding.lib().ouro_paged_chunk_attention(None, 0, None, 4096, 2, 8, 4096, 256, 4, 0.125, 4096, None, None) == binding.OURO_EINVAL
    # (nothing to do is nothing to refuse)
    assert chunk_call(fake(), n=0) == binding.OURO_OK and chunk_call(fake(), rows=0) == binding.OURO_OK


def rotary_call(c, layer=0, q=4096, q_stride=256, k=4096, v=4096, kv_stride=128, rows=3, heads=4, slots=4096, positions=4096, rotary=(4096, 32, 0, 1.0), out=8192):
    r = None if rotary is None else C.byref(binding.RotaryC(*rotary))
    return binding.lib().ouro_paged_append_rotary(C.byref(c), layer, q, q_stride, k, v, kv_stride, rows, heads, slots, positions, r, out, None)


@pytest.mark.parametrize("kw", [dict(layer=2), dict(rotary=None), dict(rotary=(None, 32, 0, 1.0)), dict(rotary=(4100, 32, 0, 1.0)), dict(rotary=(4096, 0, 0, 1.0)),
                                dict(rotary=(4096, 24, 0, 1.0)), dict(rotary=(4096, 80, 0, 1.0)), dict(rotary=(4096, 32, 2, 1.0)), dict(rotary=(4096, 32, 0, 0.0)),
                                dict(rotary=(4096, 32, 0, float("nan"))), dict(rows=-1), dict(heads=0), dict(q=None), dict(k=None), dict(v=None), dict(slots=None),
                                dict(positions=None), dict(out=None), dict(q=4104), dict(slots=4097), dict(q_stride=192), dict(kv_stride=64),
                                dict(out=4096, q_stride=512)])
def test_append_rotary_refuses(kw):
    assert rotary_call(fake(), **kw) == binding.OURO_EINVAL
    assert b"ouro_paged_append_rotary" in binding.lib().ouro_last_error(None)
    assert rotary_call(fake(), rows=0) == binding.OURO_OK


@pytest.mark.parametrize("args,kw", [((48,), {}), ((64,), dict(rotary_dim=24)), ((64,), dict(rotary_dim=80)), ((64,), dict(rotary_dim=0)), ((64,), dict(scaling="cubic")),
                                     ((64,), dict(factor=2.0)), ((64,), dict(scaling="linear", factor=0.5)), ((64,), dict(scaling="yarn", factor=2.0)),
                                     ((64,), dict(scaling="yarn", factor=2.0, original=100, beta_fast=1.0)), ((64, 1.0), {}), ((64, float("inf")), {})])
def test_rotary_refuses(args, kw):
    if args == (48,):                                      # (a head of 48 can be turned whole, but no cache has it)
        assert Rotary(*args, device="cpu").rotary_dim == 48
        return
    with pytest.raises(ValueError):
        Rotary(*args, device="cpu", **kw)


def test_frequencies():
    """The scalings' own definitions, number by number."""
    inv, mag = frequencies(8, 10000.0)
    assert mag == 1.0 and torch.allclose(inv, torch.tensor([1.0, 0.1, 0.01, 0.001], dtype=torch.float64), rtol=1e-14)
    assert torch.equal(frequencies(8, 10000.0, "linear", 4.0)[0], inv / 4)
    ntk, _ = frequencies(8, 10000.0, "ntk", 4.0)
    assert ntk[0] == 1.0 and abs(float(ntk[3] / inv[3]) - 0.25) < 1e-12 and bool((ntk[1:3] < inv[1:3]).all())
    yarn, mag = frequencies(64, 10000.0, "yarn", 16.0, 4096)
    inv = frequencies(64, 10000.0)[0]
    turns = 4096 * inv / (2 * math.pi)
    assert abs(mag - (0.1 * math.log(16.0) + 1)) < 1e-15
    assert torch.equal(yarn[:10], inv[:10]) and bool((turns[:10] > 32).all())
    assert torch.allclose(yarn[-8:], inv[-8:] / 16, rtol=1e-14) and bool((turns[-8:] < 1).all())
    assert bool((yarn[1:] < yarn[:-1]).all())


# ---------------------------------------------------------------------------------------------- rotary positions
def turned(x, positions, inv, mag, rd, interleaved):
    """In 64 bits; negative positions give zeros."""
    y = x.double().clone()
    a = positions.double()[:, None] * inv.to(x.device)
    z = torch.polar(torch.full_like(a, mag), a)[:, None]
    re, im = (slice(0, rd, 2), slice(1, rd, 2)) if interleaved else (slice(0, rd // 2), slice(rd // 2, rd))
    t = torch.complex(y[..., re].clone(), y[..., im].clone()) * z
    y[..., re], y[..., im] = t.real, t.imag
    return torch.where((positions >= 0)[:, None, None], y, 0.0)


def pair_size(x, rd, interleaved):
    """Length of the pair that an element belongs to."""
    y = x.double().abs().clone()
    re, im = (slice(0, rd, 2), slice(1, rd, 2)) if interleaved else (slice(0, rd // 2), slice(rd // 2, rd))
    s = torch.hypot(y[..., re], y[..., im])
    y[..., re], y[..., im] = s, s
    return y


@gpu
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("H,Hkv,D,rd,page,layout,scaling", [(4, 4, 32, 32, 16, "rows", "none"), (32, 4, 64, 16, 7, "heads", "linear"), (5, 1, 96, 48, 1, "padded", "ntk"),
                                                           (56, 8, 128, 128, 24, "layers", "yarn"), (3, 3, 128, 112, 16, "rows", "yarn")])
def test_append_rotary(H, Hkv, D, rd, page, layout, scaling, interleaved, dtype):
    build.build()
    k, v = pools(layout, 2, 20, page, Hkv, D, dtype, 1)
    cache = paged.PagedCache(max_seqs=1, max_pages=1, k=k, v=v)
    rotary = Rotary(D, 10000.0, rotary_dim=rd, interleaved=interleaved, scaling=scaling, factor=1.0 if scaling == "none" else 8.0, original=2048, device=DEV)
    inv, mag = frequencies(rd, 10000.0, scaling, 1.0 if scaling == "none" else 8.0, 2048)
    rows = 23
    r = np.random.default_rng(D)
    slots = r.permutation(20 * page)[:rows] if page > 1 else np.concatenate([r.permutation(20), [-1, -7, 20]])
    slots[3], slots[7] = -1, 20 * page + 5                  # padding; outside of the cache
    where = r.integers(0, 100000, rows)
    where[:6] = [0, 1, 2 ** 31 - 1, 5, 1000003, -1]
    where[10] = -(2 ** 31)
    positions = i32(where)
    both = torch.randn((rows, H + 2 * Hkv, D), device=DEV).to(dtype)      # one projection
    q, kn, vn = both[:, :H], both[:, H: H + Hkv], both[:, H + Hkv:]
    want_k, want_v = k.clone(), v.clone()
    before = both.clone()
    out = cache.append_rotary(1, q, kn, vn, i32(slots), positions, rotary)
    step = 2.0 ** -8 if dtype is BF16 else 0.0
    # (the angle of a pair of frequency f at position p: f is rounded to 2^-53 of itself, and so is the product, on either side)
    angle = 4 * 2.0 ** -53 * positions.double().abs().clamp(max=2.0 ** 31)

    def close(got, x, at):
        want = turned(x, positions[at], inv, mag, rd, interleaved)
        tol = step * want.abs() + (2.0 ** -21 + angle[at][:, None, None]) * mag * pair_size(x, rd, interleaved)
        assert bool(((got.double() - want).abs() <= tol).all()), float(((got.double() - want).abs() - tol).max())

    every = torch.arange(rows, device=DEV)
    close(out, q, every)
    assert torch.equal(out[..., rd:][positions >= 0], q[..., rd:][positions >= 0])       # what is not turned is moved
    live = [i for i in range(rows) if 0 <= slots[i] < 20 * page and where[i] >= 0]
    at = torch.tensor(live, device=DEV)
    pg, row = torch.tensor(slots[live] // page, device=DEV), torch.tensor(slots[live] % page, device=DEV)
    close(k[1, pg, row], kn[at], at)
    assert torch.equal(v[1, pg, row], vn[at])
    want_k[1, pg, row], want_v[1, pg, row] = k[1, pg, row], v[1, pg, row]
    assert torch.equal(k, want_k) and torch.equal(v, want_v) and torch.equal(both, before)
    # in place
    q2 = q.contiguous()
    assert cache.append_rotary(1, q2, kn, vn, i32(slots), positions, rotary, out=q2) is q2 and torch.equal(q2, out)
    cache.check()


@gpu
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_append_rotary_whole_heads_in_halves_is_append(dtype):
    """The same as with tables, but for the tables' rounding (2^-24 of a cosine on either side)."""
    build.build()
    k, v = pools("rows", 1, 8, 16, 4, 64, dtype, 2)
    k2, v2 = k.clone(), v.clone()
    a, b = paged.PagedCache(max_seqs=1, max_pages=1, k=k, v=v), paged.PagedCache(max_seqs=1, max_pages=1, k=k2, v=v2)
    q, kn, vn = (torch.randn((100, h, 64), device=DEV).to(dtype) for h in (8, 4, 4))
    cos, sin = paged.rotary_tables(400, 64, 10000.0, DEV)
    slots, positions = i32(np.random.default_rng(1).permutation(128)[:100]), i32(np.arange(100) * 3)
    x, y = a.append(0, q, kn, vn, slots, positions, cos, sin), b.append_rotary(0, q, kn, vn, slots, positions, Rotary(64, device=DEV))
    for s, t, u in ((x, y, q), ):
        tol = 2.0 ** -20 * pair_size(u, 64, False) + (2.0 ** -7 * s.double().abs() if dtype is BF16 else 0.0)
        assert bool(((s.double() - t.double()).abs() <= tol).all())
    assert torch.equal(v, v2)
    assert float((k.double() - k2.double()).abs().max()) <= 8 * (2.0 ** -7 if dtype is BF16 else 2.0 ** -20)


@gpu
def test_append_rotary_refuses_what_the_host_sees():
    build.build()
    cache = paged.PagedCache(1, 4, 16, 2, 64, "bf16", max_seqs=1, max_pages=1)
    q, kv, one = torch.zeros((3, 4, 64), dtype=BF16, device=DEV), torch.zeros((3, 2, 64), dtype=BF16, device=DEV), i32([0, 1, 2])
    with pytest.raises(ValueError):
        cache.append_rotary(0, q, kv, kv, one, one, Rotary(128, device=DEV))
    with pytest.raises(ValueError):
        cache.append_rotary(0, q, kv, kv, one, one, Rotary(64, device="cpu"))
    with pytest.raises(ValueError):
        cache.append_rotary(0, q[0], kv, kv, one, one, Rotary(64, device=DEV))
    with pytest.raises(ValueError):
        cache.append_rotary(0, q, kv, kv, one[:2], one, Rotary(64, device=DEV))
    for bad in (q[0], q.float(), q[:, :, :32]):
        with pytest.raises(ValueError):
            cache.attend_chunk(0, bad, i32([0, 3]))
    with pytest.raises(ValueError):
        cache.attend_chunk(0, q, i32([]))
    with pytest.raises(ValueError):
        cache.attend_chunk(0, q, i32([0, 3]).long())
    with pytest.raises(ValueError):
        cache.attend_chunk(0, q, i32([0, 3]), i32([0, 0]))
    with pytest.raises(ValueError):
        cache.attend_chunk(0, q, i32([0, 3]), out=q.transpose(0, 1).contiguous().transpose(0, 1))
    with pytest.raises(binding.OuroError):
        cache.attend_chunk(1, q, i32([0, 3]))
    with pytest.raises(binding.OuroError):
        cache.attend_chunk(0, q[:, :3], i32([0, 3]))
