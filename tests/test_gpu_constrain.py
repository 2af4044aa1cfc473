"""Rules on rows of logits (penalties, biases, grammar masks) against a plain implementation in 64 bits.

Tolerance, from the arithmetic (fixed before the first run): a quotient or product, a product and sum, a difference and a sum, each rounded to 2^-24 of a number
no larger than the sum of the parts' sizes: 2^-22 of that sum; bf16 then rounds once, half a step, 2^-8 of the result."""
import ctypes as C

import numpy as np
import pytest
import torch

from paper_2402_13720_b200 import binding, build, scores
from paper_2402_13720_b200.scores import allowed_words, constrain_logits

gpu = pytest.mark.gpu
DEV = "cuda:0"
F32, BF16 = torch.float32, torch.bfloat16


def expected(x, tokens=None, lens=None, repetition=None, presence=None, frequency=None, bias=None, mask=None):
    """Row by row in 64 bits; also the parts' sizes."""
    y, size = x.double().clone(), x.double().abs().clone()
    rows, vocab = x.shape
    if tokens is not None:
        for r in range(rows):
            n = tokens.shape[1] if lens is None else max(0, min(int(lens[r]), tokens.shape[1]))
            t = tokens[r, :n].long()
            t, c = t[(t >= 0) & (t < vocab)].unique(return_counts=True)
            rep, pres, freq = (none if v is None else float(v[r]) for v, none in ((repetition, 1.0), (presence, 0.0), (frequency, 0.0)))
            z = y[r, t]
            y[r, t] = torch.where(z > 0, z / rep, z * rep) - (freq * c + pres)
            size[r, t] = z.abs() * max(abs(rep), 1 / abs(rep)) + (abs(freq) * c + abs(pres))
    if bias is not None:
        y = y + bias.double()
        size = size + bias.double().abs()
    if mask is not None:
        y = torch.where(mask, y, torch.full_like(y, -float("inf")))
    return y, size


def close(got, want):
    y, size = want
    a = got.double()
    assert bool((torch.isnan(a) == torch.isnan(y)).all())
    inf = torch.isinf(y)
    assert torch.equal(a[inf], y[inf])
    ok = torch.isfinite(y)
    tol = 2.0 ** -22 * size + (2.0 ** -8 * y.abs() if got.dtype is BF16 else 0.0)
    assert bool(((a - y).abs() <= tol)[ok].all()), float(((a - y).abs() - tol)[ok].max())


def make(rows, vocab, dtype, width, seed, mean=0.0):
    g = torch.Generator(device=DEV).manual_seed(seed)
    x = (3 * torch.randn((rows, vocab), device=DEV, generator=g) + mean).to(dtype)
    kw = dict(tokens=(vocab * torch.rand((rows, width), device=DEV, generator=g) ** 5).int().clamp(max=vocab - 1),
              lens=torch.randint(0, width + 1, (rows,), device=DEV, generator=g).int(),
              repetition=1 + torch.rand(rows, device=DEV, generator=g), presence=torch.rand(rows, device=DEV, generator=g) - 0.3,
              frequency=torch.rand(rows, device=DEV, generator=g))
    return x, kw, g


@gpu
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,vocab,width", [(1, 1, 1), (1, 31, 5), (3, 33, 40), (5, 1000, 7), (2, 4097, 3000), (1, 32000, 411), (7, 50257, 1), (24, 64000, 700),
                                              (130, 8191, 33), (600, 8200, 20)])
@pytest.mark.parametrize("bias,mask", [(None, None), ("shared", "rows"), ("rows", "shared"), (None, "rows")])
def test_constrain(rows, vocab, width, bias, mask, dtype):
    build.build()
    x, kw, g = make(rows, vocab, dtype, width, vocab + width)
    b = None if bias is None else torch.randn((rows, vocab) if bias == "rows" else (vocab,), device=DEV, generator=g)
    m = None if mask is None else torch.rand((rows, vocab) if mask == "rows" else (vocab,), device=DEV, generator=g) < 0.6
    keep = x.clone()
    got = constrain_logits(x, **kw, bias=b, allowed=None if m is None else allowed_words(m))
    close(got, expected(x, **kw, bias=b, mask=m))
    assert torch.equal(x, keep) and got.dtype is dtype
    # without penalties
    close(constrain_logits(x, bias=b, allowed=None if m is None else allowed_words(m)), expected(x, bias=b, mask=m))
    # in place
    assert constrain_logits(x, **kw, bias=b, allowed=None if m is None else allowed_words(m), out=x) is x and torch.equal(x, got)


@gpu
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("which", ["repetition", "presence", "frequency", "lens", "none"])
def test_constrain_arguments_alone(which, dtype):
    build.build()
    x, kw, _ = make(5, 3001, dtype, 90, 4)
    kw = {"tokens": kw["tokens"], **({which: kw[which]} if which != "none" else {})}
    close(constrain_logits(x, **kw), expected(x, **kw))


@gpu
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("skew_in,skew_out", [(0, 0), (1, 1), (3, 3), (1, 2), (0, 5), (7, 7)])
def test_constrain_rows_at_any_address(skew_in, skew_out, dtype):
    """Logits, outputs, biases, masks and histories that are parts of larger tensors; what lies around the output stays."""
    build.build()
    rows, vocab = 6, 2500
    x, kw, g = make(rows, vocab, dtype, 50, 8)
    wide = torch.full((rows, vocab + 13), 9.0, device=DEV, dtype=dtype)
    wide[:, skew_in: skew_in + vocab] = x
    space = torch.full((rows, vocab + 29), 7.0, device=DEV, dtype=dtype)
    out = space[:, skew_out: skew_out + vocab]
    b = torch.randn((rows, vocab + 5), device=DEV, generator=g)[:, 3: 3 + vocab]
    m = torch.rand((rows, vocab), device=DEV, generator=g) < 0.5
    words = torch.full((rows, (vocab + 31) // 32 + 4), -1, dtype=torch.int32, device=DEV)
    words[:, 1: -3] = allowed_words(m)
    kw["tokens"] = torch.nn.functional.pad(kw["tokens"], (3, 2))[:, 3: -2]
    got = constrain_logits(wide[:, skew_in: skew_in + vocab], **kw, bias=b, allowed=words[:, 1: -3], out=out)
    close(got, expected(x, **kw, bias=b, mask=m))
    assert bool((space[:, :skew_out] == 7.0).all()) and bool((space[:, skew_out + vocab:] == 7.0).all())
    # one row of each for all
    one = {"tokens": kw["tokens"][:1].expand(rows, -1)}
    close(constrain_logits(x, **one, bias=b[0].expand(rows, -1), allowed=words[:1, 1: -3].expand(rows, -1)), expected(x, **one, bias=b[0], mask=m[0]))


@gpu
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_constrain_what_is_no_number(dtype):
    build.build()
    x, kw, g = make(4, 1000, dtype, 30, 3)
    inf, nan = float("inf"), float("nan")
    x[0, 5], x[0, 6], x[0, 7] = inf, -inf, nan
    kw["tokens"][0, :3] = torch.tensor([5, 6, 7], device=DEV)
    kw["lens"][0] = 30
    m = torch.ones((4, 1000), dtype=torch.bool, device=DEV)
    m[0, 7] = False                                         # not allowed, whatever it was
    m[1] = False                                            # nothing is allowed
    x[2] = torch.finfo(dtype).min                           # the type's lowest value
    x[3] = -inf
    got = constrain_logits(x, **kw, allowed=allowed_words(m))
    assert float(got[0, 5]) == inf and float(got[0, 6]) == -inf and float(got[0, 7]) == -inf
    assert bool(torch.isneginf(got[1]).all()) and bool(torch.isneginf(got[3]).all())
    want, size = expected(x, **kw, mask=m)
    seen = torch.zeros(1000, dtype=torch.bool, device=DEV)
    seen[kw["tokens"][2, : int(kw["lens"][2])].long()] = True
    assert torch.equal(got[2][~seen], x[2][~seen])          # untouched
    assert bool((got[2][seen] <= x[2][seen]).all())         # -inf where 32 bits or the type end
    close(got[:2], (want[:2], size[:2]))
    x[0, 9] = nan
    kw["tokens"][0, 3] = 9
    assert bool(torch.isnan(constrain_logits(x, **kw)[0, 9]))


@gpu
def test_constrain_histories():
    """Ids outside the vocabulary, lengths beyond the width or below 0, a token that is there seventy thousand times."""
    build.build()
    x, kw, g = make(4, 300, F32, 70000, 6)
    kw["tokens"][0, :] = 17
    kw["tokens"][1, ::2] = -1
    kw["tokens"][1, 1::4] = 300
    kw["tokens"][2, 5] = 2 ** 31 - 1
    kw["tokens"][2, 6] = -(2 ** 31)
    kw["lens"] = torch.tensor([70000, 2 ** 31 - 1, 100, -3], dtype=torch.int32, device=DEV)
    close(constrain_logits(x, **kw), expected(x, **kw))
    got = constrain_logits(x, tokens=kw["tokens"][:, :0], lens=torch.zeros(4, dtype=torch.int32, device=DEV))
    assert torch.equal(got, x)
    assert constrain_logits(x[:0]).shape == (0, 300)


@gpu
def test_constrain_captured():
    build.build()
    x, kw, g = make(9, 5000, BF16, 60, 2)
    out = torch.empty_like(x)
    constrain_logits(x, **kw, out=out)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        constrain_logits(x, **kw, out=out)
    x2, kw2, _ = make(9, 5000, BF16, 60, 5)
    x.copy_(x2)
    for n in kw:
        kw[n].copy_(kw2[n])
    graph.replay()
    torch.cuda.synchronize()
    close(out, expected(x, **kw))


@gpu
def test_constrain_rows_beyond_32_bit_offsets():
    build.build()
    rows, vocab = 70000, 32000                              # 2.2e9 logits
    x = torch.zeros((rows, vocab), dtype=BF16, device=DEV)
    x[-3:] = torch.randn((3, vocab), device=DEV)
    y = constrain_logits(x, tokens=torch.full((rows, 2), 11, dtype=torch.int32, device=DEV), frequency=torch.ones(rows, device=DEV))
    want = x[-3:].clone()
    want[:, 11] = (want[:, 11].float() - 2).to(BF16)
    assert torch.equal(y[-3:], want) and float(y[30000, 11]) == -2.0 and int((y[:-3] != 0).sum()) == rows - 3


@gpu
def test_constrain_then_scores():
    """What the scores make of constrained logits: the best allowed tokens, and none that is banned."""
    build.build()
    x, kw, g = make(6, 4000, F32, 100, 1)
    m = torch.rand((6, 4000), device=DEV, generator=g) < 0.01
    m[:, 3] = True
    s = scores.token_logprobs(constrain_logits(x, **kw, allowed=allowed_words(m)), None, 8)
    want = torch.log_softmax(expected(x, **kw, mask=m)[0], -1).sort(-1, descending=True)
    assert bool(m.gather(1, s.top_ids.long()).all())
    assert float((s.top_logprobs.double() - want.values[:, :8]).abs().max()) < 1e-4


@gpu
def test_constrain_refuses_tensors():
    build.build()
    x, kw, _ = make(4, 100, F32, 10, 1)
    for bad in (dict(kw, tokens=kw["tokens"].long()), dict(kw, tokens=kw["tokens"][:3]), dict(kw, tokens=kw["tokens"][0]), dict(kw, lens=kw["lens"].long()),
                dict(kw, lens=kw["lens"][:3]), dict(kw, presence=kw["presence"].double()), dict(kw, presence=kw["presence"].cpu()), dict(lens=kw["lens"]),
                dict(repetition=kw["repetition"]), dict(bias=torch.zeros(99, device=DEV)), dict(bias=torch.zeros((3, 100), device=DEV)),
                dict(bias=torch.zeros(100, device=DEV, dtype=BF16)), dict(allowed=torch.zeros(3, dtype=torch.int32, device=DEV)),
                dict(allowed=torch.zeros(4, dtype=torch.int64, device=DEV)), dict(out=torch.zeros((4, 101), device=DEV)), dict(out=x.to(BF16)),
                dict(out=torch.zeros((100, 4), device=DEV).T)):
        with pytest.raises(ValueError):
            constrain_logits(x, **bad)
    for bad in (x[0], x.half(), x.cpu(), x.T):
        with pytest.raises(ValueError):
            constrain_logits(bad)


def call(dtype=binding.OURO_F32, logits=4096, stride=100, rows=2, vocab=100, tokens=4096, token_stride=10, width=10, lens=4096, rep=4096, pres=4096, freq=4096,
         bias=None, bias_stride=0, allowed=None, allowed_stride=0, out=8192, out_stride=100):
    build.build()
    return binding.lib().ouro_constrain_logits(logits, dtype, stride, rows, vocab, tokens, token_stride, width, lens, rep, pres, freq, bias, bias_stride, allowed,
                                               allowed_stride, out, out_stride, None)


@pytest.mark.parametrize("kw", [dict(dtype=2), dict(rows=-1), dict(rows=2 ** 24 + 1), dict(vocab=0), dict(vocab=2 ** 28 + 1), dict(rows=2 ** 24, vocab=2 ** 20, stride=2 ** 20, out_stride=2 ** 20),
                                dict(logits=None), dict(out=None), dict(logits=4098), dict(out=8194), dict(dtype=binding.OURO_BF16, out=8193), dict(stride=99),
                                dict(out_stride=99), dict(logits=8192, stride=104), dict(tokens=4098), dict(lens=4097), dict(width=-1), dict(token_stride=9),
                                dict(tokens=None), dict(tokens=None, lens=None, rep=None, pres=None), dict(bias=4096, bias_stride=99), dict(bias=4098),
                                dict(allowed=4096, allowed_stride=3), dict(allowed=4097)])
def test_constrain_refuses(kw):
    assert call(**kw) == binding.OURO_EINVAL
    assert b"ouro_constrain_logits" in binding.lib().ouro_last_error(None)


def test_constrain_nothing_to_do():
    assert call(rows=0) == binding.OURO_OK


def test_allowed_words():
    m = torch.zeros((3, 70), dtype=torch.bool)
    m[0, 0] = m[0, 31] = m[0, 32] = m[1, 69] = True
    w = allowed_words(m)
    assert w.tolist() == [[-(2 ** 31) + 1, 1, 0], [0, 0, 32], [0, 0, 0]] and w.dtype is torch.int32
    assert allowed_words(m[1]).tolist() == [0, 0, 32]
