"""Attention of chunks where a call's sizes are far from one another: many more new rows than a row of the table holds, short sequences in a table for very long ones, millions of heads.  Tolerances as in test_gpu_chunk.py."""
import pytest
import torch

from paper_2402_13720_b200 import paged
from test_gpu_chunk import BF16, F32, Call

gpu = pytest.mark.gpu


@gpu
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("chunks,H,Hkv,page,max_pages", [([(16, 46500)], 64, 8, 16, 1), ([(100, 24000), (40, 3)], 64, 8, 8, 16), ([(9, 17000), (64, 64)], 64, 1, 16, 4),
                                                         ([(0, 100000), (30, 70000), (64, 2)], 16, 8, 12, 6), ([(60, 166000)], 64, 8, 16, 4)])
def test_chunk_more_new_rows_than_there_is_room_for(chunks, H, Hkv, page, max_pages, dtype):
    """Rows that see no key give zeros, however many they are, and the others what they see."""
    c = Call(chunks, H, Hkv, 32, page, dtype, max_pages=max_pages)
    out = torch.full_like(c.q, 7.0)
    out, lse = c.run(want_lse=True, out=out)
    c.check(out, lse, c.expected())
    for i, (n, m) in enumerate(chunks):
        blind = max(m - n, 0)
        at = slice(int(c.starts[i]), int(c.starts[i]) + blind)
        assert bool((out[at] == 0).all()) and bool(torch.isneginf(lse[at]).all())
    c.cache.check()


@gpu
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("chunks,H,Hkv,page,max_pages", [([(1, 1), (3, 2), (5000, 4000)], 8, 8, 1024, 1 << 20), ([(2, 2), (0, 0), (7, 7), (900, 800), (1, 1)], 8, 4, 512, 1 << 20),
                                                         ([(1, 1)] * 200, 32, 32, 1024, 1 << 17), ([(5, 5), (30, 9)], 2, 2, 1 << 15, 1 << 15)])
def test_chunk_short_sequences_in_a_wide_table(chunks, H, Hkv, page, max_pages, dtype):
    c = Call(chunks, H, Hkv, 32, page, dtype, max_pages=max_pages)
    out, lse = c.run(want_lse=True, out=torch.full_like(c.q, 7.0))
    c.check(out, lse, c.expected())
    c.cache.check()


@gpu
@pytest.mark.parametrize("dtype,page", [(F32, 1), (BF16, 1), (BF16, 8)])
def test_chunk_millions_of_heads(dtype, page):
    """A text of one token gives its value, whichever of the heads; 2^24 and more are not all numbers of 32-bit floating point."""
    heads = (1 << 24) + 12345
    k, v = (torch.zeros((1, 1, page, heads, 32), dtype=dtype, device="cuda:0") for _ in range(2))
    v[0, 0, 0].copy_(torch.arange(heads, device="cuda:0")[:, None] % 251 + 1)
    cache = paged.PagedCache(max_seqs=1, max_pages=1, k=k, v=v)
    cache.table.zero_()
    cache.lens.fill_(1)
    out = torch.zeros((1, heads, 32), dtype=dtype, device="cuda:0")
    cache.attend_chunk(0, torch.ones_like(out), torch.tensor([0, 1], dtype=torch.int32, device="cuda:0"), out=out)
    cache.check()
    assert torch.equal(out[0], v[0, 0, 0])
