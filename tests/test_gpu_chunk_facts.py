"""What the header says of attention of chunks beside its formula: how many launches a call takes, and what infinities do."""
import pytest
import torch

from paper_2402_13720_b200 import binding
from test_gpu_chunk import BF16, DEV, F32, Call, i32

gpu = pytest.mark.gpu


@gpu
@pytest.mark.parametrize("dtype,page,one,two", [(F32, 1, 192, 193), (F32, 16, 192, 208), (BF16, 1, 192, 193), (BF16, 12, 192, 204), (BF16, 8, 320, 328), (BF16, 16, 320, 336)])
def test_launches(dtype, page, one, two):
    for room, launches in ((one, 1), (two, 2)):
        c = Call([(room, 5), (3, 3)], 4, 2, 64, page, dtype, max_pages=room // page)
        want = c.expected()
        before = binding.lib().ouro_kernel_launches()
        out, lse = c.run(want_lse=True)
        assert binding.lib().ouro_kernel_launches() - before == launches
        c.check(out, lse, want)


@gpu
@pytest.mark.parametrize("page", [16, 8, 20])
@pytest.mark.parametrize("D", [64, 96])
def test_infinite_keys_in_bf16(page, D):
    """A score of -inf is that of a key that is not there, and a token that has no other gives zeros; one of +inf leaves no distribution."""
    c = Call([(400, 150), (30, 30)], 4, 2, D, page, BF16)
    c.q[:, :, 3] = c.q[:, :, 3].abs() + 0.5
    j, pg, row = c.slots(0)
    at = torch.tensor([7, 260, 261, 399])
    c.k[0, torch.tensor(pg, device=DEV)[at], torch.tensor(row, device=DEV)[at], :, 3] = -float("inf")
    _, pg1, row1 = c.slots(1)
    c.k[0, torch.tensor(pg1, device=DEV), torch.tensor(row1, device=DEV), :, 3] = -float("inf")
    want = c.expected()
    assert bool(torch.isneginf(want[2][150:]).all()) and bool((want[0][150:] == 0).all()) and bool(torch.isfinite(want[0]).all())
    out, lse = c.run(want_lse=True)
    c.check(out, lse, want)
    c.k[0, pg[260], row[260], :, 3] = float("inf")
    out = c.run()
    assert bool(torch.isfinite(out[:10]).all()) and not bool(torch.isfinite(out[10:150]).any())        # position 260 is row 10


@gpu
def test_infinite_keys_in_f32():
    """No score of f32 is -inf: an infinity among queries and keys leaves no distribution."""
    c = Call([(300, 60)], 4, 2, 64, 16, F32)
    j, pg, row = c.slots(0)
    clean = c.run()
    keep = c.k[0, pg[250], row[250]].clone()
    for x in (float("inf"), -float("inf")):
        c.k[0, pg[250], row[250], :, 3] = x
        out = c.run()
        assert torch.equal(out[:10], clean[:10]) and not bool(torch.isfinite(out[10:]).any())
    c.k[0, pg[250], row[250]] = keep
    c.q[5, 1, 7] = float("inf")
    out = c.run()
    assert not bool(torch.isfinite(out[5, 1]).any())
    out[5, 1] = clean[5, 1]
    assert torch.equal(out, clean)
