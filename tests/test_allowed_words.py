"""Masks as words: whatever type truth values come in."""
import pytest
import torch

from paper_2402_13720_b200.scores import allowed_words


@pytest.mark.parametrize("dtype", [torch.bool, torch.uint8, torch.int32, torch.float32])
def test_truth_values_of_any_type(dtype):
    g = torch.Generator().manual_seed(1)
    mask = torch.rand((3, 77), generator=g) < 0.5
    values = mask.to(dtype) if dtype is torch.bool else torch.where(mask, torch.tensor(255 if dtype is torch.uint8 else 2), torch.tensor(0)).to(dtype)
    assert torch.equal(allowed_words(values), allowed_words(mask))


@pytest.mark.parametrize("vocab", [1, 31, 32, 33, 64])
def test_bits(vocab):
    mask = torch.arange(vocab) % 3 == 0
    words = allowed_words(mask)
    assert words.shape == (-(-vocab // 32),)
    assert [bool(int(words[i // 32]) >> (i % 32) & 1) for i in range(vocab)] == mask.tolist()
