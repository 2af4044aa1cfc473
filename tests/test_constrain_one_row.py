"""Rules for a single row of logits: where its arguments' next rows would lie does not matter."""
import pytest
import torch

from paper_2402_13720_b200 import binding, build
from paper_2402_13720_b200.scores import allowed_words, constrain_logits
from test_gpu_constrain import call

gpu = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("kw", [dict(bias=4096, bias_stride=1), dict(allowed=4096, allowed_stride=1), dict(bias=4096, bias_stride=99, allowed=4096, allowed_stride=3)])
def test_strides_of_one_row_are_not_looked_at(kw):
    # (without a GPU the call ends at the launch; with one it is not made: the addresses are none)
    if torch.cuda.is_available():
        pytest.skip("the launch would be made")
    assert call(rows=1, **kw) != binding.OURO_EINVAL
    assert call(rows=2, **kw) == binding.OURO_EINVAL


@gpu
def test_one_row_of_columns():
    build.build()
    x = torch.randn((1, 300), device=DEV)
    bias = torch.randn((300, 1), device=DEV).T              # one row, whose next would begin an element further
    mask = torch.rand((1, 300), device=DEV) < 0.5
    words = allowed_words(mask).view(-1, 1).clone().T
    assert bias.stride() == (1, 1) and words.stride() == (1, 1)
    got = constrain_logits(x, bias=bias, allowed=words)
    assert torch.equal(got, torch.where(mask, x + bias, -float("inf")))
