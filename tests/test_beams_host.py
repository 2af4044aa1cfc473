"""What a beam decoder refuses before it touches the GPU."""
import pytest

from paper_2402_13720_b200 import synth
from paper_2402_13720_b200.beams import BeamDecoder


def decoder():
    d = object.__new__(BeamDecoder)                        # without a cache: nothing here gets that far
    d.m, d.beams, d.max_len = synth.ModelDesc(2, 128, 4, 2, 32, 256, 300, 64, "f32"), 4, 20
    return d


@pytest.mark.parametrize("prompt,new", [([], 4), ([1, 2], 0), ([1, 2], -1), ([1] * 17, 4), ([1, 300], 4), ([-1, 1], 4)])
def test_search_refuses(prompt, new):
    with pytest.raises(ValueError):
        decoder().search(prompt, new)


@pytest.mark.parametrize("prompt,cont", [([], [1]), ([1], []), ([], []), ([1] * 17, [1] * 4), ([300], [1]), ([1], [-1]), ([1], [2, 300])])
def test_score_refuses(prompt, cont):
    with pytest.raises(ValueError):
        decoder().score(prompt, cont)
