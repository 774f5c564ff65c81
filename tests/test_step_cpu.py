"""What a decode model refuses before it touches a device (no GPU)."""
import pytest

from paper_2609_13592_amd.step import DecodeModel, Dims


@pytest.mark.parametrize("top,first,last", [(3, 2, 2), (1, 1, 1), (4, -1, 2), (4, 1, -1), (2, 3, None),
                                            (2, None, 3), (-1, None, None)])
def test_blocks_that_do_not_fit_are_refused(top, first, last):
    dims = Dims(layers=1, d=256, hq=4, hkv=2, hd=128, ffn=384, vocab=100)
    with pytest.raises(ValueError):
        DecodeModel(0, dims, 1, 4, 0, {}, {}, top_blocks=top, first_blocks=first, last_blocks=last)
