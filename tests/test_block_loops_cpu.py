"""Refusals of a decoding loop's calls that need no device."""
import torch

from test_blocks_cpu import OK, resize


def test_an_empty_batch_has_a_free_list_all_the_same():
    assert resize(B=0) == 0 and resize(B=0, count=None, c_out=None) == 0      # in place: nothing to do
    assert resize(B=0, count=None) == 1 and resize(B=0, c_out=None) == 1
    if not torch.cuda.is_available():
        assert resize(B=0, c_out=OK + 256) in (2, 3)      # its length is written elsewhere: by the device
