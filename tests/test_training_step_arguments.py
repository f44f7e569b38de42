"""Arguments of the clipping calls that the binding refuses before anything runs; no GPU needed."""
import pytest
import torch

from paper_2510_23938_b200 import binding


class OnDevice:
    """A tensor that says it is on a GPU; nothing reads what it points to."""

    is_cuda, dtype = True, torch.float32

    def data_ptr(self):
        return 4096


@pytest.mark.parametrize("types", [None, torch.zeros(2, dtype=torch.uint8)])
def test_an_output_needs_its_offsets(types):
    with pytest.raises(AssertionError, match="out_offsets"):
        binding._out_args(OnDevice(), None, None, types, 2)
    with pytest.raises(AssertionError, match="out_offsets"):
        binding._out_args(OnDevice(), torch.zeros(3, dtype=torch.int64), None, types, 2)
    with pytest.raises(AssertionError, match="out_offsets"):
        binding._out_args(OnDevice(), torch.zeros(2, dtype=torch.int32), None, types, 2)


def test_in_place_takes_no_output_arguments():
    for offsets, dtype in ((torch.zeros(2, dtype=torch.int64), None), (None, torch.float32)):
        with pytest.raises(AssertionError, match="in place"):
            binding._out_args(None, offsets, dtype, None, 2)
    assert binding._out_args(None, None, None, None, 2) == (None, None, -1)
