"""A problem description keeps group offsets and capacities of its own (CPU only): a caller
may reuse the arrays it passed while a planned layer is between its forward and backward."""
import numpy as np
import pytest
import torch

import paper_2604_01622_amd as ec
from paper_2604_01622_amd import binding


def test_arrays_may_be_reused():
    off, cap = np.array([0, 100, 256], dtype=np.int32), np.array([100, 156], dtype=np.int32)
    P = binding.Problem(256, 128, 8, 64, off, cap, 1.0, torch.bfloat16)
    saved = ec.lib().ec_tc_saved_size(P.ref, 2)
    off[1], cap[:] = 3, 1
    assert [P.c.group_offsets[i] for i in range(3)] == [0, 100, 256]
    assert [P.c.capacity[i] for i in range(2)] == [100, 156]
    assert ec.lib().ec_tc_saved_size(P.ref, 2) == saved


def test_any_layout_of_the_arrays():
    wide = np.arange(12, dtype=np.int64).reshape(3, 4)
    for off in ([0, 4, 8], (0, 4, 8), wide[:, 0], np.array([0, 4, 8], dtype=np.int32),
                torch.tensor([0, 4, 8])):
        P = binding.Problem(8, 64, 4, 64, off, np.array([4, 4]), 1.0, torch.float32)
        assert [P.c.group_offsets[i] for i in range(3)] == [0, 4, 8] and P.K == 8
    read_only = np.array([4, 4], dtype=np.int32)
    read_only.flags.writeable = False
    assert binding.Problem(8, 64, 4, 64, [0, 4, 8], read_only, 1.0, torch.float32).K == 8


@pytest.mark.parametrize("off,cap", [([0, 8], [4, 4]), ([0, 4, 8], [4]), ([0], [8]), ([8], [8]),
                                     ([0, 8], [[8]]), ([[0, 8]], [8])])
def test_one_more_offset_than_capacities(off, cap):
    """The library takes the group count from the capacities and reads one offset more."""
    with pytest.raises(ec.ECError, match="group_offsets"):
        binding.Problem(8, 64, 4, 64, off, cap, 1.0, torch.float32)
