"""The balance gradient in place of its scores: the same bits as beside them; buffers that
overlap otherwise are refused (CPU)."""
import ctypes

import numpy as np
import pytest
import torch

import paper_2604_01622_amd as ec
from paper_2604_01622_amd import binding


def problem(lens, E):
    off = np.concatenate([[0], np.cumsum(lens)])
    return binding.Problem(int(off[-1]), 64, E, 64, off, [0] * len(lens), 2.0, torch.float32)


def test_partial_overlap_is_refused():
    L, P = ec.lib(), problem([40, 60], 8)
    S, other = 1 << 20, ctypes.c_void_p(1 << 30)
    for at in (16, 100 * 8 * 4 - 16, -16, 16 - 100 * 8 * 4):
        st = L.ec_tc_balance_backward(P.ref, 2, S, other, other, S + at, None)
        assert st == 1 and "overlap" in L.ec_last_error().decode(), at


@pytest.mark.gpu
@pytest.mark.parametrize("E,k", [(8, 2), (37, 3), (64, 8), (100, 4), (190, 5), (253, 8), (256, 8)])
@pytest.mark.parametrize("lens", [[1], [15, 16, 17], [33, 0, 64, 65, 129], [16000, 900]])
def test_gradient_in_place(lens, E, k):
    """16 and 64 tokens a chunk (batches up to 16384 tokens and past), rows of whole 16-byte
    loads and others."""
    gen = torch.Generator().manual_seed(E + len(lens))
    S = torch.softmax(torch.randn((sum(lens), E), generator=gen), 1).cuda()
    P = problem(lens, E)
    _, counts = ec.tc_balance(S, P.off, k)
    dloss = torch.linspace(-1.0, 2.0, len(lens), device="cuda")
    want = [ec.tc_balance_backward(S, counts, dloss, P.off, k, 2.0) for _ in range(2)]
    st = ec.lib().ec_tc_balance_backward(P.ref, k, S.data_ptr(), counts.data_ptr(),
                                         dloss.data_ptr(), S.data_ptr(),
                                         torch.cuda.current_stream().cuda_stream)
    assert st == 0
    assert torch.equal(want[0], want[1]) and torch.equal(want[0], S)
