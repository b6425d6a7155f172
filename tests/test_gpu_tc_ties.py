"""Experts of equal logits in token choice: the lower index is chosen, in inference as in
training, and both see the same scores to the bit."""
import numpy as np
import pytest
import torch

import paper_2604_01622_amd as ec

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("N", [50, 700, 9000])      # one wave row of tokens a workgroup and four
@pytest.mark.parametrize("E,distinct,k", [(17, 5, 3), (40, 10, 6), (64, 3, 4), (100, 7, 20),
                                          (256, 50, 8)])
def test_inference_and_training_choose_alike(E, distinct, k, N, dtype):
    """Every logit occurs in several experts, which lie in different lanes, and the k-th
    place falls among equal ones."""
    gen = torch.Generator().manual_seed(E + N)
    d, h = 128, 64
    X = torch.randn((N, d), generator=gen).to(dtype).cuda()
    rows = torch.randn((distinct, d), generator=gen).to(dtype)
    Wg = rows[torch.arange(E) % distinct].contiguous().cuda()
    W1 = (torch.randn((E, h, d), generator=gen) * 0.1).to(dtype).cuda()
    W2 = (torch.randn((E, d, h), generator=gen) * 0.1).to(dtype).cuda()
    off, cap = [0, N // 3, N], [N // 3, N - N // 3]
    S, G, slot, _, _ = ec.tc_route(X, Wg, off, cap, k)
    _, expert_rows = ec.tc_forward(X, Wg, W1, W1, W2, off, cap, k)
    _, _, counts, saved = ec.tc_train_forward(X, Wg, W1, W1, W2, off, cap, k)
    trained = saved[:N * E * 4].view(torch.float32).view(N, E)     # scores come first
    assert torch.equal(S, S[:, torch.arange(E, device="cuda") % distinct])
    assert torch.equal(S, trained)
    s = S.cpu().numpy()
    order = np.argsort(-s, axis=1, kind="stable")[:, :k]
    want = np.zeros((N, E), dtype=bool)
    np.put_along_axis(want, order, True, axis=1)
    assert np.array_equal(slot.cpu().numpy().T >= 0, want)
    assert np.array_equal(G.cpu().numpy() > 0, want)
    loads = np.stack([want[a:b].sum(0) for a, b in zip(off[:-1], off[1:])])
    assert np.array_equal(counts.cpu().numpy(), loads)
    assert np.array_equal(np.diff(expert_rows.cpu().numpy()), loads.sum(0))
