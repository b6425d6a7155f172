"""A few-token decoder whose weights are exchanged or moved between its calls."""
import pytest
import torch

import paper_2604_01622_amd as ec

pytestmark = pytest.mark.gpu

N, D, E, H = 9, 128, 6, 64


def normal(seed, shape):
    t = torch.randn(shape, generator=torch.Generator().manual_seed(seed)) * shape[-1] ** -0.5
    return t.to(torch.bfloat16).cuda()


@pytest.mark.parametrize("mx", [False, True])
def test_exchanged_and_moved(mx):
    held = ec.mx_quantize if mx else (lambda t: t)
    X = normal(0, (N, D)) * 8
    Wg = normal(1, (E, D))
    sets = [[held(normal(s + n, shape)) for n, shape in enumerate(((E, H, D), (E, H, D), (E, D, H)))]
            for s in (10, 20)]
    dec = ec.TcDecoder(Wg, *sets[0], 2, max_tokens=N)
    want = [ec.tc_decode(X, Wg, *W, 2) for W in sets]
    torch.cuda.synchronize()
    assert not torch.equal(want[0][0], want[1][0])
    for n in (0, 1, 0, 1):
        dec.W1, dec.W3, dec.W2 = sets[n]
        got = dec.forward(X)
        assert all(torch.equal(a, b) for a, b in zip(got, want[n]))
    for t in sets[1]:                           # elsewhere, the old places overwritten
        for part in (t if mx else (t,)):
            old, part.data = part.data, part.data.clone()
            old.view(torch.uint8).fill_(255)
    got = dec.forward(X)
    assert all(torch.equal(a, b) for a, b in zip(got, want[1]))
