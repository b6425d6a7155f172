"""The kernels that the packed products run as, by their names in a trace, with the rules of
the sizes beside them in tests/test_tile_forms.py."""
import pytest
import torch
from torch.profiler import ProfilerActivity, profile

import paper_2604_01622_amd as ec
from test_gpu_tc_training import check_layer
from test_tile_forms import BF16_FORMS

pytestmark = pytest.mark.gpu


def traced_step(n, d, E, h, k, dtype, hs=0):
    """Template arguments of the products of one training step, by kernel template."""
    torch.manual_seed(n)
    w = 1.0 / d ** 0.5
    draw = lambda *s: (torch.randn(s, device="cuda") * w).to(dtype)   # noqa: E731
    X = torch.randn((n, d), device="cuda").to(dtype)
    shared = (draw(hs, d), draw(hs, d), draw(d, hs)) if hs else None
    layer = ec.TcLayer(X, draw(E, d), draw(E, h, d), draw(E, h, d), draw(E, d, h), [0, n], [n], k,
                       shared=shared, training=True)
    layer.forward()
    layer.backward(X)
    torch.cuda.synchronize()
    with profile(activities=[ProfilerActivity.CUDA]) as trace:
        layer.forward()
        layer.backward(X)
        torch.cuda.synchronize()
    names = {e.key for e in trace.key_averages()}
    return {tuple(x.strip() for x in name[name.index("<") + 1:name.index(">")].split(","))
            for name in names if "gemm" in name and "<" in name}


@pytest.mark.parametrize("n,d,E,h,k,dW2,dW13", [
    (1700, 512, 17, 512, 2, ("64", "128"), ("128", "128")),
    (300, 256, 3, 256, 2, ("64", "128"), ("64", "128")),
    (500, 256, 130, 256, 2, ("128", "128"), ("128", "128")),
])
def test_fp32_weight_gradients(n, d, E, h, k, dW2, dW13):
    forms = traced_step(n, d, E, h, k, torch.float32)
    print(sorted(forms), flush=True)
    # the last argument holds the options: 16 + 1 gathers dY (dW2), 16 + 2 X (dW1/dW3)
    assert {f[:2] for f in forms if f[-1] == "17"} == {dW2}
    assert {f[:2] for f in forms if f[-1] == "18"} == {dW13}


@pytest.mark.parametrize("size,packed,shared", BF16_FORMS)
def test_bf16_training_products(size, packed, shared):
    n, d, E, h, k, hs = size
    forms = traced_step(n, d, E, h, k, torch.bfloat16, hs)
    print(sorted(forms), flush=True)
    # arguments 0, 1: the tile; 10: the stage
    tiles = {}
    for f in forms:
        tiles.setdefault(int(f[10]), set()).add((int(f[0]), int(f[1])))
    assert [tiles[tag] for tag in range(15, 21)] == [{t} for t in packed]
    assert [tiles[tag] for tag in range(9, 13) if tag in tiles] == [{t} for t in shared]


@pytest.mark.parametrize("size", [f[0] for f in BF16_FORMS if f[0][0] > 20000])
def test_training_step_of_the_shared_forms(size):
    """The shared experts' products in the tiles that the sizes of the other tests do not
    take (192 and 256 rows, 128 rows of W2)."""
    n, d, E, h, k, hs = size
    check_layer([n], d, E, h, k, 0.0, torch.bfloat16, seed=n, hs=hs)
