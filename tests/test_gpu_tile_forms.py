"""The kernels that the packed products run as, by their names in a trace, with the rules of
the sizes beside them in tests/test_tile_forms.py."""
import pytest
import torch
from torch.profiler import ProfilerActivity, profile

import paper_2604_01622_amd as ec

pytestmark = pytest.mark.gpu


def traced_step(n, d, E, h, k, dtype):
    """Template arguments of the products of one training step, by kernel template."""
    torch.manual_seed(n)
    w = 1.0 / d ** 0.5
    draw = lambda *s: (torch.randn(s, device="cuda") * w).to(dtype)   # noqa: E731
    X = torch.randn((n, d), device="cuda").to(dtype)
    layer = ec.TcLayer(X, draw(E, d), draw(E, h, d), draw(E, h, d), draw(E, d, h), [0, n], [n], k,
                       training=True)
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
