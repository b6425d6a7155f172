"""The weight's gradient of the norm over many rows, where a workgroup adds the most of them.

A workgroup of 1024 / TPR rows a step (one for rows of more than 512 pieces) out of 256 adds
rows / 256 terms of a column in sequence at most.  With u = 2^-24: a term is off by 55 u (its
row's factor 50 u, three products), the shares by rows / 256 and, of up to 16 rows a step, 16 u;
their sum by 16 lanes' 16 in sequence and the 16 lanes, 32 u: (120 + rows / 256) u of the terms'
magnitudes covers them.
"""
import pytest
import torch

import paper_2604_01622_amd as ec

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rows,d", [(6001, 4104), (9000, 4099), (20011, 2048), (70001, 64), (3001, 16384)])
def test_weight_gradient_of_many_rows(rows, d, dtype):
    gen = torch.Generator(device="cuda").manual_seed(rows)

    def normal(*shape):
        return torch.randn(shape, generator=gen, device="cuda")

    # means apart from zero, so that the partial sums grow with the rows
    H, dY = (normal(rows, d) + 1).to(dtype), (normal(rows, d) + 1).to(dtype)
    w = (1 + 0.2 * normal(d)).to(dtype)
    dX, dw = ec.rms_norm_backward(dY, H, w, 1e-6)
    h, g = H.double(), dY.double()
    terms = g * h / torch.sqrt((h * h).mean(1, keepdim=True) + 1e-6)
    off = (dw.double() - terms.sum(0)).abs() / terms.abs().sum(0)
    print(f"[dw] {rows} x {d} {dtype}: {float(off.max()) / U:.1f} u", flush=True)
    assert float(off.max()) <= (120 + rows / 256) * U
    again = ec.rms_norm_backward(dY, H, w, 1e-6)
    assert torch.equal(again[0], dX) and torch.equal(again[1], dw)
