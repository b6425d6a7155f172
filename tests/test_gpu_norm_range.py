"""The norm's backward pass at the ends of fp32's range, against the float64 oracle.

With u = 2^-24 (a rounding's half step in fp32) and b the storage type's: dx is off by
200 u (r |g| + r^3 |h| mean|g h|), as for ordinary rows, and its own rounding; where the values
that r multiplies are subnormal, a rounding is off by 2^-150 instead, times r^2 at most.
"""
import numpy as np
import pytest
import torch

from oracle import ec_ref as ref
import paper_2604_01622_amd as ec

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
DTYPES = (torch.bfloat16, torch.float32)
# every layout of a row: elements, one to four pieces a lane, unaligned pieces, dw in LDS
WIDTHS = [3, 64, 131, 2048, 4100, 8192, 12001, 16384]


def f64(t):
    return t.detach().double().cpu().numpy()


def half(dtype):
    return 2.0 ** -8 if dtype == torch.bfloat16 else U


def normal(seed, shape):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("d", WIDTHS)
@pytest.mark.parametrize("eps", [2.0 ** -149, 2.0 ** -130, 2.0 ** -127])
def test_rows_of_zeros_with_a_subnormal_eps(d, dtype, eps):
    """r = eps^-1/2 is up to 2^74.5, its square past fp32's range: dx = r g is not."""
    H = torch.zeros((3, d), dtype=dtype, device="cuda")
    w = (1 + 0.2 * normal(1, (d,))).to(dtype).cuda()
    dY, dH = (normal(n, (3, d)).to(dtype).cuda() for n in (2, 3))
    want, want_w = ref.rms_norm_backward_ref(f64(dY), f64(H), f64(w), eps)
    assert np.all(np.isfinite(want)) and np.all(want_w == 0)
    for add in (None, dH):
        dX, dw = ec.rms_norm_backward(dY, H, w, eps, dH=add)
        total = want if add is None else want + f64(add)
        assert np.all(np.abs(f64(dX) - total) <= 200 * U * np.abs(want) + half(dtype) * np.abs(total))
        assert bool((dw == 0).all())
    Y = ec.rms_norm(H, w, eps)
    assert bool((Y == 0).all())


@pytest.mark.parametrize("dtype", DTYPES)
def test_rows_beside_a_subnormal_eps(dtype):
    """Rows whose mean square is of the eps's own size, so that r^2 passes the range with h
    not zero."""
    d, eps = 512, 2.0 ** -129
    H = (2.0 ** -62 * normal(4, (5, d)).clamp(-3, 3)).to(dtype)
    H[0] = 0
    H = H.cuda()
    w = torch.ones(d, dtype=dtype, device="cuda")
    dY = normal(5, (5, d)).to(dtype).cuda()
    g, h = f64(dY), f64(H)
    want, _ = ref.rms_norm_backward_ref(g, h, f64(w), eps)
    dX, _ = ec.rms_norm_backward(dY, H, w, eps)
    r = 1.0 / np.sqrt((h * h).mean(-1, keepdims=True) + eps)
    size = r * np.abs(g) + r ** 3 * np.abs(h) * np.abs(g * h).mean(-1, keepdims=True)
    assert np.all(np.isfinite(f64(dX)))
    # squares of 2^-124 and less: each off by u of itself or 2^-150, an eps's 2^-129 by 2^-21 of
    # it at the most; r by half of that
    slack = 2.0 ** -21 + 200 * U
    assert np.all(np.abs(f64(dX) - want) <= slack * size + half(dtype) * np.abs(want))
