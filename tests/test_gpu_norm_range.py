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


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("d", WIDTHS)
def test_rows_past_the_range_of_their_squares(d, dtype):
    """A row whose sum of squares passes fp32's range is divided by infinity: Y = 0, so it gives
    dX = dH and nothing to dw, whatever the sum of weight dY H comes to."""
    H, dH = (normal(n, (4, d)).to(dtype).cuda() for n in (6, 7))
    w = (1 + 0.2 * normal(8, (d,))).to(dtype).cuda()
    dY = normal(9, (4, d)).to(dtype).cuda()
    ordinary, odd = [0, 2], [1, 3]
    want = ec.rms_norm(H, w)[ordinary]
    want_dX, _ = ec.rms_norm_backward(dY, H, w, dH=dH)
    rest = dY.clone()
    rest[odd] = 0
    _, want_dw = ec.rms_norm_backward(rest, H, w)
    H[odd] = 1e25
    dY[3] = 1e20                                 # the sum of weight dY H passes the range too
    Y = ec.rms_norm(H, w)
    assert bool((Y[odd] == 0).all()) and torch.equal(Y[ordinary], want)
    for add in (None, dH):
        dX, dw = ec.rms_norm_backward(dY, H, w, dH=add)
        assert torch.equal(dX[odd], torch.zeros_like(dX[odd]) if add is None else dH[odd])
        assert torch.equal(dw, want_dw)
    assert torch.equal(dX[ordinary], want_dX[ordinary])


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("d", WIDTHS)
def test_large_rows_up_to_the_bound(d, dtype):
    """A root mean square of 2^63.9 / sqrt(d), whose squares sum to just below 2^128."""
    rms = 2.0 ** 63.9 / np.sqrt(d)
    sign = torch.sign(normal(10, (2, d)))
    H = (rms * sign).to(dtype).cuda()
    assert float((H.double() ** 2).sum(1).max()) < 2.0 ** 128 * (1 - 2.0 ** -8)
    w = (1 + 0.2 * normal(11, (d,))).to(dtype).cuda()
    dY = normal(12, (2, d)).to(dtype).cuda()
    Y = ec.rms_norm(H, w, 1e-6)
    y = ref.rms_norm_ref(f64(H), f64(w), 1e-6)
    assert np.all(np.abs(f64(Y) - y) <= (half(dtype) + 50 * U) * np.abs(y))
    dX, dw = ec.rms_norm_backward(dY, H, w, 1e-6)
    g, h, wf = f64(dY), f64(H), f64(w)
    want, want_w = ref.rms_norm_backward_ref(g, h, wf, 1e-6)
    r = 1.0 / np.sqrt((h * h).mean(-1, keepdims=True) + 1e-6)
    size = r * np.abs(g * wf) + r ** 3 * np.abs(h) * np.abs(g * wf * h).mean(-1, keepdims=True)
    assert np.all(np.abs(f64(dX) - want) <= 200 * U * size + half(dtype) * np.abs(want))
    assert np.all(np.abs(f64(dw) - want_w) <= 120 * U * np.abs(g * h * r).sum(0))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("d", [64, 131, 4100, 16384])
def test_an_infinity_is_no_number_at_its_place(d, dtype):
    H, dH, dY = (normal(n, (3, d)).to(dtype).cuda() for n in (13, 14, 15))
    w = torch.ones(d, dtype=dtype, device="cuda")
    H[1, d // 3] = -float("inf")
    at = torch.zeros((3, d), dtype=torch.bool, device="cuda")
    at[1, d // 3] = True
    Y, (dX, dw) = ec.rms_norm(H, w), ec.rms_norm_backward(dY, H, w, dH=dH)
    assert torch.equal(torch.isnan(Y), at) and torch.equal(torch.isnan(dX), at)
    assert torch.equal(torch.isnan(dw), at[1]) and torch.equal(dX[1][~at[1]], dH[1][~at[1]])
