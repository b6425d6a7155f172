"""Eight bits with every kind of scale byte in the few-token layer's weights and tokens, codes and
scales made by hand: each finite code's value reaches Y as bf16 holds it.

A code is a multiple of 2^-9 of its scale with four leading bits, so bf16 holds it exactly from
the byte 3 (2^-133 is bf16's smallest step) up to 2^128.  Below, the nearest multiple of 2^-133, the
even one of two; from 2^128 on it is infinite; under the byte 255 no number.

The layers are made so that Y is one element times powers of two: one expert, silu(128) = 128,
ones elsewhere.  Y has the element's four bits, so it is compared exactly.  Through W1 the
element a goes through silu: exp(-a), whose argument's last bit is u |a| of it (u = 2^-24) and its
own error 2 u, sum, quotient and product; then Y's rounding, 2^-8.  Where exp(-a) passes 2^128, from
|a| = 88.72 on, a / (1 + exp(-a)) is 0 and the value left out is below 88.73 / 2^128.
"""
import numpy as np
import pytest
import torch

import paper_2604_01622_amd as ec

pytestmark = pytest.mark.gpu

ONE, P128 = 0x38, 0x70               # codes of 1 and 128
BYTES = [0, 1, 2, 3, 4, 50, 126, 127, 128, 200, 245, 246, 247, 248, 250, 253, 254, 255]
D, H = 192, 128
U, B = 2.0 ** -24, 2.0 ** -8


def hold(codes, scales):
    return ec.Mx(codes.to(torch.uint8).cuda().view(torch.float8_e4m3fn),
                 scales.to(torch.uint8).cuda().view(torch.float8_e8m0fnu))


def empty(*shape):
    """Codes of zero, scales of one."""
    return (torch.zeros(shape, dtype=torch.int64),
            torch.full((*shape[:-1], shape[-1] // 32), 127, dtype=torch.int64))


def elements(byte):
    """Values of the finite codes 0 to 126 under the scale `byte`."""
    codes = torch.arange(127, dtype=torch.uint8).view(torch.float8_e4m3fn)
    return codes.double().numpy() * 2.0 ** (byte - 127)


def layer(which, byte, f, N, sign):
    """X, W1, W3, W2 with the finite codes under the scale `byte` in one of them, times 2^f
    elsewhere; the tokens of X but the last are ordinary."""
    codes = torch.arange(127) + (128 if sign < 0 else 0)
    x, w1, w3, w2 = empty(N, D), empty(H, D), empty(H, D), empty(D, H)
    rows = torch.arange(127)
    w2[0][rows, rows] = ONE
    if which == "X":
        x[0][-1, :127], x[1][-1, :4] = codes, byte
        x[0][:, 128] = ONE
        w1[0][:, 128] = P128
        w3[0][rows, rows], w3[1][rows, rows // 32] = ONE, 127 + f
    else:
        x[0][:, 0], x[1][:, 0] = ONE, 127 + f
        x[0][:, 40] = ONE if which == "W1" else P128
        if which == "W1":
            w1[0][:127, 0], w1[1][:, 0] = codes, byte
            w3[0][:, 40] = ONE
        elif which == "W3":
            w1[0][:, 40] = ONE
            w3[0][:127, 0], w3[1][:, 0] = codes, byte
        else:
            w1[0][0, 40] = ONE
            w3[0][0, 0] = ONE
            w2[0][:] = 0
            w2[0][:127, 0], w2[1][:, 0] = codes, byte
    return [hold(*t) for t in (x, w1, w3, w2)]


def check(got, byte, f, which, sign):
    value = sign * elements(byte)
    if byte < 3:
        value = np.rint(value / 2.0 ** -133) * 2.0 ** -133
    if byte == 255:
        assert np.all(np.isnan(got))
        return
    fits = np.abs(value) < 2.0 ** 128
    assert fits.all() == (byte < 247)
    if which != "W2" and not fits.all():
        # an infinite element of a token, or of a hidden unit, meets zeros in every column of Y
        assert not np.any(np.isfinite(got))
        return
    assert not np.any(np.isfinite(got[~fits]))
    if which == "W1":
        a = value[fits] * 2.0 ** f
        want = a / (1 + np.exp(np.minimum(-a, 700)))
        slack = (B + 8 * U + 2 * U * np.abs(a)) * np.abs(want) + 88.73 * 2.0 ** -128
        off = np.abs(got[fits] - want) > slack
        assert not off.any(), (a[off], got[fits][off], want[off])
    else:
        assert np.array_equal(got[fits], 128 * value[fits] * 2.0 ** f)


@pytest.mark.parametrize("N", [1, 20, 40])
@pytest.mark.parametrize("which", ["X", "W1", "W3", "W2", "Ws1", "Ws3", "Ws2"])
def test_every_scale(which, N):
    Wg = torch.zeros((1, D), dtype=torch.bfloat16, device="cuda")
    nothing = [hold(*empty(*s)) for s in ((1, H, D), (1, H, D), (1, D, H))]
    shared = which.startswith("Ws")
    name = "W" + which[2] if shared else which
    for byte in BYTES:
        f = min(max(127 - byte, -100), 119)
        for sign in (1, -1):
            X, *W = layer(name, byte, f, N, sign)
            if shared:
                Y, _, gates = ec.tc_decode(X, Wg, *nothing, 1, shared=tuple(W))
            else:
                W = [ec.Mx(w.codes[None], w.scales[None]) for w in W]
                Y, _, gates = ec.tc_decode(X, Wg, *W, 1)
            got = Y.double().cpu().numpy()[:, :127]
            print(f"[scales] {which} byte {byte} N {N} sign {sign}", flush=True)
            check(got[-1], byte, f, name, sign)
            if name == "X":
                assert np.all(got[:-1] == 0)
            else:
                assert all(np.array_equal(g, got[-1], equal_nan=True) for g in got[:-1])
