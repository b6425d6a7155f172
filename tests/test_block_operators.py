"""The norm, the eight-bit layout and the few-token layer without a GPU: the oracle's formulas
against their definitions, automatic differentiation and differences, and the refusals of the
entry points, which happen on the host before anything is enqueued."""
import ctypes

import numpy as np
import pytest
import torch

from oracle import ec_ref as ref
import paper_2604_01622_amd as ec
from paper_2604_01622_amd import binding

EC_OK, EC_ERR_ARG, EC_ERR_SHAPE, EC_ERR_CAPACITY, EC_ERR_DTYPE, EC_ERR_ALIGN, EC_ERR_WORKSPACE = range(7)
FAKE = ctypes.c_void_p(1 << 20)       # aligned, never dereferenced: validation fails first
FAR = ctypes.c_void_p(1 << 30)
FARTHER = ctypes.c_void_p(1 << 31)
MISALIGNED = ctypes.c_void_p((1 << 20) + 8)


def at(n):
    return ctypes.c_void_p(n)


# ---- the oracle ----------------------------------------------------------------


def e4m3_numbers():
    """Every finite number of the format, from its definition: sign, four bits of exponent
    (bias 7), three of mantissa; exponent 15 with mantissa 7 is NaN."""
    out = [m * 2.0 ** -9 for m in range(8)]
    out += [(8 + m) * 2.0 ** (e - 10) for e in range(1, 16) for m in range(8) if (e, m) != (15, 7)]
    return np.array(out)


def test_e4m3_rounds_to_the_nearest_number():
    grid = e4m3_numbers()
    assert grid.max() == 448 and np.array_equal(ref.e4m3_ref(grid), grid)
    v = np.concatenate([np.random.default_rng(0).uniform(0, 448, 4000),
                        np.random.default_rng(1).uniform(0, 2.0 ** -5, 2000)])
    got = ref.e4m3_ref(v)
    assert np.all(np.isin(got, grid))
    best = np.abs(v[:, None] - grid).min(1)
    assert np.array_equal(np.abs(got - v), best)
    # halfway between neighbours: the one with an even mantissa
    mid = (grid[:-1] + grid[1:]) / 2
    even = np.where(np.arange(len(grid) - 1) % 2 == 0, grid[:-1], grid[1:])
    assert np.array_equal(ref.e4m3_ref(mid), even)
    assert np.array_equal(ref.e4m3_ref(-mid), -even)


def test_mx_scale_is_the_smallest_that_does_not_saturate():
    for top in (448.0, 448.5, 1.0, 0.875, 1.75, 1.7500001, 2.0 ** -100, 3e38, 2.0 ** -126):
        s = float(ref.mx_scale_ref(top))
        assert np.log2(s) == np.rint(np.log2(s)) and top <= 448 * s
        assert s == 2.0 ** -126 or top > 448 * s / 2
    assert ref.mx_scale_ref(0.0) == 2.0 ** -126
    assert ref.mx_scale_ref(448 * 2.0 ** -126) == 2.0 ** -126


def test_mx_codes_by_hand():
    X = np.zeros((1, 64))
    X[0, :4] = [448, -1, 0.4375, 1e-3]
    X[0, 32:35] = [896, 3.0, -17.0]
    codes, scales = ref.mx_quantize_ref(X)
    assert scales.tolist() == [[1.0, 2.0]]
    assert codes[0, :4].tolist() == [448, -1, 0.4375, 2.0 ** -9 * round(1e-3 * 512)]
    assert codes[0, 32:35].tolist() == [448, 1.5, -8.0]    # -8.5: halfway, to the even -8
    assert ref.mx_value_ref(codes, scales)[0, 34] == -16.0


@pytest.mark.parametrize("with_dH", [False, True])
def test_norm_gradients_against_autograd_and_differences(with_dH):
    rng = np.random.default_rng(3)
    H, w, dY, dH = (rng.standard_normal(s) for s in ((7, 12), (12,), (7, 12), (7, 12)))
    eps = 1e-2
    dH = dH if with_dH else None
    dX, dw = ref.rms_norm_backward_ref(dY, H, w, eps, dH)

    def total(H, w):
        y = H / torch.sqrt((H * H).mean(-1, keepdim=True) + eps) * w
        out = (y * torch.from_numpy(dY)).sum()
        return out if dH is None else out + (H * torch.from_numpy(dH)).sum()

    leaves = [torch.from_numpy(a.copy()).requires_grad_() for a in (H, w)]
    total(*leaves).backward()
    assert np.allclose(leaves[0].grad.numpy(), dX, rtol=1e-12, atol=1e-13)
    assert np.allclose(leaves[1].grad.numpy(), dw, rtol=1e-12, atol=1e-13)
    vH, vw, step = rng.standard_normal(H.shape), rng.standard_normal(w.shape), 1e-6
    up, dn = (float(total(torch.from_numpy(H + s * step * vH), torch.from_numpy(w + s * step * vw)))
              for s in (1, -1))
    want = float((dX * vH).sum() + (dw * vw).sum())
    assert (up - dn) / (2 * step) == pytest.approx(want, rel=1e-7)


def test_few_tokens_agree_with_token_choice():
    rng = np.random.default_rng(9)
    N, d, E, h, k = 13, 6, 5, 4, 3
    X, Wg, W1, W3, W2 = (rng.standard_normal(s) for s in
                         ((N, d), (E, d), (E, h, d), (E, h, d), (E, d, h)))
    shared = tuple(rng.standard_normal(s) for s in ((3, d), (3, d), (d, 3)))
    R = rng.standard_normal((N, d))
    Y, experts, gates = ref.tc_decode_ref(X, Wg, W1, W3, W2, k, 2.0, shared, R)
    want = ref.tc_forward_ref(X, Wg, W1, W3, W2, [0, N], k, [N], 2.0)
    assert np.allclose(Y, want["Y"] + ref.shared_ffn_ref(X, shared) + R, rtol=1e-12, atol=1e-12)
    for i in range(N):
        g = dict(zip(want["choice"][i], want["gate"][i]))
        assert np.allclose([g[j] for j in experts[i]], gates[i], rtol=1e-12)
        assert np.all(np.diff(gates[i]) <= 0)
    # equal logits: the lower index first
    Wg[3] = Wg[1]
    _, experts, _ = ref.tc_decode_ref(X, Wg, W1, W3, W2, E)
    assert all(list(e).index(3) == list(e).index(1) + 1 for e in experts)


# ---- refusals ------------------------------------------------------------------


def test_quantize_refusals():
    L = ec.lib()

    def call(dtype=1, rows=10, cols=64, X=FAKE, Q=FAR, s=FARTHER):
        return L.ec_mx_quantize(dtype, rows, cols, X, Q, s, None)

    assert call(dtype=2) == EC_ERR_DTYPE
    for rows, cols in ((-1, 64), (3, -32), (3, 63), (1 << 35, 32), (1 << 20, 1 << 20)):
        assert call(rows=rows, cols=cols) == EC_ERR_SHAPE
    for n in ("X", "Q", "s"):
        assert call(**{n: None}) == EC_ERR_ARG and call(**{n: MISALIGNED}) == EC_ERR_ALIGN
    assert call(Q=FAKE) == EC_ERR_ARG and call(s=FAR) == EC_ERR_ARG
    assert call(Q=at((1 << 20) + 1264)) == EC_ERR_ARG        # inside X: 10 x 64 x 2 bytes
    assert call(s=at((1 << 20) + 16)) == EC_ERR_ARG
    assert call(rows=0, X=None, Q=None, s=None) == EC_OK
    assert call(cols=0, X=None, Q=None, s=None) == EC_OK


def test_norm_refusals():
    L = ec.lib()

    def call(dtype=1, rows=10, d=64, eps=1e-6, X=FAKE, R=None, w=at(1 << 28), H=None, Y=FAR, Q=None,
             s=None):
        return L.ec_rms_norm(dtype, rows, d, eps, X, R, w, H, Y, Q, s, None)

    assert call(dtype=-1) == EC_ERR_DTYPE
    for rows, d in ((-1, 64), (1 << 31, 64), (10, 0), (10, 16385), (10, -5)):
        assert call(rows=rows, d=d) == EC_ERR_SHAPE
    for eps in (0.0, -1e-6, float("nan"), float("inf")):
        assert call(eps=eps) == EC_ERR_ARG
    for n in ("X", "w", "Y"):
        assert call(**{n: None}) == EC_ERR_ARG and call(**{n: MISALIGNED}) == EC_ERR_ALIGN
    assert call(R=FARTHER) == EC_ERR_ARG                        # the sum has no place
    assert call(H=FARTHER) == EC_ERR_ARG                        # no residual: no sum
    assert call(R=MISALIGNED, H=FARTHER) == EC_ERR_ALIGN
    assert call(R=at(1 << 29), H=MISALIGNED) == EC_ERR_ALIGN
    # eight bits
    mx = dict(Y=None, Q=FAR, s=FARTHER)
    assert call(**dict(mx, Y=at(1 << 32))) == EC_ERR_ARG
    assert call(**dict(mx, d=40)) == EC_ERR_SHAPE
    assert call(**dict(mx, Q=None)) == EC_ERR_ARG and call(**dict(mx, s=None)) == EC_ERR_ARG
    assert call(**dict(mx, s=MISALIGNED)) == EC_ERR_ALIGN
    # overlaps: 10 x 64 x 2 bytes
    assert call(Y=FAKE) == EC_ERR_ARG and call(Y=at((1 << 20) + 1264)) == EC_ERR_ARG
    assert call(Y=at((1 << 28) - 16)) == EC_ERR_ARG             # the weight
    assert call(R=FAR, H=FARTHER) == EC_ERR_ARG                 # Y is the residual
    assert call(R=FARTHER, H=FAR) == EC_ERR_ARG                 # Y is H
    assert call(R=FARTHER, H=at((1 << 20) + 16)) == EC_ERR_ARG
    assert call(R=FARTHER, H=at((1 << 31) + 16)) == EC_ERR_ARG
    assert call(**dict(mx, Q=FAKE)) == EC_ERR_ARG
    assert call(**dict(mx, s=at((1 << 30) + 16))) == EC_ERR_ARG
    assert call(rows=0, X=None, Y=None) == EC_OK


def test_norm_backward_refusals():
    L = ec.lib()
    ws = 1 << 30

    def call(dtype=1, rows=10, d=64, eps=1e-6, H=FAKE, w=at(1 << 28), dY=at(1 << 22), dH=at(1 << 24),
             dX=FAR, dw=FARTHER, p=at(1 << 33), n=ws):
        return L.ec_rms_norm_backward(dtype, rows, d, eps, H, w, dY, dH, dX, dw, p, n, None)

    assert call(dtype=7) == EC_ERR_DTYPE
    for rows, d in ((-1, 64), (1 << 31, 64), (10, 0), (10, 16385)):
        assert call(rows=rows, d=d) == EC_ERR_SHAPE
        assert L.ec_rms_norm_workspace_size(1, rows, d) == 0
    for eps in (0.0, -1.0, float("nan")):
        assert call(eps=eps) == EC_ERR_ARG
    for n in ("H", "w", "dY", "dX", "dw", "p"):
        assert call(**{n: None}) == EC_ERR_ARG, n
        assert call(**{n: MISALIGNED}) == EC_ERR_ALIGN, n
    assert call(dH=MISALIGNED) == EC_ERR_ALIGN
    need = L.ec_rms_norm_workspace_size(1, 10, 64)
    assert need > 0 and call(n=need - 1) == EC_ERR_WORKSPACE
    for base in (1 << 20, 1 << 22, 1 << 24):
        assert call(dX=at(base + 16)) == EC_ERR_ARG and call(dw=at(base + 16)) == EC_ERR_ARG
    assert call(dX=at((1 << 28) - 16)) == EC_ERR_ARG
    assert call(dw=at((1 << 30) + 16)) == EC_ERR_ARG
    assert L.ec_rms_norm_workspace_size(2, 10, 64) == 0
    assert L.ec_rms_norm_workspace_size(0, 0, 64) > 0
    # the shares of dw of at most 512 workgroups
    assert L.ec_rms_norm_workspace_size(0, 1 << 20, 16384) <= 512 * 16384 * 4


def _problem(**kw):
    args = dict(n_tokens=16, d_model=128, n_experts=8, d_ff=64, group_offsets=[0, 16], capacity=[0],
                inv_temperature=1.0, dtype=torch.bfloat16)
    args.update(kw)
    return binding.Problem(**args)


def test_decode_refusals():
    L, P = ec.lib(), _problem()
    need = L.ec_tc_decode_workspace_size(P.ref, 2)
    assert need > 0
    base = dict({n: FAKE for n in ("X", "Wg", "W1", "W3", "W2", "experts", "gates", "ws")}, Y=FAR,
                R=None, Ws1=None, Ws3=None, Ws2=None)

    def call(P=P, k=2, mx=None, n=need, **over):
        a = dict(base, **over)
        s = None if mx is None else ctypes.byref(binding._MxScales(**mx))
        return L.ec_tc_decode(P.ref, k, s, a["X"], a["Wg"], a["W1"], a["W3"], a["W2"], a["Ws1"],
                              a["Ws3"], a["Ws2"], a["R"], a["Y"], a["experts"], a["gates"],
                              a["ws"], n, None)

    for n in ("X", "Wg", "W1", "W3", "W2", "Y", "experts", "gates", "ws"):
        assert call(**{n: None}) == EC_ERR_ARG, n
        assert call(**{n: MISALIGNED}) == EC_ERR_ALIGN, n
    assert call(R=MISALIGNED) == EC_ERR_ALIGN
    assert call(n=need - 1) == EC_ERR_WORKSPACE
    for k in (0, 9, -1):
        assert call(k=k) == EC_ERR_ARG and L.ec_tc_decode_workspace_size(P.ref, k) == 0
    big = _problem(n_tokens=65, group_offsets=[0, 65])
    assert call(P=big) == EC_ERR_SHAPE and L.ec_tc_decode_workspace_size(big.ref, 2) == 0
    assert "64" in L.ec_last_error().decode()
    for bad in (dict(n_experts=257), dict(d_model=96), dict(d_ff=32), dict(d_shared=100)):
        assert call(P=_problem(**bad)) == EC_ERR_SHAPE
    assert call(P=_problem(inv_temperature=0.0)) == EC_ERR_ARG
    assert call(P=_problem(capacity=[17])) == EC_ERR_CAPACITY
    sh = _problem(d_shared=64)
    assert call(P=sh) == EC_ERR_ARG                              # shared weights missing
    assert call(Y=at((1 << 20) + 16)) == EC_ERR_ARG              # inside X
    assert call(R=at((1 << 30) + 4096 - 16)) == EC_ERR_ARG       # its rows meet Y's
    # eight bits: all weights or none, bf16 alone
    a = 1 << 21
    three = dict(W1=a, W3=a, W2=a)
    for n in three:
        assert call(mx=dict(three, **{n: None})) == EC_ERR_ARG
        assert call(mx=dict(three, **{n: a + 8})) == EC_ERR_ALIGN
    assert call(mx=dict(X=a + 4)) == EC_ERR_ALIGN
    f32 = _problem(dtype=torch.float32)
    assert call(P=f32, mx=three, n=1 << 30) == EC_ERR_DTYPE
    assert call(P=f32, mx=dict(X=a), n=1 << 30) == EC_ERR_DTYPE
    shared = dict(Ws1=FAKE, Ws3=FAKE, Ws2=FAKE)
    assert call(P=sh, mx=three, n=1 << 30, **shared) == EC_ERR_ARG   # the shared experts' scales
    none = _problem(n_tokens=0, group_offsets=[0, 0])
    assert call(P=none, n=1 << 20, X=None, Y=None, experts=None, gates=None) == EC_OK
    # the largest problem's sizes do not wrap
    top = _problem(n_tokens=64, d_model=16384, n_experts=256, d_ff=16384, group_offsets=[0, 64],
                   dtype=torch.float32)
    assert L.ec_tc_decode_workspace_size(top.ref, 256) >= 64 * 256 * 16384 * 4


def test_binding_refuses_host_tensors_and_wrong_operands():
    X = torch.zeros((4, 64))
    w = torch.ones(64)
    for call in (lambda: ec.rms_norm(X, w), lambda: ec.rms_norm_backward(X, X, w),
                 lambda: ec.mx_quantize(X)):
        with pytest.raises(ec.ECError, match="GPU"):
            call()
    for call in (lambda: ec.rms_norm(X.half(), w), lambda: ec.mx_quantize(X.double()),
                 lambda: ec.rms_norm_backward(X, X.half(), w)):
        with pytest.raises(ec.ECError, match="unsupported storage dtype"):
            call()
    for call in (lambda: ec.rms_norm(None, w), lambda: ec.mx_quantize(torch.tensor(1.0)),
                 lambda: ec.rms_norm_backward(X, 3, w)):
        with pytest.raises(ec.ECError, match="dimension"):
            call()
    Wg, W = torch.zeros((8, 64)), torch.zeros((8, 64, 64))
    with pytest.raises(ec.ECError, match="GPU"):
        ec.tc_decode(X, Wg, W, W, W, 2)
    with pytest.raises(ec.ECError, match="at most 64"):
        ec.tc_decode(torch.zeros((65, 64)), Wg, W, W, W, 2)
    with pytest.raises(ec.ECError, match="dimensions"):
        ec.tc_decode(X[0], Wg, W, W, W, 2)
    with pytest.raises(ec.ECError, match="dimensions"):
        ec.TcDecoder(Wg, W[0], W, W, 2)
    with pytest.raises(ec.ECError, match="GPU"):
        ec.TcDecoder(Wg, W, W, W, 2)
