"""The norm, the eight-bit layout and the few-token layer on the GPU against the float64 oracle.

Tolerances, from the arithmetic (u = 2^-24, a rounding's half step in fp32; b = 2^-8 in bf16):
  * codes and scales of given values: exact (a product with a power of two, one rounding).
  * norm: a row's mean square is a sum of d squares, at most 64 a lane in sequence, then 6
    steps over the wave and 16 waves: 86 u, halved by the root; the mean's product, the sum with
    eps, root and division 4 u; two products: 50 u of a value, then the output's rounding.  In
    eight bits half an e4m3 step instead, 2^-4 of the value or 2^-10 of its scale, and a scale
    may fall either way where the largest value is within 50 u of its border.
  * norm backward: dx = r g - r^3 h mean(g h): 200 u of r |g| + r^3 |h| mean|g h| covers the
    factors' 50 u each and the sum's 88 u; then the sum with dH and the rounding.
    dw: a term's 55 u, its sum over the rows of a wave (rows / 512 of them at most, or one
    workgroup's share) and over the workgroups (4 + 32 + 16): (120 + rows / 512) u of the
    terms' magnitudes.
  * few tokens: X and Wg lie on grids coarse enough that a logit is the same number whatever
    the order of its sum, so choices are equal; gates: the exponent's argument is off by u of
    itself, exp by 2 u, the sum of k by k u, division u: (2 |arg| + k + 8) u.  Y, relative
    2-norm: fp32: products of at most 16384 terms, (sqrt(16384) + a few) u each at the most and
    three in a chain, 2.4e-5, of at most 2048 terms 1e-5; bf16: Y's rounding b beside that and the activations' two parts, b^2: 1.01 b.
"""
import numpy as np
import pytest
import torch

from oracle import ec_ref as ref
import paper_2604_01622_amd as ec

pytestmark = pytest.mark.gpu

U, B = 2.0 ** -24, 2.0 ** -8
DTYPES = (torch.bfloat16, torch.float32)


def f64(t):
    return t.detach().double().cpu().numpy()


def rel_l2(got, want):
    den = np.linalg.norm(want)
    return float(np.linalg.norm(f64(got) - want) / (den if den > 0 else 1.0))


def normal(seed, shape, std=1.0):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed)) * std


def equal_bits(a, b):
    """Equal, NaN for NaN, in any type."""
    return torch.equal(a.contiguous().view(torch.uint8), b.contiguous().view(torch.uint8))


# ---- eight bits ----------------------------------------------------------------


def check_mx(X):
    q = ec.mx_quantize(X)
    torch.cuda.synchronize()
    assert q.codes.shape == X.shape and q.codes.dtype == torch.float8_e4m3fn
    assert q.scales.dtype == torch.float8_e8m0fnu
    codes, scales = ref.mx_quantize_ref(f64(X))
    assert np.array_equal(f64(q.scales), scales)
    assert np.array_equal(f64(q.codes), codes)
    return q


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("shape", [(1, 32), (7, 96), (3, 5, 64), (300, 1472), (1, 8224), (64,)])
def test_quantize(dtype, shape):
    x = normal(1, shape) * torch.exp(3 * normal(2, (*shape[:-1], 1)))
    check_mx(x.to(dtype).cuda())


@pytest.mark.parametrize("dtype", DTYPES)
def test_quantize_borders_and_extremes(dtype):
    x = normal(5, (24, 32)).to(dtype)
    x[0] = 0
    x[1, :2] = torch.tensor([448.0, -448.0])        # at the border of a scale
    x[2, 0] = 450.0                                 # above it
    x[3] *= 2.0 ** -130                             # fp32: scale at its floor
    x[4] *= 2.0 ** -140
    x[5, 7] = torch.finfo(dtype).max
    x[6] = torch.arange(32) / 16 * 1.0625           # ties between codes
    x[7] = x[7].abs() * -1
    x[8, 3] = 1.75 * 2.0 ** 20
    x[9, :] = 2.0 ** -126
    check_mx(x.cuda())


def test_quantize_of_no_numbers():
    x = normal(6, (6, 64)).cuda()
    x[1, 3], x[2, 40], x[3, 0] = float("nan"), float("inf"), -float("inf")
    q = ec.mx_quantize(x)
    byte = q.scales.view(torch.uint8).cpu()
    bad = torch.zeros((6, 2), dtype=torch.bool)
    bad[1, 0] = bad[2, 1] = bad[3, 0] = True
    assert torch.equal(byte == 255, bad)
    nan = torch.isnan(q.codes.float()).cpu().reshape(6, 2, 32)
    assert torch.equal(nan.all(-1), bad) and torch.equal(nan.any(-1), bad)
    assert ec.mx_quantize(x[:0]).codes.shape == (0, 64)


def test_quantize_past_32_bits():
    rows, cols = 2 ** 21 + 5, 2048                  # 2^32 elements and some
    x = torch.empty((rows, cols), dtype=torch.bfloat16, device="cuda")
    x.fill_(0.25)
    tail = normal(3, (7, cols)).to(torch.bfloat16).cuda()
    x[-7:] = tail
    q, want = ec.mx_quantize(x), ec.mx_quantize(tail)
    torch.cuda.synchronize()
    assert equal_bits(q.codes[-7:], want.codes) and equal_bits(q.scales[-7:], want.scales)
    assert bool((q.codes[:-7].view(torch.uint8) == 0x78).all())   # 256: 0.25 over 2^-10


# ---- norm ----------------------------------------------------------------------


def norm_inputs(rows, d, dtype, seed=0):
    size = torch.exp(normal(seed + 1, (rows, 1)))
    x = (normal(seed + 2, (rows, d)) * size).to(dtype).cuda()
    r = (normal(seed + 3, (rows, d)) * size).to(dtype).cuda()
    w = (1 + 0.2 * normal(seed + 4, (d,))).to(dtype).cuda()
    return x, r, w


def half(dtype):
    return B if dtype == torch.bfloat16 else U


def check_sum(H, x, r, dtype):
    want = f64(x) + f64(r)
    assert np.all(np.abs(f64(H) - want) <= (half(dtype) + U) * np.abs(want))


def check_norm(Y, H, w, eps, dtype):
    want = ref.rms_norm_ref(f64(H), f64(w), eps)
    assert np.all(np.abs(f64(Y) - want) <= (half(dtype) + 50 * U) * np.abs(want))


def check_norm_mx(Y, H, w, eps):
    want = ref.rms_norm_ref(f64(H), f64(w), eps)
    top = np.abs(want.reshape(*want.shape[:-1], -1, 32)).max(-1)
    scale = f64(Y.scales)
    ok = [scale == ref.mx_scale_ref(top * (1 + s * 50 * U)) for s in (-1, 0, 1)]
    assert np.all(ok[0] | ok[1] | ok[2])
    got = ref.mx_value_ref(f64(Y.codes), scale)
    step = np.maximum(np.abs(want) * 2.0 ** -4, np.repeat(scale, 32, -1) * 2.0 ** -10)
    assert np.all(np.abs(got - want) <= step * (1 + 50 * U) + 50 * U * np.abs(want))


WIDTHS = [1, 3, 4, 7, 8, 9, 15, 32, 63, 64, 96, 131, 512, 1000, 1001, 1024, 2048, 2056, 4092, 4096, 4097, 8192,
          12001, 16383, 16384]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("d", WIDTHS)
def test_norm_widths(d, dtype):
    for rows in (1, 5, 67):
        print(f"[norm] {rows} x {d} {dtype}", flush=True)
        x, r, w = norm_inputs(rows, d, dtype, d + rows)
        Y = ec.rms_norm(x, w, 1e-5)
        check_norm(Y, x, w, 1e-5, dtype)
        Y, H = ec.rms_norm(x, w, 1e-5, residual=r)
        check_sum(H, x, r, dtype)
        check_norm(Y, H, w, 1e-5, dtype)
        if d % 32 == 0:
            check_norm_mx(ec.rms_norm(x, w, 1e-5, mx=True), x, w, 1e-5)
            Yq, Hq = ec.rms_norm(x, w, 1e-5, residual=r, mx=True)
            assert torch.equal(Hq, H)
            check_norm_mx(Yq, H, w, 1e-5)


@pytest.mark.parametrize("dtype", DTYPES)
def test_norm_shapes_in_place_and_refusals(dtype):
    x, r, w = norm_inputs(30, 320, dtype)
    Y, H = ec.rms_norm(x, w, residual=r)
    Y3, H3 = ec.rms_norm(x.view(2, 15, 320), w, residual=r.view(2, 15, 320))
    assert torch.equal(Y3.view(30, 320), Y) and torch.equal(H3.view(30, 320), H)
    assert torch.equal(ec.rms_norm(x[4], w), ec.rms_norm(x, w)[4])
    for place in ("x", "r"):        # the sum in the place of an operand
        a, b = x.clone(), r.clone()
        Y2, H2 = ec.rms_norm(a, w, residual=b, sum_out=a if place == "x" else b)
        assert H2 is (a if place == "x" else b)
        assert torch.equal(Y2, Y) and torch.equal(H2, H)
    Y0, H0 = ec.rms_norm(x[:0], w, residual=r[:0], mx=True)
    assert Y0.codes.shape == (0, 320) and Y0.scales.shape == (0, 10) and H0.shape == (0, 320)
    for bad in (lambda: ec.rms_norm(x.t(), w), lambda: ec.rms_norm(x[:, ::2], w),
                lambda: ec.rms_norm(x, w[:-1]), lambda: ec.rms_norm(x, w, residual=r[:-1]),
                lambda: ec.rms_norm(x, w, sum_out=r), lambda: ec.rms_norm(x, w, eps=0.0),
                lambda: ec.rms_norm(x, w, residual=r.cpu()),
                lambda: ec.rms_norm(x[:, :40].contiguous(), w[:40].contiguous(), mx=True),
                lambda: ec.rms_norm(x.view(-1)[1:641].view(2, 320), w),     # not 16-byte aligned
                lambda: ec.rms_norm_backward(x[:-1], x, w),
                lambda: ec.rms_norm_backward(x, x, w, dH=r[:, :64])):
        with pytest.raises(ec.ECError):
            bad()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("d", [9, 131, 1003, 2048, 4099, 12002])
def test_norm_and_backward_in_place(d, dtype):
    """H over X and over the residual; dX over H, dY and dH (the library's interface): rows whose
    last piece shares elements with the one before it among them."""
    x, r, w = norm_inputs(37, d, dtype, d)
    Y, H = ec.rms_norm(x, w, residual=r)
    for place in ("x", "r"):
        a, b = x.clone(), r.clone()
        Y2, H2 = ec.rms_norm(a, w, residual=b, sum_out=a if place == "x" else b)
        assert torch.equal(Y2, Y) and torch.equal(H2, H)
    dX, dw = ec.rms_norm_backward(Y, H, w, dH=r)
    L, code = ec.lib(), {torch.float32: 0, torch.bfloat16: 1}[dtype]
    n = L.ec_rms_norm_workspace_size(code, 37, d)
    ws = torch.empty(n, dtype=torch.uint8, device="cuda")
    stream = torch.cuda.current_stream().cuda_stream
    for place in range(3):
        t = [H.clone(), Y.clone(), r.clone()]
        got = torch.empty_like(dw)
        assert L.ec_rms_norm_backward(code, 37, d, 1e-6, t[0].data_ptr(), w.data_ptr(),
                                      t[1].data_ptr(), t[2].data_ptr(), t[place].data_ptr(),
                                      got.data_ptr(), ws.data_ptr(), n, stream) == 0
        torch.cuda.synchronize()
        assert torch.equal(t[place], dX) and torch.equal(got, dw)


def test_norm_of_no_numbers_stays_in_its_row():
    x, r, w = norm_inputs(6, 96, torch.float32)
    want = ec.rms_norm(x, w)
    x2 = x.clone()
    x2[1, 5], x2[3, 7] = float("nan"), float("inf")
    x2[4] = 0
    Y, q = ec.rms_norm(x2, w), ec.rms_norm(x2, w, mx=True)
    for i in (0, 2, 5):
        assert torch.equal(Y[i], want[i])
    assert bool(torch.isnan(Y[1]).all()) and bool(torch.isnan(Y[3, 7])) and bool((Y[4] == 0).all())
    assert bool((q.scales[1].view(torch.uint8) == 255).all())
    byte = q.scales.view(torch.uint8).cpu()
    assert int(byte[3, 0]) == 255 and byte[4].tolist() == [1, 1, 1]
    dX, dw = ec.rms_norm_backward(r, x2, w)
    assert bool(torch.isfinite(dX[[0, 2, 4, 5]]).all()) and bool(torch.isnan(dX[1]).all())


def test_norm_of_squares_past_fp32():
    x, r, w = norm_inputs(3, 640, torch.float32)
    want, (dX, _) = ec.rms_norm(x, w), ec.rms_norm_backward(r, x, w)
    big = x.clone()
    big[1] = 1e25
    Y, (dX2, dw2) = ec.rms_norm(big, w), ec.rms_norm_backward(r, big, w)
    for i in (0, 2):
        assert torch.equal(Y[i], want[i]) and torch.equal(dX2[i], dX[i])
    assert bool((Y[1] == 0).all()) and bool(torch.isfinite(dw2).all())


def test_norm_past_32_bits():
    rows, d = 2 ** 20 + 3, 4096
    x = torch.empty((rows, d), dtype=torch.bfloat16, device="cuda")
    x.fill_(1.0)
    tail, r, w = norm_inputs(5, d, torch.bfloat16)
    x[-5:] = tail
    Y = ec.rms_norm(x, w)
    assert torch.equal(Y[-5:], ec.rms_norm(tail, w))
    del Y
    q = ec.rms_norm(x, w, mx=True)
    want = ec.rms_norm(tail, w, mx=True)
    assert equal_bits(q.codes[-5:], want.codes) and equal_bits(q.scales[-5:], want.scales)
    del q
    dY = torch.zeros_like(x)
    dY[-5:] = r
    dX, dw = ec.rms_norm_backward(dY, x, w)
    dXt, dwt = ec.rms_norm_backward(r, tail, w)
    assert torch.equal(dX[-5:], dXt) and bool((dX[:8] == 0).all())
    assert np.all(np.abs(f64(dw) - f64(dwt)) <= 1e-4 * np.abs(f64(dwt)) + 1e-6 * f64(dwt.abs().max()))


def check_norm_backward(dY, H, w, eps, dH, dtype):
    dX, dw = ec.rms_norm_backward(dY, H, w, eps, dH=dH)
    torch.cuda.synchronize()
    assert dw.dtype == torch.float32 and dX.dtype == dtype
    g, h, wf = f64(dY), f64(H), f64(w)
    want, want_w = ref.rms_norm_backward_ref(g, h, wf, eps, None if dH is None else f64(dH))
    r = 1.0 / np.sqrt((h * h).mean(-1, keepdims=True) + eps)
    gw = np.abs(g * wf)
    size = r * gw + r ** 3 * np.abs(h) * (gw * np.abs(h)).mean(-1, keepdims=True)
    bound = 200 * U * size + half(dtype) * np.abs(want)
    if dH is not None:
        bound += U * (np.abs(f64(dH)) + np.abs(want))
    assert np.all(np.abs(f64(dX) - want) <= bound)
    terms = np.abs(g * h * r).sum(0)
    assert np.all(np.abs(f64(dw) - want_w) <= (120 + len(h) / 512) * U * terms)
    return dX, dw


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("d", WIDTHS)
def test_norm_backward_widths(d, dtype):
    for rows in (1, 5, 67):
        print(f"[norm backward] {rows} x {d} {dtype}", flush=True)
        H, dH, w = norm_inputs(rows, d, dtype, d + rows)
        dY = normal(d + rows + 9, (rows, d)).to(dtype).cuda()
        check_norm_backward(dY, H, w, 1e-5, None, dtype)
        check_norm_backward(dY, H, w, 1e-5, dH, dtype)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows,d", [(2049, 64), (513, 2048), (3001, 131), (1100, 4100), (4100, 1024)])
def test_norm_backward_many_rows(rows, d, dtype):
    H, dH, w = norm_inputs(rows, d, dtype, rows)
    dY = normal(rows + 9, (rows, d)).to(dtype).cuda()
    a = check_norm_backward(dY, H, w, 1e-6, dH, dtype)
    b = ec.rms_norm_backward(dY, H, w, 1e-6, dH=dH)
    assert all(torch.equal(x, y) for x, y in zip(a, b))     # the same bits every time


def test_norm_backward_of_no_rows():
    w = torch.ones(64, device="cuda")
    x = torch.empty((0, 64), device="cuda")
    dX, dw = ec.rms_norm_backward(x, x, w)
    assert dX.shape == (0, 64) and bool((dw == 0).all())


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows,d", [(700, 512), (40, 131), (300, 12000)])
def test_norm_backward_in_a_graph(rows, d, dtype):
    """Captured with the eight bits of its result and replayed on other rows, with eager calls
    between the replays."""
    sets = [norm_inputs(rows, d, dtype, 10 * i) for i in range(3)]
    w = sets[0][2]

    def step(H, dY):
        dX, dw = ec.rms_norm_backward(dY, H, w, dH=H)
        return (dX, dw, *(ec.mx_quantize(dX) if d % 32 == 0 else ()))

    def equal(got, want):
        return all(equal_bits(a, b) if a.element_size() == 1 else torch.equal(a, b)
                   for a, b in zip(got, want))

    want = [step(H, dY) for H, dY, _ in sets]
    H, dY = sets[0][0].clone(), sets[0][1].clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        out = step(H, dY)
    for n in (0, 1, 2, 1, 0):
        H.copy_(sets[n][0]), dY.copy_(sets[n][1])
        graph.replay()
        again = step(*sets[n][:2])
        torch.cuda.synchronize()
        assert equal(out, want[n]) and equal(again, want[n])


def test_norm_backward_against_differences():
    """The forward kernel's own outputs, a step either way along a direction."""
    x, r, w = norm_inputs(9, 200, torch.float32, 5)
    dY, dH = normal(8, (9, 200)).cuda(), normal(9, (9, 200)).cuda()
    v = normal(10, (9, 200)).cuda() * x.abs().mean(1, keepdim=True)
    Y, H = ec.rms_norm(x, w, residual=r)
    dX, _ = ec.rms_norm_backward(dY, H, w, dH=dH)
    step = 2.0 ** -6

    def total(s):
        Y, H = ec.rms_norm(x + s * step * v, w, residual=r)
        return float((Y.double() * dY.double()).sum() + (H.double() * dH.double()).sum())

    got, want = (total(1) - total(-1)) / (2 * step), float((dX.double() * v.double()).sum())
    # the difference's own error: a third of step^2 of a third derivative of the order of the
    # terms, and 50 u of the terms over the step
    size = float((dX.double() * v.double()).abs().sum())
    assert abs(got - want) <= (step ** 2 + 100 * U / step) * size


# ---- few tokens ----------------------------------------------------------------


def layer_inputs(N, d, E, h, hs=0, dtype=torch.bfloat16, mx=False, xmx=False, seed=0):
    """X and Wg on grids (see above); weights in eight bits where asked."""
    unit = 2.0 ** round(np.log2(d ** -0.5))
    X = ((normal(seed + 1, (N, d)) * 16).round().clamp(-96, 96) / 16).to(dtype).cuda()
    Wg = ((normal(seed + 2, (E, d)) * 4).round().clamp(-15, 15) / 4 * unit).to(dtype).cuda()
    held = ec.mx_quantize if mx else (lambda t: t)
    s = d ** -0.5
    W1, W3 = (held(normal(seed + n, (E, h, d), s).to(dtype).cuda()) for n in (3, 4))
    W2 = held(normal(seed + 5, (E, d, h), s).to(dtype).cuda())
    shared = None
    if hs:
        shared = tuple(held(normal(seed + n, shape, s).to(dtype).cuda())
                       for n, shape in ((6, (hs, d)), (7, (hs, d)), (8, (d, hs))))
    return ec.mx_quantize(X) if xmx else X, Wg, W1, W3, W2, shared


def value(t):
    if isinstance(t, ec.Mx):
        return ref.mx_value_ref(f64(t.codes), f64(t.scales))
    return f64(t)


def check_decode(got, X, Wg, W1, W3, W2, k, inv_tau=1.0, shared=None, residual=None):
    Y, experts, gates = got
    torch.cuda.synchronize()
    want, e, g = ref.tc_decode_ref(value(X), value(Wg), value(W1), value(W3), value(W2), k, inv_tau,
                                   None if shared is None else [value(t) for t in shared],
                                   None if residual is None else f64(residual))
    assert experts.dtype == torch.int32 and np.array_equal(experts.cpu().numpy(), e)
    z = value(X) @ value(Wg).T
    arg = (np.take_along_axis(z, e, 1) - z.max(1, keepdims=True)) * inv_tau
    # a gate below fp32's normal numbers is off by its last bit
    assert np.all(np.abs(f64(gates) - g) <= (2 * np.abs(arg) + k + 8) * U * g + 2.0 ** -149)
    f32 = 2.4e-5 if max(value(W1).shape[1:]) > 2048 else 1e-5
    assert rel_l2(Y, want) <= (f32 if Y.dtype == torch.float32 else 1.01 * B)


FORMS = [(torch.bfloat16, False, False), (torch.bfloat16, True, False), (torch.bfloat16, True, True),
         (torch.bfloat16, False, True), (torch.float32, False, False)]


@pytest.mark.parametrize("dtype,mx,xmx", FORMS)
@pytest.mark.parametrize("N", [1, 2, 3, 15, 16, 17, 31, 32, 33, 48, 63, 64])
def test_decode_token_counts(N, dtype, mx, xmx):
    print(f"[decode] N {N} {dtype} mx {mx} {xmx}", flush=True)
    X, Wg, W1, W3, W2, sh = layer_inputs(N, 192, 12, 128, 64, dtype, mx, xmx, N)
    R = normal(N + 50, (N, 192)).to(dtype).cuda()
    check_decode(ec.tc_decode(X, Wg, W1, W3, W2, 3), X, Wg, W1, W3, W2, 3)
    check_decode(ec.tc_decode(X, Wg, W1, W3, W2, 3, 2.0, shared=sh, residual=R), X, Wg, W1, W3, W2,
                 3, 2.0, sh, R)


@pytest.mark.parametrize("dtype,mx,xmx", FORMS)
@pytest.mark.parametrize("d,E,h,hs,k", [
    (64, 1, 64, 0, 1), (64, 3, 64, 64, 3), (128, 17, 64, 128, 4), (1472, 40, 832, 640, 4),
    (2048, 8, 1024, 0, 2), (320, 256, 64, 192, 8), (64, 256, 64, 0, 256), (576, 65, 448, 0, 5),
    (64, 20, 2048, 1088, 20)])
def test_decode_shapes(d, E, h, hs, k, dtype, mx, xmx):
    for N in (1, 5, 40):
        print(f"[decode] N {N} d {d} E {E} h {h} hs {hs} k {k} {dtype} {mx} {xmx}", flush=True)
        X, Wg, W1, W3, W2, sh = layer_inputs(N, d, E, h, hs, dtype, mx, xmx, d + N)
        check_decode(ec.tc_decode(X, Wg, W1, W3, W2, k, 0.5, shared=sh), X, Wg, W1, W3, W2, k, 0.5,
                     sh)


@pytest.mark.parametrize("dtype,mx,xmx", FORMS)
@pytest.mark.parametrize("N,d,E,h,k", [
    (16, 64, 40, 64, 16), (16, 64, 40, 64, 17), (11, 128, 256, 64, 24),   # pairs at the border of
    (16, 64, 70, 128, 16), (17, 64, 70, 128, 3),                          # a choice of its own
    (3, 16384, 3, 64, 2), (64, 64, 2, 1024, 1), (33, 128, 5, 1088, 2), (20, 256, 16, 960, 16)])
def test_decode_borders(N, d, E, h, k, dtype, mx, xmx):
    print(f"[decode] N {N} d {d} E {E} h {h} k {k} {dtype} {mx} {xmx}", flush=True)
    X, Wg, W1, W3, W2, _ = layer_inputs(N, d, E, h, 0, dtype, mx, xmx, d + N)
    check_decode(ec.tc_decode(X, Wg, W1, W3, W2, k), X, Wg, W1, W3, W2, k)


@pytest.mark.parametrize("dtype", DTYPES)
def test_decode_ties_take_the_lower_expert(dtype):
    X, Wg, W1, W3, W2, _ = layer_inputs(37, 128, 96, 64, 0, dtype)
    Wg[5:] = Wg[:91].clone()[torch.arange(91) % 5]          # five logits, each many times
    got = ec.tc_decode(X, Wg, W1, W3, W2, 9)
    check_decode(got, X, Wg, W1, W3, W2, 9)
    Wg[:] = 0                                               # zeros of both signs are equal
    X[:, 0] = 1
    Wg[::2, 0] = -0.0
    got = ec.tc_decode(X, Wg, W1, W3, W2, 4)
    assert torch.equal(got[1], torch.arange(4, device="cuda", dtype=torch.int32).expand(37, 4))


@pytest.mark.parametrize("dtype,mx,xmx", FORMS)
def test_decode_every_token_on_one_expert(dtype, mx, xmx):
    X, Wg, W1, W3, W2, _ = layer_inputs(64, 128, 24, 192, 0, dtype, mx)
    Wg[:] = 0
    Wg[17, 0], Wg[3, 1] = 4.0, 4.0
    X[:, 0], X[:, 1] = 4.0, 2.0
    X = ec.mx_quantize(X) if xmx else X
    got = ec.tc_decode(X, Wg, W1, W3, W2, 2)
    check_decode(got, X, Wg, W1, W3, W2, 2)
    assert got[1].tolist() == [[17, 3]] * 64


def test_decode_agrees_with_token_choice():
    X, Wg, W1, W3, W2, sh = layer_inputs(64, 1024, 32, 512, 256)
    Y, experts, gates = ec.tc_decode(X, Wg, W1, W3, W2, 4, shared=sh)
    want, rows = ec.tc_forward(X, Wg, W1, W3, W2, [0, 64], [64], 4, shared=sh)
    assert torch.equal(torch.bincount(experts.view(-1).long(), minlength=32).cumsum(0),
                       rows[1:].long())
    # each is off the definition by its roundings: Y here, A, O and the shared Y there too
    assert rel_l2(Y, f64(want)) <= (1.01 + 2) * B


def test_decode_reads_the_chosen_experts_alone():
    X, Wg, W1, W3, W2, _ = layer_inputs(3, 128, 30, 128)
    Y, experts, _ = ec.tc_decode(X, Wg, W1, W3, W2, 2)
    rest = [j for j in range(30) if j not in set(experts.view(-1).tolist())]
    for w in (W1, W3, W2):
        w[rest] = float("nan")
    assert torch.equal(ec.tc_decode(X, Wg, W1, W3, W2, 2)[0], Y)


@pytest.mark.parametrize("dtype,mx,xmx", FORMS)
def test_decode_of_no_numbers_stays_in_its_token(dtype, mx, xmx):
    X, Wg, W1, W3, W2, sh = layer_inputs(20, 128, 16, 64, 64, dtype, mx)
    x2 = X.clone()
    x2[4, 9], x2[18, 100] = float("nan"), float("inf")
    if xmx:
        X, x2 = ec.mx_quantize(X), ec.mx_quantize(x2)
    want = ec.tc_decode(X, Wg, W1, W3, W2, 3, shared=sh)
    Y, experts, gates = ec.tc_decode(x2, Wg, W1, W3, W2, 3, shared=sh)
    keep = [i for i in range(20) if i not in (4, 18)]
    for a, b in zip((Y, experts, gates), want):
        assert torch.equal(a[keep], b[keep])
    assert bool(torch.isnan(Y[4]).all()) and bool(torch.isnan(Y[18]).any())
    assert experts[4].tolist() == [0, 1, 2] and bool(torch.isnan(gates[4]).all())
    assert int(experts.min()) >= 0 and int(experts.max()) < 16


def test_decode_far_logits_have_zero_gates():
    X, Wg, W1, W3, W2, _ = layer_inputs(5, 64, 8, 64)
    X[:, 0] = 6.0
    Wg[:, 0] = torch.tensor([60.0, 0, 0, -60, -60, 0, 0, 0])
    got = ec.tc_decode(X, Wg, W1, W3, W2, 8)
    check_decode(got, X, Wg, W1, W3, W2, 8)
    assert bool((got[2][:, 0] == 1).all()) and bool((got[2][:, 1:] == 0).all())


@pytest.mark.parametrize("dtype,mx,xmx", FORMS)
def test_decoder_buffers_and_places(dtype, mx, xmx):
    X, Wg, W1, W3, W2, sh = layer_inputs(40, 192, 10, 64, 128, dtype, mx, xmx)
    R = normal(3, (40, 192)).to(dtype).cuda()
    want = ec.tc_decode(X, Wg, W1, W3, W2, 2, shared=sh, residual=R)
    dec = ec.TcDecoder(Wg, W1, W3, W2, 2, shared=sh, max_tokens=50)
    dec.ws.fill_(255)                                       # NaN patterns, indexes far outside
    dec.Y.fill_(7), dec.experts.fill_(-5), dec.gates.fill_(-1)
    got = dec.forward(X, residual=R)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    # rows behind the tokens are left as they were
    assert bool((dec.Y[40:] == 7).all()) and bool((dec.experts[40:] == -5).all())
    assert bool((dec.gates[40:] == -1).all())
    part = ec.Mx(X.codes[:3], X.scales[:3]) if xmx else X[:3]
    got = dec.forward(part, residual=R[:3])                 # fewer tokens, the same answers
    assert torch.equal(got[0], ec.tc_decode(part, Wg, W1, W3, W2, 2, shared=sh, residual=R[:3])[0])
    got = dec.forward(ec.Mx(X.codes[:0], X.scales[:0]) if xmx else X[:0])
    assert [t.shape[0] for t in got] == [0, 0, 0]
    # out in the place of the residual, and of X
    r = R.clone()
    got = dec.forward(X, residual=r, out=r)
    assert got[0] is r and torch.equal(r, want[0])
    if not xmx:
        x = X.clone()
        assert torch.equal(dec.forward(x, residual=R, out=x)[0], want[0])
        x = X.clone()
        both = ec.tc_decode(X, Wg, W1, W3, W2, 2, shared=sh, residual=X)[0]
        assert torch.equal(dec.forward(x, residual=x, out=x)[0], both)


def test_decoder_refusals():
    X, Wg, W1, W3, W2, sh = layer_inputs(4, 64, 8, 128, 64)
    q = [ec.mx_quantize(t) for t in (W1, W3, W2)]
    qs = [ec.mx_quantize(t) for t in sh]
    dec = ec.TcDecoder(Wg, W1, W3, W2, 2, max_tokens=4)
    f32 = ec.TcDecoder(Wg.float(), W1.float(), W3.float(), W2.float(), 2)
    wrong = ec.Mx(q[0].codes, q[0].scales[:, :, :1])
    for bad in (lambda: ec.TcDecoder(Wg, q[0], W3, W2, 2), lambda: ec.TcDecoder(Wg, W1, q[1], W2, 2),
                lambda: ec.TcDecoder(Wg, *q, 2, shared=sh),
                lambda: ec.TcDecoder(Wg, W1, W3, W2, 2, shared=qs),
                lambda: ec.TcDecoder(Wg.float(), *q, 2), lambda: ec.TcDecoder(Wg, wrong, *q[1:], 2),
                lambda: ec.TcDecoder(Wg, W1, W3, W2, 0), lambda: ec.TcDecoder(Wg, W1, W3, W2, 9),
                lambda: ec.TcDecoder(Wg, W1, W3, W2, 2, max_tokens=65),
                lambda: ec.TcDecoder(Wg, W1, W3, W2, 2, max_tokens=-1),
                lambda: ec.TcDecoder(Wg, W1, W3, W2, 2, float("nan")),
                lambda: ec.TcDecoder(Wg, W1, W3, W2, 2, shared=sh[:2]),
                lambda: ec.TcDecoder(Wg[:, :32], W1, W3, W2, 2),
                lambda: dec.forward(torch.cat([X, X])), lambda: dec.forward(X[:, :32]),
                lambda: dec.forward(X.float()), lambda: dec.forward(X.cpu()),
                lambda: dec.forward(X, residual=X[:3]), lambda: dec.forward(X, out=X.float()),
                lambda: f32.forward(ec.mx_quantize(X)),
                lambda: dec.forward(X[1:], out=X[:-1])):      # out meets X one row further
        with pytest.raises(ec.ECError):
            bad()


@pytest.mark.parametrize("dtype,mx,xmx", FORMS)
def test_decode_step_in_a_graph(dtype, mx, xmx):
    """A block's step, norm and layer, captured once and replayed on other tokens, with eager
    work of the same kind between the replays."""
    _, Wg, W1, W3, W2, sh = layer_inputs(1, 256, 16, 128, 64, dtype, mx)
    w = (1 + 0.1 * normal(1, (256,))).to(dtype).cuda()
    streams = [normal(20 + i, (21, 256)).to(dtype).cuda() for i in range(3)]
    adds = [normal(30 + i, (21, 256)).to(dtype).cuda() for i in range(3)]
    dec, eager = (ec.TcDecoder(Wg, W1, W3, W2, 4, shared=sh, max_tokens=21) for _ in range(2))

    def step(layer, x, r):
        y, h = ec.rms_norm(x, w, residual=r, mx=xmx)
        return layer.forward(y, residual=h)

    want = [tuple(t.clone() for t in step(eager, x, r)) for x, r in zip(streams, adds)]
    x, r = streams[0].clone(), adds[0].clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        out = step(dec, x, r)
    for n in (0, 1, 2, 1, 0):
        x.copy_(streams[n]), r.copy_(adds[n])
        graph.replay()
        again = step(eager, streams[n], adds[n])
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want[n]))
        assert all(torch.equal(a, b) for a, b in zip(again, want[n]))


def test_decode_on_two_streams():
    args = [layer_inputs(30, 256, 16, 256, seed=s) for s in (0, 100)]
    want = [ec.tc_decode(*a[:5], 4) for a in args]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in args]
    for _ in range(5):
        got = []
        for s, a in zip(streams, args):
            s.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(s):
                got.append(ec.tc_decode(*a[:5], 4))
        torch.cuda.synchronize()
        for g, w in zip(got, want):
            assert all(torch.equal(x, y) for x, y in zip(g, w))


def test_weights_past_32_bits():
    """Experts whose weights start past 2^32 elements."""
    E, d, h = 66, 8192, 8192
    X, Wg, _, _, _, _ = layer_inputs(2, d, 1, 64)
    Wg = torch.zeros((E, d), dtype=torch.bfloat16, device="cuda")
    Wg[64:, 0] = 1.0
    X[:, 0] = 2.0
    W = [torch.empty((E, d, h), dtype=torch.bfloat16, device="cuda") for _ in range(3)]
    few = [normal(n, (2, d, h), 0.01).to(torch.bfloat16).cuda() for n in (1, 2, 3)]
    for a, b in zip(W, few):
        a[64:] = b
    got = ec.tc_decode(X, Wg, *W, 2)
    want = ec.tc_decode(X, Wg[64:].contiguous(), *few, 2)
    assert got[1].tolist() == [[64, 65]] * 2
    assert torch.equal(got[0], want[0]) and torch.equal(got[2], want[2])


# ---- together ------------------------------------------------------------------


def test_training_step_of_a_block():
    """norm with the residual -> token-choice layer with its balance loss, dropout and residual
    -> backward -> the norm's backward, which joins the two paths' gradients."""
    rng = torch.tensor([5, 1], dtype=torch.int64, device="cuda")
    N, d, E, h, k = 90, 128, 8, 64, 2
    _, Wg, W1, W3, W2, _ = layer_inputs(N, d, E, h, dtype=torch.float32)
    x, r, w = norm_inputs(N, d, torch.float32)
    dY = normal(77, (N, d)).cuda()
    y, H = ec.rms_norm(x, w, residual=r)
    layer = ec.TcLayer(y, Wg, W1, W3, W2, [0, 40, N], [40, 50], k, training=True, residual=H,
                       dropout=0.1, rng=rng)
    out = layer.forward()
    dloss = torch.tensor([0.3, -0.2], device="cuda")
    dy = layer.backward(dY, dloss)[0]
    dX, dw = ec.rms_norm_backward(dy, H, w, dH=dY)
    torch.cuda.synchronize()
    mask = ref.dropout_mask_ref(np.arange(N * d), 0.1, 5, 1).reshape(N, d)
    Hf = f64(x) + f64(r)
    yf = ref.rms_norm_ref(Hf, f64(w), 1e-6)
    want = ref.tc_train_ref(yf, f64(Wg), f64(W1), f64(W3), f64(W2), f64(dY), [0, 40, N], k, [40, 50],
                            1.0, None, Hf, mask, f64(dloss))
    dx, dwf = ref.rms_norm_backward_ref(want["dX"], Hf, f64(w), 1e-6, f64(dY))
    # products of at most 128 terms and eight in a chain, fp32: 8 (sqrt(128) + 4) u = 7e-6
    assert rel_l2(out, want["Y"]) <= 1e-5
    assert rel_l2(dX, dx) <= 1e-5 and rel_l2(dw, dwf) <= 1e-5


@pytest.mark.parametrize("mx", [False, True])
def test_serving_step_of_a_block(mx):
    _, Wg, W1, W3, W2, sh = layer_inputs(1, 512, 24, 256, 128, mx=mx)
    x, r, w = norm_inputs(33, 512, torch.bfloat16)
    y, H = ec.rms_norm(x, w, residual=r, mx=mx)
    dec = ec.TcDecoder(Wg, W1, W3, W2, 4, shared=sh, max_tokens=40)
    Y, experts, gates = dec.forward(y, residual=H)
    torch.cuda.synchronize()
    z = value(y) @ value(Wg).T
    # a choice is right if no expert left out is above one taken by more than the sum's error
    e = experts.cpu().numpy()
    slack = 512 * U * (np.abs(value(y)) @ np.abs(value(Wg)).T).max(1)
    low = np.take_along_axis(z, e, 1).min(1)
    left = z.copy()
    np.put_along_axis(left, e, -np.inf, 1)
    assert np.all(left.max(1) <= low + slack)
    want = f64(H) + ref.shared_ffn_ref(value(y), [value(t) for t in sh])
    g = np.take_along_axis(z, e, 1)
    g = np.exp(g - g.max(1, keepdims=True))
    g /= g.sum(1, keepdims=True)
    W = [value(t) for t in (W1, W3, W2)]
    for i in range(33):
        for j, s in zip(e[i], g[i]):
            want[i] += s * ref.swiglu_ffn_ref(value(y)[i:i + 1], *(t[j] for t in W))[0]
    assert rel_l2(Y, want) <= 1.01 * B
