"""The operators of token-choice training on the GPU against the float64 oracle.

Tolerances, from the arithmetic (u = half a step: 2^-24 in fp32, 2^-8 in bf16):
  * counts, masks and choices: exact.  X and Wg lie on grids coarse enough that a logit is
    the same fp32 number whatever the order of its sum (integers below 2^24 in units of one
    power of two), so the oracle's float64 scores order the experts as the kernels' do.
  * balance loss: sums in 64 bits, one rounding: 2 u.
  * its gradient from given scores: 64 bits and one rounding, u |dZ| + the 64-bit rounding of
    two terms that cancel, 2^-48 S_ij inv_tau max|b|, + half the smallest fp32 number.
  * dropout: scale, product and sum rounded in fp32 (u each), then the storage type.
  * layer, bf16: each output's relative 2-norm is off by the roundings on the way to it,
    independent of each other, so at most sqrt(n) 2^-8 with n the stored tensors on the way:
    Y: A, O, shared A, shared Y, Y; gradients: dY after dropout, H1, H3, A, dH, dXe, dZ, the
    three writes of dX.  n = 5 and 10.
  * layer, fp32: products of at most 1024 terms in fp32, (sqrt(1024) + a few) u each and
    four in a chain: 1e-5.
"""
import numpy as np
import pytest
import torch

from oracle import ec_ref as ref
import paper_2604_01622_amd as ec

pytestmark = pytest.mark.gpu

U32, UBF = 2.0 ** -24, 2.0 ** -8
GRADS = ("dX", "dWg", "dW1", "dW3", "dW2", "dWs1", "dWs3", "dWs2")


def f64(t):
    return t.detach().double().cpu().numpy()


def rel_l2(got, want):
    den = np.linalg.norm(want)
    return float(np.linalg.norm(f64(got) - want) / (den if den > 0 else 1.0))


def offsets(lens):
    return np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)


def rng_pair(seed, offset):
    wrap = lambda x: x - 2 ** 64 if x >= 2 ** 63 else x   # noqa: E731
    return torch.tensor([wrap(seed), wrap(offset)], dtype=torch.int64, device="cuda")


# ---- balance loss --------------------------------------------------------------


def scores(N, E, seed, ties=False, sharp=1.0):
    gen = torch.Generator().manual_seed(seed)
    z = torch.randn((N, E), generator=gen) * sharp + torch.randn((E,), generator=gen) * 0.5
    if ties:
        z = (z * 2).round() / 2
    return torch.softmax(z, 1).cuda()


def check_balance(S, lens, k, inv_tau=1.0):
    off = offsets(lens)
    print(f"[balance] lens {lens[:8]} E {S.shape[1]} k {k}", flush=True)
    loss, counts = ec.tc_balance(S, off, k)
    dloss = torch.linspace(0.5, -1.5, len(lens), device="cuda")
    dZ = ec.tc_balance_backward(S, counts, dloss, off, k, inv_tau)
    torch.cuda.synchronize()
    Sh = f64(S)
    want, cnt = ref.tc_balance_ref(Sh, off, k)
    assert np.array_equal(counts.cpu().numpy(), cnt)
    assert np.all(np.abs(f64(loss) - want) <= 2 * U32 * np.abs(want))
    dl = f64(dloss)
    want = ref.tc_balance_backward_ref(Sh, cnt, dl, off, k, inv_tau)
    top = np.repeat([abs(w) * S.shape[1] * cnt[g].max() / (k * max(n, 1) ** 2)
                     for g, (w, n) in enumerate(zip(dl, lens))], lens)[:, None]
    bound = U32 * np.abs(want) + 2.0 ** -48 * Sh * top * inv_tau + 2.0 ** -150
    assert np.all(np.abs(f64(dZ) - want) <= bound)


@pytest.mark.parametrize("E,k", [(1, 1), (3, 2), (8, 8), (17, 4), (40, 6), (64, 8), (65, 1),
                                 (100, 3), (128, 8), (161, 5), (256, 12)])
@pytest.mark.parametrize("ties", [False, True])
def test_balance_expert_counts(E, k, ties):
    check_balance(scores(203, E, E + k, ties), [70, 0, 1, 132], k, 2.0)


@pytest.mark.parametrize("lens", [[1], [0], [0, 0, 5, 0], [15], [16], [17], [63], [64], [65], [128],
                                  [4097], [20000], [300] * 131, [1, 700, 2, 0, 3], [256, 9],
                                  [257], [10] * 130, [65536], [65500, 36]])
def test_balance_group_lengths(lens):
    check_balance(scores(sum(lens), 24, len(lens)), lens, 3)


@pytest.mark.parametrize("E,k", [(100, 3), (129, 8), (193, 9), (256, 8), (256, 200)])
@pytest.mark.parametrize("lens", [[0, 0, 300] + [3, 0] * 80 + [700], [5000], [257, 0, 49, 289]])
def test_balance_past_64_experts(E, k, lens):
    """A group's loss comes in parts of 64 experts: empty groups, more groups than a launch
    takes, groups of many chunks; k below, at and past the eight entries that a lane sorts."""
    check_balance(scores(sum(lens), E, k), lens, k, 0.5)
    check_balance(scores(sum(lens), E, k, ties=True), lens, k)


@pytest.mark.parametrize("E,k", [(24, 3), (200, 8)])
def test_balance_in_a_graph(E, k):
    S, other, off = scores(1500, E, 1), scores(1500, E, 2), offsets([900, 0, 600])
    want = [ec.tc_balance(x, off, k) for x in (S, other)]
    buf, dloss = S.clone(), torch.tensor([1.0, 5.0, -2.0], device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        loss, counts = ec.tc_balance(buf, off, k)
        dZ = ec.tc_balance_backward(buf, counts, dloss, off, k)
    for step in range(4):
        x, (wl, wc) = (S, other)[step % 2], want[step % 2]
        buf.copy_(x)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(loss, wl) and torch.equal(counts, wc)
        assert torch.equal(dZ, ec.tc_balance_backward(x, wc, dloss, off, k))


def test_balance_ties_between_lanes_and_within_one():
    """Equal largest scores in one lane (four neighbours of 64), in several, and both."""
    for E, k in ((64, 3), (128, 8), (256, 8), (256, 12)):
        S = scores(96, E, E + 1) * 0.25
        S[:24, 4:8] = 0.5
        S[24:48, 1::16] = 0.5
        S[48:72, 4:24] = 0.5
        S[72:, E - 1] = 0.5
        check_balance(S, [96], k)


def test_balance_many_tokens():
    check_balance(scores(70001, 33, 5, sharp=2.0), [69000, 1001], 4)


@pytest.mark.parametrize("E,k", [(1, 1), (100, 2)])
def test_balance_of_the_most_tokens(E, k):
    """2^24 - 1 tokens (a problem's N 2 d < 2^31 with the smallest d): scores past 2^32 bytes,
    chunks of more tokens; one more is refused."""
    N, first = 2 ** 24 - 1, 2 ** 23 + 77
    S = torch.full((N, E), 0.5 / E, device="cuda")
    S[:, E - 1] = 0.75
    off = [0, first, N]
    loss, counts = ec.tc_balance(S, off, k)
    want = torch.zeros(2, E, dtype=torch.int32)
    sums = torch.tensor([float(S[0, 0]), float(S[0, E - 1])], dtype=torch.float64)
    for g, L in enumerate((first, N - first)):
        want[g, E - 1] = want[g, 0] = L      # the largest, then the lowest of the equal ones
        mean = sums[1] + (sums[0] if E > 1 else 0)
        assert loss[g].item() == pytest.approx(float(E / k * mean), rel=2 * U32)
    assert torch.equal(counts.cpu(), want)
    S[-1] = 0.25 / E
    dZ = ec.tc_balance_backward(S, counts, torch.tensor([1.0, 2.0 ** 20], device="cuda"), off, k)
    b = 2.0 ** 20 * E / (k * (N - first))
    last = 0.25 / E
    assert dZ[-1, E - 1].item() == pytest.approx(last * (b - min(E, 2) * last * b), rel=1e-6)
    with pytest.raises(ec.ECError, match="32-bit"):
        ec.tc_balance(S.new_empty((N + 1, 1)), [0, N + 1], 1)


def test_balance_collapsed_and_equal_scores():
    S = torch.zeros((500, 48), device="cuda")
    S[:, 7] = 1.0                                # every row the same expert: E / k ties of zero
    check_balance(S, [500], 2)
    check_balance(torch.full((130, 96), 1 / 96, device="cuda"), [100, 30], 5)


def test_balance_scores_with_nan():
    """A NaN is never chosen, and its row's other experts are: counts stay exact."""
    S = scores(100, 20, 9)
    S[3, 4] = float("nan")
    S[7] = float("nan")
    loss, counts = ec.tc_balance(S, [0, 50, 100], 3)
    want = np.zeros((2, 20), dtype=np.int64)
    for i, row in enumerate(S.cpu().numpy()):
        order = [j for j in np.lexsort((np.arange(20), -row)) if not np.isnan(row[j])]
        want[i // 50, order[:3]] += 1
    assert np.array_equal(counts.cpu().numpy(), want)
    assert np.isnan(loss[0].item()) and np.isfinite(loss[1].item())


def test_balance_agrees_with_the_choice_of_tc_route():
    X = torch.randn((300, 128), device="cuda").bfloat16()
    Wg = (0.2 * torch.randn((24, 128), device="cuda")).bfloat16()
    S, G, slot, rows, sel = ec.tc_route(X, Wg, [0, 300], [300], 4)
    _, counts = ec.tc_balance(S, [0, 300], 4)
    assert torch.equal(counts[0], rows[1:] - rows[:-1])


def test_balance_deterministic_and_in_place():
    S, off = scores(9000, 64, 3), offsets([5000, 4000])
    a, b = ec.tc_balance(S, off, 8), ec.tc_balance(S, off, 8)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


# ---- dropout -------------------------------------------------------------------


def check_dropout(n, p, dtype, residual, seed, offset, shape=None):
    gen = torch.Generator().manual_seed(n + 1)
    shape = shape or (n,)
    X = (torch.randn(shape, generator=gen) + 3.0).to(dtype).cuda()     # no zeros among them
    R = torch.randn(shape, generator=gen).to(dtype).cuda() if residual else None
    rng = rng_pair(seed, offset)
    Y = ec.dropout(X, p, rng, residual=R)
    torch.cuda.synchronize()
    m = ref.dropout_mask_ref(np.arange(n), p, seed, offset).reshape(shape)
    x, r = f64(X), f64(R) if residual else 0.0
    want = x * m + r
    got = f64(Y)
    if residual:
        assert np.array_equal(got[m == 0], f64(R)[m == 0])
    else:
        assert np.array_equal(got == 0, m == 0)
    bound = 2 * U32 * np.abs(x * m) + U32 * np.abs(want)
    if dtype == torch.bfloat16:
        bound = UBF * (np.abs(want) + bound) + bound
    assert np.all(np.abs(got - want) <= bound)
    # the gradient in X is the same call on dY: linear, so <Y - R, dY> = <X, dX>
    dY = torch.randn(shape, generator=gen).to(dtype).cuda()
    dX = f64(ec.dropout(dY, p, rng))
    assert np.array_equal(dX[m == 0], np.zeros_like(dX[m == 0]))
    want = f64(dY) * m
    bound = 2 * U32 * np.abs(want)
    if dtype == torch.bfloat16:
        bound = UBF * (np.abs(want) + bound) + bound
    assert np.all(np.abs(dX - want) <= bound)


@pytest.mark.parametrize("n", [1, 2, 3, 4, 5, 7, 8, 9, 15, 252, 257, 511, 514, 1020, 2048, 2055, 4099, 917,
                               65536, 100003])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("residual", [False, True])
def test_dropout_sizes(n, dtype, residual):
    check_dropout(n, 0.3, dtype, residual, 12345, 6)


@pytest.mark.parametrize("p", [0.0, 2.0 ** -18, 2.0 ** -16, 0.1, 0.5, 0.999, 1.0 - 2.0 ** -16, 1.0])
def test_dropout_probabilities(p):
    check_dropout(5000, p, torch.float32, True, 99, 0)


@pytest.mark.parametrize("seed,offset", [(0, 0), (2 ** 63 + 5, 1), (2 ** 64 - 1, 2 ** 64 - 1),
                                         (2 ** 32, 2 ** 33 + 7)])
def test_dropout_seeds(seed, offset):
    check_dropout(3001, 0.2, torch.bfloat16, True, seed, offset, shape=(3001, 1))


def test_dropout_of_infinities_and_nan():
    X = torch.full((4096,), float("nan"), device="cuda")
    X[1::2] = float("inf")
    rng = rng_pair(4, 2)
    Y = ec.dropout(X, 0.5, rng)
    keep = torch.from_numpy(ref.dropout_mask_ref(np.arange(4096), 0.5, 4, 2) != 0).cuda()
    assert torch.all(Y[~keep] == 0) and not torch.isfinite(Y[keep]).any()
    assert torch.all(ec.dropout(X, 1.0, rng) == 0)


def test_dropout_in_place_empty_and_without_rng():
    X, R, rng = torch.randn(999, device="cuda"), torch.randn(999, device="cuda"), rng_pair(1, 1)
    want = ec.dropout(X, 0.4, rng, residual=R)
    a, b = X.clone(), R.clone()
    assert ec.dropout(a, 0.4, rng, residual=R, out=a) is a and torch.equal(a, want)
    assert ec.dropout(X, 0.4, rng, residual=b, out=b) is b and torch.equal(b, want)
    assert torch.equal(ec.dropout(X, 0.0), X)
    assert ec.dropout(X[:0], 0.4, rng).numel() == 0
    with pytest.raises(ec.ECError):
        ec.dropout(X, 0.4)                                     # draws need rng
    with pytest.raises(ec.ECError):
        ec.dropout(X[1:], 0.4, rng)                            # not 16-byte aligned
    with pytest.raises(ec.ECError):
        ec.dropout(X.view(27, 37).t(), 0.4, rng)               # not contiguous
    with pytest.raises(ec.ECError):
        ec.dropout(X, 0.4, rng, residual=R.bfloat16())
    with pytest.raises(ec.ECError):
        ec.dropout(X, 0.4, rng, residual=R[:500])
    with pytest.raises(ec.ECError):
        ec.dropout(X, 0.4, rng.int())


def test_dropout_past_32_bits():
    """Blocks whose element numbers pass 2^32 (the counter's second word stays 0 until 2^35)."""
    n = 2 ** 32 + 1003
    X = torch.ones(n, dtype=torch.bfloat16, device="cuda")
    Y = ec.dropout(X, 0.25, rng_pair(3, 8), out=X)
    for at in (0, 2 ** 31 - 500, 2 ** 32 - 600, n - 1003):
        e = np.arange(at, at + 1003)
        assert np.array_equal(f64(Y[at:at + 1003]) != 0,
                              ref.dropout_mask_ref(e, 0.25, 3, 8) != 0), at


def test_dropout_on_another_stream_and_in_a_graph():
    """A captured call reads its seed and offset when it runs: every replay with another
    offset draws the mask of an eager call with that offset."""
    X, R, rng = torch.randn(4099, device="cuda"), torch.randn(4099, device="cuda"), rng_pair(5, 0)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        Y = ec.dropout(X, 0.2, rng, residual=R)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(Y, ec.dropout(X, 0.2, rng, residual=R))
    graph, out = torch.cuda.CUDAGraph(), torch.empty_like(X)
    with torch.cuda.graph(graph):
        ec.dropout(X, 0.2, rng, residual=R, out=out)
    seen = []
    for step in range(4):
        rng[1] = step
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, ec.dropout(X, 0.2, rng, residual=R))
        seen.append(out.clone())
    assert not torch.equal(seen[0], seen[1])


# ---- the training step ---------------------------------------------------------


def draw_layer(lens, d, E, h, dtype, seed, hs=0, skew=0.25):
    gen = torch.Generator().manual_seed(seed)
    n = lambda *s: torch.randn(s, generator=gen)   # noqa: E731
    N, w = int(sum(lens)), d ** -0.5
    X = ((n(N, d) * 16).round() + (n(d) * 4 * skew).round()).clamp(-96, 96) / 16
    Wg = (n(E, d) * 4).round().clamp(-15, 15) / 4 * 2.0 ** round(np.log2(w))
    t = {"X": X, "Wg": Wg, "W1": n(E, h, d) * w, "W3": n(E, h, d) * w, "W2": n(E, d, h) * w,
         "dY": n(N, d), "R": n(N, d)}
    sh = None
    if hs:
        sh = tuple((x * w).to(dtype).cuda() for x in (n(hs, d), n(hs, d), n(d, hs)))
    return {k: v.to(dtype).cuda() for k, v in t.items()}, sh


def step(t, sh, off, cap, k, inv_tau, p, rng, dloss, residual=True):
    args = (t["X"], t["Wg"], t["W1"], t["W3"], t["W2"])
    Y, loss, counts, saved = ec.tc_train_forward(*args, off, cap, k, inv_tau, shared=sh,
                                                 residual=t["R"] if residual else None, dropout=p,
                                                 rng=rng)
    g = ec.tc_train_backward(*args, t["dY"], saved, off, cap, k, inv_tau, shared=sh, dropout=p,
                             rng=rng, dloss=dloss)
    return {"Y": Y, "loss": loss, "counts": counts, **dict(zip(GRADS, g))}


def check_layer(lens, d, E, h, k, cf=0.0, dtype=torch.bfloat16, inv_tau=1.0, p=0.1, hs=0, seed=1,
                skew=0.25, residual=True, aux=True, cap=None):
    print(f"[layer] lens {lens} d {d} E {E} h {h} k {k} cf {cf} {dtype} p {p} hs {hs}", flush=True)
    t, sh = draw_layer(lens, d, E, h, dtype, seed, hs, skew)
    off = offsets(lens)
    cap = ec.tc_capacity(lens, E, k, cf) if cap is None else np.asarray(cap, np.int32)
    rng = rng_pair(seed * 1000 + 7, 2 ** 40 + seed)
    # a weight that makes the balance loss's gradient as large as the gates'
    dloss = torch.linspace(1.0, 2.0, len(lens), device="cuda") * (max(lens) * d ** 0.5) if aux else None
    got = step(t, sh, off, cap, k, inv_tau, p, rng, dloss, residual)
    torch.cuda.synchronize()
    h64 = {n: f64(v) for n, v in t.items()}
    mask = ref.dropout_mask_ref(np.arange(int(off[-1]) * d), p, seed * 1000 + 7, 2 ** 40 + seed)
    want = ref.tc_train_ref(h64["X"], h64["Wg"], h64["W1"], h64["W3"], h64["W2"], h64["dY"], off, k,
                            cap, inv_tau, None if sh is None else tuple(f64(w) for w in sh),
                            h64["R"] if residual else None, mask, None if dloss is None else f64(dloss))
    assert np.array_equal(got["counts"].cpu().numpy(), want["counts"])
    # scores of fp32: max error 1e-5 relative, as the router's
    assert np.all(np.abs(f64(got["loss"]) - want["loss"]) <= 1e-5 * np.abs(want["loss"]))
    errs = {n: rel_l2(got[n], want[n]) for n in ("Y",) + GRADS if n in want and n in got}
    print("[errs]", {n: f"{e:.1e}" for n, e in errs.items()}, flush=True)
    for n, e in errs.items():
        tol = 1e-5 if dtype == torch.float32 else (5 if n == "Y" else 10) ** 0.5 * UBF
        assert e <= tol, (n, e)
    return got, want


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("lens,d,E,h,k,cf,hs", [
    ([1], 64, 8, 64, 2, 0.0, 0),                      # one token
    ([70, 33, 0, 15], 128, 17, 64, 3, 1.0, 64),       # ragged, an empty group, dropped pairs
    ([300, 212], 128, 8, 192, 2, 1.25, 0),
    ([257], 192, 5, 128, 5, 0.0, 0),                  # every expert chosen
    ([129, 64], 64, 65, 64, 4, 0.0, 128),
    ([40, 500], 256, 130, 64, 8, 2.0, 0),
    ([130, 3], 64, 200, 64, 6, 0.0, 0),
    ([97], 64, 256, 128, 12, 1.0, 0),
])
def test_training_step(lens, d, E, h, k, cf, hs, dtype):
    check_layer(lens, d, E, h, k, cf, dtype, inv_tau=2.0, hs=hs)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_training_step_wide(dtype):
    # several row blocks per expert, widths that no tile divides, 16 partials a row and more
    check_layer([900, 433], 576, 6, 320, 3, 0.0, dtype, seed=3)
    check_layer([100, 60], 128, 4, 1088, 2, 1.0, dtype, seed=4)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_training_step_of_many_groups(dtype):
    check_layer([7, 0, 3] * 100, 64, 8, 64, 2, 1.0, dtype, seed=12)


@pytest.mark.parametrize("n,d,E,h,k,hs,dtype", [
    # bf16: which of the tile forms a product takes follows from its rows, experts and widths
    (700, 768, 4, 640, 2, 256, torch.bfloat16),     # 128 x 128, half-wide weight gradients
    (700, 64, 32, 512, 4, 0, torch.bfloat16),       # W1/W3 in 128 rows
    (700, 64, 48, 512, 8, 0, torch.bfloat16),       # ... 192
    (4000, 64, 48, 512, 2, 0, torch.bfloat16),      # ... 256
    (700, 1024, 32, 64, 4, 0, torch.bfloat16),      # W2 in 128 rows
    (700, 1024, 48, 64, 8, 0, torch.bfloat16),      # ... 192, dX in 256
    (4000, 1024, 48, 64, 2, 640, torch.bfloat16),   # ... 256; shared experts in 192 and 128
    (2500, 64, 48, 768, 4, 0, torch.bfloat16),      # dA in 256 rows
    (200, 64, 130, 64, 2, 0, torch.bfloat16),       # few rows an expert: every product streams
    (900, 256, 130, 256, 8, 0, torch.bfloat16),     # dW1/dW3 in 256 x 256
    (10000, 64, 200, 64, 8, 0, torch.bfloat16),     # dW2 in 256 x 256
    (300, 256, 130, 256, 4, 0, torch.float32),      # fp32 weight gradients in 128 x 128
    (900, 256, 3, 256, 2, 128, torch.float32),      # ... 64 x 128
])
def test_training_step_tile_forms(n, d, E, h, k, hs, dtype):
    check_layer([n], d, E, h, k, 0.0, dtype, seed=n, hs=hs)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_training_step_reads_nothing_it_has_not_written(dtype):
    """Workspaces, the saved buffer and the outputs full of NaN patterns change no bit."""
    t, sh = draw_layer([150, 0, 70], 128, 10, 192, dtype, 43, hs=64)
    dloss = torch.tensor([3.0, 4.0, 5.0], device="cuda")
    layer = ec.TcLayer(t["X"], t["Wg"], t["W1"], t["W3"], t["W2"], [0, 150, 150, 220], [20, 0, 20],
                       3, shared=sh, training=True, residual=t["R"], dropout=0.1,
                       rng=rng_pair(3, 0))
    runs = []
    for _ in range(2):
        for b in (layer.ws_f, layer.ws_b, layer.saved):
            b.fill_(0xFF)
        for b in (layer.Y, layer.loss, layer.dX, layer.dWg, layer.dW1, layer.dW3, layer.dW2,
                  *layer.dshared):
            b.fill_(float("nan"))
        layer.counts.fill_(-1)
        layer.forward()
        layer.ws_f.fill_(0xFF)
        out = layer.backward(t["dY"], dloss)
        runs.append([x.clone() for x in (layer.Y, layer.loss, layer.counts, *out)])
        for b in (layer.ws_f, layer.ws_b, layer.saved):
            b.zero_()
    assert all(torch.isfinite(x.float()).all() for x in runs[0])
    for b in (layer.ws_f, layer.ws_b, layer.saved):
        b.zero_()
    layer.forward()
    out = layer.backward(t["dY"], dloss)
    for a, b, c in zip(*runs, (layer.Y, layer.loss, layer.counts, *out)):
        assert torch.equal(a, b) and torch.equal(a, c)


def test_balance_reads_nothing_it_has_not_written():
    S = scores(700, 40, 8)
    P = ec.binding._balance_problem(S, [0, 300, 700], 4, 1.0)
    L = ec.lib()
    loss = torch.full((2,), float("nan"), device="cuda")
    counts = torch.full((2, 40), -1, dtype=torch.int32, device="cuda")
    ws = torch.full((L.ec_tc_workspace_size(P.ref, 4, 2),), 0xFF, dtype=torch.uint8, device="cuda")
    st = L.ec_tc_balance(P.ref, 4, S.data_ptr(), loss.data_ptr(), counts.data_ptr(), ws.data_ptr(),
                         ws.numel(), torch.cuda.current_stream().cuda_stream)
    assert st == 0
    a, b = ec.tc_balance(S, [0, 300, 700], 4)
    assert torch.equal(a, loss) and torch.equal(b, counts)


def test_training_step_many_rows_per_expert():
    check_layer([3001], 320, 4, 192, 2, 0.0, torch.bfloat16, seed=5)


@pytest.mark.parametrize("skew", [1.0, 3.0])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_training_step_with_experts_that_nobody_chose(skew, dtype):
    got, want = check_layer([60, 40], 128, 48, 64, 1, 0.0, dtype, seed=6, skew=skew)
    idle = want["counts"].sum(0) == 0
    assert idle.any()
    for n in ("dW1", "dW3", "dW2"):
        assert not got[n][torch.from_numpy(idle).cuda()].any()


@pytest.mark.parametrize("k", [1, 2])
def test_training_step_without_aux_dropout_or_residual(k):
    got, _ = check_layer([90, 31], 128, 12, 64, k, 1.0, torch.float32, p=0.0, residual=False,
                         aux=False, seed=7)
    if k == 1:
        assert not got["dWg"].any()     # the gate of one choice is 1: nothing steers the router


def test_training_step_with_no_capacity():
    """Nothing kept: the layer is the residual, the experts' gradients are zero and the
    router's are the balance loss's alone."""
    got, _ = check_layer([50, 20], 128, 8, 64, 2, dtype=torch.float32, cap=[0, 0], seed=8)
    for n in ("dW1", "dW3", "dW2"):
        assert not got[n].any()


def test_training_step_of_no_tokens():
    t, sh = draw_layer([0, 0], 128, 8, 64, torch.bfloat16, 1, hs=64)
    got = step(t, sh, [0, 0, 0], [0, 0], 2, 1.0, 0.1, rng_pair(1, 1),
               torch.ones(2, device="cuda"))
    assert got["Y"].shape == (0, 128) and not got["loss"].any() and not got["counts"].any()
    for n in GRADS[1:]:
        assert not got[n].any(), n


def test_training_step_dropping_everything():
    got, _ = check_layer([64], 128, 8, 64, 2, dtype=torch.bfloat16, p=1.0, aux=False, seed=9)
    for n in GRADS[:5]:
        assert not got[n].any(), n


def test_training_forward_equals_inference_without_dropout():
    """The same layer: the inference forward gates in the combine, the training one in the
    W1/W3 product, so they differ by the rounding of A and O alone."""
    t, sh = draw_layer([200, 90], 192, 12, 128, torch.bfloat16, 11, hs=64)
    args = (t["X"], t["Wg"], t["W1"], t["W3"], t["W2"], [0, 200, 290], [60, 30], 3)
    Y, _, counts, _ = ec.tc_train_forward(*args, shared=sh)
    Y2, rows = ec.tc_forward(*args, shared=sh)
    assert rel_l2(Y, f64(Y2)) <= 6 ** 0.5 * UBF
    assert int(rows[-1]) <= int(counts.sum())


def test_gradients_against_differences():
    """fp32 layer: the derivative along a direction of all arguments, with central differences
    of the layer's own forward.  The step is 2^-8 of each argument's size: the third-order term
    is of the order of 1e-4 of the derivative and the rounding of the sums (~1e-6 of their
    size, over the step) of 1e-3."""
    lens, k, p = [80, 41], 2, 0.2
    off = offsets(lens)
    t, sh = draw_layer(lens, 128, 6, 64, torch.float32, 21, hs=64)
    cap, rng = ec.tc_capacity(lens, 6, k, 0.0), rng_pair(9, 9)
    dloss = torch.tensor([200.0, 300.0], device="cuda")
    got = step(t, sh, off, cap, k, 1.0, p, rng, dloss)
    gen = torch.Generator().manual_seed(22)
    names = ("X", "Wg", "W1", "W3", "W2")

    def value(args, shared):
        Y, loss, counts, _ = ec.tc_train_forward(*args, off, cap, k, 1.0, shared=shared,
                                                 residual=t["R"], dropout=p, rng=rng)
        return float((Y.double() * t["dY"].double()).sum() + (loss.double() * dloss.double()).sum()), counts

    base = [t[n] for n in names] + list(sh)
    for moved in range(len(base)):
        v = torch.randn(base[moved].shape, generator=gen).cuda() * base[moved].std()
        vals = []
        eps = 2.0 ** -8 if names[moved % 5] not in ("X", "Wg") or moved > 4 else 2.0 ** -11
        for s in (1, -1):
            a = list(base)
            a[moved] = a[moved] + s * eps * v
            val, counts = value(a[:5], tuple(a[5:]))
            vals.append(val)
            if not torch.equal(counts, got["counts"]):
                vals = None      # a choice changed: not differentiable along this direction
                break
        name = (names + ("Ws1", "Ws3", "Ws2"))[moved]
        if vals is None:
            assert name in ("X", "Wg")
            continue
        want = float((got["d" + name].double() * v.double()).sum())
        assert (vals[0] - vals[1]) / (2 * eps) == pytest.approx(want, rel=5e-3, abs=0.05), name


def test_planned_layer_repeats_and_keeps_its_inputs():
    t, sh = draw_layer([130, 62], 128, 9, 64, torch.bfloat16, 31, hs=64)
    off, cap = [0, 130, 192], [40, 20]
    rng, dloss = rng_pair(2, 5), torch.tensor([3.0, 4.0], device="cuda")
    keep = {n: v.clone() for n, v in t.items()}
    want = step(t, sh, off, cap, 3, 1.0, 0.1, rng, dloss)
    layer = ec.TcLayer(t["X"], t["Wg"], t["W1"], t["W3"], t["W2"], off, cap, 3, shared=sh,
                       training=True, residual=t["R"], dropout=0.1, rng=rng)
    for _ in range(3):
        Y = layer.forward()
        g = layer.backward(t["dY"], dloss)
        assert torch.equal(Y, want["Y"]) and torch.equal(layer.loss, want["loss"])
        assert torch.equal(layer.counts, want["counts"])
        for n, x in zip(GRADS, g):
            assert torch.equal(x, want[n]), n
    for n, v in t.items():
        assert torch.equal(v, keep[n]), n
    assert rng.tolist() == [2, 5]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_training_step_in_a_graph(dtype):
    """A captured step replays to the eager step's bits, with another mask each time, the
    program's own eager work in between."""
    t, sh = draw_layer([150, 70], 128, 10, 64, dtype, 41, hs=64)
    off, cap = [0, 150, 220], [40, 20]
    rng, dloss = rng_pair(3, 0), torch.tensor([3.0, 4.0], device="cuda")
    mk = lambda: ec.TcLayer(t["X"], t["Wg"], t["W1"], t["W3"], t["W2"], off, cap, 3, shared=sh,   # noqa: E731
                            training=True, residual=t["R"], dropout=0.1, rng=rng)
    layer, eager = mk(), mk()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        layer.forward()
        layer.backward(t["dY"], dloss)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        layer.forward()
        layer.backward(t["dY"], dloss)
    last = None
    for i in range(4):
        rng[1] = i
        t["X"].copy_(torch.roll(t["X"], 1, 0))
        graph.replay()
        torch.cuda.synchronize()
        Y = eager.forward()
        g = eager.backward(t["dY"], dloss)
        assert torch.equal(layer.Y, Y) and torch.equal(layer.loss, eager.loss)
        for n, a, b in zip(GRADS, (layer.dX, layer.dWg, layer.dW1, layer.dW3, layer.dW2,
                                   *layer.dshared), g):
            assert torch.equal(a, b), n
        assert last is None or not torch.equal(last, Y)
        last = Y.clone()


def test_two_steps_on_two_streams():
    a, _ = draw_layer([100], 128, 8, 64, torch.bfloat16, 51)
    b, _ = draw_layer([90, 30], 128, 8, 64, torch.bfloat16, 52)
    ra, rb = rng_pair(1, 1), rng_pair(2, 2)
    wa = step(a, None, [0, 100], [100], 2, 1.0, 0.1, ra, None)
    wb = step(b, None, [0, 90, 120], [90, 30], 2, 1.0, 0.1, rb, None)
    torch.cuda.synchronize()
    s1, s2 = torch.cuda.Stream(), torch.cuda.Stream()
    with torch.cuda.stream(s1):
        ga = step(a, None, [0, 100], [100], 2, 1.0, 0.1, ra, None)
    with torch.cuda.stream(s2):
        gb = step(b, None, [0, 90, 120], [90, 30], 2, 1.0, 0.1, rb, None)
    torch.cuda.synchronize()
    for got, want in ((ga, wa), (gb, wb)):
        for n in ("Y", "loss", "counts") + GRADS[:5]:
            assert torch.equal(got[n], want[n]), n


def test_stage_events_of_the_training_step():
    from paper_2604_01622_amd.binding import BACKWARD_STAGES, FORWARD_STAGES, StageEvents
    t, _ = draw_layer([100], 128, 8, 64, torch.bfloat16, 61)
    layer = ec.TcLayer(t["X"], t["Wg"], t["W1"], t["W3"], t["W2"], [0, 100], [100], 2,
                       training=True)
    for stages, call in ((FORWARD_STAGES, layer.forward),
                         (BACKWARD_STAGES, lambda: layer.backward(t["dY"]))):
        ev = StageEvents(len(stages))
        ev.arm()
        try:
            call()
        finally:
            ev.disarm()
        torch.cuda.synchronize()
        assert all(x >= 0 for x in ev.durations_ms())


def test_operands_that_do_not_fit_are_refused():
    t, sh = draw_layer([64], 128, 8, 64, torch.bfloat16, 71, hs=64)
    good = dict(X=t["X"], Wg=t["Wg"], W1=t["W1"], W3=t["W3"], W2=t["W2"])

    def call(shared=None, off=(0, 64), cap=(64,), **kw):
        a = {**good, **kw}
        return ec.tc_train_forward(a["X"], a["Wg"], a["W1"], a["W3"], a["W2"], off, cap, 2,
                                   shared=shared)
    for kw in (dict(X=t["X"].float()), dict(W2=t["W1"]), dict(W3=t["W3"][:4]),
               dict(X=t["X"].t()), dict(Wg=t["Wg"].float()), dict(X=t["X"][:60]),
               dict(W1=t["W1"].cpu()), dict(shared=(sh[0], sh[1], sh[0])), dict(off=(0, 30, 64)),
               dict(cap=(65,))):
        with pytest.raises(ec.ECError):
            call(**kw)
    layer = ec.TcLayer(*good.values(), [0, 64], [64], 2, training=True)
    layer.forward()
    for bad in (t["dY"].float(), t["dY"][:10], t["dY"].cpu()):
        with pytest.raises(ec.ECError):
            layer.backward(bad)
    with pytest.raises(ec.ECError):
        layer.backward(t["dY"], torch.ones(2, device="cuda"))
    with pytest.raises(ec.ECError):
        ec.tc_train_backward(*good.values(), t["dY"], layer.saved[:64], [0, 64], [64], 2)


def test_calls_of_a_layer_out_of_order_are_refused():
    t = {"X": (64, 64), "Wg": (8, 64), "W1": (8, 64, 64), "W3": (8, 64, 64), "W2": (8, 64, 64)}
    t = {n: torch.zeros(s, device="cuda") for n, s in t.items()}
    off, cap = [0, 64], [64]
    layer = ec.TcLayer(*t.values(), off, cap, 2, training=True)
    with pytest.raises(ec.ECError, match="backward before forward"):
        layer.backward(t["X"])
    layer.forward()
    layer.backward(t["X"])
    later = ec.TcLayer(*t.values(), off, cap, 2, training=True, saved=layer.saved)
    later.backward(t["X"])
    with pytest.raises(ec.ECError, match="backward only"):
        later.forward()
    first = ec.TcLayer(*t.values(), off, cap, 2, training=True, backward=False)
    first.forward()
    with pytest.raises(ec.ECError, match="backward=False"):
        first.backward(t["X"])


def test_balance_gradient_of_the_step_is_the_standalone_one():
    """Without an output gradient the step's router gradients are the balance loss's alone:
    dX = dZ Wg and dWg = dZ^T X with dZ of tc_balance_backward on the layer's scores."""
    t, _ = draw_layer([90, 0, 41], 128, 12, 64, torch.float32, 81)
    off, cap, k = [0, 90, 90, 131], [90, 0, 41], 3
    t["dY"].zero_()
    dloss = torch.tensor([5.0, 7.0, -3.0], device="cuda")
    got = step(t, None, off, cap, k, 2.0, 0.0, None, dloss)
    S = ec.tc_route(t["X"], t["Wg"], off, cap, k, 2.0)[0]
    loss, counts = ec.tc_balance(S, off, k)
    assert torch.equal(counts, got["counts"])
    assert rel_l2(got["loss"], f64(loss)) <= 1e-6
    dZ = f64(ec.tc_balance_backward(S, counts, dloss, off, k, 2.0))
    assert rel_l2(got["dX"], dZ @ f64(t["Wg"])) <= 1e-5
    assert rel_l2(got["dWg"], dZ.T @ f64(t["X"])) <= 1e-5
    for n in ("dW1", "dW3", "dW2"):
        assert not got[n].any()


def test_two_blocks_trained_together():
    """As they are used: two token-choice blocks with residuals, dropout and balance losses,
    then dropout of the result, forward and backward, two steps with the offsets advanced,
    against the chained float64 oracle.  fp32, tolerance 1e-4: two layers of 1e-5 each, the
    second's inputs off by the first's error through weights of norm about 2."""
    lens, d, E, h, k, p = [50, 31], 128, 6, 64, 2, 0.2
    off, N = offsets(lens), 81
    cap = ec.tc_capacity(lens, E, k, 1.5)
    a, _ = draw_layer(lens, d, E, h, torch.float32, 91)
    b, _ = draw_layer(lens, d, E, h, torch.float32, 92)
    T = a["dY"]
    dl = torch.tensor([20.0, 30.0], device="cuda")
    w = lambda t: (t["Wg"], t["W1"], t["W3"], t["W2"])   # noqa: E731
    rngs = [rng_pair(11, 3 * i) for i in range(3)]
    for n in range(2):
        X = a["X"]
        H, la, ca, sa = ec.tc_train_forward(X, *w(a), off, cap, k, residual=X, dropout=p, rng=rngs[0])
        Z, lb, cb, sb = ec.tc_train_forward(H, *w(b), off, cap, k, residual=H, dropout=p, rng=rngs[1])
        out = ec.dropout(Z, p, rngs[2])
        dZ = ec.dropout(T, p, rngs[2])
        gb = ec.tc_train_backward(H, *w(b), dZ, sb, off, cap, k, dropout=p, rng=rngs[1], dloss=dl)
        dH = gb[0] + dZ
        ga = ec.tc_train_backward(X, *w(a), dH, sa, off, cap, k, dropout=p, rng=rngs[0], dloss=dl)
        dX = ga[0] + dH
        m = [ref.dropout_mask_ref(np.arange(N * d), p, 11, 3 * i + n).reshape(N, d) for i in range(3)]
        x64, wa, wb = f64(X), [f64(v) for v in w(a)], [f64(v) for v in w(b)]
        zero = np.zeros((N, d))
        h64 = ref.tc_train_ref(x64, *wa, zero, off, k, cap, 1.0, None, x64, m[0])["Y"]
        dz64 = f64(T) * m[2]
        rb = ref.tc_train_ref(h64, *wb, dz64, off, k, cap, 1.0, None, h64, m[1], f64(dl))
        dh64 = rb["dX"] + dz64
        ra = ref.tc_train_ref(x64, *wa, dh64, off, k, cap, 1.0, None, x64, m[0], f64(dl))
        assert np.array_equal(ca.cpu().numpy(), ra["counts"])
        assert np.array_equal(cb.cpu().numpy(), rb["counts"])
        for got, want in ((out, rb["Y"] * m[2]), (dX, ra["dX"] + dh64), (la, ra["loss"]),
                          (lb, rb["loss"]), *zip(gb[1:], (rb[x] for x in GRADS[1:5])),
                          *zip(ga[1:], (ra[x] for x in GRADS[1:5]))):
            assert rel_l2(got, want) <= 1e-4
        for r in rngs:
            r[1] += 1
