"""Token-choice training without a GPU: the oracle's formulas against their definitions,
automatic differentiation, differences and published values, and the refusals of the new entry
points, which happen on the host before anything is enqueued."""
import ctypes
import shutil
import subprocess

import numpy as np
import pytest
import torch

from oracle import ec_ref as ref
import paper_2604_01622_amd as ec
from paper_2604_01622_amd import binding, build

EC_OK, EC_ERR_ARG, EC_ERR_SHAPE, EC_ERR_CAPACITY, EC_ERR_DTYPE, EC_ERR_ALIGN, EC_ERR_WORKSPACE = range(7)
FAKE = ctypes.c_void_p(1 << 20)       # aligned, never dereferenced: validation fails first
FAR = ctypes.c_void_p(1 << 30)
MISALIGNED = ctypes.c_void_p((1 << 20) + 8)
NONE3 = (None, None, None)


# ---- the oracle ----------------------------------------------------------------


@pytest.mark.parametrize("counter,key,want", [
    # the published test vectors of the generator (the distribution's known answers)
    ([0, 0, 0, 0], [0, 0], [0x6627e8d5, 0xe169c58d, 0xbc57ac4c, 0x9b00dbd8]),
    ([0xffffffff] * 4, [0xffffffff] * 2, [0x408f276d, 0x41c83b0e, 0xa20bc7c6, 0x6d5451fd]),
    ([0x243f6a88, 0x85a308d3, 0x13198a2e, 0x03707344], [0xa4093822, 0x299f31d0],
     [0xd16cfe09, 0x94fdcceb, 0x5001e420, 0x24126ea1]),
])
def test_philox_known_answers(counter, key, want):
    assert [int(w) for w in ref.philox4x32_ref(np.array(counter), key)] == want


def test_dropout_mask_follows_element_seed_and_offset():
    e = np.arange(1 << 14)
    m = ref.dropout_mask_ref(e, 0.25, 7, 3)
    assert set(np.unique(m)) == {0.0, 65536 / (65536 - 16384)}
    # 2^14 draws at 1/4: standard deviation of the mean 0.0034
    assert abs((m == 0).mean() - 0.25) < 5 * 0.0034
    assert np.array_equal(m[100:200], ref.dropout_mask_ref(e[100:200], 0.25, 7, 3))
    assert not np.array_equal(m, ref.dropout_mask_ref(e, 0.25, 7, 4))
    assert not np.array_equal(m, ref.dropout_mask_ref(e, 0.25, 8, 3))
    # the elements of a block of eight draw the halves of its four words, low halves first
    w = ref.philox4x32_ref(np.array([5, 0, 3, 0]), (7, 0))
    draws = np.array([int(x) >> s & 0xffff for x in w for s in (0, 16)])
    assert np.array_equal(m[40:48] != 0, draws >= 16384)
    assert np.all(ref.dropout_mask_ref(e, 1.0, 7, 3) == 0)
    assert np.all(ref.dropout_mask_ref(e, 2.0 ** -18, 7, 3) == 1)


def test_balance_loss_by_hand():
    # an even load with equal scores costs 1, a collapsed router E / k
    S = np.full((6, 3), 1 / 3)
    S += np.array([np.roll([1e-3, 0, -1e-3], i) for i in range(6)])
    loss, counts = ref.tc_balance_ref(S, [0, 6, 6], 1)
    assert np.array_equal(counts, [[2, 2, 2], [0, 0, 0]])
    assert loss == pytest.approx([1.0, 0.0])
    S = np.array([[1.0, 0.0, 0.0, 0.0]] * 5)
    loss, counts = ref.tc_balance_ref(S, [0, 5], 1)
    assert loss == pytest.approx([4.0]) and counts.tolist() == [[5, 0, 0, 0]]
    # equal scores: the lower experts
    assert ref.tc_balance_ref(np.full((3, 5), 0.2), [0, 3], 2)[1].tolist() == [[3, 3, 0, 0, 0]]


@pytest.mark.parametrize("top_k,cf,shared,inv_tau", [(2, 1.0, False, 1.0), (3, 0.0, True, 2.0),
                                                     (1, 1.5, False, 0.5)])
def test_training_gradients_against_autograd_and_differences(top_k, cf, shared, inv_tau):
    rng = np.random.default_rng(17 + top_k)
    lens, d, E, h = [9, 0, 14], 6, 5, 4
    off = np.concatenate([[0], np.cumsum(lens)])
    N = int(off[-1])
    mk = lambda *s: rng.standard_normal(s)   # noqa: E731
    X, Wg, W1, W3, W2 = mk(N, d), mk(E, d), mk(E, h, d), mk(E, h, d), mk(E, d, h)
    dY, R = mk(N, d), mk(N, d)
    sh = (mk(3, d), mk(3, d), mk(d, 3)) if shared else None
    cap = ref.tc_capacity_ref(lens, E, top_k, cf)
    mask = ref.dropout_mask_ref(np.arange(N * d), 0.3, 5, 9).reshape(N, d)
    dloss = np.array([1.5, 2.0, -0.7])
    r = ref.tc_train_ref(X, Wg, W1, W3, W2, dY, off, top_k, cap, inv_tau, sh, R, mask, dloss)
    choice, kept = r["fwd"]["choice"], r["fwd"]["kept"]

    def total(X, Wg, W1, W3, W2, *s):
        S = torch.softmax(X @ Wg.T * inv_tau, 1)
        pick = S.gather(1, torch.from_numpy(choice))
        gate = pick / pick.sum(1, keepdim=True)
        Y = torch.zeros_like(X)
        for i in range(N):
            for n in range(top_k):
                if kept[i, n]:
                    j = int(choice[i, n])
                    a = torch.nn.functional.silu(W1[j] @ X[i]) * (W3[j] @ X[i])
                    Y = Y.index_add(0, torch.tensor([i]), (gate[i, n] * (W2[j] @ a))[None])
        if s:
            Y = Y + (torch.nn.functional.silu(X @ s[0].T) * (X @ s[1].T)) @ s[2].T
        Y = torch.from_numpy(R) + torch.from_numpy(mask) * Y
        out = (Y * torch.from_numpy(dY)).sum()
        for g, L in enumerate(lens):
            if L:
                c = torch.from_numpy(r["counts"][g]).double()
                out = out + dloss[g] * E / (top_k * L) * (c * S[off[g]:off[g + 1]].mean(0)).sum()
        return out, Y

    names = ["X", "Wg", "W1", "W3", "W2"] + (["Ws1", "Ws3", "Ws2"] if shared else [])
    args = [X, Wg, W1, W3, W2] + list(sh or ())
    leaves = [torch.from_numpy(a.copy()).requires_grad_() for a in args]
    val, Y = total(*leaves)
    val.backward()
    assert np.allclose(Y.detach().numpy(), r["Y"], rtol=1e-12, atol=1e-12)
    for n, t in zip(names, leaves):
        assert np.allclose(t.grad.numpy(), r["d" + n], rtol=1e-10, atol=1e-11), n
    # central differences along a direction in all arguments at once
    dirs = [rng.standard_normal(a.shape) for a in args]
    step = 1e-6
    with torch.no_grad():
        up, dn = (float(total(*[torch.from_numpy(a + s * step * v) for a, v in zip(args, dirs)])[0])
                  for s in (1, -1))
    want = sum(float((r["d" + n] * v).sum()) for n, v in zip(names, dirs))
    assert (up - dn) / (2 * step) == pytest.approx(want, rel=1e-6)
    if top_k == 1:   # one choice has the gate 1: only the balance loss reaches the router
        z = ref.tc_train_ref(X, Wg, W1, W3, W2, dY, off, 1, cap, inv_tau, sh, R, mask, None)
        assert not z["dWg"].any()


# ---- host arithmetic ------------------------------------------------------------


def test_one_round_splits_cover_every_row(tmp_path):
    """The splits of a shared expert's weight gradient whose tiles are one round: at most 256
    tiles wherever one split has fewer, whole chunks of 64 rows, every row once."""
    cc = shutil.which("g++")
    if cc is None:
        pytest.skip("needs g++")
    src, exe = tmp_path / "split.cpp", tmp_path / "split"
    src.write_text(r"""
#include <cstdio>
#include "row_split.h"
int main() {
  long bad = 0;
  for (int n = 1; n <= 9000; ++n)
    for (int m = 64; m <= 8192; m *= 2) {
      const int s = ec::wgrad_splits_one_round(m, 640, n);
      const ec::RowSplit r = ec::split_rows(n, s, 64);
      const int tiles = ((m + 255) / 256) * 3;
      bad += s < 1 || r.parts() > s || (long)r.full * r.chunk + r.last != n || r.last >= r.chunk ||
             (s > 1 && s * tiles > 256);
    }
  std::printf("%ld %d\n", bad, ec::wgrad_splits_one_round(1472, 640, 5451));
}
""")
    subprocess.run([cc, "-std=c++17", "-O2", "-Wall", "-Werror", "-I", build.CSRC, str(src), "-o",
                    str(exe)], check=True, capture_output=True, text=True)
    out = subprocess.run([str(exe)], check=True, capture_output=True, text=True, timeout=60).stdout
    assert out.split() == ["0", "14"]


# ---- refusals ------------------------------------------------------------------


def _problem(**kw):
    args = dict(n_tokens=256, d_model=128, n_experts=8, d_ff=64, group_offsets=[0, 100, 256],
                capacity=[100, 156], inv_temperature=1.0, dtype=torch.bfloat16)
    args.update(kw)
    return binding.Problem(**args)


def _desc(p=0.1, rng=1 << 21, residual=None):
    return binding._DropoutDesc(p, rng, residual)


def test_balance_refusals():
    L, P = ec.lib(), _problem()
    ws = 1 << 30
    ok = (FAKE, FAKE, FAKE, FAKE, ws, None)
    for k in (0, 9, -1):
        assert L.ec_tc_balance(P.ref, k, *ok) == EC_ERR_ARG
        assert L.ec_tc_balance_backward(P.ref, k, FAKE, FAKE, FAKE, FAKE, None) == EC_ERR_ARG
    assert L.ec_tc_balance(None, 2, *ok) == EC_ERR_ARG
    for n in range(4):
        a = [FAKE] * 4
        a[n] = None
        assert L.ec_tc_balance(P.ref, 2, *a, ws, None) == EC_ERR_ARG
        a[n] = MISALIGNED
        assert L.ec_tc_balance(P.ref, 2, *a, ws, None) == EC_ERR_ALIGN
        a = [FAKE] * 4
        a[n] = None
        assert L.ec_tc_balance_backward(P.ref, 2, *a, None) == EC_ERR_ARG
        a[n] = MISALIGNED
        assert L.ec_tc_balance_backward(P.ref, 2, *a, None) == EC_ERR_ALIGN
    need = L.ec_tc_workspace_size(P.ref, 2, 2)
    assert need > 0
    assert L.ec_tc_balance(P.ref, 2, FAKE, FAKE, FAKE, FAKE, need - 1, None) == EC_ERR_WORKSPACE
    bad = _problem(n_tokens=255)
    assert L.ec_tc_balance(bad.ref, 2, *ok) == EC_ERR_SHAPE
    assert L.ec_tc_workspace_size(bad.ref, 2, 2) == 0
    assert L.ec_tc_workspace_size(P.ref, 2, 5) == 0


def test_dropout_refusals():
    L = ec.lib()

    def call(dtype=1, n=1000, d=None, X=FAKE, Y=FAR):
        return L.ec_dropout(dtype, n, ctypes.byref(d or _desc()), X, Y, None)

    assert call(dtype=2) == EC_ERR_DTYPE
    assert call(n=-1) == EC_ERR_SHAPE and call(n=1 << 40) == EC_ERR_SHAPE
    assert L.ec_dropout(1, 10, None, FAKE, FAR, None) == EC_ERR_ARG
    for p in (-0.1, 1.01, float("nan"), float("inf")):
        assert call(d=_desc(p)) == EC_ERR_ARG
    assert call(d=_desc(0.1, None)) == EC_ERR_ARG
    assert call(d=_desc(0.1, (1 << 21) + 8)) == EC_ERR_ALIGN
    assert call(d=_desc(residual=(1 << 22) + 4)) == EC_ERR_ALIGN
    assert call(X=None) == EC_ERR_ARG and call(Y=None) == EC_ERR_ARG
    assert call(X=MISALIGNED) == EC_ERR_ALIGN and call(Y=MISALIGNED) == EC_ERR_ALIGN
    # overlaps other than the same buffer
    assert call(Y=ctypes.c_void_p((1 << 20) + 1984)) == EC_ERR_ARG
    assert call(d=_desc(residual=(1 << 30) + 16)) == EC_ERR_ARG
    assert call(d=_desc(residual=(1 << 30) - 1984)) == EC_ERR_ARG
    # nothing to do: accepted without a launch
    assert call(n=0, X=None, Y=None) == EC_OK


def test_training_refusals():
    L, P = ec.lib(), _problem()
    sv, wf = L.ec_tc_saved_size(P.ref, 2), L.ec_tc_workspace_size(P.ref, 2, 3)
    wb = L.ec_tc_workspace_size(P.ref, 2, 4)
    assert sv > 0 and wf > 0 and wb > 0
    d = _desc()

    def fwd(k=2, drop=d, a=None, sv_=sv, ws_=wf, P=P):
        a = dict(dict(X=FAKE, Wg=FAKE, W1=FAKE, W3=FAKE, W2=FAKE, Y=FAR, loss=FAKE, counts=FAKE,
                      saved=FAKE, ws=FAKE), **(a or {}))
        return L.ec_tc_train_forward(P.ref, k, ctypes.byref(drop), a["X"], a["Wg"], a["W1"],
                                     a["W3"], a["W2"], *NONE3, a["Y"], a["loss"], a["counts"],
                                     a["saved"], sv_, a["ws"], ws_, None)

    def bwd(k=2, drop=d, a=None, sv_=sv, ws_=wb, P=P):
        over, a = a, dict({n: FAKE for n in ("X", "Wg", "W1", "W3", "W2", "dY", "dloss", "saved", "dX",
                                    "dWg", "dW1", "dW3", "dW2", "ws")}, dX=FAR)
        a.update(over or {})
        return L.ec_tc_train_backward(P.ref, k, ctypes.byref(drop), a["X"], a["Wg"], a["W1"],
                                      a["W3"], a["W2"], *NONE3, a["dY"], a["dloss"], a["saved"],
                                      sv_, a["dX"], a["dWg"], a["dW1"], a["dW3"], a["dW2"],
                                      *NONE3, a["ws"], ws_, None)

    for call, names in ((fwd, ("X", "Wg", "W1", "W3", "W2", "Y", "loss", "counts", "saved", "ws")),
                        (bwd, ("X", "Wg", "W1", "W3", "W2", "dY", "saved", "dX", "dWg", "dW1",
                               "dW3", "dW2", "ws"))):
        for n in names:
            assert call(a={n: None}) == EC_ERR_ARG, n
            assert call(a={n: MISALIGNED}) == EC_ERR_ALIGN, n
        assert call(k=0) == EC_ERR_ARG and call(k=9) == EC_ERR_ARG
        assert call(drop=_desc(2.0)) == EC_ERR_ARG
        assert call(drop=_desc(0.5, None)) == EC_ERR_ARG
        assert call(sv_=sv - 1) == EC_ERR_WORKSPACE
        assert call(P=_problem(capacity=[101, 3])) == EC_ERR_CAPACITY
        assert call(P=_problem(d_shared=64)) == EC_ERR_ARG      # shared weights missing
    assert bwd(a={"dloss": MISALIGNED}) == EC_ERR_ALIGN
    assert fwd(ws_=wf - 1) == EC_ERR_WORKSPACE and bwd(ws_=wb - 1) == EC_ERR_WORKSPACE
    assert fwd(drop=_desc(residual=1 << 30)) == EC_ERR_ARG      # the residual is Y
    assert fwd(a={"Y": ctypes.c_void_p((1 << 20) + 4096)}) == EC_ERR_ARG    # Y inside X
    for n in ("X", "dY"):
        assert bwd(a={"dX": FAKE, ("dY" if n == "X" else "X"): ctypes.c_void_p(1 << 31)}) == EC_ERR_ARG
    assert bwd(a={"dX": ctypes.c_void_p((1 << 20) + 256 * 128 * 2 - 16)}) == EC_ERR_ARG
    # the backward's [rows, 2 h] buffer is within 2^31 elements; the inference forward's
    # [rows, h] one may be twice as long
    big = binding.Problem(65536, 64, 8, 16384, [0, 65536], [65536], 1.0, torch.bfloat16)
    assert L.ec_tc_saved_size(big.ref, 1) == 0 and "32-bit" in L.ec_last_error().decode()
    assert L.ec_tc_workspace_size(big.ref, 1, 3) == 0 and L.ec_tc_workspace_size(big.ref, 1, 4) == 0
    assert L.ec_tc_workspace_size(big.ref, 1, 1) > 0


def test_size_queries_of_training():
    L, P = ec.lib(), _problem()
    N, E, R, d, h = 256, 8, 512, 128, 64
    assert L.ec_tc_saved_size(P.ref, 2) >= 3 * N * E * 4 + 8 * R + 3 * R * h * 2
    capped = _problem(capacity=[5, 7])
    assert L.ec_tc_saved_size(capped.ref, 2) < L.ec_tc_saved_size(P.ref, 2)
    shared = _problem(d_shared=128)
    assert L.ec_tc_saved_size(shared.ref, 2) - L.ec_tc_saved_size(P.ref, 2) == 3 * N * 128 * 2
    assert L.ec_tc_workspace_size(P.ref, 2, 4) >= R * (d + 2 * h) * 2 + N * 64 * 2 + N * d * 2
    empty = _problem(n_tokens=0, group_offsets=[0, 0], capacity=[0])
    for mode in (2, 3, 4):
        assert L.ec_tc_workspace_size(empty.ref, 2, mode) > 0


def test_binding_refuses_host_tensors_and_wrong_operands():
    S = torch.zeros((4, 8))
    with pytest.raises(ec.ECError, match="GPU"):
        ec.tc_balance(S, [0, 4], 2)
    with pytest.raises(ec.ECError, match="N, E"):
        ec.tc_balance(S[0], [0, 4], 2)
    with pytest.raises(ec.ECError, match="GPU"):
        ec.dropout(S, 0.1, torch.zeros(2, dtype=torch.int64))
    with pytest.raises(ec.ECError, match="unsupported storage dtype"):
        ec.dropout(S.half(), 0.1)
    with pytest.raises(ec.ECError, match="tensor"):
        ec.dropout(None, 0.1)
    X, Wg = torch.zeros((4, 64)), torch.zeros((8, 64))
    W1, W2 = torch.zeros((8, 64, 64)), torch.zeros((8, 64, 64))
    with pytest.raises(ec.ECError, match="GPU"):
        ec.tc_train_forward(X, Wg, W1, W1, W2, [0, 4], [4], 2)
    with pytest.raises(ec.ECError, match="training=True"):
        ec.TcLayer(X, Wg, W1, W1, W2, [0, 4], [4], 2, dropout=0.1)
