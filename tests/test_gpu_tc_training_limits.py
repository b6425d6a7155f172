"""The training step of token choice at the largest sizes: buffers of packed rows whose bytes
end just below 2^32 (dH) and offsets past 2^31, against the same mathematics in 64 bits."""
import pytest
import torch

import paper_2604_01622_amd as ec

pytestmark = pytest.mark.gpu


def ffn_step(x, w1, w3, w2, g, gy, out):
    """One expert's rows: adds to out and returns y and dx of the rows, and <gy, y / g>."""
    h1, h3 = x @ w1.t(), x @ w3.t()
    s = torch.sigmoid(h1)
    a = h1 * s * h3
    y = a @ w2.t()
    q = (gy * y).sum(1)
    do = g[:, None] * gy
    da = do @ w2
    d1, d3 = da * h3 * (s + h1 * s * (1 - s)), da * h1 * s
    out["dW1"] += d1.t() @ x
    out["dW3"] += d3.t() @ x
    out["dW2"] += do.t() @ a
    return g[:, None] * y, d1 @ w1 + d3 @ w3, q


@pytest.mark.parametrize("N,E,k,dtype", [
    (2 ** 20 - 1, 1, 1, torch.bfloat16),        # one expert has every row
    (2 ** 19 - 5, 3, 2, torch.bfloat16),
    (2 ** 19 - 5, 3, 2, torch.float32),
])
def test_most_rows(N, E, k, dtype):
    d, h = 64, 1024
    assert 0.99 * 2 ** 31 < N * k * 2 * h < 2 ** 31
    print(f"[limits] N {N} E {E} k {k} {dtype}", flush=True)
    gen = torch.Generator(device="cuda").manual_seed(N + k)
    draw = lambda *s: torch.randn(s, generator=gen, device="cuda")   # noqa: E731
    w = d ** -0.5
    # logits on a grid: the same number whatever the order of its sum
    X = ((draw(N, d) * 16).round().clamp(-96, 96) / 16).to(dtype)
    Wg = ((draw(E, d) * 4).round().clamp(-15, 15) / 4 * 0.125).to(dtype)
    W1, W3, W2 = ((draw(E, h, d) * w).to(dtype), (draw(E, h, d) * w).to(dtype),
                  (draw(E, d, h) * h ** -0.5).to(dtype))
    dY = draw(N, d).to(dtype)
    off, dloss = [0, N // 2, N], torch.tensor([N / 4.0, N / 2.0], device="cuda")
    layer = ec.TcLayer(X, Wg, W1, W3, W2, off, [N // 2, N - N // 2], k, training=True)
    Y = layer.forward()
    grads = dict(zip(("dX", "dWg", "dW1", "dW3", "dW2"), layer.backward(dY, dloss)))
    torch.cuda.synchronize()

    z = X.double() @ Wg.double().t()
    S = torch.softmax(z, 1)
    chosen = torch.zeros_like(S).scatter_(1, torch.sort(z, dim=1, descending=True,
                                                        stable=True).indices[:, :k], 1.0)
    gate = S * chosen / (S * chosen).sum(1, keepdim=True)
    counts = torch.stack([chosen[a:b].sum(0) for a, b in zip(off[:-1], off[1:])])
    assert torch.equal(layer.counts.double(), counts)
    want = {"Y": torch.zeros(N, d, dtype=torch.double, device="cuda")}
    want["dX"] = torch.zeros_like(want["Y"])
    for n, v in (("dW1", W1), ("dW3", W3), ("dW2", W2)):
        want[n] = torch.zeros(v.shape, dtype=torch.double, device="cuda")
    q = torch.zeros_like(S)
    for j in range(E):
        rows = chosen[:, j].nonzero()[:, 0]
        for part in rows.split(1 << 17):
            sums = {n: want[n][j] for n in ("dW1", "dW3", "dW2")}
            y, dx, q[part, j] = ffn_step(X[part].double(), W1[j].double(), W3[j].double(),
                                         W2[j].double(), gate[part, j], dY[part].double(), sums)
            want["Y"].index_add_(0, part, y)
            want["dX"].index_add_(0, part, dx)
    dZ = gate * (q - (gate * q).sum(1, keepdim=True))
    for g, (a, b) in enumerate(zip(off[:-1], off[1:])):
        c = dloss[g].double() * E * counts[g] / (k * float(b - a) ** 2)
        dZ[a:b] += S[a:b] * (c - S[a:b] @ c[:, None])
    want["dX"] += dZ @ Wg.double()
    want["dWg"] = dZ.t() @ X.double()
    got = {"Y": Y, **grads}
    errs = {n: float((got[n].double() - v).norm() / v.norm()) for n, v in want.items() if v.any()}
    print("[errs]", {n: f"{e:.1e}" for n, e in errs.items()}, flush=True)
    # bf16: n roundings of 2^-8 at most on the way, independent of each other (Y: A, O, Y;
    # gradients: H1, H3, A, dH, dXe, dZ, two writes of dX, and the sums below).  fp32 sums of
    # up to N terms in one chain: rounding errors of random sign, sqrt(N) 2^-24 of the sum's
    # size, beside products of 1024 terms, four in a chain.
    chain = N ** 0.5 * 2.0 ** -24
    for n, e in errs.items():
        assert e <= chain + (1e-5 if dtype == torch.float32 else 3 * 2.0 ** -8), (n, e)
    # the last tokens, whose rows lie furthest
    tail = slice(N - 64, N)
    for n in ("Y", "dX"):
        e = float((got[n][tail].double() - want[n][tail]).norm() / want[n][tail].norm())
        assert e <= (1e-5 if dtype == torch.float32 else 3 * 2.0 ** -8), (n, e)
