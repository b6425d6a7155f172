"""The operators of token-choice training, over the range of sizes that users call them at.

A case names one pass through one operator:

  kind "balance"  the balance loss of token choice with its per-expert counts
                  (``tc_balance``) and, with ``grad``, the gradient that it sends to the
                  router's logits (``tc_balance_backward``)
  kind "dropout"  ``dropout`` of a tensor from a counter-based generator, onto a residual
                  or (``residual`` false) alone, which is also its backward pass
  kind "train"    a training step of the token-choice layer: ``tc_train_forward`` with the
                  balance loss, dropout and the residual of a block, then
                  ``tc_train_backward``

``api`` says how the program holds the layer: "layer" keeps a ``TcLayer`` planned once,
"call" uses the functions, which size and allocate what they need on every call.  Token
groups (sequences) are written as text, "2048x8" or "700,333,1015".
"""
import math

import numpy as np
import torch

own = False


def _ec():
    """The package: only the framework's own calls need it."""
    import paper_2604_01622_amd as ec
    return ec


def _balance(name, groups, E, top_k, **more):
    case = {"kind": "balance", "groups": groups, "E": E, "top_k": top_k, "grad": True,
            "inv_tau": 1.0, "spread": 1.0, "coarse": False}
    return _named(name, case, more)


def _dropout(name, shape, p, **more):
    case = {"kind": "dropout", "shape": shape, "p": p, "residual": True, "dtype": "bf16"}
    return _named(name, case, more)


def _train(name, groups, d, E, h, top_k, **more):
    case = {"kind": "train", "api": "call", "groups": groups, "d": d, "E": E, "h": h, "hs": 0,
            "top_k": top_k, "cf": 0.0, "p": 0.0, "residual": True, "aux": True, "inv_tau": 1.0,
            "skew": 0.25, "dtype": "bf16"}
    return _named(name, case, more)


def _named(name, case, more):
    if name:
        case["name"] = name
    case.update(more)
    return case


def listed():
    return [
        # a short sequence and few experts: a unit test, a toy model; two launches' latency
        _balance("balance_1x96_E8", "96", 8, 2),
        # the batch of the benchmark's layer, its sequences each with a loss of its own
        _balance("balance_8x2048_E64", "2048x8", 64, 8),
        # packed documents of unequal length, scores of a router that works in bf16, where
        # equal scores are common
        _balance("balance_ragged_E40", "1531,77,1,1999,640,1203", 40, 6, coarse=True, inv_tau=2.0),
        # a large batch as one group over fine experts
        _balance("balance_1x65536_E256", "65536", 256, 8, spread=1.5),
        # few rows of a width that no vector divides: the smallest call
        _dropout("dropout_f32_odd", "7x131", 0.25, dtype="f32"),
        # the output of the benchmark's layer, added to the residual stream ...
        _dropout("dropout_16384x2048", "16384x2048", 0.1),
        # ... and the gradient that goes back through it
        _dropout("dropout_back_16384x2048", "16384x2048", 0.1, residual=False),
        # a wide batch in full precision
        _dropout("dropout_f32_32768x4096", "32768x4096", 0.15, dtype="f32"),
        # the training step of the benchmark's layer under token choice, dropless top 8
        _train("train_8x2048_E64", "2048x8", 2048, 64, 1024, 8, api="layer", p=0.1),
        # a micro-batch of one short sequence: short and empty expert buffers, the weights
        # and their gradients are most of the bytes
        _train("train_1x512_E64", "512", 2048, 64, 1024, 8, p=0.1, skew=1.0),
        # packed documents, a capacity that drops pairs, shared experts, widths that no
        # tile divides
        _train("train_ragged_E40", "1531,77,1999,640,1203", 1472, 40, 832, 4, hs=640, cf=1.25,
               p=0.05, inv_tau=2.0, skew=0.5),
        # a small model in full precision
        _train("train_f32_ragged", "700,333,1015", 1024, 16, 512, 2, dtype="f32", cf=1.5, p=0.1,
               skew=0.5),
    ]


def _lengths(case):
    out = []
    for part in case["groups"].split(","):
        n, _, times = part.partition("x")
        out += [int(n)] * (int(times) if times else 1)
    return out


def _shape(case):
    rows, cols = case["shape"].split("x")
    return int(rows), int(cols)


def _log(rng, lo, hi):
    return math.exp(rng.uniform(math.log(lo), math.log(hi)))


def _width(rng, lo, hi):
    return max(1, round(_log(rng, lo, hi) / 64)) * 64


def draw(rng):
    """One more case of the ranges above."""
    most = {}
    for c in listed():
        key = (c["kind"], c.get("dtype"))
        if key not in most or work(c)["bytes"] > work(most[key])["bytes"]:
            most[key] = c
    while True:
        kind = rng.choice(["balance", "dropout", "train", "train"])
        if kind == "balance":
            E = int(_log(rng, 4, 257))
            lens = [max(1, int(_log(rng, 1, 32768))) for _ in range(rng.randint(1, 12))]
            case = _balance("", ",".join(map(str, lens)), E, rng.randint(1, max(1, min(E, 12))),
                            grad=rng.random() < 0.75, inv_tau=rng.choice([0.5, 1.0, 2.0]),
                            spread=round(rng.uniform(0.2, 3.0), 2), coarse=rng.random() < 0.3)
        elif kind == "dropout":
            case = _dropout("", "%dx%d" % (int(_log(rng, 1, 40000)), int(_log(rng, 16, 5000))),
                            round(rng.uniform(0.01, 0.6), 3), residual=rng.random() < 0.5,
                            dtype=rng.choice(["bf16", "bf16", "f32"]))
        else:
            f32 = rng.random() < 0.3
            E = rng.choice([4, 8, 16, 17, 32] if f32 else [8, 16, 24, 40, 64, 64, 96, 128])
            d = _width(rng, 64, 1024) if f32 else _width(rng, 256, 2560)
            h = _width(rng, 64, 512) if f32 else _width(rng, 128, 1536)
            lens = [int(_log(rng, 30, 1024 if f32 else 4096)) for _ in range(rng.randint(1, 6))]
            case = _train("", ",".join(map(str, lens)), d, E, h,
                          rng.choice([k for k in (1, 2, 4, 8) if k <= E // 2]),
                          api=rng.choice(["layer", "call"]), cf=rng.choice([0.0, 1.0, 1.25, 2.0]),
                          p=rng.choice([0.0, 0.05, 0.1, 0.2]), residual=rng.random() < 0.7,
                          aux=rng.random() < 0.8, inv_tau=rng.choice([0.5, 1.0, 1.0, 2.0]),
                          skew=rng.choice([0.0, 0.25, 0.5, 1.0]),
                          hs=_width(rng, 128, 1024) if rng.random() < 0.25 else 0,
                          dtype="f32" if f32 else "bf16")
        if kind == "train" and case["top_k"] == 1:
            case["aux"] = True   # one choice has the gate 1: only the balance loss steers it
        top = work(most[(kind, case.get("dtype"))])
        w = work(case)
        if w["flops"] <= top["flops"] and w["bytes"] <= top["bytes"]:
            return case


def _dtype(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _offsets(case):
    return np.concatenate([[0], np.cumsum(_lengths(case))]).astype(np.int32)


def _capacity(case):
    """Tokens that an expert keeps of each group, in plain arithmetic."""
    cf, k, E = case["cf"], case["top_k"], case["E"]
    return [n if cf <= 0 else min(n, math.ceil(cf * k * n / E - 1e-9)) for n in _lengths(case)]


def _threshold(p):
    """Dropped 16-bit draws, and the factor of what is kept."""
    t = int(np.rint(p * 65536.0))
    return t, (65536.0 / (65536 - t) if t < 65536 else 0.0)


def _dloss(case, noise):
    """Weights of the groups' balance losses beside a main loss that is a sum over tokens."""
    lens = torch.tensor(_lengths(case), dtype=torch.float32, device="cuda")
    return 0.01 * lens * (1.0 + 0.1 * noise[torch.arange(len(lens), device="cuda") % len(noise)])


def _inputs(case, seed):
    """Tensors of the case, from the seed alone."""
    gen = torch.Generator(device="cuda")

    def normal(i, shape, std=1.0):
        gen.manual_seed(seed * 16 + i)
        return torch.randn(shape, generator=gen, device="cuda") * std

    rng = torch.tensor([seed * 7919 + 11, 3 * seed + 5], dtype=torch.int64, device="cuda")
    if case["kind"] == "balance":
        N, E = sum(_lengths(case)), case["E"]
        logits = normal(0, (N, E)) + normal(1, (E,), 0.3 * case["spread"])
        logits = logits * case["spread"] * case["inv_tau"]
        if case["coarse"]:
            logits = logits.bfloat16().float()
        ex = torch.exp(logits - logits.amax(1, keepdim=True))
        return {"S": ex / ex.sum(1, keepdim=True), "dloss": _dloss(case, normal(2, (E,)))}
    dt = _dtype(case)
    if case["kind"] == "dropout":
        v = {"X": normal(0, _shape(case)).to(dt), "rng": rng, "R": None}
        if case["residual"]:
            v["R"] = normal(1, _shape(case), 2.0).to(dt)
        return v
    # X and Wg lie on a grid coarse enough that a logit is the same number whatever the order
    # of its sum, so that every program chooses the same experts (equal logits among them)
    N, d, E, h, hs = sum(_lengths(case)), case["d"], case["E"], case["h"], case["hs"]
    unit = 2.0 ** round(math.log2(1.0 / math.sqrt(d)))
    lean = (normal(9, (d,)) * 4 * case["skew"]).round()
    X = ((normal(0, (N, d)) * 16).round() + lean).clamp(-96, 96) / 16
    Wg = (normal(1, (E, d)) * 4).round().clamp(-15, 15) / 4 * unit
    w = 1.0 / math.sqrt(d)
    v = {"X": X.to(dt), "Wg": Wg.to(dt), "W1": normal(2, (E, h, d), w).to(dt),
         "W3": normal(3, (E, h, d), w).to(dt), "W2": normal(4, (E, d, h), w).to(dt),
         "dY": normal(5, (N, d)).to(dt), "R": None, "rng": rng, "shared": None, "dloss": None}
    if case["residual"]:
        v["R"] = normal(10, (N, d)).to(dt)
    if case["aux"]:
        v["dloss"] = _dloss(case, normal(11, (E,)))
    if hs:
        v["shared"] = (normal(6, (hs, d), w).to(dt), normal(7, (hs, d), w).to(dt),
                       normal(8, (d, hs), w).to(dt))
    return v


def prepare(case, seed):
    st = _inputs(case, seed)
    st["case"] = case
    if case["kind"] == "dropout":
        return st
    st["off"] = _offsets(case)
    if case["kind"] == "balance":
        return st
    st["cap"] = np.asarray(_capacity(case), dtype=np.int32)
    if own and case["api"] == "layer":
        st["layer"] = _ec().TcLayer(st["X"], st["Wg"], st["W1"], st["W3"], st["W2"], st["off"],
                                    st["cap"], case["top_k"], case["inv_tau"],
                                    shared=st["shared"], training=True, residual=st["R"],
                                    dropout=case["p"], rng=st["rng"])
    return st


_GRADS = ("dX", "dWg", "dW1", "dW3", "dW2", "dWs1", "dWs3", "dWs2")


def run(st):
    return _run_own(st) if own else _run_plain(st)


def _run_own(st):
    ec, case = _ec(), st["case"]
    if case["kind"] == "balance":
        loss, counts = ec.tc_balance(st["S"], st["off"], case["top_k"])
        out = {"loss": loss, "counts": counts}
        if case["grad"]:
            out["dZ"] = ec.tc_balance_backward(st["S"], counts, st["dloss"], st["off"],
                                               case["top_k"], case["inv_tau"])
        return out
    if case["kind"] == "dropout":
        return {"Y": ec.dropout(st["X"], case["p"], st["rng"], residual=st["R"])}
    layer = st.get("layer")
    if layer is not None:
        Y = layer.forward()
        loss, counts = layer.loss, layer.counts
        grads = layer.backward(st["dY"], st["dloss"])
    else:
        args = (st["X"], st["Wg"], st["W1"], st["W3"], st["W2"])
        plan = (st["off"], st["cap"], case["top_k"], case["inv_tau"])
        Y, loss, counts, saved = ec.tc_train_forward(*args, *plan, shared=st["shared"],
                                                     residual=st["R"], dropout=case["p"],
                                                     rng=st["rng"])
        grads = ec.tc_train_backward(*args, st["dY"], saved, *plan, shared=st["shared"],
                                     dropout=case["p"], rng=st["rng"], dloss=st["dloss"])
    out = {"Y": Y, "loss": loss, "counts": counts, **dict(zip(_GRADS, grads))}
    out["dWg"] = out["dWg"].to(st["Wg"].dtype)   # a parameter's gradient has its type
    return out


def _pairs(case):
    """Token-expert pairs that are computed (at most)."""
    return min(case["top_k"] * sum(_lengths(case)), case["E"] * sum(_capacity(case)))


def work(case):
    if case["kind"] == "dropout":
        n = math.prod(_shape(case))
        size = 2 if case["dtype"] == "bf16" else 4
        return {"bytes": n * size * (3 if case["residual"] else 2) + 16, "flops": 2 * n}
    N, E, G = sum(_lengths(case)), case["E"], len(_lengths(case))
    if case["kind"] == "balance":
        # scores in, gradients out, counts and losses; a sum and k maxima, then a dot
        # product and the gradient, per score
        grad = case["grad"]
        return {"bytes": 4 * (N * E * (2 if grad else 1) + G * E + G),
                "flops": N * E * (6 if grad else 2)}
    d, h, hs = case["d"], case["h"], case["hs"]
    size = 2 if case["dtype"] == "bf16" else 4
    weights = (E * d + 3 * E * d * h + 3 * d * hs) * size
    flops = 6 * d * (h * _pairs(case) + hs * N) + 2 * N * d * E
    # X, dY, the residual and the weights in; Y, dX and the weights' gradients out
    return {"bytes": (4 + case["residual"]) * N * d * size + 2 * weights, "flops": 3 * flops}


# ---- the plain forms: elementary operations, 32 bits -------------------------------


def _mulhilo(a, b):
    """Upper and lower halves of the 64-bit product of 32-bit values held in int64."""
    t = a * (b & 0xFFFF)
    u = a * (b >> 16) + (t >> 16)
    return u >> 16, ((u & 0xFFFF) << 16) | (t & 0xFFFF)


def _keep_plain(n, p, rng):
    """True where element e of n is kept.  Philox4x32-10 of counter (e // 8, offset) under
    key (seed) gives eight 16-bit draws, low halves first; a draw below the threshold drops."""
    t, _ = _threshold(p)
    block = torch.arange((n + 7) // 8, dtype=torch.int64, device="cuda")
    seed, offset = rng[0], rng[1]
    c = [block & 0xFFFFFFFF, block >> 32, (offset & 0xFFFFFFFF).expand_as(block),
         ((offset >> 32) & 0xFFFFFFFF).expand_as(block)]
    k0, k1 = seed & 0xFFFFFFFF, (seed >> 32) & 0xFFFFFFFF
    for _ in range(10):
        h0, l0 = _mulhilo(c[0], 0xD2511F53)
        h1, l1 = _mulhilo(c[2], 0xCD9E8D57)
        c = [h1 ^ c[1] ^ k0, l1, h0 ^ c[3] ^ k1, l0]
        k0, k1 = (k0 + 0x9E3779B9) & 0xFFFFFFFF, (k1 + 0xBB67AE85) & 0xFFFFFFFF
    draws = torch.stack([part for w in c for part in (w & 0xFFFF, w >> 16)], dim=1)
    return draws.reshape(-1)[:n] >= t


def _dropout_plain(x, p, rng):
    """x with the dropped elements zero and the others scaled, in 32 bits."""
    if _threshold(p)[0] == 0:
        return x
    keep = _keep_plain(x.numel(), p, rng).reshape(x.shape)
    return torch.where(keep, x * _threshold(p)[1], torch.zeros_like(x))


def _chosen_plain(S, k):
    """1 for each row's k largest scores, ties to the lower index."""
    best = torch.sort(S, dim=1, descending=True, stable=True).indices[:, :k]
    return torch.zeros_like(S).scatter_(1, best, 1.0)


def _balance_plain(S, chosen, off, k):
    G, E = len(off) - 1, S.shape[1]
    loss = torch.zeros(G, device="cuda")
    counts = torch.zeros(G, E, dtype=torch.int32, device="cuda")
    for g in range(G):
        a, b = int(off[g]), int(off[g + 1])
        if b > a:
            c, mean = chosen[a:b].sum(0), S[a:b].double().sum(0) / (b - a)
            counts[g] = c.int()
            loss[g] = (E * (c.double() / (k * (b - a)) * mean).sum()).float()
    return loss, counts


def _balance_back_plain(S, counts, dloss, off, k, inv_tau):
    # in 64 bits: under an even load the difference is far below its terms
    dZ, E = torch.zeros_like(S), S.shape[1]
    for g in range(len(off) - 1):
        a, b = int(off[g]), int(off[g + 1])
        if b > a:
            s = S[a:b].double()
            dS = dloss[g].double() * E * counts[g].double() / (float(k) * (b - a) * (b - a))
            dZ[a:b] = (s * (dS - (s * dS).sum(1, keepdim=True)) * inv_tau).float()
    return dZ


def _run_plain(st):
    case = st["case"]
    if case["kind"] == "balance":
        S, off, k = st["S"], st["off"], case["top_k"]
        loss, counts = _balance_plain(S, _chosen_plain(S, k), off, k)
        out = {"loss": loss, "counts": counts}
        if case["grad"]:
            out["dZ"] = _balance_back_plain(S, counts, st["dloss"], off, k, case["inv_tau"])
        return out
    if case["kind"] == "dropout":
        y = _dropout_plain(st["X"].float(), case["p"], st["rng"])
        return {"Y": (y if st["R"] is None else y + st["R"].float()).to(st["X"].dtype)}
    return _train_plain(st)


def _train_plain(st):
    case, off, k, E = st["case"], st["off"], st["case"]["top_k"], st["case"]["E"]
    dt, tau = st["X"].dtype, st["case"]["inv_tau"]
    X, Wg, dY = st["X"].float(), st["Wg"].float(), st["dY"].float()
    logits = X @ Wg.t() * tau
    ex = torch.exp(logits - logits.amax(1, keepdim=True))
    S = ex / ex.sum(1, keepdim=True)
    chosen = _chosen_plain(S, k)
    loss, counts = _balance_plain(S, chosen, off, k)
    gate = S * chosen / (S * chosen).sum(1, keepdim=True)
    kept = torch.zeros_like(chosen, dtype=torch.bool)
    for g, cap in enumerate(st["cap"]):
        a, b = int(off[g]), int(off[g + 1])
        kept[a:b] = (chosen[a:b] > 0) & (torch.cumsum(chosen[a:b], 0) <= int(cap))
    dYm = _dropout_plain(dY, case["p"], st["rng"])
    Y, dX, q = torch.zeros_like(X), torch.zeros_like(X), torch.zeros_like(S)
    grads = {n: torch.zeros(st[n[1:]].shape, dtype=dt, device="cuda") for n in ("dW1", "dW3", "dW2")}
    for j in range(E):
        i = torch.nonzero(kept[:, j])[:, 0]
        if i.numel() == 0:
            continue
        w1, w3, w2 = st["W1"][j].float(), st["W3"][j].float(), st["W2"][j].float()
        x, gy, g = X[i], dYm[i], gate[i, j, None]
        h1, h3 = x @ w1.t(), x @ w3.t()
        sg = 1.0 / (1.0 + torch.exp(-h1))
        act = h1 * sg * h3
        Y.index_add_(0, i, g * (act @ w2.t()))
        da = gy @ w2
        q[i, j] = (da * act).sum(1)
        da = da * g
        d1, d3 = da * h3 * sg * (1 + h1 * (1 - sg)), da * h1 * sg
        dX.index_add_(0, i, d1 @ w1 + d3 @ w3)
        grads["dW1"][j], grads["dW3"][j] = (d1.t() @ x).to(dt), (d3.t() @ x).to(dt)
        grads["dW2"][j] = (gy.t() @ (act * g)).to(dt)
    if st["shared"] is not None:
        w1, w3, w2 = (w.float() for w in st["shared"])
        h1, h3 = X @ w1.t(), X @ w3.t()
        sg = 1.0 / (1.0 + torch.exp(-h1))
        act = h1 * sg * h3
        Y += act @ w2.t()
        da = dYm @ w2
        d1, d3 = da * h3 * sg * (1 + h1 * (1 - sg)), da * h1 * sg
        dX += d1 @ w1 + d3 @ w3
        grads.update(dWs1=(d1.t() @ X).to(dt), dWs3=(d3.t() @ X).to(dt),
                     dWs2=(dYm.t() @ act).to(dt))
    Y = _dropout_plain(Y, case["p"], st["rng"])
    if st["R"] is not None:
        Y = Y + st["R"].float()
    dZ = gate * (q - (gate * q).sum(1, keepdim=True)) * tau
    if st["dloss"] is not None:
        dZ = dZ + _balance_back_plain(S, counts, st["dloss"], off, k, tau)
    dX = dX + dZ @ Wg
    return {"Y": Y.to(dt), "loss": loss, "counts": counts, "dX": dX.to(dt),
            "dWg": (dZ.t() @ X).to(dt), **grads}


# ---- the same in 64 bits, from the definitions --------------------------------------


def _keep64(n, p, rng):
    """The kept elements, from the generator's definition in unsigned 64-bit arithmetic."""
    u32, mask = np.uint64(32), np.uint64(0xFFFFFFFF)
    seed, offset = (np.uint64(x & 0xFFFFFFFFFFFFFFFF) for x in rng.tolist())
    x0 = np.arange((n + 7) // 8, dtype=np.uint64)
    x1, x0 = x0 >> u32, x0 & mask
    x2, x3 = np.full_like(x0, offset & mask), np.full_like(x0, offset >> u32)
    for r in range(10):
        k0 = np.uint64((int(seed & mask) + r * 0x9E3779B9) % 2 ** 32)
        k1 = np.uint64((int(seed >> u32) + r * 0xBB67AE85) % 2 ** 32)
        a, b = x0 * np.uint64(0xD2511F53), x2 * np.uint64(0xCD9E8D57)
        x0, x1, x2, x3 = (b >> u32) ^ x1 ^ k0, b & mask, (a >> u32) ^ x3 ^ k1, a & mask
    words = np.stack([x0, x1, x2, x3], axis=1).astype("<u4")
    draws = words.view("<u2").reshape(-1)[:n]
    return torch.from_numpy(draws.astype(np.int32) >= _threshold(p)[0])


def _mask64(shape, p, rng):
    """Factors of the elements: 0 or the scale."""
    t, scale = _threshold(p)
    if t == 0:
        return torch.ones(shape, dtype=torch.float64, device="cuda")
    return _keep64(math.prod(shape), p, rng).reshape(shape).cuda().double() * scale


def _ranked64(scores, k):
    """Truth values of each row's k first experts by (larger score, lower index)."""
    idx = torch.arange(scores.shape[1], device="cuda")
    out = torch.zeros(scores.shape, dtype=torch.bool, device="cuda")
    left = scores.clone()
    for _ in range(k):
        top = left.amax(1, keepdim=True)
        first = torch.where(left == top, idx, scores.shape[1]).amin(1, keepdim=True)
        out |= idx == first
        left = torch.where(idx == first, -math.inf, left)
    return out


def exact(case, seed):
    v = _inputs(case, seed)
    if case["kind"] == "balance":
        S, off, k, E = v["S"].double(), _offsets(case), case["top_k"], case["E"]
        took = _ranked64(S, k)
        loss, dZ = [], []
        for g, n in enumerate(_lengths(case)):
            s, c = S[off[g]:off[g + 1]], took[off[g]:off[g + 1]].double().sum(0)
            coef = E * c / (k * float(n) ** 2)
            loss.append((coef * s.sum(0)).sum())
            b = coef * v["dloss"][g].double()
            dZ.append(case["inv_tau"] * s * (b - s @ b[:, None]))
        out = {"loss": torch.stack(loss), "counts": None}
        if case["grad"]:
            out["dZ"] = torch.cat(dZ)
        return out
    if case["kind"] == "dropout":
        y = v["X"].double() * _mask64(_shape(case), case["p"], v["rng"])
        return {"Y": y if v["R"] is None else y + v["R"].double()}
    return _train64(case, v)


def _ffn64(x, w1, w3):
    a, b = x @ w1.t(), x @ w3.t()
    s = torch.sigmoid(a)
    return a, b, s


def _train64(case, v):
    N, d, E, k = sum(_lengths(case)), case["d"], case["E"], case["top_k"]
    off, lens = _offsets(case), _lengths(case)
    X, Wg, tau = v["X"].double(), v["Wg"].double(), case["inv_tau"]
    z = X @ Wg.t() * tau
    S = torch.softmax(z, dim=1)
    took = _ranked64(z, k)
    gate = torch.softmax(torch.where(took, z, torch.full_like(z, -math.inf)), dim=1)
    keep = took.clone()
    loss, b = [], torch.zeros_like(S)
    for g, cap in enumerate(_capacity(case)):
        rows = slice(int(off[g]), int(off[g + 1]))
        keep[rows] &= took[rows].double().cumsum(0) <= cap
        coef = E * took[rows].double().sum(0) / (k * float(lens[g]) ** 2)
        loss.append((coef * S[rows].sum(0)).sum())
        if v["dloss"] is not None:
            b[rows] = coef * v["dloss"][g].double()
    m = _mask64((N, d), case["p"], v["rng"])
    gy = v["dY"].double() * m
    acc, dX = torch.zeros_like(X), torch.zeros_like(X)
    dgate = torch.zeros_like(S)
    out = {n: torch.zeros(v[n[1:]].shape, dtype=torch.float64, device="cuda")
           for n in ("dW1", "dW3", "dW2")}
    for j in range(E):
        i = keep[:, j].nonzero().flatten()
        w1, w3, w2 = (v[n][j].double() for n in ("W1", "W3", "W2"))
        a, c, s = _ffn64(X[i], w1, w3)
        ffn = (a * s * c) @ w2.t()
        acc[i] += gate[i, j, None] * ffn
        dgate[i, j] = (gy[i] * ffn).sum(1)
        dout = gy[i] * gate[i, j, None]
        dh = dout @ w2
        da, dc = dh * c * (s + a * s * (1 - s)), dh * a * s
        dX[i] += da @ w1 + dc @ w3
        out["dW1"][j], out["dW3"][j] = da.t() @ X[i], dc.t() @ X[i]
        out["dW2"][j] = dout.t() @ (a * s * c)
    if v["shared"] is not None:
        w1, w3, w2 = (w.double() for w in v["shared"])
        a, c, s = _ffn64(X, w1, w3)
        acc += (a * s * c) @ w2.t()
        dh = gy @ w2
        da, dc = dh * c * (s + a * s * (1 - s)), dh * a * s
        dX += da @ w1 + dc @ w3
        out.update(dWs1=da.t() @ X, dWs3=dc.t() @ X, dWs2=gy.t() @ (a * s * c))
    Y = acc * m
    if v["R"] is not None:
        Y = Y + v["R"].double()
    # a softmax over the chosen logits, and the balance loss through the softmax over all
    dz = gate * (dgate - (gate * dgate).sum(1, keepdim=True))
    dz = (dz + S * (b - (S * b).sum(1, keepdim=True))) * tau
    return {"Y": Y, "loss": torch.stack(loss), "counts": None, "dX": dX + dz @ Wg,
            "dWg": dz.t() @ X, **out}
