"""Plain 64-bit forms of the mixture-of-experts operators, on host tensors, and
the error bars of the tests (each derived from the roundings it names)."""
import math

import numpy as np
import torch

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
# half a unit in the last place of the output's type, relative, and the absolute
# half spacing of its subnormals
HALF_ULP = {torch.float32: (2.0 ** -24, 2.0 ** -150), torch.bfloat16: (2.0 ** -8, 2.0 ** -134),
            torch.float16: (2.0 ** -11, 2.0 ** -25)}


def rounded(exact, dtype):
    """The error of one rounding of `exact` to dtype (and of an FP32 before it)."""
    rel, least = HALF_ULP[dtype]
    return rel * 1.01 * exact.abs() + least


def route(logits, k, scope):
    """ids, weights, offsets, rows, slots by the definition, one token at a time."""
    x = logits.double().numpy()
    T, E = x.shape
    ids = np.full((T, k), -1, np.int64)
    weights = np.zeros((T, k))
    for t in range(T):
        there = [e for e in range(E) if x[t, e] > -math.inf]
        chosen = sorted(there, key=lambda e: (-x[t, e], e))[:k]
        if not chosen:
            continue
        m = x[t, chosen[0]]
        ex = lambda e: 1.0 if x[t, e] == m else math.exp(x[t, e] - m)  # noqa: E731
        total = sum(ex(e) for e in (chosen if scope == "chosen" else there))
        ids[t, :len(chosen)] = chosen
        weights[t, :len(chosen)] = [ex(e) / total for e in chosen]
    pairs = sorted((ids[t, j], t, j) for t in range(T) for j in range(k) if ids[t, j] >= 0)
    offsets = np.zeros(E + 1, np.int64)
    rows = np.full(T * k, -1, np.int64)
    slots = np.full((T, k), -1, np.int64)
    for r, (e, t, j) in enumerate(pairs):
        rows[r], slots[t, j] = t, r
        offsets[e + 1:] += 1
    return tuple(torch.from_numpy(a) for a in (ids, weights, offsets, rows, slots))


def route_grad(logits, ids, dweights, scope):
    """d loss / d logits of the weights' formula, by its Jacobian."""
    x = logits.double()
    out = torch.zeros_like(x)
    for t in range(x.shape[0]):
        chosen = [int(e) for e in ids[t] if e >= 0]
        if not chosen:
            continue
        among = chosen if scope == "chosen" else [e for e in range(x.shape[1]) if x[t, e] > -math.inf]
        p = torch.softmax(x[t, among], 0)
        g = torch.zeros(len(among), dtype=torch.float64)
        for j, e in enumerate(chosen):
            g[among.index(e)] = float(dweights[t, j])
        out[t, among] = p * (g - (p * g).sum())
    return out


def expert_of(offsets, R):
    """The expert of each row (-1: none) from offsets as the operators read them."""
    e_of = torch.full((R,), -1, dtype=torch.int64)
    lo = 0
    for e in range(len(offsets) - 1):
        lo = min(max(int(offsets[e]), 0), R) if e else 0
        hi = min(max(int(offsets[e + 1]), lo), R)
        e_of[lo:hi] = e
    return e_of


def gathered(X, rows):
    """X[rows] in 64 bits, zeros for the entries outside X."""
    X = X.double()
    if rows is None:
        return X
    rows = rows.long()
    ok = (rows >= 0) & (rows < X.shape[0])
    out = torch.zeros((len(rows), X.shape[1]), dtype=torch.float64)
    out[ok] = X[rows[ok]]
    return out


def grouped(X, W, offsets, rows):
    """(Y, the same sums of magnitudes); W: E x K x N."""
    x = gathered(X, rows)
    R = len(x)
    Y = torch.zeros((R, W.shape[2]), dtype=torch.float64)
    S = torch.zeros_like(Y)
    e_of = expert_of(offsets, R)
    for e in range(W.shape[0]):
        at = e_of == e
        if at.any():
            Y[at] = x[at] @ W[e].double()
            S[at] = x[at].abs() @ W[e].double().abs()
    return Y, S


def wgrad(X, dY, offsets, rows):
    x, dy = gathered(X, rows), dY.double()
    E = len(offsets) - 1
    out = torch.zeros((E, x.shape[1], dy.shape[1]), dtype=torch.float64)
    S = torch.zeros_like(out)
    e_of = expert_of(offsets, len(dy))
    for e in range(E):
        at = e_of == e
        out[e] = x[at].T @ dy[at]
        S[e] = x[at].abs().T @ dy[at].abs()
    return out, S


def product_bar(exact, S, K, dtype):
    """Sums of K terms on matrix instructions: at most one rounding for each 8
    terms and eight more (the sets' sum, the left-out component products of
    FP32, 3 x 2^-26 of S), each up to 2^-23 of the sum of magnitudes; one
    rounding to the output's type."""
    return 2.0 ** -23 * (K / 8 + 8) * S + rounded(exact, dtype)


def unpacked(Q, scales, mins):
    """W in 64 bits of 4-bit entries, and a bound of the terms the kernel adds:
    (16 + q) s, 24 s and the offset."""
    q = Q.long()
    q = torch.stack((q % 16, q // 16), -1).flatten(-2).double()
    group = q.shape[-1] // scales.shape[-1]
    s = scales.double().repeat_interleave(group, -1)
    if mins is None:
        return (q - 8) * s, 55 * s.abs()
    m = mins.double().repeat_interleave(group, -1)
    return q * s + m, 47 * s.abs() + m.abs()


def check(got, exact, bar, what=""):
    got = got.detach().cpu().double()
    assert got.shape == exact.shape, (what, got.shape, exact.shape)
    assert torch.isfinite(got).all(), what
    off = (got - exact).abs()
    assert (off <= bar).all(), f"{what}: {float((off / bar.clamp(min=1e-300)).max()):.3g} times the bar"
