"""Plain 64-bit forms of the 8-bit operators and of the balance loss, on host tensors,
and their error bars."""
import math

import torch

import _moe as M


def pack(X):
    """(Q, scales) by the definition: scales rounded to FP32, Q decided in 64 bits (127 x is
    exact there, and a quotient of 31-bit numbers that is no border is 2^-33 away from one)."""
    x = X.double()
    top = x.abs().amax(-1) if x.shape[-1] else x.new_zeros(x.shape[:-1])
    bad = ~torch.isfinite(x).all(-1)
    top = torch.where(bad, 0.0, top)
    q = torch.round(127 * torch.where(bad[..., None], 0.0, x) / torch.where(top > 0, top, 1.0)[..., None])
    scales = (top.float() / 127)
    return q.to(torch.int8), torch.where(bad, math.nan, scales)


def product(X, xs, W, ws, offsets, rows):
    """Y in 64 bits; W: E x N x K.  Rows outside X are zeros."""
    x = M.gathered(X, rows)
    R = len(x)
    src = torch.arange(R) if rows is None else rows.long()
    ok = (src >= 0) & (src < X.shape[0])
    s = torch.zeros(R, dtype=torch.float64)
    s[ok] = xs.double()[src[ok]]
    Y = torch.zeros((R, W.shape[1]), dtype=torch.float64)
    e_of = torch.zeros(R, dtype=torch.int64) if offsets is None else M.expert_of(offsets, R)
    for e in range(W.shape[0]):
        at = (e_of == e) & ok
        if at.any():
            Y[at] = (x[at] @ W[e].double().T) * s[at, None] * ws[e].double()
    return Y


def product_bar(Y, dtype):
    """The sum is exact; it is rounded to FP32 and multiplied twice there, then rounded to
    the type."""
    return 2.0 ** -24 * 3.1 * Y.abs() + M.rounded(Y, dtype)


def spans(starts, T):
    """[first, end) of each sequence as the operators read the starts."""
    if starts is None:
        return [(0, T)]
    out = []
    for s in range(len(starts) - 1):
        lo = min(max(int(starts[s]), 0), T) if s else 0
        out.append((lo, min(max(int(starts[s + 1]), lo), T)))
    return out


def token(x):
    """Softmax and log of its sum of one token's logits (64 bits), None if it has none."""
    x = torch.where(torch.isnan(x), -math.inf, x)
    m = x.max()
    if m == -math.inf:
        return None
    e = torch.where(x == m, 1.0, torch.where(x > -math.inf, torch.exp(x - m), 0.0))
    return e / e.sum(), m + torch.log(e.sum())


def balance(logits, ids, starts):
    """loss, zloss, counts, tokens by the definition, one token at a time, and a bar of
    zloss: each z is off by the sum's error (34 + 36 units of 2^-24, relative, see LOSS_BAR)
    and its own roundings."""
    x = logits.double()
    T, E = x.shape
    loss, zloss, bar, counts, tokens = [], [], [], [], []
    for lo, hi in spans(starts, T):
        p, z, zb, n = torch.zeros(E, dtype=torch.float64), 0.0, 0.0, 0
        for t in range(lo, hi):
            got = token(x[t])
            if got is None:
                continue
            n += 1
            p += got[0]
            v = float(got[1])
            z += v * v
            zb += 2 * abs(v) * (70 + 4 * abs(v)) + 32 * v * v
        c = ids[lo:hi].long().reshape(-1)
        c = torch.bincount(c[(c >= 0) & (c < E)], minlength=E)
        C = int(c.sum())
        loss.append(float(E * (c * p).sum() / (C * n)) if n and C else 0.0)
        zloss.append(z / n if n else 0.0)
        bar.append((zb * 2.0 ** -24 + 2.0 ** -40) / max(n, 1))
        counts.append(c)
        tokens.append(n)
    d = lambda v: torch.tensor(v, dtype=torch.float64)  # noqa: E731
    return d(loss), d(zloss), torch.stack(counts), torch.tensor(tokens), d(bar)


# Of the loss, a sum of positive terms, relative: an exponential of a logit at most 16 below
# the largest is off by 16 + 16 + 2 units of 2^-24 (the difference's rounding, that of its
# product with log2 e, the exponential's own and the constant's); the sum of up to 512 (32 to
# a lane and 4 exchanges) by that + 36; the quotient by 2; the sum over a workgroup's tokens
# by up to 24 additions and 6 exchanges.
LOSS_BAR = 2.0 ** -24 * (34 + 34 + 36 + 2 + 30 + 2)


def balance_grad(logits, counts, tokens, dloss, dzloss, starts):
    """The gradient of the definition and its bar: p is off by 106 units of 2^-24 as above,
    the mean of the shares by 106 + 36 more, z by 70 and its own roundings, the products and
    the difference by 6."""
    x = logits.double()
    T, E = x.shape
    out, bar = torch.zeros((T, E), dtype=torch.float64), torch.zeros((T, E), dtype=torch.float64)
    for s, (lo, hi) in enumerate(spans(starts, T)):
        n = int(tokens[s])
        if n <= 0:
            continue
        f = counts[s].double()
        f = f / max(1.0, float(f.sum()))
        dl = float(dloss[s]) * E / n
        dz = 0.0 if dzloss is None else float(dzloss[s]) * 2 / n
        for t in range(lo, hi):
            got = token(x[t])
            if got is None:
                continue
            p, z = got
            mean = (p * f).sum()
            out[t] = p * (dl * (f - mean) + (dz * z if dz else 0.0))
            bar[t] = 2.0 ** -24 * 260 * p * (abs(dl) * (f + mean) + (abs(dz) * (1 + abs(z)) if dz else 0.0))
    return out, bar
