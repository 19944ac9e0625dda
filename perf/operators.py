"""Timed cases of the mixture-of-experts operators: the choice of each token's
experts and the order of their rows, the products with the experts' matrices
(forward and both gradients), the weighted sum of the experts' outputs, and the
products with 4-bit expert matrices that serve single tokens.

A case is a plain dict.  ``op`` is one of

  route    logits (T x E) -> the k experts of each token, their weights and the
           rows' order by expert; ``train``: the gradient of the logits too
  combine  y[t] = sum_j weights[t, j] z[slot(t, j)]; ``train``: the gradients of
           z and of the weights too
  product  y[r] = x[r] W[e(r)] for R rows ordered by expert, W stored E x K x N
           (``transb`` "N") or E x N x K ("T"); ``gather``: x[r] is row rows[r]
           of T token rows.  The gradient of the rows is the same call with the
           other ``transb``
  wgrad    dW[e] = sum over the rows r of e of x[r]^T dy[r], stored as W
  q4       y[r] = x[r] W[e(r)]^T with W (E x N x K) in 4 bits, one scale (and
           with ``mins`` one offset) for each ``group`` entries along K

``own`` says which side ``run`` computes: False, the plain form in elementary
torch operations in 32 bits; True, the library's operators.  Inputs are drawn
on the GPU from the seed alone.
"""
import math

import numpy as np
import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZES = {"f32": 4, "bf16": 2, "f16": 2}


def listed():
    return [
        # the router of a single token in a decoding loop: latency alone
        {"name": "route-1x64", "op": "route", "type": "f32", "T": 1, "E": 64, "k": 8,
         "scope": "all", "mask": "none", "train": False},
        # the router of a training step, some of its tokens padding (no expert at all)
        {"name": "route-16384x128-train", "op": "route", "type": "bf16", "T": 16384, "E": 128,
         "k": 8, "scope": "chosen", "mask": "padding", "train": True},
        # the experts' outputs of a small decoding batch put together
        {"name": "combine-16x4096", "op": "combine", "type": "f32", "T": 16, "D": 4096, "k": 8,
         "train": False},
        # the same in a training step with its gradients; the largest call by bytes
        {"name": "combine-8192x2048-train", "op": "combine", "type": "bf16", "T": 8192, "D": 2048,
         "k": 8, "train": True},
        # a decoding batch of few rows for each expert: the matrices' bytes bound it
        {"name": "product-f32-32rows", "op": "product", "type": "f32", "R": 32, "E": 32, "N": 2048,
         "K": 1024, "transb": "N", "gather": True},
        # single precision, the library's own accuracy: first matrix of an expert, its
        # token rows read through the router's order
        {"name": "product-f32-8192", "op": "product", "type": "f32", "R": 8192, "E": 8, "N": 2048,
         "K": 2048, "transb": "N", "gather": True},
        # the gradient of the rows with odd extents: no tile or vector boundary is met
        {"name": "product-f32-odd", "op": "product", "type": "f32", "R": 4999, "E": 13, "N": 1501,
         "K": 777, "transb": "T", "gather": False},
        # a training step of many small experts; the largest call by operations
        {"name": "product-bf16-131072", "op": "product", "type": "bf16", "R": 131072, "E": 64,
         "N": 1024, "K": 2048, "transb": "T", "gather": True},
        # the gradient of the experts' matrices in that step
        {"name": "wgrad-bf16-65536", "op": "wgrad", "type": "bf16", "R": 65536, "E": 64,
         "N": 1024, "K": 2048, "transb": "T", "gather": True},
        # one token through a dense 4-bit matrix
        {"name": "q4-bf16-1x4096", "op": "q4", "type": "bf16", "R": 1, "E": 1, "N": 4096,
         "K": 4096, "group": 128, "mins": False},
        # sixteen tokens with eight experts each, fine groups with offsets
        {"name": "q4-f16-moe", "op": "q4", "type": "f16", "R": 128, "E": 64, "N": 2048,
         "K": 2048, "group": 32, "mins": True},
        # single-precision activations of a speculative batch
        {"name": "q4-f32-40x8192", "op": "q4", "type": "f32", "R": 40, "E": 1, "N": 8192,
         "K": 8192, "group": 64, "mins": False},
    ]


MAX_PRODUCT = 2 * 131072 * 1024 * 2048     # operations of the largest listed product
MAX_COMBINE = 8192 * 8 * 2048              # entries of the largest listed sum


def _log(rng, lo, hi):
    """A whole number spread over the logarithm of [lo, hi]."""
    return min(hi, max(lo, int(round(lo * (hi / lo) ** rng.random()))))


def _extent(rng, lo, hi):
    """A matrix extent: half of them multiples of 64, the others any number."""
    n = _log(rng, lo, hi)
    if rng.random() < 0.5:
        n = max(64, n // 64 * 64)
    return n + 1 if n == 3 * 1024 else n


def draw(rng):
    """One more case of the listed ranges."""
    while True:
        op = rng.choice(["route", "combine", "product", "product", "product", "wgrad", "q4", "q4"])
        kind = rng.choice(["f32", "bf16", "f16"])
        if op == "route":
            E = rng.choice([8, 13, 16, 32, 60, 64, 128])
            return {"op": op, "type": kind, "T": _log(rng, 1, 16384), "E": E,
                    "k": rng.randint(1, 8), "scope": rng.choice(["all", "chosen"]),
                    "mask": rng.choice(["none", "padding", "limited"]),
                    "train": rng.random() < 0.5}
        if op == "combine":
            c = {"op": op, "type": kind, "T": _log(rng, 1, 8192), "D": _extent(rng, 64, 4096),
                 "k": rng.randint(1, 8), "train": rng.random() < 0.5}
            if c["T"] * c["k"] * c["D"] <= MAX_COMBINE:
                return c
            continue
        if op == "q4":
            group = rng.choice([32, 64, 128])
            E = rng.choice([1, 1, 8, 16, 64])
            c = {"op": op, "type": kind, "R": _log(rng, 1, 64 if E == 1 else 128), "E": E,
                 "N": _extent(rng, 64, 8192), "K": group * _log(rng, 2, 8192 // group),
                 "group": group, "mins": rng.random() < 0.5}
            if c["K"] == 3 * 1024:
                c["K"] += group
            if min(E, c["R"]) * c["N"] * c["K"] <= 64 * 2048 * 2048:
                return c
            continue
        c = {"op": op, "type": kind, "R": _log(rng, 1 if op == "product" else 64, 131072),
             "E": rng.choice([4, 8, 13, 32, 64]), "N": _extent(rng, 64, 4096),
             "K": _extent(rng, 64, 4096), "transb": rng.choice("NT"),
             "gather": rng.random() < 0.5}
        top = MAX_PRODUCT if kind != "f32" else MAX_PRODUCT // 4
        if (2 * c["R"] * c["N"] * c["K"] <= top and c["R"] * max(c["N"], c["K"]) <= 131072 * 2048
                and c["E"] * c["N"] * c["K"] <= 64 * 2048 * 1024):
            return c


# ---------------------------------------------------------------------------
# Inputs.

def _counts(case, seed):
    """Rows of each expert, unevenly loaded; a few rows belong to none (their
    token was padding), and one expert in sixteen gets nothing."""
    rng = np.random.default_rng([int(seed), 5])
    R, E = case["R"], case["E"]
    if E == 1:
        return np.array([R])
    p = rng.gamma(4.0, size=E)
    p[rng.permutation(E)[:E // 16]] = 0.0
    return rng.multinomial(R - R // 50, p / p.sum())


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed))
    dt = DTYPES[case["type"]]

    def normal(*shape, scale=1.0, dtype=dt):
        x = torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32)
        return x.mul_(scale).to(dtype)

    op = case["op"]
    s = {"case": case}
    if op == "route":
        T, E, k = case["T"], case["E"], case["k"]
        # some experts are liked more than others
        logits = normal(T, E, scale=1.5, dtype=torch.float32) + normal(E, dtype=torch.float32)
        if case["mask"] == "padding":
            logits[torch.rand(T, generator=gen, device="cuda") < 0.1] = -math.inf
        elif case["mask"] == "limited":
            logits[torch.rand((T, E), generator=gen, device="cuda") < 0.5] = -math.inf
        s["logits"] = logits.to(dt)
        if case["train"]:
            s["dweights"] = normal(T, k, dtype=torch.float32)
        return s
    if op == "combine":
        T, D, k = case["T"], case["D"], case["k"]
        # the order of a router: a permutation of the rows; one token in forty is padding
        s["z"] = normal(T * k, D)
        w = torch.rand((T, k), generator=gen, device="cuda") + 0.05
        dead = torch.rand(T, generator=gen, device="cuda") < 0.025
        alive = (~dead)[:, None].expand(T, k).reshape(-1)
        key = torch.where(alive, torch.rand(T * k, generator=gen, device="cuda"), 2.0)
        order = torch.argsort(key, stable=True)
        slots = torch.empty_like(order)
        slots[order] = torch.arange(T * k, device="cuda")
        s["slots"] = torch.where(alive, slots, -1).view(T, k).to(torch.int32)
        s["rows"] = torch.where(alive[order], order // k, -1).to(torch.int32)
        s["weights"] = (w / w.sum(1, keepdim=True)).masked_fill_(dead[:, None], 0.0)
        if case["train"]:
            s["dy"] = normal(T, D)
        return s
    counts = _counts(case, seed)
    R, E, N, K = case["R"], case["E"], case["N"], case["K"]
    offsets = np.concatenate([[0], np.cumsum(counts)])
    # what the host of a plain implementation plans with: the experts that have
    # rows, and the most rows of one
    s["active"] = torch.from_numpy(np.flatnonzero(counts)).cuda()
    s["most"] = int(counts.max())
    s["offsets"] = torch.from_numpy(offsets.astype(np.int32)).cuda()
    if op == "q4":
        if E == 1:
            s["offsets"] = None
        s["x"] = normal(R, K)
        s["q"] = torch.randint(0, 256, (E, N, K // 2), generator=gen, device="cuda",
                               dtype=torch.uint8)
        g = K // case["group"]
        scale = torch.rand((E, N, g), generator=gen, device="cuda").add_(0.5).mul_(0.25 / K ** 0.5)
        s["scales"] = scale.to(dt)
        s["mins"] = (scale * -7.5 * (1 + 0.2 * torch.randn(scale.shape, generator=gen, device="cuda"))
                     ).to(dt) if case["mins"] else None
        return s
    if case["gather"]:
        T = max(1, R // 4)
        s["x"] = normal(T, K)
        s["rows"] = torch.randint(0, T, (R,), generator=gen, device="cuda", dtype=torch.int32)
        s["rows"][int(offsets[-1]):] = -1
    else:
        s["x"] = normal(R, K)
        s["rows"] = None
    if op == "product":
        shape = (E, K, N) if case["transb"] == "N" else (E, N, K)
        s["w"] = normal(*shape, scale=K ** -0.5)
    else:
        s["dy"] = normal(R, N)
    return s


# ---------------------------------------------------------------------------
# The operators.

def run(state):
    return _library(state) if own else _plain(state)


def _library(s):
    import paper_2609_04663_amd as emu
    case = s["case"]
    op = case["op"]
    if op == "route":
        r = emu.moe_route(s["logits"], case["k"], case["scope"])
        out = {"ids": r.ids, "weights": r.weights, "offsets": r.offsets, "rows": r.rows,
               "slots": r.slots}
        if case["train"]:
            out["dlogits"] = emu.moe_route_grad(s["logits"], r.ids, r.weights, s["dweights"],
                                                case["scope"])
        return out
    if op == "combine":
        out = {"y": emu.moe_combine(s["z"], s["slots"], s["weights"])}
        if case["train"]:
            out["dz"], out["dweights"] = emu.moe_combine_grad(s["dy"], s["z"], s["slots"],
                                                              s["weights"], s["rows"])
        return out
    if op == "q4":
        return emu.q4_gemm(s["x"], s["q"], s["scales"], mins=s["mins"], offsets=s["offsets"])
    if op == "product":
        return emu.grouped_gemm(s["x"], s["w"], s["offsets"], transb=case["transb"],
                                rows=s["rows"])
    return emu.grouped_wgrad(s["x"], s["dy"], s["offsets"], transb=case["transb"], rows=s["rows"])


def _padded(s, R):
    """Rows of the active experts side by side: their row numbers (A x most),
    which of them exist, and for every row the place it has there."""
    off = s["offsets"].long() if s["offsets"] is not None else torch.tensor([0, R], device="cuda")
    a, most = s["active"], s["most"]
    pos = torch.arange(most, device="cuda")
    index = off[a][:, None] + pos
    real = pos < (off[a + 1] - off[a])[:, None]
    r = torch.arange(R, device="cuda")
    at = torch.searchsorted(off[a], r, right=True) - 1
    place = at * most + r - off[a][at]
    return index.clamp_(max=R - 1), real, torch.where(r < off[-1], place, 0), r < off[-1]


def _taken(x, rows, index, real):
    """x of the padded rows in 32 bits, through the gather where there is one."""
    if rows is not None:
        index = rows[index].long()
    return x.float()[index.clamp(min=0)] * real[..., None]


def _plain(s):
    case = s["case"]
    op, dt = case["op"], DTYPES[case["type"]]
    if op == "route":
        return _plain_route(s)
    if op == "combine":
        z, w, slots = s["z"].float(), s["weights"], s["slots"].long()
        w = w * (slots >= 0)
        taken = z[slots.clamp(min=0)]
        out = {"y": (taken * w[..., None]).sum(1).to(dt)}
        if case["train"]:
            dy = s["dy"].float()
            w_rows = torch.zeros(z.shape[0] + 1, device="cuda")
            w_rows[torch.where(slots >= 0, slots, z.shape[0]).reshape(-1)] = w.reshape(-1)
            rows = s["rows"].long()
            out["dz"] = (dy[rows.clamp(min=0)] * (w_rows[:-1] * (rows >= 0))[:, None]).to(dt)
            out["dweights"] = (taken * dy[:, None, :]).sum(2) * (slots >= 0)
        return out
    R, E, N, K = case["R"], case["E"], case["N"], case["K"]
    index, real, place, live = _padded(s, R)
    a = s["active"]
    if op == "wgrad":
        x = _taken(s["x"], s["rows"], index, real)
        dy = _taken(s["dy"], None, index, real)
        left, right = (x, dy) if case["transb"] == "N" else (dy, x)
        out = torch.zeros((E, left.shape[2], right.shape[2]), device="cuda")
        out[a] = torch.bmm(left.transpose(1, 2).contiguous(), right)
        return out.to(dt)
    if op == "q4":
        q = s["q"][a]
        q = torch.stack((q & 15, q >> 4), -1).view(len(a), N, K // case["group"], -1).float()
        scale = s["scales"][a].float()[..., None]
        w = q * scale + s["mins"][a].float()[..., None] if case["mins"] else (q - 8) * scale
        w = w.view(len(a), N, K)
        x = _taken(s["x"], None, index, real)
        y = torch.bmm(x, w.transpose(1, 2))
    else:
        x = _taken(s["x"], s["rows"], index, real)
        w = s["w"].float()[a]
        y = torch.bmm(x, w if case["transb"] == "N" else w.transpose(1, 2))
    return (y.view(-1, N)[place] * live[:, None]).to(dt)


def _plain_route(s):
    case = s["case"]
    T, E, k = case["T"], case["E"], case["k"]
    logits = s["logits"].float()
    value, expert = torch.sort(logits, dim=1, descending=True, stable=True)
    value, expert = value[:, :k], expert[:, :k]
    there = value > -math.inf
    top = torch.where(there[:, :1], value[:, :1], 0.0)
    over = value if case["scope"] == "chosen" else logits
    total = torch.exp(over - top).sum(1, keepdim=True)
    weights = torch.where(there, torch.exp(value - top) / total, 0.0)
    flat = torch.where(there, expert, E).reshape(-1)
    order = torch.argsort(flat, stable=True)
    slots = torch.empty_like(order)
    slots[order] = torch.arange(T * k, device="cuda")
    live = there.reshape(-1)
    offsets = torch.searchsorted(flat[order], torch.arange(E + 1, device="cuda"))
    out = {"ids": torch.where(there, expert, -1).to(torch.int32), "weights": weights,
           "offsets": offsets.to(torch.int32),
           "rows": torch.where(live[order], order // k, -1).to(torch.int32),
           "slots": torch.where(live, slots, -1).view(T, k).to(torch.int32)}
    if case["train"]:
        dw = s["dweights"]
        mean = (weights * dw * there).sum(1, keepdim=True)
        chosen = torch.zeros((T, E), device="cuda")
        chosen.scatter_(1, expert, torch.where(there, weights * dw, 0.0))
        if case["scope"] == "chosen":
            p = torch.zeros((T, E), device="cuda").scatter_(1, expert, weights)
        else:
            p = torch.where(logits > -math.inf, torch.exp(logits - top) / total, 0.0)
        out["dlogits"] = (chosen - p * mean).to(s["logits"].dtype)
    return out


def work(case):
    """Each input read once, each output written once, two operations for each
    multiply-add.  Of the experts' matrices those count that an even load of
    the rows reaches."""
    size, op = SIZES[case["type"]], case["op"]
    if op == "route":
        T, E, k = case["T"], case["E"], case["k"]
        b = size * T * E + 16 * T * k + 4 * (E + 1)
        return {"bytes": b + (size * T * E + 4 * T * k if case["train"] else 0), "flops": 4 * T * E}
    if op == "combine":
        T, D, k = case["T"], case["D"], case["k"]
        b = size * (T * k * D + T * D) + 8 * T * k
        f = 2 * T * k * D
        if case["train"]:
            return {"bytes": b + size * (T * D + T * k * D) + 8 * T * k, "flops": 5 * T * k * D}
        return {"bytes": b, "flops": f}
    R, E, N, K = case["R"], case["E"], case["N"], case["K"]
    reached = E * (1.0 - (1.0 - 1.0 / E) ** R)
    flops = 2 * R * N * K
    if op == "q4":
        w = N * K * (0.5 + size * (2 if case["mins"] else 1) / case["group"])
        return {"bytes": reached * w + size * R * (N + K), "flops": flops}
    rows_x = max(1, R // 4) if case["gather"] else R
    if op == "wgrad":
        return {"bytes": size * (rows_x * K + R * N + E * N * K), "flops": flops}
    return {"bytes": size * (rows_x * K + R * N + reached * N * K), "flops": flops}


# ---------------------------------------------------------------------------
# The definitions in 64 bits.

def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op == "route":
        x = s["logits"].double().cpu()
        T, E, k = case["T"], case["E"], case["k"]
        chosen = torch.zeros((T, E), dtype=torch.bool)
        ids = torch.empty((T, k), dtype=torch.int64)
        rest = x.clone()
        for j in range(k):
            # the largest that is left; argmax of NumPy takes the lowest index of a tie
            i = torch.from_numpy(rest.numpy().argmax(1))
            if j >= E:
                i = torch.zeros(T, dtype=torch.int64)
            ids[:, j] = i
            ok = rest.gather(1, i[:, None]) > -math.inf
            ids[:, j] = torch.where(ok[:, 0], i, -1)
            chosen |= torch.zeros_like(chosen).scatter_(1, i[:, None], ok)
            rest.scatter_(1, i[:, None], -math.inf)
        among = chosen if case["scope"] == "chosen" else x > -math.inf
        p = torch.softmax(torch.where(among, x, -math.inf), 1)
        p = torch.where(among.any(1, keepdim=True), p, 0.0)
        weights = torch.where(ids >= 0, p.gather(1, ids.clamp(min=0)), 0.0)
        out = {"ids": None, "weights": weights, "offsets": None, "rows": None, "slots": None}
        if case["train"]:
            g = torch.zeros((T, E), dtype=torch.float64)
            dw = torch.where(ids >= 0, s["dweights"].double().cpu(), 0.0)
            g.scatter_add_(1, ids.clamp(min=0), dw)
            out["dlogits"] = p * (g - (p * g).sum(1, keepdim=True))
        return out
    if op == "combine":
        z, w, slots = s["z"].double(), s["weights"].double(), s["slots"].long()
        y = torch.zeros((case["T"], case["D"]), dtype=torch.float64, device="cuda")
        dy = s["dy"].double() if case["train"] else None
        dz, dw = torch.zeros_like(z), torch.zeros_like(w)
        for j in range(case["k"]):
            t = torch.nonzero(slots[:, j] >= 0)[:, 0]
            at = slots[t, j]
            y[t] += w[t, j, None] * z[at]
            if case["train"]:
                dz[at] = w[t, j, None] * dy[t]
                dw[t, j] = (z[at] * dy[t]).sum(1)
        return {"y": y, "dz": dz, "dweights": dw} if case["train"] else {"y": y}
    R, E, N, K = case["R"], case["E"], case["N"], case["K"]
    offsets = [0, R] if s["offsets"] is None else s["offsets"].tolist()
    x = s["x"].double()
    if s.get("rows") is not None:
        x = x[s["rows"].long().clamp(min=0)]
    if op == "wgrad":
        out = torch.zeros((E, K, N) if case["transb"] == "N" else (E, N, K),
                          dtype=torch.float64, device="cuda")
    else:
        out = torch.zeros((R, N), dtype=torch.float64, device="cuda")
    for e in range(E):
        at = slice(offsets[e], offsets[e + 1])
        if at.start == at.stop:
            continue
        if op == "wgrad":
            dy = s["dy"][at].double()
            out[e] = x[at].T @ dy if case["transb"] == "N" else dy.T @ x[at]
            continue
        if op == "q4":
            q = s["q"][e].to(torch.int64)
            w = torch.empty((N, K), dtype=torch.float64, device="cuda")
            w[:, 0::2], w[:, 1::2] = q % 16, q // 16
            scale = s["scales"][e].double().repeat_interleave(case["group"], 1)
            if case["mins"]:
                w = w * scale + s["mins"][e].double().repeat_interleave(case["group"], 1)
            else:
                w = (w - 8) * scale
            w = w.T
        else:
            w = s["w"][e].double() if case["transb"] == "N" else s["w"][e].double().T
        out[at] = x[at] @ w
    return out
