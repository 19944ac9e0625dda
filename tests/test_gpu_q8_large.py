"""The 8-bit operators and the balance loss on tensors that 32-bit offsets do not span."""
import pytest
import torch

import _moe as M
import _q8 as Q

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def emu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2609_04663_amd as E
    E.lib()
    yield E
    torch.cuda.empty_cache()


def _ints(gen, *shape):
    return torch.randint(-128, 128, shape, generator=gen, device="cuda", dtype=torch.int8)


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _compare(got, x, xs, w, ws):
    ref = (x.double() @ w.double().T) * xs.double()[:, None] * ws.double()
    assert ((got.double() - ref).abs() <= Q.product_bar(ref, got.dtype)).all()


@pytest.mark.parametrize("K,rows_of_each", [(8192, 1), (8192, 200), (8191, 3)])
def test_matrices_of_5_gib(emu, K, rows_of_each):
    gen, E, N = _gen(K), 40, 16384
    W, ws = _ints(gen, E, N, K), torch.rand((E, N), generator=gen, device="cuda")
    X = _ints(gen, E * rows_of_each, K)
    xs = torch.rand(len(X), generator=gen, device="cuda")
    offsets = (torch.arange(E + 1) * rows_of_each).int().cuda()
    got = emu.q8_gemm(X, xs, W, ws, offsets, dtype=torch.float32)
    for e in (0, 31, 32, E - 1):
        at = slice(e * rows_of_each, (e + 1) * rows_of_each)
        _compare(got[at], X[at], xs[at], W[e], ws[e])


@pytest.mark.parametrize("R", [5, 700])
def test_rows_of_a_matrix_of_5_gib(emu, R):
    """Gathered from the whole of it, its last row too."""
    gen, T, K, N = _gen(R), 640000, 8192, 300
    X, xs = _ints(gen, T, K), torch.rand(T, generator=gen, device="cuda")
    W, ws = _ints(gen, N, K), torch.rand(N, generator=gen, device="cuda")
    rows = torch.randint(0, T, (R,), generator=gen, device="cuda").int()
    rows[0], rows[1], rows[2] = T - 1, 0, T
    got = emu.q8_gemm(X, xs, W, ws, rows=rows, dtype=torch.float32)
    assert (got[2] == 0).all()
    keep = torch.arange(R, device="cuda") != 2
    src = rows[keep].long()
    _compare(got[keep], X[src], xs[src], W, ws)


def test_results_of_9_gib(emu):
    gen, R, N, K = _gen(3), 40000, 60000, 64
    X, xs = _ints(gen, R, K), torch.rand(R, generator=gen, device="cuda")
    W, ws = _ints(gen, N, K), torch.rand(N, generator=gen, device="cuda")
    got = emu.q8_gemm(X, xs, W, ws, dtype=torch.float32)
    for at in (slice(0, 300), slice(35600, 36000), slice(R - 300, R)):
        _compare(got[at], X[at], xs[at], W, ws)


def test_rows_in_8_bits(emu):
    R, K = 540000, 8192
    x = torch.empty((R, K), dtype=torch.bfloat16, device="cuda").uniform_(-1, 1, generator=_gen(4))
    q, s = emu.q8_pack(x)
    for at in (slice(0, 4), slice(262140, 262148), slice(R - 4, R)):
        ref, scales = Q.pack(x[at].cpu())
        assert torch.equal(q[at].cpu(), ref) and torch.equal(s[at].cpu(), scales)
    del x
    back = emu.q8_unpack(q, s, torch.float16)
    for at in (slice(0, 4), slice(262140, 262148), slice(R - 4, R)):
        assert torch.equal(back[at], (q[at].float() * s[at, None]).half())


def test_balance_of_2_gib_of_logits(emu):
    """Every row of logits alike in its 2^21, but the last ones, a sequence of their own."""
    T, E = (1 << 21) + 5000, 1024
    row = torch.randn(E, generator=_gen(5), device="cuda").bfloat16()
    x = row.expand(T, E).contiguous()
    x[T - 5000:] = torch.randn((5000, E), generator=_gen(6), device="cuda").bfloat16()
    ids = torch.randint(0, E, (T, 2), generator=_gen(7), device="cuda").int()
    starts = torch.tensor([0, T - 5000, T], dtype=torch.int32).cuda()
    b = emu.moe_balance(x, ids, starts)
    dl = torch.tensor([2.0 ** 20, 3.0]).cuda()
    got = emu.moe_balance_grad(x, b.counts, b.tokens, dl, None, starts)
    assert b.tokens.tolist() == [T - 5000, 5000]
    for s, (lo, hi) in enumerate(((0, T - 5000), (T - 5000, T))):
        c = torch.bincount(ids[lo:hi].reshape(-1).long(), minlength=E)
        assert torch.equal(b.counts[s].long(), c)
        xs = x[lo:lo + 1] if s == 0 else x[lo:hi]
        p, f = torch.softmax(xs.double(), 1), c.double() / c.sum()
        loss = E * (f * p.mean(0)).sum()
        # 2^21 tokens: a group of lanes adds up to 300 of them
        assert abs(float(b.loss[s]) - loss) <= (Q.LOSS_BAR + 300 * 2.0 ** -24) * loss
        ref = p * float(dl[s]) * E / (hi - lo) * (f - (p @ f)[:, None])
        bar = 2.0 ** -24 * 260 * p * float(dl[s]) * E / (hi - lo) * (f + (p @ f)[:, None])
        for at in ((lo, hi - 1) if s == 0 else range(lo, hi, 999)):
            r, w = (0 if s == 0 else at - lo), got[at].double()
            assert ((w - ref[r]).abs() <= bar[r] + M.rounded(ref[r], torch.bfloat16)).all()
