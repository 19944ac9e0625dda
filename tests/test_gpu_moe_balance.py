"""The balance loss of a routing and its gradient against 64 bits."""
import math

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
    return E


def _case(seed, T, E, k, S, dt):
    """Logits with masked experts, tokens without any, and what a router makes of them; S
    sequences, with more than two of them one empty, the last tokens in none."""
    gen = torch.Generator().manual_seed(seed)
    x = (torch.randn((T, E), generator=gen) * 1.5).clamp(-7, 7).to(dt)
    x[torch.rand((T, E), generator=gen) < 0.2] = -math.inf
    x[torch.rand(T, generator=gen) < 0.1] = -math.inf
    value, ids = torch.sort(x.float(), dim=1, descending=True, stable=True)
    ids = torch.where(value > -math.inf, ids, -1)[:, :k].int().contiguous()
    starts = None
    if S > 1:
        cut = torch.sort(torch.randint(0, T + 1, (S,), generator=gen)).values
        if S > 2:
            cut[1] = cut[0]
        starts = torch.cat((torch.zeros(1), cut)).int()
    return x, ids, starts


def _gpu(t):
    return None if t is None else t.cuda()


SHAPES = [(1, 8, 1, 1), (5, 3, 3, 2), (64, 64, 8, 1), (200, 13, 4, 3), (256, 16, 2, 1), (257, 130, 8, 1),
          (700, 60, 6, 9), (900, 256, 8, 5), (333, 511, 32, 2), (300, 1000, 4, 1), (1300, 17, 2, 40)]


@pytest.mark.parametrize("kind", list(M.TYPES))
@pytest.mark.parametrize("T,E,k,S", SHAPES)
def test_losses_and_gradient(emu, kind, T, E, k, S):
    dt = M.TYPES[kind]
    x, ids, starts = _case(T + E, T, E, k, S, dt)
    loss, zloss, counts, tokens, bar = Q.balance(x, ids, starts)
    b = emu.moe_balance(x.cuda(), ids.cuda(), _gpu(starts))
    assert torch.equal(b.counts.cpu().long(), counts) and torch.equal(b.tokens.cpu().long(), tokens)
    M.check(b.loss, loss, Q.LOSS_BAR * loss + 1e-37, "loss")
    M.check(b.zloss, zloss, bar, "zloss")
    gen = torch.Generator().manual_seed(k)
    dl, dz = torch.randn(S, generator=gen), torch.randn(S, generator=gen)
    for z in (dz, None):
        ref, bar = Q.balance_grad(x, counts, tokens, dl, z, starts)
        got = emu.moe_balance_grad(x.cuda(), b.counts, b.tokens, dl.cuda(), _gpu(z), _gpu(starts))
        M.check(got, ref, bar + M.rounded(ref, dt), "dlogits")


@pytest.mark.parametrize("T,E", [(40000, 64), (70000, 8)])
def test_many_tokens(emu, T, E):
    """Spans of several loads, compared with torch in 64 bits."""
    x, ids, _ = _case(T, T, E, 2, 1, torch.float32)
    starts = torch.tensor([0, 3, 9000, 9000, T // 2, T - 77], dtype=torch.int32)
    b = emu.moe_balance(x.cuda(), ids.cuda(), starts.cuda())
    live = x.amax(1) > -math.inf
    dl = torch.tensor([1.0, -2.0, 3.0, 0.5, 1.5])
    got = emu.moe_balance_grad(x.cuda(), b.counts, b.tokens, dl.cuda(), dl.cuda(), starts.cuda()).cpu().double()
    assert (got[T - 77:] == 0).all()
    for s, (lo, hi) in enumerate(Q.spans(starts, T)):
        rows = torch.arange(lo, hi)[live[lo:hi]]
        c = torch.bincount(ids[lo:hi][ids[lo:hi] >= 0].long(), minlength=E)
        assert torch.equal(b.counts[s].cpu().long(), c) and int(b.tokens[s]) == len(rows)
        if len(rows) == 0:
            assert float(b.loss[s]) == float(b.zloss[s]) == 0
            continue
        xs = x[rows].double()
        p, z, f = torch.softmax(xs, 1), torch.logsumexp(xs, 1), c.double() / c.sum()
        loss = E * (f * p.mean(0)).sum()
        assert abs(float(b.loss[s]) - loss) <= Q.LOSS_BAR * loss
        zbar = (2 * z.abs() * (70 + 4 * z.abs()) + 32 * z * z).mean() * 2.0 ** -24
        assert abs(float(b.zloss[s]) - (z * z).mean()) <= zbar
        d, n = float(dl[s]), len(rows)
        mean = (p @ f)[:, None]
        ref = p * (d * E / n * (f - mean) + d * 2 / n * z[:, None])
        bar = 2.0 ** -24 * 260 * p * abs(d) / n * (E * (f + mean) + 2 * (1 + z.abs()[:, None]))
        M.check(got[rows], ref, bar + M.rounded(ref, torch.float32))


def test_gradient_by_differences(emu):
    """Central differences of the 64-bit losses with the counts held."""
    T, E, k = 6, 10, 3
    x, ids, starts = _case(11, T, E, k, 2, torch.float32)
    x[x == -math.inf] = -3.0
    ids = torch.topk(x, k).indices.int()
    dl, dz = torch.tensor([0.7, -1.3]), torch.tensor([0.2, 0.4])
    b = emu.moe_balance(x.cuda(), ids.cuda(), starts.cuda())
    got = emu.moe_balance_grad(x.cuda(), b.counts, b.tokens, dl.cuda(), dz.cuda(), starts.cuda()).cpu().double()

    def value(y):
        loss, zloss = Q.balance(y, ids, starts)[:2]
        return float((dl.double() * loss + dz.double() * zloss).sum())

    h = 1e-5
    for t in range(T):
        for e in range(E):
            up, down = x.double(), x.double()
            up[t, e] += h
            down[t, e] -= h
            # third derivatives are below 100, so the difference is off by h^2 / 6 of that
            assert abs(float(got[t, e]) - (value(up) - value(down)) / (2 * h)) < 1e-5


def test_infinities_nan_and_lowest_values(emu):
    gen = torch.Generator().manual_seed(3)
    x = torch.randn((12, 20), generator=gen)
    x[0] = -math.inf
    x[1] = math.nan
    x[2, ::2] = math.nan
    x[3] = torch.finfo(torch.float32).min / 2**70          # z^2 stays in range
    x[4, 7] = math.inf
    x[5, 1:] = -math.inf
    x[6, :19] = torch.finfo(torch.float32).min
    ids = torch.full((12, 2), -1, dtype=torch.int32)
    ids[2:] = torch.tensor([[7, 19]])
    ids[6, 0], ids[7, 1], ids[0, 0] = 25, -9, 3            # not experts; of a token without logits
    rest = torch.tensor([t for t in range(12) if t != 4])
    for rows in (rest, torch.tensor([4])):
        xs, i = x[rows], ids[rows].contiguous()
        loss, zloss, counts, tokens, bar = Q.balance(xs, i, None)
        b = emu.moe_balance(xs.cuda(), i.cuda())
        assert torch.equal(b.counts.cpu().long(), counts) and torch.equal(b.tokens.cpu().long(), tokens)
        M.check(b.loss, loss, Q.LOSS_BAR * loss, "loss")
        one = torch.ones(1)
        if len(rows) == 1:
            assert float(b.zloss) == math.inf
            ref, bar = Q.balance_grad(xs, counts, tokens, one, 0 * one, None)
            got = emu.moe_balance_grad(xs.cuda(), b.counts, b.tokens, one.cuda(), 0 * one.cuda())
            M.check(got, ref, bar + M.rounded(ref, torch.float32))
            got = emu.moe_balance_grad(xs.cuda(), b.counts, b.tokens, one.cuda(), one.cuda()).cpu()
            assert float(got[0, 7]) == math.inf and (got[0, torch.arange(20) != 7] == 0).all()
            continue
        M.check(b.zloss, zloss, bar, "zloss")
        ref, bar = Q.balance_grad(xs, counts, tokens, one, one, None)
        got = emu.moe_balance_grad(xs.cuda(), b.counts, b.tokens, one.cuda(), one.cuda())
        M.check(got, ref, bar + M.rounded(ref, torch.float32))


def test_nothing(emu):
    """No tokens; sequences without tokens; no choices; no tokens by the caller's count."""
    x, ids = torch.zeros((0, 9)), torch.zeros((0, 2), dtype=torch.int32)
    b = emu.moe_balance(x.cuda(), ids.cuda(), torch.zeros(4, dtype=torch.int32).cuda())
    assert b.loss.shape == (3,) and b.counts.shape == (3, 9)
    for t in b:
        assert (t == 0).all()
    zero = torch.zeros(1).cuda()
    assert emu.moe_balance_grad(x.cuda(), b.counts[:1], b.tokens[:1], zero).shape == (0, 9)
    x = torch.randn((300, 9), generator=torch.Generator().manual_seed(1)).cuda()
    none = torch.full((300, 2), -1, dtype=torch.int32).cuda()
    b = emu.moe_balance(x, none)
    assert float(b.loss) == 0 and float(b.zloss) > 0 and int(b.tokens) == 300
    one = torch.ones(1).cuda()
    assert (emu.moe_balance_grad(x, b.counts, b.tokens, one) == 0).all()
    assert (emu.moe_balance_grad(x, b.counts, 0 * b.tokens, one, one) == 0).all()
    # starts past the tokens, and descending ones, stay inside
    for starts in ([0, 500, 900], [0, -5, 300], [7, 200, 300]):
        b = emu.moe_balance(x, none, torch.tensor(starts, dtype=torch.int32).cuda())
        n = [hi - lo for lo, hi in Q.spans(starts, 300)]
        assert b.tokens.tolist() == n
    down = torch.tensor([0, 250, 100, 300], dtype=torch.int32).cuda()
    b = emu.moe_balance(x, none, down)
    three = torch.ones(3).cuda()
    assert emu.moe_balance_grad(x, b.counts, b.tokens, three, three, down).shape == x.shape


def test_rows_of_a_larger_matrix(emu):
    gen = torch.Generator().manual_seed(4)
    whole = torch.randn((300, 101), generator=gen).to(torch.bfloat16)
    part = whole[:, 3:67]
    ids = torch.randint(0, 64, (300, 3), generator=gen).int()
    loss, zloss, counts, tokens, bar = Q.balance(part, ids, None)
    b = emu.moe_balance(whole.cuda()[:, 3:67], ids.cuda())
    M.check(b.loss, loss, Q.LOSS_BAR * loss)
    M.check(b.zloss, zloss, bar)
    one = torch.ones(1)
    ref, bar = Q.balance_grad(part, counts, tokens, one, one, None)
    got = emu.moe_balance_grad(whole.cuda()[:, 3:67], b.counts, b.tokens, one.cuda(), one.cuda())
    M.check(got, ref, bar + M.rounded(ref, torch.bfloat16))


def test_a_batch_in_two_parts(emu):
    """Counts and tokens of two parts, added up, give the gradient of the whole."""
    x, ids, _ = _case(5, 900, 32, 4, 1, torch.float32)
    x, ids, one = x.cuda(), ids.cuda(), torch.ones(1).cuda()
    whole = emu.moe_balance(x, ids)
    parts = [emu.moe_balance(x[a:b], ids[a:b]) for a, b in ((0, 400), (400, 900))]
    counts, tokens = (sum(getattr(p, n) for p in parts).int() for n in ("counts", "tokens"))
    assert torch.equal(counts, whole.counts) and torch.equal(tokens, whole.tokens)
    ref = emu.moe_balance_grad(x, whole.counts, whole.tokens, one, one)
    got = torch.cat([emu.moe_balance_grad(x[a:b], counts, tokens, one, one) for a, b in ((0, 400), (400, 900))])
    assert torch.equal(got, ref)


@pytest.mark.parametrize("T", [200, 3000])
def test_in_a_graph(emu, T):
    """Captured once, replayed with other inputs and eager calls between: the same bits."""
    x, ids, starts = _case(8, T, 48, 4, 3, torch.float32)
    other, other_ids, _ = _case(9, T, 48, 4, 3, torch.float32)
    x, ids, starts, dl = x.cuda(), ids.cuda(), starts.cuda(), torch.ones(3).cuda()

    def call(x, ids):
        b = emu.moe_balance(x, ids, starts)
        return (*b, emu.moe_balance_grad(x, b.counts, b.tokens, dl, dl, starts))

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call(x, ids)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = call(x, ids)
    for data, data_ids in ((x.clone(), ids.clone()), (other.cuda(), other_ids.cuda())) * 2:
        eager = [t.clone() for t in call(data, data_ids)]
        x.copy_(data)
        ids.copy_(data_ids)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, eager))
