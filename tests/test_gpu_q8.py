"""Rows in 8-bit integers and their products against 64 bits."""
import math

import pytest
import torch

import _moe as M
import _q8 as Q
import _q8_shapes as S

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def emu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2609_04663_amd as E
    E.lib()
    return E


def _same(got, ref):
    """Equal bits of a type's values, NaN equal to NaN."""
    got = got.cpu()
    return got.dtype == ref.dtype and got.shape == ref.shape and bool(
        ((got == ref) | (torch.isnan(got) & torch.isnan(ref))).all())


LENGTHS = [1, 7, 8, 64, 129, 256, 300, 513, 1000, 1025, 2048, 2049, 4097, 8192, 8200, 16384, 16385, 40001]


@pytest.mark.parametrize("kind", list(M.TYPES))
@pytest.mark.parametrize("K", LENGTHS)
def test_pack(emu, kind, K):
    gen = torch.Generator().manual_seed(K)
    x = (torch.randn((37, K), generator=gen) * torch.exp(2 * torch.randn((37, 1), generator=gen))).to(M.TYPES[kind])
    x[3] = 0
    x[5, K // 2] = math.inf
    x[6, K - 1] = math.nan
    x[7, 0] = -math.inf
    x[8] = x[8] * 0 - 0.0
    q, scales = Q.pack(x)
    got, got_scales = emu.q8_pack(x.cuda())
    assert torch.equal(got.cpu(), q) and _same(got_scales, scales)
    for dt in M.TYPES.values():
        values = (q.float() * scales[:, None]).to(dt)
        assert _same(emu.q8_unpack(got, got_scales, dt), values)


@pytest.mark.parametrize("kind", list(M.TYPES))
def test_borders(emu, kind):
    """Entries half-way between two integers, and a unit in the last place to either side."""
    dt = M.TYPES[kind]
    tops = [127.0, 254.0, 63.5, 127.0 * 2 ** -10, 1.0, 3.0, 65.0, 1.9921875]
    if kind != "f16":
        tops += [127.0 * 2.0 ** 100, 127.0 * 2.0 ** -120, 127.0 * 2.0 ** -130, 2.0 ** 127]
    if kind == "f32":
        tops += [float(torch.nextafter(torch.tensor(127.0), torch.tensor(d))) for d in (0.0, 200.0)]
    rows = []
    for top in tops:
        half = ((2 * torch.arange(-127, 127) + 1).double() * top / 254).to(dt)
        bits = half.view(torch.int32 if kind == "f32" else torch.int16)
        near = torch.cat([half, (bits + 1).view(dt), (bits - 1).view(dt)])
        near = torch.where(near.abs() <= torch.tensor(top, dtype=dt), near, torch.zeros((), dtype=dt))
        rows.append(torch.cat([near, torch.tensor([top], dtype=dt)]))
    x = torch.stack(rows)
    q, scales = Q.pack(x)
    got, got_scales = emu.q8_pack(x.cuda())
    assert torch.equal(got.cpu(), q) and _same(got_scales, scales)


def test_subnormal_rows(emu):
    x = torch.zeros((6, 70))
    x[0] = 2.0 ** -149
    x[1] = 2.0 ** -149 * torch.arange(70)
    x[2] = torch.linspace(-1, 1, 70) * 2.0 ** -126
    x[3] = torch.linspace(-1, 1, 70) * 2.0 ** -100
    x[4] = torch.linspace(-1, 1, 70) * 3.0e38
    x[5, 69] = 2.0 ** -149
    q, scales = Q.pack(x)
    got, got_scales = emu.q8_pack(x.cuda())
    assert torch.equal(got.cpu(), q) and _same(got_scales, scales)
    for dt in M.TYPES.values():
        assert _same(emu.q8_unpack(got, got_scales, dt), (q.float() * scales[:, None]).to(dt))


@pytest.mark.parametrize("kind", list(M.TYPES))
def test_pack_of_views(emu, kind):
    gen = torch.Generator().manual_seed(2)
    whole = torch.randn((50, 333), generator=gen).to(M.TYPES[kind])
    for part in (whole[:, 5:300], whole[::2, 1:], whole[:1, 3:], whole[:0], whole.view(5, 10, 333)):
        q, scales = Q.pack(part)
        base = part.cuda() if part.dim() == 3 else None
        if base is None:                                    # the same view on the GPU
            w = whole.cuda()
            base = torch.as_strided(w, part.shape, part.stride(), part.storage_offset())
        got, got_scales = emu.q8_pack(base)
        assert got.shape == part.shape and torch.equal(got.cpu(), q) and _same(got_scales, scales)
    ints = torch.randint(-128, 128, (9, 400), generator=gen, dtype=torch.int8)
    scales = torch.rand(9, generator=gen)
    got = emu.q8_unpack(ints.cuda()[:, 7:399], scales.cuda(), M.TYPES[kind])
    assert _same(got, (ints[:, 7:399].float() * scales[:, None]).to(M.TYPES[kind]))
    for shape in ((0, 5), (3, 0)):
        got, got_scales = emu.q8_pack(torch.zeros(shape, dtype=M.TYPES[kind]).cuda())
        assert got.shape == shape and (got_scales == 0).all()
        assert emu.q8_unpack(got, got_scales).shape == shape


def test_rows_behind_a_packed_matrix_stay(emu):
    """The C entry with a leading dimension: nothing but the rows' entries is written."""
    import ctypes
    x = torch.randn((5, 21), generator=torch.Generator().manual_seed(1)).cuda()
    q = torch.full((6, 32), 99, dtype=torch.int8).cuda()
    scales = torch.full((6,), 7.0).cuda()
    P = ctypes.c_void_p
    emu.lib().emu_set_stream(P(torch.cuda.current_stream().cuda_stream))
    assert emu.lib().emu_q8_pack(0, 5, 21, P(x.data_ptr()), 21, P(q.data_ptr()), 32, P(scales.data_ptr())) == 0
    ref, ref_scales = Q.pack(x.cpu())
    assert torch.equal(q[:5, :21].cpu(), ref) and (q[:, 21:] == 99).all() and (q[5] == 99).all()
    assert _same(scales[:5], ref_scales) and float(scales[5]) == 7.0


# ---------------------------------------------------------------------------
# Products.

def _operands(seed, R, E, N, K, gather):
    gen = torch.Generator().manual_seed(seed)
    T = max(1, R // 3) if gather else R
    X = torch.randint(-128, 128, (T, K), generator=gen, dtype=torch.int8)
    W = torch.randint(-128, 128, (E, N, K), generator=gen, dtype=torch.int8)
    xs, ws = torch.rand(T, generator=gen) * 0.01 + 1e-3, torch.rand((E, N), generator=gen) * 0.01 + 1e-3
    offsets = rows = None
    if E > 1:
        cut = torch.sort(torch.randint(0, R + 1, (E,), generator=gen)).values
        if E > 2:
            cut[1] = cut[0]                                 # an expert without rows
        cut[-1] = R - R // 10                               # rows of no expert
        offsets = torch.cat((torch.zeros(1), torch.sort(cut).values)).int()
    if gather:
        rows = torch.randint(-1, T + 1, (R,), generator=gen).int()      # some outside X
    return X, xs, W, ws, offsets, rows


def _check(emu, X, xs, W, ws, offsets, rows, dt, X_=None, W_=None):
    ref = Q.product(X, xs, W, ws, offsets, rows)
    g = lambda t: None if t is None else t.cuda()  # noqa: E731
    got = emu.q8_gemm(g(X) if X_ is None else X_, g(xs), g(W) if W_ is None else W_, g(ws), g(offsets), g(rows),
                      dtype=dt)
    M.check(got, ref, Q.product_bar(ref, dt))
    return got


@pytest.mark.parametrize("gather", [False, True])
@pytest.mark.parametrize("kind", list(M.TYPES))
@pytest.mark.parametrize("R,E,N,K", S.FEW + S.SHAPES + S.ODD + S.SPLIT)
def test_product(emu, kind, R, E, N, K, gather):
    _check(emu, *_operands(R + N + K, R, E, N, K, gather), M.TYPES[kind])


@pytest.mark.parametrize("R,E,N,K", S.LARGE)
def test_large_product(emu, R, E, N, K):
    """More tiles than workgroups; compared on the GPU in 64 bits."""
    X, xs, W, ws, offsets, rows = _operands(R, R, E, N, K, True)
    g = lambda t: None if t is None else t.cuda()  # noqa: E731
    got = emu.q8_gemm(g(X), g(xs), g(W), g(ws), g(offsets), g(rows))
    e_of = (M.expert_of(offsets, R) if E > 1 else torch.zeros(R, dtype=torch.int64)).cuda()
    r = rows.cuda().long()
    ok = (r >= 0) & (r < X.shape[0]) & (e_of >= 0)
    assert (got[~ok] == 0).all()
    for e in range(E):
        at = torch.nonzero(ok & (e_of == e))[:, 0]
        if len(at) == 0:
            continue
        ref = X.cuda()[r[at]].double() @ W[e].cuda().double().T
        ref *= xs.cuda()[r[at]].double()[:, None] * ws[e].cuda().double()
        off = (got[at].double() - ref).abs()
        assert (off <= Q.product_bar(ref, torch.bfloat16)).all()


@pytest.mark.parametrize("R", [10, 400])
def test_views(emu, R):
    """Rows and matrices at any byte, rows apart, one matrix for all experts."""
    E, N, K = 3, 130, 176
    X, xs, W, ws, offsets, _ = _operands(R, R, E, N, K, False)
    for lead, ld in ((0, K + 16), (1, K + 16), (0, K + 3), (5, K)):
        bx = torch.full((lead + R * ld,), 77, dtype=torch.int8).cuda()
        vx = bx[lead:].view(R, ld)[:, :K]
        vx.copy_(X)
        bw = torch.full((lead + E * (N + 2) * ld,), 55, dtype=torch.int8).cuda()
        vw = bw[lead:].view(E, N + 2, ld)[:, :N, :K]
        vw.copy_(W)
        _check(emu, X, xs, W, ws, offsets, None, torch.float32, vx, vw)
        _check(emu, X, xs, W, ws, offsets, None, torch.float16, None, vw)
        _check(emu, X, xs, W, ws, offsets, None, torch.bfloat16, vx, None)
    one = W[:1].expand(E, N, K)
    _check(emu, X, xs, one, ws, offsets, None, torch.float32, None, W[:1].cuda().expand(E, N, K))
    odd = W[:1, :, :175].contiguous()
    _check(emu, X[:, :175].contiguous(), xs, odd.expand(E, N, 175), ws, offsets, None, torch.float32, None,
           odd.cuda().expand(E, N, 175))


@pytest.mark.parametrize("kind", list(M.TYPES))
@pytest.mark.parametrize("R", [20, 300])
def test_output_given(emu, kind, R):
    """Y's own type and leading dimension; what lies beside and behind its rows stays."""
    X, xs, W, ws, _, _ = _operands(R, R, 1, 100, 64, False)
    whole = torch.full((R + 2, 117), 5.0, dtype=M.TYPES[kind]).cuda()
    Y = whole[:R, 3:103]
    assert emu.q8_gemm(X.cuda(), xs.cuda(), W.cuda()[0], ws.cuda()[0], Y=Y) is Y
    ref = Q.product(X, xs, W, ws, None, None)
    M.check(Y, ref, Q.product_bar(ref, M.TYPES[kind]))
    assert (whole[:, :3] == 5).all() and (whole[:, 103:] == 5).all() and (whole[R:] == 5).all()


@pytest.mark.parametrize("R", [12, 300])
def test_scales_at_the_ends_of_the_range(emu, R):
    X, xs, W, ws, _, rows = _operands(R, R, 1, 200, 160, True)
    xs = 2.0 ** torch.linspace(-30, 30, len(xs))
    ws[0, :5] = torch.tensor([2.0 ** 120, 2.0 ** -140, 2.0 ** -149, 0.0, 3.0 * 2.0 ** 97])
    xs[:3] = torch.tensor([2.0 ** -120, 2.0 ** 118, 0.0])
    ref = Q.product(X, xs, W, ws, None, rows)
    got = emu.q8_gemm(X.cuda(), xs.cuda(), W.cuda(), ws.cuda(), rows=rows.cuda(), dtype=torch.float32).cpu()
    inside = ref.abs() < 3.4e38
    assert inside.any() and not inside.all()
    M.check(torch.where(inside, got, 0), torch.where(inside, ref, 0),
            Q.product_bar(torch.where(inside, ref, 0), torch.float32))
    assert (got[~inside].abs() > 3.3e38).all()
    # scales that are not finite: their rows and columns alone; rows outside X are zeros
    xs[3], ws[0, 9] = math.nan, math.inf
    got = emu.q8_gemm(X.cuda(), xs.cuda(), W.cuda(), ws.cuda(), rows=rows.cuda(), dtype=torch.float32).cpu()
    outside = (rows < 0) | (rows >= len(xs))
    assert (got[outside] == 0).all()
    assert torch.isnan(got[rows == 3]).all()
    assert not torch.isfinite(got[~outside, 9]).any()
    rest = inside & (rows != 3)[:, None]
    rest[:, 9] = False
    M.check(torch.where(rest, got, 0), torch.where(rest, ref, 0),
            Q.product_bar(torch.where(rest, ref, 0), torch.float32))


def test_nothing(emu):
    f, i8 = torch.zeros, lambda *s: torch.ones(s, dtype=torch.int8).cuda()  # noqa: E731
    one = lambda *s: torch.ones(s).cuda()  # noqa: E731
    assert emu.q8_gemm(i8(0, 8), one(0), i8(1, 5, 8), one(1, 5)).shape == (0, 5)
    assert emu.q8_gemm(i8(4, 8), one(4), i8(1, 0, 8), one(1, 0)).shape == (4, 0)
    assert (emu.q8_gemm(i8(40, 0), one(40), i8(1, 5, 0), one(1, 5)) == 0).all()
    none = f(1, dtype=torch.int32).cuda()
    assert (emu.q8_gemm(i8(40, 8), one(40), i8(0, 5, 8), one(0, 5), offsets=none) == 0).all()
    rows = torch.full((40,), 2, dtype=torch.int32).cuda()
    assert (emu.q8_gemm(i8(0, 8), one(0), i8(1, 5, 8), one(1, 5), rows=rows) == 0).all()


def test_longest_sums(emu):
    """131071 products of -128 and -128 are just below 2^31."""
    K = 131071
    X, W = torch.full((3, K), -128, dtype=torch.int8), torch.full((1, 5, K), -128, dtype=torch.int8)
    X[1] = 127
    one = torch.ones(3)
    got = emu.q8_gemm(X.cuda(), one.cuda(), W.cuda(), torch.ones((1, 5)).cuda(), dtype=torch.float32).cpu()
    assert got[0].tolist() == [float(torch.tensor(128.0 * 128 * K))] * 5
    assert got[1].tolist() == [float(torch.tensor(-127.0 * 128 * K))] * 5
    K = 131056
    X, W = X[:1, :K].expand(200, K).contiguous(), W[:, :, :K].contiguous()
    got = emu.q8_gemm(X.cuda(), torch.ones(200).cuda(), W.cuda(), torch.ones((1, 5)).cuda(), dtype=torch.float32)
    assert (got == float(torch.tensor(128.0 * 128 * K))).all()


@pytest.mark.parametrize("K", [192, 201])
def test_in_a_graph(emu, K):
    """Packed, multiplied by grouped matrices; captured once, replayed with other inputs and
    eager calls of other sizes between (the workspace's copies): the same bits."""
    gen = torch.Generator().manual_seed(6)
    R, E, N = 600, 4, 200
    x = torch.randn((R, K), generator=gen).cuda()
    wq, ws = emu.q8_pack(torch.randn((E, N, K), generator=gen).cuda())
    offsets = torch.tensor([0, 100, 100, 420, 550], dtype=torch.int32).cuda()

    def call(x):
        q, s = emu.q8_pack(x)
        return emu.q8_gemm(q, s, wq, ws, offsets)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call(x)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = call(x)
    for seed in range(3):
        data = torch.randn((R, K), generator=gen).cuda()
        eager = call(data).clone()
        x.copy_(data)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, eager)


@pytest.mark.parametrize("K,lead", [(1001, 0), (1008, 1)])
def test_few_of_many_rows_through_a_copy(emu, K, lead):
    """Rows of X that are not multiples of 16 bytes, of which the product reads fewer than X has:
    they are copied in order, their scales still by their numbers."""
    gen = torch.Generator().manual_seed(K)
    R, T, E, N = 3000, 9000, 2, 700
    whole = torch.randint(-128, 128, (T * K + lead,), generator=gen, dtype=torch.int8)
    X = whole[lead:].view(T, K)
    W = torch.randint(-128, 128, (E, N, K), generator=gen, dtype=torch.int8)
    xs, ws = torch.rand(T, generator=gen) * 0.01, torch.rand((E, N), generator=gen) * 0.01
    rows = torch.randint(-5, T + 5, (R,), generator=gen).int()
    offsets = torch.tensor([0, 1700, 2900], dtype=torch.int32)
    _check(emu, X, xs, W, ws, offsets, rows, torch.float32, whole.cuda()[lead:].view(T, K))


@pytest.mark.parametrize("R", [50, 294])
def test_split_of_some_rows(emu, R):
    """Offsets that leave rows without an expert, an output of its own type and leading
    dimension, scales that are not finite."""
    X, xs, W, ws, _, rows = _operands(R, R, 1, 130, 8128, True)
    offsets = torch.tensor([0, R - 7], dtype=torch.int32)
    ref = Q.product(X, xs, W, ws, offsets, rows)
    whole = torch.full((R + 1, 140), 5.0, dtype=torch.float16).cuda()
    ws[0, 3] = math.nan
    emu.q8_gemm(X.cuda(), xs.cuda(), W.cuda(), ws.cuda(), offsets.cuda(), rows.cuda(), Y=whole[:R, 5:135])
    got = whole[:R, 5:135].clone()
    outside = (rows < 0) | (rows >= X.shape[0]) | (torch.arange(R) >= R - 7)
    assert torch.isnan(got[~outside.cuda(), 3]).all() and (got[outside.cuda()] == 0).all()
    got[:, 3], ref[:, 3] = 0, 0
    M.check(got, ref, Q.product_bar(ref, torch.float16))
    assert (whole[:, :5] == 5).all() and (whole[:, 135:] == 5).all() and (whole[R] == 5).all()


def test_many_odd_rows_without_workspace(emu):
    """A captured call that finds no workspace reads the operands as they are."""
    X, xs, W, ws, offsets, rows = _operands(3, 2500, 3, 600, 515, True)
    ref = Q.product(X, xs, W, ws, offsets, rows)
    args = [t.cuda() for t in (X, xs, W, ws, offsets, rows)]
    eager = emu.q8_gemm(*args)
    torch.cuda.synchronize()
    emu.release_workspace()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = emu.q8_gemm(*args)
    assert emu.workspace_bytes() == 0
    for _ in range(3):
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        M.check(out, ref, Q.product_bar(ref, torch.bfloat16))
    M.check(eager, ref, Q.product_bar(ref, torch.bfloat16))


def test_on_another_stream(emu):
    """Work of one stream, results read on it after a synchronisation; two streams in turn."""
    gen = torch.Generator().manual_seed(12)
    x = torch.randn((700, 333), generator=gen).cuda()
    w = torch.randn((2, 500, 333), generator=gen).cuda()
    offsets = torch.tensor([0, 300, 700], dtype=torch.int32).cuda()
    ref = None
    torch.cuda.synchronize()
    for stream in (torch.cuda.Stream(), torch.cuda.current_stream(), torch.cuda.Stream()):
        with torch.cuda.stream(stream):
            q, s = emu.q8_pack(x)
            out = emu.q8_gemm(q, s, *emu.q8_pack(w), offsets)
            stream.synchronize()
        ref = out.clone() if ref is None else ref
        assert torch.equal(out, ref)


def test_the_run_of_them(emu):
    """Routed, packed, multiplied, activated, packed, multiplied, combined, as the example
    serves a layer; every step against its own plain form on the same inputs."""
    gen = torch.Generator().manual_seed(9)
    T, D, H, E, k = 50, 192, 320, 8, 2
    x = torch.randn((T, D), generator=gen).to(torch.bfloat16).cuda()
    W1, W2 = (torch.randn(s, generator=gen).to(torch.bfloat16).cuda() / 10 for s in ((E, H, D), (E, D, H)))
    r = emu.moe_route(torch.randn((T, E), generator=gen).cuda(), k)
    p1, p2 = emu.q8_pack(W1), emu.q8_pack(W2)
    q, s = emu.q8_pack(x)
    h = emu.q8_gemm(q, s, *p1, r.offsets, r.rows)
    ref = Q.product(q.cpu(), s.cpu(), p1[0].cpu(), p1[1].cpu(), r.offsets.cpu(), r.rows.cpu())
    M.check(h, ref, Q.product_bar(ref, torch.bfloat16))
    a = torch.nn.functional.silu(h)
    q, s = emu.q8_pack(a)
    assert torch.equal(q.cpu(), Q.pack(a.cpu())[0])
    z = emu.q8_gemm(q, s, *p2, r.offsets)
    ref = Q.product(q.cpu(), s.cpu(), p2[0].cpu(), p2[1].cpu(), r.offsets.cpu(), None)
    M.check(z, ref, Q.product_bar(ref, torch.bfloat16))
    y = emu.moe_combine(z, r.slots, r.weights)
    # against 16-bit products: each packing is off by half a 127th of a row's largest entry, 0.4 %
    # of it, some 1.2 % of a typical one; four packings, which add up at random
    full = emu.moe_combine(emu.grouped_gemm(torch.nn.functional.silu(
        emu.grouped_gemm(x, W1, r.offsets, transb="T", rows=r.rows)), W2, r.offsets, transb="T"), r.slots, r.weights)
    assert float((y.float() - full.float()).norm() / full.float().norm()) < 0.05


@pytest.mark.parametrize("kind", list(M.TYPES))
@pytest.mark.parametrize("R,K", [(9, 100), (300, 160), (900, 1600)])
def test_results_below_the_normal_range(emu, kind, R, K):
    """Subnormal results of the type: off by at most half their spacing, and by the roundings
    in FP32 before."""
    X, xs, W, ws, _, _ = _operands(R, R, 1, 140, K, False)
    top = {"f32": 2.0 ** -126, "bf16": 2.0 ** -126, "f16": 2.0 ** -14}[kind]
    xs = torch.full((R,), top / 128)
    ws = torch.full((1, 140), 1.0 / (128 * K ** 0.5 * 16))
    ref = Q.product(X, xs, W, ws, None, None)
    assert (ref.abs() < top).all() and (ref.abs() > top * 2.0 ** -8).any()
    got = emu.q8_gemm(X.cuda(), xs.cuda(), W.cuda(), ws.cuda(), dtype=M.TYPES[kind])
    # in float32 and bfloat16 the product of the scales' rounding is subnormal too
    M.check(got, ref, Q.product_bar(ref, M.TYPES[kind]) + 2.0 ** -149)


def test_two_graphs_and_eager_calls_share_the_workspace(emu):
    """Graphs of a loss over many tokens, of a product on copies and of one in splits, replayed
    in turns with eager calls between."""
    gen = torch.Generator(device="cuda").manual_seed(1)
    logits = torch.randn((5000, 64), generator=gen, device="cuda")
    ids = torch.topk(logits, 4).indices.int().contiguous()
    a, sa = emu.q8_pack(torch.randn((3000, 501), generator=gen, device="cuda"))
    b, sb = emu.q8_pack(torch.randn((700, 501), generator=gen, device="cuda"))
    c, sc = emu.q8_pack(torch.randn((50, 30000), generator=gen, device="cuda"))
    d, sd = emu.q8_pack(torch.randn((70, 30000), generator=gen, device="cuda"))
    calls = [lambda: emu.moe_balance(logits, ids)[:3], lambda: (emu.q8_gemm(a, sa, b, sb),),
             lambda: (emu.q8_gemm(c, sc, d, sd),)]
    eager = [[t.clone() for t in f()] for f in calls]
    graphs, out = [], []
    for f in calls:
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out.append(f())
        graphs.append(graph)
    for i in (0, 1, 2, 1, 0, 2, 0):
        for t in out[i]:
            t.zero_()
        graphs[i].replay()
        again = [t.clone() for t in calls[(i + 1) % 3]()]
        torch.cuda.synchronize()
        assert all(torch.equal(u, v) for u, v in zip(out[i], eager[i]))
        assert all(torch.equal(u, v) for u, v in zip(again, eager[(i + 1) % 3]))
