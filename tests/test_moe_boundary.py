"""Refusals of the mixture-of-experts entry points (no kernel is launched): the
library's EMU_EINVAL and the binding's exceptions."""
import ctypes

import pytest
import torch

import paper_2609_04663_amd as emu

P = ctypes.c_void_p(0x1000)     # never dereferenced: validation fails first
EINVAL, OK = emu.EMU_EINVAL, emu.EMU_OK


@pytest.fixture(scope="module")
def L():
    return emu.lib()


def _with(args, at, value):
    return tuple(value if i == at else a for i, a in enumerate(args))


def _refused(fn, good, bad):
    for at, value in bad:
        assert fn(*_with(good, at, value)) == EINVAL, (fn.__name__, at, value)
        assert emu.lib().emu_last_error()


def test_route(L):
    good = (0, 4, 8, 2, 0, P, 8, P, P, P, P, P)
    _refused(L.emu_moe_route, good, [(0, 3), (0, -1), (1, -1), (1, 1 << 24), (2, 0), (2, 1025), (3, 0),
                                     (3, 9), (4, 2), (6, 7), (5, None), (7, None), (8, None), (9, None),
                                     (10, None), (11, None)])
    assert L.emu_moe_route(*_with(_with(_with(good, 2, 64), 6, 64), 3, 33)) == EINVAL      # k > 32


def test_route_grad(L):
    good = (0, 4, 8, 2, 1, P, 8, P, P, P, P, 8)
    _refused(L.emu_moe_route_grad, good, [(0, 7), (1, -1), (2, 0), (3, 9), (4, -1), (6, 7), (11, 7),
                                          (5, None), (7, None), (8, None), (9, None), (10, None)])
    assert L.emu_moe_route_grad(*_with(good, 1, 0)) == OK


def test_combine(L):
    good = (1, 4, 16, 2, 8, P, 16, P, P, P, 16)
    _refused(L.emu_moe_combine, good, [(0, 3), (1, -1), (2, -1), (3, 0), (3, 33), (4, -1), (6, 15),
                                       (10, 15), (5, None), (7, None), (9, None)])
    assert L.emu_moe_combine(*_with(good, 1, 0)) == OK and L.emu_moe_combine(*_with(good, 2, 0)) == OK
    good = (1, 4, 16, 2, 8, P, 16, P, 16, P, P, P, P, 16, P)
    _refused(L.emu_moe_combine_grad, good, [(0, 3), (1, -1), (3, 0), (4, -1), (6, 15), (8, 15), (13, 15),
                                            (5, None), (7, None), (9, None), (10, None), (11, None),
                                            (12, None), (14, None)])
    assert L.emu_moe_combine_grad(*_with(_with(good, 1, 0), 4, 0)) == OK


def test_grouped(L):
    good = (2, b"N", 3, 10, 16, 8, P, 8, 10, None, P, 16, 128, P, P, 16)
    _refused(L.emu_grouped_gemm, good, [(0, 3), (1, b"X"), (2, -1), (2, 1 << 17), (3, -1), (4, -1), (5, -1),
                                        (6, None), (7, 7), (8, 9), (10, None), (11, 15), (12, -1),
                                        (13, None), (14, None), (15, 15)])
    assert L.emu_grouped_gemm(*_with(good, 3, 0)) == OK and L.emu_grouped_gemm(*_with(good, 4, 0)) == OK
    # E x N x K: the row length is K
    assert L.emu_grouped_gemm(*_with(_with(_with(good, 1, b"T"), 11, 7), 3, 0)) == EINVAL
    good = (2, b"N", 3, 10, 16, 8, P, 8, 10, None, P, 16, P, P, 16, 128)
    _refused(L.emu_grouped_wgrad, good, [(0, 3), (1, b"?"), (2, -1), (3, -1), (4, -1), (5, -1), (6, None),
                                         (7, 7), (8, 9), (10, None), (11, 15), (12, None), (13, None),
                                         (14, 15), (15, 127)])
    assert L.emu_grouped_wgrad(*_with(good, 2, 0)) == OK


def test_q4(L):
    good = (1, 2, 4, 16, 128, 64, P, 128, 4, None, P, P, None, P, P, 16)
    _refused(L.emu_q4_gemm, good, [(0, 3), (1, -1), (2, -1), (3, -1), (4, -64), (4, 96), (5, 16), (5, 256),
                                   (6, None), (7, 127), (8, 3), (10, None), (11, None), (13, None),
                                   (14, None), (15, 15)])
    assert L.emu_q4_gemm(*_with(good, 2, 0)) == OK
    good = (1, 4, 128, 32, P, 128, P, P)
    _refused(L.emu_q4_pack, good, [(0, 5), (1, -1), (2, 100), (3, 48), (4, None), (5, 127), (6, None),
                                   (7, None)])
    assert L.emu_q4_pack(*_with(good, 1, 0)) == OK


def _i(*shape):
    return torch.zeros(shape, dtype=torch.int32)


def test_binding_route():
    x = torch.zeros((4, 8))
    for bad, err in ((x.double(), TypeError), (x[0], ValueError), ("x", TypeError), (x.T, ValueError)):
        with pytest.raises(err):
            emu.moe_route(bad, 2)
    with pytest.raises(ValueError, match="scope"):
        emu.moe_route(x, 2, "some")
    with pytest.raises(TypeError, match="GPU"):
        emu.moe_route(x, 2)
    w = torch.zeros((4, 2))
    with pytest.raises(TypeError, match="ids"):
        emu.moe_route_grad(x, _i(4, 2).long(), w, w)
    with pytest.raises(ValueError, match="ids"):
        emu.moe_route_grad(x, _i(5, 2), w, w)
    with pytest.raises(ValueError, match="dweights"):
        emu.moe_route_grad(x, _i(4, 2), w, w[:, :1])
    with pytest.raises(TypeError, match="GPU"):
        emu.moe_route_grad(x, _i(4, 2), w, w)


def test_binding_combine():
    Z, w, s = torch.zeros((8, 16)), torch.zeros((4, 2)), _i(4, 2)
    with pytest.raises(TypeError, match="slots"):
        emu.moe_combine(Z, s.long(), w)
    with pytest.raises(TypeError, match="weights"):
        emu.moe_combine(Z, s, w.half())
    with pytest.raises(ValueError, match="Y must be"):
        emu.moe_combine(Z, s, w, Y=torch.zeros((4, 15)))
    with pytest.raises(TypeError, match="Y must be"):
        emu.moe_combine(Z, s, w, Y=torch.zeros((4, 16), dtype=torch.float16))
    with pytest.raises(ValueError, match="dY must be"):
        emu.moe_combine_grad(torch.zeros((3, 16)), Z, s, w, _i(8))
    with pytest.raises(ValueError, match="rows"):
        emu.moe_combine_grad(torch.zeros((4, 16)), Z, s, w, _i(7))
    with pytest.raises(TypeError, match="GPU"):
        emu.moe_combine(Z, s, w)


def test_binding_grouped():
    X, W, off = torch.zeros((10, 8)), torch.zeros((3, 8, 16)), _i(4)
    for bad, err in ((dict(W=W[:, :7]), ValueError), (dict(W=W.half()), TypeError), (dict(W=W[0]), ValueError),
                     (dict(W=W.transpose(1, 2), transb="T"), ValueError), (dict(offsets=_i(3)), ValueError),
                     (dict(offsets=None), TypeError), (dict(offsets=off.long()), TypeError),
                     (dict(rows=_i(2, 5)), ValueError), (dict(rows=torch.zeros(5)), TypeError),
                     (dict(transb="X"), ValueError), (dict(Y=torch.zeros((9, 16))), ValueError),
                     (dict(X=X.double()), TypeError), (dict(), TypeError)):
        with pytest.raises(err):
            emu.grouped_gemm(**{**dict(X=X, W=W, offsets=off), **bad})
    dY = torch.zeros((10, 16))
    for bad, err in ((dict(dY=dY[:9]), ValueError), (dict(dY=dY.half()), TypeError), (dict(rows=_i(9)), ValueError),
                     (dict(dW=torch.zeros((3, 16, 8))), ValueError), (dict(offsets="x"), ValueError),
                     (dict(transb="n"), ValueError), (dict(), TypeError)):
        with pytest.raises(err):
            emu.grouped_wgrad(**{**dict(X=X, dY=dY, offsets=off), **bad})


def test_binding_q4():
    X, s = torch.zeros((4, 128)), torch.zeros((2, 16, 2))
    Q, off = torch.zeros((2, 16, 64), dtype=torch.uint8), _i(3)
    for bad, err in ((dict(Q=Q.int()), TypeError), (dict(Q=Q[..., :32]), ValueError), (dict(scales=s[..., :1].repeat(1, 1, 3)), ValueError),
                     (dict(scales=s.half()), TypeError), (dict(scales=s[:1]), ValueError), (dict(mins=s[..., :1]), ValueError),
                     (dict(offsets=None), ValueError), (dict(offsets=_i(4)), ValueError), (dict(Y=torch.zeros((4, 17))), ValueError),
                     (dict(Q=Q[:, ::2]), ValueError), (dict(), TypeError)):
        with pytest.raises(err):
            emu.q4_gemm(**{**dict(X=X, Q=Q, scales=s, offsets=off), **bad})
    for bad, err in ((dict(W=torch.zeros(64)), ValueError), (dict(W=torch.zeros((4, 64)).double()), TypeError),
                     (dict(group=48), ValueError), (dict(W=torch.zeros((4, 96))), ValueError), (dict(), TypeError)):
        with pytest.raises(err):
            emu.q4_pack(**{**dict(W=torch.zeros((4, 64)), group=64), **bad})


def test_leading_dimensions_of_the_grouped_products(L):
    big = 1 << 31
    good = (2, b"N", 3, 10, 16, 8, P, 8, 10, None, P, 16, 128, P, P, 16)
    _refused(L.emu_grouped_gemm, good, [(7, big), (11, big), (15, big)])
    good = (2, b"N", 3, 10, 16, 8, P, 8, 10, None, P, 16, P, P, 16, 128)
    _refused(L.emu_grouped_wgrad, _with(good, 15, 8 * big), [(7, big), (11, big), (14, big)])
    # more tiles than a launch has workgroups
    good = (2, b"N", 1, 1 << 30, 1 << 20, 8, P, 8, 1 << 30, None, P, 1 << 20, 1 << 23, P, P, 1 << 20)
    assert L.emu_grouped_gemm(*good) == EINVAL
