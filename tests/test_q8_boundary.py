"""Refusals of the 8-bit operators and of the balance loss (no kernel is launched): the
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


def test_balance(L):
    good = (0, 4, 8, 2, 3, P, 8, P, P, P, P, P, P)
    _refused(L.emu_moe_balance, good, [(0, 3), (1, -1), (1, 1 << 24), (2, 0), (2, 1025), (3, 0), (3, 9), (4, 0),
                                       (4, (1 << 16) + 1), (5, None), (6, 7), (7, None), (8, None), (9, None),
                                       (10, None), (11, None), (12, None)])
    assert L.emu_moe_balance(*_with(_with(_with(good, 2, 64), 6, 64), 3, 33)) == EINVAL    # k > 32
    good = (0, 4, 8, 3, P, 8, P, P, P, P, None, P, 8)
    _refused(L.emu_moe_balance_grad, good, [(0, -1), (1, -1), (2, 0), (3, 0), (4, None), (5, 7), (6, None),
                                            (7, None), (8, None), (9, None), (11, None), (12, 7)])
    assert L.emu_moe_balance_grad(*_with(good, 1, 0)) == OK


def test_q8_rows(L):
    good = (1, 4, 100, P, 100, P, 100, P)
    _refused(L.emu_q8_pack, good, [(0, 3), (1, -1), (1, 1 << 31), (2, -1), (2, 1 << 30), (3, None), (4, 99), (5, None),
                                   (6, 99), (7, None)])
    assert L.emu_q8_pack(*_with(good, 1, 0)) == OK
    good = (1, 4, 100, P, 100, P, P, 100)
    _refused(L.emu_q8_unpack, good, [(0, 3), (1, -1), (2, -1), (3, None), (4, 99), (5, None), (6, None), (7, 99)])
    assert L.emu_q8_unpack(*_with(good, 1, 0)) == OK and L.emu_q8_unpack(*_with(good, 2, 0)) == OK


def test_q8_product(L):
    good = (2, 3, 10, 16, 8, P, 8, P, 10, None, P, 8, 128, P, P, P, 16)
    _refused(L.emu_q8_gemm, good, [(0, 3), (1, -1), (1, 1 << 17), (2, -1), (3, -1), (4, -1), (5, None), (6, 7),
                                   (7, None), (8, 9), (10, None), (11, 7), (12, -1), (13, None), (14, None),
                                   (15, None), (16, 15)])
    assert L.emu_q8_gemm(*_with(good, 2, 0)) == OK and L.emu_q8_gemm(*_with(good, 3, 0)) == OK
    long = _with(_with(_with(good, 4, 131072), 6, 131072), 11, 131072)
    assert L.emu_q8_gemm(*_with(long, 12, 16 * 131072)) == EINVAL       # sums beyond 32 bits
    huge = (2, 1, (1 << 31) - 1, 1 << 20, 8, P, 8, P, (1 << 31) - 1, None, P, 8, 0, P, None, P, 1 << 20)
    assert L.emu_q8_gemm(*huge) == EINVAL


def _i(*shape):
    return torch.zeros(shape, dtype=torch.int32)


def test_binding_balance():
    x, ids = torch.zeros((4, 8)), _i(4, 2)
    for bad, err in ((x.double(), TypeError), (x[0], ValueError), ("x", TypeError), (x.T, ValueError)):
        with pytest.raises(err):
            emu.moe_balance(bad, ids)
    with pytest.raises(TypeError, match="ids"):
        emu.moe_balance(x, ids.long())
    with pytest.raises(ValueError, match="ids"):
        emu.moe_balance(x, ids[:3])
    for bad in (_i(1), _i(2, 2), [0, 4]):
        with pytest.raises(ValueError, match="starts"):
            emu.moe_balance(x, ids, bad)
    with pytest.raises(TypeError, match="starts"):
        emu.moe_balance(x, ids, _i(3).long())
    with pytest.raises(TypeError, match="GPU"):
        emu.moe_balance(x, ids)
    counts, tokens, d = _i(1, 8), _i(1), torch.zeros(1)
    with pytest.raises(ValueError, match="counts"):
        emu.moe_balance_grad(x, _i(2, 8), tokens, d)
    with pytest.raises(ValueError, match="tokens"):
        emu.moe_balance_grad(x, counts, _i(2), d)
    with pytest.raises(TypeError, match="dloss"):
        emu.moe_balance_grad(x, counts, tokens, 1.0)
    with pytest.raises(ValueError, match="dzloss"):
        emu.moe_balance_grad(x, counts, tokens, d, torch.zeros(2))
    with pytest.raises(TypeError, match="GPU"):
        emu.moe_balance_grad(x, counts, tokens, d)


def test_binding_q8():
    x = torch.zeros((4, 8))
    for bad, err in ((x.double(), TypeError), (x[0], ValueError), ("x", ValueError), (x.T, ValueError)):
        with pytest.raises(err):
            emu.q8_pack(bad)
    with pytest.raises(TypeError, match="GPU"):
        emu.q8_pack(x)
    q, s = x.to(torch.int8), torch.zeros(4)
    with pytest.raises(TypeError, match="Q must be"):
        emu.q8_unpack(x, s)
    with pytest.raises(ValueError, match="scales"):
        emu.q8_unpack(q, s[:3])
    with pytest.raises(TypeError, match="dtype"):
        emu.q8_unpack(q, s, torch.float64)
    with pytest.raises(TypeError, match="GPU"):
        emu.q8_unpack(q, s)
    W, ws = torch.zeros((3, 5, 8), dtype=torch.int8), torch.zeros((3, 5))
    off = _i(4)
    with pytest.raises(TypeError, match="X must be"):
        emu.q8_gemm(x, s, W, ws, off)
    with pytest.raises(TypeError, match="W must be"):
        emu.q8_gemm(q, s, W.float(), ws, off)
    with pytest.raises(ValueError, match="inner"):
        emu.q8_gemm(q[:, :7], s, W, ws, off)
    with pytest.raises(ValueError, match="needs offsets"):
        emu.q8_gemm(q, s, W, ws)
    with pytest.raises(ValueError, match="xscales"):
        emu.q8_gemm(q, s[:2], W, ws, off)
    with pytest.raises(ValueError, match="wscales"):
        emu.q8_gemm(q, s, W, ws[:, :4], off)
    with pytest.raises(TypeError, match="offsets"):
        emu.q8_gemm(q, s, W, ws, off.long())
    with pytest.raises(ValueError, match="rows"):
        emu.q8_gemm(q, s, W, ws, off, rows=_i(2, 2))
    with pytest.raises(TypeError, match="dtype"):
        emu.q8_gemm(q, s, W, ws, off, dtype=torch.int8)
    with pytest.raises(ValueError, match="Y must be"):
        emu.q8_gemm(q, s, W, ws, off, Y=torch.zeros((4, 4)))
    with pytest.raises(ValueError, match="row-major"):
        emu.q8_gemm(q, s, W.transpose(1, 2), torch.zeros((3, 8)), off)
    with pytest.raises(TypeError, match="GPU"):
        emu.q8_gemm(q, s, W, ws, off)
