"""Refusals of the recurrence's, the 8-bit form's and the packed join's entry points, before any device use."""
import ctypes

import pytest
import torch

from paper_2608_21308_b200 import binding as E
from paper_2608_21308_b200 import build as libbuild


@pytest.fixture(scope="module")
def L():
    libbuild.build()
    return E.lib()


vp = ctypes.c_void_p
GOOD, WS = vp(0x10000), vp(0x100000)
BIG = 1 << 45


def fwd(L, p, change={}, ws=WS, n=BIG, save=1):
    args = [GOOD] * 8
    for i, v in change.items():
        args[i] = v
    return L.e2ttt_scan_fwd(ctypes.byref(p), *args, ws, n, save, None)


def bwd(L, p, change={}, ws=WS, n=BIG, saved=1):
    args = [GOOD] * 13
    for i, v in change.items():
        args[i] = v
    return L.e2ttt_scan_bwd(ctypes.byref(p), *args, ws, n, saved, None)


def step(L, p, change={}):
    args = [GOOD] * 8
    for i, v in change.items():
        args[i] = v
    return L.e2ttt_scan_step(ctypes.byref(p), *args, None)


@pytest.mark.parametrize("field,value,status", [
    ("B", 0, -2), ("L", 0, -2), ("D", 0, -2), ("D", (1 << 20) + 1, -2), ("L", (1 << 30) + 1, -2), ("B", (1 << 24) + 1, -2), ("io_dtype", 2, -3), ("gate", 2, -2),
    ("gate", -1, -2), ("unit_scale", 2, -2),
])
def test_bad_parameters(L, field, value, status):
    p = E.make_scan_params(1, 3, 64)
    setattr(p, field, value)
    n = ctypes.c_size_t()
    assert L.e2ttt_scan_workspace_bytes(ctypes.byref(p), 1, ctypes.byref(n)) == status
    assert fwd(L, p) == bwd(L, p) == step(L, p) == status


def test_sizes_whose_product_is_too_large(L):
    assert fwd(L, E.make_scan_params(1 << 14, 1 << 20, 128)) == -2
    assert fwd(L, E.make_scan_params(1 << 20, 1, 1 << 11)) == -2


def test_null_pointers_gates_and_save(L):
    p, plain = E.make_scan_params(1, 3, 64), E.make_scan_params(1, 3, 64, gate=E.E2TTT_GATE_NONE)
    assert L.e2ttt_scan_workspace_bytes(ctypes.byref(p), 1, None) == -1
    for i in (0, 1, 2, 3, 6, 7):               # starts (4) and h_init (5) may be missing
        assert fwd(L, p, {i: None}) == -1
    for i in (0, 1, 2, 3, 6, 8, 9, 10, 11, 12):  # so may dh_final (7)
        assert bwd(L, p, {i: None}) == -1
    for i in (0, 1, 2, 3, 5, 6, 7):
        assert step(L, p, {i: None}) == -1
    assert fwd(L, plain) == bwd(L, plain) == step(L, plain) == -1          # a gate's input without a gate
    assert bwd(L, plain, {2: None}) == -1                                  # and its gradient
    for save in (-1, 3):
        assert fwd(L, p, save=save) == bwd(L, p, saved=save) == -2
        assert L.e2ttt_scan_workspace_bytes(ctypes.byref(p), save, ctypes.byref(ctypes.c_size_t())) == -2
    assert bwd(L, p, {0: None, 1: None, 2: None}, saved=0) == -1


def test_alignment_and_workspace(L):
    for io, odd in ((E.E2TTT_F32, 0x10002), (E.E2TTT_BF16, 0x10001)):
        p = E.make_scan_params(2, 130, 65, io)
        for i in (0, 1, 2, 6):
            assert fwd(L, p, {i: vp(odd)}) == -4
        for i in (3, 5, 7):
            assert fwd(L, p, {i: vp(0x10002)}) == step(L, p, {i: vp(0x10002)}) == -4
        for i in (0, 1, 2, 6, 8, 9, 10):
            assert bwd(L, p, {i: vp(odd)}) == -4
        for i in (3, 5, 7, 11, 12):
            assert bwd(L, p, {i: vp(0x10002)}) == -4
        for save in (1, 2):
            need = E.e2ttt_scan_workspace_bytes(p, save)
            assert need % 256 == 0 and need >= 256 + 2 * 3 * 65 * 4
            assert fwd(L, p, ws=None, save=save) == fwd(L, p, n=need - 1, save=save) == bwd(L, p, n=need - 1, saved=save) == bwd(L, p, ws=None, saved=save) == -5
            assert fwd(L, p, ws=vp(0x100010), save=save) == bwd(L, p, ws=vp(0x100010), saved=save) == -4
        assert bwd(L, p, n=E.e2ttt_scan_workspace_bytes(p, 1) - 1, saved=0) == -5
        assert E.e2ttt_scan_workspace_bytes(p, 0) == 0
        # two channel blocks, three spans of 64 tokens: codes and two scale bytes a token of x, a_decay and a_in
        assert E.e2ttt_scan_workspace_bytes(p, 2) - E.e2ttt_scan_workspace_bytes(p, 1) == 3 * 2 * 2 * 192 * 66


def test_eight_bit_form(L):
    def both(p, change={}):
        args = [GOOD] * 3
        for i, v in change.items():
            args[i] = v
        a = L.e2ttt_pack8(ctypes.byref(p), *args, None)
        assert L.e2ttt_unpack8(ctypes.byref(p), args[1], args[2], args[0], None) == a
        return a

    for field, value, status in (("rows", 0, -2), ("cols", 0, -2), ("cols", (1 << 30) + 1, -2), ("rows", (1 << 40) + 1, -2), ("io_dtype", 5, -3)):
        p = E.make_pack_params(3, 40)
        setattr(p, field, value)
        assert both(p) == status
    assert both(E.make_pack_params(1 << 35, 33)) == -2
    p = E.make_pack_params(3, 40)
    for i in range(3):
        assert both(p, {i: None}) == -1
    assert both(p, {0: vp(0x10002)}) == both(E.make_pack_params(3, 40, E.E2TTT_BF16), {0: vp(0x10001)}) == -4


def test_packed_join(L):
    p = E.make_join_params(1, 2, 3, 65, gate=E.E2TTT_GATE_SILU)
    plain = E.make_join_params(1, 2, 3, 65, gate=E.E2TTT_GATE_NONE)
    keep, need = E.e2ttt_join_packed_bytes(p), E.e2ttt_join_workspace_bytes(p)
    assert keep == 3 * 3 * (160 + 8) and E.e2ttt_join_packed_bytes(plain) == 2 * 3 * (160 + 8)
    assert L.e2ttt_join_packed_bytes(ctypes.byref(p), None) == -1

    def fwd(change={}, q=p, packed=WS, n=keep):
        args = [GOOD] * 8
        for i, v in change.items():
            args[i] = v
        return L.e2ttt_join_fwd_packed(ctypes.byref(q), *args, packed, n, None)

    def bwd(change={}, q=p, packed=WS, n=keep, ws=WS, m=need):
        args = [GOOD] * 11
        for i, v in change.items():
            args[i] = v
        return L.e2ttt_join_bwd_packed(ctypes.byref(q), packed, n, *args, ws, m, None)

    for i in range(8):
        assert fwd({i: None}) == -1
    for i in range(11):
        assert bwd({i: None}) == -1
    assert fwd(q=plain) == bwd(q=plain) == -1
    assert fwd(packed=None) == fwd(n=keep - 1) == bwd(packed=None) == bwd(n=keep - 1) == bwd(ws=None) == bwd(m=need - 1) == -5
    assert fwd(packed=vp(0x100080)) == bwd(packed=vp(0x100080)) == bwd(ws=vp(0x100080)) == -4
    p.gate = 7
    assert fwd() == bwd() == -2


def test_binding_refuses_host_tensors_and_wrong_shapes():
    t = torch.zeros(1, 2, 8)
    with pytest.raises(TypeError):
        E.e2ttt_scan_fwd(E.make_scan_params(1, 2, 8), t, t, t, t, None, None, t, t)
    with pytest.raises(TypeError):
        E.e2ttt_pack8(E.make_pack_params(2, 8), t, t, t)
