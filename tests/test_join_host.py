"""Refusals of the block join's entry points, before any device use."""
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
GOOD = vp(0x10000)
WS = vp(0x100000)


@pytest.mark.parametrize("field,value,status", [
    ("B", 0, -2), ("H", 0, -2), ("L", 0, -2), ("L", (1 << 30) + 1, -2), ("d", 0, -2), ("d", 8193, -2), ("H", 129, -2), ("io_dtype", 3, -3), ("gate", 3, -2),
    ("post_eps", -1.0, -2), ("pre_eps", float("nan"), -2),
])
def test_bad_parameters(L, field, value, status):
    p = E.make_join_params(1, 2, 3, 64)
    setattr(p, field, value)
    n = ctypes.c_size_t()
    assert L.e2ttt_join_workspace_bytes(ctypes.byref(p), ctypes.byref(n)) == status
    assert L.e2ttt_join_fwd(ctypes.byref(p), *[GOOD] * 8, None) == status


def test_null_pairs_alignment_and_workspace(L):
    p = E.make_join_params(1, 2, 3, 64, gate=E.E2TTT_GATE_SILU)
    plain = E.make_join_params(1, 2, 3, 64, gate=E.E2TTT_GATE_NONE)
    need = E.e2ttt_join_workspace_bytes(p)
    assert need == 256 + 3 * 2 * 128 * 4

    def fwd(change, q=p):
        args = [GOOD] * 8
        for i, v in change.items():
            args[i] = v
        return L.e2ttt_join_fwd(ctypes.byref(q), *args, None)

    def bwd(change, q=p, ws=WS, n=need):
        args = [GOOD] * 14
        for i, v in change.items():
            args[i] = v
        return L.e2ttt_join_bwd(ctypes.byref(q), *args, ws, n, None)

    for i in range(8):
        assert fwd({i: None}) == -1           # w_pre (5) and n_out (7) come together
    for i in range(14):
        assert bwd({i: None}) == -1
    assert fwd({}, plain) == -1               # a gate's input without a gate
    assert bwd({1: None}, plain) == -1        # d_a without a gate
    assert fwd({2: vp(0x10002)}) == bwd({6: vp(0x10002)}) == fwd({3: vp(0x10001)}) == -4
    assert bwd({}, ws=None) == bwd({}, n=need - 1) == -5
    assert bwd({}, ws=vp(0x100010)) == -4


def test_binding_refuses_host_tensors():
    p = E.make_join_params(1, 1, 2, 8)
    t = torch.zeros(1, 1, 2, 8)
    with pytest.raises(TypeError):
        E.e2ttt_join_fwd(p, t, t, t, t, t, t, t, t)
