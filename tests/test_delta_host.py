"""Refusals of the gated delta rule's entry points (before any device use) and the size of its workspace."""
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
GOOD = vp(0x10000)  # never dereferenced: validation fails first
WS = vp(0x100000)


@pytest.mark.parametrize("field,value,status", [
    ("B", 0, -2), ("H", 0, -2), ("Hk", 0, -2), ("L", 0, -2), ("L", -5, -2), ("dk", 0, -2), ("dk", 129, -2), ("dv", 0, -2), ("dv", 129, -2),
    ("Hk", 3, -2), ("io_dtype", 2, -3), ("scale", float("nan"), -2), ("scale", float("inf"), -2), ("B", 1 << 25, -2), ("L", (1 << 30) + 1, -2),
])
def test_bad_parameters(L, field, value, status):
    p = E.make_delta_params(1, 4, 2, 64, 64, 64)
    setattr(p, field, value)
    n = ctypes.c_size_t()
    assert L.e2ttt_delta_workspace_bytes(ctypes.byref(p), 0, ctypes.byref(n)) == status
    assert L.e2ttt_delta_step(ctypes.byref(p), *[GOOD] * 8, None) == status


def test_null_alignment_and_workspace(L):
    p = E.make_delta_params(1, 2, 1, 64, 64, 64)
    need = E.e2ttt_delta_workspace_bytes(p, 1)

    def fwd(i=None, value=None, ws=WS, n=need):
        args = [GOOD] * 8
        if i is not None:
            args[i] = value
        return L.e2ttt_delta_fwd(ctypes.byref(p), *args, ws, n, 1, None)

    def bwd(i=None, value=None, ws=WS, n=need):
        args = [GOOD] * 14
        if i is not None:
            args[i] = value
        return L.e2ttt_delta_bwd(ctypes.byref(p), *args, ws, n, 1, None)

    for i in (0, 1, 2, 3, 4, 6, 7):  # 5: S_init may be NULL
        assert fwd(i, None) == -1
    for i in (0, 1, 2, 3, 4, 6, 8, 9, 10, 11, 12, 13):  # 5, 7: S_init, dS_final
        assert bwd(i, None) == -1
    assert fwd(0, vp(0x10002)) == bwd(0, vp(0x10002)) == -4    # fp32 queries at two bytes
    assert fwd(5, vp(0x10002)) == bwd(7, vp(0x10001)) == -4
    assert fwd(ws=None) == bwd(ws=None) == -5
    assert fwd(n=need - 1) == bwd(n=need - 1) == -5
    assert fwd(ws=vp(0x100080)) == bwd(ws=vp(0x100080)) == -4
    assert L.e2ttt_delta_workspace_bytes(ctypes.byref(p), 0, None) == -1
    assert L.e2ttt_delta_workspace_bytes(None, 0, ctypes.byref(ctypes.c_size_t())) == -1
    for i in range(8):
        args = [GOOD] * 8
        args[i] = None
        assert L.e2ttt_delta_step(ctypes.byref(p), *args, None) == -1


def test_binding_refuses_host_tensors_and_other_shapes():
    p = E.make_delta_params(1, 2, 1, 64, 64, 64)
    t = torch.zeros(1, 1, 64, 64)
    with pytest.raises(TypeError):
        E.e2ttt_delta_step(p, t, t, t, t, t, t, t, t)


def test_workspace_grows_with_the_tokens_and_with_saved_states(L):
    size = lambda B, H, Hk, n, dk, dv, io, save: E.e2ttt_delta_workspace_bytes(E.make_delta_params(B, H, Hk, n, dk, dv, io), save)  # noqa: E731
    a = size(4, 16, 16, 4096, 128, 128, E.E2TTT_BF16, 0)
    assert a == 256 + 64 * 128 * (2 * 32 * 128 * 2 + 9216)
    assert size(4, 16, 16, 4096, 128, 128, E.E2TTT_F32, 0) > a
    assert size(4, 16, 4, 4096, 128, 128, E.E2TTT_BF16, 0) < a
    assert size(4, 16, 16, 4096, 128, 128, E.E2TTT_BF16, 1) > 3 * a
    assert size(1, 1, 1, 1, 1, 1, E.E2TTT_BF16, 0) >= 256 + 9216
    # sizes past 32 bits
    assert size(8, 16, 16, 1 << 20, 128, 128, E.E2TTT_F32, 1) > 1 << 35
