"""Gated delta rule: bounds of 0 beside large states and adjoints.  The product of two scales may leave fp32's range there, and nothing may become NaN of it."""
import numpy as np
import pytest

from oracle import delta as O
from tests.test_gpu_delta import Run, _make, check

pytestmark = pytest.mark.gpu

SHAPES = [(1, 2, 2, 128, 64, 64), (4, 20, 20, 128, 64, 32)]  # the columns of a slice over two warps; one warp per slice


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("case", ["zeros", "reset", "reset later", "one key", "unwritten", "far"])
def test_a_large_state_over_chunks_of_zeros(io, shape, case):
    """A chunk of padding (no keys, no values, no output gradients) has bounds of 0 beside a state and an adjoint of 2^50."""
    x, d = _make(*shape, io, seed=31)
    big = np.float32(2.0 ** 50)
    x["S"] *= big
    d["dS_final"] *= big
    x["log_gamma"][:] = 0
    c = slice(32, 64)
    for t in () if case == "far" else (x["q"], d["d_o"]) if case == "unwritten" else (x["k"], x["q"], x["v"], d["d_o"]):
        t[:, :, c] = 0
    if case == "reset":
        x["log_gamma"][:, :, 32] = -np.inf
    if case == "reset later":
        x["log_gamma"][:, :, 40] = -np.inf
    if case == "one key":  # one large key behind a reset
        x["log_gamma"][:, :, 63] = -np.inf
        x["k"][:, :, 63, 0] = 4096
        x["eta"][:, :, 63] = 0
    if case in ("unwritten", "far"):  # learning rates of 0
        x["eta"][:, :, c] = 0
    if case == "unwritten":  # large values that nothing writes
        x["v"][:, :, c] *= big
    if case == "far":  # a chunk that reads what is e^-60 of the state, and adds to no adjoint but its own
        x["log_gamma"][:, :, 32] = -60
        d["dS_final"][:] = 0
        d["d_o"][:, :, 64:] = 0
    o, S = O.forward(**x, scale=1.0)
    ref = O.backward(**x, scale=1.0, **d)
    r = Run(x, io, 1.0)
    check(r.fwd(1), {"o": o, "S": S})
    check(r.bwd(d), ref, dict(x, scale=1.0, **d))
    check(r.fwd(0), {"o": o, "S": S}, dict(x, scale=1.0))


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("values,gradients", [(50, 50), (50, -50), (-50, 50), (-50, -50)])
def test_ends_of_the_range_of_magnitudes(io, shape, values, gradients):
    x, d = _make(*shape, io, seed=37)
    for t, n in ((x["v"], values), (x["S"], values), (d["d_o"], gradients), (d["dS_final"], gradients)):
        t *= np.float32(2.0 ** (n - np.sign(n) * 3))  # the largest of them are within 2^3 of the typical ones
    o, S = O.forward(**x, scale=1.0)
    r = Run(x, io, 1.0)
    check(r.fwd(1), {"o": o, "S": S})
    check(r.bwd(d), O.backward(**x, scale=1.0, **d), dict(x, scale=1.0, **d))
    check(r.step(), {"o": o, "S": S})
