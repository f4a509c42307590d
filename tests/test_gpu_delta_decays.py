"""Gradient of the decays' logarithms over the whole range of decays, judged against its own size.

A token that forgets the state makes its gradient exp(log_gamma) times what it would be, and everything that the gradient is a sum of with it, so the
error is relative to the tensor's norm whatever the decay.  Tolerance: a value is a sum of products of three computed quantities (e, dP or dO, the state or
its adjoint), each behind at most four products with operands of 22 bits: errors of 2^-22 / sqrt(3) each, 12 of them with random signs, 4.8e-7, and
some ten truncations of 2^-24 in the mean, 6e-7: 2e-6.
"""
import numpy as np
import pytest
import torch

from oracle import delta as O
from tests.test_gpu_delta import Run, _make

pytestmark = pytest.mark.gpu
TOL = 2e-6


def _near(got, ref, tol=TOL):
    got = got.double().cpu().numpy()
    assert np.isfinite(got).all()
    err, size = np.linalg.norm(got - ref), np.linalg.norm(ref)
    assert err <= tol * size, (err / size, size)


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("start", [True, False])
@pytest.mark.parametrize("log_gamma", [0.0, -0.01, -1.0, -3.0, -8.0, -16.0, -40.0])
@pytest.mark.parametrize("shape", [(1, 4, 4, 256, 64, 64), (2, 6, 2, 97, 72, 100), (4, 10, 5, 130, 128, 64)])
def test_one_steady_decay(io, start, log_gamma, shape):
    x, d = _make(*shape, io, seed=21, start=start)
    x["log_gamma"][:] = log_gamma
    r = Run(x, io, shape[4] ** -0.5)
    r.fwd(1)
    _near(r.bwd(d)["d_log_gamma"], O.backward(**x, scale=shape[4] ** -0.5, **d)["d_log_gamma"])


@pytest.mark.parametrize("io", ["f32", "bf16"])
def test_without_a_start_state_the_first_token_has_no_gradient(io):
    for L in (1, 40, 70):
        x, d = _make(1, 3, 3, L, 64, 64, io, seed=22, start=False)
        r = Run(x, io, 1.0)
        r.fwd(1)
        assert (r.bwd(d)["d_log_gamma"][:, :, 0] == 0).all()


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("at", [20, 32, 50, 64, 75])
def test_a_document_behind_a_reset_leaves_the_one_before_alone(io, at):
    """The second document's values and gradients are 2^10 times the first's: at one scale with them the first keeps 22 - 10 + 11 bits or more (the second
    terms reach 2^-37 of the largest value)."""
    x, d = _make(1, 4, 4, 120, 64, 64, io, seed=23)
    x["log_gamma"][:, :, at] = -np.inf
    x["v"][:, :, at:] *= np.float32(1024)
    d["d_o"][:, :, at:] *= np.float32(1024)
    r = Run(x, io, 1.0)
    r.fwd(1)
    got, ref = r.bwd(d)["d_log_gamma"], O.backward(**x, scale=1.0, **d)["d_log_gamma"]
    _near(got[:, :, :at], ref[:, :, :at])
    _near(got[:, :, at:], ref[:, :, at:])
    assert (got[:, :, at] == 0).all()
