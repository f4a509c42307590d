"""Logits without bound, masked ones, kept in 8 bits: they count as they do in the forward, from -43 (and, where a sigmoid is 1, to 43), and cost their block of 32 channels nothing more.
Tolerances are those of the recurrence's own test; sums behind a shut gate are as in its test of gates wide open and shut."""
import numpy as np
import pytest

from oracle import pack8 as K
from oracle import scan as O
from tests import test_gpu_scan as S

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("gate", [True, False])
@pytest.mark.parametrize("L,D", [(150, 64), (150, 66), (150, 65), (1100, 72)])
@pytest.mark.parametrize("far", [np.inf, 3e38, 1000.0, 44.0])
def test_unbounded_logits(io, gate, L, D, far):
    x, d = S.make(1, L, D, io, gate, True, True, seed=30)
    far = S.inputs.round_bf16(np.array([far], np.float32)).item() if io == "bf16" and np.isfinite(far) else np.float32(far)
    x["r"][:, ::7, 3], x["r"][:, 1::5, 40], x["r"][:, 20:30, 61] = -far, far, -far
    if gate:
        x["g"][:, ::6, 5], x["g"][:, 2::9, 41], x["g"][:, 40:50, 62] = -far, far, -far
    run = S.Run(x, io, "packed")
    out, got = run.fwd(), run.bwd(d)
    x["r"], x["g"] = (None if x[n] is None else np.clip(x[n], -43.0, 43.0) for n in ("r", "g"))
    kept = tuple(None if x[n] is None else K.through(x[n]) for n in ("x", "r", "g"))
    extra = 43 * 2.0 ** -22 if io == "bf16" else 0.0  # the rounding of the exponential's argument
    S.check_forward(out, x, io, extra)
    ref, mag = O.backward(**x, **d, kept=kept)
    tol = 2 * S.share(io, L, extra) + S.GATE[io]
    assert set(got) == set(ref)
    for n, t in got.items():
        S.near(n, t, ref[n], mag[n], tol + (L / 8 + 80) * 2.0 ** -24 if n == "d_rate" else tol)


@pytest.mark.parametrize("io", ["f32", "bf16"])
def test_a_nan_beside_an_unbounded_logit_is_still_a_nan(io):
    x, d = S.make(1, 70, 64, io, seed=31)
    x["r"][0, 10, 4], x["r"][0, 10, 9] = -np.inf, np.nan
    run = S.Run(x, io, "packed")
    run.fwd()
    got = run.bwd(d)
    assert not np.isfinite(got["da_decay"][0, 10, :32].float().cpu().numpy()).any()
    assert np.isfinite(got["da_decay"][0, :, 32:].float().cpu().numpy()).all()
