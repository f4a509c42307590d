"""Gated linear recurrence over many turns of a CTA: long sequences by the copy engine, whose stages are filled, stored from and filled again, by one CTA a sequence and by
clusters of 2, 3, 4, 6, 7 and 8, both directions, against the oracle in 64 bits, with long documents.  Tolerances are those of the recurrence's own test."""
import numpy as np
import pytest

from oracle import pack8 as K
from oracle import scan as O
from tests import test_gpu_scan as S

pytestmark = pytest.mark.gpu


def through(x):
    """What x is after being packed and read back, all blocks at once."""
    if x is None:
        return None
    x = np.asarray(x, np.float64)
    D = x.shape[-1]
    v = np.zeros((*x.shape[:-1], -(-D // 32) * 32))
    v[..., :D] = x
    v = v.reshape(-1, 32)
    m, e = np.frexp(np.abs(v).max(1))
    unit = np.exp2(np.maximum(e - np.where(m <= 127 / 128, 7, 6), -126.0))[:, None]
    return (np.rint(v / unit) * unit).reshape(*x.shape[:-1], -1)[..., :D]


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("B,L,D", [(140, 900, 64), (74, 1000, 64), (45, 1000, 72), (30, 1500, 72), (37, 2000, 64), (1, 20000, 64)])
def test_many_turns(io, B, L, D):
    x, d = S.make(B, L, D, io, seed=22)
    x["starts"] = (np.random.default_rng(23).random((B, L)) < 0.002).astype(np.uint8)
    kept = tuple(through(x[n]) for n in ("x", "r", "g"))
    assert np.array_equal(kept[0][0, :40], K.through(x["x"][0, :40]))
    tol = S.share(io, L)
    back = 2 * tol + S.GATE[io]
    h, last, mag = O.forward(**x)
    for save in ("states", "packed"):
        run = S.Run(x, io, save)
        out = run.fwd()
        S.near("h", out["h"], h, mag, tol)
        S.near("h_final", out["h_final"], last, mag[:, -1], tol)
        ref, terms = O.backward(**x, **d, kept=kept if save == "packed" else None)
        got = run.bwd(d)
        assert set(got) == set(ref)
        for n, t in got.items():
            S.near(n, t, ref[n], terms[n], back + (L / 8 + 64 + 16 * B) * 2.0 ** -24 if n == "d_rate" else back)
