"""The block join's oracle: its adjoint against differences."""
import numpy as np
import pytest

from oracle import join as O


@pytest.mark.parametrize("kind", ["none", "sigmoid", "silu"])
@pytest.mark.parametrize("pre", [True, False])
def test_adjoint_against_central_differences(kind, pre):
    rng = np.random.default_rng(0)
    B, H, L, d = 2, 3, 2, 4
    D = H * d
    x = {"o": rng.standard_normal((B, H, L, d)), "a": None if kind == "none" else rng.standard_normal((B, L, D)), "x": rng.standard_normal((B, L, D)),
         "w_post": rng.standard_normal(D), "res_scale": rng.standard_normal(D), "w_pre": rng.standard_normal(D) if pre else None}
    eps = dict(kind=kind, post_eps=0.1, pre_eps=0.2)
    d_x, d_n = rng.standard_normal((2, B, L, D))

    def loss(**change):
        xo, n = O.forward(**{**x, **change}, **eps)
        return (xo * d_x).sum() + ((n * d_n).sum() if pre else 0.0)

    got = O.backward(**x, **eps, d_x_out=d_x, d_n=d_n if pre else None)
    assert set(got) == {"d_" + n for n in x if x[n] is not None}
    h = 1e-6
    for n in x:
        if x[n] is None:
            continue
        for at in [tuple(rng.integers(0, k) for k in x[n].shape) for _ in range(8)]:
            up, down = x[n].copy(), x[n].copy()
            up[at] += h
            down[at] -= h
            assert abs((loss(**{n: up}) - loss(**{n: down})) / (2 * h) - got["d_" + n][at]) < 1e-7, n
