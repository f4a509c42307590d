"""The oracle of the gated delta rule: its adjoint against differences, its start from zeros, its relation to the plain outer product."""
import numpy as np
import pytest

from oracle import delta as O


def _case(seed, B=1, H=4, Hk=2, L=5, dk=3, dv=4):
    rng = np.random.default_rng(seed)
    q, k = rng.standard_normal((2, B, Hk, L, dk)) * 0.5
    return {"q": q, "k": k, "v": rng.standard_normal((B, H, L, dv)), "eta": rng.uniform(0, 1, (B, H, L)),
            "log_gamma": -rng.uniform(0, 1, (B, H, L)), "S": rng.standard_normal((B, H, dv, dk))}


@pytest.mark.parametrize("name,grad", [("q", "dq"), ("k", "dk"), ("v", "dv"), ("eta", "d_eta"), ("log_gamma", "d_log_gamma"), ("S", "dS")])
def test_adjoint_against_central_differences(name, grad):
    x = _case(3)
    rng = np.random.default_rng(4)
    d_o, dS = rng.standard_normal(x["v"].shape), rng.standard_normal(x["S"].shape)

    def loss(**change):
        o, S = O.forward(**{**x, **change}, scale=0.7)
        return (o * d_o).sum() + (S * dS).sum()

    got = O.backward(**x, scale=0.7, d_o=d_o, dS_final=dS)[grad]
    h = 1e-6  # truncation h^2 = 1e-12, rounding 1e-16 |loss| / h ~ 1e-9
    for at in [tuple(rng.integers(0, n) for n in x[name].shape) for _ in range(12)]:
        up, down = x[name].copy(), x[name].copy()
        up[at] += h
        down[at] -= h
        assert abs((loss(**{name: up}) - loss(**{name: down})) / (2 * h) - got[at]) < 1e-7


def test_first_token_from_zeros_and_a_forgotten_state():
    x = _case(5)
    o, S = O.forward(**{**x, "S": None}, scale=1.0)
    k = np.repeat(x["k"], 2, 1)[:, :, 0]
    q = np.repeat(x["q"], 2, 1)[:, :, 0]
    assert np.allclose(o[:, :, 0], x["eta"][:, :, 0, None] * x["v"][:, :, 0] * (k * q).sum(-1, keepdims=True))
    x["log_gamma"][:, :, 2] = -np.inf  # tokens from 2 on see nothing of what was before
    o1, S1 = O.forward(**x, scale=1.0)
    tail = {n: (x[n][:, :, 2:] if n != "S" else None) for n in x}
    o2, S2 = O.forward(**tail, scale=1.0)
    assert np.allclose(o1[:, :, 2:], o2) and np.allclose(S1, S2)


def test_recomputing_tokens_in_two_calls():
    x = _case(7, L=9)
    o, S = O.forward(**x, scale=0.3)
    a = {n: (x[n][:, :, :4] if n != "S" else x[n]) for n in x}
    o1, S1 = O.forward(**a, scale=0.3)
    b = {n: (x[n][:, :, 4:] if n != "S" else S1) for n in x}
    o2, S2 = O.forward(**b, scale=0.3)
    assert np.allclose(np.concatenate([o1, o2], 2), o) and np.allclose(S2, S)
