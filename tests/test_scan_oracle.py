"""The recurrence's oracle: its gradients against central differences of its own forward, and the 8-bit form's against its definition."""
import numpy as np
import pytest

from oracle import pack8 as K
from oracle import scan as O


@pytest.mark.parametrize("gate", [True, False])
@pytest.mark.parametrize("unit", [True, False])
@pytest.mark.parametrize("docs", [True, False])
def test_gradients_are_differences(gate, unit, docs):
    rng = np.random.default_rng(3)
    B, L, D = 2, 7, 3
    t = {n: rng.standard_normal((B, L, D)) for n in ("x", "r", "g", "d_h")}
    rate, h0, end = rng.uniform(0.05, 2.0, D), rng.standard_normal((B, D)), rng.standard_normal((B, D))
    starts = np.zeros((B, L), np.uint8)
    starts[0, 3] = starts[1, 0] = 1
    args = {"x": t["x"], "r": t["r"], "g": t["g"] if gate else None, "rate": rate, "starts": starts if docs else None, "h0": h0, "unit": unit}

    def loss():
        h, last, _ = O.forward(**args)
        return (h * t["d_h"]).sum() + (last * end).sum()

    grads, terms = O.backward(**args, d_h=t["d_h"], dh_final=end)
    names = {"x": "d_x", "r": "da_decay", "rate": "d_rate", "h0": "dh_init", **({"g": "da_in"} if gate else {})}
    for n, m in names.items():
        flat, want = args[n].reshape(-1), grads[m].reshape(-1)
        assert (np.abs(want) <= terms[m].reshape(-1) + 1e-12).all()
        for j in range(flat.size):
            keep, step = flat[j], 1e-6
            flat[j] = keep + step
            up = loss()
            flat[j] = keep - step
            down = loss()
            flat[j] = keep
            assert abs((up - down) / (2 * step) - want[j]) < 2e-8 * max(1.0, np.abs(want).max()) * 10, (m, j)


def test_kept_inputs_equal_to_the_inputs_change_nothing():
    rng = np.random.default_rng(4)
    B, L, D = 1, 150, 5
    x, r, g, d_h = (rng.standard_normal((B, L, D)) for _ in range(4))
    a = O.backward(x, r, g, np.full(D, 0.1), None, None, True, d_h, None)[0]
    b = O.backward(x, r, g, np.full(D, 0.1), None, None, True, d_h, None, kept=(x, r, g))[0]
    for n in a:
        assert np.array_equal(a[n], b[n]), n


def test_eight_bits_are_off_by_half_a_step_and_the_scale_is_the_smallest():
    rng = np.random.default_rng(5)
    x = rng.standard_normal((9, 70)) * np.exp(rng.standard_normal((9, 1)) * 6)
    x[0, :32] = 0
    x[1, 33] = 127.0
    x[1, 34:] = 0.5
    codes, scales = K.pack(x)
    back = K.unpack(codes, scales)
    for j in range(3):
        v, e = x[:, 32 * j:32 * j + 32], scales[:, j].astype(int) - 127
        big = np.abs(v).max(1)
        assert (127 * 2.0 ** e >= big).all() and ((127 * 2.0 ** (e - 1) < big) | (big == 0)).all()
        assert (np.abs(back[:, 32 * j:32 * j + 32] - v) <= 2.0 ** (e - 1.0)[:, None]).all()
        assert (np.abs(back[:, 32 * j:32 * j + 32] - v).max(1) <= big / 127 * (1 + 1e-12)).all()
    assert scales[1, 1] == 127 and (scales[0, 0], codes[0, 0]) == (1, 0)
    assert np.isnan(K.through(np.array([[1.0, np.inf] + [2.0] * 31])))[0].sum() == 32
