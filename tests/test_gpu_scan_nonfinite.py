"""Gated linear recurrence: which values a NaN or an infinity reaches.  Compared with the recurrence in 64 bits, token by token: the same values are finite, and no others, whatever the decays
(products of decays that underflow in 32 bits cut nothing off; only a start does), rows (copy engine, words, values) and number of CTAs per sequence."""
import numpy as np
import pytest
import torch

from oracle import pack8 as K
from oracle import scan as O
from tests import test_gpu_scan as S

pytestmark = pytest.mark.gpu
STARTS = (100, 229)  # both within a run of eight tokens, and of sixteen


def same(got, ref):
    for n, t in got.items():
        finite, want = torch.isfinite(t).cpu().numpy(), np.isfinite(ref[n])
        assert np.array_equal(finite, want), (n, np.argwhere(finite != want)[:5], int((finite != want).sum()))


def make(L, D, io, docs, where, t, bad, gate=True, unit=True):
    x, d = S.make(1, L, D, io, gate, unit, seed=20)
    x["rate"][::3] = 60.0  # four tokens' decays underflow
    x["rate"][1::6] = 2.0  # a hundred tokens' do
    x["r"] = np.abs(x["r"])
    if docs:
        x["starts"] = np.zeros((1, L), np.uint8)
        x["starts"][0, [s for s in (*STARTS, 1500) if s < L]] = 1
    for c in (3, 40, 61):  # rates of 60, of 2, and near 1
        (d if where == "d_h" else x)[where][0, t, c] = bad
    return x, d


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("docs", [False, True])
@pytest.mark.parametrize("L,D", [(333, 64), (333, 66), (333, 65), (2100, 72)])
@pytest.mark.parametrize("where,t,bad", [("x", 0, np.inf), ("x", 37, np.nan), ("r", 102, np.nan), ("g", 107, np.nan), ("d_h", 290, np.nan), ("d_h", 103, -np.inf)])
def test_the_values_that_are_not_finite_are_the_definitions(io, docs, L, D, where, t, bad):
    x, d = make(L, D, io, docs, where, t, bad)
    with np.errstate(invalid="ignore", over="ignore"):
        h, last, _ = O.forward(**x)
        grads = {save: O.backward(**x, **d, kept=kept)[0] for save, kept in (("states", None), ("packed", tuple(K.through(x[n]) for n in ("x", "r", "g"))))}
    for save, ref in grads.items():
        run = S.Run(x, io, save)
        same(run.fwd(), {"h": h, "h_final": last})
        same(run.bwd(d), ref)
    if L < 1000:
        same(S.Run(x, io).step(), {"h": h, "h_final": last})


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("docs", [False, True])
def test_without_an_input_gate_and_unit_scale(io, docs):
    x, d = make(333, 72, io, docs, "x", 3, np.inf, gate=False, unit=False)
    with np.errstate(invalid="ignore", over="ignore"):
        h, last, _ = O.forward(**x)
        ref = O.backward(**x, **d)[0]
    run = S.Run(x, io)
    same(run.fwd(), {"h": h, "h_final": last})
    same(run.bwd(d), ref)


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("gate,unit", [(True, True), (True, False), (False, True)])
@pytest.mark.parametrize("D", [64, 66, 65])
@pytest.mark.parametrize("L", [333, 2100])
def test_the_decay_logit_of_a_start_is_not_used(io, gate, unit, D, L):
    """A NaN there changes nothing, bit for bit, and its gradient is zero."""
    x, d = S.make(1, L, D, io, gate, unit, seed=21)
    x["starts"] = np.zeros((1, L), np.uint8)
    first = np.array([0, *STARTS, 230, 255, L - 1])
    x["starts"][0, first] = 1
    outs = []
    for logit in (-43.0, np.nan):
        x["r"][0, first] = logit
        outs.append({})
        for save in ("none", "states", "packed"):
            run = S.Run(x, io, save)
            outs[-1].update({(save, n): t for n, t in {**run.fwd(), **run.bwd(d)}.items()})
        outs[-1].update({("step", n): t for n, t in S.Run(x, io).step().items()})
    for n, t in outs[0].items():
        assert torch.equal(t, outs[1][n]), n
        if n[1] == "da_decay":
            assert not bool(t[0, first].any())
