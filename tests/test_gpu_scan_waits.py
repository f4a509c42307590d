"""Gated linear recurrence: device-side waits that give up, made to by a limit of no cycles.  Nothing finite comes out of what was not waited for, starts or not; the calls end, and the next
ones run clean."""
import pytest
import torch

from paper_2608_21308_b200 import binding as E
from tests import test_gpu_scan as S

pytestmark = pytest.mark.gpu


@pytest.fixture
def impatient():
    yield lambda: E.e2ttt_selftest_scan_wait_limit(0)
    E.e2ttt_selftest_scan_wait_limit(-1)


def nothing(out, starts=None):
    for n, t in out.items():
        known = torch.isnan(t)
        if n == "da_decay" and starts is not None:  # a start's is 0 whatever the inputs are
            known = known | torch.tensor(starts != 0, device="cuda")[..., None] & (t == 0)
        assert bool(known.all()), (n, torch.argwhere(~known)[:4])


# clusters of eight by the copy engine; several turns of one CTA and of clusters of two; clusters without the copy engine
@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("save", ["states", "packed"])
@pytest.mark.parametrize("gate,unit", [(True, True), (False, False)])
@pytest.mark.parametrize("B,L,D,docs", [(1, 2100, 72, True), (300, 600, 64, True), (1, 50, 64, True), (1, 1000, 66, False), (1, 1000, 65, False)])
def test_waits_that_give_up(impatient, io, save, gate, unit, B, L, D, docs):
    x, d = S.make(B, L, D, io, gate, unit, docs, seed=24)
    run = S.Run(x, io, save)
    clean = run.fwd()
    grads = run.bwd(d)
    impatient()
    nothing(run.bwd(d), x["starts"])
    out = run.fwd()
    nothing(out)
    E.e2ttt_selftest_scan_wait_limit(-1)
    if save == "packed" and docs:  # what was left for the reverse pass is nothing either
        got = run.bwd(d)
        nothing({n: got[n] for n in ("d_x", "da_decay") if gate or n != "d_x"}, x["starts"])
    for n, t in {**run.fwd(), **run.bwd(d)}.items():
        assert torch.equal(t, {**clean, **grads}[n]), n
