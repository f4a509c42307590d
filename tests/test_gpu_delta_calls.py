"""Gated delta rule: what a call gives beside other calls of the same inputs."""
import pytest
import torch

from oracle import delta as O
from tests.test_gpu_delta import SHAPES, Run, _make, check

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("shape", SHAPES)
def test_outputs_do_not_depend_on_whether_states_are_saved(io, shape):
    x, _ = _make(*shape, io, seed=41)
    r = Run(x, io, 0.25)
    kept = {n: t.clone() for n, t in r.fwd(1).items()}
    for n, t in r.fwd(0).items():
        assert torch.equal(t, kept[n]), n
    o, S = O.forward(**x, scale=0.25)
    check(kept, {"o": o, "S": S})  # to the tolerance of fp32 sums, whatever is kept
