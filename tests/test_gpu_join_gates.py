"""Block join: the gate's derivative over the whole range of its input, value by value.

Without a second norm the adjoint of x_out is d_x_out as given, and d_a = d_x_out res_scale w_post y0 sig (1 - sig) is a product: some ten roundings of 2^-24, a
reciprocal root, an exponential and a reciprocal of 2^-22 at most: 2e-6 of the value.  With bf16 the exponential's argument is rounded too: up to 2^-24 of
|a| log2(e) <= 116, 5e-6 of the value; and the output by half a step.
"""
import numpy as np
import pytest
import torch

from oracle import join as O
from paper_2608_21308_b200 import binding as E
from tests.test_gpu_join import EPS, Run, _make

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("kind", ["sigmoid", "silu"])
@pytest.mark.parametrize("shape", [(1, 4, 40, 64), (1, 1, 20, 4500)])  # weights and gates kept in registers, and not
def test_gate_gradient_where_the_gate_is_open_or_shut(io, kind, shape):
    x, d = _make(*shape, io, kind, False, seed=6)
    x["a"][:] = np.resize(np.concatenate([np.linspace(2, 80, 157), -np.linspace(2, 80, 157)]), x["a"].shape).astype(np.float32)
    if io == "bf16":
        x["a"] = torch.tensor(x["a"]).bfloat16().float().numpy()
    # the sigmoid's derivative is even, and sig (1 - sig) exact in 64 bits where sig is the smaller part
    ref = O.backward(**dict(x, a=-np.abs(x["a"]) if kind == "sigmoid" else x["a"]), kind=kind, **EPS, **d)["d_a"]
    t = Run(x, io, kind).bwd(d)["d_a"]
    got, half = t.double().cpu().numpy(), torch.finfo(t.dtype).eps / 2
    # Below the smallest normal value, 2^-126 (a factor of 1e-3 is enough at a = 80: exp(-80) = 2^-115), the type's steps are of one size, eps 2^-126, and
    # half of one is what a value may be off by.
    least = half * torch.finfo(t.dtype).smallest_normal
    over = np.abs(got - ref) - (half + (2e-6 if io == "f32" else 1e-5)) * np.abs(ref) - least
    assert over.max() <= 0, (over / np.abs(ref)).max()
