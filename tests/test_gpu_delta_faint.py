"""Gated delta rule: a slice, a chunk or a document that is small beside others keeps its gradients."""
import numpy as np
import pytest

from oracle import delta as O
from tests.test_gpu_delta import Run, _make, check

pytestmark = pytest.mark.gpu

SHAPES = [(1, 2, 2, 128, 64, 64), (4, 20, 20, 128, 64, 32)]  # the columns of a slice over two warps; one warp per slice


def _norm(got, ref):
    got = got.double().cpu().numpy()
    assert np.isfinite(got).all()
    return np.linalg.norm(got - ref) / np.linalg.norm(ref)


# The smaller part is 2^-26 of the larger one, whose scale it shares: largest value in [2^12, 2^14), fp16's smallest step 2^-24.  Where the scale comes from the
# larger part's largest value itself, the smaller part's root mean square, a quarter of its largest, is 2^-15 or more and a step's error 2^-24 / sqrt(12): 2^-10.8
# of it.  e's scale comes from a bound: its largest value, 4, against (4 + 2-norm of 16 rows of a state, 10) times row sums of T up to 3: some 2^3.4 above, 2^-7.4.
# With one term that is what dq and dk of such tokens are made of, beside other operands' 2^-10.8 and less: below 2^-7.
SMALL, NEAR = np.float32(2.0 ** -26), 2.0 ** -7


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("shape", [(1, 2, 2, 128, 64, 64), (1, 2, 1, 64, 128, 128), (4, 20, 20, 64, 64, 32)])
def test_small_value_rows_beside_large_ones(io, shape):
    x, d = _make(*shape, io, seed=32)
    x["v"][..., 16:] *= SMALL
    x["S"][:, :, 16:] *= SMALL
    d["d_o"][..., :16] = 0
    d["dS_final"][:, :, :16] = 0
    r = Run(x, io, 1.0)
    r.fwd(1)
    got, ref = r.bwd(d), O.backward(**x, scale=1.0, **d)
    for n in ("dq", "dk"):
        assert _norm(got[n], ref[n]) <= NEAR, n


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("at", [32, 20, 40])
def test_a_faint_document_behind_another_in_one_block(io, at):
    x, d = _make(1, 2, 2, 64, 64, 64, io, seed=33)
    x["log_gamma"][:, :, at] = -np.inf
    x["v"][:, :, at:] *= SMALL
    r = Run(x, io, 1.0)
    r.fwd(1)
    got, ref = r.bwd(d), O.backward(**x, scale=1.0, **d)
    for n in ("dq", "dk"):
        assert _norm(got[n][:, :, at:], ref[n][:, :, at:]) <= NEAR, n


@pytest.mark.parametrize("io", ["f32", "bf16"])
def test_faint_keys_and_queries_of_one_chunk(io):
    """With keys of 2^-26 of their neighbours' the second chunk's queries see their own chunk only through them."""
    x, d = _make(1, 2, 2, 64, 64, 64, io, seed=34)
    x["log_gamma"][:, :, 32] = -np.inf
    x["k"][:, :, 32:] *= SMALL
    r = Run(x, io, 1.0)
    r.fwd(1)
    got, ref = r.bwd(d), O.backward(**x, scale=1.0, **d)
    for n in ("dq", "dk"):
        assert _norm(got[n][:, :, 32:], ref[n][:, :, 32:]) <= NEAR, n


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("ratio", [18, 20, 22])
def test_faint_output_gradients_under_a_large_adjoint(io, shape, ratio):
    """The adjoint of one column of the state is 2^ratio, what the outputs' gradients put into the others is of the order of 1.  The walk adds both at one
    scale, from a bound that may be 2^10 above what it bounds, and there are steps down to 2^-37 of it: 2^-27, or 2^-5 of a unit with 2^22, at worst.
    One key in all tokens and 2-norms leave the bound some 2^5 above: 2^-10 of a unit."""
    x, d = _make(*shape, io, seed=35)
    x["log_gamma"][:] = 0
    x["S"][:] = 0
    x["k"][:], x["k"][..., 0] = 0, 1
    x["q"][..., 0] = 0
    d["dS_final"][:] = 0
    d["dS_final"][..., 0] = 2.0 ** ratio
    r = Run(x, io, 1.0)
    r.fwd(1)
    got, ref = r.bwd(d), O.backward(**x, scale=1.0, **d)
    assert _norm(got["dS"][..., 1:], ref["dS"][..., 1:]) <= 2.0 ** -8


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("shape", SHAPES)
def test_large_adjoints_of_tokens_that_see_nothing_beside_small_ones_under_a_large_state(io, shape):
    """One block: the first chunk has values of 2^50 in its state and adjoints of its errors of the order of 1, the second chunk the other way round."""
    x, d = _make(*shape, io, seed=36)
    big = np.float32(2.0 ** 50)
    x["S"] *= big
    d["dS_final"] *= big
    x["log_gamma"][:] = 0
    for t in (x["k"], x["q"], x["v"], d["d_o"]):
        t[:, :, 32:64] = 0
    x["log_gamma"][:, :, 32] = -95
    x["k"][:, :, 33, 1] = 1
    o, S = O.forward(**x, scale=1.0)
    r = Run(x, io, 1.0)
    check(r.fwd(1), {"o": o, "S": S})
    check(r.bwd(d), O.backward(**x, scale=1.0, **d), dict(x, scale=1.0, **d))
