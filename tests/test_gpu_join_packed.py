"""The block join with its inputs kept in 8 bits: the forward is the join's bit for bit, the reverse pass the adjoint at the values that are read back.

Tolerances are those of the block join's own test: half a step of the output's type, and 1e-5 of the largest magnitude (of the terms, for d_o) for the fp32 arithmetic.
"""
import numpy as np
import pytest
import torch

from oracle import join as O
from oracle import pack8 as K
from paper_2608_21308_b200 import binding as E
from tests import test_gpu_join as J

pytestmark = pytest.mark.gpu


class Run(J.Run):
    def __init__(self, x, io, kind):
        super().__init__(x, io, kind)
        self.packed = torch.full((E.e2ttt_join_packed_bytes(self.p),), 0xff, dtype=torch.uint8, device="cuda")

    def fwd(self):
        xo = torch.full_like(self.io[2], 7.0)
        n = None if self.w[2] is None else torch.full_like(xo, 7.0)
        E.e2ttt_join_fwd_packed(self.p, *self.io, *self.w, xo, n, self.packed)
        return {"x_out": xo, **({} if n is None else {"n": n})}

    def bwd(self, d):
        ws = torch.empty(E.e2ttt_join_workspace_bytes(self.p), dtype=torch.uint8, device="cuda").fill_(0xff)
        like = lambda t: None if t is None else torch.full_like(t, 7.0)  # noqa: E731
        out = {"d_" + n: like(t) for n, t in zip(("o", "a", "x", "w_post", "res_scale", "w_pre"), self.io + self.w)}
        E.e2ttt_join_bwd_packed(self.p, self.packed, *self.w, J._dev(d["d_x_out"], self.kind), J._dev(d["d_n"], self.kind), *out.values(), ws)
        return {n: t for n, t in out.items() if t is not None}


def kept(x):
    """The inputs as they are read back: o in blocks of 32 columns of a token's row, across heads."""
    B, H, L, d = x["o"].shape
    o = K.through(np.moveaxis(x["o"], 1, 2).reshape(B, L, H * d)).reshape(B, L, H, d)
    return {**x, "o": np.moveaxis(o, 2, 1), "x": K.through(x["x"]), "a": None if x["a"] is None else K.through(x["a"])}


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("kind,pre", [("silu", True), ("sigmoid", False), ("none", True)])
@pytest.mark.parametrize("shape", J.SHAPES)
def test_forward_and_backward(io, kind, pre, shape):
    x, d = J._make(*shape, io, kind, pre)
    r = Run(x, io, kind)
    plain, got = J.Run(x, io, kind).fwd(), r.fwd()
    for n, t in plain.items():
        assert torch.equal(t, got[n]), n
    back = r.bwd(d)
    J.check(back, O.backward(**kept(x), kind=kind, **J.EPS, **d, terms=True))
    for n, t in r.bwd(d).items():
        assert torch.equal(t, back[n]), n  # repeats bit for bit


@pytest.mark.parametrize("io", ["f32", "bf16"])
def test_unaligned_in_place_and_values_already_in_eight_bits(io):
    x, d = J._make(2, 5, 50, 24, io, "silu", True, seed=1)
    x = {n: (kept(x)[n].astype(np.float32) if n in ("o", "a", "x") else t) for n, t in x.items()}  # they pack to themselves: the join's own gradients
    r, base = Run(x, io, "silu"), J.Run(x, io, "silu")
    out = base.fwd()
    want = base.bwd(d)
    shift = lambda t: None if t is None else torch.cat([t.new_zeros(1), t.flatten()])[1:].view(t.shape)  # noqa: E731
    r.fwd()
    for n, t in r.bwd(d).items():
        assert torch.equal(t, want[n]), n
    r.packed.fill_(0xff)
    E.e2ttt_join_fwd_packed(r.p, *r.io, *r.w, r.io[2], r.io[1], r.packed)  # x_out over x, n over a
    assert torch.equal(r.io[2], out["x_out"]) and torch.equal(r.io[1], out["n"])
    for n, t in r.bwd(d).items():
        assert torch.equal(t, want[n]), n
    r = Run(x, io, "silu")
    r.io, r.w = [shift(t) for t in r.io], [shift(t) for t in r.w]
    r.fwd()
    J.check(r.bwd(d), O.backward(**x, kind="silu", **J.EPS, **d, terms=True))


def test_a_block_that_is_not_finite_reaches_its_token_only():
    x, d = J._make(2, 4, 20, 64, "bf16", "silu", True, seed=2)
    r = Run(x, "bf16", "silu")
    r.fwd()
    clean = r.bwd(d)
    x["x"][1, 7, 40] = np.inf
    r = Run(x, "bf16", "silu")
    r.fwd()
    got = r.bwd(d)
    for n in ("d_x", "d_a"):
        keep = torch.ones_like(got[n], dtype=torch.bool)
        keep[1, 7] = False
        assert torch.equal(got[n][keep], clean[n][keep]), n
        assert not bool(torch.isfinite(got[n][1, 7, 32:64]).any())
    keep = torch.ones_like(got["d_o"], dtype=torch.bool)
    keep[1, :, 7] = False
    assert torch.equal(got["d_o"][keep], clean["d_o"][keep])
