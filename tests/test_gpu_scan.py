"""Gated linear recurrence against its oracle in 64 bits: forward, reverse pass (from states, from 8-bit inputs, from nothing), recurrent step.

Tolerances, per value: half a step of the output's type relative to the value, plus a share of the sum of the magnitudes of the terms that the value is made of (the oracle
gives it).  That share, in fp32 arithmetic:
  gates    a term is a product of i, s and decays.  With bf16 I/O a sigmoid is off by 2^-22 (exponential) + 2^-23 (reciprocal) + the rounding of the exponential's
           argument, |x| 2^-24: some 2^-21 for |x| up to 5; s by half of that and its root; a decay over a log decay of S by S times that, and terms with S above 4 are under
           2 % of the sum: 2^-21 (1 + 1/2 + 4) + 2^-22 < 3e-6.  With fp32 I/O a dozen roundings of 2^-24 in their place.  GATE = 4e-6 and 2e-6.
  walk     a tile of at least 64 tokens adds at most 16 roundings of the full sum: (L / 4 + 32) 2^-24.
A gradient is a product of two such sums and two more gates: twice the share and GATE.  d_rate adds up over tokens: a thread adds up L / 8 of a sequence, warps, parts and
sequences follow: (L / 8 + 64 + 16 B) 2^-24 more.
"""
import numpy as np
import pytest
import torch

from oracle import pack8 as K
from oracle import scan as O
from paper_2608_21308_b200 import binding as E
from paper_2608_21308_b200 import inputs

pytestmark = pytest.mark.gpu
GATE = {"bf16": 4e-6, "f32": 2e-6}
SAVE = {"none": E.E2TTT_SAVE_NONE, "states": E.E2TTT_SAVE_STATES, "packed": E.E2TTT_SAVE_PACKED}


def make(B, L, D, io, gate=True, unit=True, docs=False, seed=0, rate=None):
    rng = np.random.default_rng(seed)
    rnd = inputs.round_bf16 if io == "bf16" else (lambda a: a.astype(np.float32))
    f = lambda *s: rng.standard_normal(s).astype(np.float32)  # noqa: E731
    lo, hi = rate or (0.9, 0.999)
    x = {"x": rnd(f(B, L, D)), "r": rnd(f(B, L, D)), "g": rnd(f(B, L, D)) if gate else None, "rate": -np.log(rng.uniform(lo, hi, D)).astype(np.float32),
         "starts": (rng.random((B, L)) < 0.02).astype(np.uint8) if docs else None, "h0": f(B, D), "unit": unit}
    return x, {"d_h": rnd(f(B, L, D)), "dh_final": f(B, D)}


def dev(a, io=None):
    if a is None:
        return None
    t = torch.tensor(a, device="cuda")
    return t if a.dtype == np.uint8 else t.to(torch.bfloat16 if io == "bf16" else torch.float32).contiguous()


class Run:
    def __init__(self, x, io, save="states"):
        B, L, D = x["x"].shape
        self.p = E.make_scan_params(B, L, D, E.E2TTT_F32 if io == "f32" else E.E2TTT_BF16, E.E2TTT_GATE_NONE if x["g"] is None else E.E2TTT_GATE_SIGMOID, int(x["unit"]))
        self.io, self.save = io, SAVE[save]
        self.x, self.r, self.g = (dev(x[n], io) for n in ("x", "r", "g"))
        self.rate, self.starts, self.h0 = dev(x["rate"]), dev(x["starts"]), dev(x["h0"])
        n = E.e2ttt_scan_workspace_bytes(self.p, self.save or E.E2TTT_SAVE_STATES)
        self.ws = torch.full((n,), 0xff, dtype=torch.uint8, device="cuda")

    def fwd(self):
        h, last = torch.full_like(self.x, 7.0), torch.full((self.p.B, self.p.D), 7.0, device="cuda")
        E.e2ttt_scan_fwd(self.p, self.x, self.r, self.g, self.rate, self.starts, self.h0, h, last, self.ws if self.save else None, self.save)
        return {"h": h, "h_final": last}

    def bwd(self, d):
        out = {"d_x": torch.full_like(self.x, 7.0), "da_decay": torch.full_like(self.x, 7.0), "da_in": None if self.g is None else torch.full_like(self.x, 7.0),
               "d_rate": torch.full_like(self.rate, 7.0), "dh_init": torch.full((self.p.B, self.p.D), 7.0, device="cuda")}
        x, r, g = (None, None, None) if self.save == E.E2TTT_SAVE_PACKED else (self.x, self.r, self.g)
        E.e2ttt_scan_bwd(self.p, x, r, g, self.rate, self.starts, self.h0, dev(d["d_h"], self.io), dev(d["dh_final"]), *out.values(), self.ws, self.save)
        return {n: t for n, t in out.items() if t is not None}

    def step(self):
        h, last = torch.full_like(self.x, 7.0), torch.full((self.p.B, self.p.D), 7.0, device="cuda")
        E.e2ttt_scan_step(self.p, self.x, self.r, self.g, self.rate, self.starts, self.h0, h, last)
        return {"h": h, "h_final": last}


def share(io, L, extra=0.0):
    return GATE[io] + (L / 4 + 32) * 2.0 ** -24 + extra


def near(n, t, ref, mag, tol):
    y = t.double().cpu().numpy()
    assert np.isfinite(y).all(), n
    half = torch.finfo(t.dtype).eps / 2
    # below 2^-126 a factor may be flushed to zero; those that meet it are at most 64
    over = np.abs(y - ref) - half * np.abs(ref) * (1 + half) - tol * mag - 2.0 ** -120
    assert over.max() <= 0, (n, over.max(), np.abs(ref).max(), np.linalg.norm(y - ref) / np.linalg.norm(ref))


def check_forward(got, x, io, extra=0.0):
    h, last, mag = O.forward(**x)
    tol = share(io, h.shape[1], extra)
    near("h", got["h"], h, mag, tol)
    near("h_final", got["h_final"], last, mag[:, -1], tol)


def check_backward(got, x, d, io, packed, extra=0.0):
    kept = tuple(None if x[n] is None else K.through(x[n]) for n in ("x", "r", "g")) if packed else None
    ref, mag = O.backward(**x, **d, kept=kept)
    B, L = x["x"].shape[:2]
    tol = 2 * share(io, L, extra) + GATE[io]
    assert set(got) == set(ref)
    for n, t in got.items():
        near(n, t, ref[n], mag[n], tol + (L / 8 + 64 + 16 * B) * 2.0 ** -24 if n == "d_rate" else tol)


SHAPES = [  # B, L, D
    (1, 1, 1), (3, 1, 130), (1, 2, 64), (2, 63, 7), (1, 64, 66), (2, 65, 65), (1, 127, 2), (1, 128, 601), (3, 129, 64), (1, 777, 200), (2, 1000, 72), (1, 2500, 33),
    (5, 300, 8), (1, 520, 128),
]


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("gate,unit,docs", [(True, True, False), (True, True, True), (False, True, True), (True, False, False), (False, False, True)])
@pytest.mark.parametrize("save", ["states", "packed"])
@pytest.mark.parametrize("shape", SHAPES)
def test_forward_and_backward(io, gate, unit, docs, save, shape):
    x, d = make(*shape, io, gate, unit, docs)
    r = Run(x, io, save)
    out = r.fwd()
    check_forward(out, x, io)
    grads = r.bwd(d)
    check_backward(grads, x, d, io, save == "packed")
    for n, t in {**r.fwd(), **r.bwd(d)}.items():
        assert torch.equal(t, {**out, **grads}[n]), n  # repeats bit for bit


@pytest.mark.parametrize("io", ["f32", "bf16"])
def test_wide_and_many_sequences(io):
    for shape in ((2, 300, 2048), (40, 70, 130)):
        x, d = make(*shape, io, docs=True)
        for save in ("states", "packed"):
            r = Run(x, io, save)
            check_forward(r.fwd(), x, io)
            check_backward(r.bwd(d), x, d, io, save == "packed")


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("rate", [(1e-4, 0.05), (0.5, 0.9), (0.99999, 0.9999999)])
def test_fast_and_slow_channels(io, rate):
    """Decays far from 1 (the exponential in place of the series), around the line between them, and so near to 1 that 1 - a is under the rounding of a."""
    x, d = make(2, 400, 70, io, rate=rate, seed=1)
    r = Run(x, io)
    check_forward(r.fwd(), x, io)
    check_backward(r.bwd(d), x, d, io, False)


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("save", ["states", "packed"])
def test_no_start_state_no_end_gradient_and_states_computed_again(io, save):
    x, d = make(2, 150, 70, io, docs=True, seed=2)
    x["h0"], d["dh_final"] = None, None
    r = Run(x, io, save)
    r.p.B = 2
    check_forward(r.fwd(), x, io)
    grads = r.bwd(d)
    check_backward(grads, x, d, io, save == "packed")
    if save == "states":
        again = Run(x, io, "none")
        for n, t in again.bwd(d).items():
            assert torch.equal(t, grads[n]), n


@pytest.mark.parametrize("io", ["f32", "bf16"])
def test_saving_changes_no_output(io):
    x, _ = make(2, 333, 130, io, docs=True, seed=3)
    base = Run(x, io, "none").fwd()
    for save in ("states", "packed"):
        for n, t in Run(x, io, save).fwd().items():
            assert torch.equal(t, base[n]), (save, n)


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("D", [64, 72, 66, 65])
def test_tensors_at_any_element(io, D):
    x, d = make(2, 140, D, io, docs=True, seed=4)
    shift = lambda t: None if t is None else torch.cat([t.new_zeros(1), t.flatten()])[1:].view(t.shape)  # noqa: E731
    for save in ("states", "packed"):
        r = Run(x, io, save)
        for n in ("x", "r", "g", "rate", "starts", "h0"):
            setattr(r, n, shift(getattr(r, n)))
        check_forward(r.fwd(), x, io)
        out = [shift(torch.zeros(s, device="cuda", dtype=t)) for s, t in [(r.x.shape, r.x.dtype)] * 3 + [((D,), torch.float32), ((2, D), torch.float32)]]
        E.e2ttt_scan_bwd(r.p, r.x, r.r, r.g, r.rate, r.starts, r.h0, shift(dev(d["d_h"], io)), shift(dev(d["dh_final"])), *out, r.ws, r.save)
        check_backward(dict(zip(("d_x", "da_decay", "da_in", "d_rate", "dh_init"), out)), x, d, io, save == "packed")


@pytest.mark.parametrize("io", ["f32", "bf16"])
def test_state_in_place(io):
    x, d = make(3, 200, 96, io, seed=5)
    r = Run(x, io)
    out, grads = r.fwd(), r.bwd(d)
    state, h = r.h0.clone(), torch.empty_like(r.x)
    E.e2ttt_scan_fwd(r.p, r.x, r.r, r.g, r.rate, r.starts, state, h, state, r.ws, r.save)
    assert torch.equal(state, out["h_final"]) and torch.equal(h, out["h"])
    end, rest = dev(d["dh_final"]), [torch.empty_like(grads[n]) for n in ("d_x", "da_decay", "da_in", "d_rate")]
    E.e2ttt_scan_bwd(r.p, r.x, r.r, r.g, r.rate, r.starts, r.h0, dev(d["d_h"], io), end, *rest, end, r.ws, r.save)
    for n, t in zip(("d_x", "da_decay", "da_in", "d_rate", "dh_init"), (*rest, end)):
        assert torch.equal(t, grads[n]), n


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("gate,unit,docs", [(True, True, True), (False, True, False), (True, False, True)])
@pytest.mark.parametrize("shape", [(1, 1, 1), (1, 1, 2048), (64, 1, 768), (3, 4, 65), (2, 9, 130), (200, 2, 2)])
def test_step(io, gate, unit, docs, shape):
    x, _ = make(*shape, io, gate, unit, docs, seed=6)
    r = Run(x, io)
    got = r.step()
    check_forward(got, x, io)
    state = r.h0.clone()
    E.e2ttt_scan_step(r.p, r.x, r.r, r.g, r.rate, r.starts, state, torch.empty_like(r.x), state)
    assert torch.equal(state, got["h_final"])


@pytest.mark.parametrize("io", ["f32", "bf16"])
def test_a_prompt_and_then_tokens_on_its_state(io):
    B, L, D, cut = 2, 210, 70, 203
    x, _ = make(B, L, D, io, docs=True, seed=7)
    part = lambda lo, hi, h0: {n: (t[:, lo:hi] if n in ("x", "r", "g", "starts") else t) for n, t in x.items()} | {"h0": h0}  # noqa: E731
    one = Run(part(0, cut, x["h0"]), io)
    got = one.fwd()
    h, state = [got["h"]], got["h_final"]
    for t in range(cut, L):
        r = Run(part(t, t + 1, x["h0"]), io)
        r.h0 = state
        o = r.step()
        h.append(o["h"])
        state = o["h_final"]
    check_forward({"h": torch.cat(h, 1), "h_final": state}, x, io)


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("save", ["states", "packed"])
def test_gates_wide_open_and_shut(io, save):
    """Logits far out: the derivative of an open gate is what is left of 1; a shut decay gate keeps the state and lets nothing in (unit scale)."""
    x, d = make(1, 140, 64, io, seed=8)
    x["r"][:, :, :8], x["r"][:, :, 8:16] = 30.0, -30.0
    x["g"][:, :, 16:24], x["g"][:, :, 24:32] = 30.0, -30.0
    x["r"][:, 70, 32:], x["g"][:, 71, 32:] = 40.0, -40.0
    x["r"][:, :, 40] = 0.0
    x["rate"][48:56] = 60.0
    r = Run(x, io, save)
    # bf16: the rounding of the exponential's argument, |x| 2^-24, in a sigmoid, s and a decay.  Both: token 71 lets nothing in, so that all there is of h is what one decay leaves,
    # and where the rate is 60 its logarithm S is up to 60: off by S times the error of log a, of four roundings (exponential, sum, reciprocal, product) of 2^-24, or 2^-21 in bf16
    extra = 40 * 2.0 ** -22 + 60 * 2.0 ** -21 if io == "bf16" else 60 * 2.0 ** -22
    check_forward(r.fwd(), x, io, extra)
    check_backward(r.bwd(d), x, d, io, save == "packed", extra)


@pytest.mark.parametrize("io", ["f32", "bf16"])
def test_logits_without_bound_and_a_rate_of_zero(io):
    """Nothing is NaN at infinite logits or where a_t is 1: there the derivative of s_t is taken as 0.  Logits count from -43 on."""
    x, d = make(1, 100, 64, io, seed=9)
    x["r"][:, 5:9, :4], x["r"][:, 20, 4:8], x["g"][:, 30, :4], x["g"][:, 31, :4] = -np.inf, np.inf, -np.inf, np.inf
    x["r"][:, :, 60] = -np.inf
    x["rate"][63] = 0.0
    r = Run(x, io)
    out, got = r.fwd(), r.bwd(d)
    x["r"], x["g"] = (np.maximum(x[n], -43.0) for n in ("r", "g"))
    check_forward(out, x, io)
    check_backward(got, x, d, io, False)


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("save", ["states", "packed"])
@pytest.mark.parametrize("where,bad", [("x", np.nan), ("x", np.inf), ("r", np.nan), ("g", np.nan)])
@pytest.mark.parametrize("D", [70, 72])
def test_what_a_nan_reaches(io, save, where, bad, D):
    """A channel's NaN stays in it, between two starts; in 8 bits its block of 32 channels is NaN at that token."""
    B, L = 2, 300
    x, d = make(B, L, D, io, seed=10)
    x["starts"] = np.zeros((B, L), np.uint8)
    x["starts"][0, [100, 229]] = 1
    clean = Run(x, io, save)
    h, grads = clean.fwd(), clean.bwd(d)
    x[where][0, 150, 40] = bad
    r = Run(x, io, save)
    got, back = r.fwd(), r.bwd(d)
    keep = torch.ones(B, L, D, dtype=torch.bool, device="cuda")
    keep[0, 150:229, 40] = False
    assert torch.equal(got["h"][keep], h["h"][keep]) and torch.equal(got["h_final"], h["h_final"])
    assert not torch.isfinite(got["h"][0, 150, 40])
    wide = slice(32, 64) if save == "packed" else slice(40, 41)
    keep[0, 100:229, wide] = False
    for n in ("d_x", "da_decay", "da_in"):
        assert torch.equal(back[n][keep], grads[n][keep]), n
    assert torch.equal(back["dh_init"], grads["dh_init"])
    cols = torch.ones(D, dtype=torch.bool, device="cuda")
    cols[wide] = False
    assert torch.equal(back["d_rate"][cols], grads["d_rate"][cols])


def test_a_sequence_does_not_depend_on_what_is_in_the_others():
    x, d = make(3, 500, 130, "bf16", docs=True, seed=11)
    y, e = make(3, 500, 130, "bf16", docs=True, seed=12)
    for n in ("x", "r", "g", "starts", "h0"):
        y[n][1] = x[n][1]
    for n in d:
        e[n][1] = d[n][1]
    y["rate"] = x["rate"]
    for save in ("states", "packed"):
        a, b = Run(x, "bf16", save), Run(y, "bf16", save)
        a, b = {**a.fwd(), **a.bwd(d)}, {**b.fwd(), **b.bwd(e)}
        for n in a:
            if n != "d_rate":
                assert torch.equal(a[n][1], b[n][1]), n


def test_more_than_two_to_the_31_elements():
    """The last tokens lie 2^31 elements into every tensor; behind a start they have to come out as they do alone, forward and back.  Going back, the long call has its
    tiles in several parts, whose sums are rounded elsewhere: a value may be rounded to the next step of bf16, 2^-7 of it."""
    L, D, n = (1 << 20) + 64, 2048, 64
    g = torch.Generator(device="cuda").manual_seed(0)
    x, r = (torch.zeros(1, L, D, device="cuda", dtype=torch.bfloat16) for _ in range(2))
    for t in (x, r):
        t[:, -n:].copy_(torch.randn(1, n, D, device="cuda", generator=g))
    rate = 0.01 + 0.09 * torch.rand(D, device="cuda", generator=g)
    starts = torch.zeros(1, L, dtype=torch.uint8, device="cuda")
    starts[:, -n] = 1
    h, last = torch.empty_like(x), torch.empty(1, D, device="cuda")
    p = E.make_scan_params(1, L, D, E.E2TTT_BF16, E.E2TTT_GATE_NONE)
    ws = torch.empty(E.e2ttt_scan_workspace_bytes(p, 2), dtype=torch.uint8, device="cuda")
    E.e2ttt_scan_fwd(p, x, r, None, rate, starts, None, h, last, ws, 2)
    end = torch.randn(1, D, device="cuda", generator=g)
    out = [torch.empty_like(rate), torch.empty_like(last)]
    x1, r1, h1 = (t[:, -n:].clone() for t in (x, r, h))
    dr = torch.empty_like(x)
    E.e2ttt_scan_bwd(p, None, None, None, rate, starts, None, h, end, r, dr, None, *out, ws, 2)  # d_h = h, and d_x where r was
    p1 = E.make_scan_params(1, n, D, E.E2TTT_BF16, E.E2TTT_GATE_NONE)
    ws1 = torch.empty(E.e2ttt_scan_workspace_bytes(p1, 2), dtype=torch.uint8, device="cuda")
    h2, last1, out1 = torch.empty_like(h1), torch.empty_like(last), [torch.empty_like(t) for t in out]
    E.e2ttt_scan_fwd(p1, x1, r1, None, rate, starts[:, -n:].contiguous(), None, h2, last1, ws1, 2)
    assert torch.equal(h2, h1) and torch.equal(last1, last)
    dx1, dr1 = torch.empty_like(x1), torch.empty_like(x1)
    E.e2ttt_scan_bwd(p1, None, None, None, rate, starts[:, -n:].contiguous(), None, h1, end, dx1, dr1, None, *out1, ws1, 2)
    for got, alone in ((r[:, -n:], dx1), (dr[:, -n:], dr1)):
        got, alone = got.float(), alone.float()
        assert bool(((got - alone).abs() <= 2.0 ** -7 * alone.abs() + 1e-5 * alone.abs().max()).all())
    assert not bool(r[:, :-n].any()) and not bool(h[:, :-n].any())  # nothing came before


@pytest.mark.parametrize("io", ["f32", "bf16"])
def test_unaligned_outputs_only(io):
    """Inputs that the copy engine could read, gradients and states that it could not write."""
    x, d = make(1, 140, 64, io, docs=True, seed=15)
    shift = lambda s, t: torch.zeros(int(np.prod(s)) + 1, device="cuda", dtype=t)[1:].view(s)  # noqa: E731
    for save in ("states", "packed"):
        r = Run(x, io, save)
        h, last = shift(r.x.shape, r.x.dtype), shift(r.h0.shape, torch.float32)
        E.e2ttt_scan_fwd(r.p, r.x, r.r, r.g, r.rate, r.starts, r.h0, h, last, r.ws, r.save)
        check_forward({"h": h, "h_final": last}, x, io)
        out = [shift(r.x.shape, r.x.dtype) for _ in range(3)] + [torch.empty_like(r.rate), torch.empty_like(r.h0)]
        E.e2ttt_scan_bwd(r.p, r.x, r.r, r.g, r.rate, r.starts, r.h0, dev(d["d_h"], io), dev(d["dh_final"]), *out, r.ws, r.save)
        check_backward(dict(zip(("d_x", "da_decay", "da_in", "d_rate", "dh_init"), out)), x, d, io, save == "packed")


@pytest.mark.parametrize("B,L,D", [(1, 20000, 128), (9, 1500, 1024), (150, 129, 64), (300, 200, 64)])
def test_every_way_of_sharing_a_sequence(B, L, D):
    """Few channels and many tokens (clusters of eight), several rounds of smaller clusters, one CTA a sequence; the second half of a long sequence, from the state of the first,
    is what it is in one piece."""
    x, _ = make(B, L, D, "bf16", docs=False, seed=16)
    r = Run(x, "bf16", "none")
    whole = r.fwd()
    cut = L // 2
    part = lambda lo, hi, h0: {**{n: t[:, lo:hi] if n in ("x", "r", "g") else t for n, t in x.items()}, "h0": h0}  # noqa: E731
    one = Run(part(0, cut, x["h0"]), "bf16", "none").fwd()
    two = Run(part(cut, L, one["h_final"].cpu().numpy()), "bf16", "none").fwd()
    h = torch.cat([one["h"], two["h"]], 1).float()
    big = float(whole["h_final"].abs().max())
    # states in fp32 agree to both calls' shares; h is rounded to bf16 in both: one step of it, 2^-7, apart at most
    tol = 2 * share("bf16", L) * 40
    assert bool(((two["h_final"] - whole["h_final"]).abs() <= tol * big).all())
    assert bool(((h - whole["h"].float()).abs() <= 2.0 ** -7 * h.abs() + tol * big).all())


def test_graphs_of_two_streams_and_replays():
    x, d = make(2, 200, 128, "bf16", docs=True, seed=13)
    y, _ = make(2, 200, 128, "bf16", docs=True, seed=14)
    runs = [Run(x, "bf16", s) for s in ("states", "packed")]
    for r in runs:
        r.fwd(), r.bwd(d)
    dh, end = dev(d["d_h"], "bf16"), dev(d["dh_final"])
    graphs = []
    for r in runs:
        out = [torch.empty_like(t) for t in (r.x, r.h0, r.x, r.x, r.x, r.rate, r.h0)]
        stream, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
        stream.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(stream), torch.cuda.graph(graph, stream=stream):
            E.e2ttt_scan_fwd(r.p, r.x, r.r, r.g, r.rate, r.starts, r.h0, out[0], out[1], r.ws, r.save)
            E.e2ttt_scan_bwd(r.p, r.x, r.r, r.g, r.rate, r.starts, r.h0, dh, end, *out[2:], r.ws, r.save)
        graphs.append((graph, out, stream))
    for r in runs:
        for n in ("x", "r", "g", "starts", "h0"):
            getattr(r, n).copy_(dev(y[n], "bf16" if n in ("x", "r", "g") else None))
    torch.cuda.synchronize()
    for graph, _, stream in graphs:  # both at the same time, each on its own workspace
        with torch.cuda.stream(stream):
            graph.replay()
    torch.cuda.synchronize()
    y["rate"] = x["rate"]
    for (_, out, _), save in zip(graphs, ("states", "packed")):
        check_forward({"h": out[0], "h_final": out[1]}, y, "bf16")
        check_backward(dict(zip(("d_x", "da_decay", "da_in", "d_rate", "dh_init"), out[2:])), y, d, "bf16", save == "packed")
