"""Gated delta rule against its oracle in 64 bits: whole sequences, reverse pass, recurrent form.

Tolerances, per value: half a step of the output's type relative to the value (bf16 2^-8, fp32 2^-24) plus TOL of the tensor's largest
magnitude.  TOL: an operand of 32 bits is two fp16 terms (2^-22), a product of the chain has two such operands and sums at most
3 x 8 + 3 x 2 partial results that are truncated (2^-23 each, partial sums at most about the sum of the magnitudes); four dependent products
per chunk: 4 (2 x 2^-22 + 30 x 2^-23) = 1.6e-5 of the sum of the magnitudes if all errors had one sign.  They do not, and no sum here exceeds its
largest magnitude's row by more than sqrt(128): 2e-5 of the largest magnitude holds for the worst value.
bf16 outputs of a forward without saved states come from products with one fp16 term (half a step: 2^-11) of the start state, of u and of A: an output
is off by at most 2^-11 of the magnitudes of what the state puts into it and 2 x 2^-11 of what the chunk's tokens do: 2^-10 of the sum of magnitudes.
The gradients of bf16 queries and keys come from products with one term as well: dq's of the state, or of e and then of their product's matrix (2 x 2^-11);
dk's of dP, of e or the state or its adjoint, and of their products' matrices (3 x 2^-11 at most), of the sum of magnitudes.
"""
import numpy as np
import pytest
import torch

from oracle import delta as O
from paper_2608_21308_b200 import binding as E
from paper_2608_21308_b200 import inputs

pytestmark = pytest.mark.gpu
TOL = 2e-5


def _make(B, H, Hk, L, dk, dv, io, seed=0, gates="model", start=True):
    rng = np.random.default_rng(seed)
    rnd = inputs.round_bf16 if io == "bf16" else (lambda a: a.astype(np.float32))

    def unit(*shape):
        x = rng.standard_normal(shape)
        return rnd((x / np.linalg.norm(x, axis=-1, keepdims=True)).astype(np.float32))

    x = {"q": unit(B, Hk, L, dk), "k": unit(B, Hk, L, dk), "v": rnd(rng.standard_normal((B, H, L, dv)).astype(np.float32)),
         "eta": (1 / (1 + np.exp(-rng.standard_normal((B, H, L))))).astype(np.float32),
         "log_gamma": (-rng.uniform(0, 0.3, (B, H, L))).astype(np.float32),
         "S": (0.3 * rng.standard_normal((B, H, dv, dk))).astype(np.float32) if start else None}
    if gates == "edges":  # no decay, strong decay, a forgotten state, nothing written, everything written
        x["log_gamma"] = rng.choice(np.array([0, -0.01, -3, -40, -np.inf], np.float32), (B, H, L), p=[0.4, 0.3, 0.2, 0.05, 0.05])
        x["eta"] = rng.choice(np.array([0, 1e-9, 0.5, 1], np.float32), (B, H, L))
    d = {"d_o": rnd(rng.standard_normal((B, H, L, dv)).astype(np.float32)),
         "dS_final": (0.1 * rng.standard_normal((B, H, dv, dk))).astype(np.float32)}
    return x, d


def _dev(a, io=None):
    return None if a is None else torch.tensor(a, device="cuda").to(torch.bfloat16 if io == "bf16" else torch.float32).contiguous()


class Run:
    def __init__(self, x, io, scale):
        B, H, L, dv = x["v"].shape
        Hk, dk = x["q"].shape[1], x["q"].shape[-1]
        self.p = E.make_delta_params(B, H, Hk, L, dk, dv, E.E2TTT_F32 if io == "f32" else E.E2TTT_BF16, scale)
        self.q, self.k, self.v = (_dev(x[n], io) for n in "qkv")
        self.eta, self.lg, self.S = _dev(x["eta"]), _dev(x["log_gamma"]), _dev(x["S"])
        self.o = torch.full_like(self.v, 7.0)
        self.S_out = torch.full((B, H, dv, dk), 7.0, device="cuda")
        self.io = io

    def workspace(self, save):
        ws = torch.empty(E.e2ttt_delta_workspace_bytes(self.p, save), dtype=torch.uint8, device="cuda")
        return ws.fill_(0xff)  # NaNs in every word that the kernels should write first

    def fwd(self, save=0, ws=None):
        self.ws = self.workspace(save) if ws is None else ws
        E.e2ttt_delta_fwd(self.p, self.q, self.k, self.v, self.eta, self.lg, self.S, self.o, self.S_out, self.ws, save)
        assert E.e2ttt_device_status(self.ws) == 0
        return {"o": self.o, "S": self.S_out}

    def bwd(self, d, saved=1):
        if not saved:
            self.ws = self.workspace(1)
        out = {"dq": torch.full_like(self.q, 7.0), "dk": torch.full_like(self.k, 7.0), "dv": torch.full_like(self.v, 7.0),
               "d_eta": torch.full_like(self.eta, 7.0), "d_log_gamma": torch.full_like(self.eta, 7.0), "dS": torch.full_like(self.S_out, 7.0)}
        E.e2ttt_delta_bwd(self.p, self.q, self.k, self.v, self.eta, self.lg, self.S, _dev(d["d_o"], self.io), _dev(d["dS_final"]),
                          *out.values(), self.ws, saved)
        assert E.e2ttt_device_status(self.ws) == 0
        return out

    def step(self):
        E.e2ttt_delta_step(self.p, self.q, self.k, self.v, self.eta, self.lg, self.S, self.o, self.S_out)
        return {"o": self.o, "S": self.S_out}


def check(got, ref, single=None):
    """single: the inputs, where the outputs (with `d_o` among them: dq and dk) are of products with one term."""
    terms = {}
    if single is not None and next(iter(got.values())).dtype == torch.bfloat16:
        if "d_o" in single:
            m = O.gradient_magnitudes(**single)
            terms = {"dq": 2.0 ** -10 * m["dq"], "dk": 3 * 2.0 ** -11 * m["dk"]}
        else:
            terms = {"o": 2.0 ** -10 * O.magnitudes(**single)}
    for n, t in got.items():
        y, r = t.double().cpu().numpy(), ref[n]
        half = torch.finfo(t.dtype).eps / 2
        assert np.isfinite(y).all(), n
        over = np.abs(y - r) - half * np.abs(r) - TOL * np.abs(r).max() - terms.get(n, 0.0)
        assert over.max() <= 0, (n, over.max(), np.abs(r).max(), np.linalg.norm(y - r) / np.linalg.norm(r))


SHAPES = [  # B, H, Hk, L, dk, dv
    (1, 1, 1, 1, 64, 64), (1, 2, 1, 31, 128, 128), (2, 2, 2, 32, 64, 64), (1, 3, 3, 33, 128, 128), (1, 4, 2, 64, 72, 100), (1, 2, 2, 65, 128, 16),
    (2, 6, 2, 97, 72, 100), (1, 1, 1, 200, 128, 128), (1, 2, 1, 130, 1, 1), (1, 1, 1, 70, 17, 33), (3, 5, 5, 129, 65, 127), (9, 16, 4, 96, 64, 64),
    (1, 13, 13, 128, 128, 128),
    # more slices than SMs: a warp for all of a slice's columns, four slices (two with fp32) or fewer in a CTA, the last CTA not full
    (2, 16, 16, 70, 128, 128), (3, 16, 4, 100, 128, 100), (5, 8, 2, 96, 96, 80),
    # narrow keys and wide values
    (2, 4, 2, 130, 48, 120), (6, 8, 4, 70, 64, 128),
]


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("shape", SHAPES)
def test_forward(io, shape):
    x, _ = _make(*shape, io)
    o, S = O.forward(**x, scale=0.25)
    check(Run(x, io, 0.25).fwd(), {"o": o, "S": S}, dict(x, scale=0.25))


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("shape", SHAPES)
def test_backward(io, shape):
    x, d = _make(*shape, io, seed=1)
    o, S = O.forward(**x, scale=0.25)
    r = Run(x, io, 0.25)
    check(r.fwd(1), {"o": o, "S": S})
    got = r.bwd(d)
    check(got, O.backward(**x, scale=0.25, **d), dict(x, scale=0.25, **d))
    again = r.bwd(d, saved=0)
    for n in got:
        assert torch.equal(got[n], again[n]), n


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("shape", [(1, 2, 2, 1, 128, 128), (2, 6, 2, 3, 72, 100), (1, 1, 1, 40, 17, 33), (3, 2, 1, 2, 64, 64), (5, 16, 16, 1, 128, 128), (1, 1, 1, 1, 1, 1)])
def test_step(io, shape):
    x, _ = _make(*shape, io, seed=2)
    o, S = O.forward(**x, scale=0.5)
    check(Run(x, io, 0.5).step(), {"o": o, "S": S})


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("start", [True, False])
def test_edges_of_the_gates(io, start):
    x, d = _make(2, 4, 2, 150, 64, 64, io, seed=3, gates="edges", start=start)
    if not start:
        d["dS_final"] = None
    o, S = O.forward(**x, scale=1.0)
    r = Run(x, io, 1.0)
    check(r.fwd(1), {"o": o, "S": S})
    check(r.bwd(d), O.backward(**x, scale=1.0, **d), dict(x, scale=1.0, **d))
    if start:
        check(r.step(), {"o": o, "S": S})


@pytest.mark.parametrize("io", ["f32", "bf16"])
def test_no_decay_over_many_chunks(io):
    """The plain delta rule: nothing fades, so what a chunk gets wrong stays."""
    x, d = _make(1, 2, 2, 1024, 64, 64, io, seed=4)
    x["log_gamma"][:] = 0
    o, S = O.forward(**x, scale=1.0)
    r = Run(x, io, 1.0)
    check(r.fwd(1), {"o": o, "S": S})
    check(r.bwd(d), O.backward(**x, scale=1.0, **d), dict(x, scale=1.0, **d))


@pytest.mark.parametrize("size", [1e-12, 1e-4, 1e4])
def test_magnitudes_far_from_one(size):
    """Values, states and gradients far outside fp16's range; keys and queries stay the unit vectors that the rule is stable for."""
    for io in ("f32", "bf16"):
        x, d = _make(1, 2, 1, 100, 64, 48, io, seed=5)
        rnd = inputs.round_bf16 if io == "bf16" else (lambda a: a.astype(np.float32))
        x["v"], x["S"] = rnd(x["v"] * np.float32(size)), x["S"] * np.float32(size)
        d["d_o"], d["dS_final"] = rnd(d["d_o"] / np.float32(size)), d["dS_final"] / np.float32(size)
        o, S = O.forward(**x, scale=1.0)
        r = Run(x, io, 1.0)
        check(r.fwd(1), {"o": o, "S": S})
        check(r.bwd(d), O.backward(**x, scale=1.0, **d), dict(x, scale=1.0, **d))


def test_small_keys_of_one_chunk_beside_large_ones():
    x, d = _make(1, 2, 1, 128, 64, 64, "f32", seed=6)
    x["k"][:, :, 32:64] *= np.float32(1e-5)
    x["q"][:, :, 64:96] *= np.float32(1e-7)
    x["k"][:, :, 96:] = 0
    o, S = O.forward(**x, scale=1.0)
    r = Run(x, "f32", 1.0)
    check(r.fwd(1), {"o": o, "S": S})
    check(r.bwd(d), O.backward(**x, scale=1.0, **d), dict(x, scale=1.0, **d))


@pytest.mark.parametrize("io", ["f32", "bf16"])
def test_states_chain_and_may_be_updated_in_place(io):
    x, _ = _make(2, 2, 2, 96, 128, 64, io, seed=7)
    whole = Run(x, io, 1.0).fwd()
    cut = lambda a, lo, hi: a[:, :, lo:hi]  # noqa: E731
    S, parts = _dev(x["S"]), []
    for lo, hi in ((0, 64), (64, 93), (93, 96)):
        r = Run({**{n: cut(x[n], lo, hi) for n in ("q", "k", "v", "eta", "log_gamma")}, "S": x["S"]}, io, 1.0)
        r.S = r.S_out = S
        parts.append((r.fwd() if hi < 96 else r.step())["o"])
    o, Sf = O.forward(**x, scale=1.0)
    check({"o": torch.cat(parts, 2), "S": S}, {"o": o, "S": Sf}, dict(x, scale=1.0))
    check(whole, {"o": o, "S": Sf}, dict(x, scale=1.0))


@pytest.mark.parametrize("io", ["f32", "bf16"])
def test_unaligned_tensors(io):
    """Tensors that start one element past a 16-byte boundary."""
    x, d = _make(1, 2, 2, 70, 64, 64, io, seed=8)
    r = Run(x, io, 1.0)
    shift = lambda t: torch.cat([t.new_zeros(1), t.flatten()])[1:].view(t.shape)  # noqa: E731
    base, grads = {n: t.clone() for n, t in r.fwd(1).items()}, r.bwd(d)
    for n in ("q", "k", "v", "o", "eta", "lg", "S", "S_out"):
        setattr(r, n, shift(getattr(r, n)))
    got = r.fwd(1)
    for n in got:
        assert torch.equal(got[n], base[n]), n
    for n, t in r.bwd(d).items():
        assert torch.equal(t, grads[n]), n
    o, S = O.forward(**x, scale=1.0)
    check(r.step(), {"o": o, "S": S})


def test_a_sequence_does_not_depend_on_its_neighbours_and_nothing_behind_the_outputs_is_written():
    x, d = _make(3, 4, 2, 77, 64, 80, "bf16", seed=9)
    r = Run(x, "bf16", 1.0)
    big = torch.full((3 * 4 * 77 * 80 + 512,), 5.0, device="cuda", dtype=torch.bfloat16)
    r.o = big[: 3 * 4 * 77 * 80].view(3, 4, 77, 80)
    got, grads = r.fwd(1), r.bwd(d)
    assert (big[3 * 4 * 77 * 80:] == 5.0).all()
    one = Run({n: a[1:2] for n, a in x.items()}, "bf16", 1.0)
    alone = one.fwd(1)
    assert torch.equal(alone["o"], got["o"][1:2]) and torch.equal(alone["S"], got["S"][1:2])
    for n, t in one.bwd({n: a[1:2] for n, a in d.items()}).items():
        assert torch.equal(t, grads[n][1:2]), n


def test_graph_replay_on_a_side_stream_with_new_inputs():
    x, d = _make(1, 2, 2, 100, 64, 64, "bf16", seed=10)
    y, _ = _make(1, 2, 2, 100, 64, 64, "bf16", seed=11)
    r = Run(x, "bf16", 1.0)
    r.fwd(1)
    r.bwd(d)
    out = {n: torch.empty_like(t) for n, t in (("dq", r.q), ("dk", r.k), ("dv", r.v), ("d_eta", r.eta), ("d_log_gamma", r.eta), ("dS", r.S_out))}
    d_o, dS = _dev(d["d_o"], "bf16"), _dev(d["dS_final"])
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(stream), torch.cuda.graph(graph, stream=stream):
        E.e2ttt_delta_fwd(r.p, r.q, r.k, r.v, r.eta, r.lg, r.S, r.o, r.S_out, r.ws, 1)
        E.e2ttt_delta_bwd(r.p, r.q, r.k, r.v, r.eta, r.lg, r.S, d_o, dS, *out.values(), r.ws, 1)
    for n, t in (("q", r.q), ("k", r.k), ("v", r.v)):
        t.copy_(_dev(y[n], "bf16"))
    r.eta.copy_(_dev(y["eta"])), r.lg.copy_(_dev(y["log_gamma"])), r.S.copy_(_dev(y["S"]))
    graph.replay()
    torch.cuda.synchronize()
    o, S = O.forward(**y, scale=1.0)
    check({"o": r.o, "S": r.S_out}, {"o": o, "S": S})
    check(out, O.backward(**y, scale=1.0, **d), dict(y, scale=1.0, **d))


def test_two_streams_with_workspaces_of_their_own():
    runs = []
    for seed in (12, 13):
        x, _ = _make(2, 4, 4, 333, 128, 128, "bf16", seed=seed)
        runs.append((x, Run(x, "bf16", 1.0), torch.cuda.Stream()))
    for _, r, s in runs:
        r.ws = r.workspace(0)
        s.wait_stream(torch.cuda.current_stream())
    for _ in range(3):
        for _, r, s in runs:
            E.e2ttt_delta_fwd(r.p, r.q, r.k, r.v, r.eta, r.lg, r.S, r.o, r.S_out, r.ws, 0, stream=s)
    torch.cuda.synchronize()
    for x, r, _ in runs:
        o, S = O.forward(**x, scale=1.0)
        check({"o": r.o, "S": r.S_out}, {"o": o, "S": S}, dict(x, scale=1.0))


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("eta", [1.0, 1.5])
def test_one_key_in_all_tokens(io, eta):
    """What is written is read, and taken out, by every token: T's rows alternate in sign, their magnitudes sum to 1 + eta / (1 - |1 - eta|) <= 4,
    which times the operands' 2^-22 and the three products in a row stays below the tolerance."""
    x, d = _make(1, 2, 1, 100, 64, 48, io, seed=14)
    x["k"][:] = x["k"][:, :, :1]
    x["eta"][:], x["log_gamma"][:] = eta, 0
    o, S = O.forward(**x, scale=1.0)
    r = Run(x, io, 1.0)
    check(r.fwd(1), {"o": o, "S": S})
    check(r.bwd(d), O.backward(**x, scale=1.0, **d), dict(x, scale=1.0, **d))


def test_gradient_of_the_start_state_over_that_of_the_end():
    x, d = _make(3, 16, 4, 100, 128, 100, "bf16", seed=15)
    r = Run(x, "bf16", 1.0)
    r.fwd(1)
    want = r.bwd(d)
    dS = _dev(d["dS_final"])
    out = {n: torch.empty_like(t) for n, t in want.items()}
    out["dS"] = dS
    E.e2ttt_delta_bwd(r.p, r.q, r.k, r.v, r.eta, r.lg, r.S, _dev(d["d_o"], "bf16"), dS, *out.values(), r.ws, 1)
    for n in want:
        assert torch.equal(out[n], want[n]), n


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("shape", [(1, 3, 3, 300, 64, 64), (4, 16, 16, 300, 128, 64)])  # the columns of a slice over two warps; one warp per slice
def test_a_value_that_is_not_finite(io, bad, shape):
    """It reaches its own chunk and what follows it, nothing before it and no other head."""
    x, d = _make(*shape, io, seed=16)
    clean = Run(x, io, 1.0)
    good, grads = clean.fwd(1), clean.bwd(d)
    for name in ("v", "k", "eta"):
        r = Run(x, io, 1.0)
        t = getattr(r, name)
        t[0, 1, 170] = bad
        got = r.fwd(1)
        assert not torch.isfinite(got["o"][0, 1, 170]).all() or not torch.isfinite(got["o"][0, 1, 171]).all()
        assert torch.equal(got["o"][0, 1, :160], good["o"][0, 1, :160])
        back = r.bwd(d)
        for m in (0, 2):
            assert torch.equal(got["o"][0, m], good["o"][0, m]) and torch.equal(got["S"][0, m], good["S"][0, m])
            for n in back:
                assert torch.equal(back[n][0, m], grads[n][0, m]), (name, n)


def test_more_than_two_to_the_31_elements():
    """The last head starts 2^31 elements into q, k, v and o; it has to come out as it does alone."""
    H, L, d = 17, 1 << 20, 128
    g = torch.Generator(device="cuda").manual_seed(0)
    p = E.make_delta_params(1, H, H, L, d, d, E.E2TTT_BF16, 1.0)
    one = E.make_delta_params(1, 1, 1, L, d, d, E.E2TTT_BF16, 1.0)
    q, k, v = (torch.zeros(1, H, L, d, device="cuda", dtype=torch.bfloat16) for _ in range(3))
    eta, lg = torch.zeros(1, H, L, device="cuda"), torch.zeros(1, H, L, device="cuda")
    for t in (q, k, v):
        t[:, -1] = torch.randn(1, L, d, device="cuda", generator=g) / d ** 0.5
    eta[:, -1], lg[:, -1] = torch.rand(1, L, device="cuda", generator=g), -torch.rand(1, L, device="cuda", generator=g)
    o, S = torch.empty_like(v), torch.empty(1, H, d, d, device="cuda")
    ws = torch.empty(E.e2ttt_delta_workspace_bytes(p, 0), dtype=torch.uint8, device="cuda")
    E.e2ttt_delta_fwd(p, q, k, v, eta, lg, None, o, S, ws, 0)
    last = [t[:, -1:] for t in (q, k, v, eta, lg)]
    o1, S1 = torch.empty_like(last[2]), torch.empty(1, 1, d, d, device="cuda")
    E.e2ttt_delta_fwd(one, *last, None, o1, S1, ws, 0)
    assert torch.equal(o[:, -1:], o1) and torch.equal(S[:, -1:], S1)
    assert (o[:, :-1] == 0).all() and bool((o1 != 0).any())


def test_a_workspace_of_more_than_two_to_the_32_bytes():
    """The same for what the reverse pass keeps of the sequences."""
    H, L, d = 17, 1 << 17, 128
    g = torch.Generator(device="cuda").manual_seed(1)
    rnd = lambda *s: torch.randn(*s, device="cuda", generator=g)  # noqa: E731
    q, k, v, d_o = ((rnd(1, H, L, d) / d ** 0.5).bfloat16() for _ in range(4))
    eta, lg = torch.rand(1, H, L, device="cuda", generator=g), -torch.rand(1, H, L, device="cuda", generator=g)

    def run(h):
        p = E.make_delta_params(1, h, h, L, d, d, E.E2TTT_BF16, 1.0)
        x = [t[:, -h:] for t in (q, k, v, eta, lg)]
        n = E.e2ttt_delta_workspace_bytes(p, 1)
        ws = torch.empty(n, dtype=torch.uint8, device="cuda")
        S = torch.empty(1, h, d, d, device="cuda")
        out = [torch.empty_like(t) for t in x] + [S.clone()]
        E.e2ttt_delta_bwd(p, *x, None, d_o[:, -h:], None, *out, ws, 0)
        assert E.e2ttt_device_status(ws) == 0
        return n, out

    (n, all_), (_, last) = run(H), run(1)
    assert n > 1 << 32
    for a, b in zip(all_, last):
        assert torch.equal(a[:, -1:], b)


def test_step_with_more_than_two_to_the_31_values_of_state():
    B, H, d = 8200, 16, 128
    g = torch.Generator(device="cuda").manual_seed(2)
    rnd = lambda *s: torch.randn(*s, device="cuda", generator=g)  # noqa: E731
    S = torch.empty(B, H, d, d, device="cuda")
    S[:-1], S[-1] = 0, rnd(H, d, d)
    x = [(rnd(B, H, 1, d) / d ** 0.5).bfloat16() for _ in range(3)] + [torch.rand(B, H, 1, device="cuda", generator=g), -torch.rand(B, H, 1, device="cuda", generator=g)]
    one, o, o1, S1 = [t[-1:].contiguous() for t in x], torch.empty_like(x[2]), torch.empty_like(x[2][-1:]), S[-1:].clone()
    E.e2ttt_delta_step(E.make_delta_params(1, H, H, 1, d, d, E.E2TTT_BF16, 1.0), *one, S1, o1, S1)
    E.e2ttt_delta_step(E.make_delta_params(B, H, H, 1, d, d, E.E2TTT_BF16, 1.0), *x, S, o, S)
    assert torch.equal(o[-1:], o1) and torch.equal(S[-1:], S1)


def test_prepared_tokens_run_through_the_rule_and_back():
    """e2ttt_prepare_fwd's queries, keys, eta and gamma (its logarithm) are what the rule takes."""
    B, H, L, d = 1, 2, 75, 64
    g = torch.Generator(device="cuda").manual_seed(0)
    rnd = lambda *s: torch.randn(*s, device="cuda", generator=g)  # noqa: E731
    p = E.make_params(B, H, L, d, 4 * d, 1, E.E2TTT_MLP_GELU, E.E2TTT_BF16)
    gp = E.e2ttt_gate_params(0.5, 32.0, 0.1, 1e-12)
    raw = [rnd(B, H, L, d).bfloat16() for _ in range(2)]
    logits = [rnd(B, H, L) for _ in range(3)]
    q, k = torch.empty_like(raw[0]), torch.empty_like(raw[0])
    eta, beta, gamma = (torch.empty(B, H, L, device="cuda") for _ in range(3))
    E.e2ttt_prepare_fwd(p, gp, *raw, *logits, q, k, eta, beta, gamma)
    x = {"q": q.float().cpu().numpy(), "k": k.float().cpu().numpy(), "v": rnd(B, H, L, d).bfloat16().float().cpu().numpy(),
         "eta": eta.cpu().numpy(), "log_gamma": gamma.log().cpu().numpy(), "S": None}
    o, S = O.forward(**x, scale=1.0)
    check(Run(x, "bf16", 1.0).fwd(), {"o": o, "S": S}, dict(x, scale=1.0))
