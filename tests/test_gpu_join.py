"""Block join against its oracle in 64 bits, forward and reverse pass.

Tolerances, per value: half a step of the output's type relative to the value, plus TOL of the tensor's largest magnitude for the fp32 arithmetic
in between.  A value passes at most some 20 roundings of 2^-24 and two reciprocal roots and one exponential of 2^-21, and sums whose
rounding is below n 2^-24 of the sum of magnitudes: 1e-5 of the largest.  The vectors' gradients are sums over all tokens of such values.
d_o is the difference of two terms, dy / rms and its part along o: a rounding of either is relative to the term, not to the difference (with heads of one
value it leaves eps / o^2 of them), so the largest magnitude that counts is the terms'.
"""
import numpy as np
import pytest
import torch

from oracle import delta as OD
from oracle import join as O
from paper_2608_21308_b200 import binding as E
from paper_2608_21308_b200 import inputs

pytestmark = pytest.mark.gpu
TOL = 1e-5
GATES = {"none": E.E2TTT_GATE_NONE, "sigmoid": E.E2TTT_GATE_SIGMOID, "silu": E.E2TTT_GATE_SILU}
EPS = dict(post_eps=1e-6, pre_eps=1e-5)


def _make(B, H, L, d, io, kind, pre, seed=0):
    rng = np.random.default_rng(seed)
    rnd = inputs.round_bf16 if io == "bf16" else (lambda a: a.astype(np.float32))
    D = H * d
    f = lambda *s: rng.standard_normal(s).astype(np.float32)  # noqa: E731
    x = {"o": rnd(0.3 * f(B, H, L, d)), "a": None if kind == "none" else rnd(f(B, L, D)), "x": rnd(f(B, L, D)),
         "w_post": 1 + np.float32(0.1) * f(D), "res_scale": np.float32(0.5) + np.float32(0.1) * f(D),
         "w_pre": 1 + np.float32(0.1) * f(D) if pre else None}
    return x, {"d_x_out": rnd(f(B, L, D)), "d_n": rnd(f(B, L, D)) if pre else None}


def _dev(a, io=None):
    return None if a is None else torch.tensor(a, device="cuda").to(torch.bfloat16 if io == "bf16" else torch.float32).contiguous()


class Run:
    def __init__(self, x, io, kind):
        B, H, L, d = x["o"].shape
        self.p = E.make_join_params(B, H, L, d, E.E2TTT_F32 if io == "f32" else E.E2TTT_BF16, GATES[kind], **EPS)
        self.io = [_dev(x[n], io) for n in ("o", "a", "x")]
        self.w = [_dev(x[n]) for n in ("w_post", "res_scale", "w_pre")]
        self.kind = io

    def fwd(self):
        xo = torch.full_like(self.io[2], 7.0)
        n = None if self.w[2] is None else torch.full_like(xo, 7.0)
        E.e2ttt_join_fwd(self.p, *self.io, *self.w, xo, n)
        return {"x_out": xo, **({} if n is None else {"n": n})}

    def bwd(self, d):
        ws = torch.empty(E.e2ttt_join_workspace_bytes(self.p), dtype=torch.uint8, device="cuda").fill_(0xff)
        like = lambda t: None if t is None else torch.full_like(t, 7.0)  # noqa: E731
        out = {"d_" + n: like(t) for n, t in zip(("o", "a", "x", "w_post", "res_scale", "w_pre"), self.io + self.w)}
        E.e2ttt_join_bwd(self.p, *self.io, *self.w, _dev(d["d_x_out"], self.kind), _dev(d["d_n"], self.kind), *out.values(), ws)
        return {n: t for n, t in out.items() if t is not None}


def check(got, ref):
    ref, terms = ref if isinstance(ref, tuple) else (ref, {})
    for n, t in got.items():
        y, r = t.double().cpu().numpy(), ref[n]
        half = torch.finfo(t.dtype).eps / 2
        assert np.isfinite(y).all(), n
        over = np.abs(y - r) - half * np.abs(r) - TOL * np.abs(terms.get(n, r)).max()
        assert over.max() <= 0, (n, over.max(), np.abs(r).max(), np.linalg.norm(y - r) / np.linalg.norm(r))


SHAPES = [  # B, H, L, d
    (1, 1, 1, 1), (1, 16, 1, 128), (2, 12, 37, 64), (1, 1, 19, 768), (3, 1, 5, 4096), (1, 3, 7, 100), (2, 5, 3, 17), (1, 2, 9, 96), (1, 2, 4, 258),
    (1, 1, 3, 8192), (1, 64, 2, 128), (1, 1, 2, 4999), (4, 4, 400, 32), (1, 40, 700, 8), (2, 7, 1, 3), (1, 1, 1, 33),
]


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("kind,pre", [("silu", True), ("sigmoid", False), ("none", True)])
@pytest.mark.parametrize("shape", SHAPES)
def test_forward_and_backward(io, kind, pre, shape):
    x, d = _make(*shape, io, kind, pre)
    xo, n = O.forward(**x, kind=kind, **EPS)
    r = Run(x, io, kind)
    check(r.fwd(), {"x_out": xo, "n": n})
    got = r.bwd(d)
    check(got, O.backward(**x, kind=kind, **EPS, **d, terms=True))
    for m, t in r.bwd(d).items():
        assert torch.equal(t, got[m]), m  # repeats bit for bit


@pytest.mark.parametrize("io", ["f32", "bf16"])
def test_in_place_and_unaligned(io):
    x, d = _make(2, 4, 50, 64, io, "silu", True, seed=1)
    r = Run(x, io, "silu")
    base, grads = r.fwd(), r.bwd(d)
    shift = lambda t: None if t is None else torch.cat([t.new_zeros(1), t.flatten()])[1:].view(t.shape)  # noqa: E731
    r2 = Run(x, io, "silu")
    r2.io, r2.w = [shift(t) for t in r2.io], [shift(t) for t in r2.w]
    xo, n = O.forward(**x, kind="silu", **EPS)
    check(r2.fwd(), {"x_out": xo, "n": n})  # other pieces, other order of the sums
    check(r2.bwd(d), O.backward(**x, kind="silu", **EPS, **d, terms=True))
    E.e2ttt_join_fwd(r.p, *r.io, *r.w, r.io[2], r.io[1])  # x_out over x, n over a
    assert torch.equal(r.io[2], base["x_out"]) and torch.equal(r.io[1], base["n"])
    r = Run(x, io, "silu")
    dx = _dev(d["d_x_out"], io)
    out = {m: torch.empty_like(t) for m, t in grads.items()}
    out["d_x"] = dx  # d_x over d_x_out
    ws = torch.empty(E.e2ttt_join_workspace_bytes(r.p), dtype=torch.uint8, device="cuda")
    E.e2ttt_join_bwd(r.p, *r.io, *r.w, dx, _dev(d["d_n"], io), *[out["d_" + m] for m in ("o", "a", "x", "w_post", "res_scale", "w_pre")], ws)
    for m in grads:
        assert torch.equal(out[m], grads[m]), m


@pytest.mark.parametrize("io", ["f32", "bf16"])
def test_rows_of_zeros_and_extreme_gates(io):
    x, d = _make(1, 4, 6, 32, io, "sigmoid", True, seed=2)
    x["o"][0, 1, 2] = 0
    x["x"][0, 3] = 0
    x["o"][0, :, 3] = 0     # a token whose x_out is zero: n is zero, its gradients 1 / sqrt(eps) large but finite
    x["a"][0, 4] = 300
    x["a"][0, 5] = -300
    with np.errstate(over="ignore"):
        xo, n = O.forward(**x, kind="sigmoid", **EPS)
        ref = O.backward(**x, kind="sigmoid", **EPS, **d, terms=True)
    r = Run(x, io, "sigmoid")
    check(r.fwd(), {"x_out": xo, "n": n})
    check(r.bwd(d), ref)


def test_a_token_does_not_depend_on_the_others():
    x, d = _make(3, 4, 700, 64, "bf16", "silu", True, seed=3)
    r = Run(x, "bf16", "silu")
    got, grads = r.fwd(), r.bwd(d)
    cut = {n: (a[1:2] if n in ("o", "a", "x") else a) for n, a in x.items()}
    one = Run(cut, "bf16", "silu")
    for n, t in one.fwd().items():
        assert torch.equal(t, got[n][1:2]), n
    for n, t in one.bwd({n: a[1:2] for n, a in d.items()}).items():
        if n in ("d_o", "d_a", "d_x"):
            assert torch.equal(t, grads[n][1:2]), n


def test_more_than_two_to_the_31_elements():
    """The last tokens lie 2^31 elements into every tensor; they have to come out as they do alone."""
    H, L, d, n = 16, (1 << 20) + 64, 128, 64
    g = torch.Generator(device="cuda").manual_seed(0)
    o, a, x = (torch.zeros(*s, device="cuda", dtype=torch.bfloat16) for s in ((1, H, L, d), (1, L, H * d), (1, L, H * d)))
    for t in (o[:, :, -n:], a[:, -n:], x[:, -n:]):
        t.copy_(torch.randn(t.shape, device="cuda", generator=g))
    w = [1 + 0.1 * torch.randn(H * d, device="cuda", generator=g) for _ in range(3)]
    xo, no = torch.empty_like(x), torch.empty_like(x)
    E.e2ttt_join_fwd(E.make_join_params(1, H, L, d, E.E2TTT_BF16, E.E2TTT_GATE_SILU, **EPS), o, a, x, *w, xo, no)
    tail = [t.contiguous() for t in (o[:, :, -n:], a[:, -n:], x[:, -n:])]
    x1, n1 = torch.empty_like(tail[2]), torch.empty_like(tail[2])
    E.e2ttt_join_fwd(E.make_join_params(1, H, n, d, E.E2TTT_BF16, E.E2TTT_GATE_SILU, **EPS), *tail, *w, x1, n1)
    assert torch.equal(xo[:, -n:], x1) and torch.equal(no[:, -n:], n1)


def test_graph_replay_and_a_side_stream():
    x, d = _make(2, 4, 33, 64, "bf16", "silu", True, seed=4)
    y, _ = _make(2, 4, 33, 64, "bf16", "silu", True, seed=5)
    r = Run(x, "bf16", "silu")
    r.fwd(), r.bwd(d)
    xo, n = torch.empty_like(r.io[2]), torch.empty_like(r.io[2])
    out = {"d_" + m: torch.empty_like(t) for m, t in zip(("o", "a", "x", "w_post", "res_scale", "w_pre"), r.io + r.w)}
    ws = torch.empty(E.e2ttt_join_workspace_bytes(r.p), dtype=torch.uint8, device="cuda")
    dx, dn = _dev(d["d_x_out"], "bf16"), _dev(d["d_n"], "bf16")
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(stream), torch.cuda.graph(graph, stream=stream):
        E.e2ttt_join_fwd(r.p, *r.io, *r.w, xo, n)
        E.e2ttt_join_bwd(r.p, *r.io, *r.w, dx, dn, *out.values(), ws)
    for t, m in zip(r.io, ("o", "a", "x")):
        t.copy_(_dev(y[m], "bf16"))
    for t, m in zip(r.w, ("w_post", "res_scale", "w_pre")):
        t.copy_(_dev(y[m]))
    graph.replay()
    torch.cuda.synchronize()
    a, b = O.forward(**y, kind="silu", **EPS)
    check({"x_out": xo, "n": n}, {"x_out": a, "n": b})
    check(out, O.backward(**y, kind="silu", **EPS, **d, terms=True))


def test_a_block_of_prepare_rule_and_join_forward_and_back():
    """The operators as a layer uses them: prepared tokens, the gated delta rule, the join; the reverse passes hand their gradients on."""
    B, H, L, dh = 1, 2, 75, 64
    g = torch.Generator(device="cuda").manual_seed(0)
    rnd = lambda *s: torch.randn(*s, device="cuda", generator=g)  # noqa: E731
    f32 = dict(device="cuda", dtype=torch.float32)
    pp = E.make_params(B, H, L, dh, 4 * dh, 1, E.E2TTT_MLP_GELU, E.E2TTT_F32)
    gp = E.e2ttt_gate_params(0.5, 32.0, 0.1, 1e-12)
    raw, logits = [rnd(B, H, L, dh) for _ in range(2)], [rnd(B, H, L) for _ in range(3)]
    q, k = torch.empty_like(raw[0]), torch.empty_like(raw[0])
    eta, beta, gamma = (torch.empty(B, H, L, **f32) for _ in range(3))
    E.e2ttt_prepare_fwd(pp, gp, *raw, *logits, q, k, eta, beta, gamma)
    lg = gamma.log()
    dp = E.make_delta_params(B, H, H, L, dh, dh, E.E2TTT_F32, 1.0)
    v, o, S = rnd(B, H, L, dh), torch.empty(B, H, L, dh, **f32), torch.empty(B, H, dh, dh, **f32)
    ws = torch.empty(E.e2ttt_delta_workspace_bytes(dp, 1), dtype=torch.uint8, device="cuda")
    E.e2ttt_delta_fwd(dp, q, k, v, eta, lg, None, o, S, ws, 1)
    jp = E.make_join_params(B, H, L, dh, E.E2TTT_F32, E.E2TTT_GATE_SILU, **EPS)
    x, a, w = rnd(B, L, H * dh), rnd(B, L, H * dh), [1 + 0.1 * rnd(H * dh) for _ in range(3)]
    xo, n = torch.empty_like(x), torch.empty_like(x)
    E.e2ttt_join_fwd(jp, o, a, x, *w, xo, n)
    dxo, dn = rnd(B, L, H * dh), rnd(B, L, H * dh)
    d_o, d_a, d_x = torch.empty_like(o), torch.empty_like(a), torch.empty_like(x)
    jw = torch.empty(E.e2ttt_join_workspace_bytes(jp), dtype=torch.uint8, device="cuda")
    E.e2ttt_join_bwd(jp, o, a, x, *w, dxo, dn, d_o, d_a, d_x, *[torch.empty_like(t) for t in w], jw)
    grads = {m: torch.empty_like(t) for m, t in (("dq", q), ("dk", k), ("dv", v), ("d_eta", eta), ("d_log_gamma", eta), ("dS", S))}
    E.e2ttt_delta_bwd(dp, q, k, v, eta, lg, None, d_o, None, *grads.values(), ws, 1)
    num = lambda t: t.double().cpu().numpy()  # noqa: E731
    args = dict(q=num(q), k=num(k), v=num(v), eta=num(eta), log_gamma=num(lg), S=None, scale=1.0)
    ro, rS = OD.forward(**args)
    join = dict(a=num(a), x=num(x), w_post=num(w[0]), res_scale=num(w[1]), w_pre=num(w[2]), kind="silu", **EPS)
    rx, rn = O.forward(o=ro, **join)
    # o may be off by 2e-5 of its largest magnitude (the rule's tolerance); y = o / rms magnifies that by max |o| / min rms, and d_o, with y in both
    # of its factors, twice
    grow = np.abs(ro).max() / np.sqrt((ro ** 2).mean(-1)).min()
    near = lambda t, r: np.abs(num(t) - r).max() <= 2 * 2e-5 * grow * np.abs(r).max()  # noqa: E731
    assert grow < 100
    assert near(xo, rx) and near(n, rn)
    rj = O.backward(o=ro, **join, d_x_out=num(dxo), d_n=num(dn))
    assert near(d_o, rj["d_o"]) and near(d_x, rj["d_x"]) and near(d_a, rj["d_a"])
    ref = OD.backward(**args, d_o=rj["d_o"], dS_final=None)
    for m, t in grads.items():
        assert near(t, ref[m]), m
