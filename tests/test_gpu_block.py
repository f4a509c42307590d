"""Token preparation, gated delta rule and block join as one block, forward and back to the preparation's own inputs.

Tolerances as in the block join's test: the rule's outputs and gradients are off by 2e-5 of a tensor's largest value; the norm behind them magnifies that by
max |o| / min rms, twice where it stands in both factors; the preparation's own derivatives multiply by at most 1 / |silu(q)| and tau, and are taken relative to
what they give.
"""
import numpy as np
import pytest
import torch

from oracle import delta as OD
from oracle import join as OJ
from oracle import prepare as OP
from paper_2608_21308_b200 import binding as E

pytestmark = pytest.mark.gpu
EPS = dict(post_eps=1e-6, pre_eps=1e-5)


@pytest.mark.parametrize("L", [1, 75, 130])
def test_forward_and_back_to_the_raw_queries_keys_and_gates(L):
    B, H, dh = 2, 2, 64
    g = torch.Generator(device="cuda").manual_seed(7)
    rnd = lambda *s: torch.randn(*s, device="cuda", generator=g)  # noqa: E731
    num = lambda t: t.double().cpu().numpy()  # noqa: E731
    pp = E.make_params(B, H, L, dh, 4 * dh, 1, E.E2TTT_MLP_GELU, E.E2TTT_F32)
    gates = (0.5, 32.0, 0.1)
    gp = E.e2ttt_gate_params(*gates, 1e-12)
    raw, logits = [rnd(B, H, L, dh) for _ in range(2)], [rnd(B, H, L) for _ in range(3)]
    q, k = torch.empty_like(raw[0]), torch.empty_like(raw[0])
    eta, beta, gamma = (torch.empty(B, H, L, device="cuda") for _ in range(3))
    E.e2ttt_prepare_fwd(pp, gp, *raw, *logits, q, k, eta, beta, gamma)
    lg = gamma.log()
    dp = E.make_delta_params(B, H, H, L, dh, dh, E.E2TTT_F32, 1.0)
    v, S0 = rnd(B, H, L, dh), 0.3 * rnd(B, H, dh, dh)
    o, S = torch.empty_like(v), torch.empty_like(S0)
    ws = torch.empty(E.e2ttt_delta_workspace_bytes(dp, 1), dtype=torch.uint8, device="cuda")
    E.e2ttt_delta_fwd(dp, q, k, v, eta, lg, S0, o, S, ws, 1)
    jp = E.make_join_params(B, H, L, dh, E.E2TTT_F32, E.E2TTT_GATE_SILU, **EPS)
    x, a, w = rnd(B, L, H * dh), rnd(B, L, H * dh), [1 + 0.1 * rnd(H * dh) for _ in range(3)]
    xo, n = torch.empty_like(x), torch.empty_like(x)
    E.e2ttt_join_fwd(jp, o, a, x, *w, xo, n)

    dxo, dn, dS_final = rnd(B, L, H * dh), rnd(B, L, H * dh), 0.1 * rnd(B, H, dh, dh)
    d_o, d_a, d_x = torch.empty_like(o), torch.empty_like(a), torch.empty_like(x)
    jw = torch.empty(E.e2ttt_join_workspace_bytes(jp), dtype=torch.uint8, device="cuda")
    E.e2ttt_join_bwd(jp, o, a, x, *w, dxo, dn, d_o, d_a, d_x, *[torch.empty_like(t) for t in w], jw)
    dq, dk, dv, d_eta, d_lg, dS0 = (torch.empty_like(t) for t in (q, k, v, eta, eta, S0))
    E.e2ttt_delta_bwd(dp, q, k, v, eta, lg, S0, d_o, dS_final, dq, dk, dv, d_eta, d_lg, dS0, ws, 1)
    d_gamma, d_beta = d_lg / gamma, torch.zeros_like(beta)  # the rule takes gamma's logarithm, and has no momentum
    back = [torch.empty_like(t) for t in (*raw, *logits)]
    E.e2ttt_prepare_bwd(pp, gp, *raw, *logits, dq, dk, d_eta, d_beta, d_gamma, *back)

    r_eta, r_beta, r_gamma = OP.gates(*[num(t) for t in logits], *gates)
    args = dict(q=OP.silu_l2norm(num(raw[0])), k=OP.silu_l2norm(num(raw[1])), v=num(v), eta=r_eta, log_gamma=np.log(r_gamma), S=num(S0), scale=1.0)
    ro, rS = OD.forward(**args)
    join = dict(a=num(a), x=num(x), w_post=num(w[0]), res_scale=num(w[1]), w_pre=num(w[2]), kind="silu", **EPS)
    rx, rn = OJ.forward(o=ro, **join)
    grow = np.abs(ro).max() / np.sqrt((ro ** 2).mean(-1)).min()
    assert grow < 100
    near = lambda t, r: np.abs(num(t) - r).max() <= 2 * 2e-5 * grow * np.abs(r).max()  # noqa: E731
    assert near(xo, rx) and near(n, rn) and near(S, rS)
    rj = OJ.backward(o=ro, **join, d_x_out=num(dxo), d_n=num(dn))
    rd = OD.backward(**args, d_o=rj["d_o"], dS_final=num(dS_final))
    for m, t in (("dq", dq), ("dk", dk), ("dv", dv), ("d_eta", d_eta), ("d_log_gamma", d_lg), ("dS", dS0)):
        assert near(t, rd[m]), m
    ref = [OP.silu_l2norm_vjp(num(raw[0]), rd["dq"]), OP.silu_l2norm_vjp(num(raw[1]), rd["dk"]),
           *OP.gates_vjp(*[num(t) for t in logits], *gates, rd["d_eta"], np.zeros_like(r_beta), rd["d_log_gamma"] / r_gamma)]
    for m, t, r in zip(("q_raw", "k_raw", "a_eta", "a_beta", "a_alpha"), back, ref):
        assert near(t, r), m
