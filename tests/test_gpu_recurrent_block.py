"""A recurrent block's training step as a layer runs it: recurrence, join, both with their inputs in 8 bits, back through both; and its decoding steps.

Tolerances: the recurrence's outputs are off by its own share (its test derives it: under 2e-5 of a tensor's largest magnitude here); the join's norm magnifies that by
max |h| / min rms, twice where it stands in both factors.  The join's inputs in 8 bits add a rounding of their own: h as the join reads it back is taken from the GPU.
"""
import numpy as np
import pytest
import torch

from oracle import join as OJ
from oracle import pack8 as K
from oracle import scan as OS
from paper_2608_21308_b200 import binding as E

pytestmark = pytest.mark.gpu
EPS = dict(post_eps=1e-6, pre_eps=1e-5)


@pytest.mark.parametrize("L", [1, 75, 200])
def test_training_step(L):
    B, D = 2, 96
    g = torch.Generator(device="cuda").manual_seed(3)
    rnd = lambda *s: torch.randn(*s, device="cuda", generator=g)  # noqa: E731
    num = lambda t: t.double().cpu().numpy()  # noqa: E731
    x, r, gi = (rnd(B, L, D) for _ in range(3))
    rate, h0 = 0.01 + 0.1 * torch.rand(D, device="cuda", generator=g), rnd(B, D)
    starts = (torch.rand(B, L, device="cuda", generator=g) < 0.03).to(torch.uint8)
    sp = E.make_scan_params(B, L, D)
    ws = torch.empty(E.e2ttt_scan_workspace_bytes(sp, E.E2TTT_SAVE_PACKED), dtype=torch.uint8, device="cuda")
    h, last = torch.empty_like(x), torch.empty_like(h0)
    E.e2ttt_scan_fwd(sp, x, r, gi, rate, starts, h0, h, last, ws, E.E2TTT_SAVE_PACKED)
    # one head of the whole width: h [B,L,D] is o [B,1,L,D]
    jp = E.make_join_params(B, 1, L, D, E.E2TTT_F32, E.E2TTT_GATE_SILU, **EPS)
    res, a, w = rnd(B, L, D), rnd(B, L, D), [1 + 0.1 * rnd(D) for _ in range(3)]
    packed = torch.empty(E.e2ttt_join_packed_bytes(jp), dtype=torch.uint8, device="cuda")
    xo, n = torch.empty_like(res), torch.empty_like(res)
    E.e2ttt_join_fwd_packed(jp, h.view(B, 1, L, D), a, res, *w, xo, n, packed)
    keep = num(h)
    dxo, dn, end = rnd(B, L, D), rnd(B, L, D), rnd(B, D)
    d_h, d_a, d_res, d_w = torch.empty_like(h), torch.empty_like(a), torch.empty_like(res), [torch.empty_like(t) for t in w]
    jw = torch.empty(E.e2ttt_join_workspace_bytes(jp), dtype=torch.uint8, device="cuda")
    inputs = {"x": num(x), "r": num(r), "g": num(gi), "rate": num(rate), "starts": starts.cpu().numpy(), "h0": num(h0), "unit": True}
    join = dict(a=num(a), x=num(res), w_post=num(w[0]), res_scale=num(w[1]), w_pre=num(w[2]), kind="silu", **EPS)
    for t in (x, r, gi, h, a, res):
        t.fill_(float("nan"))  # the reverse passes read none of them
    E.e2ttt_join_bwd_packed(jp, packed, *w, dxo, dn, d_h.view(B, 1, L, D), d_a, d_res, *d_w, jw)
    out = {m: torch.empty_like(t) for m, t in (("d_x", x), ("da_decay", x), ("da_in", x), ("d_rate", rate), ("dh_init", h0))}
    E.e2ttt_scan_bwd(sp, None, None, None, rate, starts, h0, d_h, end, *out.values(), ws, E.E2TTT_SAVE_PACKED)

    rh, rlast, _ = OS.forward(**inputs)
    rx, rn = OJ.forward(o=rh[:, None], **join)
    grow = np.abs(rh).max() / np.sqrt((rh ** 2).mean(-1)).min()
    assert grow < 100
    near = lambda t, ref: np.abs((t if isinstance(t, np.ndarray) else num(t)) - ref).max() <= 2 * 2e-5 * grow * np.abs(ref).max()  # noqa: E731
    assert near(keep, rh) and near(last, rlast) and near(xo, rx) and near(n, rn)
    rj = OJ.backward(o=K.through(keep)[:, None], **{**join, "a": K.through(join["a"]), "x": K.through(join["x"])}, d_x_out=num(dxo), d_n=num(dn))
    assert near(d_h, rj["d_o"][:, 0]) and near(d_a, rj["d_a"]) and near(d_res, rj["d_x"])
    for m, t in zip(("d_w_post", "d_res_scale", "d_w_pre"), d_w):
        assert near(t, rj[m]), m
    ref, _ = OS.backward(**inputs, d_h=rj["d_o"][:, 0], dh_final=num(end), kept=tuple(K.through(inputs[m]) for m in ("x", "r", "g")))
    for m, t in out.items():
        assert near(t, ref[m]), m


def test_decoding_continues_a_prompt():
    """Prompt through the whole-sequence form, then token by token: recurrence and join give what they give over the whole sequence."""
    B, L, D, cut = 2, 40, 128, 36
    g = torch.Generator(device="cuda").manual_seed(4)
    rnd = lambda *s: torch.randn(*s, device="cuda", generator=g)  # noqa: E731
    x, r, gi, a, res = (rnd(B, L, D).bfloat16() for _ in range(5))
    rate, w = 0.01 + 0.1 * torch.rand(D, device="cuda", generator=g), [1 + 0.1 * rnd(D) for _ in range(3)]

    def run(lo, hi, state, step):
        n = hi - lo
        t = [v[:, lo:hi].contiguous() for v in (x, r, gi, a, res)]
        sp = E.make_scan_params(B, n, D, E.E2TTT_BF16)
        h, out = torch.empty_like(t[0]), torch.empty(B, D, device="cuda")
        if step:
            E.e2ttt_scan_step(sp, *t[:3], rate, None, state, h, out)
        else:
            E.e2ttt_scan_fwd(sp, *t[:3], rate, None, state, h, out)
        xo, no = torch.empty_like(h), torch.empty_like(h)
        E.e2ttt_join_fwd(E.make_join_params(B, 1, n, D, E.E2TTT_BF16, E.E2TTT_GATE_SILU, **EPS), h.view(B, 1, n, D), t[3], t[4], *w, xo, no)
        return h, out, xo, no

    whole = run(0, L, None, False)
    state = run(0, cut, None, False)[1]
    for t in range(cut, L):
        h, state, xo, no = run(t, t + 1, state, True)
        for got, ref in zip((h, xo, no), (whole[0], whole[2], whole[3])):
            ref = ref[:, t:t + 1].float()
            # both are roundings of values that agree to 2e-5: at most one step of bf16 apart, 2^-7; the join carries a step of h on, once through the product and once through the norm
            assert bool(((got.float() - ref).abs() <= 3 * 2.0 ** -7 * ref.abs().clamp(min=1.0)).all())
    assert bool(((state - whole[1]).abs() <= 2e-5 * whole[1].abs().max()).all())
