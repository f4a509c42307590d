"""Gated delta rule: what a call gives beside other calls of the same inputs."""
import pytest
import torch

from oracle import delta as O
from paper_2608_21308_b200 import binding as E
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


def _as_alone(got, alone, name):
    """What one sequence gives in a batch and alone, by kernels that cut a state differently: both are within 2e-5 of the exact tensor's largest value
    (times at most 16 norms / sqrt(elements): below 2^-9 of the norm) before they are rounded to the type, bf16 dq and dk within 3 x 2^-11 of their terms."""
    assert torch.isfinite(alone).all(), name
    err, size = (got.double() - alone.double()).norm(), alone.double().norm()
    assert err <= 2.0 ** -7 * size and size > 0, (name, err / size)


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("B", [2, 5, 30])  # 10, 25 and 150 slices of 16 value rows: the last is past one slice for an SM
def test_a_sequence_in_batches_of_any_size(io, B):
    x, d = _make(B, 5, 5, 77, 64, 16, io, seed=42)
    o, S = O.forward(**x, scale=1.0)
    r = Run(x, io, 1.0)
    check(r.fwd(1), {"o": o, "S": S})
    got = r.bwd(d)
    check(got, O.backward(**x, scale=1.0, **d), dict(x, scale=1.0, **d))
    one = Run({n: a[1:2] for n, a in x.items()}, io, 1.0)
    alone = {**one.fwd(1), **one.bwd({n: a[1:2] for n, a in d.items()})}
    for n, t in {"o": r.o, "S": r.S_out, **got}.items():
        if B * 5 <= 148:  # the same kernel: bit for bit
            assert torch.equal(t[1:2], alone[n]), n
        _as_alone(t[1:2], alone[n], n)


def test_more_than_two_to_the_31_elements_with_a_warp_per_slice():
    H, L, d = 20, 1 << 20, 128  # 160 slices; the last head starts 19 x 2^27 elements into q, k, v and o
    g = torch.Generator(device="cuda").manual_seed(3)
    q, k, v = (torch.zeros(1, H, L, d, device="cuda", dtype=torch.bfloat16) for _ in range(3))
    eta, lg = torch.zeros(1, H, L, device="cuda"), torch.zeros(1, H, L, device="cuda")
    for t in (q, k, v):
        t[:, -1] = torch.randn(1, L, d, device="cuda", generator=g) / d ** 0.5
    eta[:, -1], lg[:, -1] = torch.rand(1, L, device="cuda", generator=g), -torch.rand(1, L, device="cuda", generator=g)
    o, S = torch.empty_like(v), torch.empty(1, H, d, d, device="cuda")
    p, one = (E.make_delta_params(1, h, h, L, d, d, E.E2TTT_BF16, 1.0) for h in (H, 1))
    ws = torch.empty(E.e2ttt_delta_workspace_bytes(p, 0), dtype=torch.uint8, device="cuda")
    E.e2ttt_delta_fwd(p, q, k, v, eta, lg, None, o, S, ws, 0)
    last = [t[:, -1:] for t in (q, k, v, eta, lg)]
    o1, S1 = torch.empty_like(last[2]), torch.empty(1, 1, d, d, device="cuda")
    E.e2ttt_delta_fwd(one, *last, None, o1, S1, ws, 0)
    _as_alone(o[:, -1:], o1, "o"), _as_alone(S[:, -1:], S1, "S")
    assert (o[:, :-1] == 0).all()


def test_a_workspace_of_more_than_two_to_the_32_bytes_with_a_warp_per_slice():
    H, L, d = 20, 1 << 17, 128
    g = torch.Generator(device="cuda").manual_seed(4)
    rnd = lambda *s: torch.randn(*s, device="cuda", generator=g)  # noqa: E731
    q, k, v, d_o = ((rnd(1, H, L, d) / d ** 0.5).bfloat16() for _ in range(4))
    eta, lg = torch.rand(1, H, L, device="cuda", generator=g), -torch.rand(1, H, L, device="cuda", generator=g)

    def run(h):
        p = E.make_delta_params(1, h, h, L, d, d, E.E2TTT_BF16, 1.0)
        x = [t[:, -h:] for t in (q, k, v, eta, lg)]
        ws = torch.empty(E.e2ttt_delta_workspace_bytes(p, 1), dtype=torch.uint8, device="cuda")
        out = [torch.empty_like(t) for t in x] + [torch.empty(1, h, d, d, device="cuda")]
        E.e2ttt_delta_bwd(p, *x, None, d_o[:, -h:], None, *out, ws, 0)
        assert E.e2ttt_device_status(ws) == 0
        return ws.numel(), out

    (n, all_), (_, last) = run(H), run(1)
    assert n > 1 << 32
    for name, a, b in zip(("dq", "dk", "dv", "d_eta", "d_log_gamma", "dS"), all_, last):
        _as_alone(a[:, -1:], b, name)
