"""The linear-memory operators and the block join, as measurable cases.

A case is one call pattern of a program that holds a gated delta layer next to (or in place of) its E2-TTT layers:

  delta_forward  e2ttt_delta_fwd: prefill of whole sequences with the gated delta rule
  delta_train    the same with saved states and e2ttt_delta_bwd on them: one layer's training step
  delta_step     e2ttt_delta_step: the recurrent form, one or a few tokens of every sequence on its state
  join_forward   e2ttt_join_fwd: norm after the block, gate, residual scale and sum, norm before the next block
  join_train     e2ttt_join_fwd and e2ttt_join_bwd

The rule, per sequence and head, with a state S [dv, dk] (rows are outputs, as in every fast-weight matrix of the library):

  S'_t = exp(log_gamma_t) S_{t-1},   e_t = v_t - S'_t k_t,   S_t = S'_t + eta_t e_t k_t^T,   o_t = scale S_t q_t

The join, per token:  y = o / rms(o per head) * w_post,  x_out = x + res_scale * gate(a) * y,  n = x_out / rms(x_out) * w_pre.

Shapes are those of the benchmark configurations and tests: heads of 64 or 128, 1 to 16 heads, a batch of 1 to 8 (decoding: up to 64 requests),
sequences of one token to 32768; narrower and odd heads, query and key heads that several value heads share, and ragged lengths are what
the any-shape promise of the interface stands for.  Values: q and k are SiLU + L2-normalised rows (what the preparation step hands over),
v, residuals and output gradients N(0, 1), learning rates sigmoid(N(0, 1)), decays -A dt with A in 1..16 per head and dt = softplus(N(0, 1) - 4).
"""
from __future__ import annotations

import math

import torch

own = False

EPS = 1e-6


def _delta(name, op, B, H, Hk, L, dk, dv, io="bf16", start=True):
    c = {"op": op, "B": B, "H": H, "Hk": Hk, "L": L, "dk": dk, "dv": dv, "io": io, "start": start}
    return dict(c, name=name) if name else c


def _join(name, op, B, H, L, d, gate="silu", io="bf16", pre=True):
    c = {"op": op, "B": B, "H": H, "L": L, "d": d, "gate": gate, "io": io, "pre": pre}
    return dict(c, name=name) if name else c


def listed():
    return [
        # one token of one request, 16 heads: the smallest call of a decoder, launch and host latency
        _delta("delta step 1", "delta_step", 1, 16, 16, 1, 128, 128),
        # one token of each of 64 requests at the 1.3B layer shape: reads and writes 2 x 67 MB of state
        _delta("delta step 64", "delta_step", 64, 16, 16, 1, 128, 128),
        # prefill of one short ragged prompt at the 125M layer shape
        _delta("delta prefill short", "delta_forward", 1, 12, 12, 333, 64, 64),
        # prefill at the 1.3B layer shape
        _delta("delta prefill 1.3B", "delta_forward", 4, 16, 16, 4096, 128, 128),
        # prefill of one long context: few sequences, many chunks
        _delta("delta prefill long", "delta_forward", 1, 16, 16, 32768, 128, 128),
        # the checking mode: fp32 I/O, odd widths, two query and key heads for six value heads, from a zero state, both directions
        _delta("delta train f32 odd", "delta_train", 2, 6, 2, 777, 72, 100, io="f32", start=False),
        # training step at the 125M layer shape
        _delta("delta train 125M", "delta_train", 8, 12, 12, 2048, 64, 64),
        # training step at the 1.3B layer shape, four query and key heads for sixteen value heads
        _delta("delta train 1.3B", "delta_train", 4, 16, 4, 4096, 128, 128),
        # the join of one token of each of 8 requests
        _join("join step", "join_forward", 8, 16, 1, 128),
        # the join of a prefill at the 1.3B layer shape
        _join("join prefill 1.3B", "join_forward", 4, 16, 4096, 128),
        # training step of the join behind an output projection: one norm over the whole width of the 125M model, fp32
        _join("join train 125M f32", "join_train", 8, 1, 1000, 768, gate="sigmoid", io="f32"),
        # training step of the join at the 1.3B layer shape
        _join("join train 1.3B", "join_train", 4, 16, 4096, 128),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["delta_step", "delta_forward", "delta_forward", "delta_train", "delta_train", "join_forward", "join_train"])
    io = rng.choice(["bf16", "bf16", "bf16", "f32"])
    if op.startswith("join"):
        H, d = rng.choice([(1, rng.randint(64, 2048)), (rng.randint(1, 16), rng.choice([32, 64, 96, 128, rng.randint(16, 128)]))])
        tokens = _log_int(rng, 1, max(1, 16 * 1024 * 2048 // (H * d) // (2 if io == "f32" else 1)))
        B = min(tokens, rng.randint(1, 8))
        return _join(None, op, B, H, max(1, tokens // B), d, rng.choice(["none", "sigmoid", "silu"]), io, rng.random() < 0.8)
    Hk = rng.randint(1, 16)
    H = Hk * rng.choice([r for r in (1, 1, 2, 3, 4) if Hk * r <= 16])
    dk, dv = rng.choice([(64, 64), (128, 128), (128, 128), (rng.randint(16, 128), rng.randint(16, 128))])
    if op == "delta_step":
        return _delta(None, op, _log_int(rng, 1, 64), H, Hk, rng.choice([1, 1, 1, 2, 4]), dk, dv, io, True)
    B = rng.randint(1, 8)
    L = _log_int(rng, 2, min(32768 if op == "delta_forward" else 4096, 4 * 16 * 4096 // (B * H) // (4 if io == "f32" else 1)))
    return _delta(None, op, B, H, Hk, L, dk, dv, io, rng.random() < 0.5)


def prepare(case, seed):
    dev = torch.device("cuda")
    g = torch.Generator(device=dev)
    g.manual_seed(seed)
    io = torch.float32 if case["io"] == "f32" else torch.bfloat16

    def randn(*shape):
        return torch.randn(*shape, device=dev, generator=g)

    s = {"case": case}
    B, H, L = case["B"], case["H"], case["L"]
    if case["op"].startswith("join"):
        d = case["d"]
        D = H * d
        s["o"] = (0.3 * randn(B, H, L, d)).to(io)
        s["x"] = randn(B, L, D).to(io)
        s["a"] = randn(B, L, D).to(io) if case["gate"] != "none" else None
        s["w_post"], s["w_pre"] = 1.0 + 0.1 * randn(D), 1.0 + 0.1 * randn(D)
        s["res_scale"] = 0.5 + 0.1 * randn(D)
        s["x_out"], s["n"] = torch.empty_like(s["x"]), torch.empty_like(s["x"])
        if case["op"] == "join_train":
            s["d_x_out"], s["d_n"] = randn(B, L, D).to(io), randn(B, L, D).to(io)
            s["d_o"], s["d_x"], s["d_a"] = torch.empty_like(s["o"]), torch.empty_like(s["x"]), torch.empty_like(s["x"])
            s["d_w"] = [torch.empty_like(s["w_post"]) for _ in range(3)]
        return s
    Hk, dk, dv = case["Hk"], case["dk"], case["dv"]
    s["q"], s["k"] = (torch.nn.functional.normalize(torch.nn.functional.silu(randn(B, Hk, L, dk)), dim=-1).to(io) for _ in range(2))
    s["v"] = randn(B, H, L, dv).to(io)
    s["eta"] = torch.sigmoid(randn(B, H, L))
    decay = 1.0 + 15.0 * torch.rand(1, H, 1, device=dev, generator=g)
    s["log_gamma"] = -decay * torch.nn.functional.softplus(randn(B, H, L) - 4.0)
    s["S"] = 0.3 * randn(B, H, dv, dk) if case["start"] else None
    s["o"] = torch.empty_like(s["v"])
    s["S_out"] = torch.empty(B, H, dv, dk, device=dev)
    if case["op"] == "delta_train":
        s["d_o"] = randn(B, H, L, dv).to(io)
        s["dS_out"] = 0.1 * randn(B, H, dv, dk)
        s["d_qkv"] = [torch.empty_like(s[n]) for n in ("q", "k", "v")]
        s["d_eta"], s["d_log_gamma"] = torch.empty_like(s["eta"]), torch.empty_like(s["eta"])
        s["dS"] = torch.empty_like(s["S_out"])
    return s


def _scale(case):
    return case["dk"] ** -0.5


# ---- plain forms -----------------------------------------------------------------------------------------------
CHUNK = 64


def _plain_delta(q, k, v, eta, log_gamma, S, scale):
    """The rule chunk by chunk in 32 bits: within a chunk e = (I + N)^-1 (v - b S0 k), N the strictly lower part of D (k k^T) eta."""
    B, H, L, dv = v.shape
    dk, r = q.shape[-1], H // q.shape[1]
    C = min(CHUNK, L)
    n = -(-L // C)

    def cut(x):  # [B, H, L, ..] -> [B, H, n, C, ..], padded with zeros: tokens that write and read nothing
        x = torch.cat([x, x.new_zeros(x.shape[0], x.shape[1], n * C - L, *x.shape[3:])], 2) if n * C != L else x
        return x.reshape(x.shape[0], x.shape[1], n, C, *x.shape[3:])

    q, k = (x.repeat_interleave(r, 1) if r > 1 else x for x in (q, k))
    q, k, v, eta, log_gamma = cut(q), cut(k), cut(v), cut(eta), cut(log_gamma)
    run_sum = log_gamma.double().clamp(min=-1000.0).cumsum(-1)  # in 64 bits: the differences of long sums lose what matters in 32
    low = torch.ones(C, C, dtype=torch.bool, device=v.device).tril()
    D = (run_sum.unsqueeze(-1) - run_sum.unsqueeze(-2)).masked_fill(~low, -math.inf).exp().float()
    b, end = run_sum.exp().float().unsqueeze(-1), (run_sum[..., -1:] - run_sum).exp().float().unsqueeze(-1)
    N = -(((k @ k.transpose(-1, -2)) * D * eta.unsqueeze(-2)).tril(-1)).double()
    eye = torch.eye(C, dtype=torch.float64, device=v.device)
    T = eye + N
    power = N
    for _ in range(max(0, (C - 1).bit_length() - 1)):  # the sum of N^j, j < C, by squaring; in 64 bits: its terms cancel
        power = power @ power
        T = T @ (eye + power)
    T = T.float()
    A = (q @ k.transpose(-1, -2)) * D
    out = []
    for c in range(n):
        e = T[:, :, c] @ (v[:, :, c] - b[:, :, c] * (k[:, :, c] @ S.transpose(-1, -2)))
        u = eta[:, :, c].unsqueeze(-1) * e
        out.append(b[:, :, c] * (q[:, :, c] @ S.transpose(-1, -2)) + A[:, :, c] @ u)
        S = b[:, :, c, -1:] * S + (end[:, :, c] * u).transpose(-1, -2) @ k[:, :, c]
    return scale * torch.cat(out, 2)[:, :, :L], S


def _run_delta(s):
    case = s["case"]
    io = s["v"].dtype
    train = case["op"] == "delta_train"
    with torch.set_grad_enabled(train):
        x = [s[n].detach().float().requires_grad_(train) for n in ("q", "k", "v", "eta", "log_gamma")]
        S = (s["S"] if s["S"] is not None else torch.zeros_like(s["S_out"])).detach().requires_grad_(train)
        o, S_out = _plain_delta(*x, S, _scale(case))
    out = {"o": o.detach().to(io), "S": S_out.detach()}
    if train:
        d = torch.autograd.grad((o, S_out), (*x, S), (s["d_o"].float(), s["dS_out"]))
        out.update(dq=d[0].to(io), dk=d[1].to(io), dv=d[2].to(io), d_eta=d[3], d_log_gamma=d[4], dS=d[5])
    return out


def _gate(a, kind):
    sig = 1.0 / (1.0 + torch.exp(-a))
    return sig if kind == "sigmoid" else a * sig


def _plain_join(o, a, x, w_post, res_scale, w_pre, kind, pre):
    B, H, L, d = o.shape
    y = o / torch.sqrt((o * o).mean(-1, keepdim=True) + EPS)
    y = y.transpose(1, 2).reshape(B, L, H * d) * w_post
    x_out = x + res_scale * (y if a is None else _gate(a, kind) * y)
    if not pre:
        return (x_out,)
    return x_out, x_out / torch.sqrt((x_out * x_out).mean(-1, keepdim=True) + EPS) * w_pre


def _run_join(s):
    case = s["case"]
    io = s["x"].dtype
    train, pre = case["op"] == "join_train", case["pre"]
    names = ["o", "x", "w_post", "res_scale"] + (["w_pre"] if pre else []) + (["a"] if s["a"] is not None else [])
    with torch.set_grad_enabled(train):
        x = {n: s[n].detach().float().requires_grad_(train) for n in names}
        res = _plain_join(x["o"], x.get("a"), x["x"], x["w_post"], x["res_scale"], x.get("w_pre"), case["gate"], pre)
    out = {n: t.detach().to(io) for n, t in zip(("x_out", "n"), res)}
    if train:
        d = torch.autograd.grad(res, [x[n] for n in names], [s["d_x_out"].float(), s["d_n"].float()][: len(res)])
        out.update({"d_" + n: t.to(s[n].dtype) for n, t in zip(names, d)})
    return out


# ---- the library's calls ---------------------------------------------------------------------------------------
def _workspace(s, size):
    if "ws" not in s:  # a program keeps one for all of its calls
        s["ws"] = torch.empty(size, dtype=torch.uint8, device=s["o"].device)
    return s["ws"]


def _own_delta(s):
    from paper_2608_21308_b200 import binding as E
    case = s["case"]
    if "p" not in s:
        s["p"] = E.make_delta_params(case["B"], case["H"], case["Hk"], case["L"], case["dk"], case["dv"],
                                     E.E2TTT_F32 if case["io"] == "f32" else E.E2TTT_BF16, _scale(case))
    p = s["p"]
    if case["op"] == "delta_step":
        E.e2ttt_delta_step(p, s["q"], s["k"], s["v"], s["eta"], s["log_gamma"], s["S"], s["o"], s["S_out"])
        return {"o": s["o"], "S": s["S_out"]}
    train = case["op"] == "delta_train"
    ws = _workspace(s, 0) if "ws" in s else _workspace(s, E.e2ttt_delta_workspace_bytes(p, int(train)))
    E.e2ttt_delta_fwd(p, s["q"], s["k"], s["v"], s["eta"], s["log_gamma"], s["S"], s["o"], s["S_out"], ws, int(train))
    out = {"o": s["o"], "S": s["S_out"]}
    if train:
        dq, dk, dv = s["d_qkv"]
        E.e2ttt_delta_bwd(p, s["q"], s["k"], s["v"], s["eta"], s["log_gamma"], s["S"], s["d_o"], s["dS_out"], dq, dk, dv,
                          s["d_eta"], s["d_log_gamma"], s["dS"], ws, 1)
        out.update(dq=dq, dk=dk, dv=dv, d_eta=s["d_eta"], d_log_gamma=s["d_log_gamma"], dS=s["dS"])
    return out


def _own_join(s):
    from paper_2608_21308_b200 import binding as E
    case = s["case"]
    pre = case["pre"]
    if "p" not in s:
        s["p"] = E.make_join_params(case["B"], case["H"], case["L"], case["d"], E.E2TTT_F32 if case["io"] == "f32" else E.E2TTT_BF16,
                                    {"none": E.E2TTT_GATE_NONE, "sigmoid": E.E2TTT_GATE_SIGMOID, "silu": E.E2TTT_GATE_SILU}[case["gate"]], EPS, EPS)
    p = s["p"]
    w_pre, n = (s["w_pre"], s["n"]) if pre else (None, None)
    E.e2ttt_join_fwd(p, s["o"], s["a"], s["x"], s["w_post"], s["res_scale"], w_pre, s["x_out"], n)
    out = {"x_out": s["x_out"], **({"n": n} if pre else {})}
    if case["op"] == "join_train":
        ws = _workspace(s, 0) if "ws" in s else _workspace(s, E.e2ttt_join_workspace_bytes(p))
        d_post, d_res, d_pre = s["d_w"]
        d_a = s["d_a"] if s["a"] is not None else None
        E.e2ttt_join_bwd(p, s["o"], s["a"], s["x"], s["w_post"], s["res_scale"], w_pre, s["d_x_out"], s["d_n"] if pre else None,
                         s["d_o"], d_a, s["d_x"], d_post, d_res, d_pre if pre else None, ws)
        out.update(d_o=s["d_o"], d_x=s["d_x"], d_w_post=d_post, d_res_scale=d_res)
        if pre:
            out["d_w_pre"] = d_pre
        if d_a is not None:
            out["d_a"] = d_a
    return out


def run(state):
    join = state["case"]["op"].startswith("join")
    if own:
        return _own_join(state) if join else _own_delta(state)
    return _run_join(state) if join else _run_delta(state)


def work(case):
    """Each input read once, each output written once; the products of the token-wise rule only."""
    e = 4 if case["io"] == "f32" else 2
    B, H, L = case["B"], case["H"], case["L"]
    if case["op"].startswith("join"):
        n = B * L * H * case["d"]
        gate = case["gate"] != "none"
        fwd = n * e * (2 + gate + 1 + case["pre"])
        if case["op"] == "join_forward":
            return {"bytes": fwd, "flops": 20 * n}
        # what both directions share (o, a, x) is read once
        return {"bytes": fwd + n * e * (1 + case["pre"] + 2 + gate), "flops": 60 * n}
    Hk, dk, dv = case["Hk"], case["dk"], case["dv"]
    tokens, state = B * L, 4 * B * H * dk * dv
    io = tokens * (2 * Hk * dk + 2 * H * dv) * e + 8 * tokens * H
    states = state * (2 if case["start"] else 1)
    flops = 6 * tokens * H * dk * dv
    if case["op"] != "delta_train":
        return {"bytes": io + states, "flops": flops}
    return {"bytes": 2 * io + states + 2 * state, "flops": 3 * flops}


# ---- the definitions in 64 bits, token by token ------------------------------------------------------------------
def _exact_delta(s):
    case = s["case"]
    B, H, L, dk, dv = (case[n] for n in ("B", "H", "L", "dk", "dv"))
    Hk = case["Hk"]
    scale, r = _scale(case), H // Hk
    q, k = ((s[n].double().unsqueeze(2).expand(B, Hk, r, L, dk).reshape(B * H, L, dk)) for n in ("q", "k"))
    v = s["v"].double().reshape(B * H, L, dv)
    eta = s["eta"].double().reshape(B * H, L, 1)
    gamma = s["log_gamma"].double().exp().reshape(B * H, L, 1, 1)
    S = s["S"].double().reshape(B * H, dv, dk) if s["S"] is not None else torch.zeros(B * H, dv, dk, dtype=torch.float64, device=v.device)
    o = torch.empty_like(v)
    e = torch.empty_like(v)
    train = case["op"] == "delta_train"
    seg, kept = 64, []
    for t in range(L):
        if train and t % seg == 0:
            kept.append(S.clone())
        S = gamma[:, t] * S
        e[:, t] = v[:, t] - (S @ k[:, t].unsqueeze(-1)).squeeze(-1)
        S = torch.baddbmm(S, (eta[:, t] * e[:, t]).unsqueeze(-1), k[:, t].unsqueeze(-2))
        o[:, t] = scale * (S @ q[:, t].unsqueeze(-1)).squeeze(-1)
    out = {"o": o.reshape(B, H, L, dv), "S": S.reshape(B, H, dv, dk)}
    if not train:
        return out
    d_o = s["d_o"].double().reshape(B * H, L, dv)
    X = s["dS_out"].double().reshape(B * H, dv, dk)
    dq, d_k, d_v = torch.empty_like(q), torch.empty_like(k), torch.empty_like(v)
    d_eta, d_lg = torch.empty_like(eta), torch.empty_like(eta)
    for j in range(len(kept) - 1, -1, -1):
        before, after = [], []  # gamma S_{t-1} and S_t of the segment's tokens
        S = kept[j]
        for t in range(j * seg, min(L, j * seg + seg)):
            before.append(gamma[:, t] * S)
            S = torch.baddbmm(before[-1], (eta[:, t] * e[:, t]).unsqueeze(-1), k[:, t].unsqueeze(-2))
            after.append(S)
        for t in range(min(L, j * seg + seg) - 1, j * seg - 1, -1):
            Sp, St = before.pop(), after.pop()
            dq[:, t] = scale * (d_o[:, t].unsqueeze(-2) @ St).squeeze(-2)
            X = torch.baddbmm(X, scale * d_o[:, t].unsqueeze(-1), q[:, t].unsqueeze(-2))
            Xk = (X @ k[:, t].unsqueeze(-1)).squeeze(-1)
            de = eta[:, t] * Xk
            d_eta[:, t] = (e[:, t] * Xk).sum(-1, keepdim=True)
            d_k[:, t] = ((eta[:, t] * e[:, t]).unsqueeze(-2) @ X).squeeze(-2) - (de.unsqueeze(-2) @ Sp).squeeze(-2)
            d_v[:, t] = de
            X = torch.baddbmm(X, -de.unsqueeze(-1), k[:, t].unsqueeze(-2))
            d_lg[:, t] = (X * Sp).sum((-1, -2)).unsqueeze(-1)
            X = gamma[:, t] * X
    group = lambda x: x.reshape(B, Hk, r, L, dk).sum(2)  # noqa: E731
    out.update(dq=group(dq), dk=group(d_k), dv=d_v.reshape(B, H, L, dv), d_eta=d_eta.reshape(B, H, L), d_log_gamma=d_lg.reshape(B, H, L),
               dS=X.reshape(B, H, dv, dk))
    return out


def _exact_join(s):
    case = s["case"]
    B, H, L, d = (case[n] for n in ("B", "H", "L", "d"))
    D = H * d
    o = s["o"].double().permute(0, 2, 1, 3)  # [B, L, H, d]
    x, w, c = s["x"].double(), s["w_post"].double(), s["res_scale"].double()
    inv = (o.square().mean(-1, keepdim=True) + EPS).rsqrt()
    y0 = (o * inv).reshape(B, L, D)
    if s["a"] is None:
        g, dg = torch.ones_like(x), None
    else:
        a = s["a"].double()
        sig = torch.sigmoid(a)
        g, dg = (sig, sig * (1 - sig)) if case["gate"] == "sigmoid" else (a * sig, sig * (1 + a * (1 - sig)))
    x_out = x + c * g * w * y0
    out = {"x_out": x_out}
    if case["pre"]:
        wp = s["w_pre"].double()
        m = (x_out.square().mean(-1, keepdim=True) + EPS).rsqrt()
        out["n"] = x_out * m * wp
    if case["op"] == "join_forward":
        return out
    dx = s["d_x_out"].double()
    if case["pre"]:
        dn = s["d_n"].double()
        h = x_out * m
        dh = dn * wp
        out["d_w_pre"] = (dn * h).sum((0, 1))
        dx = dx + m * (dh - h * (dh * h).mean(-1, keepdim=True))
    out["d_x"] = dx
    out["d_res_scale"] = (dx * g * w * y0).sum((0, 1))
    out["d_w_post"] = (dx * c * g * y0).sum((0, 1))
    if dg is not None:
        out["d_a"] = dx * c * w * y0 * dg
    dy = (dx * c * g * w).reshape(B, L, H, d)
    yh = y0.reshape(B, L, H, d)
    out["d_o"] = (inv * (dy - yh * (dy * yh).mean(-1, keepdim=True))).permute(0, 2, 1, 3)
    return out


def exact(case, seed):
    s = prepare(case, seed)
    with torch.no_grad():
        return _exact_join(s) if case["op"].startswith("join") else _exact_delta(s)
