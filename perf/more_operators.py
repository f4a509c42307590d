"""The gated linear recurrence and the 8-bit activation checkpoints, as measurable cases.

A case is one call pattern of a program that holds recurrent blocks next to (or in place of) its E2-TTT layers:

  scan_forward  e2ttt_scan_fwd: prefill of whole sequences with the gated linear recurrence
  scan_train    the same with saved states, or with its inputs kept in 8 bits, and e2ttt_scan_bwd on them: one layer's training step
  scan_step     e2ttt_scan_step: one or a few tokens of every sequence on its state
  pack          e2ttt_pack8 and e2ttt_unpack8: an activation put away in 8 bits and read back
  join_train    e2ttt_join_fwd_packed and e2ttt_join_bwd_packed: the block join's training step, its inputs kept in 8 bits

The recurrence, per sequence and channel, with learned rates and a logit of decay and of input per token:

  a_t = exp(-rate sigmoid(r_t)),   i_t = sigmoid(g_t),   s_t = sqrt(1 - a_t^2),   h_t = a_t h_{t-1} + s_t i_t x_t

(s_t = 1 without unit scale, i_t = 1 without an input gate; a token that starts a document has a_t = 0 and s_t = 1).  With its inputs kept in 8 bits, the reverse
pass is the adjoint at the inputs that are read back; the states it multiplies are walked again from them, from the forward's own state before every 64th token,
which is kept in 32 bits.  8-bit checkpoints: a row is cut into
blocks of 32 values; a block's scale is 2^e, e the smallest integer with 127 2^e >= max |x|, its codes are the integers nearest to x 2^-e (ties to even).

Shapes are those of the benchmark configurations and tests: widths of 768 (12 heads of 64) and 2048 (16 heads of 128), a batch of 1 to 8 (decoding: up to 64
requests), sequences of one token to 32768; other widths and ragged lengths are what the any-shape promise of the interface stands for.  Values: activations,
logits and output gradients N(0, 1), rates -log(u) with u uniform in 0.9 .. 0.999 (a channel forgets over 10 to 1000 tokens with an open decay gate), documents of
some 500 tokens where there are several in a row.
"""
from __future__ import annotations

import math

import torch

own = False

EPS = 1e-6
BLOCK = 32
SPAN = 64  # tokens between two states that the recurrence keeps


def _scan(name, op, B, L, D, io="bf16", gate=True, unit=True, docs=False, save="states"):
    c = {"op": op, "B": B, "L": L, "D": D, "io": io, "gate": gate, "unit": unit, "docs": docs}
    if op == "scan_train":
        c["save"] = save
    return dict(c, name=name) if name else c


def _pack(name, rows, cols, io="bf16"):
    c = {"op": "pack", "rows": rows, "cols": cols, "io": io}
    return dict(c, name=name) if name else c


def _join(name, B, H, L, d, gate="silu", io="bf16", pre=True):
    c = {"op": "join_train", "B": B, "H": H, "L": L, "d": d, "gate": gate, "io": io, "pre": pre}
    return dict(c, name=name) if name else c


def listed():
    return [
        # one token of one request at the 1.3B width: the smallest call of a decoder, launch and host latency
        _scan("scan step 1", "scan_step", 1, 1, 2048),
        # one token of each of 64 requests
        _scan("scan step 64", "scan_step", 64, 1, 2048),
        # prefill of one short ragged prompt at the 125M width
        _scan("scan prefill short", "scan_forward", 1, 333, 768),
        # prefill at the 1.3B layer shape
        _scan("scan prefill 1.3B", "scan_forward", 4, 4096, 2048),
        # prefill of one long context: few channels, many tokens
        _scan("scan prefill long", "scan_forward", 1, 32768, 2048),
        # the checking mode: fp32 I/O, an odd width, several documents in a row, no input gate, both directions
        _scan("scan train f32 odd", "scan_train", 2, 777, 601, io="f32", gate=False, docs=True),
        # training step at the 125M layer shape, inputs kept in 8 bits
        _scan("scan train 125M packed", "scan_train", 8, 2048, 768, save="packed"),
        # training step at the 1.3B layer shape
        _scan("scan train 1.3B", "scan_train", 4, 4096, 2048),
        # a ragged fp32 activation put away and read back
        _pack("pack ragged f32", 1000, 777, io="f32"),
        # the residual stream of the 1.3B layer shape put away and read back
        _pack("pack 1.3B", 16384, 2048),
        # training step of the join behind an output projection at the 125M width, fp32, inputs kept in 8 bits
        _join("join train 125M f32 packed", 8, 1, 1000, 768, gate="sigmoid", io="f32"),
        # training step of the join at the 1.3B layer shape, inputs kept in 8 bits
        _join("join train 1.3B packed", 4, 16, 4096, 128),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["scan_step", "scan_forward", "scan_forward", "scan_train", "scan_train", "scan_train", "pack", "join_train", "join_train"])
    io = rng.choice(["bf16", "bf16", "bf16", "f32"])
    most = 4 * 4096 * 2048 // (2 if io == "f32" else 1)  # values of a tensor
    if op == "pack":
        cols = rng.choice([768, 2048, rng.randint(1, 4096), rng.randint(1, 4096)])
        return _pack(None, _log_int(rng, 1, max(1, most // cols)), cols, io)
    if op == "join_train":
        H, d = rng.choice([(1, rng.randint(64, 2048)), (rng.randint(1, 16), rng.choice([32, 64, 96, 128, rng.randint(16, 128)]))])
        tokens = _log_int(rng, 1, max(1, most // (H * d)))
        B = min(tokens, rng.randint(1, 8))
        return _join(None, B, H, max(1, tokens // B), d, rng.choice(["none", "sigmoid", "silu"]), io, rng.random() < 0.8)
    D = rng.choice([768, 2048, _log_int(rng, 16, 2048), _log_int(rng, 16, 2048)])
    gate, unit, docs = rng.random() < 0.8, rng.random() < 0.8, rng.random() < 0.3
    if op == "scan_step":
        return _scan(None, op, _log_int(rng, 1, 64), rng.choice([1, 1, 1, 2, 4]), D, io, gate, unit, docs)
    B = rng.randint(1, 8)
    L = _log_int(rng, 2, min(32768, max(2, most // (B * D))))
    return _scan(None, op, B, L, D, io, gate, unit, docs, rng.choice(["states", "packed"]))


def prepare(case, seed):
    dev = torch.device("cuda")
    g = torch.Generator(device=dev)
    g.manual_seed(seed)
    io = torch.float32 if case["io"] == "f32" else torch.bfloat16

    def randn(*shape):
        return torch.randn(*shape, device=dev, generator=g)

    s = {"case": case}
    if case["op"] == "pack":
        # rows of differing size, as a residual stream's tokens are
        s["x"] = (torch.exp(randn(case["rows"], 1)) * randn(case["rows"], case["cols"])).to(io)
        s["codes"] = torch.empty(s["x"].shape, dtype=torch.int8, device=dev)
        s["scales"] = torch.empty(case["rows"], -(-case["cols"] // BLOCK), dtype=torch.uint8, device=dev)
        s["back"] = torch.empty_like(s["x"])
        return s
    B, L = case["B"], case["L"]
    if case["op"] == "join_train":
        H, d = case["H"], case["d"]
        D = H * d
        s["o"] = (0.3 * randn(B, H, L, d)).to(io)
        s["x"] = randn(B, L, D).to(io)
        s["a"] = randn(B, L, D).to(io) if case["gate"] != "none" else None
        s["w_post"], s["w_pre"] = 1.0 + 0.1 * randn(D), 1.0 + 0.1 * randn(D)
        s["res_scale"] = 0.5 + 0.1 * randn(D)
        s["x_out"], s["n"] = torch.empty_like(s["x"]), torch.empty_like(s["x"])
        s["d_x_out"], s["d_n"] = randn(B, L, D).to(io), randn(B, L, D).to(io)
        s["d_o"], s["d_x"], s["d_a"] = torch.empty_like(s["o"]), torch.empty_like(s["x"]), torch.empty_like(s["x"])
        s["d_w"] = [torch.empty_like(s["w_post"]) for _ in range(3)]
        return s
    D = case["D"]
    s["x"], s["r"] = randn(B, L, D).to(io), randn(B, L, D).to(io)
    s["g"] = randn(B, L, D).to(io) if case["gate"] else None
    s["rate"] = -torch.log(0.9 + 0.099 * torch.rand(D, device=dev, generator=g))
    s["starts"] = (torch.rand(B, L, device=dev, generator=g) < 0.002).to(torch.uint8) if case["docs"] else None
    s["h0"] = 0.3 * randn(B, D)
    s["h"], s["h_out"] = torch.empty_like(s["x"]), torch.empty_like(s["h0"])
    if case["op"] == "scan_train":
        s["d_h"], s["dh_out"] = randn(B, L, D).to(io), randn(B, D)
        s["d_x"], s["d_r"] = torch.empty_like(s["x"]), torch.empty_like(s["r"])
        s["d_g"] = torch.empty_like(s["g"]) if case["gate"] else None
        s["d_rate"], s["dh0"] = torch.empty_like(s["rate"]), torch.empty_like(s["h0"])
    return s


# ---- plain forms -----------------------------------------------------------------------------------------------
def _plain_codes(x):
    """(codes, scales) of x [.., n] in blocks of 32, in 64 bits: codes and their powers of two are then exact."""
    n = x.shape[-1]
    pad = -n % BLOCK
    y = torch.nn.functional.pad(x.double(), (0, pad)).reshape(*x.shape[:-1], -1, BLOCK)
    m, e = torch.frexp(y.abs().amax(-1, keepdim=True))  # max |x| = m 2^e, m in [0.5, 1)
    e = torch.where(m > 127.0 / 128.0, e - 6, e - 7).clamp(-126, 121)
    scale = torch.ldexp(torch.ones_like(m), e)
    return torch.round(y / scale), scale


def _plain_packed(x):
    """The values that x's 8-bit checkpoint stands for, in 32 bits."""
    codes, scale = _plain_codes(x)
    return (codes * scale).flatten(-2)[..., : x.shape[-1]].float()


def _plain_prefix(c, b, reverse=False):
    """y_t = (1 - c_t) y_{t-1} + b_t along dimension 1 from zero (or y_t = (1 - c_t) y_{t+1} + b_t): distances of 1, 2, 4, .. in turn.  What is forgotten, c, is
    what is kept of the decays: 1 - c is rounded where it is next to 1, and over a long memory that adds up."""
    if reverse:
        return _plain_prefix(c.flip(1), b.flip(1)).flip(1)
    step, L = 1, c.shape[1]
    c, b = c.clone(), b.clone()
    while step < L:
        far = b[:, :-step].clone()
        b[:, step:] = b[:, step:] + (far - c[:, step:] * far)
        c[:, step:] = c[:, step:] + c[:, :-step].clone() * (1.0 - c[:, step:])
        step *= 2
    return b


def _run_scan(s):
    case = s["case"]
    io = s["x"].dtype
    x, r, g = s["x"].float(), s["r"].float(), None if s["g"] is None else s["g"].float()

    def gates():
        sg = 1.0 / (1.0 + torch.exp(-r))
        la = -s["rate"] * sg
        i = torch.ones_like(x) if g is None else 1.0 / (1.0 + torch.exp(-g))
        c = -torch.expm1(la)  # 1 - a
        scale = torch.sqrt(-torch.expm1(2.0 * la)) if case["unit"] else torch.ones_like(x)
        first = None
        if s["starts"] is not None:
            first = (s["starts"] != 0).unsqueeze(-1)
            c, scale = c.masked_fill(first, 1.0), scale.masked_fill(first, 1.0)
        return sg, la, c, i, scale, first

    def states(c, b):
        b = b.clone()
        b[:, 0] += (1.0 - c[:, 0]) * s["h0"]
        return _plain_prefix(c, b)

    sg, la, c, i, scale, first = gates()
    h = states(c, scale * i * x)
    out = {"h": h.to(io), "h_out": h[:, -1]}
    if case["op"] != "scan_train":
        return out
    if case["save"] == "packed":
        x, r, g = (None if t is None else _plain_packed(t) for t in (x, r, g))
        sg, la, c, i, scale, first = gates()
        kept = torch.cat([s["h0"].unsqueeze(1), h[:, SPAN - 1:-1:SPAN]], 1)
        c1, b = c.clone(), scale * i * x
        b[:, ::SPAN] += (1.0 - c[:, ::SPAN]) * kept
        c1[:, ::SPAN] = 1.0
        h = _plain_prefix(c1, b)
    else:
        kept = None
    before = torch.cat([s["h0"].unsqueeze(1), h[:, :-1]], 1)
    if kept is not None:
        before[:, ::SPAN] = kept
    d = s["d_h"].float().clone()
    d[:, -1] += s["dh_out"]
    lam = _plain_prefix(torch.cat([c[:, 1:], torch.ones_like(c[:, :1])], 1), d, reverse=True)
    a = 1.0 - c
    out["dh0"] = a[:, 0] * lam[:, 0]
    out["d_x"] = (lam * scale * i).to(io)
    if g is not None:
        out["d_g"] = (lam * scale * x * i * (1.0 - i)).to(io)
    d_la = a * lam * (before - a * i * x / scale) if case["unit"] else a * lam * before
    if first is not None:
        d_la = d_la.masked_fill(first, 0.0)
    out["d_r"] = (d_la * la * (1.0 - sg)).to(io)
    out["d_rate"] = -(d_la * sg).sum((0, 1))
    return out


def _run_step(s):
    case = s["case"]
    h, out = s["h0"], []
    for t in range(case["L"]):
        x, r = s["x"][:, t].float(), s["r"][:, t].float()
        la = -s["rate"] / (1.0 + torch.exp(-r))
        b = x if s["g"] is None else x / (1.0 + torch.exp(-s["g"][:, t].float()))
        a = torch.exp(la)
        y = a * h + (torch.sqrt(-torch.expm1(2.0 * la)) * b if case["unit"] else b)
        h = y if s["starts"] is None else torch.where(s["starts"][:, t, None] != 0, b, y)
        out.append(h)
    return {"h": torch.stack(out, 1).to(s["x"].dtype), "h_out": h}


def _run_pack(s):
    return {"back": _plain_packed(s["x"]).to(s["x"].dtype)}


def _gate(a, kind):
    sig = 1.0 / (1.0 + torch.exp(-a))
    return sig if kind == "sigmoid" else a * sig


def _plain_join(o, a, x, w_post, res_scale, w_pre, d, kind, pre):
    """o, a, x [B,L,D]: rows of tokens, heads of d columns."""
    y = o.reshape(*o.shape[:2], -1, d)
    y = (y / torch.sqrt((y * y).mean(-1, keepdim=True) + EPS)).reshape(o.shape) * w_post
    x_out = x + res_scale * (y if a is None else _gate(a, kind) * y)
    if not pre:
        return (x_out,)
    return x_out, x_out / torch.sqrt((x_out * x_out).mean(-1, keepdim=True) + EPS) * w_pre


def _run_join(s):
    case = s["case"]
    io, pre = s["x"].dtype, case["pre"]
    B, H, L, d = (case[n] for n in ("B", "H", "L", "d"))
    acts = {"o": s["o"].float().transpose(1, 2).reshape(B, L, H * d), "x": s["x"].float()}
    if s["a"] is not None:
        acts["a"] = s["a"].float()
    weights = {n: s[n] for n in ["w_post", "res_scale"] + (["w_pre"] if pre else [])}

    def form(t):
        return _plain_join(t["o"], t.get("a"), t["x"], t["w_post"], t["res_scale"], t.get("w_pre"), d, case["gate"], pre)

    with torch.no_grad():
        out = {n: t.to(io) for n, t in zip(("x_out", "n"), form({**acts, **weights}))}
        kept = {n: _plain_packed(t) for n, t in acts.items()}
    leaves = {n: t.detach().requires_grad_(True) for n, t in {**kept, **weights}.items()}
    res = form(leaves)
    grads = torch.autograd.grad(res, list(leaves.values()), [s["d_x_out"].float(), s["d_n"].float()][: len(res)])
    grads = dict(zip(leaves, grads))
    grads["o"] = grads["o"].reshape(B, L, H, d).transpose(1, 2)
    out.update({"d_" + n: t.to(s[n].dtype).contiguous() for n, t in grads.items()})
    return out


# ---- the library's calls ---------------------------------------------------------------------------------------
def _own_scan(s):
    from paper_2608_21308_b200 import binding as E
    case = s["case"]
    if "p" not in s:
        s["p"] = E.make_scan_params(case["B"], case["L"], case["D"], E.E2TTT_F32 if case["io"] == "f32" else E.E2TTT_BF16,
                                    E.E2TTT_GATE_SIGMOID if case["gate"] else E.E2TTT_GATE_NONE, int(case["unit"]))
    p = s["p"]
    if case["op"] == "scan_step":
        E.e2ttt_scan_step(p, s["x"], s["r"], s["g"], s["rate"], s["starts"], s["h0"], s["h"], s["h_out"])
        return {"h": s["h"], "h_out": s["h_out"]}
    train = case["op"] == "scan_train"
    save = (E.E2TTT_SAVE_PACKED if case["save"] == "packed" else E.E2TTT_SAVE_STATES) if train else E.E2TTT_SAVE_NONE
    if "ws" not in s:  # a program keeps one per layer
        s["ws"] = torch.empty(E.e2ttt_scan_workspace_bytes(p, save), dtype=torch.uint8, device=s["x"].device)
    E.e2ttt_scan_fwd(p, s["x"], s["r"], s["g"], s["rate"], s["starts"], s["h0"], s["h"], s["h_out"], s["ws"], save)
    out = {"h": s["h"], "h_out": s["h_out"]}
    if train:
        x, r, g = (None, None, None) if case["save"] == "packed" else (s["x"], s["r"], s["g"])
        E.e2ttt_scan_bwd(p, x, r, g, s["rate"], s["starts"], s["h0"], s["d_h"], s["dh_out"], s["d_x"], s["d_r"], s["d_g"], s["d_rate"], s["dh0"],
                         s["ws"], save)
        out.update(dh0=s["dh0"], d_x=s["d_x"], **({} if s["d_g"] is None else {"d_g": s["d_g"]}), d_r=s["d_r"], d_rate=s["d_rate"])
    return out


def _own_pack(s):
    from paper_2608_21308_b200 import binding as E
    if "p" not in s:
        s["p"] = E.make_pack_params(s["case"]["rows"], s["case"]["cols"], E.E2TTT_F32 if s["case"]["io"] == "f32" else E.E2TTT_BF16)
    E.e2ttt_pack8(s["p"], s["x"], s["codes"], s["scales"])
    E.e2ttt_unpack8(s["p"], s["codes"], s["scales"], s["back"])
    return {"back": s["back"]}


def _own_join(s):
    from paper_2608_21308_b200 import binding as E
    case = s["case"]
    pre = case["pre"]
    if "p" not in s:
        s["p"] = E.make_join_params(case["B"], case["H"], case["L"], case["d"], E.E2TTT_F32 if case["io"] == "f32" else E.E2TTT_BF16,
                                    {"none": E.E2TTT_GATE_NONE, "sigmoid": E.E2TTT_GATE_SIGMOID, "silu": E.E2TTT_GATE_SILU}[case["gate"]], EPS, EPS)
        s["packed"] = torch.empty(E.e2ttt_join_packed_bytes(s["p"]), dtype=torch.uint8, device=s["x"].device)
        s["ws"] = torch.empty(E.e2ttt_join_workspace_bytes(s["p"]), dtype=torch.uint8, device=s["x"].device)
    p = s["p"]
    w_pre, n, d_n, d_pre = (s["w_pre"], s["n"], s["d_n"], s["d_w"][2]) if pre else (None, None, None, None)
    d_a = s["d_a"] if s["a"] is not None else None
    E.e2ttt_join_fwd_packed(p, s["o"], s["a"], s["x"], s["w_post"], s["res_scale"], w_pre, s["x_out"], n, s["packed"])
    E.e2ttt_join_bwd_packed(p, s["packed"], s["w_post"], s["res_scale"], w_pre, s["d_x_out"], d_n, s["d_o"], d_a, s["d_x"], s["d_w"][0], s["d_w"][1], d_pre, s["ws"])
    out = {"x_out": s["x_out"], **({"n": n} if pre else {}), "d_o": s["d_o"], "d_x": s["d_x"], **({} if d_a is None else {"d_a": d_a})}
    out.update(d_w_post=s["d_w"][0], d_res_scale=s["d_w"][1], **({"d_w_pre": d_pre} if pre else {}))
    return out


def run(state):
    op = state["case"]["op"]
    if own:
        return _own_pack(state) if op == "pack" else _own_join(state) if op == "join_train" else _own_scan(state)
    return {"pack": _run_pack, "join_train": _run_join, "scan_step": _run_step}.get(op, _run_scan)(state)


def work(case):
    """Each input read once, each output written once; what an 8-bit checkpoint itself takes lies between the passes and is not counted, but for `pack`,
    whose output it is."""
    e = 4 if case["io"] == "f32" else 2
    if case["op"] == "pack":
        n = case["rows"] * case["cols"]
        blocks = case["rows"] * -(-case["cols"] // BLOCK)
        return {"bytes": 2 * (n * (e + 1) + blocks), "flops": 6 * n}
    if case["op"] == "join_train":
        n = case["B"] * case["L"] * case["H"] * case["d"]
        gate = case["gate"] != "none"
        return {"bytes": n * e * (2 + gate + 1 + case["pre"] + 1 + case["pre"] + 2 + gate), "flops": 70 * n}
    n, ends = case["B"] * case["L"] * case["D"], 4 * case["B"] * case["D"]
    fwd = n * e * (3 + case["gate"])
    if case["op"] != "scan_train":
        return {"bytes": fwd + 2 * ends, "flops": 20 * n}
    return {"bytes": fwd + n * e * (3 + case["gate"]) + 4 * ends, "flops": 60 * n}


# ---- the definitions in 64 bits, token by token ------------------------------------------------------------------
def _exact_packed(x):
    """x's 8-bit checkpoint by its definition: the smallest power of two that holds the block, found by trying."""
    n = x.shape[-1]
    x = x.double()
    blocks = list(range(0, n, BLOCK))
    big = torch.stack([x[..., c:c + BLOCK].abs().amax(-1) for c in blocks], -1)
    e = torch.floor(torch.log2(big.clamp(min=1e-300) / 127.0)) - 1.0
    for _ in range(3):
        e = torch.where(127.0 * torch.exp2(e) < big, e + 1.0, e)
    unit = torch.exp2(e.clamp(-126.0, 121.0)).repeat_interleave(BLOCK, -1)[..., :n]
    return torch.round(x / unit) * unit


def _exact_scan(s):
    case = s["case"]
    train = case["op"] == "scan_train"
    L = case["L"]

    def series(name):
        return None if s[name] is None else s[name].double().transpose(0, 1).contiguous()  # [L,B,D]

    x, r, g = (series(n) for n in ("x", "r", "g"))
    rate, h0 = s["rate"].double(), s["h0"].double()
    start = None if s["starts"] is None else (s["starts"].t() != 0).unsqueeze(-1)

    def walk(x, r, g, known=None):
        la = -rate * torch.sigmoid(r)
        one_less = -torch.expm1(2.0 * la)  # 1 - a^2
        if not case["unit"]:
            one_less = torch.ones_like(la)
        a = la.exp()
        if start is not None:
            a, one_less = torch.where(start, 0.0, a), torch.where(start, 1.0, one_less)
        u = x if g is None else x * torch.sigmoid(g)
        b = one_less.sqrt() * u
        before, last = torch.empty_like(x), h0
        for t in range(L):
            if known is not None and t % SPAN == 0:
                last = known[t]
            before[t] = last
            last = torch.addcmul(b[t], a[t], last)
        return la, one_less, a, u, before, last

    la, one_less, a, u, before, last = walk(x, r, g)
    out = {"h": torch.cat([before[1:], last.unsqueeze(0)]).transpose(0, 1), "h_out": last}
    if not train:
        return out
    if case["save"] == "packed":
        x, r, g = (None if t is None else _exact_packed(t) for t in (x, r, g))
        la, one_less, a, u, before, _ = walk(x, r, g, before)
    lam = s["d_h"].double().transpose(0, 1).contiguous()
    lam[L - 1] += s["dh_out"].double()
    for t in range(L - 2, -1, -1):
        lam[t].addcmul_(a[t + 1], lam[t + 1])
    out["dh0"] = a[0] * lam[0]
    root = one_less.sqrt()
    out["d_x"] = lam * root if g is None else lam * root * torch.sigmoid(g)
    if g is not None:
        out["d_g"] = lam * root * u * torch.sigmoid(-g)
    to_a = lam * before
    if case["unit"]:
        to_a = to_a - lam * u * a / root  # through sqrt(1 - a^2)
    to_la = a * to_a
    if start is not None:
        to_la = torch.where(start, 0.0, to_la)
    out["d_r"] = to_la * la * torch.sigmoid(-r)
    out["d_rate"] = -(to_la * torch.sigmoid(r)).sum((0, 1))
    for n in ("d_x", "d_g", "d_r"):
        if n in out:
            out[n] = out[n].transpose(0, 1)
    return out


def _exact_join(s):
    case = s["case"]
    B, H, L, d = (case[n] for n in ("B", "H", "L", "d"))
    D = H * d
    w, c = s["w_post"].double(), s["res_scale"].double()
    wp = s["w_pre"].double() if case["pre"] else None

    def forward(o, a, x):
        o = o.reshape(B, L, H, d)
        inv = (o.square().mean(-1, keepdim=True) + EPS).rsqrt()
        y0 = (o * inv).reshape(B, L, D)
        if a is None:
            gate, slope = torch.ones_like(x), None
        else:
            sig, rest = torch.sigmoid(a), torch.sigmoid(-a)
            gate, slope = (sig, sig * rest) if case["gate"] == "sigmoid" else (a * sig, sig * (1 + a * rest))
        x_out = x + c * gate * w * y0
        m = (x_out.square().mean(-1, keepdim=True) + EPS).rsqrt()
        return inv, y0, gate, slope, x_out, m

    acts = [s["o"].double().permute(0, 2, 1, 3).reshape(B, L, D), None if s["a"] is None else s["a"].double(), s["x"].double()]
    *_, x_out, m = forward(*acts)
    out = {"x_out": x_out}
    if case["pre"]:
        out["n"] = x_out * m * wp
    inv, y0, gate, slope, x_out, m = forward(*[None if t is None else _exact_packed(t) for t in acts])
    dx = s["d_x_out"].double()
    if case["pre"]:
        dn = s["d_n"].double()
        unit = x_out * m
        dh = dn * wp
        d_pre = (dn * unit).sum((0, 1))
        dx = dx + m * (dh - unit * (dh * unit).mean(-1, keepdim=True))
    dy = (dx * c * gate * w).reshape(B, L, H, d)
    yh = y0.reshape(B, L, H, d)
    out["d_o"] = (inv * (dy - yh * (dy * yh).mean(-1, keepdim=True))).permute(0, 2, 1, 3)
    out["d_x"] = dx
    if slope is not None:
        out["d_a"] = dx * c * w * y0 * slope
    out["d_w_post"] = (dx * c * gate * y0).sum((0, 1))
    out["d_res_scale"] = (dx * gate * w * y0).sum((0, 1))
    if case["pre"]:
        out["d_w_pre"] = d_pre
    return out


def exact(case, seed):
    s = prepare(case, seed)
    with torch.no_grad():
        if case["op"] == "pack":
            return {"back": _exact_packed(s["x"])}
        return _exact_join(s) if case["op"] == "join_train" else _exact_scan(s)
