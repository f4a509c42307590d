"""Gated linear recurrence in fp64, token by token, and its adjoint: test infrastructure."""
from __future__ import annotations

import numpy as np


def _sigmoid(x):
    e = np.exp(-np.abs(x))
    return np.where(x > 0, 1 / (1 + e), e / (1 + e))


def _gates(x, r, g, rate, starts, unit):
    x, r, rate = (np.asarray(t, np.float64) for t in (x, r, rate))
    la = -rate * _sigmoid(r)
    a = np.exp(la)
    s = np.sqrt(-np.expm1(2 * la)) if unit else np.ones_like(x)
    i = np.ones_like(x) if g is None else _sigmoid(np.asarray(g, np.float64))
    if starts is not None:
        first = np.asarray(starts)[..., None] != 0
        a, s = np.where(first, 0.0, a), np.where(first, 1.0, s)
    return x, la, a, s, i


def _walk(a, b, h0, known=None):
    """The state before every token and the last one; every 64th is taken from `known` where there is one."""
    before, h = np.empty_like(b), h0
    for t in range(b.shape[1]):
        if known is not None and t % 64 == 0:
            h = known[:, t]
        before[:, t] = h
        h = np.where(a[:, t] == 0, 0.0, a[:, t] * h) + b[:, t]  # a document's first token forgets a NaN too
    return before, h


def forward(x, r, g, rate, starts, h0, unit):
    """(h, h_final, magnitude of h's terms)"""
    x, _, a, s, i = _gates(x, r, g, rate, starts, unit)
    h0 = np.zeros_like(x[:, 0]) if h0 is None else np.asarray(h0, np.float64)
    before, last = _walk(a, s * i * x, h0)
    mag, big = _walk(a, np.abs(s * i * x), np.abs(h0))
    after = lambda t, end: np.concatenate([t[:, 1:], end[:, None]], 1)  # noqa: E731
    return after(before, last), last, after(mag, big)


def backward(x, r, g, rate, starts, h0, unit, d_h, dh_final, kept=None):
    """kept: the inputs as the reverse pass reads them, (x, r, g), where that is not what the forward read.  Returns the gradients and the magnitudes of the terms that
    each of them is a sum of."""
    h0 = np.zeros_like(np.asarray(x, np.float64)[:, 0]) if h0 is None else np.asarray(h0, np.float64)
    x_, la, a, s, i = _gates(x, r, g, rate, starts, unit)
    before, _ = _walk(a, s * i * x_, h0)
    mag, _ = _walk(a, np.abs(s * i * x_), np.abs(h0))
    if kept is not None:
        x, r, g = kept
        x_, la, a, s, i = _gates(x, r, g, rate, starts, unit)
        before, _ = _walk(a, s * i * x_, h0, before)
        mag, _ = _walk(a, np.abs(s * i * x_), np.abs(h0), mag)
    x, r = x_, np.asarray(r, np.float64)
    L = x.shape[1]
    d_h = np.asarray(d_h, np.float64)
    end = np.zeros_like(h0) if dh_final is None else np.asarray(dh_final, np.float64)

    def adjoint(d, v):
        lam = np.empty_like(d)
        for t in range(L - 1, -1, -1):
            lam[:, t] = d[:, t] + v
            v = np.where(a[:, t] == 0, 0.0, a[:, t] * lam[:, t])
        return lam, v

    lam, d0 = adjoint(d_h, end)
    big, big0 = adjoint(np.abs(d_h), np.abs(end))
    u = i * x
    with np.errstate(divide="ignore", invalid="ignore"):
        through_s = np.where(s > 0, a * u / s, 0.0) if unit else np.zeros_like(x)
    first = np.zeros(x.shape[:2] + (1,), bool) if starts is None else np.asarray(starts)[..., None] != 0
    before, mag = np.where(first, 0.0, before), np.where(first, 0.0, mag)
    dla = np.where(first, 0.0, a * lam * (before - through_s))
    dla_big = np.where(first, 0.0, a * big * (mag + np.abs(through_s)))
    sg, rest = _sigmoid(r), _sigmoid(-r)
    out = {"d_x": lam * s * i, "da_decay": dla * la * rest, "d_rate": -(dla * sg).sum((0, 1)), "dh_init": d0}
    terms = {"d_x": big * s * i, "da_decay": dla_big * np.abs(la) * rest, "d_rate": (dla_big * sg).sum((0, 1)), "dh_init": big0}
    if g is not None:
        closed = _sigmoid(-np.asarray(g, np.float64))
        out["da_in"], terms["da_in"] = lam * s * u * closed, big * s * np.abs(u) * closed
    return out, terms
