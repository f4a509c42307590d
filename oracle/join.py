"""Block join in fp64 and its adjoint: test infrastructure."""
from __future__ import annotations

import numpy as np


def _gate(a, kind):
    if kind == "none":
        return 1.0, 0.0
    sig = 1.0 / (1.0 + np.exp(-a))
    return (sig, sig * (1 - sig)) if kind == "sigmoid" else (a * sig, sig * (1 + a * (1 - sig)))


def _parts(o, a, x, w_post, res_scale, kind, eps):
    B, H, L, d = o.shape
    yh = np.moveaxis(o, 1, 2)
    inv = 1 / np.sqrt((yh ** 2).mean(-1, keepdims=True) + eps)
    y0 = (yh * inv).reshape(B, L, H * d)
    g, dg = _gate(a, kind)
    return y0, inv, g, dg, x + res_scale * g * w_post * y0


def forward(o, a, x, w_post, res_scale, w_pre, kind, post_eps, pre_eps):
    o, x, w_post, res_scale = (np.asarray(t, np.float64) for t in (o, x, w_post, res_scale))
    a = None if a is None else np.asarray(a, np.float64)
    x_out = _parts(o, a, x, w_post, res_scale, kind, post_eps)[-1]
    if w_pre is None:
        return x_out, None
    return x_out, x_out / np.sqrt((x_out ** 2).mean(-1, keepdims=True) + pre_eps) * np.asarray(w_pre, np.float64)


def backward(o, a, x, w_post, res_scale, w_pre, kind, post_eps, pre_eps, d_x_out, d_n, terms=False):
    """terms: also the magnitudes of the two terms whose difference d_o is."""
    o, x, w_post, res_scale, dx = (np.asarray(t, np.float64) for t in (o, x, w_post, res_scale, d_x_out))
    a = None if a is None else np.asarray(a, np.float64)
    B, H, L, d = o.shape
    y0, inv, g, dg, x_out = _parts(o, a, x, w_post, res_scale, kind, post_eps)
    out = {}
    if w_pre is not None:
        w_pre, d_n = np.asarray(w_pre, np.float64), np.asarray(d_n, np.float64)
        m = 1 / np.sqrt((x_out ** 2).mean(-1, keepdims=True) + pre_eps)
        h, dh = x_out * m, d_n * w_pre
        out["d_w_pre"] = (d_n * h).sum((0, 1))
        dx = dx + m * (dh - h * (dh * h).mean(-1, keepdims=True))
    out["d_x"] = dx
    out["d_res_scale"] = (dx * g * w_post * y0).sum((0, 1))
    out["d_w_post"] = (dx * res_scale * g * y0).sum((0, 1))
    if a is not None:
        out["d_a"] = dx * res_scale * w_post * y0 * dg
    dy, yh = (dx * res_scale * g * w_post).reshape(B, L, H, d), y0.reshape(B, L, H, d)
    along = yh * (dy * yh).mean(-1, keepdims=True)
    out["d_o"] = np.moveaxis(inv * (dy - along), 2, 1)
    return (out, {"d_o": np.moveaxis(inv * (np.abs(dy) + np.abs(along)), 2, 1)}) if terms else out
