"""Gated delta rule in fp64, token by token, and its adjoint: test infrastructure, no code shared with the GPU path."""
from __future__ import annotations

import numpy as np


def magnitudes(q, k, v, eta, log_gamma, S, scale):
    """Sums of the magnitudes of an output's terms: what the start state, and every token's update, put into it."""
    q, k, v, eta, log_gamma = (np.asarray(x, np.float64) for x in (q, k, v, eta, log_gamma))
    B, H, L, dv = v.shape
    r = H // q.shape[1]
    q, k = np.repeat(q, r, 1), np.repeat(k, r, 1)
    S = np.zeros((B, H, dv, q.shape[-1])) if S is None else np.array(S, np.float64)
    A, o = np.abs(S), np.zeros_like(v)
    for t in range(L):
        g = np.exp(log_gamma[:, :, t])[..., None, None]
        S, A = g * S, g * A
        e = v[:, :, t] - np.einsum("bhij,bhj->bhi", S, k[:, :, t])
        step = (eta[:, :, t, None] * e)[..., :, None] * k[:, :, t, None, :]
        S, A = S + step, A + np.abs(step)
        o[:, :, t] = abs(scale) * np.einsum("bhij,bhj->bhi", A, np.abs(q[:, :, t]))
    return o


def forward(q, k, v, eta, log_gamma, S, scale):
    """q, k [B,Hk,L,dk], v [B,H,L,dv], eta, log_gamma [B,H,L], S [B,H,dv,dk] or None -> o, S_final (all fp64)."""
    q, k, v, eta, log_gamma = (np.asarray(x, np.float64) for x in (q, k, v, eta, log_gamma))
    B, H, L, dv = v.shape
    r = H // q.shape[1]
    q, k = np.repeat(q, r, 1), np.repeat(k, r, 1)
    S = np.zeros((B, H, dv, q.shape[-1])) if S is None else np.array(S, np.float64)
    o = np.zeros_like(v)
    for t in range(L):
        S = np.exp(log_gamma[:, :, t])[..., None, None] * S
        e = v[:, :, t] - np.einsum("bhij,bhj->bhi", S, k[:, :, t])
        S = S + (eta[:, :, t, None] * e)[..., :, None] * k[:, :, t, None, :]
        o[:, :, t] = scale * np.einsum("bhij,bhj->bhi", S, q[:, :, t])
    return o, S


def backward(q, k, v, eta, log_gamma, S, scale, d_o, dS_final):
    """Adjoints of q, k, v, eta, log_gamma and the start state, from those of o and the final state (None: zeros)."""
    q0, k0, v, eta, log_gamma, d_o = (np.asarray(x, np.float64) for x in (q, k, v, eta, log_gamma, d_o))
    B, H, L, dv = v.shape
    Hk, dk = q0.shape[1], q0.shape[-1]
    r = H // Hk
    q, k = np.repeat(q0, r, 1), np.repeat(k0, r, 1)
    S = np.zeros((B, H, dv, dk)) if S is None else np.array(S, np.float64)
    decayed, after, es = [], [], []
    for t in range(L):
        Sp = np.exp(log_gamma[:, :, t])[..., None, None] * S
        e = v[:, :, t] - np.einsum("bhij,bhj->bhi", Sp, k[:, :, t])
        S = Sp + (eta[:, :, t, None] * e)[..., :, None] * k[:, :, t, None, :]
        decayed.append(Sp), after.append(S), es.append(e)
    X = np.zeros((B, H, dv, dk)) if dS_final is None else np.array(dS_final, np.float64)
    dq, d_k, d_v = np.zeros_like(q), np.zeros_like(k), np.zeros_like(v)
    d_eta, d_lg = np.zeros_like(eta), np.zeros_like(eta)
    for t in range(L - 1, -1, -1):
        dq[:, :, t] = scale * np.einsum("bhi,bhij->bhj", d_o[:, :, t], after[t])
        X = X + scale * d_o[:, :, t, :, None] * q[:, :, t, None, :]
        Xk = np.einsum("bhij,bhj->bhi", X, k[:, :, t])
        d_eta[:, :, t] = (es[t] * Xk).sum(-1)
        de = eta[:, :, t, None] * Xk
        d_k[:, :, t] = np.einsum("bhi,bhij->bhj", eta[:, :, t, None] * es[t], X) - np.einsum("bhi,bhij->bhj", de, decayed[t])
        d_v[:, :, t] = de
        X = X - de[..., :, None] * k[:, :, t, None, :]
        d_lg[:, :, t] = (X * decayed[t]).sum((-1, -2))
        X = np.exp(log_gamma[:, :, t])[..., None, None] * X
    group = lambda x: x.reshape(B, Hk, r, L, dk).sum(2)  # noqa: E731
    return {"dq": group(dq), "dk": group(d_k), "dv": d_v, "d_eta": d_eta, "d_log_gamma": d_lg, "dS": X}


def gradient_magnitudes(q, k, v, eta, log_gamma, S, scale, d_o, dS_final):
    """Sums of the magnitudes of the terms of dq and dk: every token's part in the state and in its adjoint with its magnitude."""
    de = np.abs(backward(q, k, v, eta, log_gamma, S, scale, d_o, dS_final)["dv"])
    q, k, v, eta, log_gamma, d_o = (np.asarray(x, np.float64) for x in (q, k, v, eta, log_gamma, d_o))
    B, H, L, dv = v.shape
    Hk, dk = q.shape[1], q.shape[-1]
    r = H // Hk
    q, k, scale, d_o = np.abs(np.repeat(q, r, 1)), np.repeat(k, r, 1), abs(scale), np.abs(d_o)
    S = np.zeros((B, H, dv, dk)) if S is None else np.array(S, np.float64)
    A, decayed, after, us = np.abs(S), [], [], []
    for t in range(L):
        g = np.exp(log_gamma[:, :, t])[..., None, None]
        S, A = g * S, g * A
        u = eta[:, :, t, None] * (v[:, :, t] - np.einsum("bhij,bhj->bhi", S, k[:, :, t]))
        step = u[..., :, None] * k[:, :, t, None, :]
        decayed.append(A)
        S, A = S + step, A + np.abs(step)
        after.append(A), us.append(np.abs(u))
    X = np.zeros((B, H, dv, dk)) if dS_final is None else np.abs(np.array(dS_final, np.float64))
    dq, d_k = np.zeros_like(q), np.zeros_like(k)
    for t in range(L - 1, -1, -1):
        dq[:, :, t] = scale * np.einsum("bhi,bhij->bhj", d_o[:, :, t], after[t])
        X = X + scale * d_o[:, :, t, :, None] * q[:, :, t, None, :]
        d_k[:, :, t] = np.einsum("bhi,bhij->bhj", us[t], X) + np.einsum("bhi,bhij->bhj", de[:, :, t], decayed[t])
        X = np.exp(log_gamma[:, :, t])[..., None, None] * (X + de[:, :, t, :, None] * np.abs(k[:, :, t, None, :]))
    return {"dq": dq.reshape(B, Hk, r, L, dk).sum(2), "dk": d_k.reshape(B, Hk, r, L, dk).sum(2)}
