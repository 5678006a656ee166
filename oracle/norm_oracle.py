"""fp64 CPU oracle of the residual stream and norms between two blocks.  TEST INFRASTRUCTURE ONLY.

    N = norm(Y; gamma_post),  H = X + s gate_j N,  Xn = norm(H; gamma_pre),     norm(V; g) = V / sqrt(mean(V^2) + eps) g

and the derivative of L = sum(dH * H) + sum(dXn * Xn), token by token: with V^ = V rstd and G = dnorm * g,
dV = rstd (G - V^ mean(G V^)).  None stands for: no norm (gammas), ones (gates), zeros (X, dH, dXn).
Pinned by tests/test_step_pins.py: torch autograd in float64, central differences."""
from __future__ import annotations

import numpy as np


def _hat(V, eps):
    r = 1.0 / np.sqrt(np.mean(V * V, axis=1, keepdims=True) + eps)
    return V * r, r


def _gates(gates, offsets, T, d):
    G = np.ones((T, d))
    if gates is not None:
        for j, (a, b) in enumerate(zip(offsets[:-1], offsets[1:])):
            if gates[j] is not None:
                G[a:b] = gates[j]
    return G


def forward(X, Y, offsets, eps, s=1.0, gamma_post=None, gamma_pre=None, gates=None):
    Y = np.asarray(Y, dtype=np.float64)
    T, d = Y.shape
    N = Y if gamma_post is None else _hat(Y, eps)[0] * gamma_post
    H = (0.0 if X is None else np.asarray(X, dtype=np.float64)) + s * _gates(gates, offsets, T, d) * N
    return H, None if gamma_pre is None else _hat(H, eps)[0] * gamma_pre


def backward(X, Y, offsets, eps, dH, dXn, s=1.0, gamma_post=None, gamma_pre=None, gates=None):
    """dict of dX, dY, dgamma_post, dgamma_pre, dgates and, under "abs_" names, the sums of the absolute terms of each."""
    Y = np.asarray(Y, dtype=np.float64)
    T, d = Y.shape
    G = _gates(gates, offsets, T, d)
    H, _ = forward(X, Y, offsets, eps, s, gamma_post, gamma_pre, gates)
    D = np.zeros((T, d)) if dH is None else np.asarray(dH, dtype=np.float64).copy()
    aD = np.abs(D)
    out = {}
    if dXn is not None:
        dXn = np.asarray(dXn, dtype=np.float64)
        Hh, r2 = _hat(H, eps)
        g = dXn * gamma_pre
        D += r2 * (g - Hh * np.mean(g * Hh, axis=1, keepdims=True))
        aD += r2 * (np.abs(g) + np.abs(Hh) * np.mean(np.abs(g * Hh), axis=1, keepdims=True))
        out["dgamma_pre"], out["abs_dgamma_pre"] = (dXn * Hh).sum(axis=0), np.abs(dXn * Hh).sum(axis=0)
    elif gamma_pre is not None:
        out["dgamma_pre"] = out["abs_dgamma_pre"] = np.zeros(d)
    dN, adN = s * G * D, np.abs(s * G) * aD
    out["dX"], out["abs_dX"] = D, aD
    if gamma_post is None:
        N = Y
        out["dY"], out["abs_dY"] = dN, adN
    else:
        Yh, r1 = _hat(Y, eps)
        N = Yh * gamma_post
        g, ag = dN * gamma_post, adN * np.abs(gamma_post)
        out["dY"] = r1 * (g - Yh * np.mean(g * Yh, axis=1, keepdims=True))
        out["abs_dY"] = r1 * (ag + np.abs(Yh) * np.mean(ag * np.abs(Yh), axis=1, keepdims=True))
        out["dgamma_post"], out["abs_dgamma_post"] = (dN * Yh).sum(axis=0), (adN * np.abs(Yh)).sum(axis=0)
    seg = list(zip(offsets[:-1], offsets[1:]))
    out["dgates"] = [(s * D * N)[a:b].sum(axis=0) for a, b in seg]
    out["abs_dgates"] = [(abs(s) * aD * np.abs(N))[a:b].sum(axis=0) for a, b in seg]
    return out
