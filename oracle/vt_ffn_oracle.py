"""fp64 definition of the gated feed-forward block and of its backward pass (numpy, no code shared with the library).

    g = x Wg^T     u = x Wu^T     a = act(g) u     y = a Wd^T
    da = dy Wd     du = da act(g)     dg = da u act'(g)     dx = dg Wg + du Wu     dWg = dg^T x     dWu = du^T x     dWd = dy^T a"""
from __future__ import annotations

import numpy as np


def act(g: np.ndarray, kind: str) -> np.ndarray:
    if kind == "silu":
        return g / (1.0 + np.exp(-g))
    return 0.5 * g * (1.0 + np.tanh(np.sqrt(2.0 / np.pi) * (g + 0.044715 * g ** 3)))


def act_slope(g: np.ndarray, kind: str) -> np.ndarray:
    if kind == "silu":
        s = 1.0 / (1.0 + np.exp(-g))
        return s + g * s * (1.0 - s)
    t = np.tanh(np.sqrt(2.0 / np.pi) * (g + 0.044715 * g ** 3))
    return 0.5 * (1.0 + t) + 0.5 * g * (1.0 - t * t) * np.sqrt(2.0 / np.pi) * (1.0 + 3 * 0.044715 * g * g)


def forward(x, Wg, Wu, Wd, kind: str) -> dict:
    x, Wg, Wu, Wd = (np.asarray(t, np.float64) for t in (x, Wg, Wu, Wd))
    g, u = x @ Wg.T, x @ Wu.T
    a = act(g, kind) * u
    return {"g": g, "u": u, "a": a, "y": a @ Wd.T}


def backward(x, Wg, Wu, Wd, dy, kind: str) -> dict:
    x, Wg, Wu, Wd, dy = (np.asarray(t, np.float64) for t in (x, Wg, Wu, Wd, dy))
    f = forward(x, Wg, Wu, Wd, kind)
    da = dy @ Wd
    du, dg = da * act(f["g"], kind), da * f["u"] * act_slope(f["g"], kind)
    return {"da": da, "dg": dg, "du": du, "grad_x": dg @ Wg + du @ Wu, "grad_W_gate": dg.T @ x, "grad_W_up": du.T @ x,
            "grad_W_down": dy.T @ f["a"]}
