"""Float64 oracle of the layers around the whitening (norm, gated block, 8-bit product), written from their formulas; no code
shared with the GPU path."""
from __future__ import annotations

import numpy as np
from scipy.special import erf

ACTS = ("silu", "gelu", "gelu_tanh", "relu")


def f64(x):
    return np.asarray(x, dtype=np.float64)


def rms_norm(h, w, eps):
    """Rows of h over their root mean square, times w (or ones)."""
    h = f64(h)
    y = h / np.sqrt(np.mean(h * h, axis=1, keepdims=True) + eps)
    return y if w is None else y * f64(w)


def rms_norm_grad(h, w, eps, dy, dh=None):
    """(gradient with respect to h with that of the residual path added, gradient with respect to w)."""
    h, dy = f64(h), f64(dy)
    rho = 1.0 / np.sqrt(np.mean(h * h, axis=1, keepdims=True) + eps)
    v = dy if w is None else dy * f64(w)
    dx = rho * v - h * rho ** 3 * np.mean(v * h, axis=1, keepdims=True)
    return (dx if dh is None else dx + f64(dh)), np.sum(dy * h * rho, axis=0)


def int8_steps(y):
    """(y in steps of a 127th of its row's largest entry, that step): what the nearest integers are taken of."""
    y = f64(y)
    top = np.max(np.abs(y), axis=1, keepdims=True)
    with np.errstate(invalid="ignore", divide="ignore"):
        steps = np.where(top > 0, y * 127.0 / top, 0.0)
    return steps, top[:, 0] / 127.0


def act(kind, g):
    g = f64(g)
    if kind == "silu":
        return g / (1 + np.exp(-g))
    if kind == "gelu":
        return 0.5 * g * (1 + erf(g / np.sqrt(2)))
    if kind == "gelu_tanh":
        return 0.5 * g * (1 + np.tanh(np.sqrt(2 / np.pi) * (g + 0.044715 * g ** 3)))
    return np.maximum(g, 0.0)


def act_slope(kind, g):
    g = f64(g)
    if kind == "silu":
        s = 1 / (1 + np.exp(-g))
        return s * (1 + g * (1 - s))
    if kind == "gelu":
        return 0.5 * (1 + erf(g / np.sqrt(2))) + g * np.exp(-0.5 * g * g) / np.sqrt(2 * np.pi)
    if kind == "gelu_tanh":
        k = np.sqrt(2 / np.pi)
        t = np.tanh(k * (g + 0.044715 * g ** 3))
        return 0.5 * (1 + t) + 0.5 * g * (1 - t * t) * k * (1 + 3 * 0.044715 * g * g)
    return (g > 0).astype(np.float64)


def projections(X, Wg, Wu, bg=None, bu=None):
    g, u = f64(X) @ f64(Wg).T, f64(X) @ f64(Wu).T
    return (g if bg is None else g + f64(bg)), (u if bu is None else u + f64(bu))


def gated(X, Wg, Wu, kind, bg=None, bu=None):
    g, u = projections(X, Wg, Wu, bg, bu)
    return act(kind, g) * u


def gated_grad_from(dg, du, X, Wg, Wu, mu=None):
    """(dX, dWg, dWu, dbg, dbu) for given gradients of the two projections; weights' gradients of the rows centred on mu."""
    dg, du, Xc = f64(dg), f64(du), f64(X) - (0.0 if mu is None else f64(mu))
    return dg @ f64(Wg) + du @ f64(Wu), dg.T @ Xc, du.T @ Xc, dg.sum(0), du.sum(0)


def gated_grad(X, Wg, Wu, kind, dH, bg=None, bu=None, mu=None):
    g, u = projections(X, Wg, Wu, bg, bu)
    dH = f64(dH)
    return gated_grad_from(dH * u * act_slope(kind, g), dH * act(kind, g), X, Wg, Wu, mu)


def int8_product(Xq, sx, Wq, sw, b=None):
    y = (np.asarray(Xq, dtype=np.int64) @ np.asarray(Wq, dtype=np.int64).T) * f64(sx)[:, None] * f64(sw)
    return y if b is None else y + f64(b)
