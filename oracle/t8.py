"""Oracle of the 8-bit layers with a scale for each token (the reference of include/qc_t8.h): numpy, float64.
Quantiser decisions are float32 divisions rounded half to even, as elsewhere in this package."""
from __future__ import annotations

import numpy as np

F32 = np.float32


def act(name: str, v):
    """(value, derivative) of the gates' activations: v times the logistic function of v, or of 2 y = 2 sqrt(2 / pi) (v + 0.044715 v^3), which is
    (1 + tanh(y)) / 2 and, other than that, keeps its digits where it is small."""
    v = np.asarray(v, dtype=np.float64)
    c = 2 * np.sqrt(2 / np.pi)
    with np.errstate(over="ignore"):
        t, slope = (v, np.ones_like(v)) if name == "silu" else (c * (v + 0.044715 * v ** 3), c * (1 + 3 * 0.044715 * v ** 2))
        z = np.exp(-np.abs(t))
        s, o = np.where(t >= 0, 1, z) / (1 + z), np.where(t >= 0, z, 1) / (1 + z)
        return v * s, s + v * slope * s * o


def codes(v):
    """(codes int64 [M, K], scale float32 [M]) of float32 rows; a row that is not finite: zeros and NaN."""
    v = np.asarray(v, dtype=F32)
    with np.errstate(all="ignore"):
        top = np.abs(v).max(1)
        bad = ~np.isfinite(top)
        scale = (top / F32(127)).astype(F32)
        scale = np.where(scale == 0, F32(1), scale)
        q = np.clip(np.rint(v / scale[:, None]), -127, 127)
    q[bad] = 0
    return q.astype(np.int64), np.where(bad, F32("nan"), scale).astype(F32)


def rho(h, eps):
    """float64."""
    h = np.asarray(h, np.float64)
    return 1 / np.sqrt((h * h).mean(1) + np.float64(F32(eps)))


def norm(h, weight, eps):
    """The float32 rows that are quantised: two float32 products."""
    with np.errstate(all="ignore"):
        y = np.asarray(h, F32) * rho(h, eps).astype(F32)[:, None]
        return y if weight is None else y * np.asarray(weight, F32)


def norm_grad(h, weight, eps, dy, dh=None):
    """(dx, dweight), float64."""
    h, dy = np.asarray(h, np.float64), np.asarray(dy, np.float64)
    r = rho(h, eps)[:, None]
    g = dy if weight is None else dy * np.asarray(weight, np.float64)
    dx = r * (g - h * r * r * (g * h).mean(1, keepdims=True))
    return dx if dh is None else dx + np.asarray(dh, np.float64), (dy * h * r).sum(0)


def gated(x, gate, name):
    """The float32 rows that are quantised."""
    with np.errstate(all="ignore"):
        return (act(name, gate)[0] * np.asarray(x, np.float64)).astype(F32)


def gated_grad(x, gate, name, dv):
    a, d = act(name, gate)
    return dv * a, dv * np.asarray(x, np.float64) * d


def linear(qx, xs, qw, ws, bias=None):
    """The sums are whole numbers below 2^53: exact."""
    y = (np.asarray(qx, np.float64) @ np.asarray(qw, np.float64).T) * (np.asarray(xs, np.float64)[:, None] * np.asarray(ws, np.float64))
    return y if bias is None else y + np.asarray(bias, np.float64)


def linear_grad(dy, qw, ws):
    return (np.asarray(dy, np.float64) * np.asarray(ws, np.float64)) @ np.asarray(qw, np.float64)
