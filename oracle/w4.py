"""Oracle of the operators on 4-bit weights with a scale per group (the reference of include/qc_w4.h): numpy, float64.
Quantiser decisions are float32 divisions rounded half to even, as elsewhere in this package."""
from __future__ import annotations

import numpy as np

from .quant import pack_w4, unpack_w4

F32 = np.float32


def group_quant(W, group: int, asymmetric: bool):
    """(unsigned codes int64 [N, K], scale float32 [N, G], zero points int64 [N, G]); the last group may be short."""
    W = np.asarray(W, dtype=F32)
    N, K = W.shape
    G = -(-K // group)
    u, scale, zero = np.empty((N, K), np.int64), np.empty((N, G), F32), np.full((N, G), 8, np.int64)
    for g in range(G):
        w = W[:, g * group:(g + 1) * group]
        if asymmetric:
            lo, hi = np.minimum(w.min(1), F32(0)), np.maximum(w.max(1), F32(0))
            s = ((hi - lo) / F32(15)).astype(F32)
        else:
            s = (np.abs(w).max(1) / F32(7)).astype(F32)
        s = np.where(s == 0, F32(1), s)
        if asymmetric:
            zero[:, g] = np.clip(np.rint(-lo / s), 0, 15)
        q = np.rint(w / s[:, None]).astype(np.int64) + zero[:, g:g + 1]
        u[:, g * group:(g + 1) * group] = np.clip(q, 0 if asymmetric else 1, 15)
        scale[:, g] = s
    return u, scale, zero


def values(u, scale, zero, group: int):
    """The matrix the codes stand for, float64."""
    K = u.shape[1]
    full = lambda v: np.repeat(np.asarray(v, dtype=np.float64), group, axis=1)[:, :K]  # noqa: E731
    return (u - full(zero)) * full(scale)


def pack(u):
    return pack_w4(np.asarray(u) - 8)


def unpack(p):
    return unpack_w4(p).astype(np.int64) + 8


def act(name: str, v):
    """(value, derivative) of the gate's activation."""
    v = np.asarray(v, dtype=np.float64)
    if name == "silu":
        e = np.where(v >= 0, 1 / (1 + np.exp(-np.abs(v))), np.exp(-np.abs(v)) / (1 + np.exp(-np.abs(v))))
        return v * e, e + v * e * (1 - e)
    c = np.sqrt(2 / np.pi)
    t = np.tanh(c * (v + 0.044715 * v ** 3))
    return 0.5 * v * (1 + t), 0.5 * (1 + t) + 0.5 * v * (1 - t * t) * c * (1 + 3 * 0.044715 * v ** 2)


def linear(x, W, b=None):
    y = np.asarray(x, np.float64) @ np.asarray(W, np.float64).T
    return y if b is None else y + np.asarray(b, np.float64)


def gated(x, Wg, Wu, bg, bu, name: str):
    return act(name, linear(x, Wg, bg))[0] * linear(x, Wu, bu)


def gated_grad(x, Wg, Wu, bg, bu, name: str, dh):
    a, d = act(name, linear(x, Wg, bg))
    return dh * linear(x, Wu, bu) * d, dh * a
