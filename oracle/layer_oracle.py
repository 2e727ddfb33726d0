"""Plain fp64 CPU oracle of the position-wise operators around the attention.

TEST INFRASTRUCTURE.  Only ``tests/`` may import, call or time this module.  It
shares no code with the HIP path.

* ``rms_norm``: the residual's addition and the root-mean-square norm.
* ``e4m3``: values of the OCP 8-bit float, round to nearest even, by their grid.
* ``linear``: the matrix product with scales, bias, activation and residual.
"""
from __future__ import annotations

import math

import numpy as np

__all__ = ["rms_norm", "e4m3", "linear"]

E4M3_MAX = 448.0
TINY = 2.0 ** -96


def rms_norm(x, weight, eps, residual=None):
    """(h, y): h = x + residual, y = h / sqrt(mean(h^2) + eps) * weight."""
    h = np.asarray(x, dtype=np.float64)
    if residual is not None:
        h = h + np.asarray(residual, dtype=np.float64)
    ms = (h * h).sum(axis=-1, keepdims=True) / h.shape[-1]
    return h, h / np.sqrt(ms + eps) * np.asarray(weight, dtype=np.float64)


def e4m3(v) -> np.ndarray:
    """v rounded to e4m3: steps of 2^(e-3) in [2^e, 2^(e+1)), of 2^-9 below 2^-6."""
    v = np.asarray(v, dtype=np.float64)
    a = np.abs(v)
    e = np.floor(np.log2(np.maximum(a, 2.0 ** -6)))
    step = 2.0 ** (e - 3)
    q = np.minimum(np.rint(a / step) * step, E4M3_MAX)     # rint: ties to even
    return np.copysign(q, v)


def linear(x, w, bias=None, act="none", residual=None, x_scale=None, w_scale=None) -> np.ndarray:
    """act(x_scale w_scale (x w^T) + bias) + residual; x [R, K], w [N, K]."""
    y = np.asarray(x, dtype=np.float64) @ np.asarray(w, dtype=np.float64).T
    if x_scale is not None:
        y = y * np.asarray(x_scale, dtype=np.float64)[:, None]
    if w_scale is not None:
        y = y * np.asarray(w_scale, dtype=np.float64)[None, :]
    if bias is not None:
        y = y + np.asarray(bias, dtype=np.float64)
    if act == "relu":
        y = np.maximum(y, 0.0)
    elif act == "gelu":
        y = 0.5 * y * (1.0 + np.vectorize(math.erf)(y / math.sqrt(2.0))) if y.size else y
    elif act == "silu":
        with np.errstate(over="ignore"):
            y = y / (1.0 + np.exp(-y))
    elif act != "none":
        raise ValueError(act)
    return y if residual is None else y + np.asarray(residual, dtype=np.float64)
