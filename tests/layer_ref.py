"""The formulas around the attention of a layer in 64 bits, on the CPU: rotary
tables, rotation, the norms of queries and keys, and their gradients, written
straight from their definitions; and the error that float32 arithmetic on them
may have."""
from __future__ import annotations

import math

import numpy as np

# half a step of a type, relative to the value
HALF = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}
F32 = 2.0 ** -24


def table(pos, dims, theta=10000.0, scaling="none", factor=1.0, orig_len=0.0, fast=32.0, slow=1.0, magnitude=1.0):
    """cos, sin [N, sum(dims) / 2] of positions [N, len(dims)]."""
    pos = np.asarray(pos, np.float64)
    cols = []
    for a, dim in enumerate(dims):
        th = theta * factor ** (dim / (dim - 2)) if scaling == "ntk" else theta
        for i in range(dim // 2):
            w = th ** (-2.0 * i / dim)
            if scaling == "linear":
                w /= factor
            elif scaling == "ramp":
                t = (orig_len * w / (2 * math.pi) - slow) / (fast - slow)
                t = min(1.0, max(0.0, t))
                w = w * t + w / factor * (1 - t)
            cols.append(pos[:, a] * w)
    ang = np.stack(cols, 1)
    return np.cos(ang) * magnitude, np.sin(ang) * magnitude


def rotate(x, cos, sin, layout, transpose=False):
    """x [B, N, H, d]; cos, sin [N, r] or [B, N, r]."""
    if cos is None:
        return x.copy()
    r = cos.shape[-1]
    c, s = np.asarray(cos, np.float64), np.asarray(sin, np.float64)
    if c.ndim == 2:
        c, s = c[None], s[None]
    c, s = c[:, :, None], (-s if transpose else s)[:, :, None]
    y = x.copy()
    for i in range(r):
        a, b = (2 * i, 2 * i + 1) if layout == "interleaved" else (i, r + i)
        y[..., a] = x[..., a] * c[..., i] - x[..., b] * s[..., i]
        y[..., b] = x[..., b] * c[..., i] + x[..., a] * s[..., i]
    return y


def normalised(x, norm, eps):
    """(n, 1 / deviation), the second with a last dim of 1."""
    if norm == "layer":
        x = x - x.mean(-1, keepdims=True)
    r = 1.0 / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
    return x * r, r


def forward(x, w, b, cos, sin, norm, eps, layout):
    n, _ = normalised(x, norm, eps)
    y = n * (1.0 if w is None else w) + (0.0 if b is None else b)
    return rotate(y, cos, sin, layout)


def forward_scale(x, w, b, norm, eps):
    """What the error of a float32 result is in proportion to, per head: the
    normalised values before any cancellation (the mean's subtraction, the
    pair's sum)."""
    _, r = normalised(x, norm, eps)
    w = 1.0 if w is None else np.abs(w).max()
    b = 0.0 if b is None else np.abs(b).max()
    return 2 * (np.abs(x).max(-1, keepdims=True) * r * 2 * w + b)


def backward(x, w, g, cos, sin, norm, eps, layout):
    """dx, dw, db and the scale of dx's error per head."""
    n, r = normalised(x, norm, eps)
    h = rotate(g, cos, sin, layout, transpose=True)
    gw = h if w is None else h * w
    dx = gw - n * (gw * n).mean(-1, keepdims=True)
    if norm == "layer":
        dx = dx - gw.mean(-1, keepdims=True)
    axes = tuple(range(x.ndim - 1))
    gmax = (2 * np.abs(g).max(-1, keepdims=True)) * (1.0 if w is None else np.abs(w).max())
    nmax = 2 * np.abs(x).max(-1, keepdims=True) * r
    scale = r * gmax * (2 + nmax * nmax)
    return dx * r, (h * n).sum(axes), h.sum(axes), scale


def sums_scale(x, g, norm, eps):
    """Sum of the absolute terms of dw and of db (a rotated pair's terms are at
    most both of its elements)."""
    n, _ = normalised(x, norm, eps)
    axes = tuple(range(x.ndim - 1))
    big = 2 * np.abs(g).max(-1, keepdims=True)
    return (big * (np.abs(n) + 2 * np.abs(x).max(-1, keepdims=True) * F32)).sum(axes), (big + 0 * n).sum(axes)
