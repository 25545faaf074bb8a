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


# -- the attention's gradients --------------------------------------------------
def attention(q, k, v):
    """out [B, Nq, H, d] and lse [B, H, Nq] of full attention."""
    qh, kh, vh = (np.moveaxis(x, 2, 1) for x in (q, k, v))
    s = qh @ np.swapaxes(kh, 2, 3) / math.sqrt(q.shape[-1])
    if s.shape[-1] == 0:
        return np.zeros_like(q), np.full(s.shape[:3], -np.inf)
    m = s.max(-1, keepdims=True)
    p = np.exp(s - m)
    t = p.sum(-1, keepdims=True)
    return np.moveaxis(p / t @ vh, 1, 2), (m + np.log(t))[..., 0]


def attention_bwd(q, k, v, out, lse, dout, dlse=None, dtype="bf16"):
    """{name: (gradient, worst error, error's deviation)} of dq, dk, dv.

    The worst error counts, for every term of a gradient's sum, half a step of P
    or dS where they are rounded to the operand type, the float32 error of the
    exponent (a product of d + 4 roundings of the dot product and of
    lse * sqrt(d)) and of dout . v - D, one rounding for every addition of the
    sum, and half a step of the result.  The deviation takes the operands'
    roundings as independent (their squares add) and the rest as they are."""
    qh, kh, vh, oh, gh = (np.moveaxis(np.asarray(x, np.float64), 2, 1) for x in (q, k, v, out, dout))
    d = q.shape[-1]
    scale = 1 / math.sqrt(d)
    T = lambda x: np.swapaxes(x, 2, 3)
    none = np.isneginf(lse)
    lf = np.where(none, 0.0, lse)[..., None]
    alive = ~none[..., None]
    s = qh @ T(kh) * scale
    P = np.where(alive, np.exp(np.where(alive, s - lf, 0.0)), 0.0)
    oh = np.where(alive, oh, 0.0)
    D = (gh * oh).sum(-1, keepdims=True) - (0.0 if dlse is None else np.where(alive, dlse[..., None], 0.0))
    gv = gh @ T(vh)
    S = P * (gv - D)
    op = HALF[dtype] if dtype == "bf16" else 0.0   # rounding of P and dS as operands
    steps = (d + 8) * F32
    eP = steps * (scale * (np.abs(qh) @ T(np.abs(kh))) + np.abs(lf)) + 4 * F32
    eS = P * (steps * (np.abs(gh) @ T(np.abs(vh)) + (np.abs(gh) * np.abs(oh)).sum(-1, keepdims=True)
                       + (0.0 if dlse is None else np.abs(dlse[..., None])))) + np.abs(S) * (eP + 4 * F32)
    eS = np.where(alive, eS, 0.0)
    back = lambda x: np.moveaxis(x, 1, 2)
    res = {}
    for name, W, E, X, f, n in (("dq", S, eS, kh, scale, k.shape[1]), ("dk", T(S), T(eS), qh, scale, q.shape[1]),
                                ("dv", T(P), T(P * eP), gh, 1.0, q.shape[1])):
        want = W @ X * f
        small = (E @ np.abs(X) + (n + 20) * F32 * (np.abs(W) @ np.abs(X))) * f
        worst = small + op * (np.abs(W) @ np.abs(X)) * f + HALF[dtype] * np.abs(want) * 1.01
        dev = small + op * np.sqrt((W * W) @ (X * X)) * f + HALF[dtype] * np.abs(want)
        res[name] = tuple(back(x) for x in (want, worst, dev))
    return res
