"""The 64-bit formulas that the kernels are checked against, against
differences and against facts fixed outside them."""
from __future__ import annotations

import numpy as np
import pytest

from tests import layer_ref as ref


def _inputs(seed, d, rot):
    rng = np.random.default_rng(seed)
    x, g = rng.standard_normal((2, 3, 2, d)), rng.standard_normal((2, 3, 2, d))
    w, b = 1 + 0.3 * rng.standard_normal(d), 0.2 * rng.standard_normal(d)
    cos, sin = ref.table(rng.integers(0, 50, (3, 1)), [rot]) if rot else (None, None)
    return x, g, w, b, cos, sin


@pytest.mark.parametrize("layout", ["interleaved", "half"])
@pytest.mark.parametrize("norm,rot", [("rms", 0), ("rms", 16), ("layer", 8), ("layer", 24)])
def test_gradients_by_differences(norm, rot, layout):
    d, eps, h = 24, 1e-3, 1e-6
    x, g, w, b, cos, sin = _inputs(3, d, rot)
    f = lambda x, w, b: (ref.forward(x, w, b, cos, sin, norm, eps, layout) * g).sum()
    dx, dw, db, _ = ref.backward(x, w, g, cos, sin, norm, eps, layout)
    rng = np.random.default_rng(4)
    for _ in range(20):
        i = tuple(rng.integers(0, n) for n in x.shape)
        e = np.zeros_like(x)
        e[i] = h
        assert abs((f(x + e, w, b) - f(x - e, w, b)) / (2 * h) - dx[i]) < 1e-7
    for j in range(d):
        e = np.zeros(d)
        e[j] = h
        assert abs((f(x, w + e, b) - f(x, w - e, b)) / (2 * h) - dw[j]) < 1e-7
        assert abs((f(x, w, b + e) - f(x, w, b - e)) / (2 * h) - db[j]) < 1e-7


def test_rotation_facts():
    rng = np.random.default_rng(5)
    x = rng.standard_normal((1, 4, 2, 16))
    cos, sin = ref.table(np.arange(4)[:, None], [16])
    for layout in ("interleaved", "half"):
        y = ref.rotate(x, cos, sin, layout)
        assert np.allclose(ref.rotate(y, cos, sin, layout, True), x)          # its transpose undoes it
        assert np.allclose((y ** 2).sum(-1), (x ** 2).sum(-1))                # lengths stay
        assert np.array_equal(y[:, 0], x[:, 0])                              # position 0 turns by nothing
        # products of two rotated rows depend on the distance of their positions
        q = ref.rotate(np.broadcast_to(x[:, :1], x.shape), cos, sin, layout)
        k = ref.rotate(np.broadcast_to(x[:, 1:2], x.shape), cos, sin, layout)
        assert np.allclose((q[:, 1] * k[:, 0]).sum(-1), (q[:, 3] * k[:, 2]).sum(-1))


def test_table_facts():
    pos = np.array([[0, 0], [1, 7], [1000, 3]])
    c, s = ref.table(pos, [8, 4], theta=100.0)
    assert c.shape == (3, 6) and np.allclose(c ** 2 + s ** 2, 1)
    assert np.isclose(c[1, 0], np.cos(1.0)) and np.isclose(s[1, 4], np.sin(7.0)) and np.isclose(s[2, 5], np.sin(0.3))
    # linear: positions divided; ntk: the fastest kept, the slowest divided
    c2, _ = ref.table(pos * 4, [8, 4], theta=100.0, scaling="linear", factor=4.0)
    assert np.allclose(c2, c)
    one = np.array([[1.0]])
    f0, f1 = (np.arctan2(*ref.table(one, [8], 100.0, k, 3.0)[::-1]) for k in ("none", "ntk"))
    assert np.isclose(f1[0, 0], f0[0, 0]) and np.isclose(f1[0, 3], f0[0, 3] / 3)
    # ramp: turns over the original length decide
    f2 = np.arctan2(*ref.table(one, [8], 100.0, "ramp", 3.0, orig_len=100.0, fast=10.0, slow=1.0)[::-1])
    turns = 100.0 * f0 / (2 * np.pi)
    assert np.allclose(f2[turns >= 10], f0[turns >= 10]) and np.allclose(f2[turns <= 1], f0[turns <= 1] / 3)


def test_attention_gradients_by_differences():
    """Of the outputs and of the log-sum-exp, and of a sequence in two chunks."""
    rng = np.random.default_rng(6)
    B, nq, nk, H, d = 1, 3, 5, 2, 8
    q, k, v = rng.standard_normal((B, nq, H, d)), rng.standard_normal((B, nk, H, d)), rng.standard_normal((B, nk, H, d))
    g, e = rng.standard_normal((B, nq, H, d)), rng.standard_normal((B, H, nq))

    def loss(q, k, v):
        o, l = ref.attention(q, k, v)
        return (o * g).sum() + (l * e).sum()

    out, lse = ref.attention(q, k, v)
    got = ref.attention_bwd(q, k, v, out, lse, g, e)
    h = 1e-6
    for x, name, at in ((q, "dq", 0), (k, "dk", 1), (v, "dv", 2)):
        for _ in range(12):
            i = tuple(rng.integers(0, n) for n in x.shape)
            step = np.zeros_like(x)
            step[i] = h
            up, dn = ([*(y + (s * step if j == at else 0) for j, y in enumerate((q, k, v)))] for s in (1, -1))
            assert abs((loss(*up) - loss(*dn)) / (2 * h) - got[name][0][i]) < 1e-7, name
    # chunks with the whole sequence's out and lse: parts of dq add up, dk and dv are the chunks'
    whole = ref.attention_bwd(q, k, v, out, lse, g)
    parts = [ref.attention_bwd(q, k[:, a:b], v[:, a:b], out, lse, g) for a, b in ((0, 2), (2, 5))]
    assert np.allclose(sum(p["dq"][0] for p in parts), whole["dq"][0])
    for n in ("dk", "dv"):
        assert np.allclose(np.concatenate([p[n][0] for p in parts], 1), whole[n][0])
