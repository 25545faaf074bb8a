"""The stage micro-step with norms and rotation of queries and keys: the bits
of its parts called one after another, and the formulas in 64 bits.

Bounds: a projection is good to half a bf16 step (2^-8) plus float32 sums; the
norm divides by the deviation of values with that error, at most twice it
relative to the largest value of the head, and rounds once more."""
from __future__ import annotations

import math

import numpy as np
import pytest

import paper_2411_01738_amd as xd
from tests import layer_ref as ref
from tests.gpu_util import to_np, torch_mod

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("B,L,N,H,d,C,off,norm,rot,layout", [
    (2, 96, 320, 2, 72, 160, 64, "rms", 72, "half"), (1, 130, 300, 3, 64, 192, 170, "layer", 48, "interleaved"),
    (2, 64, 256, 2, 128, 256, 0, "rms", 0, "interleaved"), (1, 1, 128, 2, 64, 64, 127, "none", 64, "interleaved")])
def test_stage_step_qk(B, L, N, H, d, C, off, norm, rot, layout):
    torch = torch_mod()
    g = torch.Generator().manual_seed(400 + L)
    r = lambda *s, scale=1.0: (torch.randn(*s, generator=g) * scale).bfloat16().cuda()
    x, wo = r(B, L, C), r(H * d, C, scale=1 / math.sqrt(H * d))
    wq, wk, wv = (r(C, H * d, scale=1 / math.sqrt(C)) for _ in range(3))
    kv0 = r(2, B, N, H, d)
    kw = dict(norm=norm, eps=1e-5, layout=layout)
    if norm != "none":
        kw.update(wq=1 + r(d, scale=0.3), wk=1 + r(d, scale=0.3))
    if norm == "layer":
        kw.update(bq=r(d, scale=0.2), bk=r(d, scale=0.2))
    if rot:
        table = [torch.empty(N, rot // 2, device="cuda") for _ in range(2)]
        xd.xdit_rope_table(torch.arange(N, device="cuda")[:, None], [rot], *table)
        kw.update(cos=table[0][off:off + L], sin=table[1][off:off + L])
    stage_kw = {("norm_" + n if n[0] in "wb" else n): v for n, v in kw.items()}

    def buffers():
        return [torch.full((B, L, H, d), float("nan"), device="cuda", dtype=torch.bfloat16) for _ in range(4)] + [
            torch.full((B, L, C), float("nan"), device="cuda", dtype=torch.bfloat16)]

    q, k, v, o, y = buffers()
    kv = kv0.clone()
    xd.xdit_stage_step(x, wq, wk, wv, wo, kv, off, q, k, v, o, y, **stage_kw)
    # its parts: the projections of the plain step, the norms and rotation, the patch step
    q1, k1, v1, o1, y1 = buffers()
    xd.xdit_stage_step(x, wq, wk, wv, wo, kv0.clone(), off, q1, k1, v1, o1, y1)
    raw = q1.clone(), k1.clone()
    xd.xdit_qk_norm_rope(q1, k1, q1, k1, **kw)
    kv1 = kv0.clone()
    xd.xdit_patch_attn(q1, kv1, off, L, k1, v1, o1)
    for a, b in ((q, q1), (k, k1), (v, v1), (o, o1), (kv, kv1)):
        assert torch.equal(a, b)
    # y = o wo as the plain step forms it
    assert np.abs(to_np(y) - to_np(o).reshape(B, L, H * d).astype(np.float64) @ to_np(wo).astype(np.float64)).max() <= 3e-2
    f = lambda t: None if t is None else to_np(t).astype(np.float64)
    c, s = (None, None) if not rot else (kw["cos"].cpu().numpy(), kw["sin"].cpu().numpy())
    for got, w, wn, bn, raw_t in ((q, wq, "wq", "bq", raw[0]), (k, wk, "wk", "bk", raw[1])):
        X = (f(x) @ f(w)).reshape(B, L, H, d)
        W, Bn = f(kw.get(wn)), f(kw.get(bn))
        if norm == "none":
            want, scale = ref.rotate(X, c, s, layout), 2 * np.abs(X).max(-1, keepdims=True)
        else:
            want, scale = ref.forward(X, W, Bn, c, s, norm, 1e-5, layout), ref.forward_scale(X, W, Bn, norm, 1e-5)
        err = np.abs(f(got) - want)
        assert (err <= 2.0 ** -8 * np.abs(want) + 3 * 2.0 ** -8 * scale).all(), err.max()
        assert np.sqrt((err ** 2).mean()) <= 2.0 ** -7 * np.sqrt((want ** 2).mean())


@pytest.mark.parametrize("norm,layout", [("rms", "interleaved"), ("layer", "half"), ("none", "half")])
def test_a_table_per_batch(norm, layout):
    """Each batch at its own positions: the queries and keys of a call per batch
    with that batch's table."""
    torch = torch_mod()
    B, L, N, H, d, C, off = 3, 40, 96, 2, 64, 128, 24
    g = torch.Generator().manual_seed(460)
    r = lambda *s, scale=1.0: (torch.randn(*s, generator=g) * scale).bfloat16().cuda()
    x, kv, wo = r(B, L, C), r(2, B, N, H, d), r(H * d, C, scale=0.1)
    wq, wk, wv = (r(C, H * d, scale=C ** -0.5) for _ in range(3))
    cos, sin = (torch.empty(B, L, d // 2, device="cuda") for _ in range(2))
    for b in range(B):
        xd.xdit_rope_table(torch.arange(L, device="cuda")[:, None] + 1000 * b + off, [d], cos[b], sin[b])
    w = dict(wq=1 + r(d, scale=0.3), wk=1 + r(d, scale=0.3)) if norm != "none" else {}
    new = lambda *s: torch.full(s, float("nan"), device="cuda", dtype=torch.bfloat16)
    q, k, v, o = (new(B, L, H, d) for _ in range(4))
    y = new(B, L, C)
    got_kv = kv.clone()
    xd.xdit_stage_step(x, wq, wk, wv, wo, got_kv, off, q, k, v, o, y, norm=norm, cos=cos, sin=sin, layout=layout,
                       **{"norm_" + n: t for n, t in w.items()})
    # the projections of the plain step, then batch by batch
    q1, k1, v1, o1 = (new(B, L, H, d) for _ in range(4))
    xd.xdit_stage_step(x, wq, wk, wv, wo, kv.clone(), off, q1, k1, v1, o1, new(B, L, C))
    for b in range(B):
        xd.xdit_qk_norm_rope(q1[b:b + 1], k1[b:b + 1], q1[b:b + 1], k1[b:b + 1], norm=norm, cos=cos[b], sin=sin[b], layout=layout, **w)
    assert torch.equal(q, q1) and torch.equal(k, k1) and not torch.equal(q[0], q[1])
    want_kv = kv.clone()
    xd.xdit_patch_attn(q1, want_kv, off, L, k1, v1, o1)
    assert torch.equal(o, o1) and torch.equal(got_kv, want_kv) and torch.isfinite(y).all()


def test_stream_and_graph():
    """On a stream of its own, and captured and replayed with other inputs: the
    bits of the eager call."""
    torch = torch_mod()
    B, L, N, H, d, C, off = 2, 64, 160, 2, 72, 128, 48
    g = torch.Generator().manual_seed(470)
    r = lambda *s, scale=1.0: (torch.randn(*s, generator=g) * scale).bfloat16().cuda()
    x, kv0, wo, w = r(B, L, C), r(2, B, N, H, d), r(H * d, C, scale=0.1), 1 + r(d, scale=0.3)
    wq, wk, wv = (r(C, H * d, scale=C ** -0.5) for _ in range(3))
    cos, sin = (torch.empty(L, d // 2, device="cuda") for _ in range(2))
    xd.xdit_rope_table(torch.arange(L, device="cuda")[:, None] + off, [d], cos, sin)

    def buffers():
        return [kv0.clone(), *(torch.zeros(B, L, H, d, device="cuda", dtype=torch.bfloat16) for _ in range(4)),
                torch.zeros(B, L, C, device="cuda", dtype=torch.bfloat16)]

    def call(b):
        xd.xdit_stage_step(x, wq, wk, wv, wo, b[0], off, *b[1:], norm="rms", norm_wq=w, norm_wk=w, cos=cos, sin=sin, layout="half")

    eager, side, cap = buffers(), buffers(), buffers()
    call(eager)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        call(side)
    torch.cuda.current_stream().wait_stream(s)
    for a, b in zip(eager, side):
        assert torch.equal(a, b)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(cap)
    for i in range(4):
        x.copy_(r(B, L, C))
        w.copy_(1 + r(d, scale=0.3))
        graph.replay()
        call(eager)
        torch.cuda.synchronize()
        for a, b in zip(eager, cap):
            assert torch.equal(a, b), f"replay {i}"


def test_refusals():
    torch = torch_mod()
    z = lambda *s, dt=torch.bfloat16: torch.zeros(*s, device="cuda", dtype=dt)
    B, L, N, H, d, C = 1, 8, 16, 2, 64, 64
    x, w, wo, kv, y = z(B, L, C), z(C, H * d), z(H * d, C), z(2, B, N, H, d), z(B, L, C)
    q, k, v, o = (z(B, L, H, d) for _ in range(4))
    t = z(L, 32, dt=torch.float32)
    step = lambda **kw: xd.xdit_stage_step(x, w, w, w, wo, kv, 4, q, k, v, o, y, **kw)
    for kw in (dict(norm="other"), dict(norm="rms", norm_bq=z(d)), dict(norm_wq=z(d)), dict(norm="rms", cos=t), dict(cos=t[:4], sin=t[:4]),
               dict(norm="rms", norm_wq=z(32)), dict(norm="rms", norm_wq=q[0, 0, 0]), dict(norm="rms", eps=-1.0),
               dict(norm="rms", norm_wk=kv[0, 0, 0, 0])):
        with pytest.raises(xd.XditError):
            step(**kw)
            pytest.fail(f"{list(kw)} was taken")
    torch.cuda.synchronize()
    assert not any(a.any() for a in (q, k, v, o, y, kv))
