"""The attention's gradients against the formulas in 64 bits
(tests/layer_ref.py, which also derives the bounds): every element within the
worst error, and the root mean square within the operands' roundings taken as
independent, so that a row left out cannot hide under the worst case."""
from __future__ import annotations

import numpy as np
import pytest

import paper_2411_01738_amd as xd
from tests import layer_ref as ref
from tests.gpu_util import tdtype, torch_mod

pytestmark = pytest.mark.gpu


def _np(t):
    return t.float().cpu().numpy().astype(np.float64)


def _inputs(seed, B, nq, nk, H, d, dtype, dlse=False, scale=1.0):
    torch = torch_mod()
    g = torch.Generator().manual_seed(seed)
    r = lambda *s: (torch.randn(*s, generator=g) * scale).to(tdtype(dtype)).cuda()
    q, k, v, dout = r(B, nq, H, d), r(B, nk, H, d), r(B, nk, H, d), r(B, nq, H, d)
    o, l = ref.attention(_np(q), _np(k), _np(v))
    out = torch.from_numpy(o).to(tdtype(dtype)).cuda().contiguous()
    lse = torch.from_numpy(l).float().cuda()
    e = torch.randn(B, H, nq, generator=g).cuda() if dlse else None
    return q, k, v, out, lse, dout, e


def _grads(q, k, fill=float("nan"), dq=None, dkv=None):
    torch = torch_mod()
    new = lambda t, dt: torch.full(t.shape, fill, device="cuda", dtype=dt or t.dtype)
    return new(q, dq), new(k, dkv), new(k, dkv)


def _ws(q, nk, fill=True):
    torch = torch_mod()
    n = xd.chunk_attn_bwd_workspace_bytes(q, nk)
    ws = torch.empty(n, device="cuda", dtype=torch.uint8)
    if n:
        ws.view(torch.float32).fill_(float("nan"))
    return ws


def _check(got, want, what):
    for name, t in got.items():
        w, worst, dev = want[name]
        err = np.abs(_np(t) - w)
        bad = ~(err <= worst)
        assert not bad.any(), f"{what} {name}: {bad.sum()} of {bad.size} off, worst {np.nanmax(err - worst):.3e} over"
        if w.size:
            a, b = np.sqrt((err ** 2).mean()), np.sqrt((dev ** 2).mean())
            assert a <= b, f"{what} {name}: rms {a:.3e} over {b:.3e}"


def _run(seed, B, nq, nk, H, d, dtype, dlse=False, scale=1.0):
    q, k, v, out, lse, dout, e = _inputs(seed, B, nq, nk, H, d, dtype, dlse, scale)
    dq, dk, dv = _grads(q, k)
    xd.xdit_chunk_attn_bwd(q, k, v, out, lse, dout, dq, dk, dv, dlse=e, workspace=_ws(q, nk))
    want = ref.attention_bwd(_np(q), _np(k), _np(v), _np(out), _np(lse), _np(dout), None if e is None else _np(e), dtype)
    _check(dict(dq=dq, dk=dk, dv=dv), want, f"{dtype} {B}x{H} {nq}x{nk} d{d}")


# lengths around a block of 32, a tile of 64, a workgroup of 128 rows; one row
SIZES = [(1, 1), (1, 2), (33, 1), (31, 32), (64, 65), (32, 33), (96, 128), (129, 127), (130, 300), (257, 64), (5, 700), (700, 3)]


@pytest.mark.parametrize("d", [64, 72, 128])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_lengths(dtype, d):
    for i, (nq, nk) in enumerate(SIZES):
        B, H = ((1, 1), (2, 3), (1, 5))[i % 3]
        print(f"[bwd] {dtype} d{d} {B}x{H} {nq}x{nk}", flush=True)
        _run(100 + i, B, nq, nk, H, d, dtype, dlse=i % 2 == 1)


@pytest.mark.parametrize("dtype,d,B,H,nq,nk", [("bf16", 64, 1, 2, 33, 2500), ("bf16", 72, 1, 1, 1, 4100), ("bf16", 128, 1, 2, 20, 2100),
                                               ("bf16", 64, 1, 2, 2500, 40), ("bf16", 72, 1, 1, 3000, 1), ("bf16", 128, 1, 1, 2000, 130),
                                               ("f32", 64, 1, 1, 7, 1500), ("f32", 72, 1, 2, 1500, 9), ("f32", 128, 1, 1, 129, 900)])
def test_long_sweeps_of_few_rows(dtype, d, B, H, nq, nk):
    """Sweeps cut into parts that are joined."""
    _run(200, B, nq, nk, H, d, dtype, dlse=True)


def _sampled(seed, B, nq, nk, H, d, dtype, heads, dlse):
    """A call on the forward kernels' out and lse; some of its heads against the
    formulas."""
    torch = torch_mod()
    g = torch.Generator(device="cuda").manual_seed(seed)
    r = lambda n: torch.randn(B, n, H, d, generator=g, device="cuda").to(tdtype(dtype))
    q, k, v, dout = r(nq), r(nk), r(nk), r(nq)
    out, lse = torch.empty_like(q), torch.empty(B, H, nq, device="cuda")
    xd.xdit_chunk_attn(q, k, v, out, lse)
    e = torch.randn(B, H, nq, generator=g, device="cuda") if dlse else None
    dq, dk, dv = _grads(q, k)
    ws = _ws(q, nk)
    xd.xdit_chunk_attn_bwd(q, k, v, out, lse, dout, dq, dk, dv, dlse=e, workspace=ws)
    assert all(torch.isfinite(t).all() for t in (dq, dk, dv))
    for b, h in heads:
        at = lambda t: _np(t[b:b + 1, :, h:h + 1])
        row = lambda t: None if t is None else _np(t[b:b + 1, h:h + 1])
        want = ref.attention_bwd(at(q), at(k), at(v), at(out), row(lse), at(dout), row(e), dtype)
        _check(dict(dq=dq[b:b + 1, :, h:h + 1], dk=dk[b:b + 1, :, h:h + 1], dv=dv[b:b + 1, :, h:h + 1]), want,
               f"{dtype} {B}x{H} {nq}x{nk} d{d} head {b},{h}")
    return ws.numel()


# tiles of 64 streamed rows at bf16 head dims 64 and 72, of 32 otherwise: 11 and
# more in both sweeps of every call, in one round of workgroups and in several
@pytest.mark.parametrize("dtype,B,H,nq,nk", [("bf16", 1, 16, 715, 1030), ("bf16", 3, 16, 1100, 700), ("f32", 1, 16, 330, 450),
                                             ("f32", 2, 32, 410, 345)])
@pytest.mark.parametrize("d", [64, 72, 128])
def test_long_sweeps_of_many_rows(dtype, B, H, nq, nk, d):
    ws = _sampled(205, B, nq, nk, H, d, dtype, [(0, 0), (0, 7), (B - 1, H - 1)], dlse=B != 2)
    # nothing beyond two float32 per query row: no partials, so no sweep was cut
    assert ws == (8 * B * H * nq + 255) // 256 * 256


@pytest.mark.parametrize("dtype,B,H,nq,nk,d", [("bf16", 2, 24, 4429, 4429, 64), ("bf16", 2, 16, 4096, 4096, 72),
                                               ("bf16", 1, 24, 4224, 4224, 128), ("f32", 2, 16, 1024, 1024, 72)])
def test_whole_sequences(dtype, B, H, nq, nk, d):
    """The joint sequence of SD3, Pixart's, one chunk of Flux, a float32 share."""
    _sampled(206, B, nq, nk, H, d, dtype, [(B - 1, 5)], dlse=False)


@pytest.mark.parametrize("dtype,nq,nk,H,d", [("bf16", 261000, 4, 32, 128), ("bf16", 5, 261000, 32, 128), ("f32", 130000, 3, 32, 128),
                                             ("f32", 2, 130000, 32, 128)])
def test_the_largest_batch(dtype, nq, nk, H, d):
    """One batch of a tensor up to the 2 GiB that a call takes."""
    es = 2 if dtype == "bf16" else 4
    assert (1 << 31) - (1 << 24) < (max(nq, nk) + 256) * H * d * es < 1 << 31
    _sampled(207, 1, nq, nk, H, d, dtype, [(0, 0), (0, H - 1)], dlse=True)


@pytest.mark.parametrize("d", [64, 72, 128])
def test_many_heads(d):
    _run(210, 2, 150, 170, 17, d, "bf16")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_peaked_rows(dtype):
    """Scores of a large spread: most probabilities vanish, a few are one."""
    _run(220, 1, 200, 190, 2, 64, dtype, scale=4.0)


@pytest.mark.parametrize("dtype,d", [("bf16", 64), ("bf16", 72), ("bf16", 128), ("f32", 72)])
def test_sums(dtype, d):
    """accum: the gradients are added to float32 sums, one side or both; cut
    sweeps too."""
    torch = torch_mod()
    f32 = torch.float32
    for nq, nk in ((70, 90), (9, 1700), (1700, 9)):
        q, k, v, out, lse, dout, _ = _inputs(300, 1, nq, nk, 2, d, dtype)
        plain = _grads(q, k)
        xd.xdit_chunk_attn_bwd(q, k, v, out, lse, dout, *plain, workspace=_ws(q, nk))
        for aq, ak in ((True, False), (False, True), (True, True)):
            base = [torch.randn(*t.shape, device="cuda") for t in plain]
            acc = _grads(q, k)
            acc = [b.clone() if on else a for a, b, on in zip(acc, base, (aq, ak, ak))]
            xd.xdit_chunk_attn_bwd(q, k, v, out, lse, dout, *acc, accum_dq=aq, accum_dkv=ak, workspace=_ws(q, nk))
            zero = [torch.zeros_like(b) if on else a for a, b, on in zip(_grads(q, k), base, (aq, ak, ak))]
            xd.xdit_chunk_attn_bwd(q, k, v, out, lse, dout, *zero, accum_dq=aq, accum_dkv=ak, workspace=_ws(q, nk))
            for a, z, b, p, on in zip(acc, zero, base, plain, (aq, ak, ak)):
                if on:
                    assert a.dtype == f32 and torch.equal(a, z + b)     # one addition
                    assert torch.equal(z.to(p.dtype), p)                # of what the plain call rounds
                else:
                    assert torch.equal(a, p)


def test_rows_without_keys():
    """lse = -inf: the row has no part in any gradient, its out is not read."""
    torch = torch_mod()
    for dtype, d in (("bf16", 64), ("bf16", 128), ("f32", 72)):
        nq, nk = 140, 70
        q, k, v, out, lse, dout, e = _inputs(310, 1, nq, nk, 2, d, dtype, dlse=True)
        dead = torch.zeros(1, 2, nq, dtype=torch.bool, device="cuda")
        dead[:, 0, ::3] = True
        dead[:, 1, 100:] = True
        lse[dead] = float("-inf")
        rows = dead.transpose(1, 2)
        out[rows] = float("nan")
        dq, dk, dv = _grads(q, k)
        xd.xdit_chunk_attn_bwd(q, k, v, out, lse, dout, dq, dk, dv, dlse=e, workspace=_ws(q, nk))
        assert not dq[rows].any()
        want = ref.attention_bwd(_np(q), _np(k), _np(v), np.nan_to_num(_np(out)), _np(lse), _np(dout), _np(e), dtype)
        _check(dict(dq=dq, dk=dk, dv=dv), want, dtype)
        lse.fill_(float("-inf"))  # no row has a key
        xd.xdit_chunk_attn_bwd(q, k, v, out, lse, dout, dq, dk, dv, dlse=e, workspace=_ws(q, nk))
        assert not dq.any() and not dk.any() and not dv.any()


@pytest.mark.parametrize("dtype,d", [("bf16", 64), ("bf16", 72), ("bf16", 128), ("f32", 64)])
def test_rows_without_keys_hold_anything_finite(dtype, d):
    """Their out and dlse are NaN, their q and dout far above the others'."""
    nq, nk = 140, 70
    q, k, v, out, lse, dout, e = _inputs(311, 1, nq, nk, 2, d, dtype, dlse=True)
    dead = torch_mod().zeros(1, 2, nq, dtype=torch_mod().bool, device="cuda")
    dead[:, 0, 1::3] = True
    dead[:, 1, 90:] = True
    rows = dead.transpose(1, 2)
    lse[dead], e[dead], out[rows], q[rows], dout[rows] = float("-inf"), float("nan"), float("nan"), 1e15, -1e15
    dq, dk, dv = _grads(q, k)
    xd.xdit_chunk_attn_bwd(q, k, v, out, lse, dout, dq, dk, dv, dlse=e, workspace=_ws(q, nk))
    assert not dq[rows].any()
    # for the formulas and their error the rows are rows of zeros
    for t in (out, q, dout):
        t[rows] = 0.0
    want = ref.attention_bwd(_np(q), _np(k), _np(v), _np(out), _np(lse), _np(dout), np.nan_to_num(_np(e)), dtype)
    _check(dict(dq=dq, dk=dk, dv=dv), want, dtype)


def test_strongly_negative_lse():
    """Rows whose scores lie far below zero: padding keys of a tile, whose score
    would be zero, must not reach them."""
    torch = torch_mod()
    for dtype, d in (("bf16", 64), ("bf16", 72), ("bf16", 128), ("f32", 64)):
        nq, nk = 40, 45
        q = torch.full((1, nq, 1, d), 6.0, device="cuda").to(tdtype(dtype))
        q[:, ::2] = 5.0
        k = (-6.0 + torch.arange(nk, device="cuda").view(1, nk, 1, 1) % 3 / 64).expand(1, nk, 1, d).contiguous().to(tdtype(dtype))
        v = torch.randn(1, nk, 1, d, device="cuda").to(tdtype(dtype))
        dout = torch.randn(1, nq, 1, d, device="cuda").to(tdtype(dtype))
        o, l = ref.attention(_np(q), _np(k), _np(v))
        assert l.max() < -200
        out, lse = torch.from_numpy(o).to(tdtype(dtype)).cuda().contiguous(), torch.from_numpy(l).float().cuda()
        dq, dk, dv = _grads(q, k)
        xd.xdit_chunk_attn_bwd(q, k, v, out, lse, dout, dq, dk, dv, workspace=_ws(q, nk))
        want = ref.attention_bwd(_np(q), _np(k), _np(v), _np(out), _np(lse), _np(dout), None, dtype)
        _check(dict(dq=dq, dk=dk, dv=dv), want, f"{dtype} d{d}")


def test_far_into_long_tensors():
    """Batches past 2^32 bytes of the queries' tensors, then of the keys': the
    last one's gradients against the formulas."""
    torch = torch_mod()
    B, H, d = 273, 32, 128
    for nq, nk in ((2000, 4), (4, 2000)):
        new = lambda n: torch.zeros(B, n, H, d, device="cuda", dtype=torch.bfloat16)
        q, k, v, out, dout = new(nq), new(nk), new(nk), new(nq), new(nq)
        assert max(t.numel() for t in (q, k)) * 2 > 1 << 32
        lse = torch.zeros(B, H, nq, device="cuda")
        last = _inputs(320, 1, nq, nk, H, d, "bf16")
        for t, s in zip((q, k, v, out, lse, dout), last):
            t[-1:] = s
        got = _grads(q, k)
        xd.xdit_chunk_attn_bwd(q, k, v, out, lse, dout, *got, workspace=_ws(q, nk))
        want = ref.attention_bwd(*(_np(t) for t in last[:6]), None, "bf16")
        _check(dict(zip(("dq", "dk", "dv"), (t[-1:] for t in got))), want, f"{nq}x{nk}")
        assert not any(t[:-1].any() for t in got)


@pytest.mark.parametrize("accum", [False, True])
def test_several_launches(accum):
    """More workgroups than a launch holds: batches go out in three parts (16
    heads of one query and one key: 524287 batches at a time), with the bits of
    a call for each part, and the formulas at the parts' borders."""
    torch = torch_mod()
    step, H, d = 524287, 16, 64
    B = 2 * step + 3
    g = torch.Generator(device="cuda").manual_seed(325)
    f32 = torch.float32
    new = lambda dt: torch.randn(B, 1, H, d, generator=g, device="cuda", dtype=torch.bfloat16).to(dt)
    q, k, v, out, dout = (new(torch.bfloat16) for _ in range(5))
    lse, dlse = (torch.randn(B, H, 1, generator=g, device="cuda") for _ in range(2))
    lse = ((q.float() * k.float()).sum(-1).transpose(1, 2) * d ** -0.5 + lse.abs()).contiguous()
    base = [torch.ones(B, 1, H, d, device="cuda", dtype=f32) if accum else torch.full_like(q, float("nan")) for _ in range(3)]
    kw = dict(accum_dq=accum, accum_dkv=accum)
    got = [t.clone() for t in base]
    xd.xdit_chunk_attn_bwd(q, k, v, out, lse, dout, *got, dlse=dlse, workspace=_ws(q, 1), **kw)
    for a, b in ((0, step), (step, 2 * step), (2 * step, B)):
        part = [t[a:b].clone() for t in base]
        xd.xdit_chunk_attn_bwd(*(t[a:b] for t in (q, k, v, out, lse, dout)), *part, dlse=dlse[a:b], workspace=_ws(q[a:b], 1), **kw)
        for x, y in zip(got, part):
            assert torch.equal(x[a:b], y), f"batches {a}.."
    for a in (0, step - 1, 2 * step - 1, B - 2):
        args = [_np(t[a:a + 2]) for t in (q, k, v, out, lse, dout, dlse)]
        want = ref.attention_bwd(*args, "bf16")
        grads = [t[a:a + 2] - 1.0 if accum else t[a:a + 2] for t in got]
        if accum:  # the sum with 1 and the difference round once each
            want = {n: (w, *(x + 2.0 ** -24 * (1 + 2 * np.abs(w)) for x in bounds)) for n, (w, *bounds) in want.items()}
        _check(dict(zip(("dq", "dk", "dv"), grads)), want, f"batches {a}..")


def test_empty_sides():
    torch = torch_mod()
    z = lambda *s, dt=torch.bfloat16: torch.zeros(*s, device="cuda", dtype=dt)
    q, e, lse = z(1, 40, 2, 64), z(1, 0, 2, 64), z(1, 2, 40, dt=torch.float32)
    dq, none, none2 = _grads(q, e)
    xd.xdit_chunk_attn_bwd(q, e, e.clone(), q.clone(), lse.fill_(float("-inf")), q.clone(), dq, none, none2, workspace=_ws(q, 0))
    assert torch.equal(dq, torch.zeros_like(dq))
    k = z(1, 30, 2, 64)
    _, dk, dv = _grads(e, k)
    xd.xdit_chunk_attn_bwd(e, k, k.clone(), e.clone(), z(1, 2, 0, dt=torch.float32), e.clone(), e.clone(), dk, dv,
                           workspace=_ws(e, 30))
    assert torch.equal(dk, torch.zeros_like(dk)) and torch.equal(dv, torch.zeros_like(dv))
    acc = torch.ones(1, 40, 2, 64, device="cuda")
    xd.xdit_chunk_attn_bwd(q, e, e.clone(), q.clone(), lse, q.clone(), acc, none, none2, accum_dq=True, workspace=_ws(q, 0))
    assert torch.equal(acc, torch.ones_like(acc))


@pytest.mark.parametrize("dtype,d", [("bf16", 64), ("bf16", 72), ("bf16", 128), ("f32", 128)])
def test_ring(dtype, d):
    """Forward and backward of a ring over three uneven chunks, as one GPU runs
    it: the running (out, lse), then per chunk its dk, dv and its part of dq."""
    torch = torch_mod()
    B, nq, H, cuts = 1, 150, 3, (0, 130, 131, 290)
    q, k, v, _, _, dout, _ = _inputs(320, B, nq, cuts[-1], H, d, dtype)
    parts = [(k[:, a:b].contiguous(), v[:, a:b].contiguous()) for a, b in zip(cuts, cuts[1:])]
    out, lse = torch.empty_like(q), torch.full((B, H, nq), float("-inf"), device="cuda")
    for kr, vr in parts:
        xd.xdit_chunk_attn_accum(q, kr, vr, out, lse)
    dq = torch.zeros(q.shape, device="cuda")
    for (kr, vr), a, b in zip(parts, cuts, cuts[1:]):
        _, dk, dv = _grads(q, kr)
        xd.xdit_chunk_attn_bwd(q, kr, vr, out, lse, dout, dq, dk, dv, accum_dq=True, workspace=_ws(q, b - a))
        want = ref.attention_bwd(_np(q), _np(kr), _np(vr), _np(out), _np(lse), _np(dout), None, dtype)
        _check(dict(dk=dk, dv=dv), want, f"chunk {a}..{b}")
    want = ref.attention_bwd(_np(q), _np(k), _np(v), _np(out), _np(lse), _np(dout), None, dtype)
    _check(dict(dq=dq), want, "dq")


def test_partials_and_merge():
    """Gradients through chunk partials and their merge: out = sum w_r o_r with
    w_r = exp(lse_r - L) gives do_r = w_r g and dlse_r = w_r (g . o_r - g . out);
    the chunks' gradients with these equal those with the merged out and lse."""
    torch = torch_mod()
    B, nq, nk, H, d = 1, 90, 200, 2, 64
    q, k, v, _, _, g, _ = _inputs(330, B, nq, nk, H, d, "f32")
    cuts = ((0, 120), (120, 200))
    outs, lses = [torch.empty_like(q) for _ in cuts], [torch.empty(B, H, nq, device="cuda") for _ in cuts]
    ks, vs = [k[:, a:b].contiguous() for a, b in cuts], [v[:, a:b].contiguous() for a, b in cuts]
    for r in range(2):
        xd.xdit_chunk_attn(q, ks[r], vs[r], outs[r], lses[r])
    out, lse = torch.empty_like(q), torch.empty(B, H, nq, device="cuda")
    xd.xdit_lse_merge(outs, lses, 2, out, lse)
    sums = [torch.zeros_like(q) for _ in range(2)]
    for r in range(2):
        w = torch.exp(lses[r] - lse)
        dot = lambda o: (g * o).sum(-1).transpose(1, 2)
        do = (w.transpose(1, 2)[..., None] * g).contiguous()
        got = []
        for s, args, e in ((sums[0], (outs[r], lses[r], do), (w * (dot(outs[r]) - dot(out))).contiguous()), (sums[1], (out, lse, g), None)):
            _, dk, dv = _grads(q, ks[r])
            xd.xdit_chunk_attn_bwd(q, ks[r], vs[r], *args, s, dk, dv, dlse=e, accum_dq=True, workspace=_ws(q, ks[r].shape[1]))
            got.append((dk, dv))
        for a, b in zip(*got):
            assert (a - b).abs().max() <= 2e-5 * b.abs().max()
    # both forms of float32: a thousand roundings of 2^-24 at most
    assert (sums[0] - sums[1]).abs().max() <= 6e-5 * sums[1].abs().max()


def test_same_bits_streams_and_graphs():
    """Twice the same call, on a stream of its own, and captured and replayed
    with other inputs, sweeps cut and uncut: the same bits."""
    torch = torch_mod()
    for B, H, nq, nk, d in ((2, 16, 300, 400, 72), (1, 2, 20, 1500, 128)):
        q, k, v, out, lse, dout, e = _inputs(340, B, nq, nk, H, d, "bf16", dlse=True)
        ws = [_ws(q, nk) for _ in range(2)]

        def call(g, w):
            xd.xdit_chunk_attn(q, k, v, out, lse)
            xd.xdit_chunk_attn_bwd(q, k, v, out, lse, dout, *g, dlse=e, workspace=w)

        first, second, side, cap = (_grads(q, k) for _ in range(4))
        call(first, ws[0])
        call(second, ws[1])
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            call(side, ws[0])
        torch.cuda.current_stream().wait_stream(s)
        for a, b, c in zip(first, second, side):
            assert torch.equal(a, b) and torch.equal(a, c)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            call(cap, ws[1])
        for i in range(4):
            q.copy_(torch.randn_like(q))
            dout.copy_(torch.randn_like(q))
            for t in cap:
                t.zero_()
            graph.replay()
            call(first, ws[0])
            torch.cuda.synchronize()
            for a, b in zip(first, cap):
                assert torch.equal(a, b), f"replay {i}"


@pytest.mark.parametrize("norm,layout", [("rms", "interleaved"), ("layer", "half")])
def test_a_layer_forward_and_backward(norm, layout):
    """Table, norms and rotation, attention over two chunks, and all their
    gradients, float32, from one fused projection's output; against the same in
    64 bits.  Each of the four kernels on the way is good to about a thousand
    roundings of 2^-24 relative to the largest value it forms; three passes of
    that bound the result at 2e-4 of the gradient's norm."""
    torch = torch_mod()
    B, N, H, d, rot, eps = 2, 75, 3, 64, 48, 1e-6
    g = torch.Generator().manual_seed(350)
    qkv = torch.randn(B, N, 3 * H, d, generator=g).cuda()
    w = {n: (1 + 0.3 * torch.randn(d, generator=g)).cuda() for n in ("wq", "wk")}
    b = {n: (0.2 * torch.randn(d, generator=g)).cuda() for n in ("bq", "bk")} if norm == "layer" else {}
    dout = torch.randn(B, N, H, d, generator=g).cuda()
    pos = torch.stack([torch.arange(N), torch.arange(N) % 7], 1).cuda()
    cos, sin = torch.empty(N, rot // 2, device="cuda"), torch.empty(N, rot // 2, device="cuda")
    xd.xdit_rope_table(pos, [16, 32], cos, sin)
    q0, k0, v0 = (qkv[:, :, i * H:(i + 1) * H] for i in range(3))
    q, k, v = (torch.empty(B, N, H, d, device="cuda") for _ in range(3))
    kw = dict(norm=norm, eps=eps, cos=cos, sin=sin, layout=layout)
    xd.xdit_qk_norm_rope(q0, k0, q, k, **kw, **w, **b)
    v.copy_(v0)
    out, lse = torch.empty_like(q), torch.full((B, H, N), float("-inf"), device="cuda")
    cuts = ((0, 40), (40, N))
    ks, vs = [k[:, x:y].contiguous() for x, y in cuts], [v[:, x:y].contiguous() for x, y in cuts]
    for r in range(2):
        xd.xdit_chunk_attn_accum(q, ks[r], vs[r], out, lse)
    dq, dk, dv = torch.zeros_like(q), torch.empty_like(q), torch.empty_like(q)
    for r, (x, y) in enumerate(cuts):
        _, dkr, dvr = _grads(q, ks[r])
        xd.xdit_chunk_attn_bwd(q, ks[r], vs[r], out, lse, dout, dq, dkr, dvr, accum_dq=True, workspace=_ws(q, y - x))
        dk[:, x:y], dv[:, x:y] = dkr, dvr
    dqkv = torch.full_like(qkv, float("nan"))
    dw = {"d" + n: torch.empty(d, device="cuda") for n in ("wq", "wk", *b)}
    ws = torch.empty(xd.qk_norm_rope_bwd_workspace_bytes(q0, k0), device="cuda", dtype=torch.uint8)
    xd.xdit_qk_norm_rope_bwd(q0, k0, dq, dk, dqkv[:, :, :H], dqkv[:, :, H:2 * H], **kw, **w, **dw, workspace=ws)
    dqkv[:, :, 2 * H:] = dv

    f = lambda t: None if t is None else _np(t)
    c, s = ref.table(pos.cpu().numpy(), [16, 32])
    Q0, K0, V = (f(qkv[:, :, i * H:(i + 1) * H]) for i in range(3))
    Q = ref.forward(Q0, f(w["wq"]), f(b.get("bq")), c, s, norm, eps, layout)
    K = ref.forward(K0, f(w["wk"]), f(b.get("bk")), c, s, norm, eps, layout)
    O, L = ref.attention(Q, K, V)
    back = ref.attention_bwd(Q, K, V, O, L, f(dout), None, "f32")
    gq = ref.backward(Q0, f(w["wq"]), back["dq"][0], c, s, norm, eps, layout)
    gk = ref.backward(K0, f(w["wk"]), back["dk"][0], c, s, norm, eps, layout)
    want = {"dqkv": (dqkv, np.concatenate([gq[0], gk[0], back["dv"][0]], 2)), "dwq": (dw["dwq"], gq[1]), "dwk": (dw["dwk"], gk[1])}
    if b:
        want.update(dbq=(dw["dbq"], gq[2]), dbk=(dw["dbk"], gk[2]))
    for name, (got, exact) in want.items():
        err = np.linalg.norm(f(got) - exact) / np.linalg.norm(exact)
        assert err <= 2e-4, f"{name}: {err:.2e}"


def test_both_call_paths_agree(monkeypatch):
    torch = torch_mod()
    nat = xd._load_native()
    taken = []

    class Rec:
        def __getattr__(self, name):
            def call(*a):
                taken.append((name, getattr(nat, name)(*a)))
                return taken[-1][1]
            return call

    q, k, v, out, lse, dout, e = _inputs(360, 1, 50, 60, 2, 64, "bf16", dlse=True)
    got = []
    for path in (Rec(), False):
        monkeypatch.setattr(xd, "_native", path)
        g = [torch.zeros(q.shape, device="cuda"), *_grads(q, k)[1:]]
        xd.xdit_chunk_attn_bwd(q, k, v, out, lse, dout, *g, dlse=e, accum_dq=True, workspace=_ws(q, 60))
        got.append(g)
    assert taken == [("chunk_bwd", 0)]
    for a, b in zip(*got):
        assert torch.equal(a, b)


def test_refusals(monkeypatch):
    torch = torch_mod()
    nat = xd._load_native()
    q, k, v, out, lse, dout, e = _inputs(370, 1, 40, 50, 2, 64, "bf16", dlse=True)
    ws = _ws(q, 50)
    dq, dk, dv = _grads(q, k, fill=0.0)
    good = dict(q=q, k=k, v=v, out=out, lse=lse, dout=dout, dq=dq, dk=dk, dv=dv, dlse=e, workspace=ws)
    bad = [dict(q=q.float()), dict(k=k[:, :49]), dict(v=v.cpu()), dict(out=out[:, :39].contiguous()), dict(lse=None),
           dict(lse=lse.half()), dict(dout=dout.transpose(1, 2)), dict(dout=None), dict(dq=dq.float()), dict(dq=dq, accum_dq=True),
           dict(dk=dk.float()), dict(dk=dk.float(), accum_dkv=True), dict(dv=dv[:, :1]), dict(dlse=e[:, :, :5].contiguous()),
           dict(workspace=None), dict(workspace=ws[:16]), dict(workspace=ws[16:]), dict(dq=q), dict(dq=out), dict(dk=dv), dict(dv=v),
           dict(dq=dout), dict(dk=None)]
    for path in (nat, False):
        monkeypatch.setattr(xd, "_native", path)
        for x in bad:
            with pytest.raises(xd.XditError):
                xd.xdit_chunk_attn_bwd(**{**good, **x})
                pytest.fail(f"{list(x)} was taken")
    torch.cuda.synchronize()
    assert not dq.any() and not dk.any() and not dv.any()
