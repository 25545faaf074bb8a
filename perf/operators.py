"""Timing cases of the operators around the attention of one layer: rotary
positions, the norms of queries and keys that go with them, and the gradients
of both and of the attention itself.

listed() names the fixed cases, draw() makes more over the same ranges,
prepare() builds a case's inputs on the GPU, run() is one pass, work() the
bytes and operations no implementation can do without, exact() the result in
64 bits.

A case's fields: op, dtype ("bf16" or "f32", of the activations), and per op
  table     N positions of len(dims) axes (`dims` as "16+56+56"), as whole
            numbers or fractional ("pos"), the first one `first`; theta;
            scaling "none", "linear", "ntk" or "ramp" with its factor and the
            original length, and the magnitude of the table
  rope      x of [B, N, H, d], its first `rot` dims rotated; layout; transpose
            (the gradient)
  norm      queries [B, N, H, d] and keys [B, N, Hk, d] normalised per head
            (norm "rms" or "layer", weights of `wtype`) and rotated (rot = 0:
            not rotated); fused: they are views of one projection's output
  norm_bwd  gradients of norm
  attn_bwd  gradients of the attention of nq queries over `chunks` chunks
            that share nk keys; dlse: the log-sum-exp has a gradient too; ring:
            the queries' gradient summed in float32 over the chunks, and
            the output and log-sum-exp those of all chunks
"""
from __future__ import annotations

import math

import torch

own = False


def listed():
    return [
        # The rotary table of Flux at 2048px, one GPU's shard of the joint
        # sequence: text and two image axes.
        dict(name="flux_table", op="table", dtype="f32", N=4224, dims="16+56+56", pos="whole", first=0, theta=10000.0,
             scaling="none", factor=1.0, orig=0, magnitude=1.0),
        # A long sequence far from its start, frequencies scaled by how often
        # they turn within the original length.
        dict(name="long_table", op="table", dtype="f32", N=131072, dims="128", pos="whole", first=1 << 20, theta=500000.0,
             scaling="ramp", factor=8.0, orig=16384, magnitude=1.2079441541679836),
        # One token of one head set: all latency.
        dict(name="token_rope", op="rope", dtype="bf16", B=1, N=1, H=24, d=128, rot=128, layout="half", transpose=False),
        # The gradient through the rotation of CogVideoX's video rows.
        dict(name="cog_rope_bwd", op="rope", dtype="bf16", B=1, N=17550, H=48, d=64, rot=64, layout="interleaved",
             transpose=True),
        # A float32 caller: few rows, part of each head rotated.
        dict(name="tiny_norm_f32", op="norm", dtype="f32", B=2, N=77, H=2, Hk=2, d=64, rot=32, layout="half", norm="rms",
             wtype="f32", fused=False),
        # Flux: RMS norms and rotation of one shard's queries and keys, as the
        # fused projection leaves them.
        dict(name="flux_norm", op="norm", dtype="bf16", B=1, N=4224, H=24, Hk=24, d=128, rot=128, layout="interleaved",
             norm="rms", wtype="bf16", fused=True),
        # SD3's text rows, training: norms with no rotation.
        dict(name="sd3_text_norm_bwd", op="norm_bwd", dtype="bf16", B=2, N=333, H=24, Hk=24, d=64, rot=0,
             layout="interleaved", norm="rms", wtype="bf16", fused=False),
        # CogVideoX, training: layer norms with weight and bias, then the
        # rotation, of the whole video.
        dict(name="cog_norm_bwd", op="norm_bwd", dtype="bf16", B=1, N=17550, H=48, Hk=48, d=64, rot=64,
             layout="interleaved", norm="layer", wtype="f32", fused=False),
        # The tiny float32 model's chunk: all latency.
        dict(name="tiny_bwd_f32", op="attn_bwd", dtype="f32", B=1, H=2, d=64, nq=256, nk=64, chunks=1, dlse=False, ring=False),
        # SD3's text queries over the joint sequence: few query rows, odd sizes.
        dict(name="sd3_text_bwd", op="attn_bwd", dtype="bf16", B=2, H=24, d=64, nq=333, nk=4429, chunks=1, dlse=False,
             ring=False),
        # One chunk of Pixart's sequence-parallel share, its partial merged
        # with the others afterwards.
        dict(name="pixart_bwd", op="attn_bwd", dtype="bf16", B=2, H=16, d=72, nq=1024, nk=1024, chunks=1, dlse=True,
             ring=False),
        # Flux 2048px: two steps of the ring that one GPU's queries go
        # through; the largest.
        dict(name="flux_ring_bwd", op="attn_bwd", dtype="bf16", B=1, H=24, d=128, nq=4224, nk=8448, chunks=2, dlse=False,
             ring=True),
    ]


# (heads, head dim) of the models, whole and split over tensor-parallel ranks
_HEADS = [(16, 72), (8, 72), (24, 64), (12, 64), (48, 64), (6, 64), (24, 128), (12, 128), (3, 128)]
_MOST_FLOPS = {"bf16": 1.0e12, "f32": 2.0e10}  # of an attn_bwd case


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the listed ones' ranges: one row to whole videos, any
    remainder, every layout, norm, type and scaling."""
    op = rng.choice(["table", "rope", "norm", "norm", "norm_bwd", "norm_bwd", "attn_bwd", "attn_bwd", "attn_bwd", "attn_bwd"])
    f32 = rng.random() < 0.2
    H, d = rng.choice(_HEADS)
    B = rng.choice([1, 1, 2])
    c = dict(op=op, dtype="f32" if f32 or op == "table" else "bf16")
    if op == "table":
        dims = rng.choice(["16+56+56", "16+24+24", "32+32", "128", "64", "72", "40+24"])
        kind = rng.choice(["none", "linear", "ntk", "ramp"])
        c.update(N=_log(rng, 1, 131072), dims=dims, pos=rng.choice(["whole", "fraction"]), first=_log(rng, 1, 1 << 20) - 1,
                 theta=rng.choice([10000.0, 256.0, 500000.0]), scaling=kind, factor=1.0 if kind == "none" else rng.uniform(1.0, 16.0),
                 orig=_log(rng, 512, 16384), magnitude=rng.choice([1.0, rng.uniform(0.8, 1.5)]))
        return c
    c.update(B=B, H=H, d=d)
    layout = rng.choice(["interleaved", "half"])
    rot = rng.choice([d, d, 8 * rng.randint(1, d // 8)])
    if op == "rope":
        c.update(N=min(_log(rng, 1, 20000), int(5.0e7 / (B * H * d))), rot=rot, layout=layout, transpose=rng.random() < 0.5)
    elif op in ("norm", "norm_bwd"):
        c.update(N=min(_log(rng, 1, 20000), int((2.5e7 if f32 else 5.0e7) / (B * H * d))), Hk=rng.choice([H, H, max(1, H // 3)]),
                 rot=rng.choice([0, rot, rot, rot]), layout=layout, norm=rng.choice(["rms", "rms", "layer"]),
                 wtype=rng.choice(["f32", c["dtype"]]), fused=rng.random() < 0.4)
    else:
        most = _MOST_FLOPS[c["dtype"]]
        chunks = rng.choice([1, 1, 1, 2, 3])
        nk = _log(rng, chunks, 18000)
        nq = max(1, min(_log(rng, 1, 18000), int(most / (10.0 * B * H * d * nk))))
        ring = chunks > 1
        c.update(nq=nq, nk=nk, chunks=chunks, dlse=not ring and rng.random() < 0.4, ring=ring)
    return c


# -- inputs -------------------------------------------------------------------
class _Draws:
    """Normal tensors on the GPU from one seed, in call order."""

    def __init__(self, case, seed):
        self.g = torch.Generator(device="cuda")
        self.g.manual_seed(seed)
        self.dt = _type(case["dtype"])

    def f32(self, *shape, scale=1.0):
        return torch.randn(shape, generator=self.g, device="cuda", dtype=torch.float32) * scale

    def io(self, *shape, scale=1.0):
        return self.f32(*shape, scale=scale).to(self.dt)


def _type(name):
    return torch.bfloat16 if name == "bf16" else torch.float32


def _dims(case):
    return [int(x) for x in case["dims"].split("+")]


def _chunks(case):
    """Row ranges of the key chunks, near-equal."""
    n, k = case["nk"], case["chunks"]
    return [(n * r // k, n * (r + 1) // k) for r in range(k)]


def _angles(g, N, rot):
    """A rotary table of N positions on one axis from a random start."""
    first = torch.randint(0, 100000, (1,), generator=g.g, device="cuda")
    pos = (first + torch.arange(N, device="cuda")).double()
    inv = 10000.0 ** (-torch.arange(0, rot, 2, device="cuda", dtype=torch.float64) / rot)
    a = pos[:, None] * inv
    return torch.cos(a).float(), torch.sin(a).float()


def _norm_inputs(case, g):
    B, N, H, Hk, d = (case[x] for x in ("B", "N", "H", "Hk", "d"))
    if case["fused"]:  # views of one projection's output, the values' heads behind the keys'
        qkv = g.io(B, N, H + 2 * Hk, d, scale=1.5)
        q, k = qkv[:, :, :H], qkv[:, :, H:H + Hk]
    else:
        q, k = g.io(B, N, H, d, scale=1.5), g.io(B, N, Hk, d, scale=1.5)
    wt = _type(case["wtype"])
    st = dict(q=q, k=k, wq=(1.0 + g.f32(d, scale=0.3)).to(wt), wk=(1.0 + g.f32(d, scale=0.3)).to(wt), bq=None, bk=None,
              cos=None, sin=None, eps=1e-6)
    if case["norm"] == "layer":
        st.update(bq=g.f32(d, scale=0.2).to(wt), bk=g.f32(d, scale=0.2).to(wt))
    if case["rot"]:
        st["cos"], st["sin"] = _angles(g, N, case["rot"])
    return st


def prepare(case, seed):
    g = _Draws(case, seed)
    st = dict(case=case)
    new = lambda x, dt=None: torch.empty(x.shape, device="cuda", dtype=dt or x.dtype)  # noqa: E731
    op = case["op"]
    if op == "table":
        N, dims = case["N"], _dims(case)
        shift = torch.randint(0, 4096, (1, len(dims)), generator=g.g, device="cuda")
        pos = case["first"] + shift + torch.arange(N, device="cuda")[:, None] % torch.tensor(
            [N] + [128] * (len(dims) - 1), device="cuda")
        if case["pos"] == "fraction":  # a grid of another resolution, stretched onto the trained one
            pos = (pos.double() * 0.59375).float()
        st.update(pos=pos.contiguous(), cos=torch.empty(N, sum(dims) // 2, device="cuda"),
                  sin=torch.empty(N, sum(dims) // 2, device="cuda"))
    elif op == "rope":
        st["x"] = g.io(case["B"], case["N"], case["H"], case["d"])
        st["cos"], st["sin"] = _angles(g, case["N"], case["rot"])
        st["y"] = new(st["x"])
    elif op == "norm":
        st.update(_norm_inputs(case, g))
        st.update(yq=new(st["q"]), yk=new(st["k"]))
    elif op == "norm_bwd":
        st.update(_norm_inputs(case, g))
        st.update(gq=g.io(*st["q"].shape), gk=g.io(*st["k"].shape), dq=new(st["q"]), dk=new(st["k"]))
        for n in ("wq", "wk", "bq", "bk"):
            st["d" + n] = None if st[n] is None else new(st[n], torch.float32)
    else:
        B, H, d, nq, nk = (case[x] for x in ("B", "H", "d", "nq", "nk"))
        q, k, v = g.io(B, nq, H, d), g.io(B, nk, H, d), g.io(B, nk, H, d)
        s = _mm(_heads(q), _heads(k).transpose(2, 3)) * d ** -0.5
        lse = torch.logsumexp(s, 3)
        out = _mm(torch.exp(s.sub_(lse[..., None])), _heads(v)).transpose(1, 2).to(g.dt).contiguous()
        del s
        parts = _chunks(case)
        st.update(q=q, k=[k[:, a:b].contiguous() for a, b in parts], v=[v[:, a:b].contiguous() for a, b in parts], out=out,
                  lse=lse.contiguous(), dout=g.io(B, nq, H, d), dlse=g.f32(B, H, nq) if case["dlse"] else None)
        st.update(dq=new(q, torch.float32 if case["ring"] else None), dk=[new(x) for x in st["k"]], dv=[new(x) for x in st["v"]])
    return st


# -- the plain form -----------------------------------------------------------
def _heads(x):
    """[B, N, H, d] as float32 [B, H, N, d]."""
    return x.float().transpose(1, 2).contiguous()


def _mm(a, b):
    return torch.matmul(a.contiguous(), b.contiguous())


def _rotate(x, cos, sin, layout, transpose):
    """The first 2 * cos.shape[-1] dims of float32 x [B, N, H, d] rotated."""
    if cos is None:
        return x
    r = cos.shape[-1]
    c, s = cos[:, None], -sin[:, None] if transpose else sin[:, None]
    y = torch.empty_like(x)
    y[..., 2 * r:] = x[..., 2 * r:]
    a, b = (slice(0, 2 * r, 2), slice(1, 2 * r, 2)) if layout == "interleaved" else (slice(0, r), slice(r, 2 * r))
    y[..., a] = x[..., a] * c - x[..., b] * s
    y[..., b] = x[..., b] * c + x[..., a] * s
    return y


def _stats(x, norm, eps):
    """x shifted by its mean (layer norm), and the factor that normalises it."""
    if norm == "layer":
        x = x - x.mean(-1, keepdim=True)
    return x, torch.rsqrt((x * x).mean(-1, keepdim=True) + eps)


def _norm_fwd(x, w, b, st):
    c = st["case"]
    x, r = _stats(x.float(), c["norm"], st["eps"])
    y = x * r * w.float()
    if b is not None:
        y = y + b.float()
    return _rotate(y, st["cos"], st["sin"], c["layout"], False).to(st["q"].dtype)


def _norm_bwd(x, w, b, g, st):
    c = st["case"]
    g = _rotate(g.float(), st["cos"], st["sin"], c["layout"], True)
    x, r = _stats(x.float(), c["norm"], st["eps"])
    n = x * r
    gw = g * w.float()
    dx = gw - n * (gw * n).mean(-1, keepdim=True)
    if c["norm"] == "layer":
        dx = dx - gw.mean(-1, keepdim=True)
    return (dx * r).to(st["q"].dtype), (g * n).sum((0, 1, 2)), None if b is None else g.sum((0, 1, 2))


def _table(pos, case):
    freq = []
    for dim in _dims(case):
        theta, f = case["theta"], case["factor"]
        if case["scaling"] == "ntk":
            theta = theta * f ** (dim / (dim - 2))
        inv = theta ** (-torch.arange(0, dim, 2, device=pos.device, dtype=torch.float64) / dim)
        if case["scaling"] == "linear":
            inv = inv / f
        elif case["scaling"] == "ramp":
            share = ((case["orig"] * inv / (2 * math.pi) - 1.0) / (32.0 - 1.0)).clamp(0, 1)
            inv = inv * (share + (1 - share) / f)
        freq.append(inv)
    a = torch.cat([pos[:, i:i + 1].double() * inv for i, inv in enumerate(freq)], 1)
    return (torch.cos(a) * case["magnitude"]).float(), (torch.sin(a) * case["magnitude"]).float()


def _attn_bwd(q, k, v, out, lse, dout, dlse):
    """Gradients in float32 [B, N, H, d] of one chunk's attention."""
    q, k, v, out, dout = (_heads(x) for x in (q, k, v, out, dout))
    scale = q.shape[-1] ** -0.5
    p = torch.exp(_mm(q, k.transpose(2, 3)) * scale - lse[..., None])
    delta = (dout * out).sum(-1)
    if dlse is not None:
        delta = delta - dlse
    dv = _mm(p.transpose(2, 3), dout)
    ds = p.mul_(_mm(dout, v.transpose(2, 3)) - delta[..., None]).mul_(scale)
    return tuple(x.transpose(1, 2) for x in (_mm(ds, k), _mm(ds.transpose(2, 3), q), dv))


def _plain(st):
    case = st["case"]
    op = case["op"]
    if op == "table":
        cos, sin = _table(st["pos"], case)
        return dict(cos=cos, sin=sin)
    if op == "rope":
        x = st["x"]
        return dict(y=_rotate(x.float(), st["cos"], st["sin"], case["layout"], case["transpose"]).to(x.dtype))
    if op == "norm":
        return dict(q=_norm_fwd(st["q"], st["wq"], st["bq"], st), k=_norm_fwd(st["k"], st["wk"], st["bk"], st))
    if op == "norm_bwd":
        dq, dwq, dbq = _norm_bwd(st["q"], st["wq"], st["bq"], st["gq"], st)
        dk, dwk, dbk = _norm_bwd(st["k"], st["wk"], st["bk"], st["gk"], st)
        return dict(dq=dq, dk=dk, dwq=dwq, dwk=dwk, dbq=dbq, dbk=dbk)
    got = [_attn_bwd(st["q"], k, v, st["out"], st["lse"], st["dout"], st["dlse"]) for k, v in zip(st["k"], st["v"])]
    dt = st["q"].dtype
    return dict(dq=sum(x[0] for x in got).to(dt).contiguous(), dk=[x[1].to(dt).contiguous() for x in got],
                dv=[x[2].to(dt).contiguous() for x in got])


# -- the framework's calls ----------------------------------------------------
def _workspace(st, name, size):
    """The workspace that a program keeps for its calls of one shape."""
    if name not in st:
        n = size()
        st[name] = torch.empty(n, device="cuda", dtype=torch.uint8) if n else None
    return st[name]


def _own(st):
    import paper_2411_01738_amd as xd

    case = st["case"]
    op = case["op"]
    if op == "table":
        xd.xdit_rope_table(st["pos"], _dims(case), st["cos"], st["sin"], theta=case["theta"], scaling=case["scaling"],
                           factor=case["factor"], orig_len=case["orig"], magnitude=case["magnitude"])
        return dict(cos=st["cos"], sin=st["sin"])
    if op == "rope":
        xd.xdit_rope(st["x"], st["cos"], st["sin"], st["y"], layout=case["layout"], transpose=case["transpose"])
        return dict(y=st["y"])
    if op == "norm":
        xd.xdit_qk_norm_rope(st["q"], st["k"], st["yq"], st["yk"], norm=case["norm"], eps=st["eps"], wq=st["wq"], wk=st["wk"],
                             bq=st["bq"], bk=st["bk"], cos=st["cos"], sin=st["sin"], layout=case["layout"])
        return dict(q=st["yq"], k=st["yk"])
    if op == "norm_bwd":
        ws = _workspace(st, "ws", lambda: xd.qk_norm_rope_bwd_workspace_bytes(st["q"], st["k"]))
        xd.xdit_qk_norm_rope_bwd(st["q"], st["k"], st["gq"], st["gk"], st["dq"], st["dk"], norm=case["norm"], eps=st["eps"],
                                 wq=st["wq"], wk=st["wk"], cos=st["cos"], sin=st["sin"], layout=case["layout"], dwq=st["dwq"],
                                 dwk=st["dwk"], dbq=st["dbq"], dbk=st["dbk"], workspace=ws)
        return {n: st[n] for n in ("dq", "dk", "dwq", "dwk", "dbq", "dbk")}
    if case["ring"]:
        st["dq"].zero_()
    for r, (k, v) in enumerate(zip(st["k"], st["v"])):
        ws = _workspace(st, "ws%d" % r, lambda: xd.chunk_attn_bwd_workspace_bytes(st["q"], k.shape[1]))
        xd.xdit_chunk_attn_bwd(st["q"], k, v, st["out"], st["lse"], st["dout"], st["dq"], st["dk"][r], st["dv"][r],
                               dlse=st["dlse"], accum_dq=case["ring"], workspace=ws)
    return dict(dq=st["dq"].to(st["q"].dtype), dk=st["dk"], dv=st["dv"])


def run(state):
    return _own(state) if own else _plain(state)


# -- floors -------------------------------------------------------------------
def work(case):
    op, es = case["op"], 2 if case["dtype"] == "bf16" else 4
    if op == "table":
        dims = _dims(case)
        cols = sum(dims) // 2
        return dict(bytes=case["N"] * ((8 if case["pos"] == "whole" else 4) * len(dims) + 8.0 * cols), flops=50.0 * case["N"] * cols)
    B, H, d = case["B"], case["H"], case["d"]
    if op == "attn_bwd":
        nq, nk = case["nq"], case["nk"]
        b = es * B * H * d * (4.0 * nq + 4.0 * nk) + 4.0 * B * H * nq * (2 if case["dlse"] else 1)
        return dict(bytes=b, flops=10.0 * B * H * nq * nk * d)
    N = case["N"]
    heads = H if op == "rope" else H + case["Hk"]
    rows = B * N * heads * d
    moved = 3 if op == "norm_bwd" else 2
    each = 3.0 * case["rot"] / d + (0 if op == "rope" else 5 if op == "norm" else 14)
    return dict(bytes=float(moved * es * rows) + 4.0 * N * case["rot"], flops=each * rows)


# -- 64 bits ------------------------------------------------------------------
def _turn(x, cos, sin, layout, sign):
    """Rotation in complex128: each pair times cos + i sign sin."""
    if cos is None:
        return x
    r = cos.shape[1]
    z = torch.complex(cos.double(), sign * sin.double())[None, :, None, :]
    head, rest = x[..., :2 * r], x[..., 2 * r:]
    if layout == "half":
        w = torch.complex(head[..., :r].contiguous(), head[..., r:].contiguous()) * z
        return torch.cat((w.real, w.imag, rest), -1)
    w = torch.view_as_complex(head.reshape(*head.shape[:-1], r, 2).contiguous()) * z
    return torch.cat((torch.view_as_real(w).flatten(-2), rest), -1)


def _exact_norm(st, x, w, b, g):
    """Forward (g None) or the gradients, from the definition of the variance."""
    c, d = st["case"], x.shape[-1]
    x, w = x.double(), w.double()
    if c["norm"] == "layer":
        m = x.sum(-1, keepdim=True) / d
        sd = (((x - m) ** 2).sum(-1, keepdim=True) / d + st["eps"]).sqrt()
        n = (x - m) / sd
    else:
        sd = ((x ** 2).sum(-1, keepdim=True) / d + st["eps"]).sqrt()
        n = x / sd
    if g is None:
        return _turn(n * w + (0 if b is None else b.double()), st["cos"], st["sin"], c["layout"], 1.0)
    g = _turn(g.double(), st["cos"], st["sin"], c["layout"], -1.0)
    dn = g * w
    back = dn - n * (dn * n).sum(-1, keepdim=True) / d
    if c["norm"] == "layer":
        back = back - dn.sum(-1, keepdim=True) / d
    flat = lambda t: t.reshape(-1, d).sum(0)  # noqa: E731
    return back / sd, flat(g * n), None if b is None else flat(g)


def _exact_attn(st):
    """One (batch, head) at a time, from P = exp(s - lse) and dS = P (dP - D)."""
    q, out, dout, lse = st["q"], st["out"], st["dout"], st["lse"].double()
    B, nq, H, d = q.shape
    dq = torch.zeros(q.shape, device="cuda", dtype=torch.float64)
    dk = [torch.zeros(k.shape, device="cuda", dtype=torch.float64) for k in st["k"]]
    dv = [torch.zeros(k.shape, device="cuda", dtype=torch.float64) for k in st["k"]]
    for b in range(B):
        for h in range(H):
            Q, O, G = (x[b, :, h].double() for x in (q, out, dout))
            D = (O * G).sum(1)
            if st["dlse"] is not None:
                D = D - st["dlse"][b, h].double()
            for r, (k, v) in enumerate(zip(st["k"], st["v"])):
                K, V = k[b, :, h].double(), v[b, :, h].double()
                P = (Q @ K.T / math.sqrt(d) - lse[b, h][:, None]).exp()
                dv[r][b, :, h] = P.T @ G
                S = P * (G @ V.T - D[:, None]) / math.sqrt(d)
                dq[b, :, h] += S @ K
                dk[r][b, :, h] = S.T @ Q
    return dict(dq=dq, dk=dk, dv=dv)


def exact(case, seed):
    st = prepare(case, seed)
    op = case["op"]
    if op == "table":
        cols, at = [], 0
        for a, dim in enumerate(_dims(case)):
            for i in range(dim // 2):
                f = case["factor"]
                theta = case["theta"] if case["scaling"] != "ntk" else case["theta"] * math.pow(f, dim / (dim - 2))
                w = math.exp(-math.log(theta) * 2 * i / dim)
                if case["scaling"] == "linear":
                    w /= f
                elif case["scaling"] == "ramp":
                    turns = case["orig"] * w / (2 * math.pi)
                    keep = min(1.0, max(0.0, (turns - 1.0) / 31.0))
                    w = keep * w + (1.0 - keep) * w / f
                cols.append(st["pos"][:, a].double() * w)
                at += 1
        ang = torch.stack(cols, 1)
        return dict(cos=case["magnitude"] * torch.cos(ang), sin=case["magnitude"] * torch.sin(ang))
    if op == "rope":
        return dict(y=_turn(st["x"].double(), st["cos"], st["sin"], case["layout"], -1.0 if case["transpose"] else 1.0))
    if op == "norm":
        return dict(q=_exact_norm(st, st["q"], st["wq"], st["bq"], None), k=_exact_norm(st, st["k"], st["wk"], st["bk"], None))
    if op == "norm_bwd":
        dq, dwq, dbq = _exact_norm(st, st["q"], st["wq"], st["bq"], st["gq"])
        dk, dwk, dbk = _exact_norm(st, st["k"], st["wk"], st["bk"], st["gk"])
        return dict(dq=dq, dk=dk, dwq=dwq, dwk=dwk, dbq=dbq, dbk=dbk)
    return _exact_attn(st)
