"""Single operators of a transformer layer and of a training step, as cases that can be timed: through the binding's entry
points where `own` is true, else in their plain form in elementary torch operations.

A case's `op` and what one pass of it is:
  qk_rope     RMS norm of every query and key head and the rotation by position, of a packed projection [rows, (A + 2 Ak) d];
              with `train` the gradient behind it too
  attention   softmax attention of the visible pairs: a window of W positions (0 = all), S first tokens that stay visible,
              causal or not, A query heads on Ak key heads, sequences of their own lengths (`ragged`); with `train` the
              gradients behind it too
  clip        the global norm of a list of gradients, and the clipped gradients (the tensors of L encoder layers of H, F)
  gated_ffn   y = (act(x Wg + bg) * (x Wu + bu)) Wo + bo; with `train` the gradients behind it too
dtype: "f32" or "bf16", of every tensor but the statistics."""
import math

import numpy as np
import torch

own = False

DEVICE = "cuda:0"
EPS = 1e-6
MAX_NORM = 1.0
TABLE = 16384            # positions of the rotation table


def _rope(name, dtype, rows, A, Ak, d, rot, half, norm, train):
    c = dict(op="qk_rope", dtype=dtype, rows=rows, A=A, Ak=Ak, d=d, rot=rot, half=half, norm=norm, train=train)
    return dict(c, name=name) if name else c


def _attn(name, dtype, b, s, A, Ak, d, W, S, causal, ragged, train):
    c = dict(op="attention", dtype=dtype, b=b, s=s, A=A, Ak=Ak, d=d, W=W, S=S, causal=causal, ragged=ragged, train=train)
    return dict(c, name=name) if name else c


def _clip(name, dtype, L, H, F, sigma):
    c = dict(op="clip", dtype=dtype, L=L, H=H, F=F, sigma=sigma)
    return dict(c, name=name) if name else c


def _ffn(name, dtype, T, H, F, act, train):
    c = dict(op="gated_ffn", dtype=dtype, T=T, H=H, F=F, act=act, train=train)
    return dict(c, name=name) if name else c


def listed():
    return [
        # a short prompt's rows: a launch's latency
        _rope("rope_16_rows", "bf16", 16, 16, 16, 64, 64, True, True, False),
        # one task of a stage trained on long sequences, with shared key heads
        _rope("rope_train_32k", "bf16", 32768, 32, 8, 128, 128, True, True, True),
        # fp32, interleaved pairs, a part of the head, an odd number of rows
        _rope("rope_train_f32_part", "f32", 3001, 12, 4, 64, 32, False, True, True),
        # one sample of the short sequences the encoder stages have (heads of 64)
        _attn("attn_512", "bf16", 1, 512, 16, 16, 64, 128, 4, True, False, False),
        # a micro-batch of encoder sequences of different lengths, local attention with global first tokens
        _attn("attn_train_local", "bf16", 4, 1987, 16, 16, 64, 256, 8, False, True, True),
        # a long sequence with shared key heads
        _attn("attn_train_8k", "bf16", 1, 8192, 16, 4, 128, 1024, 16, True, False, True),
        # an fp32 stage
        _attn("attn_train_f32", "f32", 2, 777, 12, 6, 64, 200, 1, True, True, True),
        # the gradients of a small stage
        _clip("clip_small", "f32", 2, 256, 1024, 0.01),
        # all layers of a 24-layer encoder 1024 wide: 302M gradients
        _clip("clip_24_layers", "f32", 24, 1024, 4096, 0.01),
        # few rows: the weights are what is read
        _ffn("ffn_16_rows", "bf16", 16, 1024, 4096, "silu", False),
        # one task of four micro-batches of a wide layer
        _ffn("ffn_train_8k", "bf16", 8192, 2048, 8192, "silu", True),
        # an fp32 stage, ragged sizes
        _ffn("ffn_train_f32", "f32", 1000, 768, 2040, "gelu", True),
    ]


def draw(rng):
    def logint(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    op = rng.choice(["qk_rope", "attention", "attention", "clip", "gated_ffn"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    train = rng.random() < 0.6
    if op == "qk_rope":
        d = rng.choice([32, 64, 64, 80, 96, 128, 128, 256])
        Ak = rng.choice([1, 2, 4, 8])
        A = Ak * rng.choice([1, 2, 4])
        rot = rng.choice([d, d, d // 2])
        rows = min(logint(1, 32768), 32768 * 40 * 128 // ((A + Ak) * d))
        return _rope("", dtype, rows, A, Ak, d, rot, rng.random() < 0.5, rng.random() < 0.8, train)
    if op == "attention":
        d = rng.choice([32, 64, 64, 80, 128])
        Ak = rng.choice([1, 2, 4, 8])
        A = Ak * rng.choice([1, 2, 4])
        s = logint(24, 6000)
        b = rng.choice([1, 2, 3, 4])
        while b * A * s * s > 16 * 8192 ** 2 // (4 if dtype == "f32" else 2):
            if b > 1:
                b -= 1
            else:
                s = s * 3 // 4
        W = rng.choice([0, logint(16, 2048), logint(16, 2048)])
        return _attn("", dtype, b, s, A, Ak, d, W, rng.choice([0, 1, 4, 17, 64]), rng.random() < 0.7, rng.random() < 0.4, train)
    if op == "clip":
        return _clip("", dtype, rng.randint(1, 6), 8 * logint(8, 128), logint(100, 5000), rng.choice([1e-5, 0.01, 0.3]))
    H, F = 8 * logint(16, 256), 8 * logint(32, 1024)
    T = min(logint(1, 8192), 8192 * 2048 * 8192 // (H * F) // (8 if dtype == "f32" else 1))
    return _ffn("", dtype, T, H, F, rng.choice(["silu", "gelu"]), train)


# ---------------------------------------------------------------- inputs
def _type(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _size(case):
    return 2 if case["dtype"] == "bf16" else 4


def layer_shapes(L, H, F):
    """The tensors of L encoder layers, in the order a stage holds them."""
    one = [(H, H), (H,)] * 4 + [(H,), (H,), (H, F), (F,), (F, H), (H,), (H,), (H,)]
    return one * L


def prepare(case, seed):
    g = torch.Generator(device=DEVICE).manual_seed(seed)
    dt = _type(case)

    def normal(*shape, scale=1.0, mean=0.0, t=dt):
        return (torch.randn(*shape, generator=g, device=DEVICE) * scale + mean).to(t)

    def room(*shape, t=dt):
        return torch.empty(*shape, dtype=t, device=DEVICE)

    st = dict(case=case)
    op = case["op"]
    if op == "qk_rope":
        rows, A, Ak, d, rot = (case[k] for k in ("rows", "A", "Ak", "d", "rot"))
        st["x"] = normal(rows, (A + 2 * Ak) * d)
        st["gq"], st["gk"] = normal(d, scale=0.2, mean=1.0), normal(d, scale=0.2, mean=1.0)
        st["pos"] = torch.randint(0, TABLE, (rows,), generator=g, device=DEVICE, dtype=torch.int32)
        inv = 10000.0 ** (-2.0 * torch.arange(rot // 2, device=DEVICE, dtype=torch.float64) / rot)
        angle = torch.arange(TABLE, device=DEVICE, dtype=torch.float64)[:, None] * inv
        st["table"] = torch.stack([angle.cos(), angle.sin()], dim=-1).float().contiguous()     # [positions, rot / 2, 2]
        st["y"] = room(rows, (A + Ak) * d)
        if case["train"]:
            st["dy"] = normal(rows, (A + Ak) * d)
            st["dx"] = room(rows, (A + Ak) * d)
            st["dgq"], st["dgk"] = room(d, t=torch.float32), room(d, t=torch.float32)
    elif op == "attention":
        b, s, A, Ak, d = (case[k] for k in ("b", "s", "A", "Ak", "d"))
        st["qkv"] = normal(b * s, (A + 2 * Ak) * d)
        lens = torch.randint(max(1, s // 2), s + 1, (b,), generator=g, device=DEVICE, dtype=torch.int32)
        lens[0] = s
        st["lens"] = lens if case["ragged"] else None
        st["ctx"] = room(b * s, A * d)
        st["lse"] = room(b, A, s, t=torch.float32)
        if case["train"]:
            st["dctx"] = normal(b * s, A * d)
            st["ctx32"] = room(b * s, A * d, t=torch.float32)
            st["dqkv"] = room(b * s, (A + 2 * Ak) * d)
    elif op == "clip":
        shapes = layer_shapes(case["L"], case["H"], case["F"])
        sizes = [math.prod(x) for x in shapes]
        st["flat"] = normal(sum(sizes), scale=case["sigma"])
        st["out"] = room(sum(sizes))
        st["grads"] = [x.view(sh) for x, sh in zip(st["flat"].split(sizes), shapes)]
        st["clipped"] = [x.view(sh) for x, sh in zip(st["out"].split(sizes), shapes)]
        st["norm"] = room(2, t=torch.float32)
    else:
        T, H, F = (case[k] for k in ("T", "H", "F"))
        st["x"] = normal(T, H)
        st["w_in"], st["b_in"] = normal(H, 2 * F, scale=0.02), normal(2 * F, scale=0.02)
        st["w_out"], st["b_out"] = normal(F, H, scale=0.02), normal(H, scale=0.02)
        st["y"], st["h"] = room(T, H), room(T, F)
        if case["train"]:
            st["dy"] = normal(T, H)
            st["gu"], st["dgu"], st["dx"] = room(T, 2 * F), room(T, 2 * F), room(T, H)
            st["dw_in"], st["db_in"], st["dw_out"], st["db_out"] = room(H, 2 * F), room(2 * F), room(F, H), room(H)
    return st


# ---------------------------------------------------------------- one pass
def run(st):
    op = st["case"]["op"]
    if own:
        return dict(qk_rope=_own_rope, attention=_own_attention, clip=_own_clip, gated_ffn=_own_ffn)[op](st)
    return dict(qk_rope=_plain_rope, attention=_plain_attention, clip=_plain_clip, gated_ffn=_plain_ffn)[op](st)


def _rotate(n, c, s, half):
    """n [..., rot]: every pair (a, b) to (a c - b s, a s + b c)."""
    if half:
        a, b = n.chunk(2, dim=-1)
        return torch.cat([a * c - b * s, a * s + b * c], dim=-1)
    a, b = n[..., 0::2], n[..., 1::2]
    return torch.stack([a * c - b * s, a * s + b * c], dim=-1).flatten(-2)


def _plain_rope(st):
    case = st["case"]
    rows, A, Ak, d, rot, half = (case[k] for k in ("rows", "A", "Ak", "d", "rot", "half"))
    x = st["x"][:, : (A + Ak) * d].float().view(rows, A + Ak, d)
    cs = st["table"][st["pos"].long()]
    c, s = cs[:, None, :, 0], cs[:, None, :, 1]
    gamma = torch.cat([st["gq"].float().expand(A, d), st["gk"].float().expand(Ak, d)])
    rstd = (x.square().mean(-1, keepdim=True) + EPS).rsqrt()
    n = x * rstd * gamma if case["norm"] else x
    y = torch.cat([_rotate(n[..., :rot], c, s, half), n[..., rot:]], dim=-1)
    out = [y.reshape(rows, -1).to(st["x"].dtype)]
    if case["train"]:
        dy = st["dy"].float().view(rows, A + Ak, d)
        dn = torch.cat([_rotate(dy[..., :rot], c, -s, half), dy[..., rot:]], dim=-1)
        if case["norm"]:
            xh = x * rstd
            dg = (dn * xh).sum(0)
            t = dn * gamma
            dx = rstd * (t - xh * (t * xh).mean(-1, keepdim=True))
            out += [dx.reshape(rows, -1).to(st["x"].dtype), dg[:A].sum(0), dg[A:].sum(0)]
        else:
            out += [dn.reshape(rows, -1).to(st["x"].dtype)]
    return out


def _own_rope(st):
    from paper_2007_01045_amd import binding as B
    case = st["case"]
    rows, A, Ak, d = (case[k] for k in ("rows", "A", "Ak", "d"))
    es, x, y = _size(case), st["x"].data_ptr(), st["y"].data_ptr()
    dtype = B.DTYPE_BF16 if case["dtype"] == "bf16" else B.DTYPE_F32
    norm = case["norm"]
    stream = torch.cuda.current_stream().cuda_stream
    common = dict(rows=rows, A=A, Ak=Ak, d=d, rot=case["rot"], interleaved=int(not case["half"]), eps=EPS,
                  q=x, k=x + A * d * es, ldq=(A + 2 * Ak) * d, ldk=(A + 2 * Ak) * d,
                  gamma_q=st["gq"].data_ptr() if norm else None, gamma_k=st["gk"].data_ptr() if norm else None,
                  positions=st["pos"].data_ptr(), table=st["table"].data_ptr(), max_pos=TABLE)
    ld = (A + Ak) * d
    B.dapple_qk_rope_fwd(dtype, B.qk_rope_desc(yq=y, yk=y + A * d * es, ldyq=ld, ldyk=ld, **common), stream)
    out = [st["y"]]
    if case["train"]:
        dy, dx = st["dy"].data_ptr(), st["dx"].data_ptr()
        desc = B.qk_rope_desc(dyq=dy, dyk=dy + A * d * es, lddyq=ld, lddyk=ld, dq=dx, dk=dx + A * d * es, lddq=ld, lddk=ld,
                              dgamma_q=st["dgq"].data_ptr() if norm else None,
                              dgamma_k=st["dgk"].data_ptr() if norm else None, **common)
        ws = torch.empty(B.dapple_qk_rope_workspace(dtype, desc), dtype=torch.uint8, device=DEVICE)
        desc.workspace = ws.data_ptr()
        B.dapple_qk_rope_bwd(dtype, desc, stream)
        out += [st["dx"], st["dgq"], st["dgk"]] if norm else [st["dx"]]
    return out


def _visible(case, lens):
    """[b or 1, s, s]: whether query i sees key j."""
    s, W, S = case["s"], case["W"], case["S"]
    i, j = torch.arange(s, device=DEVICE)[:, None], torch.arange(s, device=DEVICE)[None, :]
    ok = torch.ones(s, s, dtype=torch.bool, device=DEVICE)
    if W:
        ok = ((i - j).abs() < W) | (j < S)
    if case["causal"]:
        ok = ok & (j <= i)
    ok = ok[None]
    if lens is not None:
        ok = ok & (i < lens[:, None, None]) & (j < lens[:, None, None])
    return ok


def _plain_attention(st):
    case = st["case"]
    b, s, A, Ak, d = (case[k] for k in ("b", "s", "A", "Ak", "d"))
    G, dt = A // Ak, st["qkv"].dtype
    q, k, v = (t.float().view(b, s, -1, d).transpose(1, 2) for t in st["qkv"].split([A * d, Ak * d, Ak * d], dim=1))
    q = q.reshape(b, Ak, G * s, d)                     # the G query heads of a key head one behind the other
    k, v = k.contiguous(), v.contiguous()
    scale = d ** -0.5
    hide = ~_visible(case, st["lens"])[:, None, None]
    t = (q @ k.transpose(-1, -2)).view(b, Ak, G, s, s).mul_(scale).masked_fill_(hide, -math.inf)
    top = t.amax(-1, keepdim=True).clamp_min(-1e30)    # (a row that sees nothing)
    p = t.sub_(top).exp_()
    z = p.sum(-1, keepdim=True)
    lse = ((top + z.log()) * math.log2(math.e)).view(b, A, s)
    p.div_(z.clamp_min(1e-30))
    ctx = p.view(b, Ak, G * s, s) @ v

    def rows(t):                                       # [b, Ak, heads * s, d] -> [b s, heads d]
        return t.reshape(b, -1, s, d).transpose(1, 2).reshape(b * s, -1)

    out = [rows(ctx).to(dt), lse]
    if case["train"]:
        dc = st["dctx"].float().view(b, s, A, d).transpose(1, 2).reshape(b, Ak, G * s, d)
        seen = (~hide).any(-1).expand(b, 1, 1, s).expand(b, Ak, G, s).reshape(b, Ak, G * s, 1)
        dc = dc.masked_fill(~seen, 0.0)
        delta = (dc * ctx).sum(-1, keepdim=True)
        dv = p.view(b, Ak, G * s, s).transpose(-1, -2) @ dc
        ds = (dc @ v.transpose(-1, -2)).sub_(delta).mul_(p.view(b, Ak, G * s, s)).mul_(scale)
        dq, dk = ds @ k, ds.transpose(-1, -2) @ q
        out.append(torch.cat([rows(dq), rows(dk), rows(dv)], dim=1).to(dt))
    return out


def _own_attention(st):
    from paper_2007_01045_amd import binding as B
    case = st["case"]
    b, s, A, Ak, d = (case[k] for k in ("b", "s", "A", "Ak", "d"))
    dtype = B.DTYPE_BF16 if case["dtype"] == "bf16" else B.DTYPE_F32
    es, ld, x = _size(case), (A + 2 * Ak) * d, st["qkv"].data_ptr()
    train = case["train"]
    stream = torch.cuda.current_stream().cuda_stream
    desc = B.attention_window_desc(q=x, k=x + A * d * es, v=x + (A + Ak) * d * es, ctx=st["ctx"].data_ptr(), lse=st["lse"].data_ptr(),
                                   ctx32=st["ctx32"].data_ptr() if train else None,
                                   lens=st["lens"].data_ptr() if st["lens"] is not None else None,
                                   b=b, s=s, A=A, Ak=Ak, d=d, ldq=ld, ldk=ld, ldv=ld, window=case["W"], sinks=case["S"],
                                   causal=int(case["causal"]))
    B.dapple_attention_window_fwd(dtype, desc, stream)
    out = [st["ctx"], st["lse"]]
    if train:
        dx = st["dqkv"].data_ptr()
        desc.dctx, desc.dq, desc.dk, desc.dv = st["dctx"].data_ptr(), dx, dx + A * d * es, dx + (A + Ak) * d * es
        desc.lddq = desc.lddk = desc.lddv = ld
        ws = torch.empty(B.dapple_attention_window_workspace(dtype, desc), dtype=torch.uint8, device=DEVICE)
        desc.workspace = ws.data_ptr()
        B.dapple_attention_window_bwd(dtype, desc, stream)
        out.append(st["dqkv"])
    return out


def _plain_clip(st):
    norm = torch.stack([g.double().square().sum() for g in st["grads"]]).sum().sqrt()
    factor = (MAX_NORM / norm).clamp_max(1.0)
    clipped = torch.cat([(g.float() * factor.float()).reshape(-1) for g in st["grads"]])
    return [torch.stack([norm, factor]).float(), clipped.to(st["flat"].dtype)]


def _own_clip(st):
    from paper_2007_01045_amd import binding as B
    dtype = B.DTYPE_BF16 if st["case"]["dtype"] == "bf16" else B.DTYPE_F32
    stream = torch.cuda.current_stream().cuda_stream
    grads, sizes = [g.data_ptr() for g in st["grads"]], [g.numel() for g in st["grads"]]
    ws = torch.empty(B.dapple_grad_norm_workspace(sizes), dtype=torch.uint8, device=DEVICE)
    B.dapple_grad_norm(dtype, grads, sizes, MAX_NORM, st["norm"].data_ptr(), ws.data_ptr(), stream_ptr=stream)
    B.dapple_grad_clip(dtype, grads, [g.data_ptr() for g in st["clipped"]], sizes, st["norm"].data_ptr(), stream)
    return [st["norm"], st["out"]]


def _act(g, kind):
    """The activation and its derivative."""
    if kind == "silu":
        f = torch.sigmoid(g)
        return g * f, f * (1 + g * (1 - f))
    f = 0.5 * (1 + torch.erf(g * 0.5 ** 0.5))
    return g * f, f + g * torch.exp(-0.5 * g * g) * (2 * math.pi) ** -0.5


def _plain_ffn(st):
    case = st["case"]
    dt = st["x"].dtype
    x, w_in, w_out = (st[k].float() for k in ("x", "w_in", "w_out"))
    g, u = (x @ w_in + st["b_in"].float()).chunk(2, dim=1)
    a, da = _act(g, case["act"])
    h = a * u
    out = [h @ w_out + st["b_out"].float()]
    if case["train"]:
        dy = st["dy"].float()
        dh = dy @ w_out.t()
        dgu = torch.cat([dh * u * da, dh * a], dim=1)
        out += [dgu @ w_in.t(), x.t() @ dgu, dgu.sum(0), h.t() @ dy, dy.sum(0)]
    return [t.to(dt) for t in out]


def _own_ffn(st):
    from paper_2007_01045_amd import binding as B
    case = st["case"]
    dtype = B.DTYPE_BF16 if case["dtype"] == "bf16" else B.DTYPE_F32
    stream = torch.cuda.current_stream().cuda_stream
    p = lambda *names: {n: st[n].data_ptr() for n in names}  # noqa: E731
    desc = B.gated_ffn_desc(T=case["T"], H=case["H"], F=case["F"], act=B.ACT_SILU if case["act"] == "silu" else B.ACT_GELU,
                            gu=st["gu"].data_ptr() if case["train"] else None,
                            **p("x", "w_in", "b_in", "w_out", "b_out", "h", "y"))
    B.dapple_gated_ffn_fwd(dtype, desc, stream)
    out = [st["y"]]
    if case["train"]:
        names = ("dx", "dw_in", "db_in", "dw_out", "db_out")
        desc.dy, desc.dgu = st["dy"].data_ptr(), st["dgu"].data_ptr()
        desc.dx, desc.dw_in, desc.db_in, desc.dw_out, desc.db_out = (st[n].data_ptr() for n in names)
        ws = torch.empty(B.dapple_gated_ffn_workspace(dtype, desc), dtype=torch.uint8, device=DEVICE)
        desc.workspace = ws.data_ptr()
        B.dapple_gated_ffn_bwd(dtype, desc, stream)
        out += [st[n] for n in names]
    return out


# ---------------------------------------------------------------- what a pass cannot do without
def _pairs(case):
    """Visible pairs of one full-length sequence and head."""
    s, W, S = case["s"], case["W"], case["S"]
    i = np.arange(s, dtype=np.int64)
    lo = np.maximum(0, i - W + 1) if W else np.zeros_like(i)
    hi = i + 1 if case["causal"] else (np.minimum(s, i + W) if W else np.full_like(i, s))
    first = np.minimum(np.minimum(lo, S), i + 1) if case["causal"] else np.minimum(lo, S)
    return int((hi - lo + first).sum())


def work(case):
    es, train = _size(case), case.get("train")
    if case["op"] == "qk_rope":
        n = case["rows"] * (case["A"] + case["Ak"]) * case["d"]
        table = min(case["rows"], TABLE) * case["rot"] * 4
        return {"bytes": n * es * (4 if train else 2) + table + case["rows"] * 4, "flops": n * (20 if train else 8)}
    if case["op"] == "attention":
        b, s, A, Ak, d = (case[k] for k in ("b", "s", "A", "Ak", "d"))
        pairs = b * A * _pairs(case)
        if case["ragged"]:
            pairs = int(pairs * (0.75 * (b - 1) + 1) / b)
        io = b * s * (A + 2 * Ak) * d * es * (2 if train else 1) + b * s * A * d * es * (2 if train else 1) + b * A * s * 4
        return {"bytes": io, "flops": pairs * d * (14 if train else 4)}
    if case["op"] == "clip":
        n = sum(math.prod(x) for x in layer_shapes(case["L"], case["H"], case["F"]))
        return {"bytes": 2 * n * es + 8, "flops": 3 * n}
    T, H, F = (case[k] for k in ("T", "H", "F"))
    io = (2 * T * H + 3 * H * F + 2 * F + H) * es
    if train:
        io += (2 * T * H + 3 * H * F + 2 * F + H) * es
    return {"bytes": io, "flops": 6 * T * H * F * (3 if train else 1)}


# ---------------------------------------------------------------- the definitions in 64 bits
def exact(case, seed):
    st = prepare(case, seed)
    with torch.enable_grad():
        return dict(qk_rope=_exact_rope, attention=_exact_attention, clip=_exact_clip, gated_ffn=_exact_ffn)[case["op"]](st)


def _leaf(t):
    return t.detach().double().requires_grad_(True)


def _exact_rope(st):
    case = st["case"]
    rows, A, Ak, d, rot = (case[k] for k in ("rows", "A", "Ak", "d", "rot"))
    q, k, _ = st["x"].split([A * d, Ak * d, Ak * d], dim=1)
    cs = torch.view_as_complex(st["table"].double())[st["pos"].long()]          # e^(i angle)
    ys, dxs, dgs = [], [], []
    for t, gam, heads, at in ((q, st["gq"], A, 0), (k, st["gk"], Ak, A)):
        t, gam = _leaf(t), _leaf(gam)
        n = t.view(rows, heads, d)
        if case["norm"]:
            n = n / torch.sqrt((n * n).sum(-1, keepdim=True) / d + EPS) * gam
        r = n[..., :rot]
        pairs = r.unflatten(-1, (2, rot // 2)).transpose(-1, -2) if case["half"] else r.unflatten(-1, (rot // 2, 2))
        r = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * cs[:, None])
        r = (r.transpose(-1, -2) if case["half"] else r).flatten(-2)
        y = torch.cat([r, n[..., rot:]], dim=-1).reshape(rows, heads * d)
        ys.append(y.detach())
        if case["train"]:
            y.backward(st["dy"][:, at * d : (at + heads) * d].double())
            dxs.append(t.grad)
            dgs.append(gam.grad)
    out = [torch.cat(ys, dim=1)]
    if case["train"]:
        out += [torch.cat(dxs, dim=1)] + (dgs if case["norm"] else [])
    return out


def _exact_attention(st):
    case = st["case"]
    b, s, A, Ak, d = (case[k] for k in ("b", "s", "A", "Ak", "d"))
    x = _leaf(st["qkv"])
    ctx = torch.zeros(b * s, A * d, dtype=torch.float64, device=DEVICE)
    lse = torch.full((b, A, s), -math.inf, dtype=torch.float64, device=DEVICE)
    dx = torch.zeros_like(x)
    for i in range(b):
        n = int(st["lens"][i]) if case["ragged"] else s
        at = torch.arange(n, device=DEVICE)
        gap = at[:, None] - at[None, :]
        seen = torch.ones(n, n, dtype=torch.bool, device=DEVICE)
        if case["W"]:
            seen = torch.logical_or(gap.abs() < case["W"], (at < case["S"]).expand(n, n))
        if case["causal"]:
            seen = torch.logical_and(seen, gap >= 0)
        far = torch.where(seen, 0.0, -math.inf).double()
        for h in range(A):
            kv = h // (A // Ak)
            cols = [slice((o + c) * d, (o + c + 1) * d) for o, c in ((0, h), (A, kv), (A + Ak, kv))]
            q, k, v = (_leaf(x[i * s : i * s + n, c]) for c in cols)
            t = q @ k.t().contiguous() / math.sqrt(d) + far
            y = torch.softmax(t, dim=-1) @ v
            rows = slice(i * s, i * s + n)
            ctx[rows, h * d : (h + 1) * d] = y.detach()
            lse[i, h, :n] = torch.logsumexp(t.detach(), dim=-1) / math.log(2.0)
            if case["train"]:
                y.backward(st["dctx"][rows, h * d : (h + 1) * d].double())
                for c, t in zip(cols, (q, k, v)):
                    dx[rows, c] += t.grad
    return [ctx, lse] + ([dx] if case["train"] else [])


def _exact_clip(st):
    g = st["flat"].double()
    norm = torch.linalg.vector_norm(g)
    factor = MAX_NORM / max(MAX_NORM, float(norm))
    return [torch.tensor([float(norm), factor], dtype=torch.float64, device=DEVICE), g * factor]


def _exact_ffn(st):
    case = st["case"]
    F = case["F"]
    x, w_in, b_in, w_out, b_out = (_leaf(st[k]) for k in ("x", "w_in", "b_in", "w_out", "b_out"))
    g, u = x @ w_in[:, :F] + b_in[:F], x @ w_in[:, F:] + b_in[F:]
    a = g / (1 + torch.exp(-g)) if case["act"] == "silu" else g * torch.special.ndtr(g)
    y = (a * u) @ w_out + b_out
    out = [y.detach()]
    if case["train"]:
        y.backward(st["dy"].double())
        out += [x.grad, w_in.grad, b_in.grad, w_out.grad, b_out.grad]
    return out
