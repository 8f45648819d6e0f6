"""Attention of the visible pairs, forward and backward, against float64 on the same inputs.

Tolerances, element by element.  With bf16 inputs the probabilities and dS are rounded once for their products (half a step,
r = 2^-8 of each) and every output once more; e = 2^-13 covers the fp32 arithmetic: a logit is a sum of at most 128 products,
off by 128 * 2^-24 of the sum of their sizes, which is below 10 here (2^-13 of a probability), and so are dP and delta.  delta
is taken from a ctx that has the error of the rounded probabilities (and of its own rounding without ctx32).  These bounds add
all errors up; so each row of a head is also held to 4 r (fp32: 4 e) of its norm, which a lost or an extra pair would not pass."""
import math

import pytest
import torch

from paper_2007_01045_amd import binding as B

pytestmark = pytest.mark.gpu
TD = {B.DTYPE_F32: torch.float32, B.DTYPE_BF16: torch.bfloat16}
GUARD = 7.0


def normal(seed, *shape):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(*shape, generator=g, device="cuda")


class Case:
    """Packed q, k, v [b s, ld] with `pad` columns behind them, likewise the gradients; what lies behind a sequence's end is NaN."""

    def __init__(self, dtype, b, s, A, Ak, d, W=0, S=0, causal=False, lens=None, scale=0.0, ctx32=True, pad=8, seed=1):
        self.__dict__.update(locals())
        td, self.rows, self.ld, self.ldc = TD[dtype], b * s, (A + 2 * Ak) * d + pad, A * d + pad
        self.qkv, self.dctx = normal(seed, self.rows, self.ld).to(td), normal(seed + 1, self.rows, self.ldc).to(td)
        self.n = [s] * b if lens is None else [min(max(x, 0), s) for x in lens]
        self.lens_dev = None if lens is None else torch.tensor(lens, dtype=torch.int32, device="cuda")
        for i, n in enumerate(self.n):
            self.qkv[i * s + n:(i + 1) * s] = math.nan
            self.dctx[i * s + n:(i + 1) * s] = math.nan
        self.ctx = torch.full((self.rows, self.ldc), GUARD, device="cuda").to(td)
        self.c32 = torch.full((self.rows, self.ldc), GUARD, device="cuda")
        self.lse = torch.full((b, A, s), GUARD, device="cuda")
        self.dqkv = torch.full((self.rows, self.ld), GUARD, device="cuda").to(td)

    def desc(self):
        es, (A, Ak, d) = self.qkv.element_size(), (self.A, self.Ak, self.d)
        x, g = self.qkv.data_ptr(), self.dqkv.data_ptr()
        k, v = A * d * es, (A + Ak) * d * es
        t = B.attention_window_desc(q=x, k=x + k, v=x + v, ctx=self.ctx.data_ptr(), ctx32=self.c32.data_ptr() if self.ctx32 else None,
                                    lse=self.lse.data_ptr(), lens=None if self.lens is None else self.lens_dev.data_ptr(),
                                    dctx=self.dctx.data_ptr(), dq=g, dk=g + k, dv=g + v, b=self.b, s=self.s, A=A, Ak=Ak, d=d,
                                    window=self.W, sinks=self.S, causal=int(self.causal), ldq=self.ld, ldk=self.ld, ldv=self.ld,
                                    ldc=self.ldc, lddc=self.ldc, lddq=self.ld, lddk=self.ld, lddv=self.ld, scale=self.scale)
        self.ws = torch.full((B.dapple_attention_window_workspace(self.dtype, t),), 0xff, dtype=torch.uint8, device="cuda")
        t.workspace = self.ws.data_ptr()
        return t

    def run(self, stream=None):
        t = self.desc()
        B.dapple_attention_window_fwd(self.dtype, t, stream)
        B.dapple_attention_window_bwd(self.dtype, t, stream)

    def check(self):
        b, s, A, Ak, d, G = self.b, self.s, self.A, self.Ak, self.d, self.A // self.Ak
        bf = self.dtype == B.DTYPE_BF16
        r, e = (2.0 ** -8 if bf else 0.0), 2.0 ** -13
        rc = r if self.ctx32 or not bf else 2 * r
        scale = self.scale or d ** -0.5
        for t, n in ((self.ctx, A * d), (self.dqkv, (A + 2 * Ak) * d)) + (((self.c32, A * d),) if self.ctx32 else ()):
            assert bool((t[:, n:] == GUARD).all()), "a column between the rows was written"
        for bi, n in enumerate(self.n):
            rows = slice(bi * s, bi * s + n)
            for t, w in ((self.ctx, A * d), (self.dqkv, (A + 2 * Ak) * d)) + (((self.c32, A * d),) if self.ctx32 else ()):
                assert bool((t[bi * s + n:(bi + 1) * s, :w] == 0).all()), "a row behind the end is not zero"
            assert bool((self.lse[bi, :, n:] == -math.inf).all())
            if n == 0:
                continue
            i, j = torch.arange(n, device="cuda")[:, None], torch.arange(n, device="cuda")[None, :]
            ok = torch.ones(n, n, dtype=torch.bool, device="cuda")
            if self.W:
                ok = ((i - j).abs() < self.W) | (j < self.S)
            if self.causal:
                ok &= j <= i
            part = lambda t, at, heads: t[rows, at * d:(at + heads) * d].double().view(n, heads, d).transpose(0, 1)  # noqa: E731
            q, k, v = part(self.qkv, 0, A), part(self.qkv, A, Ak), part(self.qkv, A + Ak, Ak)
            g = part(self.dctx, 0, A)
            k, v = (x.repeat_interleave(G, 0) for x in (k, v))
            mm = lambda x, y: x @ y.transpose(1, 2).contiguous()  # noqa: E731
            tt = lambda x, y: x.transpose(1, 2).contiguous() @ y  # noqa: E731
            t = (mm(q, k) * scale).masked_fill(~ok, -math.inf)
            lse = torch.logsumexp(t, -1)
            p = torch.exp(t - lse[..., None])
            pv = p @ v.abs()
            ctx = p @ v
            self.close("ctx", part(self.ctx, 0, A), ctx, (r + e) * pv + r * ctx.abs(), 4 * max(r, e))
            if self.ctx32:
                self.close("ctx32", part(self.c32, 0, A), ctx, (r + e) * pv, 4 * max(r, e))
            assert float((self.lse[bi, :, :n].double() - lse / math.log(2)).abs().max()) < 2 * e
            dabs = (g.abs() * pv).sum(-1, keepdim=True)
            ds = p * (mm(g, v) - (g * ctx).sum(-1, keepdim=True))
            err = (r + e) * ds.abs() + p * (e * mm(g.abs(), v.abs()) + (rc + e) * dabs)
            share = lambda x: x.view(Ak, G, n, d).sum(1)  # noqa: E731
            dq, dk, dv = scale * (ds @ k), scale * share(tt(ds, q)), share(tt(p, g))
            self.close("dq", part(self.dqkv, 0, A), dq, scale * (err @ k.abs()) + r * dq.abs(), 4 * max(rc, e))
            self.close("dk", part(self.dqkv, A, Ak), dk, scale * share(tt(err, q.abs())) + r * dk.abs(), 4 * max(rc, e))
            self.close("dv", part(self.dqkv, A + Ak, Ak), dv, (r + e) * share(tt(p, g.abs())) + r * dv.abs(), 4 * max(r, e))

    def close(self, what, got, want, tol, row):
        off = (got - want).abs()
        assert bool((off <= tol + 1e-12).all()), (what, float((off / (tol + 1e-12)).max()))
        norm = want.square().sum(-1).sqrt()
        rms = float(norm.square().mean().sqrt())
        if rms > 1e-3:      # (a row that sees itself alone has dq = 0)
            far = off.square().sum(-1).sqrt() - row * (norm + rms)
            assert float(far.max()) <= 0, (what, "row", int(far.argmax()))


F, H = B.DTYPE_F32, B.DTYPE_BF16
CASES = [  # dtype, b, s, A, Ak, d, W, S, causal, lens
    (H, 1, 1, 1, 1, 64, 0, 0, True, None), (H, 2, 2, 2, 1, 64, 1, 0, True, None), (H, 1, 63, 2, 2, 32, 7, 0, True, None),
    (H, 1, 64, 1, 1, 64, 0, 0, True, None), (H, 2, 65, 2, 1, 128, 16, 1, True, None), (H, 1, 127, 4, 4, 64, 0, 0, False, None),
    (H, 3, 130, 6, 2, 64, 33, 5, False, [130, 1, 77]), (H, 2, 200, 4, 1, 80, 64, 64, True, [0, 200]),
    (H, 2, 517, 4, 2, 64, 100, 3, True, None), (H, 2, 517, 4, 2, 64, 100, 70, False, [517, 400]), (H, 1, 700, 8, 1, 128, 129, 130, True, [650]),
    (H, 4, 333, 3, 3, 8, 40, 2, False, [333, 64, 65, 2]), (H, 1, 300, 2, 2, 96, 64, 0, True, None), (H, 1, 260, 5, 5, 40, 300, 7, False, None),
    (H, 16, 517, 8, 8, 64, 50, 4, True, None), (H, 2, 1030, 16, 4, 128, 256, 16, True, None), (H, 9, 140, 16, 16, 128, 1, 3, False, None),
    (H, 2, 385, 4, 4, 32, 64, 200, True, [385, 192]), (H, 1, 2100, 4, 2, 64, 0, 0, True, None), (H, 1, 2100, 2, 1, 64, 300, 1, False, [2099]),
    (H, 4, 530, 32, 8, 128, 150, 20, True, [530, 1, 300, 511]), (H, 2, 1100, 28, 28, 104, 0, 0, True, None), (H, 3, 700, 32, 4, 72, 64, 0, False, None),
    (F, 1, 1, 1, 1, 16, 0, 0, True, None), (F, 2, 33, 2, 1, 4, 5, 1, True, None), (F, 1, 64, 2, 2, 64, 0, 0, False, None),
    (F, 3, 130, 6, 2, 64, 33, 5, False, [130, 1, 77]), (F, 2, 200, 4, 1, 80, 64, 64, True, [0, 200]), (F, 2, 517, 4, 2, 20, 100, 3, True, None),
    (F, 1, 700, 8, 1, 128, 129, 130, True, [650]), (F, 18, 260, 4, 4, 32, 50, 4, True, None), (F, 2, 333, 3, 3, 36, 40, 100, False, [333, 64]),
]


@pytest.mark.parametrize("case", CASES, ids=lambda c: "-".join("x" if v is None else str(v).replace(", ", "_") for v in c))
def test_forward_and_backward(case):
    c = Case(*case)
    c.run()
    c.check()


@pytest.mark.parametrize("dtype", [F, H])
def test_scale_and_bf16_ctx_alone(dtype):
    c = Case(dtype, 2, 150, 4, 2, 64, 40, 3, True, scale=0.05, ctx32=False)
    c.run()
    c.check()
    assert bool((c.c32 == GUARD).all())


@pytest.mark.parametrize("dtype", [F, H])
def test_lengths_outside_the_sequence_are_clamped(dtype):
    c = Case(dtype, 3, 70, 2, 1, 64, 20, 2, True, lens=[-5, 1000, 69])
    c.run()
    c.check()


@pytest.mark.parametrize("dtype", [F, H])
def test_large_logits(dtype):
    # logits of several hundred, and rows whose maximum comes late: the running maximum carries
    c = Case(dtype, 1, 300, 2, 2, 64, 90, 4, True)
    c.qkv[:, :128] *= torch.linspace(0.5, 20, 300, device="cuda")[:, None].to(c.qkv.dtype)
    t = c.desc()
    B.dapple_attention_window_fwd(dtype, t)
    q, k, v = (c.qkv[:, at * 64:(at + 2) * 64].double().view(300, 2, 64).transpose(0, 1) for at in (0, 2, 4))
    i = torch.arange(300, device="cuda")
    ok = (i[None] <= i[:, None]) & ((i[:, None] - i[None] < 90) | (i[None] < 4))
    logits = q @ k.transpose(1, 2).contiguous() / 8
    p = torch.softmax(logits.masked_fill(~ok, -math.inf), -1)
    # a logit of size x is off by 64 * 2^-24 of the sum of its products' sizes, a probability by that factor
    far = 2.0 ** -18 * (q.abs() @ k.abs().transpose(1, 2).contiguous() / 8).amax(-1, keepdim=True)
    r = 2.0 ** -8 if dtype == H else 0.0
    got = c.ctx[:, :128].double().view(300, 2, 64).transpose(0, 1)
    want = p @ v
    assert bool(((got - want).abs() <= (2 * far + r + 2.0 ** -13) * (p @ v.abs()) + r * want.abs()).all())


def test_gradient_against_differences():
    # fp32; the quotient's error: h^2 of the third derivative's part, and the roundings of a sum of about 50 over h
    c = Case(F, 1, 20, 2, 1, 8, 6, 2, True, pad=0)
    c.run()
    grad, x0, h = c.dqkv.clone(), c.qkv.clone(), 2.0 ** -6
    t = c.desc()

    def f():
        B.dapple_attention_window_fwd(F, t)
        return float((c.ctx.double() * c.dctx.double()).sum())

    for row, col in ((0, 3), (7, 9), (0, 17), (13, 20), (19, 25), (5, 30)):
        vals = []
        for sgn in (1, -1):
            c.qkv.copy_(x0)
            c.qkv[row, col] += sgn * h
            vals.append(f())
        c.qkv.copy_(x0)
        assert abs((vals[0] - vals[1]) / (2 * h) - float(grad[row, col])) < 20 * h * h + 2.0 ** -24 * 200 / h


def test_offsets_beyond_32_bits():
    b, s, ld, d = 3, 200, 5_000_000, 64      # the last sequence begins past 2^31 elements (6 GB)
    x = torch.empty(b * s, ld, dtype=torch.bfloat16, device="cuda")
    at = ld - 3 * d
    small = normal(3, b * s, 3 * d).bfloat16()
    x[:, at:] = small
    ctx, lse = torch.empty(b * s, d, dtype=torch.bfloat16, device="cuda"), torch.empty(b, 1, s, device="cuda")
    want, lse2 = torch.empty_like(ctx), torch.empty_like(lse)
    p = x.data_ptr() + at * 2
    kw = dict(b=b, s=s, A=1, Ak=1, d=d, window=50, sinks=2, causal=1)
    B.dapple_attention_window_fwd(H, B.attention_window_desc(q=p, k=p + 2 * d, v=p + 4 * d, ctx=ctx.data_ptr(), lse=lse.data_ptr(),
                                                             ldq=ld, ldk=ld, ldv=ld, **kw))
    p = small.data_ptr()
    B.dapple_attention_window_fwd(H, B.attention_window_desc(q=p, k=p + 2 * d, v=p + 4 * d, ctx=want.data_ptr(), lse=lse2.data_ptr(),
                                                             ldq=3 * d, ldk=3 * d, ldv=3 * d, **kw))
    assert torch.equal(ctx, want) and torch.equal(lse, lse2)


@pytest.mark.parametrize("dtype", [F, H])
def test_same_bits_on_another_stream_and_in_a_graph(dtype):
    c = Case(dtype, 2, 400, 8, 2, 64, 70, 9, True, lens=[400, 311])
    c.run()
    torch.cuda.synchronize()
    outs = (c.ctx, c.c32, c.lse, c.dqkv)
    want = [t.clone() for t in outs]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        c.run(side.cuda_stream)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(outs, want))
    t = c.desc()

    def run():
        sp = torch.cuda.current_stream().cuda_stream
        B.dapple_attention_window_fwd(dtype, t, sp)
        B.dapple_attention_window_bwd(dtype, t, sp)

    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    for k in range(3):
        c.qkv.mul_(-0.75)
        run()
        torch.cuda.synchronize()
        eager = [x.clone() for x in outs]
        for x in outs:
            x.fill_(GUARD)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip([x[:, :c.A * c.d] if x.dim() == 2 else x for x in outs],
                                                     [x[:, :c.A * c.d] if x.dim() == 2 else x for x in eager])), k
        assert torch.equal(c.dqkv[:, :c.ld - c.pad], eager[3][:, :c.ld - c.pad]), k


@pytest.mark.parametrize("case", [  # many tiles of sinks: their walks in parts of their own length, or whole, beside whole and cut ones
    (H, 4, 1500, 16, 16, 64, 64, 700, True, [1500, 3, 1111, 699]), (H, 4, 1500, 16, 16, 64, 64, 1400, True, None),
    (H, 2, 1500, 32, 8, 128, 64, 600, True, [1500, 900]), (H, 1, 1300, 4, 2, 128, 64, 600, False, None), (H, 1, 2500, 2, 2, 32, 500, 1500, True, None),
    (F, 2, 700, 8, 4, 32, 40, 300, False, [700, 301]), (F, 3, 900, 8, 8, 64, 30, 860, True, None)],
    ids=lambda c: "-".join("x" if v is None else str(v).replace(", ", "_") for v in c))
def test_many_sinks(case):
    c = Case(*case)
    c.run()
    c.check()


@pytest.mark.parametrize("case", [  # fp32 in groups of four waves: from 512 tiles of 64 rows on, a wide head's forward from 192 on
    (F, 4, 260, 32, 8, 32, 50, 4, True, [260, 0, 77, 259]), (F, 4, 260, 32, 32, 16, 0, 0, False, None), (F, 3, 450, 24, 8, 64, 100, 7, False, [450, 64, 333]),
    (F, 2, 330, 48, 16, 128, 70, 3, True, None), (F, 3, 333, 12, 4, 128, 40, 2, True, [333, 1, 200]), (F, 3, 333, 12, 12, 72, 0, 0, False, None),
    # and with walks of few key heads in parts: fp32, and bf16 in workgroups of four waves
    (F, 1, 600, 64, 2, 36, 0, 0, True, None), (F, 1, 600, 64, 2, 128, 200, 70, False, [577]), (F, 2, 300, 64, 2, 64, 60, 1, True, [300, 131]),
    (H, 1, 600, 64, 2, 64, 0, 0, True, None), (H, 1, 600, 64, 2, 64, 200, 130, False, [577]), (H, 2, 300, 64, 2, 32, 60, 1, True, [300, 131])],
    ids=lambda c: "-".join("x" if v is None else str(v).replace(", ", "_") for v in c))
def test_many_tiles(case):
    c = Case(*case)
    c.run()
    c.check()
