"""The gated feed-forward block, forward and backward, against float64 on the same inputs.

Tolerances, element by element: bf16 calls round g, u, h, dg, du and every bf16 output once (r = 2^-8 of each); a sum of n fp32
products is off by at most n 2^-24 of the sum of their sizes; the activation's functions by 2^-20 (1 + |g|).  Each error is carried
through the formulas with sizes in the place of values (act' and act'' are below 1.13 and 0.8 in size).  These bounds add
everything up; the 2-norm over a tensor is held to 6e-3 (fp32 2e-5) as the products' tests do."""
import math

import pytest
import torch

from paper_2007_01045_amd import binding as B

pytestmark = pytest.mark.gpu
TD = {B.DTYPE_F32: torch.float32, B.DTYPE_BF16: torch.bfloat16}
F32, BF = B.DTYPE_F32, B.DTYPE_BF16
GUARD = 7.0


def act_of(g, act):
    if act == B.ACT_SILU:
        f = torch.sigmoid(g)
        return g * f, f * (1 + g * (1 - f))
    f = torch.special.ndtr(g)
    return g * f, f + g * torch.exp(-0.5 * g * g) / math.sqrt(2 * math.pi)


class Case:
    def __init__(self, dtype, T, H, F, act=B.ACT_SILU, bias=True, pad=0, accumulate=0, dx=True, dw=True, keep=True, seed=1):
        self.__dict__.update(locals())
        td, self.ld = TD[dtype], H + pad
        gen = torch.Generator(device="cuda").manual_seed(seed)
        normal = lambda s, *n: (s * torch.randn(*n, generator=gen, device="cuda")).to(td)  # noqa: E731
        self.x, self.dy = normal(1, T, self.ld), normal(1, T, self.ld)
        self.x[:, H:] = math.nan
        self.dy[:, H:] = math.nan
        self.w_in, self.w_out = normal(H ** -0.5, H, 2 * F), normal(F ** -0.5, F, H)
        self.b_in, self.b_out = (normal(0.5, 2 * F), normal(0.5, H)) if bias else (None, None)
        full = lambda *n, t=td: torch.full(n, GUARD, device="cuda").to(t)  # noqa: E731
        self.gu, self.h, self.y = full(T, 2 * F), full(T, F), full(T, self.ld)
        self.dgu, self.out_dx = full(T, 2 * F), full(T, self.ld)
        gt = torch.float32 if accumulate else td
        self.grads = [full(H, 2 * F, t=gt), full(2 * F, t=gt), full(F, H, t=gt), full(H, t=gt)] if dw else [None] * 4

    def desc(self):
        p = lambda t: None if t is None else t.data_ptr()  # noqa: E731
        dw_in, db_in, dw_out, db_out = self.grads
        d = B.gated_ffn_desc(x=p(self.x), w_in=p(self.w_in), b_in=p(self.b_in), w_out=p(self.w_out), b_out=p(self.b_out),
                             gu=p(self.gu) if self.keep else None, h=p(self.h), y=p(self.y), dy=p(self.dy), dgu=p(self.dgu),
                             dx=p(self.out_dx) if self.dx else None, dw_in=p(dw_in), db_in=p(db_in) if self.bias else None, dw_out=p(dw_out),
                             db_out=p(db_out) if self.bias else None, T=self.T, H=self.H, F=self.F, act=self.act,
                             accumulate=self.accumulate, ldx=self.ld, ldy=self.ld, lddy=self.ld, lddx=self.ld)
        self.ws = torch.full((B.dapple_gated_ffn_workspace(self.dtype, d),), 0xff, dtype=torch.uint8, device="cuda")
        d.workspace = self.ws.data_ptr()
        return d

    def run(self, stream=None):
        d = self.desc()
        B.dapple_gated_ffn_fwd(self.dtype, d, stream)
        if self.keep:
            B.dapple_gated_ffn_bwd(self.dtype, d, stream)

    def close(self, what, got, want, tol):
        off = (got.double() - want).abs()
        assert bool((off <= tol + 1e-10).all()), (what, float((off / (tol + 1e-10)).max()))
        norm = float(want.norm())
        if norm > 1e-3 and want.numel() > 64:
            assert float(off.norm()) <= (2e-5 if self.dtype == F32 else 6e-3) * norm, (what, float(off.norm()) / norm)

    def check(self):
        T, H, F, r = self.T, self.H, self.F, (2.0 ** -8 if self.dtype == BF else 0.0)
        u24 = 2.0 ** -24
        x, dy = self.x[:, :H].double(), self.dy[:, :H].double()
        w_in, w_out = self.w_in.double(), self.w_out.double()
        b_in, b_out = (self.b_in.double(), self.b_out.double()) if self.bias else (0.0, 0.0)
        gu = x @ w_in + b_in
        egu = (H + 2) * u24 * (x.abs() @ w_in.abs() + (b_in.abs() if self.bias else 0.0))
        (g, u), (eg, eu) = gu.chunk(2, 1), egu.chunk(2, 1)
        a, da = act_of(g, self.act)
        ea = 2.0 ** -20 * (1 + g.abs())
        h = a * u
        eh = r * h.abs() + (1 + r) * ((ea + 1.13 * eg) * u.abs() + a.abs() * eu)
        y = h @ w_out + b_out
        ey = eh @ w_out.abs() + (F + 2) * u24 * (h.abs() @ w_out.abs() + (b_out.abs() if self.bias else 0.0)) + r * y.abs()
        self.close("y", self.y[:, :H], y, ey)
        self.close("h", self.h, h, eh)
        if not self.keep:
            assert bool((self.gu == GUARD).all())
            return
        self.close("gu", self.gu, gu, egu + r * gu.abs())
        dh = dy @ w_out.t().contiguous()
        edh = (H + 2) * u24 * (dy.abs() @ w_out.t().abs().contiguous())
        rg, ru = r * g.abs() + eg, r * u.abs() + eu          # of the g and u that the backward reads
        dg, du = dh * u * da, dh * a
        edg = edh * (u * da).abs() + dh.abs() * ((0.8 * rg + ea) * (u.abs() + ru) + da.abs() * ru) + r * dg.abs()
        edu = edh * a.abs() + dh.abs() * (1.13 * rg + ea) + r * du.abs()
        dgu, ed = torch.cat([dg, du], 1), torch.cat([edg, edu], 1) * (1 + r)
        self.close("dgu", self.dgu, dgu, ed)
        wt = w_in.t().contiguous()
        if self.dx:
            dx = dgu @ wt
            self.close("dx", self.out_dx[:, :H], dx, ed @ wt.abs() + (2 * F + 2) * u24 * (dgu.abs() @ wt.abs()) + r * dx.abs())
        for t in (self.y, self.out_dx):
            assert bool((t[:, H:] == GUARD).all()), "a column between the rows was written"
        if not self.dx:
            assert bool((self.out_dx == GUARD).all())
        if not self.dw:
            return
        rw, start = (0.0, GUARD) if self.accumulate else (r, 0.0)
        s = (T + 3) * u24
        for what, got, want, tol in (
                ("dw_in", self.grads[0], x.t().contiguous() @ dgu, x.abs().t().contiguous() @ (ed + s * dgu.abs())),
                ("db_in", self.grads[1], dgu.sum(0), (ed + s * dgu.abs()).sum(0)),
                ("dw_out", self.grads[2], h.t().contiguous() @ dy, (eh + s * h.abs()).t().contiguous() @ dy.abs()),
                ("db_out", self.grads[3], dy.sum(0), s * dy.abs().sum(0))):
            if what.startswith("db") and not self.bias:
                assert bool((got == GUARD).all())
            else:
                self.close(what, got, start + want, tol + rw * want.abs() + 2 * u24 * (start + want.abs()))


SHAPES = [(1, 8, 8), (5, 64, 128), (16, 128, 256), (33, 72, 40), (130, 64, 200), (300, 256, 512), (1000, 96, 1000), (1030, 128, 1544),
          (2049, 128, 264), (8200, 64, 1544), (8200, 72, 1544), (700, 1096, 96),
          (32, 1032, 520), (31, 264, 2056), (17, 2048, 40)]


@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "-".join(map(str, s)))
def test_forward_and_backward(dtype, shape):
    for kw in (dict(act=B.ACT_SILU), dict(act=B.ACT_GELU, pad=8, accumulate=1)):
        c = Case(dtype, *shape, **kw)
        c.run()
        c.check()


@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("kw", [dict(bias=False), dict(bias=False, accumulate=1), dict(dx=False), dict(dw=False), dict(keep=False),
                                dict(keep=False, bias=False), dict(act=B.ACT_GELU, keep=False, pad=16)], ids=str)
def test_what_is_not_wanted(dtype, kw):
    for shape in ((20, 64, 72), (520, 136, 200)):
        c = Case(dtype, *shape, **kw)
        c.run()
        c.check()


@pytest.mark.parametrize("shape", [(16, 40, 2048), (13, 64, 2056), (32, 72, 4168), (29, 4104, 16), (2, 4104, 8), (17, 64, 64)],
                         ids=lambda s: "-".join(map(str, s)))
def test_few_rows(shape):
    # depths of more and of less than a wave's part, columns that end inside sixteen
    for kw in (dict(pad=8), dict(act=B.ACT_GELU, bias=False), dict(keep=False)):
        c = Case(BF, *shape, **kw)
        c.run()
        c.check()


@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("accumulate", [0, 1])
def test_large_weight_gradients(dtype, accumulate):
    # bf16: tiles of 256x256 and of 256x128, with rests in every direction
    c = Case(dtype, 75, 1912, 4360, accumulate=accumulate)
    c.run()
    c.check()


@pytest.mark.parametrize("shape", [(2100, 1604, 1212), (1002, 772, 1020), (645, 1028, 1036), (700, 1036, 4), (1, 4, 5124), (2570, 36, 516)],
                         ids=lambda s: "-".join(map(str, s)))
def test_fp32_tiles(shape):
    # large and small tiles, each with rests in every direction; products with a step or less of depth
    for kw in (dict(), dict(act=B.ACT_GELU, pad=4, accumulate=1), dict(bias=False, dx=False), dict(keep=False, bias=False), dict(dw=False)):
        c = Case(F32, *shape, **kw)
        c.run()
        c.check()


@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("accumulate", [0, 1])
@pytest.mark.parametrize("shape", [(20, 64, 72), (700, 1096, 96), (4100, 64, 1544), (75, 1912, 4360)], ids=lambda s: "-".join(map(str, s)))
def test_one_bias_gradient(dtype, accumulate, shape):
    # either of the two without the other: the same bits as with both, and nothing written for the other
    c = Case(dtype, *shape, accumulate=accumulate)
    c.run()
    want = [t.clone() for t in c.grads]
    for keep in (1, 3):
        for t in c.grads:
            t.fill_(GUARD)
        d = c.desc()
        if keep == 1:
            d.db_out = None
        else:
            d.db_in = None
        B.dapple_gated_ffn_bwd(dtype, d)
        for i, (got, w) in enumerate(zip(c.grads, want)):
            assert torch.equal(got, torch.full_like(w, GUARD) if i == 4 - keep else w), (keep, i)


def test_fp32_only_shapes():
    # multiples of four
    for shape in ((3, 12, 20), (77, 100, 36), (513, 260, 132)):
        for kw in (dict(), dict(pad=4, accumulate=1), dict(keep=False)):
            c = Case(F32, *shape, **kw)
            c.run()
            c.check()


@pytest.mark.parametrize("act", [B.ACT_SILU, B.ACT_GELU])
@pytest.mark.parametrize("dtype", [F32, BF])
def test_large_gates(dtype, act):
    # gates of +-300: the exponentials end at 0 and at infinity
    c = Case(dtype, 40, 64, 64, act)
    c.b_in[:32] = 300.0
    c.b_in[32:64] = -300.0
    c.run()
    assert all(bool(t.isfinite().all()) for t in (c.y, c.h, c.dgu, c.out_dx, *c.grads))
    c.check()


def test_gradient_against_differences():
    # fp32; h^2 of the third derivative's part, and the roundings of a sum of about 100 over h
    c = Case(F32, 6, 16, 12, B.ACT_SILU)
    c.run()
    step, d = 2.0 ** -6, c.desc()

    def f():
        B.dapple_gated_ffn_fwd(F32, d)
        return float((c.y.double() * c.dy.double()).sum())

    for t, grad, at in ((c.x, c.out_dx.clone(), (3, 5)), (c.w_in, c.grads[0].clone(), (7, 3)), (c.w_in, c.grads[0].clone(), (2, 20)),
                        (c.b_in, c.grads[1].clone(), (4,)), (c.w_out, c.grads[2].clone(), (11, 15)), (c.b_out, c.grads[3].clone(), (9,))):
        old, vals = float(t[at]), []
        for sgn in (1, -1):
            t[at] = old + sgn * step
            vals.append(f())
        t[at] = old
        assert abs((vals[0] - vals[1]) / (2 * step) - float(grad[at])) < 30 * step * step + 2.0 ** -24 * 400 / step


@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("accumulate", [0, 1])
def test_same_bits_on_another_stream_and_in_a_graph(dtype, accumulate):
    c = Case(dtype, 200, 128, 264, accumulate=accumulate)
    outs = (c.y, c.h, c.gu, c.dgu, c.out_dx, *c.grads)
    c.run()
    torch.cuda.synchronize()
    want = [t.clone() for t in outs]
    side = torch.cuda.Stream()
    for t in c.grads:
        t.fill_(GUARD)
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        c.run(side.cuda_stream)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(outs, want))
    d = c.desc()

    def run():
        sp = torch.cuda.current_stream().cuda_stream
        B.dapple_gated_ffn_fwd(dtype, d, sp)
        B.dapple_gated_ffn_bwd(dtype, d, sp)

    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    for k in range(3):
        c.x.mul_(-0.75)
        for t in outs:
            t.fill_(GUARD)
        run()
        torch.cuda.synchronize()
        eager = [t.clone() for t in outs]
        for t in outs:
            t.fill_(GUARD)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, eager)), k


@pytest.mark.parametrize("shape", [(16, 64, 4096), (16, 64, 4104), (9, 128, 9000), (32, 72, 8192), (32, 72, 8200), (1, 72, 8200), (20, 4096, 72),
                                   (20, 4104, 72), (16, 4096, 64), (16, 4104, 64)], ids=lambda s: "-".join(map(str, s)))
def test_few_rows_of_many_columns(shape):
    # on either side of the columns from which on few rows are the tiles' again, each product
    for kw in (dict(), dict(act=B.ACT_GELU, pad=8, accumulate=1)):
        c = Case(BF, *shape, **kw)
        c.run()
        c.check()


@pytest.mark.parametrize("shape,kw", [
    ((4090, 36, 1020), dict(act=B.ACT_GELU)),                      # gate and value
    ((4090, 2044, 36), dict(pad=4)),                               # the output product
    ((4090, 36, 2044), dict(bias=False, accumulate=1)),            # dh with the gate's gradient
    ((2040, 2044, 2044), dict()), ((2040, 2044, 2044), dict(accumulate=1, act=B.ACT_GELU)),      # the last gradients, dx with them
    ((100, 2044, 2804), dict(dx=False)), ((100, 2044, 2804), dict(dx=False, bias=False, accumulate=1)),
    ((4090, 36, 1020), dict(keep=False, bias=False))], ids=str)
def test_fp32_wide_tiles(shape, kw):
    # two 128-wide tiles for each unit, with rests in every direction
    c = Case(F32, *shape, **kw)
    c.run()
    c.check()
