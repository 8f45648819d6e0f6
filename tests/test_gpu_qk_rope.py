"""Head norms with the rotation by position, forward and backward, and the table of angles, against float64.

Tolerances.  A sum over a head of up to 256 columns is a chain of at most 32 additions per lane and a tree of six: rstd is
off by at most (38 / 2 + 3) 2^-24 with its own rounding and the division, a column by less than 2^-19 of the two columns its
pair is made of; dx by 2^-19 of its two terms, the mean of which is a sum of the same kind.  bf16 results have half a step,
2^-8, of themselves on top.  dgamma: chains of at most 512 additions at these sizes, 2^-15 of the sum of the terms' sizes."""
import math

import numpy as np
import pytest
import torch

from paper_2007_01045_amd import binding as B

pytestmark = pytest.mark.gpu
TD = {B.DTYPE_F32: torch.float32, B.DTYPE_BF16: torch.bfloat16}
DTYPES = [B.DTYPE_F32, B.DTYPE_BF16]
GUARD = 7.0


def turn(n, c, s, rot, inter):
    """n [..., d] with its first `rot` columns turned; the sizes of the pairs' columns beside it."""
    y, size = n.clone(), n.abs()
    if rot:
        i = torch.arange(rot // 2, device=n.device)
        a, b = (2 * i, 2 * i + 1) if inter else (i, i + rot // 2)
        y[..., a] = n[..., a] * c - n[..., b] * s
        y[..., b] = n[..., a] * s + n[..., b] * c
        size[..., a] = size[..., b] = n[..., a].abs() + n[..., b].abs()
    return y, size


def normal(seed, *shape, scale=1.0, mean=0.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(*shape, generator=g, device="cuda") * scale + mean


class Case:
    """One projection [rows, ld] whose first columns (after `lead`) are the query heads, key heads behind them."""

    def __init__(self, dtype, rows, A, Ak, d, rot, inter, norm=True, lead=0, tail=0, positions=True, seq=0, seed=1):
        self.__dict__.update(locals())
        self.td, self.ld, self.n = TD[dtype], lead + (A + Ak) * d + tail, (A + Ak) * d
        self.x, self.dy = (normal(seed + i, rows, self.ld).to(self.td) for i in (0, 1))
        self.gam = [normal(seed + 2 + i, d, scale=0.3, mean=1.0).to(self.td) for i in (0, 1)]
        self.max_pos = 5000
        self.table = torch.empty(self.max_pos, max(rot // 2, 1), 2, device="cuda")
        if rot:
            B.dapple_rope_table(self.table.data_ptr(), self.max_pos, rot)
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.pos = torch.randint(0, self.max_pos, (rows,), generator=g, device="cuda", dtype=torch.int32) if positions else None
        self.y, self.dx = (torch.full((rows, self.ld), GUARD, device="cuda").to(self.td) for _ in range(2))
        self.dg = [torch.full((d,), 3.0, device="cuda") for _ in range(2)]

    def desc(self, y=None, dx=None, accumulate=0):
        es, ld, k = self.x.element_size(), self.ld, self.A * self.d * self.x.element_size()
        at = lambda t: t.data_ptr() + self.lead * es  # noqa: E731
        y, dx = at(self.y if y is None else y), at(self.dx if dx is None else dx)
        d = B.qk_rope_desc(q=at(self.x), k=at(self.x) + k, yq=y, yk=y + k, dyq=at(self.dy), dyk=at(self.dy) + k, dq=dx, dk=dx + k,
                           table=self.table.data_ptr() if self.rot else None,
                           positions=self.pos.data_ptr() if self.pos is not None else None, rows=self.rows, A=self.A, Ak=self.Ak, d=self.d,
                           rot=self.rot, interleaved=int(self.inter), seq=self.seq, max_pos=self.max_pos, accumulate=accumulate,
                           ldq=ld, ldk=ld, ldyq=ld, ldyk=ld, lddyq=ld, lddyk=ld, lddq=ld, lddk=ld, eps=1e-6)
        if self.norm:
            d.gamma_q, d.gamma_k = (t.data_ptr() for t in self.gam)
            d.dgamma_q, d.dgamma_k = (t.data_ptr() for t in self.dg)
            self.ws = torch.full((B.dapple_qk_rope_workspace(self.dtype, d),), 0xff, dtype=torch.uint8, device="cuda")
            d.workspace = self.ws.data_ptr()
        return d

    def heads(self, t):
        return t[:, self.lead:self.lead + self.n].double().view(self.rows, self.A + self.Ak, self.d)

    def want(self):
        """y, dx, dgamma and what their errors may be."""
        row = torch.arange(self.rows, device="cuda")
        pos = self.pos.long() if self.pos is not None else (row % self.seq if self.seq else row)
        cs = self.table[pos].double()
        c, s = (cs[:, None, :, i] if self.rot else None for i in (0, 1))
        x, dy = self.heads(self.x), self.heads(self.dy)
        gam = torch.cat([self.gam[0].double().expand(self.A, self.d), self.gam[1].double().expand(self.Ak, self.d)])
        half = 2.0 ** -8 if self.dtype == B.DTYPE_BF16 else 0.0
        e = 2.0 ** -19
        if not self.norm:
            y, size = turn(x, c, s, self.rot, self.inter)
            dx, dsize = turn(dy, c, -s, self.rot, self.inter)
            return (y, e * size + half * y.abs()), (dx, e * dsize + half * dx.abs()), None
        rstd = 1 / torch.sqrt(x.square().mean(-1, keepdim=True) + 1e-6)
        xh = x * rstd
        y, size = turn(xh * gam, c, s, self.rot, self.inter)
        dn, dsize = turn(dy, c, -s if self.rot else None, self.rot, self.inter)
        t = dn * gam
        dx = rstd * (t - xh * (t * xh).mean(-1, keepdim=True))
        tol = rstd * e * (dsize * gam.abs() + xh.abs() * (dsize * gam.abs() * xh.abs()).mean(-1, keepdim=True)) + half * dx.abs()
        terms = dn * xh
        dg = [terms[:, :self.A].sum((0, 1)), terms[:, self.A:].sum((0, 1))]
        big = (dsize * xh.abs())
        dgt = [2.0 ** -15 * big[:, :self.A].sum((0, 1)), 2.0 ** -15 * big[:, self.A:].sum((0, 1))]
        return (y, e * size + half * y.abs()), (dx, tol), list(zip(dg, dgt))

    def check(self, got, pair):
        want, tol = pair
        off = (self.heads(got) - want).abs()
        assert bool((off <= tol).all()), float((off / tol.clamp_min(1e-300)).max())
        outside = torch.ones(self.ld, dtype=torch.bool, device="cuda")
        outside[self.lead:self.lead + self.n] = False
        assert bool((got[:, outside] == GUARD).all()), "a column between the rows was written"


SHAPES = [  # rows, A, Ak, d, rot, interleaved, lead, tail
    (1, 1, 1, 64, 64, False, 0, 0), (1, 16, 4, 128, 128, False, 0, 0), (5, 3, 1, 64, 64, True, 0, 0), (77, 12, 4, 128, 64, False, 8, 16),
    (130, 7, 0, 64, 32, True, 0, 8), (300, 4, 2, 80, 80, False, 0, 0), (33, 5, 5, 80, 20, False, 0, 0), (33, 5, 5, 80, 20, True, 0, 0),
    (64, 2, 2, 256, 256, False, 0, 0), (64, 2, 2, 256, 96, True, 0, 0), (19, 3, 2, 36, 18, False, 0, 0), (19, 3, 2, 36, 18, True, 0, 2),
    (40, 2, 1, 255, 254, False, 1, 0), (21, 2, 3, 7, 6, False, 1, 3), (9, 4, 4, 64, 0, False, 0, 0), (4500, 2, 1, 32, 32, False, 0, 0),
    (50, 3, 1, 104, 64, False, 0, 0), (50, 3, 1, 96, 2, True, 4, 4), (11, 1, 1, 2, 2, True, 0, 0), (70, 40, 1, 64, 64, False, 0, 0)]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("norm", [True, False])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "-".join(str(int(v)) for v in s))
def test_forward_and_backward(dtype, norm, shape):
    rows, A, Ak, d, rot, inter, lead, tail = shape
    if not norm and not rot:
        pytest.skip("neither a norm nor a rotation: refused")
    c = Case(dtype, rows, A, Ak, d, rot, inter, norm, lead, tail, positions=rows % 2 == 1, seq=0 if rows < 100 else 97)
    desc = c.desc()
    B.dapple_qk_rope_fwd(dtype, desc)
    B.dapple_qk_rope_bwd(dtype, desc)
    y, dx, dg = c.want()
    c.check(c.y, y)
    c.check(c.dx, dx)
    if norm:
        for got, (want, tol), heads in zip(c.dg, dg, (A, Ak)):
            if heads:
                assert bool(((got.double() - want).abs() <= tol).all())
        first = [t.clone() for t in c.dg]
        desc = c.desc(accumulate=1)     # added to what is there
        B.dapple_qk_rope_bwd(dtype, desc)
        for got, one, heads in zip(c.dg, first, (A, Ak)):
            if heads:
                assert torch.equal(got, one + one)


@pytest.mark.parametrize("dtype", DTYPES)
def test_in_place(dtype):
    c = Case(dtype, 50, 4, 2, 64, 32, False, lead=8)
    desc = c.desc()
    B.dapple_qk_rope_fwd(dtype, desc)
    B.dapple_qk_rope_bwd(dtype, desc)
    y, dx = c.y.clone(), c.dx.clone()
    B.dapple_qk_rope_bwd(dtype, c.desc(dx=c.dy))
    assert torch.equal(c.heads(c.dy), c.heads(dx))
    B.dapple_qk_rope_fwd(dtype, c.desc(y=c.x))
    assert torch.equal(c.heads(c.x), c.heads(y))


def test_gradient_against_differences():
    # d(sum y dy) / dx by central differences of the kernel's own forward, fp32: the difference quotient's error is the third
    # derivative's part, h^2, and two roundings of a sum of about 20, 2^-24 20 / h
    c = Case(B.DTYPE_F32, 3, 1, 1, 16, 8, True)
    desc = c.desc()
    B.dapple_qk_rope_bwd(B.DTYPE_F32, desc)
    dx, x0, h = c.dx.clone(), c.x.clone(), 2.0 ** -6

    def f():
        B.dapple_qk_rope_fwd(B.DTYPE_F32, desc)
        return float((c.heads(c.y) * c.heads(c.dy)).sum())

    for r, col in ((0, 0), (0, 9), (1, 17), (2, 31), (2, 3)):
        vals = []
        for sgn in (1, -1):
            c.x.copy_(x0)
            c.x[r, col] += sgn * h
            vals.append(f())
        c.x.copy_(x0)
        assert abs((vals[0] - vals[1]) / (2 * h) - float(dx[r, col])) < 10 * h * h + 2.0 ** -24 * 100 / h


@pytest.mark.parametrize("dtype", DTYPES)
def test_what_is_not_finite_stays_where_it_is(dtype):
    for inter in (False, True):
        c = Case(dtype, 8, 2, 1, 64, 32, inter, norm=False)
        c.x[3, 40] = math.inf                     # a column that does not turn, of head 0
        c.x[4, 64 + 33] = math.nan
        c.pos[5], c.pos[6] = -1, c.max_pos        # positions that the table does not have
        B.dapple_qk_rope_fwd(dtype, c.desc())
        bad = ~torch.isfinite(c.heads(c.y))
        where = torch.zeros_like(bad)
        where[3, 0, 40] = where[4, 1, 33] = True
        where[5:7, :, :32] = True
        assert torch.equal(bad, where)


def test_offsets_beyond_32_bits():
    # the last row begins past 2^31 elements (4.8 GB of bf16)
    rows, ld, d = 40000, 60000, 64
    x = torch.empty(rows, ld, dtype=torch.bfloat16, device="cuda")
    x[-3:] = normal(4, 3, ld).bfloat16()
    table = torch.empty(rows, d // 2, 2, device="cuda")
    B.dapple_rope_table(table.data_ptr(), rows, d)
    y = torch.empty(rows, d, dtype=torch.bfloat16, device="cuda")
    q = x.data_ptr() + (ld - d) * 2
    x[:, ld - d:] = x[-1, ld - d:]
    desc = B.qk_rope_desc(q=q, yq=y.data_ptr(), table=table.data_ptr(), rows=rows, A=1, d=d, rot=d, max_pos=rows, ldq=ld)
    B.dapple_qk_rope_fwd(B.DTYPE_BF16, desc)
    cs = table.double()
    want, size = turn(x[-1, ld - d:].double().expand(rows, d), cs[..., 0], cs[..., 1], d, False)
    assert bool(((y.double() - want).abs() <= 2.0 ** -19 * size + 2.0 ** -8 * want.abs()).all())


def test_replayed_graph():
    c = Case(B.DTYPE_BF16, 333, 4, 2, 64, 64, False)
    desc = c.desc()

    def run():
        sp = torch.cuda.current_stream().cuda_stream
        B.dapple_qk_rope_fwd(B.DTYPE_BF16, desc, sp)
        B.dapple_qk_rope_bwd(B.DTYPE_BF16, desc, sp)

    run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    for k in range(3):
        c.x.mul_(-0.5), c.dy.add_(0.25)
        run()
        torch.cuda.synchronize()
        eager = [t.clone() for t in (c.y, c.dx, *c.dg)]
        for t in (c.y, c.dx, *c.dg):
            t.fill_(GUARD)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a[:, :c.n] if a.dim() > 1 else a, b[:, :c.n] if b.dim() > 1 else b) for a, b in zip(eager, (c.y, c.dx, *c.dg))), k


@pytest.mark.parametrize("rot,base,factor,original,magnitude", [
    (64, 10000.0, 1.0, 0, 1.0), (2, 10000.0, 1.0, 0, 1.0), (256, 500000.0, 1.0, 0, 1.0), (64, 10000.0, 8.0, 0, 1.0),
    (128, 10000.0, 4.0, 2048, 1.1386), (96, 1e6, 0.5, 512, 0.5)])
def test_table(rot, base, factor, original, magnitude):
    # each entry is a float64 value rounded once: half a step of the entry, and 2^-30 where it is near zero (the device's and
    # the host's angles of 3e5 radians agree to 1e-10)
    n = 300000 if rot <= 64 else 5000
    t = torch.full((n, rot // 2, 2), math.nan, device="cuda")
    B.dapple_rope_table(t.data_ptr(), n, rot, base, factor, original, 1.0, 32.0, magnitude)
    i = np.arange(rot // 2)
    w = base ** (-2.0 * i / rot)
    g = np.clip((original * w / (2 * np.pi) - 1.0) / 31.0, 0.0, 1.0) if original else np.zeros(rot // 2)
    angle = np.arange(n)[:, None] * (w * (g + (1 - g) / factor))
    got = t.cpu().numpy().astype(np.float64)
    for k, f in ((0, np.cos), (1, np.sin)):
        want = magnitude * f(angle)
        assert (np.abs(got[..., k] - want) <= 2.0 ** -24 * np.abs(want) * 1.01 + 2.0 ** -30).all()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("shape", [(5, 12, 4, 64, 64, False), (4200, 3, 1, 64, 32, True), (7, 5, 3, 7, 6, False), (6, 9, 0, 96, 0, False)],
                         ids=lambda s: "-".join(str(int(v)) for v in s))
def test_without_eps(dtype, shape):
    # heads that do not fill a wave's passes, whose absent ones must not reach dgamma; no head is zero
    rows, A, Ak, d, rot, inter = shape
    c = Case(dtype, rows, A, Ak, d, rot, inter)
    for accumulate in (0, 1):
        for t in c.dg:
            t.fill_(3.0)
        desc = c.desc(accumulate=accumulate)
        desc.eps = 0.0
        B.dapple_qk_rope_fwd(dtype, desc)
        B.dapple_qk_rope_bwd(dtype, desc)
        x, dy = c.heads(c.x), c.heads(c.dy)
        cs = c.table[c.pos.long()].double()
        cos, sin = (cs[:, None, :, i] if rot else None for i in (0, 1))
        gam = torch.cat([c.gam[0].double().expand(A, d), c.gam[1].double().expand(Ak, d)])
        rstd = 1 / torch.sqrt(x.square().mean(-1, keepdim=True))
        xh, half, e = x * rstd, 2.0 ** -8 if dtype == B.DTYPE_BF16 else 0.0, 2.0 ** -19      # (as in want())
        y, size = turn(xh * gam, cos, sin, rot, inter)
        dn, dsize = turn(dy, cos, -sin if rot else None, rot, inter)
        t = dn * gam
        dx = rstd * (t - xh * (t * xh).mean(-1, keepdim=True))
        c.check(c.y, (y, e * size + half * y.abs()))
        c.check(c.dx, (dx, rstd * e * (dsize * gam.abs() + xh.abs() * (dsize * gam.abs() * xh.abs()).mean(-1, keepdim=True)) + half * dx.abs()))
        for got, at, heads in zip(c.dg, (slice(0, A), slice(A, A + Ak)), (A, Ak)):
            if heads:
                start = 3.0 * accumulate
                want, tol = start + (dn * xh)[:, at].sum((0, 1)), 2.0 ** -15 * (start + (dsize * xh.abs())[:, at].sum((0, 1)))
                assert bool(((got.double() - want).abs() <= tol).all()), (accumulate, at)
