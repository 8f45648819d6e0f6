"""Dropout, residual sum and norm, forward and backward, against float64 on the same inputs and the mask of tests/dropout_util.py.

Tolerances.  r: half a step of the type that an output is rounded to (bf16 2^-8, fp32 2^-24).  z: before its last addition x + bias,
1 / (1 - p) and their product are rounded to fp32, each by 2^-24 at most, so m |x + bias| is off by 3 * 2^-24 and 2^-22 bounds that; the addition's
own rounding (before one to bf16) is below 2^-23 of what it adds.  The norm is checked from the z that was stored: a mean of H values is off by the depth of its sum (at most 4 * 8 in a lane, 6 + 8
across) times 2^-24 of mean |z|, below 2^-18 mean |z|, and h by that times rstd and by 2^-18 of itself for rstd: e (1 + |h|) with
e = 2^-18 (1 + rstd mean |z|).  A gradient is a sum of three such terms.  Sums over rows are at most 200 deep here: 2^-16 of their terms' sizes."""
import math

import numpy as np
import pytest
import torch

from paper_2007_01045_amd import binding as B
from tests.dropout_util import keep_mask

pytestmark = pytest.mark.gpu
F, H16 = B.DTYPE_F32, B.DTYPE_BF16
TD = {F: torch.float32, H16: torch.bfloat16}
R = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}
LAYER, RMS, NONE = B.NORM_LAYER, B.NORM_RMS, B.NORM_NONE
GUARD, EPS = 7.0, 1e-5


class Case:
    """Tensors with `pad` columns behind every row; pad odd: rows begin anywhere."""

    def __init__(self, dtype, rows, H, norm=LAYER, p=0.1, stream32=False, bias=True, residual=True, gamma=True, beta=True, carry=True, pad=0,
                 accumulate=0, site=5, seed=1, mean=0.5, skip=0):
        self.__dict__.update(locals())
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.td, self.zt = TD[dtype], torch.float32 if stream32 else TD[dtype]
        ld = H + pad

        def buf(t, fill=None):      # `skip` elements in front: an odd address
            x = torch.full((rows * ld + skip,), GUARD, device="cuda").to(t)
            v = x[skip:].view(rows, ld)
            if fill is not None:
                v[:, :H] = fill.to(t)
            return v

        rn = lambda sc, m=0.0: torch.randn(rows, H, generator=g, device="cuda") * sc + m  # noqa: E731
        vec = lambda sc, m=0.0: (torch.randn(H, generator=g, device="cuda") * sc + m).to(self.td)  # noqa: E731
        self.x, self.res = buf(self.td, rn(1)), buf(self.zt, rn(2, mean)) if residual else None
        self.b = vec(0.5) if bias else None
        self.ga = vec(0.2, 1) if gamma and norm != NONE else None
        self.be = vec(0.3) if beta and norm == LAYER else None
        self.dy, self.dz = buf(self.td, rn(1)), buf(self.zt, rn(1)) if carry or norm == NONE else None
        self.rng = torch.randint(-(1 << 62), 1 << 62, (2,), generator=g, device="cuda")
        self.z, self.y, self.stats = buf(self.zt), buf(self.td), torch.full((rows, 2), GUARD, device="cuda")
        self.dx, self.dr = buf(self.td), buf(self.zt)
        self.sums = [torch.full((H,), 3.0, device="cuda") for _ in range(3)]      # dbias, dgamma, dbeta
        self.want_sums = [True, norm != NONE, norm == LAYER]

    def desc(self, **kw):
        q = lambda t: None if t is None else t.data_ptr()  # noqa: E731
        ld = self.H + self.pad
        d = B.dropout_norm_desc(x=q(self.x), bias=q(self.b), residual=q(self.res), gamma=q(self.ga), beta=q(self.be), rng=q(self.rng), z=q(self.z),
                                y=q(self.y), stats=q(self.stats), dy=q(self.dy), dz=q(self.dz), dx=q(self.dx), dresidual=q(self.dr),
                                rows=self.rows, H=self.H, norm=self.norm, stream32=int(self.stream32), accumulate=self.accumulate, site=self.site,
                                ldx=ld, ldr=ld, ldz=ld, ldy=ld, lddy=ld, lddz=ld, lddx=ld, lddr=ld, p=self.p, eps=EPS)
        for name, t, on in zip(("dbias", "dgamma", "dbeta"), self.sums, self.want_sums):
            setattr(d, name, q(t) if on else None)
        self.ws = torch.full((B.dapple_dropout_norm_workspace(self.dtype, d),), 0xff, dtype=torch.uint8, device="cuda")
        d.workspace = q(self.ws)
        for k, v in kw.items():
            setattr(d, k, v)
        return d

    def run(self, stream=None, **kw):
        d = self.desc(**kw)
        B.dapple_dropout_norm_fwd(self.dtype, d, stream)
        B.dapple_dropout_norm_bwd(self.dtype, d, stream)

    def mask(self):
        seed, step = (int(v) & (2 ** 64 - 1) for v in self.rng.tolist())
        level = round(65536 * float(np.float32(self.p)))
        if level == 0:
            return torch.ones(self.rows, self.H, dtype=torch.float64, device="cuda")
        keep = torch.from_numpy(keep_mask(seed, step, self.site, self.rows, self.H, self.p)).cuda()
        return keep.double() * (65536 / (65536 - level) if level < 65536 else 0.0)

    def check(self):
        H, n = self.H, lambda t: 0.0 if t is None else t.double()
        rd, rz = R[self.td], R[self.zt]
        for t in [self.z, self.y, self.dx, self.dr]:
            assert bool((t[:, H:] == GUARD).all()), "a column between the rows was written"
        m = self.mask()
        x = n(self.x[:, :H]) + n(self.b)
        res = n(self.res[:, :H]) if self.res is not None else 0.0
        z = m * x + res
        self.close("z", self.z, z, 2.0 ** -22 * m * x.abs() + 2.0 ** -23 * abs(res), rz)
        z = self.z[:, :H].double()
        g = n(self.dz[:, :H]) if self.dz is not None else torch.zeros_like(z)
        tol = 2.0 ** -23 * g.abs()
        old = 3.0 if self.accumulate else 0.0
        if self.norm != NONE:
            mean = z.mean(-1, keepdim=True) if self.norm == LAYER else 0.0
            rstd = ((z - mean).square().mean(-1, keepdim=True) + EPS).rsqrt()
            h = (z - mean) * rstd
            e = 2.0 ** -18 * (1 + rstd * z.abs().mean(-1, keepdim=True))
            ga = n(self.ga) if self.ga is not None else torch.ones(H, dtype=torch.float64, device="cuda")
            y = h * ga + n(self.be)
            self.close("y", self.y, y, e * (1 + h.abs()) * ga.abs() + 2.0 ** -22 * y.abs() + 2.0 ** -22 * abs(n(self.be)), rd)
            st = self.stats.double()
            assert bool(((st[:, 1:] - rstd).abs() <= e * rstd).all())
            assert bool(((st[:, :1] - mean).abs() * rstd <= e).all())
            dy = n(self.dy[:, :H])
            t = dy * ga
            d = t - h * (t * h).mean(-1, keepdim=True) - (t.mean(-1, keepdim=True) if self.norm == LAYER else 0.0)
            g = g + rstd * d
            ta = t.abs()
            tol = tol + rstd * e * (ta + ta.mean(-1, keepdim=True) + 3 * (1 + h.abs()) * (ta * (1 + h.abs())).mean(-1, keepdim=True))
            if self.norm == LAYER:
                self.total("dbeta", 2, dy.sum(0) + old, 2.0 ** -16 * dy.abs().sum(0))
            self.total("dgamma", 1, (dy * h).sum(0) + old, ((2.0 ** -16 + e) * dy.abs() * (1 + h.abs())).sum(0))
        self.close("dresidual", self.dr, g, tol, rz)
        self.close("dx", self.dx, m * g, m * (tol + 2.0 ** -23 * g.abs()), rd)
        self.total("dbias", 0, (m * g).sum(0) + old, (m * (tol + 2.0 ** -16 * g.abs())).sum(0))

    def close(self, what, got, want, tol, r):
        got = got[:, :self.H].double()
        off = (got - want).abs() - (tol + r * (want.abs() + tol) + 1e-30)
        assert float(off.max()) <= 0, (what, float(off.max()), int(off.argmax()))

    def total(self, what, i, want, tol):
        off = (self.sums[i].double() - want).abs() - (tol + 2.0 ** -22 * (1 + want.abs()))
        assert float(off.max()) <= 0, (what, float(off.max()), int(off.argmax()))


CASES = [  # dtype, rows, H, norm, p, stream32
    (H16, 1, 1, LAYER, 0.1, False), (H16, 1, 8, RMS, 0.5, False), (H16, 3, 7, LAYER, 0.1, True), (H16, 5, 64, NONE, 0.3, False), (H16, 16, 512, LAYER, 0.1, False),
    (H16, 33, 513, RMS, 0.1, True), (H16, 70, 1024, LAYER, 0.1, True), (H16, 67, 1001, LAYER, 0.25, False), (H16, 9, 1025, LAYER, 0.1, False),
    (H16, 40, 2048, RMS, 0.0, False), (H16, 17, 2055, LAYER, 0.1, True), (H16, 21, 4096, RMS, 0.1, False), (H16, 6, 4097, LAYER, 0.1, False),
    (H16, 5, 8192, LAYER, 0.1, True), (H16, 3, 8200, RMS, 0.1, False), (H16, 4, 16384, LAYER, 0.1, False), (H16, 3, 16383, LAYER, 0.9, True), (H16, 3, 700, NONE, 0.0, True),
    (H16, 2500, 24, LAYER, 0.1, False), (H16, 9000, 40, RMS, 0.1, False), (H16, 3001, 1100, LAYER, 0.1, False), (H16, 12, 256, LAYER, 1.0, False),
    (F, 1, 1, LAYER, 0.1, False), (F, 2, 3, RMS, 0.5, False), (F, 19, 250, LAYER, 0.1, False), (F, 30, 1024, LAYER, 0.1, True), (F, 31, 1001, RMS, 0.2, False),
    (F, 11, 2047, LAYER, 0.1, False), (F, 9, 4096, NONE, 0.1, False), (F, 5, 8191, LAYER, 0.1, False), (F, 3, 16384, LAYER, 0.1, False), (F, 1200, 520, LAYER, 0.1, False),
    (H16, 600, 8200, LAYER, 0.1, True), (H16, 520, 16384, LAYER, 0.1, False), (F, 530, 12288, LAYER, 0.1, False), (F, 520, 8208, RMS, 0.1, False),
]
ids = lambda c: "-".join(str(v) for v in c)  # noqa: E731


@pytest.mark.parametrize("case", CASES, ids=ids)
@pytest.mark.parametrize("pad", [0, 3])
def test_forward_and_backward(case, pad):
    c = Case(*case, pad=pad, skip=pad // 3)
    c.run()
    c.check()


@pytest.mark.parametrize("dtype", [F, H16])
@pytest.mark.parametrize("off", ["bias", "residual", "gamma", "beta", "carry"])
def test_without_one_of_the_inputs(dtype, off):
    for norm in (LAYER, RMS, NONE):
        c = Case(dtype, 50, 300, norm, **{off: False})
        c.run()
        c.check()


@pytest.mark.parametrize("dtype", [F, H16])
def test_outputs_not_wanted_and_sums_added(dtype):
    c = Case(dtype, 60, 700, accumulate=1)
    c.run()
    c.check()
    want = [t.clone() for t in (c.y, c.dx, c.dr, *c.sums)]
    for t in c.sums:
        t.fill_(3)
    c.dr.fill_(GUARD)
    B.dapple_dropout_norm_bwd(dtype, c.desc(dx=None, dresidual=None))
    assert all(torch.equal(a, b) for a, b in zip(c.sums, want[3:])) and bool((c.dr == GUARD).all())
    c.z.fill_(GUARD)
    c.stats.fill_(GUARD)
    c.y.fill_(0)
    B.dapple_dropout_norm_fwd(dtype, c.desc(z=None, stats=None))
    assert torch.equal(c.y, want[0]) and bool((c.z == GUARD).all()) and bool((c.stats == GUARD).all())
    c = Case(dtype, 60, 700)
    c.run()
    want = [t.clone() for t in (c.dx, c.dr)]
    c.dx.fill_(0)
    B.dapple_dropout_norm_bwd(dtype, c.desc(dbias=None, dgamma=None, dbeta=None, workspace=None))
    assert torch.equal(c.dx, want[0]) and torch.equal(c.dr, want[1])


@pytest.mark.parametrize("dtype", [F, H16])
def test_in_place(dtype):
    a, b = Case(dtype, 77, 1000), Case(dtype, 77, 1000)
    a.run()
    q = lambda t: t.data_ptr()  # noqa: E731
    d = b.desc(z=q(b.res), y=q(b.x), dresidual=q(b.dz), dx=q(b.dy))
    B.dapple_dropout_norm_fwd(dtype, d)
    B.dapple_dropout_norm_bwd(dtype, d)
    for got, want in ((b.res, a.z), (b.x, a.y), (b.dz, a.dr), (b.dy, a.dx)):
        assert torch.equal(got, want)
    assert all(torch.equal(x, y) for x, y in zip(a.sums, b.sums))


def test_masks_of_steps_sites_and_seeds_differ():
    c = Case(F, 64, 1000, NONE, 0.5, residual=False, bias=False)
    c.x.fill_(1.0)
    masks = []
    for seed, step, site in ((1, 2, 3), (2, 2, 3), (1, 3, 3), (1, 2, 4), (1 + (1 << 32), 2, 3), (1, 2 + (1 << 32), 3)):
        c.rng.copy_(torch.tensor([seed, step]))
        B.dapple_dropout_norm_fwd(F, c.desc(site=site))
        masks.append(c.z.clone())
        assert bool(((c.z == 0) | (c.z == 2)).all())
        assert abs(float(c.z.mean()) - 1) < 6 / math.sqrt(64000)      # six standard deviations
    for i in range(len(masks)):
        for j in range(i):
            assert abs(float((masks[i] == masks[j]).double().mean()) - 0.5) < 3 / math.sqrt(64000)      # likewise


def test_infinite_and_nan_elements_that_are_dropped():
    c = Case(F, 40, 500, NONE, 0.5)
    drop = c.mask() == 0
    c.x[drop] = math.nan
    c.x[:, :10][drop[:, :10]] = math.inf
    c.run()
    assert bool(c.z.isfinite().all()) and torch.equal(c.z[drop], c.res[drop])


def test_gradient_against_differences():
    # fp32; the quotient's error: h^2 of the third derivative's part, and the roundings of a sum of about 200 terms over h
    c = Case(F, 6, 37, LAYER, 0.3)
    c.run()
    sums = [t.clone() for t in c.sums]
    h = 2.0 ** -6

    def f():
        B.dapple_dropout_norm_fwd(F, c.desc())
        return float((c.y.double() * c.dy.double()).sum() + (c.z.double() * c.dz.double()).sum())

    for t, grad, at in ((c.x, c.dx, [(0, 3), (5, 36), (2, 0)]), (c.res, c.dr, [(1, 7), (4, 20)]), (c.b, sums[0], [5, 30]), (c.ga, sums[1], [0, 36]), (c.be, sums[2], [8])):
        for i in at:
            old, vals = t[i].clone(), []
            for sgn in (1, -1):
                t[i] = old + sgn * h
                vals.append(f())
            t[i] = old
            assert abs((vals[0] - vals[1]) / (2 * h) - float(grad[i])) < 40 * h * h + 2.0 ** -24 * 800 / h, (i,)


@pytest.mark.parametrize("dtype", [F, H16])
def test_same_bits_on_another_stream_and_in_a_graph(dtype):
    c = Case(dtype, 300, 1000)
    outs = (c.z, c.y, c.stats, c.dx, c.dr, *c.sums)
    c.run()
    torch.cuda.synchronize()
    want = [t.clone() for t in outs]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        c.run(side.cuda_stream)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(outs, want))
    d = c.desc()
    held = c.ws      # the graph's own: an eager run brings another
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        sp = torch.cuda.current_stream().cuda_stream
        B.dapple_dropout_norm_fwd(dtype, d, sp)
        B.dapple_dropout_norm_bwd(dtype, d, sp)
    last = None
    for k in range(3):      # another step: another mask
        c.rng[1] += 1
        c.run()
        torch.cuda.synchronize()
        eager = [x.clone() for x in outs]
        assert last is None or not torch.equal(last, eager[0])
        last = eager[0]
        for x in outs:
            x.fill_(GUARD)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, eager)), k
    del held


def test_offsets_beyond_32_bits():
    rows, H, ld = 500, 72, 9_000_001      # the last rows lie past 2^32 elements (9 GB); an odd stride
    x = torch.empty(rows * ld, dtype=torch.bfloat16, device="cuda").view(rows, ld)
    small = Case(H16, rows, H)
    x[:, :H] = small.x
    small.run()
    want = [t.clone() for t in (small.z, small.y, small.dx)]
    d = small.desc(x=x.data_ptr(), ldx=ld, z=x.data_ptr() + 2 * 128, ldz=ld, y=x.data_ptr() + 2 * 256, ldy=ld, dx=x.data_ptr() + 2 * 512, lddx=ld)
    B.dapple_dropout_norm_fwd(H16, d)
    B.dapple_dropout_norm_bwd(H16, d)
    for at, w in zip((128, 256, 512), want):
        assert torch.equal(x[:, at:at + H], w)
