"""Rows of a table and the table's gradient, against float64 on the same inputs.

Tolerances: a row of y is one product, rounded once: the same bits as torch's.  A sum of n rows is off by at most n * 2^-24 of its terms'
sizes (its depth is less), by 2^-23 for the scale and the sum before it, and half a step of the type it is rounded to."""
import pytest
import torch

from paper_2007_01045_amd import binding as B

pytestmark = pytest.mark.gpu
F, H16 = B.DTYPE_F32, B.DTYPE_BF16
TD = {F: torch.float32, H16: torch.bfloat16}
GUARD = 7.0


class Case:
    def __init__(self, dtype, rows, V, H, scale=0.75, kind="some", pad=0, skip=0, accumulate=0, seed=1):
        self.__dict__.update(locals())
        g = torch.Generator(device="cuda").manual_seed(seed)
        td = TD[dtype]
        ld = H + pad

        def buf(n, t, fill=True):
            x = torch.full((n * ld + skip,), GUARD, device="cuda").to(t)[skip:].view(n, ld)
            if fill:
                x[:, :H] = torch.randn(n, H, generator=g, device="cuda").to(t)
            return x

        self.table, self.dy, self.y = buf(V, td), buf(rows, td), buf(rows, td, False)
        self.dtable = buf(V, torch.float32 if accumulate else td, bool(accumulate))
        u = torch.rand(rows, generator=g, device="cuda", dtype=torch.float64)
        self.ids = {"some": lambda: ((V + 1.0) ** u).floor().long() - 1, "uniform": lambda: (u * V).long(), "same": lambda: torch.full_like(u, V - 1).long(),
                    "none": lambda: torch.where(u < 0.5, -1, V), "pads": lambda: torch.where(u < 0.6, (V * u / 0.6).long(), torch.where(u < 0.8, -7, 2 ** 31 - 1)),
                    "rising": lambda: torch.arange(rows, device="cuda") * V // rows, "falling": lambda: V - 1 - torch.arange(rows, device="cuda") * V // rows}[kind]()
        self.ids = self.ids.clamp(-7 if kind in ("pads", "none") else 0, 2 ** 31 - 1 if kind in ("pads", "none") else V - 1).int()

    def desc(self):
        q, ld = (lambda t: t.data_ptr()), self.H + self.pad
        d = B.embedding_desc(table=q(self.table), ids=q(self.ids), y=q(self.y), dy=q(self.dy), dtable=q(self.dtable), rows=self.rows, V=self.V, H=self.H,
                             accumulate=self.accumulate, ldt=ld, ldy=ld, lddy=ld, lddt=ld, scale=self.scale)
        self.ws = torch.full((B.dapple_embedding_workspace(self.dtype, d),), 0xff, dtype=torch.uint8, device="cuda")
        d.workspace = q(self.ws)
        return d

    def run(self, stream=None):
        d = self.desc()
        B.dapple_embedding_fwd(self.dtype, d, stream)
        B.dapple_embedding_bwd(self.dtype, d, stream)

    def run_and_check(self):
        H, V = self.H, self.V
        old = self.dtable.double()[:, :H]
        self.run()
        ids = self.ids.long()
        ok = (ids >= 0) & (ids < V)
        at = torch.where(ok, ids, 0)
        want = (self.table[at, :H].float() * self.scale).to(TD[self.dtype]) * ok[:, None]
        assert torch.equal(self.y[:, :H], want)
        for t in (self.y, self.dtable):
            assert bool((t[:, H:] == GUARD).all()), "a column between the rows was written"
        dy = (self.dy[:, :H].double() * self.scale) * ok[:, None]
        grad = torch.zeros(V, H, dtype=torch.float64, device="cuda").index_add_(0, at, dy)
        size = torch.zeros(V, H, dtype=torch.float64, device="cuda").index_add_(0, at, dy.abs())
        n = torch.bincount(at[ok], minlength=V).double()[:, None]
        r = 2.0 ** -8 if self.dtype == H16 and not self.accumulate else 2.0 ** -24
        if self.accumulate:
            grad, size = grad + old, size + old.abs()
        off = (self.dtable[:, :H].double() - grad).abs() - ((n * 2.0 ** -24 + 2.0 ** -22) * size + r * grad.abs())
        assert float(off.max()) <= 0, (float(off.max()), divmod(int(off.argmax()), H))
        gone = n[:, 0] == 0
        assert torch.equal(self.dtable[gone, :H].double(), old[gone] if self.accumulate else torch.zeros_like(old[gone]))


CASES = [  # dtype, rows, V, H, kind
    (H16, 1, 1, 1, "same"), (H16, 1, 5, 8, "uniform"), (H16, 2, 2, 3, "same"), (H16, 15, 3, 64, "some"), (H16, 16, 3, 64, "same"), (H16, 17, 1, 100, "same"),
    (H16, 33, 511, 512, "uniform"), (H16, 64, 512, 513, "rising"), (H16, 100, 30522, 1024, "some"), (H16, 1000, 7, 40, "some"), (H16, 1023, 4, 8, "pads"),
    (H16, 1025, 1, 250, "same"), (H16, 5000, 1 << 20, 24, "uniform"), (H16, 4097, 300, 1025, "some"), (H16, 3000, 100, 16, "none"), (H16, 9000, 2000, 72, "falling"),
    (H16, 70000, 1000, 8, "some"), (H16, 200001, 50, 5, "some"), (H16, 140000, 3, 20, "same"), (H16, 3000, 4000, 2047, "some"), (H16, 2500, 40, 4100, "pads"),
    (F, 1, 1, 1, "same"), (F, 31, 9, 4, "some"), (F, 3001, 517, 250, "pads"), (F, 2049, 70000, 33, "some"), (F, 40000, 2, 12, "uniform"), (F, 16, 16, 600, "rising"),
    (F, 1000, 262143, 16, "uniform"), (F, 1000, 262144, 16, "uniform"), (F, 66000, 512, 30, "uniform"),
]


@pytest.mark.parametrize("case", CASES, ids=lambda c: "-".join(str(v) for v in c))
@pytest.mark.parametrize("accumulate", [0, 1])
@pytest.mark.parametrize("pad", [0, 5])
def test_forward_and_backward(case, accumulate, pad):
    dtype, rows, V, H, kind = case
    Case(dtype, rows, V, H, kind=kind, accumulate=accumulate, pad=pad, skip=pad // 5).run_and_check()


@pytest.mark.parametrize("dtype", [F, H16])
def test_same_bits_on_another_stream_and_in_a_graph(dtype):
    c = Case(dtype, 5000, 900, 300)
    c.run()
    torch.cuda.synchronize()
    outs = (c.y, c.dtable)
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
        B.dapple_embedding_fwd(dtype, d, sp)
        B.dapple_embedding_bwd(dtype, d, sp)
    for k in range(3):
        c.ids.copy_(torch.roll(c.ids, 17) // 2)
        c.dy.mul_(-0.5)
        c.run()
        torch.cuda.synchronize()
        eager = [x.clone() for x in outs]
        for x in outs:
            x.fill_(GUARD)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, eager)), k
    del held


def test_offsets_beyond_32_bits():
    rows, V, H, ld = 700, 600, 40, 8_000_001      # the last rows lie past 2^32 elements (9.6 GB)
    a = Case(H16, rows, V, H, kind="uniform")
    a.run()
    big = torch.zeros(V * ld, dtype=torch.bfloat16, device="cuda").view(V, ld)
    big[:, :H] = a.table
    d = a.desc()
    y, want = a.y.clone(), a.dtable.clone()
    a.y.zero_()
    d.table, d.ldt, d.dtable, d.lddt = big.data_ptr(), ld, big.data_ptr() + 2 * 64, ld
    B.dapple_embedding_fwd(H16, d)
    B.dapple_embedding_bwd(H16, d)
    assert torch.equal(a.y, y) and torch.equal(big[:, 64:64 + H], want) and bool((big[:, 64 + H:200] == 0).all())


def test_gradient_against_differences():
    # linear in the table: the quotient is off by the roundings of a sum of 40 * 12 terms alone
    c = Case(F, 40, 6, 12)
    c.run()
    grad, d = c.dtable.clone(), c.desc()
    f = lambda: float((c.y.double() * c.dy.double()).sum()) if B.dapple_embedding_fwd(F, d) is None else 0  # noqa: E731
    for at in ((0, 0), (3, 7), (5, 11)):
        old, vals = c.table[at].clone(), []
        for sgn in (1, -1):
            c.table[at] = old + sgn
            vals.append(f())
        c.table[at] = old
        assert abs((vals[0] - vals[1]) / 2 - float(grad[at])) < 2.0 ** -24 * 480 * 8
