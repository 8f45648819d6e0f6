"""The embedding and the end of a block at sizes that choose other paths than small calls do: rows and tables that are not kept in the
memory-side cache, workgroups that take several rows each.  The cases and tolerances are those of test_gpu_embedding.py and
test_gpu_dropout_norm.py (sums over rows: 4133 rows are 17 to a workgroup, 16 workgroups to a wave and 16 waves, 49 deep)."""
import pytest
import torch

from paper_2007_01045_amd import binding as B
from tests import test_gpu_dropout_norm as N
from tests import test_gpu_embedding as E

pytestmark = pytest.mark.gpu
F, H16 = B.DTYPE_F32, B.DTYPE_BF16
MiB = 1 << 20


# from 128 MiB of rows, and of table, on
FAR = [  # dtype, rows, V, H, kind
    (H16, 65536, 66000, 1024, "some"), (H16, 65537, 65600, 1027, "pads"), (H16, 1 << 20, 1000, 64, "uniform"), (H16, 3000, 30000, 2304, "uniform"),
    (F, 33000, 40001, 1024, "pads"), (F, 70001, 67200, 501, "some"), (F, 4200, 10, 8192, "same"),
]


@pytest.mark.parametrize("case", FAR, ids=lambda c: "-".join(str(v) for v in c))
@pytest.mark.parametrize("accumulate", [0, 1])
@pytest.mark.parametrize("pad", [0, 5])
def test_embedding_of_large_rows_and_tables(case, accumulate, pad):
    dtype, rows, V, H, kind = case
    es = 2 if dtype == H16 else 4
    assert max(rows, V) * H * es >= 128 * MiB
    c = E.Case(dtype, rows, V, H, kind=kind, accumulate=accumulate, pad=pad, skip=pad // 5)
    c.run_and_check()
    if not accumulate:
        first = c.dtable.clone()
        c.dtable[:, :H] = 3
        c.run()
        assert torch.equal(c.dtable, first)


# rows beyond the forward's workgroups: 2048 for one or two waves to a row (four rows each in the first case), 4096 above
ROWS = [(4 * 2048 * 2 + 5, 200), (2 * 2048 + 1, 520), (2 * 2048 + 1, 1000), (4096 + 37, 1100), (4096 + 37, 4100), (4096 + 37, 8200)]


@pytest.mark.parametrize("rows, H", ROWS)
@pytest.mark.parametrize("dtype, stream32, norm, pad", [(H16, False, N.LAYER, 0), (H16, True, N.RMS, 3), (H16, True, N.LAYER, 8), (F, False, N.LAYER, 0), (F, False, N.RMS, 3)])
def test_norm_of_several_rows_to_a_workgroup(rows, H, dtype, stream32, norm, pad):
    c = N.Case(dtype, rows, H, norm, 0.1, stream32, pad=pad, skip=pad % 8 // 3)
    c.run()
    c.check()
    # outputs in their inputs' place: a row that is loaded ahead is not the one that is written
    d = N.Case(dtype, rows, H, norm, 0.1, stream32, pad=pad, skip=pad % 8 // 3)
    q = lambda t: t.data_ptr()  # noqa: E731
    desc = d.desc(z=q(d.res), y=q(d.x), dresidual=q(d.dz), dx=q(d.dy))
    B.dapple_dropout_norm_fwd(dtype, desc)
    B.dapple_dropout_norm_bwd(dtype, desc)
    for got, want in ((d.res, c.z), (d.x, c.y), (d.dz, c.dr), (d.dy, c.dx)):
        assert torch.equal(got, want)
    assert all(torch.equal(x, y) for x, y in zip(c.sums, d.sums))
