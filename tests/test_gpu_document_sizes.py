"""Attention of packed documents at sizes that choose other paths than short rows do; the cases and tolerances are those of
test_gpu_attention_docs.py."""
import pytest
import torch

from paper_2007_01045_amd import binding as B
from tests.test_gpu_attention_docs import Case, F, H, name

pytestmark = pytest.mark.gpu


def test_spans_of_more_than_2_to_the_30_documents():
    # almost all of them empty; the sum of two of their indices is beyond an int
    n, rows = (1 << 30) + 1000, 100
    ends = torch.zeros(n, dtype=torch.int32, device="cuda")
    ends[-3:] = torch.tensor([40, 40, 90], dtype=torch.int32, device="cuda")
    spans = torch.full((4 * rows + 1,), -9, dtype=torch.int32, device="cuda")
    B.dapple_doc_spans(ends.data_ptr(), n, rows, spans.data_ptr())
    lo, hi, qlo, qhi = spans[:-1].view(4, rows).cpu().tolist()
    assert int(spans[-1]) == 90
    for i in range(rows):
        begin, end = (0, 40) if i < 40 else (40, 90)
        assert (lo[i], hi[i], qlo[i], qhi[i]) == ((begin, i + 1, i, end) if i < 90 else (90,) * 4), i


def short(n, of=200):
    """n documents of 30 to 30 + of rows"""
    return [30 + (t * 53) % of for t in range(n)]


# rows beyond 64 tiles of queries (ranked in groups of neighbours where a launch has more than 256 of them) and 256 of keys (more than the plan has
# threads), walks of one document that are cut among many that are not
LONG = [  # dtype, rows, docs, A, Ak, d, causal, prefix, W, cap, slope
    (H, 9000, short(20) + [2400] + short(25) + [1], 8, 4, 64, True, None, 0, 0.0, 0.05), (H, 20011, short(60) + [2800, 1900] + short(40), 4, 1, 32, True, True, 0, 30.0, 0.0),
    (H, 18000, [2300] + short(100), 1, 1, 64, False, None, 0, 0.0, 0.0), (H, 34000, short(130) + [2800] + short(80), 4, 2, 64, True, True, 0, 0.0, 0.0),
    (H, 34000, short(130) + [2800] + short(90), 8, 2, 128, True, None, 0, 50.0, 0.0), (H, 33333, short(200) + [2000, 33], 4, 4, 80, False, None, 300, 50.0, 0.05),
    (F, 8300, short(30) + [1700] + short(15), 2, 1, 64, True, None, 0, 0.0, 0.0), (F, 17000, short(50) + [1800] + short(40), 4, 2, 32, True, True, 0, 20.0, 0.05),
]
# heads wider than 64 whose dq is in the launch of dk and dv: every kind of logits
WIDE = [(H, 2100, [900, 0, 700, 450], 32, 8, 128, causal, causal or None, W, cap, slope)
        for causal, W, cap, slope in ((True, 0, 0.0, 0.0), (True, 0, 50.0, 0.0), (True, 0, 50.0, 0.1), (True, 0, 0.0, 0.1), (False, 150, 30.0, 0.1))]
# more documents than are searched in LDS, a few of them empty
MANY = [(dtype, 4500, [0, 1, 2, 3, 4] * 420 + [200], 4, 2, 64, True, True, 0, 20.0, 0.1) for dtype in (F, H)]


@pytest.mark.parametrize("case", LONG + WIDE + MANY, ids=name)
def test_forward_and_backward(case):
    c = Case(*case)
    c.run()
    c.check()
    first = c.dqkv.clone()      # (the plan lists its parts in an order that may change: no result goes by it)
    c.dqkv.fill_(3)
    c.run()
    w = c.ld - c.pad
    assert torch.equal(c.dqkv[:, :w], first[:, :w])


@pytest.mark.parametrize("rows", [2090, 2091, 2092, 9000])
def test_spans_of_many_documents(rows):
    # one row each but for an empty one behind every seventh, and a long one: 2047, 2048, 2049 and 9944 of them
    docs = [n for t in range(rows - 300) for n in ((1, 0) if t % 7 == 0 else (1,))] + [290]
    ends = torch.tensor(docs).cumsum(0).int().cuda()
    spans = torch.full((4 * rows + 1,), -9, dtype=torch.int32, device="cuda")
    B.dapple_doc_spans(ends.data_ptr(), len(docs), rows, spans.data_ptr(), causal=0)
    length = torch.tensor(docs, device="cuda")
    end = ends.long().repeat_interleave(length)
    begin = (ends - length).long().repeat_interleave(length)
    behind = torch.full((10,), rows - 10, device="cuda")
    lo, hi, qlo, qhi = spans[:-1].view(4, rows).long()
    assert int(spans[-1]) == rows - 10
    for got, want in ((lo, begin), (hi, end), (qlo, begin), (qhi, end)):
        assert torch.equal(got, torch.cat([want, behind]))


@pytest.mark.parametrize("s, A, Ak, d, W", [(300, 4, 2, 64, 90), (3000, 4, 1, 64, 0), (2500, 16, 4, 128, 0), (2500, 32, 8, 128, 700)])
@pytest.mark.parametrize("dtype", [F, H])
def test_gradients_equal_to_the_window_operator(dtype, s, A, Ak, d, W):
    """One document, no cap, no slopes: dq is of the same products in the same order, dk and dv of the same products, whose walks may be cut
    elsewhere.  A sum of m products in whatever order is off by m * 2^-24 of their sizes at most, and both are rounded once (r)."""
    c = Case(dtype, s, [s], A, Ak, d, True, None, W, pad=0)
    c.run()
    got = c.dqkv.clone()
    t = c.desc()
    w = B.attention_window_desc(**{n: getattr(t, n) for n in ("q", "k", "v", "ctx", "ctx32", "lse", "dctx", "dq", "dk", "dv", "ldq", "ldk", "ldv", "ldc", "lddc", "lddq",
                                                               "lddk", "lddv")}, b=1, s=s, A=A, Ak=Ak, d=d, window=W, causal=1)
    ws = torch.empty(B.dapple_attention_window_workspace(dtype, w), dtype=torch.uint8, device="cuda")
    w.workspace = ws.data_ptr()
    c.dqkv.zero_()
    B.dapple_attention_window_fwd(dtype, w)
    B.dapple_attention_window_bwd(dtype, w)
    assert torch.equal(got[:, :A * d], c.dqkv[:, :A * d])
    heads = lambda t, at, n: t[:, at * d:(at + n) * d].double().view(s, n, d).transpose(0, 1)  # noqa: E731
    q, k, v, g = heads(c.qkv, 0, A), heads(c.qkv, A, Ak), heads(c.qkv, A + Ak, Ak), heads(c.dctx, 0, A)
    i = torch.arange(s, device="cuda")
    gap = i[:, None] - i[None, :]
    hidden = (gap < 0) | (gap >= (W or s))
    r, m = (2.0 ** -8 if dtype == H else 2.0 ** -24), s * A // Ak
    scale = d ** -0.5
    for h in range(Ak):
        sizes = [torch.zeros(s, d, dtype=torch.float64, device="cuda") for _ in range(2)]
        for a in range(h * A // Ak, (h + 1) * A // Ak):
            p = torch.softmax((q[a] @ k[h].T.contiguous() * scale).masked_fill_(hidden, float("-inf")), -1)
            ds = p * (g[a] @ v[h].T.contiguous() - (g[a] * (p @ v[h])).sum(-1, keepdim=True))
            sizes[0] += scale * (ds.abs().T.contiguous() @ q[a].abs())
            sizes[1] += p.T.contiguous() @ g[a].abs()
        for at, size in ((A + h, sizes[0]), (A + Ak + h, sizes[1])):
            one, two = (x[:, at * d:(at + 1) * d].double() for x in (got, c.dqkv))
            # (dS near 0 is itself off by 2^-13 of its terms at most, the probabilities by as much of themselves: the sizes' twice is enough)
            assert bool(((one - two).abs() <= 2 * m * 2.0 ** -24 * 2 * size + r * (one.abs() + two.abs()) + 1e-12).all()), (at, "differs")


# more key heads than a launch has shares, one, one and two of them; a bias that rises with the distance; prefixes beyond a tile of queries
OTHERS = [(H, 1100, [1090], 200, 200, 64, True, None, 0, 0.0, 0.0), (H, 300, [100, 190], 256, 256, 32, False, None, 0, 20.0, 0.0), (F, 700, [690], 172, 172, 16, True, None, 0, 0.0, 0.0),
          (H, 500, [170, 320], 8, 2, 64, True, None, 0, 0.0, -0.1), (H, 500, [320, 170], 8, 2, 128, False, None, 0, 30.0, -0.1), (F, 500, [320, 170], 4, 2, 64, True, True, 0, 0.0, -0.1),
          (H, 900, [800, 77], 4, 2, 64, True, [500, 77], 0, 0.0, 0.1), (H, 900, [800, 77], 4, 2, 128, True, [500, 100], 300, 0.0, 0.0), (F, 900, [800, 77], 4, 2, 64, True, [500, 0], 0, 0.0, 0.0)]


@pytest.mark.parametrize("case", OTHERS, ids=name)
def test_other_heads_slopes_and_prefixes(case):
    c = Case(*case)
    c.run()
    c.check()


@pytest.mark.parametrize("dtype", [F, H])
def test_tensors_of_their_own_strides(dtype):
    # as they lie in one buffer, and each in a buffer of its own with another stride: the same bits
    c = Case(dtype, 333, [100, 33, 180], 4, 2, 64, True, True, 0, 30.0, 0.1)
    c.run()
    A, Ak, d, rows = c.A, c.Ak, c.d, c.rows
    td, t = c.qkv.dtype, c.desc()
    room = lambda heads, more, kind=td: torch.full((rows, heads * d + more), 7.0, device="cuda").to(kind)  # noqa: E731
    q, k, v, g = room(A, 16), room(Ak, 0), room(Ak, 40), room(A, 72)
    for to, src, at, heads in ((q, c.qkv, 0, A), (k, c.qkv, A, Ak), (v, c.qkv, A + Ak, Ak), (g, c.dctx, 0, A)):
        to[:, :heads * d] = src[:, at * d:(at + heads) * d]
    ctx, c32, lse, dq, dk, dv = room(A, 24), room(A, 24, torch.float32), torch.empty_like(c.lse), room(A, 8), room(Ak, 56), room(Ak, 0)
    for n, x in dict(q=q, k=k, v=v, ctx=ctx, ctx32=c32, lse=lse, dctx=g, dq=dq, dk=dk, dv=dv).items():
        setattr(t, n, x.data_ptr())
    for n, x in dict(ldq=q, ldk=k, ldv=v, ldc=ctx, lddc=g, lddq=dq, lddk=dk, lddv=dv).items():
        setattr(t, n, x.shape[1])
    t.ldk = t.lddv = 0      # (dense)
    B.dapple_attention_docs_fwd(dtype, t)
    B.dapple_attention_docs_bwd(dtype, t)
    for got, want, at, heads in ((ctx, c.ctx, 0, A), (c32, c.c32, 0, A), (dq, c.dqkv, 0, A), (dk, c.dqkv, A, Ak), (dv, c.dqkv, A + Ak, Ak)):
        assert torch.equal(got[:, :heads * d], want[:, at * d:(at + heads) * d]) and bool((got[:, heads * d:] == 7).all())
    assert torch.equal(lse, c.lse)


@pytest.mark.parametrize("dtype", [F, H])
def test_offsets_beyond_32_bits(dtype):
    # rows up to the last that the operator takes at this stride (below 2^30 - 4096 elements, 4 GiB in fp32); the documents at the end are checked
    rows, docs = 1 << 20, [200, 1, 320, 55]
    pad = 1016 - 4 * 64
    n = sum(docs)
    front = [1] * 63 + [1 << 10] * 1023
    front += [rows - n - 7 - sum(front)]
    c = Case(dtype, rows, front + docs, 2, 1, 64, True, None, 0, 0.0, 0.1, pad=pad)
    assert c.ld == 1016 and rows * c.ld < (1 << 30) - 4096
    c.run()
    at = rows - n - 7
    assert c.len == rows - 7
    small = Case(dtype, n + 7, docs, 2, 1, 64, True, None, 0, 0.0, 0.1, pad=pad)
    small.qkv, small.dctx, small.ctx, small.c32, small.dqkv, small.lse = c.qkv[at:], c.dctx[at:], c.ctx[at:], c.c32[at:], c.dqkv[at:], c.lse[:, at:]
    small.check()


@pytest.mark.parametrize("cap", [2.0 ** -20, 1.0, 50.0, 1024.0])
@pytest.mark.parametrize("dtype", [F, H])
def test_how_far_capped_logits_are_off(dtype, cap):
    """Documents of one row: lse is the logit.  fp32: tanh's argument has three roundings and tanh two.  bf16, (1 - e) / (1 + e) with e = 2^-|a|: e is off
    by its last place, 2^-24 at most, which is half of that of t; a by three roundings, 1.4 * 2^-24 of t at most; the reciprocal by its last place, 2 *
    2^-24 of t, and sum, difference and product by 3 * 2^-24.  Both: the constants and products around it and log2 of the sum, five
    roundings of the logit more.  Together below 2^-20 of the logit, and in bf16 2^-24 of the cap."""
    rows = 20000
    x = torch.cat([torch.linspace(-12, 12, rows // 2, device="cuda"), 2.0 ** torch.linspace(-20, 4, rows // 2, device="cuda")]) * cap
    c = Case(dtype, rows, [1] * rows, 1, 1, 8, cap=cap, scale=1.0, pad=0)
    c.qkv.zero_()
    c.qkv[:, 0], c.qkv[:, 8] = x.to(c.qkv.dtype), 1
    c.make_spans()
    B.dapple_attention_docs_fwd(dtype, c.desc())
    logit = cap * torch.tanh(c.qkv[:, 0].double() / cap)
    off = (c.lse[0].double() * 0.6931471805599453 - logit).abs() - 2.0 ** -20 * logit.abs()
    assert float(off.max()) <= (cap * 2.0 ** -24 if dtype == H else 0.0), float(off.max()) / cap
