"""The operators around and in a layer run together, as a training step over packed documents uses them:
   z0 = dropout(scale * table[ids]), h = layer norm(z0);  q, k, v = h Wqkv;  c = attention of the documents (capped, with prefixes and bias);
   z1 = z0 + dropout(c Wo + bo), y = RMS norm(z1);  loss = sum of y dy + z1 dz
forward and backward, against float64 autograd on the same inputs and masks.

Tolerances, relative 2-norms.  bf16: a gradient comes through at most twelve tensors that were rounded to bf16 (2^-9 of a tensor in the
2-norm, at most), which the steps behind them pass on at most doubled here: 12 * 2 * 2^-9 = 0.047.  fp32: each of six products of at most
600 terms is off by at most 600 * 2^-24 of its terms' sizes, sums that cancel by a fourth at most: 6 * 4 * 600 * 2^-24 = 9e-4."""
import math

import numpy as np
import pytest
import torch

from paper_2007_01045_amd import binding as B
from tests.dropout_util import keep_mask

pytestmark = pytest.mark.gpu
TD = {B.DTYPE_F32: torch.float32, B.DTYPE_BF16: torch.bfloat16}
TOL = {B.DTYPE_F32: 9e-4, B.DTYPE_BF16: 0.047}
T, A, Ak, d, V, P, EPS, CAP, SCALE = 393, 4, 2, 64, 211, 0.1, 1e-5, 20.0, 1.5
H, N = A * d, (A + 2 * Ak) * d
DOCS, PREFIX = [150, 1, 0, 77, 130], [10, 1, 0, 200, 0]


class Step:
    def __init__(self, dtype, seed=1):
        self.dtype, td, f32 = dtype, TD[dtype], torch.float32
        gen = torch.Generator(device="cuda").manual_seed(seed)
        normal = lambda sc, *n, t=td: (sc * torch.randn(*n, generator=gen, device="cuda")).to(t)  # noqa: E731
        room = lambda *n, t=td: torch.empty(*n, dtype=t, device="cuda")  # noqa: E731
        self.table, self.w_qkv, self.w_o, self.b_o = normal(1, V, H), normal(H ** -0.5, H, N), normal(H ** -0.5, H, H), normal(0.3, H)
        self.g0, self.be0, self.g1 = normal(0.2, H) + 1, normal(0.2, H), normal(0.2, H) + 1
        self.ids = torch.randint(-5, V, (T,), generator=gen, device="cuda").int()
        self.ends, self.prefix = torch.tensor(DOCS).cumsum(0).int().cuda(), torch.tensor(PREFIX).int().cuda()
        self.slopes = 0.25 * 0.5 ** torch.arange(A, device="cuda", dtype=f32)
        self.rng = torch.tensor([1234567890123 + seed, 7], device="cuda")
        self.dy, self.dz1 = normal(1, T, H), normal(1, T, H, t=f32)
        self.e, self.h, self.o, self.y, self.ctx, self.qkv = room(T, H), room(T, H), room(T, H), room(T, H), room(T, H), room(T, N)
        self.z0, self.z1, self.ctx32, self.lse = room(T, H, t=f32), room(T, H, t=f32), room(T, H, t=f32), room(A, T, t=f32)
        self.s0, self.s1, self.spans = room(T, 2, t=f32), room(T, 2, t=f32), room(4 * T + 1, t=torch.int32)
        self.do, self.dz0, self.dctx, self.dqkv, self.dh, self.de = room(T, H), room(T, H, t=f32), room(T, H), room(T, N), room(T, H), room(T, H)
        self.dtable, self.dw_qkv, self.dw_o = room(V, H, t=f32), room(H, N, t=f32), room(H, H, t=f32)
        self.db_o, self.dg0, self.dbe0, self.dg1 = (room(H, t=f32) for _ in range(4))
        p = lambda t: t.data_ptr()  # noqa: E731
        es = self.e.element_size()
        self.emb = B.embedding_desc(table=p(self.table), ids=p(self.ids), y=p(self.e), dy=p(self.de), dtable=p(self.dtable), rows=T, V=V, H=H,
                                    accumulate=1, scale=SCALE)
        common = dict(rng=p(self.rng), rows=T, H=H, stream32=1, p=P, eps=EPS)
        self.n0 = B.dropout_norm_desc(x=p(self.e), gamma=p(self.g0), beta=p(self.be0), z=p(self.z0), y=p(self.h), stats=p(self.s0), dy=p(self.dh),
                                      dz=p(self.dz0), dx=p(self.de), dgamma=p(self.dg0), dbeta=p(self.dbe0), norm=B.NORM_LAYER, site=0, **common)
        self.n1 = B.dropout_norm_desc(x=p(self.o), bias=p(self.b_o), residual=p(self.z0), gamma=p(self.g1), z=p(self.z1), y=p(self.y), stats=p(self.s1),
                                      dy=p(self.dy), dz=p(self.dz1), dx=p(self.do), dresidual=p(self.dz0), dbias=p(self.db_o), dgamma=p(self.dg1),
                                      norm=B.NORM_RMS, site=1, **common)
        q, g, k, v = p(self.qkv), p(self.dqkv), A * d * es, (A + Ak) * d * es
        self.att = B.attention_docs_desc(q=q, k=q + k, v=q + v, ctx=p(self.ctx), ctx32=p(self.ctx32), lse=p(self.lse), spans=p(self.spans),
                                         slopes=p(self.slopes), dctx=p(self.dctx), dq=g, dk=g + k, dv=g + v, rows=T, A=A, Ak=Ak, d=d, ldq=N, ldk=N,
                                         ldv=N, lddq=N, lddk=N, lddv=N, cap=CAP)
        self.ws = []
        for desc, size in ((self.emb, B.dapple_embedding_workspace), (self.n0, B.dapple_dropout_norm_workspace),
                           (self.n1, B.dapple_dropout_norm_workspace), (self.att, B.dapple_attention_docs_workspace)):
            self.ws.append(torch.empty(size(dtype, desc), dtype=torch.uint8, device="cuda"))
            desc.workspace = p(self.ws[-1])

    def step(self, stream=None):
        dt, p = self.dtype, lambda t: t.data_ptr()  # noqa: E731

        def gemm(a, b, c, **kw):
            B.dapple_gemm(dt, B.dapple_gemm_desc(A=p(a), B=p(b), C=p(c), batch=1, **kw), stream)

        for g in (self.dtable, self.dw_qkv, self.dw_o):
            g.zero_()
        B.dapple_doc_spans(p(self.ends), len(DOCS), T, p(self.spans), prefix_ptr=p(self.prefix), stream_ptr=stream)
        B.dapple_embedding_fwd(dt, self.emb, stream)
        B.dapple_dropout_norm_fwd(dt, self.n0, stream)
        gemm(self.h, self.w_qkv, self.qkv, M=T, N=N, K=H, lda=H, ldb=N, ldc=N, b_kstrided=1)
        B.dapple_attention_docs_fwd(dt, self.att, stream)
        gemm(self.ctx, self.w_o, self.o, M=T, N=H, K=H, lda=H, ldb=H, ldc=H, b_kstrided=1)
        B.dapple_dropout_norm_fwd(dt, self.n1, stream)
        B.dapple_dropout_norm_bwd(dt, self.n1, stream)
        weight = dict(a_kstrided=1, b_kstrided=1, epi=B.EPI_ACC32)
        gemm(self.ctx, self.do, self.dw_o, M=H, N=H, K=T, lda=H, ldb=H, ldc=H, **weight)
        gemm(self.do, self.w_o, self.dctx, M=T, N=H, K=H, lda=H, ldb=H, ldc=H)
        B.dapple_attention_docs_bwd(dt, self.att, stream)
        gemm(self.h, self.dqkv, self.dw_qkv, M=H, N=N, K=T, lda=H, ldb=N, ldc=N, **weight)
        gemm(self.dqkv, self.w_qkv, self.dh, M=T, N=H, K=N, lda=N, ldb=N, ldc=H)
        B.dapple_dropout_norm_bwd(dt, self.n0, stream)
        B.dapple_embedding_bwd(dt, self.emb, stream)

    def outputs(self):
        return [self.y, self.z1, self.dtable, self.dg0, self.dbe0, self.dw_qkv, self.dw_o, self.db_o, self.dg1]

    def mask(self, site):
        level = round(65536 * float(np.float32(P)))
        seed, step = self.rng.tolist()
        return torch.from_numpy(keep_mask(seed, step, site, T, H, P)).cuda().double() * (65536 / (65536 - level))

    def want(self):
        leaves = [t.double().requires_grad_(True) for t in (self.table, self.g0, self.be0, self.w_qkv, self.w_o, self.b_o, self.g1)]
        table, g0, be0, w_qkv, w_o, b_o, g1 = leaves
        inside = self.ids >= 0
        z0 = SCALE * table[self.ids.clamp_min(0).long()] * inside[:, None] * self.mask(0)
        h = torch.nn.functional.layer_norm(z0, (H,), g0, be0, EPS)
        q, k, v = (h @ w_qkv).view(T, -1, d).transpose(0, 1).split([A, Ak, Ak], dim=0)
        k, v = k.repeat_interleave(A // Ak, 0), v.repeat_interleave(A // Ak, 0)
        doc, place = torch.full((T,), -1, device="cuda"), torch.zeros(T, device="cuda").long()
        at = 0
        for n, length in enumerate(DOCS):
            doc[at:at + length] = n
            place[at:at + length] = torch.arange(length, device="cuda")
            at += length
        gap = place[:, None] - place[None, :]
        free = place < torch.tensor(PREFIX, device="cuda")[doc.clamp_min(0)]
        ok = (doc[:, None] == doc[None, :]) & (doc[:, None] >= 0) & ((gap >= 0) | free[None, :])
        t = CAP * torch.tanh(q @ k.transpose(1, 2).contiguous() * d ** -0.5 / CAP) - self.slopes.double()[:, None, None] * gap.abs()
        pr = torch.softmax(t.masked_fill(~ok, -1e300), -1) * ok
        o = (pr @ v.contiguous()).transpose(0, 1).reshape(T, H) @ w_o + b_o
        z1 = z0 + o * self.mask(1)
        y = z1 * torch.rsqrt(z1.square().mean(-1, keepdim=True) + EPS) * g1
        grads = torch.autograd.grad((y * self.dy.double()).sum() + (z1 * self.dz1.double()).sum(), leaves)
        return [y.detach(), z1.detach(), *grads]


@pytest.mark.parametrize("dtype", [B.DTYPE_F32, B.DTYPE_BF16])
def test_a_step_and_its_gradients(dtype):
    s = Step(dtype)
    s.step()
    for n, (got, want) in enumerate(zip(s.outputs(), s.want())):
        assert bool(got.isfinite().all()), n
        assert float((got.double() - want).norm()) <= TOL[dtype] * float(want.norm()), (n, float((got.double() - want).norm() / want.norm()))
    # absent tokens have no gradient
    absent = torch.ones(V, dtype=torch.bool, device="cuda")
    absent[s.ids[s.ids >= 0].long()] = False
    assert bool((s.dtable[absent] == 0).all()) and math.isfinite(float(s.dtable.sum()))


@pytest.mark.parametrize("dtype", [B.DTYPE_F32, B.DTYPE_BF16])
def test_two_steps_on_two_streams_and_in_a_graph(dtype):
    one, two = Step(dtype, 1), Step(dtype, 2)
    want = []
    for s in (one, two):
        s.step()
        torch.cuda.synchronize()
        want.append([t.clone() for t in s.outputs()])
        for t in s.outputs():
            t.fill_(7)
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    for _ in range(3):
        for s, st in zip((one, two), streams):
            with torch.cuda.stream(st):
                s.step(st.cuda_stream)
    torch.cuda.synchronize()
    for s, w in zip((one, two), want):
        assert all(torch.equal(x, y) for x, y in zip(s.outputs(), w))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        one.step(torch.cuda.current_stream().cuda_stream)
        two.step(torch.cuda.current_stream().cuda_stream)
    for k in range(3):      # other masks, documents and tokens in the same graph
        for s in (one, two):
            s.rng[1] += 1
            s.ends.copy_(torch.tensor([100 + k, 100 + k, 160, 161, 350 + k]).int())
            s.ids.copy_(torch.roll(s.ids, 5))
            s.step()
        torch.cuda.synchronize()
        eager = [[t.clone() for t in s.outputs()] for s in (one, two)]
        for s in (one, two):
            for t in s.outputs():
                t.fill_(7)
        graph.replay()
        torch.cuda.synchronize()
        for s, w in zip((one, two), eager):
            assert all(torch.equal(x, y) for x, y in zip(s.outputs(), w)), k
