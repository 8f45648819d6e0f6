"""The operators of a layer and a training step run together, as a layer with shared key heads and a gated feed-forward block uses them:
   qkv = x Wqkv;  q, k normed and turned in place;  ctx = attention(q, k, v);  y = block(ctx);  loss = sum of y dy
forward and backward, the gradients' norm and their clipping, against float64 autograd on the same inputs.

Tolerances, relative 2-norms.  bf16: a gradient comes through at most twelve tensors that were rounded to bf16 (2^-9 of a tensor in the
2-norm, at most), which the steps behind them pass on at most doubled here: 12 * 2 * 2^-9 = 0.047.  fp32: each of six products of at most
600 terms is off by at most 600 * 2^-24 of its terms' sizes, sums that cancel by a fourth at most (terms of random signs, square root of
600 of 600, would be worse, were their errors not random with them): 6 * 4 * 600 * 2^-24 = 9e-4."""
import pytest
import torch

from paper_2007_01045_amd import binding as B

pytestmark = pytest.mark.gpu
TD = {B.DTYPE_F32: torch.float32, B.DTYPE_BF16: torch.bfloat16}
TOL = {B.DTYPE_F32: 9e-4, B.DTYPE_BF16: 0.047}
b, s, A, Ak, d, F, WINDOW, SINKS, EPS, MAX_NORM = 3, 147, 4, 2, 64, 520, 40, 3, 1e-6, 0.5
H, N, T = A * d, (A + 2 * Ak) * d, b * s
LENS = [147, 0, 93]


class Layer:
    def __init__(self, dtype, seed=1):
        self.dtype, td = dtype, TD[dtype]
        gen = torch.Generator(device="cuda").manual_seed(seed)
        normal = lambda sc, *n: (sc * torch.randn(*n, generator=gen, device="cuda")).to(td)  # noqa: E731
        self.x, self.dy = normal(1, T, H), normal(1, T, H)
        self.w_qkv = normal(H ** -0.5, H, N)
        self.gq, self.gk = (normal(0.2, d) + 1 for _ in range(2))
        self.w_in, self.b_in, self.w_out, self.b_out = normal(H ** -0.5, H, 2 * F), normal(0.3, 2 * F), normal(F ** -0.5, F, H), normal(0.3, H)
        self.lens = torch.tensor(LENS, dtype=torch.int32, device="cuda")
        # padded rows: positions of another sequence's, outside the table in the last ones; dy is zero there
        self.pos = torch.arange(s, dtype=torch.int32, device="cuda").repeat(b).contiguous()
        self.seen = (torch.arange(s, device="cuda") < self.lens[:, None]).reshape(-1)
        self.dy[~self.seen] = 0
        self.table = torch.empty(s, d // 2, 2, device="cuda")
        B.dapple_rope_table(self.table.data_ptr(), s, d)
        room = lambda *n, t=td: torch.empty(*n, dtype=t, device="cuda")  # noqa: E731
        self.qkv, self.turned, self.ctx, self.ctx32 = room(T, N), room(T, (A + Ak) * d), room(T, H), room(T, H, t=torch.float32)
        self.lse, self.gu, self.h, self.y = room(b, A, s, t=torch.float32), room(T, 2 * F), room(T, F), room(T, H)
        self.dgu, self.dctx, self.dqkv = room(T, 2 * F), room(T, H), room(T, N)
        f32 = torch.float32
        self.grads = [room(H, N, t=f32), room(d, t=f32), room(d, t=f32), room(H, 2 * F, t=f32), room(2 * F, t=f32), room(F, H, t=f32), room(H, t=f32)]
        self.norm = room(2, t=f32)
        self.clipped = [torch.empty_like(g) for g in self.grads]
        es, p = self.x.element_size(), lambda t: t.data_ptr()  # noqa: E731
        k, v, dk, dv = p(self.qkv) + H * es, p(self.qkv) + (H + Ak * d) * es, p(self.dqkv) + H * es, p(self.dqkv) + (H + Ak * d) * es
        lt = (A + Ak) * d
        self.rope = B.qk_rope_desc(q=p(self.qkv), k=k, gamma_q=p(self.gq), gamma_k=p(self.gk), positions=p(self.pos), table=p(self.table),
                                   yq=p(self.turned), yk=p(self.turned) + H * es, dyq=p(self.dqkv), dyk=dk, dq=p(self.dqkv), dk=dk,
                                   dgamma_q=p(self.grads[1]), dgamma_k=p(self.grads[2]), rows=T, A=A, Ak=Ak, d=d, rot=d, max_pos=s, accumulate=1,
                                   ldq=N, ldk=N, ldyq=lt, ldyk=lt, lddyq=N, lddyk=N, lddq=N, lddk=N, eps=EPS)
        self.attn = B.attention_window_desc(q=p(self.turned), k=p(self.turned) + H * es, v=v, ctx=p(self.ctx), ctx32=p(self.ctx32), lse=p(self.lse),
                                            lens=p(self.lens), dctx=p(self.dctx), dq=p(self.dqkv), dk=dk, dv=dv, b=b, s=s, A=A, Ak=Ak, d=d,
                                            window=WINDOW, sinks=SINKS, causal=1, ldq=lt, ldk=lt, ldv=N, lddq=N, lddk=N, lddv=N)
        self.ffn = B.gated_ffn_desc(x=p(self.ctx), w_in=p(self.w_in), b_in=p(self.b_in), w_out=p(self.w_out), b_out=p(self.b_out), gu=p(self.gu),
                                    h=p(self.h), y=p(self.y), dy=p(self.dy), dgu=p(self.dgu), dx=p(self.dctx), dw_in=p(self.grads[3]),
                                    db_in=p(self.grads[4]), dw_out=p(self.grads[5]), db_out=p(self.grads[6]), T=T, H=H, F=F, act=B.ACT_SILU, accumulate=1)
        self.ptrs, self.sizes = [p(g) for g in self.grads], [g.numel() for g in self.grads]
        self.ws = []
        for desc, size in ((self.rope, B.dapple_qk_rope_workspace(dtype, self.rope)), (self.attn, B.dapple_attention_window_workspace(dtype, self.attn)),
                           (self.ffn, B.dapple_gated_ffn_workspace(dtype, self.ffn))):
            self.ws.append(torch.empty(size, dtype=torch.uint8, device="cuda"))
            desc.workspace = p(self.ws[-1])
        self.norm_ws = torch.empty(B.dapple_grad_norm_workspace(self.sizes), dtype=torch.uint8, device="cuda")

    def gemm(self, stream, **kw):
        B.dapple_gemm(self.dtype, B.dapple_gemm_desc(batch=1, **kw), stream)

    def step(self, stream=None):
        for g in self.grads:
            g.zero_()
        dt, p = self.dtype, lambda t: t.data_ptr()  # noqa: E731
        self.gemm(stream, A=p(self.x), B=p(self.w_qkv), C=p(self.qkv), M=T, N=N, K=H, lda=H, ldb=N, ldc=N, b_kstrided=1)
        B.dapple_qk_rope_fwd(dt, self.rope, stream)
        B.dapple_attention_window_fwd(dt, self.attn, stream)
        B.dapple_gated_ffn_fwd(dt, self.ffn, stream)
        B.dapple_gated_ffn_bwd(dt, self.ffn, stream)
        B.dapple_attention_window_bwd(dt, self.attn, stream)
        B.dapple_qk_rope_bwd(dt, self.rope, stream)          # (in place on the queries' and keys' columns of dqkv)
        self.gemm(stream, A=p(self.x), B=p(self.dqkv), C=p(self.grads[0]), M=H, N=N, K=T, lda=H, ldb=N, ldc=N, a_kstrided=1, b_kstrided=1,
                  epi=B.EPI_ACC32)
        B.dapple_grad_norm(B.DTYPE_F32, self.ptrs, self.sizes, MAX_NORM, p(self.norm), p(self.norm_ws), 1.0, stream)
        B.dapple_grad_clip(B.DTYPE_F32, self.ptrs, [p(c) for c in self.clipped], self.sizes, p(self.norm), stream)

    def outputs(self):
        return [self.y, self.norm, *self.grads, *self.clipped]

    def want(self):
        leaf = lambda t: t.double().requires_grad_(True)  # noqa: E731
        w_qkv, gq, gk, w_in, b_in, w_out, b_out = leaves = [leaf(t) for t in (self.w_qkv, self.gq, self.gk, self.w_in, self.b_in, self.w_out, self.b_out)]
        qkv = (self.x.double() @ w_qkv).view(b, s, -1, d)
        q, k, v = qkv.split([A, Ak, Ak], dim=2)
        angle = torch.arange(s, device="cuda", dtype=torch.float64)[:, None] * 10000.0 ** (-2 * torch.arange(d // 2, device="cuda", dtype=torch.float64) / d)
        c, sn = angle.cos()[None, :, None], angle.sin()[None, :, None]

        def turn(t, gamma):
            n = t * torch.rsqrt(t.square().mean(-1, keepdim=True) + EPS) * gamma
            x1, x2 = n.chunk(2, dim=-1)
            return torch.cat([x1 * c - x2 * sn, x1 * sn + x2 * c], dim=-1)

        q, k = turn(q, gq), turn(k, gk).repeat_interleave(A // Ak, dim=2)
        v = v.repeat_interleave(A // Ak, dim=2)
        i, j = torch.arange(s, device="cuda")[:, None], torch.arange(s, device="cuda")[None, :]
        ok = (((i - j).abs() < WINDOW) | (j < SINKS)) & (j <= i)
        ok = (ok[None] & (i < self.lens[:, None, None]) & (j < self.lens[:, None, None]))[:, None]
        sc = (q.transpose(1, 2) @ k.transpose(1, 2).transpose(-1, -2).contiguous()) * d ** -0.5
        pr = torch.softmax(sc.masked_fill(~ok, -1e300), dim=-1) * ok
        ctx = (pr @ v.transpose(1, 2).contiguous()).transpose(1, 2).reshape(T, H)
        g, u = (ctx @ w_in + b_in).chunk(2, dim=1)
        y = (g * torch.sigmoid(g) * u) @ w_out + b_out
        grads = torch.autograd.grad((y * self.dy.double()).sum(), leaves)
        norm = torch.stack([t.square().sum() for t in grads]).sum().sqrt()
        factor = min(1.0, MAX_NORM / float(norm))
        return [y.detach(), torch.tensor([float(norm), factor], dtype=torch.float64, device="cuda"), *grads, *[t * factor for t in grads]]


@pytest.mark.parametrize("dtype", [B.DTYPE_F32, B.DTYPE_BF16])
def test_a_layer_and_its_gradients(dtype):
    layer = Layer(dtype)
    layer.step()
    for n, (got, want) in enumerate(zip(layer.outputs(), layer.want())):
        assert bool(got.isfinite().all()), n
        assert float((got.double() - want).norm()) <= TOL[dtype] * float(want.norm()), (n, float((got.double() - want).norm() / want.norm()))
    clipped = torch.cat([c.reshape(-1).double() for c in layer.clipped]).norm()
    assert float(clipped) <= MAX_NORM * (1 + 2.0 ** -20)
    # what padding holds does not matter
    want = [t.clone() for t in layer.outputs()]
    layer.x.view(b, s, H)[2, LENS[2]:] = 3.0
    layer.step()
    got = layer.outputs()
    rows = layer.seen
    assert torch.equal(got[0][rows], want[0][rows])
    assert all(torch.equal(x, y) for x, y in zip(got[2:9], want[2:9]))


@pytest.mark.parametrize("dtype", [B.DTYPE_F32, B.DTYPE_BF16])
def test_two_layers_on_two_streams_and_in_a_graph(dtype):
    one, two = Layer(dtype, 1), Layer(dtype, 2)
    want = []
    for layer in (one, two):
        layer.step()
        torch.cuda.synchronize()
        want.append([t.clone() for t in layer.outputs()])
        for t in layer.outputs():
            t.fill_(7)
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    for _ in range(3):
        for layer, st in zip((one, two), streams):
            with torch.cuda.stream(st):
                layer.step(st.cuda_stream)
    torch.cuda.synchronize()
    for layer, w in zip((one, two), want):
        assert all(torch.equal(x, y) for x, y in zip(layer.outputs(), w))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        one.step(torch.cuda.current_stream().cuda_stream)
        two.step(torch.cuda.current_stream().cuda_stream)
    for k in range(3):
        for layer in (one, two):
            layer.x.mul_(0.75)
            layer.step()
        torch.cuda.synchronize()
        eager = [[t.clone() for t in layer.outputs()] for layer in (one, two)]
        for layer in (one, two):
            for t in layer.outputs():
                t.fill_(7)
        graph.replay()
        torch.cuda.synchronize()
        for layer, w in zip((one, two), eager):
            assert all(torch.equal(x, y) for x, y in zip(layer.outputs(), w)), k
