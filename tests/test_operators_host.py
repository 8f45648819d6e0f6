"""What the operators of dapple_kernels.h refuse, checked on the host: every call here returns before anything is enqueued
(the pointers are no memory)."""
import math

import pytest

from paper_2007_01045_amd import binding as B

P = 0x10000        # an aligned address that nothing looks at


def refused(code, f, *args, **kw):
    with pytest.raises(B.StageError) as e:
        f(*args, **kw)
    assert e.value.code == code, (e.value, args, kw)
    assert str(e.value).split(": ", 1)[1], "the refusal gives no reason"


def test_grad_norm_refusals():
    ok = dict(dtype=B.DTYPE_F32, grad_ptrs=[P, P], sizes=[3, 5], max_norm=1.0, norm_ptr=P, workspace_ptr=P, grad_scale=1.0)
    for code, change in [(B.STAGE_E_NULL, dict(norm_ptr=None)), (B.STAGE_E_NULL, dict(workspace_ptr=None)),
                         (B.STAGE_E_NULL, dict(grad_ptrs=None)), (B.STAGE_E_NULL, dict(grad_ptrs=[P, None])),
                         (B.STAGE_E_CONFIG, dict(dtype=2)), (B.STAGE_E_CONFIG, dict(sizes=[3, -1])),
                         (B.STAGE_E_CONFIG, dict(sizes=[3, 1 << 41])), (B.STAGE_E_CONFIG, dict(max_norm=0.0)),
                         (B.STAGE_E_CONFIG, dict(max_norm=-1.0)), (B.STAGE_E_CONFIG, dict(max_norm=math.nan)),
                         (B.STAGE_E_CONFIG, dict(grad_scale=math.inf)), (B.STAGE_E_CONFIG, dict(grad_scale=math.nan)),
                         (B.STAGE_E_CONFIG, dict(grad_ptrs=[P, P + 2])), (B.STAGE_E_CONFIG, dict(workspace_ptr=P + 4)),
                         (B.STAGE_E_CONFIG, dict(norm_ptr=P + 2))]:
        refused(code, B.dapple_grad_norm, **dict(ok, **change))
    refused(B.STAGE_E_CONFIG, B.dapple_grad_norm, **dict(ok, dtype=B.DTYPE_BF16, grad_ptrs=[P, P + 1]))
    refused(B.STAGE_E_CONFIG, B.dapple_grad_norm_workspace, [-1])
    assert B.dapple_grad_norm_workspace([]) > 0 and B.dapple_grad_norm_workspace([0, 0]) > 0
    assert B.dapple_grad_norm_workspace([1, 0, 1]) == 2 * B.dapple_grad_norm_workspace([1])


def test_grad_clip_refusals():
    ok = dict(dtype=B.DTYPE_F32, grad_ptrs=[P, P], out_ptrs=[P, P], sizes=[3, 5], norm_ptr=P)
    for code, change in [(B.STAGE_E_NULL, dict(norm_ptr=None)), (B.STAGE_E_NULL, dict(grad_ptrs=None)),
                         (B.STAGE_E_NULL, dict(out_ptrs=[P, None])), (B.STAGE_E_CONFIG, dict(dtype=-1)),
                         (B.STAGE_E_CONFIG, dict(sizes=[-3, 5])), (B.STAGE_E_CONFIG, dict(out_ptrs=[P, P + 1]))]:
        refused(code, B.dapple_grad_clip, **dict(ok, **change))


def test_clipped_adam_refusals():
    cfg = B.make_config(1, 64, 4, 128, 16, 2, 2, B.DTYPE_F32, flags=B.FLAG_DRY_RUN)
    h = B.stage_init(cfg, None, None, 0)
    try:
        B.stage_apply_adam_clipped(h, None, None, None, None, 1, 1e-3, None)      # (a dry run has no device memory)
        refused(B.STAGE_E_CONFIG, B.stage_apply_adam_clipped, h, P, P, P, P, 0, 1e-3, P)
        refused(B.STAGE_E_CONFIG, B.stage_apply_adam_clipped, h, P, P, P, P, 1, 1e-3, P, eps=0.0)
        B.stage_fwd(h, 0, None, None)
        refused(B.STAGE_E_BAD_ORDER, B.stage_apply_adam_clipped, h, P, P, P, P, 1, 1e-3, P)
    finally:
        B.stage_destroy(h)
    refused(B.STAGE_E_NULL, B.stage_apply_adam_clipped, None, P, P, P, P, 1, 1e-3, P)


def test_qk_rope_refusals():
    ok = dict(q=P, k=P, gamma_q=P, gamma_k=P, positions=P, table=P, yq=P, yk=P, dyq=P, dyk=P, dq=P, dk=P, dgamma_q=P, dgamma_k=P,
              workspace=P, rows=4, A=2, Ak=1, d=64, rot=32, interleaved=0, seq=0, max_pos=16, eps=1e-6)
    null, conf = B.STAGE_E_NULL, B.STAGE_E_CONFIG
    both = [(null, dict(q=None)), (null, dict(k=None)), (null, dict(table=None)), (conf, dict(rows=0)), (conf, dict(A=0)), (conf, dict(Ak=-1)),
            (conf, dict(d=0)), (conf, dict(d=257)), (conf, dict(rot=33)), (conf, dict(rot=66)), (conf, dict(rot=-2)), (conf, dict(max_pos=0)),
            (conf, dict(seq=-1)), (conf, dict(gamma_k=None)), (conf, dict(gamma_q=None)), (conf, dict(gamma_q=None, gamma_k=None, rot=0)),
            (conf, dict(eps=-1.0)), (conf, dict(eps=math.nan)), (conf, dict(ldq=127)), (conf, dict(ldk=-64)), (conf, dict(q=P + 1)),
            (conf, dict(table=P + 4)), (conf, dict(positions=P + 2)), (conf, dict(interleaved=1, ldq=129)),
            (conf, dict(interleaved=1, k=P + 2)), (conf, dict(interleaved=1, d=63, rot=32))]
    for dt in (B.DTYPE_BF16, 2):
        for code, change in both if dt == B.DTYPE_BF16 else [(conf, {})]:
            for f in (B.dapple_qk_rope_fwd, B.dapple_qk_rope_bwd):
                refused(code, f, dt, B.qk_rope_desc(**dict(ok, **change)))
    for change in (dict(yq=None), dict(yk=None)):
        refused(null, B.dapple_qk_rope_fwd, B.DTYPE_F32, B.qk_rope_desc(**dict(ok, **change)))
    for change in (dict(dyq=None), dict(dyk=None), dict(dq=None), dict(dk=None), dict(workspace=None)):
        refused(null, B.dapple_qk_rope_bwd, B.DTYPE_F32, B.qk_rope_desc(**dict(ok, **change)))
    refused(conf, B.dapple_qk_rope_bwd, B.DTYPE_F32, B.qk_rope_desc(**dict(ok, workspace=P + 8)))
    refused(conf, B.dapple_qk_rope_bwd, B.DTYPE_F32, B.qk_rope_desc(**dict(ok, dgamma_q=P + 2)))
    refused(conf, B.dapple_qk_rope_workspace, B.DTYPE_F32, B.qk_rope_desc(**dict(ok, rows=0)))
    assert B.dapple_qk_rope_workspace(B.DTYPE_F32, B.qk_rope_desc(**ok)) >= 2 * 64 * 4


def test_rope_table_refusals():
    refused(B.STAGE_E_NULL, B.dapple_rope_table, None, 4, 8)
    for args, kw in [((0, 8), {}), ((4, 0), {}), ((4, 7), {}), ((4, 258), {}), ((4, 8), dict(base=0.0)), ((4, 8), dict(base=math.nan)),
                     ((4, 8), dict(factor=0.0)), ((4, 8), dict(factor=math.inf)), ((4, 8), dict(original=-1)),
                     ((4, 8), dict(original=16, low=2.0, high=2.0)), ((4, 8), dict(magnitude=math.nan))]:
        refused(B.STAGE_E_CONFIG, B.dapple_rope_table, P, *args, **kw)
    refused(B.STAGE_E_CONFIG, B.dapple_rope_table, P + 4, 4, 8)


def test_attention_window_refusals():
    ok = dict(q=P, k=P, v=P, ctx=P, lse=P, dctx=P, dq=P, dk=P, dv=P, workspace=P, b=1, s=100, A=4, Ak=2, d=64, window=10, sinks=2, causal=1)
    null, conf = B.STAGE_E_NULL, B.STAGE_E_CONFIG
    both = [(null, dict(q=None)), (null, dict(k=None)), (null, dict(v=None)), (null, dict(ctx=None)), (null, dict(lse=None)), (conf, dict(b=0)),
            (conf, dict(s=0)), (conf, dict(A=0)), (conf, dict(Ak=0)), (conf, dict(Ak=3)), (conf, dict(d=0)), (conf, dict(d=60)), (conf, dict(d=136)),
            (conf, dict(window=-1)), (conf, dict(sinks=-1)), (conf, dict(scale=-1.0)), (conf, dict(scale=math.inf)), (conf, dict(scale=math.nan)),
            (conf, dict(ldq=255)), (conf, dict(ldq=260)), (conf, dict(ldk=-8)), (conf, dict(ldv=1 << 23)), (conf, dict(s=1 << 22, ldq=264)),
            (conf, dict(q=P + 8)), (conf, dict(ctx32=P + 4)), (conf, dict(lse=P + 2)), (conf, dict(lens=P + 1)),
            (conf, dict(b=1 << 20, s=1 << 12)), (conf, dict(b=1 << 16, A=1 << 15, Ak=1 << 15, s=1))]
    for code, change in both:
        for f in (B.dapple_attention_window_fwd, B.dapple_attention_window_bwd):
            refused(code, f, B.DTYPE_BF16, B.attention_window_desc(**dict(ok, **change)))
    for change in (dict(dctx=None), dict(dq=None), dict(dk=None), dict(dv=None), dict(workspace=None)):
        refused(null, B.dapple_attention_window_bwd, B.DTYPE_F32, B.attention_window_desc(**dict(ok, **change)))
    for change in (dict(dctx=P + 8), dict(dv=P + 4), dict(lddq=258), dict(workspace=P + 8)):
        refused(conf, B.dapple_attention_window_bwd, B.DTYPE_F32, B.attention_window_desc(**dict(ok, **change)))
    refused(conf, B.dapple_attention_window_fwd, 2, B.attention_window_desc(**ok))
    refused(conf, B.dapple_attention_window_fwd, B.DTYPE_F32, B.attention_window_desc(**dict(ok, d=66)))
    refused(conf, B.dapple_attention_window_workspace, B.DTYPE_BF16, B.attention_window_desc(**dict(ok, d=4)))
    for dt in (B.DTYPE_F32, B.DTYPE_BF16):
        assert B.dapple_attention_window_workspace(dt, B.attention_window_desc(**ok)) >= 4 * 4 * 100


def test_gated_ffn_refusals():
    ok = dict(x=P, w_in=P, b_in=P, w_out=P, b_out=P, gu=P, h=P, y=P, dy=P, dgu=P, dx=P, dw_in=P, db_in=P, dw_out=P, db_out=P, workspace=P,
              T=10, H=64, F=128)
    null, conf = B.STAGE_E_NULL, B.STAGE_E_CONFIG
    both = [(null, dict(x=None)), (null, dict(w_in=None)), (null, dict(w_out=None)), (null, dict(h=None)), (conf, dict(T=0)), (conf, dict(H=0)),
            (conf, dict(F=0)), (conf, dict(H=68)), (conf, dict(F=132)), (conf, dict(act=2)), (conf, dict(ldx=56)), (conf, dict(ldy=68)),
            (conf, dict(lddx=-64)), (conf, dict(T=1 << 22)), (conf, dict(H=1 << 16, F=1 << 14)), (conf, dict(T=1 << 20, ldx=1 << 10)),
            (conf, dict(w_out=P + 8)), (conf, dict(h=P + 8)), (conf, dict(gu=P + 4))]
    for code, change in both:
        for f in (B.dapple_gated_ffn_fwd, B.dapple_gated_ffn_bwd):
            refused(code, f, B.DTYPE_BF16, B.gated_ffn_desc(**dict(ok, **change)))
    refused(null, B.dapple_gated_ffn_fwd, B.DTYPE_F32, B.gated_ffn_desc(**dict(ok, y=None)))
    refused(conf, B.dapple_gated_ffn_fwd, B.DTYPE_F32, B.gated_ffn_desc(**dict(ok, H=66)))
    refused(conf, B.dapple_gated_ffn_fwd, B.DTYPE_F32, B.gated_ffn_desc(**dict(ok, x=P + 8)))
    refused(conf, B.dapple_gated_ffn_fwd, 3, B.gated_ffn_desc(**ok))
    for change in (dict(dy=None), dict(gu=None), dict(dgu=None), dict(workspace=None)):
        refused(null, B.dapple_gated_ffn_bwd, B.DTYPE_F32, B.gated_ffn_desc(**dict(ok, **change)))
    for change in (dict(dw_in=None), dict(dw_out=None), dict(dw_in=None, dw_out=None), dict(workspace=P + 4), dict(db_in=P + 4), dict(dy=P + 4),
                   dict(dgu=P + 8), dict(dw_in=P + 8), dict(dx=P + 8)):
        refused(conf, B.dapple_gated_ffn_bwd, B.DTYPE_F32, B.gated_ffn_desc(**dict(ok, **change)))
    refused(conf, B.dapple_gated_ffn_workspace, B.DTYPE_BF16, B.gated_ffn_desc(**dict(ok, F=12)))
    for dt in (B.DTYPE_F32, B.DTYPE_BF16):
        assert B.dapple_gated_ffn_workspace(dt, B.gated_ffn_desc(**ok)) > 0


def test_sizes_beyond_a_launch():
    # 2^32 work-items; workspaces and tensors of these sizes are conceivable, so they are refused before anything is enqueued
    rope = dict(q=P, k=P, gamma_q=P, gamma_k=P, table=P, yq=P, yk=P, dyq=P, dyk=P, dq=P, dk=P, workspace=P, rows=1 << 26, A=1, Ak=1, d=8, rot=8,
                max_pos=16)
    for f in (B.dapple_qk_rope_fwd, B.dapple_qk_rope_bwd, B.dapple_qk_rope_workspace):
        refused(B.STAGE_E_CONFIG, f, B.DTYPE_BF16, B.qk_rope_desc(**rope))
    refused(B.STAGE_E_CONFIG, B.dapple_rope_table, P, 1 << 24, 256)
    attn = dict(q=P, k=P, v=P, ctx=P, lse=P, dctx=P, dq=P, dk=P, dv=P, workspace=P, d=8)
    for sizes in (dict(b=1 << 16, s=1 << 10, A=1, Ak=1), dict(b=1 << 16, s=1, A=2, Ak=1), dict(b=1 << 8, s=1 << 15, A=32, Ak=1),
                  dict(b=1, s=1 << 27, A=1, Ak=1), dict(b=0x7fffffff, s=0x7fffffff, A=0x7fffffff, Ak=1)):
        for f in (B.dapple_attention_window_fwd, B.dapple_attention_window_bwd, B.dapple_attention_window_workspace):
            refused(B.STAGE_E_CONFIG, f, B.DTYPE_BF16, B.attention_window_desc(**attn, **sizes))


def test_attention_workspace_is_bounded():
    # fp32 sums of parts of walks: their number must not grow with sinks times rows
    for dt, wide in ((B.DTYPE_BF16, 128), (B.DTYPE_F32, 128), (B.DTYPE_BF16, 64), (B.DTYPE_F32, 32)):
        for b, s, A, Ak in ((1, 32768, 32, 8), (4, 8192, 16, 16), (1, 65536, 1, 1), (1, (1 << 24) - 64, 1, 1), (3, 5000, 48, 2), (64, 300, 16, 1)):
            for window in (1, 64, 1000, 0):
                for sinks in (0, 1, 17, 1000, s // 8, s // 2, s - 1, s):
                    for causal in (0, 1):
                        desc = B.attention_window_desc(b=b, s=s, A=A, Ak=Ak, d=wide, window=window, sinks=sinks, causal=causal)
                        size = B.dapple_attention_window_workspace(dt, desc)
                        assert 4 * b * A * s <= size < 4 * b * A * s + (1 << 28), (dt, wide, b, s, A, Ak, window, sinks, causal, size)


def test_the_last_sizes_of_a_launch():
    # one step further than what a launch of 2^32 - 1 work-items holds is refused, the step before is not (the workspaces say so)
    rope = dict(A=1, Ak=1, d=8)
    assert B.dapple_qk_rope_workspace(B.DTYPE_F32, B.qk_rope_desc(rows=(1 << 26) - 4, **rope)) > 0
    refused(B.STAGE_E_CONFIG, B.dapple_qk_rope_workspace, B.DTYPE_F32, B.qk_rope_desc(rows=(1 << 26) - 3, **rope))
    size = lambda dt, **kw: B.dapple_attention_window_workspace(dt, B.attention_window_desc(d=8, **kw))  # noqa: E731
    ok = dict(q=P, k=P, v=P, ctx=P, lse=P, dctx=P, dq=P, dk=P, dv=P, workspace=P, d=8)
    for dt in (B.DTYPE_F32, B.DTYPE_BF16):
        assert size(dt, b=4, s=(1 << 24) - 1, A=1, Ak=1) > 0
        for kw in (dict(b=1, s=(1 << 26) - 3, A=1, Ak=1),                  # rows
                   dict(b=65535, s=1, A=128, Ak=1), dict(b=65535, s=32, A=127, Ak=1),   # query and key heads: 512 work-items to one's rows
                   dict(b=1, s=1 << 22, A=63, Ak=1, d=64, ldq=4096)):
            kw = dict(ok, **kw)
            for f in (B.dapple_attention_window_bwd, B.dapple_attention_window_workspace):
                refused(B.STAGE_E_CONFIG, f, dt, B.attention_window_desc(**kw))
        assert size(dt, b=65535, s=32, A=126, Ak=1) > 0
    most = (1 << 38) - (1 << 22)
    for sizes in ([most], [1 << 31] * 127 + [(1 << 31) - (1 << 22)]):
        assert B.dapple_grad_norm_workspace(sizes) > 0
        refused(B.STAGE_E_CONFIG, B.dapple_grad_norm_workspace, sizes + [1])


def test_gated_ffn_rows_of_2_to_the_24():
    ok = dict(x=P, w_in=P, w_out=P, h=P, y=P, gu=P, dy=P, dgu=P, workspace=P, T=1, H=8, F=8)
    for change in (dict(F=1 << 23), dict(ldx=1 << 24), dict(H=1 << 24)):
        desc = B.gated_ffn_desc(**dict(ok, **change))
        for f in (B.dapple_gated_ffn_fwd, B.dapple_gated_ffn_bwd, B.dapple_gated_ffn_workspace):
            with pytest.raises(B.StageError) as e:
                f(B.DTYPE_BF16, desc)
            assert e.value.code == B.STAGE_E_CONFIG and "2^24" in str(e.value)
        assert B.dapple_gated_ffn_workspace(B.DTYPE_F32, desc) > 0
    for change in (dict(F=(1 << 23) - 8), dict(ldx=(1 << 24) - 8, lddy=(1 << 24) - 8), dict(ldy=1 << 24)):
        assert B.dapple_gated_ffn_workspace(B.DTYPE_BF16, B.gated_ffn_desc(**dict(ok, **change))) > 0
    refused(B.STAGE_E_CONFIG, B.dapple_gated_ffn_bwd, B.DTYPE_BF16, B.gated_ffn_desc(**dict(ok, lddy=1 << 24)))


def test_philox_reference():
    # the vectors that the generator's authors publish for ten rounds of four words
    from tests.dropout_util import philox
    full = 0xffffffff
    for ctr, key, want in (([0] * 4, [0] * 2, [0x6627e8d5, 0xe169c58d, 0xbc57ac4c, 0x9b00dbd8]),
                           ([full] * 4, [full] * 2, [0x408f276d, 0x41c83b0e, 0xa20bc7c6, 0x6d5451fd]),
                           ([0x243f6a88, 0x85a308d3, 0x13198a2e, 0x03707344], [0xa4093822, 0x299f31d0], [0xd16cfe09, 0x94fdcceb, 0x5001e420, 0x24126ea1])):
        assert [int(x) for x in philox(ctr, key)] == want


def test_dropout_norm_refusals():
    ok = dict(x=P, bias=P, residual=P, gamma=P, beta=P, rng=P, z=P, y=P, stats=P, dy=P, dz=P, dx=P, dresidual=P, dbias=P, dgamma=P, dbeta=P, workspace=P,
              rows=10, H=64, norm=B.NORM_LAYER, p=0.1, eps=1e-5)
    null, conf = B.STAGE_E_NULL, B.STAGE_E_CONFIG
    both = [(null, dict(rng=None)), (conf, dict(rows=0)), (conf, dict(H=0)), (conf, dict(H=16385)), (conf, dict(norm=3)), (conf, dict(norm=-1)), (conf, dict(p=-0.1)),
            (conf, dict(p=1.1)), (conf, dict(p=math.nan)), (conf, dict(eps=-1.0)), (conf, dict(eps=math.nan)), (conf, dict(ldx=63)), (conf, dict(lddr=-1)),
            (conf, dict(rows=(1 << 26) + 1)), (conf, dict(rows=1 << 26, H=512)), (conf, dict(rng=P + 4)), (conf, dict(stats=P + 2)), (conf, dict(z=P + 1)),
            (conf, dict(stream32=1, z=P + 2)), (conf, dict(gamma=P + 1)), (conf, dict(norm=B.NORM_NONE)), (conf, dict(norm=B.NORM_NONE, beta=None, gamma=P)),
            (conf, dict(norm=B.NORM_RMS))]
    for code, change in both:
        for f in (B.dapple_dropout_norm_fwd, B.dapple_dropout_norm_bwd):
            refused(code, f, B.DTYPE_BF16, B.dropout_norm_desc(**dict(ok, **change)))
    none = dict(norm=B.NORM_NONE, gamma=None, beta=None, dgamma=None, dbeta=None)
    for change in (dict(x=None), dict(y=None), dict(none, z=None)):
        refused(null, B.dapple_dropout_norm_fwd, B.DTYPE_F32, B.dropout_norm_desc(**dict(ok, **change)))
    for change in (dict(dy=None), dict(z=None), dict(stats=None), dict(workspace=None), dict(none, dz=None),
                   dict(dx=None, dresidual=None, dbias=None, dgamma=None, dbeta=None)):
        refused(null, B.dapple_dropout_norm_bwd, B.DTYPE_F32, B.dropout_norm_desc(**dict(ok, **change)))
    for change in (dict(workspace=P + 8), dict(dx=P + 2), dict(dbias=P + 2), dict(dz=P + 2), dict(norm=B.NORM_RMS, beta=None)):
        refused(conf, B.dapple_dropout_norm_bwd, B.DTYPE_F32, B.dropout_norm_desc(**dict(ok, **change)))
    refused(conf, B.dapple_dropout_norm_fwd, 2, B.dropout_norm_desc(**ok))
    size = lambda rows, H: B.dapple_dropout_norm_workspace(B.DTYPE_BF16, B.dropout_norm_desc(rows=rows, H=H))  # noqa: E731
    assert size(1, 1) >= 12 and size(1 << 26, 504) > 0 and size((1 << 21) - 1, 16384) > 0
    for sizes in ((1 << 26, 512), (1 << 21, 16384), (0, 8), (8, 16385)):
        refused(conf, size, *sizes)


def test_embedding_refusals():
    ok = dict(table=P, ids=P, y=P, dy=P, dtable=P, workspace=P, rows=10, V=100, H=64, scale=1.0)
    null, conf = B.STAGE_E_NULL, B.STAGE_E_CONFIG
    both = [(null, dict(ids=None)), (conf, dict(rows=0)), (conf, dict(V=0)), (conf, dict(H=0)), (conf, dict(rows=(1 << 28) + 1)), (conf, dict(V=(1 << 28) + 1)),
            (conf, dict(H=(1 << 16) + 1)), (conf, dict(scale=math.inf)), (conf, dict(scale=math.nan)), (conf, dict(ldt=63)), (conf, dict(lddt=-64)), (conf, dict(ids=P + 2))]
    for code, change in both:
        for f in (B.dapple_embedding_fwd, B.dapple_embedding_bwd):
            refused(code, f, B.DTYPE_BF16, B.embedding_desc(**dict(ok, **change)))
    for change in (dict(table=None), dict(y=None)):
        refused(null, B.dapple_embedding_fwd, B.DTYPE_F32, B.embedding_desc(**dict(ok, **change)))
    for change in (dict(dy=None), dict(dtable=None), dict(workspace=None)):
        refused(null, B.dapple_embedding_bwd, B.DTYPE_F32, B.embedding_desc(**dict(ok, **change)))
    for change in (dict(workspace=P + 8), dict(dy=P + 1), dict(accumulate=1, dtable=P + 2)):
        refused(conf, B.dapple_embedding_bwd, B.DTYPE_BF16, B.embedding_desc(**dict(ok, **change)))
    refused(conf, B.dapple_embedding_fwd, B.DTYPE_BF16, B.embedding_desc(**dict(ok, y=P + 1)))
    refused(conf, B.dapple_embedding_fwd, -1, B.embedding_desc(**ok))
    size = lambda rows, V, H: B.dapple_embedding_workspace(B.DTYPE_BF16, B.embedding_desc(rows=rows, V=V, H=H))  # noqa: E731
    for rows, V, H in ((1, 1, 1), (65536, 30522, 1024), (1 << 28, 1 << 28, 1 << 16)):
        assert 16 * rows <= size(rows, V, H) <= 16 * rows + (1 << 16) * H + (1 << 19)
    refused(conf, size, 0, 1, 1)


def test_attention_docs_refusals():
    ok = dict(q=P, k=P, v=P, ctx=P, lse=P, spans=P, slopes=P, dctx=P, dq=P, dk=P, dv=P, workspace=P, rows=100, A=4, Ak=2, d=64)
    null, conf = B.STAGE_E_NULL, B.STAGE_E_CONFIG
    both = [(null, dict(q=None)), (null, dict(k=None)), (null, dict(v=None)), (null, dict(ctx=None)), (null, dict(lse=None)), (null, dict(spans=None)),
            (conf, dict(rows=0)), (conf, dict(A=0)), (conf, dict(Ak=3)), (conf, dict(d=60)), (conf, dict(d=136)), (conf, dict(scale=-1.0)),
            (conf, dict(scale=math.nan)), (conf, dict(cap=-1.0)), (conf, dict(cap=1e-7)), (conf, dict(cap=1025.0)), (conf, dict(cap=math.inf)),
            (conf, dict(cap=math.nan)), (conf, dict(ldq=255)), (conf, dict(ldk=-8)), (conf, dict(ldv=1 << 23)), (conf, dict(rows=1 << 22, ldq=264)),
            (conf, dict(q=P + 8)), (conf, dict(ctx32=P + 4)), (conf, dict(lse=P + 2)), (conf, dict(spans=P + 2)), (conf, dict(slopes=P + 1)),
            (conf, dict(rows=(1 << 26) - 7)), (conf, dict(scale=1e38, cap=2.0 ** -20)), (conf, dict(scale=1e-38, cap=1024.0))]
    for code, change in both:
        for f in (B.dapple_attention_docs_fwd, B.dapple_attention_docs_bwd):
            refused(code, f, B.DTYPE_BF16, B.attention_docs_desc(**dict(ok, **change)))
    for change in (dict(dctx=None), dict(dq=None), dict(dk=None), dict(dv=None), dict(workspace=None)):
        refused(null, B.dapple_attention_docs_bwd, B.DTYPE_F32, B.attention_docs_desc(**dict(ok, **change)))
    for change in (dict(dctx=P + 8), dict(dv=P + 4), dict(lddq=258), dict(workspace=P + 8)):
        refused(conf, B.dapple_attention_docs_bwd, B.DTYPE_F32, B.attention_docs_desc(**dict(ok, **change)))
    refused(conf, B.dapple_attention_docs_fwd, 2, B.attention_docs_desc(**ok))
    refused(conf, B.dapple_attention_docs_workspace, B.DTYPE_BF16, B.attention_docs_desc(**dict(ok, d=4)))
    for dt in (B.DTYPE_F32, B.DTYPE_BF16):
        for rows, A, Ak, d in ((100, 4, 2, 64), (1, 1, 1, 8), (65536, 32, 8, 128), (8192, 16, 4, 128), (1 << 22, 1, 1, 64), (3000, 64, 1, 32)):
            assert 4 * A * rows <= B.dapple_attention_docs_workspace(dt, B.attention_docs_desc(rows=rows, A=A, Ak=Ak, d=d)) < 4 * A * rows + (1 << 28)


def test_doc_spans_refusals():
    null, conf = B.STAGE_E_NULL, B.STAGE_E_CONFIG
    ok = dict(ends_ptr=P, n=3, rows=10, spans_ptr=P)
    for code, change in ((null, dict(ends_ptr=None)), (null, dict(spans_ptr=None)), (conf, dict(n=-1)), (conf, dict(rows=0)), (conf, dict(rows=(1 << 26) - 7)),
                         (conf, dict(window=-1)), (conf, dict(causal=0, prefix_ptr=P)), (conf, dict(ends_ptr=P + 2)), (conf, dict(prefix_ptr=P + 1)),
                         (conf, dict(spans_ptr=P + 2))):
        refused(code, B.dapple_doc_spans, **dict(ok, **change))
