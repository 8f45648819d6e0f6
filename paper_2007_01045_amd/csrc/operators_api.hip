// C ABI of the operators in the second part of dapple_kernels.h: argument checks on the host, and forwarding to the
// launchers.
#include <hip/hip_runtime.h>

#include <cmath>

#include "../../include/dapple_kernels.h"
#include "../../include/dapple_stage.h"
#include "kernels.h"

using namespace dapple;

static bool bad_dtype(int dt) { return dt != STAGE_DTYPE_F32 && dt != STAGE_DTYPE_BF16; }
static Dtype type_of(int dt) { return dt == STAGE_DTYPE_BF16 ? DT_BF16 : DT_F32; }
static bool aligned_to(const void* p, size_t a) { return (uintptr_t)p % a == 0; }
static int rc_of(hipError_t e) {
  return e == hipSuccess ? STAGE_OK : set_error(STAGE_E_DEVICE, "a launch failed: %s", hipGetErrorString(e));
}

// ------------------------------------------------------------------ attention of visible pairs
// the launcher's arguments; sizes_only: what the size of the workspace depends on
static int win_args(int dtype, const dapple_attention_window_desc* d, bool bwd, bool sizes_only, AttnWinArgs& a) {
  if (!d) return set_error(STAGE_E_NULL, "the descriptor is NULL");
  if (bad_dtype(dtype)) return set_error(STAGE_E_CONFIG, "dtype %d", dtype);
  if (d->b < 1 || d->s < 1 || d->A < 1 || d->Ak < 1 || d->A % d->Ak || d->d < 1)
    return set_error(STAGE_E_CONFIG, "%d sequences of %d rows, %d query heads on %d key heads of %d columns", d->b, d->s, d->A, d->Ak, d->d);
  if (d->window < 0 || d->sinks < 0) return set_error(STAGE_E_CONFIG, "window %d, sinks %d", d->window, d->sinks);
  if (!(d->scale >= 0.f) || !std::isfinite(d->scale)) return set_error(STAGE_E_CONFIG, "scale must be positive and finite (0: 1/sqrt(d))");
  const int v = dtype == STAGE_DTYPE_BF16 ? 8 : 4;
  if (d->d % v || d->d > 128) return set_error(STAGE_E_CONFIG, "heads of %d columns: multiples of %d up to 128 are taken", d->d, v);
  // (A launch has fewer than 2^32 work-items: 512 to 32 rows of a head, 64 to a row.  The gradient's holds key heads beside query heads,
  // and up to 2048 parts of walks: see make_plan.)
  const long row_blocks = (long)d->b * ((d->s + 31L) / 32);
  if (d->s >= 1 << 27 || (long)d->b * d->s > (1L << 26) - 4 || (long)d->b * d->A >= 1L << 23 || row_blocks * d->A >= 1L << 23 || (long)d->b * d->Ak >= 1L << 16)
    return set_error(STAGE_E_CONFIG, "2^26 - 3 rows, 2^16 key heads of all sequences or 2^23 times 32 rows of a head and more");
  if (bwd && row_blocks * ((long)d->A + d->Ak) >= (1L << 23) - 2048)
    return set_error(STAGE_E_CONFIG, "2^23 - 2048 times 32 rows of a head, key heads included, and more");
  a.b = d->b; a.s = d->s; a.A = d->A; a.Ak = d->Ak; a.d = d->d; a.causal = d->causal != 0;
  a.W = d->window < d->s ? d->window : 0;   // (a window of s positions and more hides nothing)
  a.S = d->sinks < d->s ? d->sinks : d->s;
  a.scale = d->scale > 0.f ? d->scale : 1.0f / sqrtf((float)d->d);
  const struct { int given; int heads; int* to; } lds[] = {{d->ldq, d->A, &a.ldq}, {d->ldk, d->Ak, &a.ldk}, {d->ldv, d->Ak, &a.ldv},
      {d->ldc, d->A, &a.ldc}, {d->lddc, d->A, &a.lddc}, {d->lddq, d->A, &a.lddq}, {d->lddk, d->Ak, &a.lddk}, {d->lddv, d->Ak, &a.lddv}};
  for (const auto& l : lds) {
    const long dense = (long)l.heads * d->d;
    if (dense >= 1 << 23 || l.given < 0 || (l.given && l.given < dense))
      return set_error(STAGE_E_CONFIG, "a row stride of %d for %ld columns", l.given, dense);
    *l.to = l.given ? l.given : (int)dense;
  }
  if (sizes_only) return STAGE_OK;
  if (!d->q || !d->k || !d->v || !d->ctx || !d->lse) return set_error(STAGE_E_NULL, "q, k, v, ctx and lse must not be NULL");
  if (bwd && (!d->dctx || !d->dq || !d->dk || !d->dv || !d->workspace))
    return set_error(STAGE_E_NULL, "dctx, dq, dk, dv and workspace must not be NULL");
  a.q = d->q; a.k = d->k; a.v = d->v; a.ctx = d->ctx; a.ctx32 = d->ctx32; a.lse = d->lse; a.lens = d->lens;
  if (bwd) { a.dctx = d->dctx; a.dq = d->dq; a.dk = d->dk; a.dv = d->dv; }
  if (!aligned_to(a.lse, 4) || !aligned_to(a.lens, 4) || (bwd && !aligned_to(d->workspace, 16)))
    return set_error(STAGE_E_CONFIG, "lse, lens or workspace not aligned");
  if (!attn_win_takes(type_of(dtype), a))
    return set_error(STAGE_E_CONFIG, "tensors must be 16-byte aligned, row strides multiples of %d below 2^23, a sequence below 2^30 elements", v);
  return STAGE_OK;
}

extern "C" {

int dapple_attention_window_fwd(int dtype, const dapple_attention_window_desc* d, void* stream) {
  AttnWinArgs a{};
  const int rc = win_args(dtype, d, false, false, a);
  return rc != STAGE_OK ? rc : rc_of(launch_attn_win_fwd(type_of(dtype), a, (hipStream_t)stream));
}

int64_t dapple_attention_window_workspace(int dtype, const dapple_attention_window_desc* d) {
  AttnWinArgs a{};
  const int rc = win_args(dtype, d, true, true, a);
  return rc != STAGE_OK ? rc : attn_win_workspace(type_of(dtype), a);
}

int dapple_attention_window_bwd(int dtype, const dapple_attention_window_desc* d, void* stream) {
  AttnWinArgs a{};
  const int rc = win_args(dtype, d, true, false, a);
  return rc != STAGE_OK ? rc : rc_of(launch_attn_win_bwd(type_of(dtype), a, d->workspace, (hipStream_t)stream));
}

}  // extern "C"

// ------------------------------------------------------------------ attention of packed documents
static int docs_args(int dtype, const dapple_attention_docs_desc* d, bool bwd, bool sizes_only, AttnWinArgs& a) {
  if (!d) return set_error(STAGE_E_NULL, "the descriptor is NULL");
  // (one sequence; a workgroup of the gradient's first launch beside four rows each is the plan's)
  if (d->rows > (1 << 26) - 8) return set_error(STAGE_E_CONFIG, "2^26 - 7 rows and more");
  dapple_attention_window_desc w{};
  w.q = d->q; w.k = d->k; w.v = d->v; w.ctx = d->ctx; w.ctx32 = d->ctx32; w.lse = d->lse; w.dctx = d->dctx; w.dq = d->dq; w.dk = d->dk; w.dv = d->dv;
  w.workspace = d->workspace; w.b = 1; w.s = d->rows; w.A = d->A; w.Ak = d->Ak; w.d = d->d;
  w.ldq = d->ldq; w.ldk = d->ldk; w.ldv = d->ldv; w.ldc = d->ldc; w.lddc = d->lddc; w.lddq = d->lddq; w.lddk = d->lddk; w.lddv = d->lddv;
  w.scale = d->scale;
  const int rc = win_args(dtype, &w, bwd, sizes_only, a);
  if (rc != STAGE_OK || sizes_only) return rc;
  if (!(d->cap == 0.f || (d->cap >= 0x1p-20f && d->cap <= 0x1p10f))) return set_error(STAGE_E_CONFIG, "cap must be 0 or lie in [2^-20, 2^10]");
  if (!d->spans) return set_error(STAGE_E_NULL, "spans must not be NULL");
  if (!aligned_to(d->spans, 4) || !aligned_to(d->slopes, 4)) return set_error(STAGE_E_CONFIG, "spans or slopes not aligned");
  a.spans = d->spans; a.slopes = d->slopes;
  if (d->cap > 0.f) {
    a.cap2 = (float)(d->cap * 1.4426950408889634);
    a.bend = a.scale / d->cap;
    if (!std::isnormal(a.bend) || !std::isnormal(1.f / a.bend)) return set_error(STAGE_E_CONFIG, "scale %g over cap %g", a.scale, d->cap);
  }
  return STAGE_OK;
}

extern "C" {

int dapple_doc_spans(const int32_t* ends, const int32_t* prefix, int n, int rows, int causal, int window, int32_t* spans, void* stream) {
  if (!spans || (n > 0 && !ends)) return set_error(STAGE_E_NULL, "spans, and ends of a document, must not be NULL");
  if (n < 0 || rows < 1 || rows > (1 << 26) - 8) return set_error(STAGE_E_CONFIG, "%d documents, %d rows (1 to 2^26 - 8)", n, rows);
  if (window < 0) return set_error(STAGE_E_CONFIG, "window %d", window);
  if (prefix && !causal) return set_error(STAGE_E_CONFIG, "a prefix without causal");
  if (!aligned_to(ends, 4) || !aligned_to(prefix, 4) || !aligned_to(spans, 4)) return set_error(STAGE_E_CONFIG, "ends, prefix or spans not aligned");
  return rc_of(launch_doc_spans(ends, prefix, n, rows, causal != 0, window < rows ? window : 0, spans, (hipStream_t)stream));
}

int dapple_attention_docs_fwd(int dtype, const dapple_attention_docs_desc* d, void* stream) {
  AttnWinArgs a{};
  const int rc = docs_args(dtype, d, false, false, a);
  return rc != STAGE_OK ? rc : rc_of(launch_attn_docs_fwd(type_of(dtype), a, (hipStream_t)stream));
}

int64_t dapple_attention_docs_workspace(int dtype, const dapple_attention_docs_desc* d) {
  AttnWinArgs a{};
  const int rc = docs_args(dtype, d, true, true, a);
  return rc != STAGE_OK ? rc : attn_docs_workspace(type_of(dtype), a);
}

int dapple_attention_docs_bwd(int dtype, const dapple_attention_docs_desc* d, void* stream) {
  AttnWinArgs a{};
  const int rc = docs_args(dtype, d, true, false, a);
  return rc != STAGE_OK ? rc : rc_of(launch_attn_docs_bwd(type_of(dtype), a, d->workspace, (hipStream_t)stream));
}

}  // extern "C"

// ------------------------------------------------------------------ head norms and rotation
// the launcher's arguments; workspace_only: what the size of the workspace depends on
static int rope_args(int dtype, const dapple_qk_rope_desc* d, bool bwd, bool workspace_only, QkRopeArgs& a) {
  if (!d) return set_error(STAGE_E_NULL, "the descriptor is NULL");
  if (bad_dtype(dtype)) return set_error(STAGE_E_CONFIG, "dtype %d", dtype);
  if (d->rows < 1 || d->A < 1 || d->Ak < 0 || d->d < 1 || d->d > 256)
    return set_error(STAGE_E_CONFIG, "rows %d, heads %d and %d of %d columns (at most 256)", d->rows, d->A, d->Ak, d->d);
  if (d->rows > (1 << 26) - 4) return set_error(STAGE_E_CONFIG, "2^26 - 3 rows and more");   // (a launch has fewer than 2^32 work-items)
  if (workspace_only) return STAGE_OK;
  if (d->rot < 0 || d->rot % 2 || d->rot > d->d) return set_error(STAGE_E_CONFIG, "%d of %d columns to turn", d->rot, d->d);
  if (d->seq < 0 || (d->rot && d->max_pos < 1)) return set_error(STAGE_E_CONFIG, "seq %d, max_pos %d", d->seq, d->max_pos);
  const bool keys = d->Ak > 0, norm = d->gamma_q != nullptr;
  if (keys && norm != (d->gamma_k != nullptr)) return set_error(STAGE_E_CONFIG, "one gamma without the other");
  if (!norm && !d->rot) return set_error(STAGE_E_CONFIG, "neither a norm nor a rotation");
  if (norm && !(d->eps >= 0.f)) return set_error(STAGE_E_CONFIG, "eps must not be negative");
  if (d->rot && !d->table) return set_error(STAGE_E_NULL, "table is NULL");
  if (((!bwd || norm) && (!d->q || (keys && !d->k))) || (!bwd && (!d->yq || (keys && !d->yk))) ||
      (bwd && (!d->dyq || !d->dq || (keys && (!d->dyk || !d->dk)))))
    return set_error(STAGE_E_NULL, "a tensor is NULL");
  a.q = d->q; a.gamma_q = d->gamma_q; a.yq = d->yq; a.dyq = d->dyq; a.dq = d->dq; a.dgamma_q = norm ? d->dgamma_q : nullptr;
  if (keys) {
    a.k = d->k; a.gamma_k = d->gamma_k; a.yk = d->yk; a.dyk = d->dyk; a.dk = d->dk; a.dgamma_k = norm ? d->dgamma_k : nullptr;
  }
  a.positions = d->positions; a.table = d->table;
  a.rows = d->rows; a.A = d->A; a.Ak = d->Ak; a.d = d->d; a.rot = d->rot; a.interleaved = d->interleaved != 0; a.seq = d->seq;
  a.max_pos = d->max_pos; a.accumulate = d->accumulate != 0; a.eps = d->eps;
  const struct { int given; int heads; int* to; } lds[] = {{d->ldq, d->A, &a.ldq}, {d->ldk, d->Ak, &a.ldk},
      {d->ldyq, d->A, &a.ldyq}, {d->ldyk, d->Ak, &a.ldyk}, {d->lddyq, d->A, &a.lddyq}, {d->lddyk, d->Ak, &a.lddyk},
      {d->lddq, d->A, &a.lddq}, {d->lddk, d->Ak, &a.lddk}};
  for (const auto& l : lds) {
    const long dense = (long)l.heads * d->d;
    if (dense > 0x7fffffffL || l.given < 0 || (l.given && l.given < dense))
      return set_error(STAGE_E_CONFIG, "a row stride of %d for %ld columns", l.given, dense);
    *l.to = l.given ? l.given : (int)dense;
  }
  const size_t es = dtype == STAGE_DTYPE_BF16 ? 2 : 4;
  const void* ps[] = {a.q, a.k, a.gamma_q, a.gamma_k, bwd ? a.dyq : a.yq, bwd ? a.dyk : a.yk, bwd ? a.dq : nullptr, bwd ? a.dk : nullptr};
  for (const void* p : ps)
    if (!aligned_to(p, es)) return set_error(STAGE_E_CONFIG, "a tensor is not aligned to its elements");
  if (!aligned_to(a.table, 8) || !aligned_to(a.positions, 4) || !aligned_to(a.dgamma_q, 4) || !aligned_to(a.dgamma_k, 4))
    return set_error(STAGE_E_CONFIG, "table, positions or dgamma not aligned");
  if (!qk_rope_takes(type_of(dtype), a, bwd))
    return set_error(STAGE_E_CONFIG, "interleaved pairs need an even d, even strides and addresses aligned to two elements");
  return STAGE_OK;
}

extern "C" {

int dapple_qk_rope_fwd(int dtype, const dapple_qk_rope_desc* d, void* stream) {
  QkRopeArgs a{};
  const int rc = rope_args(dtype, d, false, false, a);
  return rc != STAGE_OK ? rc : rc_of(launch_qk_rope_fwd(type_of(dtype), a, (hipStream_t)stream));
}

int64_t dapple_qk_rope_workspace(int dtype, const dapple_qk_rope_desc* d) {
  QkRopeArgs a{};
  const int rc = rope_args(dtype, d, true, true, a);
  return rc != STAGE_OK ? rc : (int64_t)qk_rope_blocks(d->rows) * 2 * d->d * 4;
}

int dapple_qk_rope_bwd(int dtype, const dapple_qk_rope_desc* d, void* stream) {
  QkRopeArgs a{};
  const int rc = rope_args(dtype, d, true, false, a);
  if (rc != STAGE_OK) return rc;
  if (a.dgamma_q || a.dgamma_k) {
    if (!d->workspace) return set_error(STAGE_E_NULL, "workspace is NULL");
    if (!aligned_to(d->workspace, 16)) return set_error(STAGE_E_CONFIG, "workspace not aligned to 16 bytes");
  }
  return rc_of(launch_qk_rope_bwd(type_of(dtype), a, (float*)d->workspace, (hipStream_t)stream));
}

int dapple_rope_table(float* table, int max_pos, int rot, double base, double factor, int original, double low, double high,
                      double magnitude, void* stream) {
  if (!table) return set_error(STAGE_E_NULL, "table is NULL");
  if (max_pos < 1 || rot < 2 || rot % 2 || rot > 256 || (long)max_pos * rot > 0x7fffffffL) return set_error(STAGE_E_CONFIG, "max_pos %d, rot %d", max_pos, rot);
  if (!(base > 0) || !std::isfinite(base) || !(factor > 0) || !std::isfinite(factor) || !std::isfinite(magnitude) || original < 0 ||
      (original > 0 && !(low < high && std::isfinite(low) && std::isfinite(high))))
    return set_error(STAGE_E_CONFIG, "base and factor must be positive and finite, low below high");
  if (!aligned_to(table, 8)) return set_error(STAGE_E_CONFIG, "table not aligned to 8 bytes");
  double f[128];
  for (int i = 0; i < rot / 2; ++i) {
    const double w = std::pow(base, -2.0 * i / rot);
    double g = 0.0;
    if (original > 0) g = std::fmin(1.0, std::fmax(0.0, (original * w / (2.0 * M_PI) - low) / (high - low)));
    f[i] = w * (g + (1.0 - g) / factor);
  }
  return rc_of(launch_rope_table(table, max_pos, rot / 2, f, magnitude, (hipStream_t)stream));
}

}  // extern "C"

// ------------------------------------------------------------------ gated feed-forward block
static int ffn_args(int dtype, const dapple_gated_ffn_desc* d, bool bwd, bool sizes_only, GatedFfnArgs& a) {
  if (!d) return set_error(STAGE_E_NULL, "the descriptor is NULL");
  if (bad_dtype(dtype)) return set_error(STAGE_E_CONFIG, "dtype %d", dtype);
  const int v = dtype == STAGE_DTYPE_BF16 ? 8 : 4;
  const long most = (1L << 30) - 4096;
  if (d->T < 1 || d->H < 1 || d->F < 1 || d->H % v || d->F % v)
    return set_error(STAGE_E_CONFIG, "%d rows, %d and %d columns: the columns must be multiples of %d", d->T, d->H, d->F, v);
  if (2L * d->T * d->F >= most || 2L * d->H * d->F >= most) return set_error(STAGE_E_CONFIG, "T * 2F or H * 2F of 2^30 - 4096 and more");
  if (d->act != DAPPLE_ACT_SILU && d->act != DAPPLE_ACT_GELU) return set_error(STAGE_E_CONFIG, "activation %d", d->act);
  a.T = d->T; a.H = d->H; a.F = d->F; a.silu = d->act == DAPPLE_ACT_SILU; a.accumulate = d->accumulate != 0;
  const struct { int given; int* to; } lds[] = {{d->ldx, &a.ldx}, {d->ldy, &a.ldy}, {d->lddy, &a.lddy}, {d->lddx, &a.lddx}};
  for (const auto& l : lds) {
    *l.to = l.given ? l.given : d->H;
    if (*l.to < d->H || *l.to % v || (long)d->T * *l.to >= most) return set_error(STAGE_E_CONFIG, "a row stride of %d", l.given);
  }
  // (64 rows of an operand are counted in 31 bits of bytes: see gemm_uses_mfma)
  if (dtype == STAGE_DTYPE_BF16 && (2L * d->F >= 1 << 24 || a.ldx >= 1 << 24 || (bwd && a.lddy >= 1 << 24)))
    return set_error(STAGE_E_CONFIG, "2F or a stride of x or dy of 2^24 and more");
  if (sizes_only) return STAGE_OK;
  if (!d->x || !d->w_in || !d->w_out || !d->h) return set_error(STAGE_E_NULL, "x, w_in, w_out and h must not be NULL");
  if (!bwd && !d->y) return set_error(STAGE_E_NULL, "y must not be NULL");
  if (bwd && (!d->dy || !d->gu || !d->dgu || !d->workspace)) return set_error(STAGE_E_NULL, "dy, gu, dgu and workspace must not be NULL");
  if (bwd && (!d->dw_in != !d->dw_out || (!d->dw_in && (d->db_in || d->db_out))))
    return set_error(STAGE_E_CONFIG, "dw_in and dw_out are wanted both or not at all, biases' gradients with them");
  a.x = d->x; a.w_in = d->w_in; a.b_in = d->b_in; a.w_out = d->w_out; a.b_out = d->b_out; a.gu = d->gu; a.h = d->h; a.y = d->y;
  if (bwd) {
    a.dy = d->dy; a.dgu = d->dgu; a.dx = d->dx; a.dw_in = d->dw_in; a.db_in = d->db_in; a.dw_out = d->dw_out; a.db_out = d->db_out;
    if (!aligned_to(d->workspace, 16) || !aligned_to(a.db_in, 16) || !aligned_to(a.db_out, 16))
      return set_error(STAGE_E_CONFIG, "workspace, db_in or db_out not aligned to 16 bytes");
  }
  if (!gated_ffn_takes(type_of(dtype), a, bwd)) return set_error(STAGE_E_CONFIG, "a tensor is not aligned to 16 bytes");
  return STAGE_OK;
}

extern "C" {

int dapple_gated_ffn_fwd(int dtype, const dapple_gated_ffn_desc* d, void* stream) {
  GatedFfnArgs a{};
  const int rc = ffn_args(dtype, d, false, false, a);
  return rc != STAGE_OK ? rc : rc_of(launch_gated_ffn_fwd(type_of(dtype), a, (hipStream_t)stream));
}

int64_t dapple_gated_ffn_workspace(int dtype, const dapple_gated_ffn_desc* d) {
  GatedFfnArgs a{};
  const int rc = ffn_args(dtype, d, true, true, a);
  return rc != STAGE_OK ? rc : gated_ffn_workspace(type_of(dtype), a);
}

int dapple_gated_ffn_bwd(int dtype, const dapple_gated_ffn_desc* d, void* stream) {
  GatedFfnArgs a{};
  const int rc = ffn_args(dtype, d, true, false, a);
  return rc != STAGE_OK ? rc : rc_of(launch_gated_ffn_bwd(type_of(dtype), a, d->workspace, (hipStream_t)stream));
}

}  // extern "C"

// ------------------------------------------------------------------ dropout, residual sum and norm
static int norm_args(int dtype, const dapple_dropout_norm_desc* d, bool bwd, bool sizes_only, DropNormArgs& a) {
  if (!d) return set_error(STAGE_E_NULL, "the descriptor is NULL");
  if (bad_dtype(dtype)) return set_error(STAGE_E_CONFIG, "dtype %d", dtype);
  if (d->rows < 1 || d->H < 1 || d->H > 16384) return set_error(STAGE_E_CONFIG, "%d rows of %d columns (at most 16384)", d->rows, d->H);
  // (a group of eight elements is counted in 32 bits; so are a launch's work-items)
  if (d->rows > 1 << 26 || (long)d->rows * ((d->H + 7) / 8) >= 1L << 32) return set_error(STAGE_E_CONFIG, "2^26 rows or 2^32 groups of eight columns and more");
  if (sizes_only) return STAGE_OK;
  if (d->norm != DAPPLE_NORM_NONE && d->norm != DAPPLE_NORM_LAYER && d->norm != DAPPLE_NORM_RMS) return set_error(STAGE_E_CONFIG, "norm %d", d->norm);
  if (!(d->p >= 0.f && d->p <= 1.f)) return set_error(STAGE_E_CONFIG, "p must lie in [0, 1]");
  const bool norm = d->norm != DAPPLE_NORM_NONE;
  if (norm && !(d->eps >= 0.f)) return set_error(STAGE_E_CONFIG, "eps must not be negative");
  if (!norm && (d->gamma || d->beta || (bwd && (d->dgamma || d->dbeta)))) return set_error(STAGE_E_CONFIG, "gamma or beta without a norm");
  if (d->norm == DAPPLE_NORM_RMS && (d->beta || (bwd && d->dbeta))) return set_error(STAGE_E_CONFIG, "an RMS norm has no beta");
  a.rows = d->rows; a.H = d->H; a.norm = d->norm; a.stream32 = d->stream32 != 0; a.accumulate = d->accumulate != 0;
  a.site = (uint32_t)d->site; a.level = (uint32_t)std::nearbyint(65536.0 * d->p); a.eps = d->eps;
  a.up = a.level < 65536 ? (float)(65536.0 / (65536.0 - a.level)) : 0.f;
  if (a.level && !d->rng) return set_error(STAGE_E_NULL, "rng must not be NULL");
  a.rng = a.level ? d->rng : nullptr;
  const struct { int given; int* to; } lds[] = {{d->ldx, &a.ldx}, {d->ldr, &a.ldr}, {d->ldz, &a.ldz}, {d->ldy, &a.ldy},
      {d->lddy, &a.lddy}, {d->lddz, &a.lddz}, {d->lddx, &a.lddx}, {d->lddr, &a.lddr}};
  for (const auto& l : lds) {
    if (l.given && l.given < d->H) return set_error(STAGE_E_CONFIG, "a row stride of %d for %d columns", l.given, d->H);
    *l.to = l.given ? l.given : d->H;
  }
  if (!bwd && (!d->x || (norm ? !d->y : !d->z))) return set_error(STAGE_E_NULL, "x, and y (without a norm: z), must not be NULL");
  if (bwd && (norm ? !d->dy || !d->z || !d->stats : !d->dz)) return set_error(STAGE_E_NULL, "dy, z and stats (without a norm: dz) must not be NULL");
  if (bwd && !d->dx && !d->dresidual && !d->dbias && !d->dgamma && !d->dbeta) return set_error(STAGE_E_NULL, "no gradient is wanted");
  const size_t es = dtype == STAGE_DTYPE_BF16 ? 2 : 4, zs = a.stream32 ? 4 : es;
  a.gamma = d->gamma;
  a.z = d->z; a.stats = d->stats;
  if (!bwd) {
    a.x = d->x; a.bias = d->bias; a.residual = d->residual; a.beta = d->beta; a.y = norm ? d->y : nullptr;
  } else {
    a.dy = norm ? d->dy : nullptr; a.dz = d->dz; a.dx = d->dx; a.dr = d->dresidual; a.dbias = d->dbias; a.dgamma = d->dgamma; a.dbeta = d->dbeta;
    if (a.dbias || a.dgamma || a.dbeta) {
      if (!d->workspace) return set_error(STAGE_E_NULL, "workspace is NULL");
      if (!aligned_to(d->workspace, 16)) return set_error(STAGE_E_CONFIG, "workspace not aligned to 16 bytes");
      a.partial = (float*)d->workspace;
    }
  }
  for (const void* p : {a.x, a.bias, a.gamma, a.beta, (const void*)a.y, a.dy, (const void*)a.dx})
    if (!aligned_to(p, es)) return set_error(STAGE_E_CONFIG, "a tensor is not aligned to its elements");
  for (const void* p : {a.residual, (const void*)a.z, a.dz, (const void*)a.dr})
    if (!aligned_to(p, zs)) return set_error(STAGE_E_CONFIG, "a tensor of the stream is not aligned to its elements");
  for (const void* p : {a.stats, a.dbias, a.dgamma, a.dbeta})
    if (!aligned_to(p, 4)) return set_error(STAGE_E_CONFIG, "stats or a sum is not aligned to its elements");
  if (!aligned_to(a.rng, 8)) return set_error(STAGE_E_CONFIG, "rng not aligned to 8 bytes");
  return STAGE_OK;
}

extern "C" {

int dapple_dropout_norm_fwd(int dtype, const dapple_dropout_norm_desc* d, void* stream) {
  DropNormArgs a{};
  const int rc = norm_args(dtype, d, false, false, a);
  return rc != STAGE_OK ? rc : rc_of(launch_dropout_norm_fwd(type_of(dtype), a, (hipStream_t)stream));
}

int64_t dapple_dropout_norm_workspace(int dtype, const dapple_dropout_norm_desc* d) {
  DropNormArgs a{};
  const int rc = norm_args(dtype, d, true, true, a);
  return rc != STAGE_OK ? rc : (int64_t)dropout_norm_blocks(d->rows, d->H) * 3 * d->H * 4;
}

int dapple_dropout_norm_bwd(int dtype, const dapple_dropout_norm_desc* d, void* stream) {
  DropNormArgs a{};
  const int rc = norm_args(dtype, d, true, false, a);
  return rc != STAGE_OK ? rc : rc_of(launch_dropout_norm_bwd(type_of(dtype), a, (hipStream_t)stream));
}

}  // extern "C"

// ------------------------------------------------------------------ embedding
static int embedding_args(int dtype, const dapple_embedding_desc* d, bool bwd, bool sizes_only, EmbeddingArgs& a) {
  if (!d) return set_error(STAGE_E_NULL, "the descriptor is NULL");
  if (bad_dtype(dtype)) return set_error(STAGE_E_CONFIG, "dtype %d", dtype);
  if (d->rows < 1 || d->V < 1 || d->H < 1 || d->rows > 1 << 28 || d->V > 1 << 28 || d->H > 1 << 16)
    return set_error(STAGE_E_CONFIG, "%d rows (at most 2^28) of a table of %d (at most 2^28) by %d (at most 2^16)", d->rows, d->V, d->H);
  a.rows = d->rows; a.V = d->V; a.H = d->H;
  if (sizes_only) return STAGE_OK;
  if (!std::isfinite(d->scale)) return set_error(STAGE_E_CONFIG, "scale must be finite");
  a.accumulate = d->accumulate != 0; a.scale = d->scale;
  const struct { int given; int* to; } lds[] = {{d->ldt, &a.ldt}, {d->ldy, &a.ldy}, {d->lddy, &a.lddy}, {d->lddt, &a.lddt}};
  for (const auto& l : lds) {
    if (l.given && l.given < d->H) return set_error(STAGE_E_CONFIG, "a row stride of %d for %d columns", l.given, d->H);
    *l.to = l.given ? l.given : d->H;
  }
  if (!d->ids || (bwd ? !d->dy || !d->dtable || !d->workspace : !d->table || !d->y))
    return set_error(STAGE_E_NULL, bwd ? "ids, dy, dtable and workspace must not be NULL" : "table, ids and y must not be NULL");
  const size_t es = dtype == STAGE_DTYPE_BF16 ? 2 : 4;
  a.ids = d->ids;
  if (bwd) { a.dy = d->dy; a.dtable = d->dtable; } else { a.table = d->table; a.y = d->y; }
  if (!aligned_to(a.table, es) || !aligned_to(a.y, es) || !aligned_to(a.dy, es) || !aligned_to(a.dtable, a.accumulate ? 4 : es) || !aligned_to(a.ids, 4))
    return set_error(STAGE_E_CONFIG, "a tensor is not aligned to its elements");
  if (bwd && !aligned_to(d->workspace, 16)) return set_error(STAGE_E_CONFIG, "workspace not aligned to 16 bytes");
  return STAGE_OK;
}

extern "C" {

int dapple_embedding_fwd(int dtype, const dapple_embedding_desc* d, void* stream) {
  EmbeddingArgs a{};
  const int rc = embedding_args(dtype, d, false, false, a);
  return rc != STAGE_OK ? rc : rc_of(launch_embedding_fwd(type_of(dtype), a, (hipStream_t)stream));
}

int64_t dapple_embedding_workspace(int dtype, const dapple_embedding_desc* d) {
  EmbeddingArgs a{};
  const int rc = embedding_args(dtype, d, true, true, a);
  return rc != STAGE_OK ? rc : embedding_workspace(a);
}

int dapple_embedding_bwd(int dtype, const dapple_embedding_desc* d, void* stream) {
  EmbeddingArgs a{};
  const int rc = embedding_args(dtype, d, true, false, a);
  return rc != STAGE_OK ? rc : rc_of(launch_embedding_bwd(type_of(dtype), a, d->workspace, (hipStream_t)stream));
}

}  // extern "C"

// ------------------------------------------------------------------ gradient norm
static int check_sizes(const int64_t* sizes, int n) {
  if (n < 0) return set_error(STAGE_E_CONFIG, "%d tensors", n);
  if (n > 0 && !sizes) return set_error(STAGE_E_NULL, "sizes must not be NULL");
  int64_t total = 0;
  for (int i = 0; i < n; ++i) {
    if (sizes[i] < 0) return set_error(STAGE_E_CONFIG, "tensor %d has %lld elements", i, (long long)sizes[i]);
    // (a launch of up to 128 tensors has fewer than 2^24 workgroups of 256: see grad_norm.hip)
    constexpr int64_t most = (1LL << 38) - (1LL << 22);
    if (sizes[i] > most || (total += sizes[i]) > most) return set_error(STAGE_E_CONFIG, "more than 2^38 - 2^22 elements");
  }
  return STAGE_OK;
}

static int check_tensors(int dtype, const void* const* t, const int64_t* sizes, int n, const char* what) {
  if (n > 0 && !t) return set_error(STAGE_E_NULL, "%s must not be NULL", what);
  const size_t es = dtype == STAGE_DTYPE_BF16 ? 2 : 4;
  for (int i = 0; i < n; ++i) {
    if (sizes[i] == 0) continue;
    if (!t[i]) return set_error(STAGE_E_NULL, "%s[%d] is NULL", what, i);
    if (!aligned_to(t[i], es)) return set_error(STAGE_E_CONFIG, "%s[%d] is not aligned to its elements", what, i);
  }
  return STAGE_OK;
}

extern "C" {

int64_t dapple_grad_norm_workspace(const int64_t* sizes, int n) {
  const int rc = check_sizes(sizes, n);
  if (rc != STAGE_OK) return rc;
  const int64_t b = grad_norm_blocks(sizes, n);
  return 8 * (b > 0 ? b : 1);
}

int dapple_grad_norm(int dtype, const void* const* grads, const int64_t* sizes, int n, float grad_scale, float max_norm,
                     float* norm_dev, void* workspace, void* stream) {
  if (!norm_dev || !workspace) return set_error(STAGE_E_NULL, "norm_dev and workspace must not be NULL");
  if (bad_dtype(dtype)) return set_error(STAGE_E_CONFIG, "dtype %d", dtype);
  int rc = check_sizes(sizes, n);
  if (rc == STAGE_OK) rc = check_tensors(dtype, grads, sizes, n, "grads");
  if (rc != STAGE_OK) return rc;
  if (!(max_norm > 0.f)) return set_error(STAGE_E_CONFIG, "max_norm must be positive");
  if (!std::isfinite(grad_scale)) return set_error(STAGE_E_CONFIG, "grad_scale must be finite");
  if (!aligned_to(workspace, 8) || !aligned_to(norm_dev, 4)) return set_error(STAGE_E_CONFIG, "workspace or norm_dev not aligned");
  return rc_of(launch_grad_norm(type_of(dtype), grads, sizes, n, grad_scale, max_norm, norm_dev, (double*)workspace, (hipStream_t)stream));
}

int dapple_grad_clip(int dtype, const void* const* grads, void* const* outs, const int64_t* sizes, int n, const float* norm_dev,
                     void* stream) {
  if (!norm_dev) return set_error(STAGE_E_NULL, "norm_dev must not be NULL");
  if (bad_dtype(dtype)) return set_error(STAGE_E_CONFIG, "dtype %d", dtype);
  if (!aligned_to(norm_dev, 4)) return set_error(STAGE_E_CONFIG, "norm_dev not aligned");
  void* const* const to = outs ? outs : (void* const*)grads;
  int rc = check_sizes(sizes, n);
  if (rc == STAGE_OK) rc = check_tensors(dtype, grads, sizes, n, "grads");
  if (rc == STAGE_OK) rc = check_tensors(dtype, to, sizes, n, "outs");
  if (rc != STAGE_OK) return rc;
  return rc_of(launch_grad_clip(type_of(dtype), grads, to, sizes, n, norm_dev, (hipStream_t)stream));
}

}  // extern "C"
