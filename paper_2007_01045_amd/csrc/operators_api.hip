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
