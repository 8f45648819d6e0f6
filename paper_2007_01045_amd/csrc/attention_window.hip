// Attention with a window and first tokens that stay visible: the kernels of attention_window.h with their own mask and plain logits.
#include "attention_window.h"

namespace dapple {

static bool al16(const void* p) { return ((uintptr_t)p & 15) == 0; }

bool attn_win_takes(Dtype dt, const AttnWinArgs& a) {
  const int v = dt == DT_BF16 ? 8 : 4;
  if (a.d % v || a.d > 128) return false;
  for (int ld : {a.ldq, a.ldk, a.ldv, a.ldc, a.lddc, a.lddq, a.lddk, a.lddv})
    // (a sequence's bytes are counted in 32 bits, and so are those of a block of 64 rows)
    if (ld % v || ld >= (1 << 23) || (long)a.s * ld >= (1L << 30) - 4096) return false;
  for (const void* p : {a.q, a.k, a.v, (const void*)a.ctx, (const void*)a.ctx32, a.dctx, (const void*)a.dq, (const void*)a.dk, (const void*)a.dv})
    if (!al16(p)) return false;
  return true;
}

int64_t attn_win_workspace(Dtype dt, AttnWinArgs a) {
  make_plan(dt, a);
  const int kt = key_tile(dt, a);
  const int width = pick_width(dt, a.d, [](auto D) { return (int)decltype(D)::value; });
  return (int64_t)delta_bytes(a) + (int64_t)a.b * a.Ak * a.plan.slots * 2 * kt * width * 4;
}

hipError_t launch_attn_win_fwd(Dtype dt, const AttnWinArgs& a, hipStream_t st) {
  return dt == DT_BF16 ? attn_win_fwd_launch_bf16<MASK_WINDOW, SCORE_PLAIN>(a, st) : attn_win_fwd_launch_f32<MASK_WINDOW, SCORE_PLAIN>(a, st);
}

hipError_t launch_attn_win_bwd(Dtype dt, const AttnWinArgs& a, void* workspace, hipStream_t st) {
  return dt == DT_BF16 ? attn_win_bwd_launch_bf16<MASK_WINDOW, SCORE_PLAIN>(a, workspace, st) : attn_win_bwd_launch_f32<MASK_WINDOW, SCORE_PLAIN>(a, workspace, st);
}

}  // namespace dapple
