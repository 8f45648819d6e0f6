// Attention of packed documents (attention_docs.hip), fp32: one kernel for plain logits, one that looks at cap and slopes when it runs
#include "attention_window.h"

namespace dapple {

static bool plain(const AttnWinArgs& a) { return !(a.cap2 > 0.f) && !a.slopes; }

hipError_t launch_attn_docs_fwd_f32(const AttnWinArgs& a, hipStream_t st) {
  return plain(a) ? attn_win_fwd_launch_f32<MASK_SPANS, SCORE_PLAIN>(a, st) : attn_win_fwd_launch_f32<MASK_SPANS, SCORE_BOTH>(a, st);
}

hipError_t launch_attn_docs_bwd_f32(const AttnWinArgs& a, void* workspace, hipStream_t st) {
  return plain(a) ? attn_win_bwd_launch_f32<MASK_SPANS, SCORE_PLAIN>(a, workspace, st) : attn_win_bwd_launch_f32<MASK_SPANS, SCORE_BOTH>(a, workspace, st);
}

}  // namespace dapple
