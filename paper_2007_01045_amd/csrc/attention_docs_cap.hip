// Attention of packed documents (attention_docs.hip) with capped logits: forward, and the gradient without slopes
#include "attention_window.h"

namespace dapple {

hipError_t launch_attn_docs_fwd_cap(const AttnWinArgs& a, hipStream_t st) {
  return a.slopes ? attn_win_fwd_launch_bf16<MASK_SPANS, SCORE_BOTH>(a, st) : attn_win_fwd_launch_bf16<MASK_SPANS, SCORE_CAP>(a, st);
}

hipError_t launch_attn_docs_bwd_cap(const AttnWinArgs& a, void* workspace, hipStream_t st) {
  return attn_win_bwd_launch_bf16<MASK_SPANS, SCORE_CAP>(a, workspace, st);
}

}  // namespace dapple
