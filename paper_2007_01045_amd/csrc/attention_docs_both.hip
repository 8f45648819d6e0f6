// Attention of packed documents (attention_docs.hip), the gradient of logits that are capped and lowered
#include "attention_window.h"

namespace dapple {

hipError_t launch_attn_docs_bwd_both(const AttnWinArgs& a, void* workspace, hipStream_t st) {
  return attn_win_bwd_launch_bf16<MASK_SPANS, SCORE_BOTH>(a, workspace, st);
}

}  // namespace dapple
