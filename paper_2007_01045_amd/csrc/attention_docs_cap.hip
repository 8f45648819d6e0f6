// Attention of packed documents (attention_docs.hip), the gradient of capped logits
#include "attention_window.h"

namespace dapple {

hipError_t launch_attn_docs_bwd_cap(const AttnWinArgs& a, void* workspace, hipStream_t st) {
  return attn_win_bwd_launch_bf16<MASK_SPANS, SCORE_CAP>(a, workspace, st);
}

}  // namespace dapple
