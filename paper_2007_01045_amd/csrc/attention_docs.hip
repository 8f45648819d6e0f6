// Attention of packed documents: the kernels of attention_window.h with runs of visible rows from arrays, and logits that are capped,
//   t = cap tanh(scale q k / cap),  dt / d(scale q k) = 1 - (t / cap)^2,
// and lowered by slope |i - j|.  A row sees the rows of its own document: backwards (causal), also what lies in the document's prefix, or
// all of it, |i - j| < W if there is a window.  That is one run of rows, [key_lo, key_hi), whose ends never fall from row to row, and so
// are the rows that see a row, [query_lo, query_hi): doc_spans writes the four down once for all layers and heads of a step, and
// the kernels walk and skip by them as they do by a window.
#include "attention_window.h"

namespace dapple {

// ------------------------------------------------------------------ spans
// spans[0 .. 3][rows]: key_lo, key_hi, query_lo, query_hi; behind them the number of rows that documents hold.  Document t holds the rows
// from ends[t - 1] (0) to ends[t].  Rows behind the last see nothing.
constexpr int NEAR_ENDS = 2048;   // as many are searched in LDS
__global__ __launch_bounds__(256) void doc_spans_kernel(const int32_t* __restrict__ ends, const int32_t* __restrict__ prefix, int n, int rows, int causal, int window,
                                                        int32_t* __restrict__ spans) {
  __shared__ int32_t near[NEAR_ENDS];
  const int i = blockIdx.x * 256 + threadIdx.x;
  const int len = n > 0 ? min(max(ends[n - 1], 0), rows) : 0;
  if (n <= NEAR_ENDS) {
    for (int t = threadIdx.x; t < n; t += 256) near[t] = ends[t];
    __syncthreads();
  }
  if (i == 0) spans[4L * rows] = len;
  if (i >= rows) return;
  int v[4] = {len, len, len, len};
  if (i < len) {
    auto end_of = [&](int t) { return n <= NEAR_ENDS ? near[t] : ends[t]; };
    int lo = 0, hi = n - 1;   // the first document that ends behind row i
    while (lo < hi) {
      const int mid = lo + ((hi - lo) >> 1);   // (the sum of two may be beyond an int)
      if (end_of(mid) > i) hi = mid;
      else lo = mid + 1;
    }
    // (ends that are not ascending: some document, within the rows)
    const int begin = lo ? min(max(end_of(lo - 1), 0), i) : 0, end = min(max(end_of(lo), i + 1), len);
    const int free = causal && prefix ? min(max(prefix[lo], 0), end - begin) + begin : begin;   // first row behind the prefix
    v[0] = begin;
    v[1] = causal ? max(i + 1, free) : end;
    v[2] = causal && i >= free ? i : begin;
    v[3] = end;
    if (window) {   // (below rows)
      v[0] = max(v[0], i - window + 1);
      v[1] = min(v[1], i + window);
      v[2] = max(v[2], i - window + 1);
      v[3] = min(v[3], i + window);
    }
  }
#pragma unroll
  for (int k = 0; k < 4; ++k) spans[(long)k * rows + i] = v[k];
}

hipError_t launch_doc_spans(const int32_t* ends, const int32_t* prefix, int n, int rows, int causal, int window, int32_t* spans, hipStream_t st) {
  hipLaunchKernelGGL(doc_spans_kernel, dim3((rows + 255) / 256), dim3(256), 0, st, ends, prefix, n, rows, causal, window, spans);
  return hipGetLastError();
}

// ------------------------------------------------------------------ launchers
int64_t attn_docs_workspace(Dtype dt, AttnWinArgs a) {
  make_docs_plan(dt, a);
  const int width = pick_width(dt, a.d, [](auto D) { return (int)decltype(D)::value; });
  return (int64_t)(delta_bytes(a) + table_bytes(a)) + (int64_t)a.Ak * a.plan.slots * 2 * a.plan.kt * width * 4;
}

hipError_t launch_attn_docs_fwd(Dtype dt, const AttnWinArgs& a, hipStream_t st) {
  if (dt != DT_BF16) return launch_attn_docs_fwd_f32(a, st);
  if (a.cap2 > 0.f) return launch_attn_docs_fwd_cap(a, st);
  return a.slopes ? attn_win_fwd_launch_bf16<MASK_SPANS, SCORE_SLOPE>(a, st) : attn_win_fwd_launch_bf16<MASK_SPANS, SCORE_PLAIN>(a, st);
}

hipError_t launch_attn_docs_bwd(Dtype dt, const AttnWinArgs& a, void* workspace, hipStream_t st) {
  if (dt != DT_BF16) return launch_attn_docs_bwd_f32(a, workspace, st);
  if (a.cap2 > 0.f) return a.slopes ? launch_attn_docs_bwd_both(a, workspace, st) : launch_attn_docs_bwd_cap(a, workspace, st);
  return a.slopes ? attn_win_bwd_launch_bf16<MASK_SPANS, SCORE_SLOPE>(a, workspace, st) : attn_win_bwd_launch_bf16<MASK_SPANS, SCORE_PLAIN>(a, workspace, st);
}

}  // namespace dapple
