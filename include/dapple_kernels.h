/*
 * dapple_kernels.h -- kernel-level entry points of the stage library.
 *
 * The forward and backward tasks of a stage (dapple_stage.h) are sequences of the
 * kernels in the first part.  They are exported so that each can be checked against the CPU
 * oracle on its own and timed on its own; they add no functionality.  The second part
 * holds operators of layers and training steps that a stage does not build itself.  All
 * pointers are DEVICE pointers owned by the caller, `stream` is a hipStream_t
 * (NULL = default stream), work is enqueued and not waited for, the return value
 * is 0 or a negative STAGE_E_* code (see dapple_stage.h).
 * dtype: 0 = fp32, 1 = bf16 storage with fp32 accumulation.
 */
#ifndef DAPPLE_KERNELS_H
#define DAPPLE_KERNELS_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

enum {
  DAPPLE_EPI_BIAS = 1,  /* t = acc + bias[n] */
  DAPPLE_EPI_ADD = 2,   /* t += aux[m,n]  (residual branch) */
  DAPPLE_EPI_MUL = 4,   /* t *= aux[m,n]  (GELU' gate in the FFN backward) */
  DAPPLE_EPI_GELU = 8,  /* C = GELU(t), C2 = GELU'(t) */
  DAPPLE_EPI_ACC32 = 16, /* C is fp32 and C += t  (weight-gradient accumulation over
                            micro-batches, section V-B-3 of the DAPPLE paper) */
  DAPPLE_EPI_OUT32 = 32, /* C is fp32 and C = t */
  DAPPLE_EPI_AUX32 = 64, /* aux is fp32 although the product is bf16 (the unrounded residual stream) */
  DAPPLE_EPI_BSUM = 128, /* bsum[n] += sum_k B(n,k): the bias gradient (column sums of the output gradient)
                            in the launch of the weight gradient; both operands k-strided, batch 1 */
  DAPPLE_EPI_ROWDOT = 256 /* rowdot[j*M + m] = sum over the columns n in [32j, 32j+32) of C[m,n] (as stored,
                            rounded to bf16) * aux[m,n]; aux is neither added nor multiplied in.  The stage
                            backward B_s uses it on the product that makes the attention output's gradient:
                            the row sums rowsum(dctx o ctx) per head that the softmax backward needs are then
                            two of these blocks.  bf16 MFMA path only (anything else: STAGE_E_CONFIG), no other
                            epilogue than BIAS and AUX32 beside it, batch 1 */
};

/* C[m,n] = epilogue(sum_k A(m,k) B(n,k)).  A k-contiguous operand is X(r,k) =
 * X[r*ld + k]; a k-strided one is X(r,k) = X[k*ld + r].  K may be cut in segments
 * of kseg_len (0 = one segment): segment i reads A + i*segA, B + i*segB.  batch
 * (0 = 1) instances at element strides sA, sB, sC, sBias.  k_valid (0 = K): rows k
 * >= k_valid of a k-strided operand read as zero.  The linear layers of an
 * encoder layer, their data gradients and their weight gradients are all
 * instances of this product. */
typedef struct {
  const void* A;
  const void* B;
  void* C;
  void* C2;
  const void* bias;
  const void* aux;
  float* bsum;    /* DAPPLE_EPI_BSUM: fp32 [N], accumulated into */
  float* rowdot;  /* DAPPLE_EPI_ROWDOT: fp32 [ceil(N/32)][M], overwritten */
  int32_t M, N, K;
  int32_t lda, ldb, ldc, ldaux;
  int32_t a_kstrided, b_kstrided;
  int32_t kseg_len;
  int64_t segA, segB;
  int32_t batch;
  int64_t sA, sB, sC, sBias;
  int32_t k_valid;
  int32_t epi;
  int32_t tile;   /* 0 = automatic; else one configuration of the MFMA kernel, for tests and timing:
                   * 1: 256x256 tile, four-stage ring of 32-wide k-tiles; 2: 256x128, three stages of 64;
                   * 3: 128x128, two stages of 64; 4: 128x64, three stages of 64; 5: 128x128, four stages of 32
                   * (both operands k-strided; any other layout gets 3); 6: 128x128, five stages of 64; 7: 64x64,
                   * four stages of 64; 8: 128x128 in four waves, four stages of 32 (A k-contiguous; else 5 or 3);
                   * 9: 32x64 and 10: 32x32, four stages of 64 (A k-contiguous; else 7); 12: 128x64 in four stages
                   * (A k-contiguous; else 7); any other number is 7.  K segments that are no multiple of 64
                   * have 3 and 4 where an operand is k-contiguous (any other number: chosen between them) */
} dapple_gemm_desc;

/* Returns 1 if the bf16 MFMA kernel takes this problem, 0 if the plain kernel does. */
int dapple_gemm(int dtype, const dapple_gemm_desc* d, void* stream);
/* What dapple_gemm would launch (host only; nothing is enqueued).  Returns as dapple_gemm does; with 1, plan_out[0..3] are
 * the rows and columns of a workgroup's tile, the depth of a k-tile, and the k-tiles each workgroup runs (a ring is filled
 * in whole turns: k-tiles of zeros are among them). */
int dapple_gemm_plan(int dtype, const dapple_gemm_desc* d, int32_t* plan_out);
/* What a stage would launch for this product: on a stream that may use `units` compute units (0 = all), with another
 * stream's products beside it if `shared` is not 0 (a data gradient beside the weight gradients).  plan_out[0..3] as
 * above, [4] the waves of a workgroup, [5] the stages of its ring. */
int dapple_gemm_plan_beside(int dtype, const dapple_gemm_desc* d, int units, int shared, int32_t* plan_out);

/* Attention of one layer.  q,k,v,ctx,dctx,dq,dk,dv: [b*s, H], head h in columns
 * [h*d, (h+1)*d), d = H / A.  lse [b,A,s] fp32: log2-domain logsumexp of the scaled
 * logits (written by fwd, read by bwd).  delta [b,A,s] fp32: scratch of bwd.
 * fwd: ctx = softmax(q k^T / sqrt(d)) v.  bwd: dq, dk, dv from dctx. */
int dapple_attention_fwd(int dtype, const void* q, const void* k, const void* v, void* ctx, float* lse,
                         int b, int s, int A, int H, void* stream);
int dapple_attention_bwd(int dtype, const void* q, const void* k, const void* v, const void* ctx,
                         const float* lse, const void* dctx, void* dq, void* dk, void* dv, float* delta,
                         int b, int s, int A, int H, void* stream);

/* y = LN(z) over the last dimension H (biased variance, eps inside the root);
 * stats[2r] = mean, stats[2r+1] = 1/sqrt(var+eps). */
int dapple_layernorm_fwd(int dtype, const void* z, const void* gamma, const void* beta, void* y,
                         float* stats, int rows, int H, float eps, void* stream);
/* dz from dy; dgamma += sum_r dy*xhat, dbeta += sum_r dy, dbias += sum_r dz (each
 * fp32 [H], NULL to skip).  partial: fp32 scratch of ceil(rows/8)*3*H elements. */
int dapple_layernorm_bwd(int dtype, const void* dy, const void* z, const float* stats, const void* gamma,
                         void* dz, float* partial, float* dgamma, float* dbeta, float* dbias, int rows,
                         int H, void* stream);
/* out[c] += sum_r X[r*ld + c]; partial: fp32 scratch of ceil(rows/64)*cols elements. */
int dapple_colsum(int dtype, const void* X, int rows, int cols, int ld, float* partial, float* out,
                  void* stream);


/* dapple_colsum for callers that cannot allocate or bring a workspace (code under HIP graph capture, serving
 * loops, harnesses that forbid hipMalloc): the same two kernels and the same summation order, bit for bit, with
 * the partial sums in an array built into the library's device code (one copy of
 * DAPPLE_COLSUM_STATIC_MAX_FLOATS floats = 4 MiB per GPU, held until the process ends).  Allocates nothing and
 * frees nothing; the array's device address is looked up on the first call on a device (a host-side query, no
 * allocation).  ceil(rows/64)*cols must not exceed DAPPLE_COLSUM_STATIC_MAX_FLOATS, else STAGE_E_CONFIG
 * (stage_last_error() says by how much) and nothing is enqueued.  X [rows, ld] and out [cols] are device
 * pointers owned by the caller as in dapple_colsum.  All calls on one GPU share the one array: calls that may
 * overlap on that GPU (different streams, no ordering between them) race; calls on one stream are safe. */
#define DAPPLE_COLSUM_STATIC_MAX_FLOATS (1 << 20)
int dapple_colsum_static(int dtype, const void* X, int rows, int cols, int ld, float* out, void* stream);

/* ------------------------------------------------------------------ operators of layers and training steps
 * Checked on the host before anything is enqueued: a refused call returns STAGE_E_NULL or STAGE_E_CONFIG and
 * stage_last_error() says why.  Nothing is allocated and nothing waited for; results are the same bits from call to call;
 * every call can be captured into a HIP graph (after one eager call of the same kind).  The calling thread's current device is the
 * stream's.  `workspace` is device memory of
 * the size that the operator's *_workspace function returns (host only; a negative code for sizes that would be refused),
 * 16-byte aligned, whose contents do not matter before or after: calls that may overlap need one each. */

/* Attention with a window, first tokens that stay visible, shared key heads and sequences of their own lengths.
 * b sequences of s rows; row r of q holds A heads of d columns (head h in columns [h d, (h+1) d) of q + r*ldq), k and v hold
 * Ak heads, Ak divides A, query head h reads key head h / (A / Ak).  Query i sees key j of its sequence where
 *   j < len  and  (causal = 0 or j <= i)  and  (window = 0 or |i - j| < window or j < sinks)
 * lens: device int32 [b], clamped to [0, s]; NULL = s.  Rows at and behind len see nothing and are seen by nobody; what q, k, v
 * and dctx hold there is not used, and their ctx, dq, dk, dv are set to 0, their lse to -infinity.  Before len, inputs are finite.
 * fwd: ctx = softmax(scale q k^T) v of the visible keys, lse [b,A,s] fp32 = log2 of the sum of 2^(scale log2(e) q k).  ctx32 (may be
 * NULL): an unrounded fp32 ctx in ctx's layout; given to bwd, the row sums of dctx*ctx come from it (a bf16 ctx costs dq and dk
 * accuracy where gradients are sums of many layers').
 * bwd: dq, dk, dv from dctx and the ctx, ctx32 (or NULL) and lse of fwd; dk and dv are summed over the heads that share them.
 * workspace: below 4 b A s bytes + 256 MiB, whatever window and sinks.
 * scale > 0; 0 = 1/sqrt(d).  Row strides in elements, 0 = dense; q, k, v may be columns of one buffer, and dq, dk, dv of another;
 * outputs overlap no input.  bf16: d and strides multiples of 8; fp32: of 4; d <= 128, strides below 2^23, s * stride below 2^30 - 4096,
 * b * s up to 2^26 - 4, b * Ak below 2^16, b * A * ceil(s / 32) below 2^23, bwd b * (A + Ak) * ceil(s / 32) below 2^23 - 2048; all tensors
 * 16-byte aligned.  Probabilities and dS are rounded once to bf16 in bf16 calls, for their products. */
typedef struct {
  const void* q;
  const void* k;
  const void* v;
  void* ctx;
  float* ctx32;
  float* lse;
  const int32_t* lens;
  const void* dctx;
  void* dq;
  void* dk;
  void* dv;
  void* workspace; /* bwd */
  int32_t b, s, A, Ak, d, window, sinks, causal;
  int32_t ldq, ldk, ldv, ldc, lddc, lddq, lddk, lddv; /* ldc: of ctx and ctx32 */
  float scale;
} dapple_attention_window_desc;
int dapple_attention_window_fwd(int dtype, const dapple_attention_window_desc* d, void* stream);
int64_t dapple_attention_window_workspace(int dtype, const dapple_attention_window_desc* d);
int dapple_attention_window_bwd(int dtype, const dapple_attention_window_desc* d, void* stream);

/* Attention of packed documents: rows of one long row of tokens that see their own document only, with capped logits and a bias that
 * falls with the distance.  q [rows, A heads of d], k and v [rows, Ak heads] and shared key heads as above.
 * Document t holds the rows from ends[t - 1] (0) to ends[t]; what row i sees of its document, from begin to end:
 *   (causal = 0 or j <= i or j < begin + prefix[t])  and  (window = 0 or |i - j| < window)
 * dapple_doc_spans writes that down as runs of rows, spans int32 [4 * rows + 1], once for all calls on the same rows (all layers, both
 * directions, any head counts and types).  ends: device int32 [n], ascending (equal ones: an empty document), clamped to [0, rows]; prefix:
 * device int32 [n], clamped to the document, NULL = 0, only with causal.  Rows from ends[n - 1] on see nothing and are seen by nobody;
 * what q, k, v and dctx hold there is not used, their ctx, dq, dk, dv are set to 0, their lse to -infinity.  Before them, inputs are finite.
 *   logit = t - slopes[h] |i - j|,   t = cap tanh(scale q k / cap), or scale q k with cap = 0
 * slopes: device fp32 [A], NULL = 0; finite, and constants (they have no gradient).  cap: 0 or 2^-20 to 2^10.  scale > 0; 0 = 1/sqrt(d);
 * scale / cap and cap / scale that fp32 does not hold as normal numbers are refused.
 * bf16 calls make tanh of an exponential and a reciprocal: a logit, and with it lse, is off by 2^-24 cap + 2^-20 |logit| at most in fwd, the
 * logits of bwd by 2^-21 cap.  fp32 calls keep fp32's precision.
 * fwd: ctx, lse [A, rows] fp32 = log2 of the sum of 2^(log2(e) logit), ctx32 (may be NULL) as above.  bwd: dq, dk, dv from dctx and the ctx, ctx32
 * (or NULL) and lse of fwd.  spans holds what dapple_doc_spans left, of the same rows (other contents: wrong results, nothing worse).
 * Strides, alignment, limits (with b = 1, s = rows; up to 2^26 - 8), rounding and overlaps as for dapple_attention_window; workspace: below
 * 4 A rows bytes + 256 MiB. */
typedef struct {
  const void* q;
  const void* k;
  const void* v;
  void* ctx;
  float* ctx32;
  float* lse;
  const int32_t* spans;
  const float* slopes;
  const void* dctx;
  void* dq;
  void* dk;
  void* dv;
  void* workspace; /* bwd */
  int32_t rows, A, Ak, d;
  int32_t ldq, ldk, ldv, ldc, lddc, lddq, lddk, lddv; /* ldc: of ctx and ctx32 */
  float scale, cap;
} dapple_attention_docs_desc;
int dapple_doc_spans(const int32_t* ends, const int32_t* prefix, int n, int rows, int causal, int window, int32_t* spans, void* stream);
int dapple_attention_docs_fwd(int dtype, const dapple_attention_docs_desc* d, void* stream);
int64_t dapple_attention_docs_workspace(int dtype, const dapple_attention_docs_desc* d);
int dapple_attention_docs_bwd(int dtype, const dapple_attention_docs_desc* d, void* stream);

/* RMS norm of every query and key head and the rotation by position, in one pass (forward), and its gradient.
 * Row r of q holds A heads of d columns, head h in columns [h d, (h+1) d) of q + r*ldq; k holds Ak heads likewise (Ak = 0: no
 * keys, its pointers are not looked at).  Per head:
 *   n = x * gamma / sqrt(mean(x^2) + eps)         gamma_q for queries, gamma_k for keys, [d]; both NULL: n = x
 *   the first `rot` columns turn in pairs, (a, b) -> (a c - b s, a s + b c), (c, s) = table[position][pair]:
 *     interleaved = 0: pair i is columns i and i + rot/2;   1: columns 2i and 2i + 1
 *   columns from rot on are n's.  rot = 0: no rotation (table is not looked at).
 * table: fp32 [max_pos][rot/2][2], as dapple_rope_table or the caller makes it.  positions: int32 [rows], NULL = r % seq (seq 0:
 * r); a position outside [0, max_pos) reads nothing and gives NaN in the columns that turn (backward: and in dgamma).
 * Types: q, k, gammas and outputs of dtype; table, dgamma and all arithmetic fp32.  Row strides in elements, 0 = dense.  An
 * output may be its input (yq = q with ldyq = ldq, dq = dyq, ...), else they do not overlap.  Limits: d <= 256, rot even and <= d,
 * 1 <= rows <= 2^26 - 4; interleaved needs d and the strides even and addresses aligned to two elements; everything aligned to 16 bytes
 * (d, rot/2 or interleaved rot, strides, addresses) is fastest.
 * Backward: dyq, dyk in, dq, dk out (q and k are read only with gammas), dgamma_q, dgamma_k [d] fp32: set, or with accumulate != 0
 * added to; NULL = not wanted.  workspace only where a dgamma is wanted. */
typedef struct {
  const void* q;
  const void* k;
  const void* gamma_q;
  const void* gamma_k;
  const int32_t* positions;
  const float* table;
  void* yq;
  void* yk;
  const void* dyq;
  const void* dyk;
  void* dq;
  void* dk;
  float* dgamma_q;
  float* dgamma_k;
  void* workspace;
  int32_t rows, A, Ak, d, rot, interleaved, seq, max_pos, accumulate;
  int32_t ldq, ldk, ldyq, ldyk, lddyq, lddyk, lddq, lddk;
  float eps;
} dapple_qk_rope_desc;
int dapple_qk_rope_fwd(int dtype, const dapple_qk_rope_desc* d, void* stream);
int64_t dapple_qk_rope_workspace(int dtype, const dapple_qk_rope_desc* d);
int dapple_qk_rope_bwd(int dtype, const dapple_qk_rope_desc* d, void* stream);
/* table[p][i] = magnitude * (cos, sin)(p * f_i), i < rot/2, angles and functions in 64 bits.  With w_i = base^(-2i/rot):
 *   factor = 1: f_i = w_i;   original = 0: f_i = w_i / factor (positions interpolated)
 *   original > 0, the context that the model was trained on: by parts, f_i = w_i (g + (1 - g) / factor), g = 0 for pairs that turn
 *   at most `low` times within it, 1 from `high` times on, linear in the turns between.
 * rot even and at most 256, max_pos * rot below 2^31. */
int dapple_rope_table(float* table, int max_pos, int rot, double base, double factor, int original, double low, double high,
                      double magnitude, void* stream);

/* The gated feed-forward block:  g = x Wg + bg,  u = x Wu + bu,  h = act(g) * u,  y = h Wo + bo, and its gradients.
 * x [T, H], y [T, H] at row strides ldx, ldy; w_in [H, 2F]: the columns of Wg, then those of Wu; b_in [2F] likewise; w_out [F, H],
 * b_out [H]; biases may be NULL.  h [T, F] and gu [T, 2F] (g and u, before the activation) are dense: h is always written (the second
 * product reads it), gu only if given; both are what the backward needs.  act: SiLU g / (1 + e^-g) or GELU (erf).
 * bwd: from x, the weights, gu, h and dy: dgu [T, 2F] (dense, always written), dx (NULL = not wanted), and the weights' gradients
 * dw_in, dw_out (both or neither) with db_in, db_out (NULL = not wanted).  accumulate = 0: these four are of dtype and set;
 * accumulate != 0: fp32, and added to, as a stage sums its micro-batches.
 * Outputs overlap no input.  bf16: H, F and strides multiples of 8; fp32: of 4; all 16-byte aligned; T * 2F, T * stride and H * 2F
 * below 2^30 - 4096; bf16: 2F, ldx and lddy below 2^24.  bf16 calls round g, u, h, dg and du once each (products are summed in fp32). */
enum { DAPPLE_ACT_SILU = 0, DAPPLE_ACT_GELU = 1 };
typedef struct {
  const void* x;
  const void* w_in;
  const void* b_in;
  const void* w_out;
  const void* b_out;
  void* gu;
  void* h;
  void* y;
  const void* dy;
  void* dgu;
  void* dx;
  void* dw_in;
  void* db_in;
  void* dw_out;
  void* db_out;
  void* workspace; /* bwd */
  int32_t T, H, F, act, accumulate;
  int32_t ldx, ldy, lddy, lddx; /* in elements, 0 = H */
} dapple_gated_ffn_desc;
int dapple_gated_ffn_fwd(int dtype, const dapple_gated_ffn_desc* d, void* stream);
int64_t dapple_gated_ffn_workspace(int dtype, const dapple_gated_ffn_desc* d);
int dapple_gated_ffn_bwd(int dtype, const dapple_gated_ffn_desc* d, void* stream);

/* The end of a block: dropout, the residual sum and a norm in one pass, and their gradients.
 *   z = residual + m (x + bias),   y = norm(z) gamma + beta,   m = 1 / (1 - p) where an element is kept, else 0
 *   norm: layer (z - mean) / sqrt(var + eps), RMS z / sqrt(mean(z^2) + eps) (no beta), or none (y, dy, stats are not looked at)
 * rows of H columns, row r of a tensor at r times its stride.  bias, residual, gamma, beta [H]: NULL = 0, 0, 1, 0.  z may be NULL where it
 * is not wanted (the backward of a norm reads it, and stats [rows][2], mean and 1 / sqrt(...), NULL = not wanted).  What is normed is z
 * as it is stored (z NULL too).
 * The mask is made again where it is needed and never stored: element (r, c) belongs to group r * ceil(H / 8) + c / 8, whose four words
 * are Philox4x32-10 of the counter (group, low and high word of rng[1], site) under the key (low and high word of rng[0]); half word
 * c % 8, low halves first, decides: it is kept where that is not below 65536 p, rounded (p is that / 65536 then in 1 / (1 - p), too;
 * p = 1 drops everything).  rng: DEVICE memory, a seed and the number of the step, read when the kernel runs: a captured graph
 * draws another mask where its owner changes them between replays, but not between forward and backward.  site: tells the calls of a step
 * apart.  p = 0: rng is not looked at.
 * bwd: from dy, z and stats, and dz (what comes in through z otherwise; NULL = 0; without a norm it must be given):
 *   g = dz + norm's gradient at dy gamma;   dresidual = g,  dx = m g;   dbias = sum of dx over the rows, dgamma of dy norm(z), dbeta of dy
 * each NULL = not wanted; the sums are fp32 [H], of unrounded values, set, or with accumulate != 0 added to; workspace only where one is
 * wanted.
 * Types: dtype; residual, z, dz and dresidual fp32 with stream32 != 0; statistics and arithmetic fp32.  An output may be an input of the
 * same type and stride (z = residual, dresidual = dz, dx = dy, ...), else they do not overlap.  H <= 16384, rows <= 2^26, rows *
 * ceil(H / 8) < 2^32; any strides and addresses of whole elements. */
enum { DAPPLE_NORM_NONE = 0, DAPPLE_NORM_LAYER = 1, DAPPLE_NORM_RMS = 2 };
typedef struct {
  const void* x;
  const void* bias;
  const void* residual;
  const void* gamma;
  const void* beta;
  const uint64_t* rng;
  void* z;
  void* y;
  float* stats;
  const void* dy;
  const void* dz;
  void* dx;
  void* dresidual;
  float* dbias;
  float* dgamma;
  float* dbeta;
  void* workspace;
  int32_t rows, H, norm, stream32, accumulate, site;
  int32_t ldx, ldr, ldz, ldy, lddy, lddz, lddx, lddr; /* in elements, 0 = H */
  float p, eps;
} dapple_dropout_norm_desc;
int dapple_dropout_norm_fwd(int dtype, const dapple_dropout_norm_desc* d, void* stream);
int64_t dapple_dropout_norm_workspace(int dtype, const dapple_dropout_norm_desc* d);
int dapple_dropout_norm_bwd(int dtype, const dapple_dropout_norm_desc* d, void* stream);

/* Rows of a table:  y[r] = scale * table[ids[r]], and the table's gradient  dtable[v] = scale * sum of dy[r] over the rows with ids[r] = v.
 * table [V, H], ids int32 [rows].  An id outside [0, V) (padding) reads nothing, gives a row of zeros and has no gradient.
 * bwd: accumulate = 0: dtable is of dtype and set, rows of absent ids to zero; accumulate != 0: fp32, and added to, rows of absent ids
 * are not touched.  Sums in fp32, each id's rows in an order that sizes and ids alone decide.
 * Outputs overlap no input.  rows, V <= 2^28, H <= 2^16; any strides and addresses of whole elements; workspace: 16 bytes a row, and at most
 * 64 KiB a column and 512 KiB. */
typedef struct {
  const void* table;
  const int32_t* ids;
  void* y;
  const void* dy;
  void* dtable;
  void* workspace; /* bwd */
  int32_t rows, V, H, accumulate;
  int32_t ldt, ldy, lddy, lddt; /* in elements, 0 = H */
  float scale;
} dapple_embedding_desc;
int dapple_embedding_fwd(int dtype, const dapple_embedding_desc* d, void* stream);
int64_t dapple_embedding_workspace(int dtype, const dapple_embedding_desc* d);
int dapple_embedding_bwd(int dtype, const dapple_embedding_desc* d, void* stream);

/* The global norm of n gradient tensors, all of one dtype: grads and sizes are HOST arrays of n device pointers (aligned to
 * their elements) and element counts (0 is allowed, its pointer is not looked at).
 *   norm_dev[0] = |grad_scale| * sqrt(sum of all squares)      (squares and sums in 64 bits)
 *   norm_dev[1] = min(1, max_norm / norm_dev[0]), 0 if the norm is not finite
 * grad_scale: what the gradients are multiplied with later (1 / samples for accumulated sums).  max_norm > 0, may be
 * infinite.  The gradients of all stages of a model may be given in one call, up to 2^38 - 2^22 elements in all.  workspace: 8-byte
 * aligned is enough. */
int64_t dapple_grad_norm_workspace(const int64_t* sizes, int n);
int dapple_grad_norm(int dtype, const void* const* grads, const int64_t* sizes, int n, float grad_scale, float max_norm,
                     float* norm_dev, void* workspace, void* stream);
/* outs[i] = grads[i] * norm_dev[1], zeros if norm_dev[0] is not finite (grad_scale is not applied).  outs: HOST array of n
 * device pointers, NULL = in place; outs[i] is grads[i] or overlaps none of the tensors, and no tensor is listed twice.
 * stage_apply_adam_clipped (dapple_stage.h) takes norm_dev itself and needs no clipped copy. */
int dapple_grad_clip(int dtype, const void* const* grads, void* const* outs, const int64_t* sizes, int n,
                     const float* norm_dev, void* stream);

#ifdef __cplusplus
}
#endif
#endif
