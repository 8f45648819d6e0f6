// The gated feed-forward block, forward and backward, as products:
//   g = x Wg + bg,  u = x Wu + bu,  h = act(g) u,  y = h Wo + bo
//   dh = dy Wo^T,  du = dh act(g),  dg = dh u act'(g),  dx = [dg du] [Wg Wu]^T,  dW = x^T [dg du],  dWo = h^T dy, biases: column sums
// bf16: h leaves the product that makes g and u, dg and du the one that makes dh (gemm_gate.hip); the others are products as the
// encoder layers have them.  Bound by the matrix cores, 6 T H F flops forward and 12 backward; few rows by reading the weights.
// fp32: the same shape where the products have tiles enough (gated_ffn_f32.hip); with fewer of them they go to the kernels that
// split K over a workgroup's waves (gemm_f32.hip), and the activations are passes of their own.
#include "device_common.h"
#include "kernels.h"

namespace dapple {

// what a pass does per four columns of a row:  ACT: h = act(h);  MUL: h = act(gu) gu[F];  GRAD: dgu, whose value half holds dh
enum class Pass { ACT, MUL, GRAD };
template <Pass P>
__global__ __launch_bounds__(256) void gate_pass_f32(const float* __restrict__ gu, float* io, long n4, int F4, bool silu) {
  const long stride = (long)gridDim.x * 256;
  for (long i = (long)blockIdx.x * 256 + threadIdx.x; i < n4; i += stride) {
    f32x4* const p = (f32x4*)io;
    const long at = P == Pass::ACT ? i : i / F4 * 2 * F4 + i % F4;   // of the gate, in [T, 2F]
    const f32x4 g = P == Pass::ACT ? p[i] : ((const f32x4*)gu)[at];
    f32x4 a, da;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      float x, y;
      gate_act(silu, g[e], x, y);
      a[e] = x;
      da[e] = y;
    }
    if constexpr (P == Pass::ACT) p[i] = a;
    else {
      const f32x4 u = ((const f32x4*)gu)[at + F4];
      if constexpr (P == Pass::MUL) p[i] = a * u;
      else {
        const f32x4 dh = p[at + F4];
        p[at] = dh * u * da;
        p[at + F4] = dh * a;
      }
    }
  }
}

__global__ __launch_bounds__(256) void zero_f32_kernel(float* a, int na, float* b, int nb) {
  for (int i = blockIdx.x * 256 + threadIdx.x; i < na + nb; i += gridDim.x * 256) (i < na ? a[i] : b[i - na]) = 0.f;
}

// C[m, n] = sum over k of A(m, k) B(n, k); a, b: k-strided
static GemmArgs product(const void* A, int lda, bool a, const void* B, int ldb, bool b, void* C, int ldc, int M, int N, int K) {
  GemmArgs g{};
  g.A = A; g.lda = lda; g.a_kstrided = a; g.B = B; g.ldb = ldb; g.b_kstrided = b; g.C = C; g.ldc = ldc;
  g.M = g.m_valid = M; g.N = g.n_valid = N; g.K = g.kseg_len = g.k_valid = K; g.batch = 1;
  return g;
}
static void with_bias(GemmArgs& g, const void* bias) {
  g.bias = bias;
  if (bias) g.epi |= EPI_BIAS;
}

static GemmArgs fwd_in(const GatedFfnArgs& a, void* C, int ldc) { return product(a.x, a.ldx, false, a.w_in, 2 * a.F, true, C, ldc, a.T, 2 * a.F, a.H); }
static GemmArgs fwd_out(const GatedFfnArgs& a) {
  GemmArgs g = product(a.h, a.F, false, a.w_out, a.H, true, a.y, a.ldy, a.T, a.H, a.F);
  with_bias(g, a.b_out);
  return g;
}
static GemmArgs bwd_dh(const GatedFfnArgs& a, void* C) { return product(a.dy, a.lddy, false, a.w_out, a.H, false, C, 2 * a.F, a.T, a.F, a.H); }
static GemmArgs bwd_dx(const GatedFfnArgs& a) { return product(a.dgu, 2 * a.F, false, a.w_in, 2 * a.F, false, a.dx, a.lddx, a.T, a.H, 2 * a.F); }
static GemmArgs bwd_dw(const GatedFfnArgs& a, bool in, float* bsum) {
  GemmArgs g = in ? product(a.x, a.ldx, true, a.dgu, 2 * a.F, true, a.dw_in, 2 * a.F, a.H, 2 * a.F, a.T)
                  : product(a.h, a.F, true, a.dy, a.lddy, true, a.dw_out, a.H, a.F, a.H, a.T);
  if (a.accumulate) g.epi |= EPI_ACC32;
  if (bsum) {
    g.epi |= EPI_BSUM;
    g.bsum = bsum;
  }
  return g;
}

// The tile of a weight gradient's product (T rows deep): 256x256 or 256x128 where three quarters of the 256 units get one, else 0,
// the choice for the encoder layers (128x128, eight waves).  With the bias' sums, T = 8192: 2048 x 16384 756 -> 468 us (256x256),
// 8192 x 2048 273 -> 215; 1024 x 8192 139 -> 131 (256x128; 256x256 166), T = 2048, 4096 x 2048 38 -> 36 (49).
static int dw_tile(const GemmArgs& g) {
  auto tiles = [&](int m, int n) { return (long)((g.M + m - 1) / m) * ((g.N + n - 1) / n); };
  return tiles(256, 256) >= 192 ? 1 : tiles(256, 128) >= 192 ? 2 : 0;
}

bool gated_ffn_takes(Dtype dt, const GatedFfnArgs& a, bool bwd) {
  auto takes = [&](const GemmArgs& g) { return dt == DT_BF16 ? gemm_uses_mfma(dt, g) : gemm_f32_takes(g); };
  float some = 0.f;
  auto al16 = [](const void* p) { return (uintptr_t)p % 16 == 0; };
  if (!al16(a.b_in) || !al16(a.b_out) || !al16(a.gu) || !al16(a.dgu) || !al16(a.h)) return false;
  if (!bwd) return takes(fwd_in(a, a.h, 2 * a.F)) && takes(fwd_out(a));
  return takes(bwd_dh(a, a.dgu)) && (!a.dx || takes(bwd_dx(a))) && (!a.dw_in || (takes(bwd_dw(a, true, &some)) && takes(bwd_dw(a, false, &some))));
}

int64_t gated_ffn_workspace(Dtype dt, const GatedFfnArgs& a) {
  return dt == DT_F32 ? gated_ffn_f32_workspace(a) : 16;   // (bf16: none)
}

static unsigned pass_blocks(long n) { return (unsigned)((n + 255) / 256 < 65536 ? (n + 255) / 256 : 65536); }

hipError_t launch_gated_ffn_fwd(Dtype dt, const GatedFfnArgs& a, hipStream_t st) {
  hipError_t e;
  const RingPlan ring = dt == DT_F32 ? gated_ffn_f32_plan(a) : RingPlan{};
  if (dt == DT_BF16) {
    GemmArgs g = fwd_in(a, a.h, a.F);
    g.N = a.F;
    g.C2 = a.gu;
    g.ldaux = 2 * a.F;
    with_bias(g, a.b_in);
    if (a.silu) g.epi |= EPI_SILU;
    e = gemm_rows_takes(g, true) ? launch_rows_gate_fwd(g, st) : launch_gate_fwd(g, st);
  } else if (ring.in) {
    e = launch_ring_f32_in(a, st);
  } else {
    const long n4 = (long)a.T * a.F / 4;
    if (a.gu) {
      GemmArgs g = fwd_in(a, a.gu, 2 * a.F);
      with_bias(g, a.b_in);
      e = launch_gemm(dt, g, st);
      if (e != hipSuccess) return e;
      hipLaunchKernelGGL(gate_pass_f32<Pass::MUL>, dim3(pass_blocks(n4)), dim3(256), 0, st, (const float*)a.gu, (float*)a.h, n4, a.F / 4, a.silu);
      e = hipGetLastError();
    } else {   // the gate in h's place, and the value times it
      for (int part = 0; part < 2; ++part) {
        GemmArgs g = fwd_in(a, a.h, a.F);
        g.N = g.n_valid = a.F;
        g.B = (const float*)a.w_in + part * a.F;
        with_bias(g, a.b_in ? (const float*)a.b_in + part * a.F : nullptr);
        if (part) {
          g.epi |= EPI_MUL;
          g.aux = a.h;
          g.ldaux = a.F;
        }
        e = launch_gemm(dt, g, st);
        if (e != hipSuccess) return e;
        if (!part) hipLaunchKernelGGL(gate_pass_f32<Pass::ACT>, dim3(pass_blocks(n4)), dim3(256), 0, st, nullptr, (float*)a.h, n4, a.F / 4, a.silu);
        e = hipGetLastError();
        if (e != hipSuccess) return e;
      }
    }
  }
  if (e != hipSuccess) return e;
  if (ring.out) return launch_ring_f32_out(a, st);
  return dt == DT_BF16 && gemm_rows_takes(fwd_out(a), false) ? launch_rows(fwd_out(a), st) : launch_gemm(dt, fwd_out(a), st);
}

hipError_t launch_gated_ffn_bwd(Dtype dt, const GatedFfnArgs& a, void* workspace, hipStream_t st) {
  hipError_t e;
  const RingPlan ring = dt == DT_F32 ? gated_ffn_f32_plan(a) : RingPlan{};
  if (dt == DT_BF16) {
    GemmArgs g = bwd_dh(a, a.dgu);
    g.aux = a.gu;
    g.ldaux = 2 * a.F;
    if (a.silu) g.epi |= EPI_SILU;
    e = gemm_rows_takes(g, false) ? launch_rows_gate_bwd(g, st) : launch_gate_bwd(g, st);
  } else if (ring.dh) {
    e = launch_ring_f32_dh(a, st);
  } else {
    const long n4 = (long)a.T * a.F / 4;
    e = launch_gemm(dt, bwd_dh(a, (float*)a.dgu + a.F), st);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(gate_pass_f32<Pass::GRAD>, dim3(pass_blocks(n4)), dim3(256), 0, st, (const float*)a.gu, (float*)a.dgu, n4, a.F / 4, a.silu);
    e = hipGetLastError();
  }
  if (e == hipSuccess && a.dx && !ring.dx) e = dt == DT_BF16 && gemm_rows_takes(bwd_dx(a), false) ? launch_rows(bwd_dx(a), st) : launch_gemm(dt, bwd_dx(a), st);
  if (e == hipSuccess && (ring.dx || ring.dw)) e = launch_ring_f32_grads(a, ring, workspace, st);
  if (e != hipSuccess || !a.dw_in || ring.dw) return e;
  GemmArgs win = bwd_dw(a, true, nullptr), wout = bwd_dw(a, false, nullptr);
  if (dt == DT_BF16) win.tile = dw_tile(win), wout.tile = dw_tile(wout);
  // Both in one launch where they have no large tiles.  The biases' sums leave the products as the gradients are wanted: with kernels of
  // their own that cleared them and rounded them to bf16, and two launches, 300 rows of 512 x 2048 took 35 us for 26, 8192 of 128 x 512 84 for 50.
  const bool set16 = dt == DT_BF16 && !a.accumulate;
  if ((a.accumulate || set16) && !win.tile && !wout.tile) {
    WgradGroup w{};
    w.p[0] = WgradProblem{a.x, a.dgu, (float*)a.dw_in, (float*)a.db_in, a.H, 2 * a.F, a.ldx, 2 * a.F, 2 * a.F};
    w.p[1] = WgradProblem{a.h, a.dy, (float*)a.dw_out, (float*)a.db_out, a.F, a.H, a.F, a.lddy, a.H};
    w.n = 2;
    w.K = w.kseg = a.T;
    w.set = set16;
    return launch_wgrad_group(dt, w, st);
  }
  if (dt == DT_F32 && !a.accumulate && (a.db_in || a.db_out)) {   // (the fp32 products add to them)
    const int ni = a.db_in ? 2 * a.F : 0, no = a.db_out ? a.H : 0;
    hipLaunchKernelGGL(zero_f32_kernel, dim3((ni + no + 255) / 256), dim3(256), 0, st, (float*)a.db_in, ni, (float*)a.db_out, no);
    e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  auto with_sum = [&](GemmArgs& g, void* sum) {
    g.bsum = (float*)sum;
    if (sum) g.epi |= EPI_BSUM | (set16 ? EPI_BSUM_BF16 : 0);
  };
  with_sum(win, a.db_in);
  with_sum(wout, a.db_out);
  e = launch_gemm(dt, win, st);
  return e == hipSuccess ? launch_gemm(dt, wout, st) : e;
}

}  // namespace dapple
