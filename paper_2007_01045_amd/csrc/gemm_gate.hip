// The two bf16 products of a gated feed-forward block that have an activation in their epilogue (GATE of gemm_mfma.h).
// Forward: act(x Wg + bg) * (x Wu + bu).  One product over the packed weights [H, 2F]: a tile of BN columns takes BN / 2 columns
// of the gate and the same ones of the value, in blocks of 32 by turns, so that each wave holds both of a column and the
// block's hidden row leaves the kernel finished: x is read once, and the two projections reach memory only if the caller keeps them.
// Backward: dh = dy Wo^T never reaches memory; the epilogue reads the two projections and writes their gradients.
#include "gemm_mfma.h"

namespace dapple {

template <int BM, int BN, int WGM, int WGN, int NS, bool BKS, int BK, bool KT, int GATE>
__global__ __launch_bounds__(64 * WGM * WGN, (GemmTile<BM, BN, WGM, WGN, NS, false, BKS, BK, KT>::MIN_WAVES)) void gemm_gate_kernel(GemmArgs g, int tiles_m, int tiles_n) {
  gemm_mfma_tile<BM, BN, WGM, WGN, NS, false, BKS, BK, false, KT, false, false, GATE>(g, tiles_m, tiles_n, blockIdx.x, 0);
}

template <int BM, int BN, int WGM, int WGN, int NS, bool BKS, int BK, bool KT, int GATE>
static hipError_t launch(const GemmArgs& g, hipStream_t st) {
  typedef GemmTile<BM, BN, WGM, WGN, NS, false, BKS, BK, KT> CFG;
  auto kern = gemm_gate_kernel<BM, BN, WGM, WGN, NS, BKS, BK, KT, GATE>;
  static const hipError_t rc = hipFuncSetAttribute((const void*)kern, hipFuncAttributeMaxDynamicSharedMemorySize, (int)CFG::LDS_BYTES);
  if (rc != hipSuccess) return rc;
  constexpr int BNC = GATE == 1 ? BN / 2 : BN;
  const int tiles_m = (g.M + BM - 1) / BM, tiles_n = (g.N + BNC - 1) / BNC;
  hipLaunchKernelGGL(kern, dim3(tiles_m * tiles_n), dim3(CFG::NT), CFG::LDS_BYTES, st, g, tiles_m, tiles_n);
  return hipGetLastError();
}

static long tiles(const GemmArgs& g, long m, long n) { return ((g.M + m - 1) / m) * ((g.N + n - 1) / n); }

// Tiles as in gemm.hip: the largest of which three quarters of the 256 units get one
hipError_t launch_gate_fwd(const GemmArgs& g, hipStream_t st) {
  const bool short_k = g.K % 64 != 0;
  if (short_k) return tiles(g, 128, 64) >= 192 ? launch<128, 128, 4, 2, 2, true, 64, true, 1>(g, st) : launch<64, 64, 2, 1, 4, true, 64, true, 1>(g, st);
  if (tiles(g, 256, 128) >= 192) return launch<256, 256, 2, 4, 4, true, 32, false, 1>(g, st);
  if (tiles(g, 128, 64) >= 192) return launch<128, 128, 4, 2, 2, true, 64, false, 1>(g, st);
  if (tiles(g, 32, 32) <= 256) return launch<32, 64, 1, 1, 4, true, 64, false, 1>(g, st);
  return launch<64, 64, 2, 1, 4, true, 64, false, 1>(g, st);
}

hipError_t launch_gate_bwd(const GemmArgs& g, hipStream_t st) {
  const bool short_k = g.K % 64 != 0;
  if (short_k) return tiles(g, 128, 128) >= 192 ? launch<128, 128, 2, 4, 2, false, 64, true, 2>(g, st) : launch<64, 64, 2, 2, 4, false, 64, true, 2>(g, st);
  if (tiles(g, 256, 256) >= 192) return launch<256, 256, 2, 4, 4, false, 32, false, 2>(g, st);
  if (tiles(g, 128, 128) >= 192) return launch<128, 128, 2, 4, 2, false, 64, false, 2>(g, st);
  if (tiles(g, 32, 32) <= 256) return launch<32, 32, 1, 1, 4, false, 64, false, 2>(g, st);
  return launch<64, 64, 2, 2, 4, false, 64, false, 2>(g, st);
}

}  // namespace dapple
