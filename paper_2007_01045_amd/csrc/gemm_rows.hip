// The products of a gated feed-forward block (bf16) whose other side has at most 32 rows.  What bounds them is reading the weights
// once, and how many compute units read: one draws 20-30 GB/s of what is not in its L2, whatever it has in flight.  So a workgroup
// takes 16 columns (of the gate and the same of the value), a quarter of an L2 line's, eight waves an eighth of the depth each, all of a
// wave's part (up to 512 rows of a weight) requested before the first is used, and the waves' sums are added in LDS in wave order.
// A k-strided weight goes through a piece of LDS of the wave's own and is read back transposed; a k-contiguous one is loaded as fragments.
#include "device_common.h"
#include "kernels.h"

namespace dapple {

constexpr int RW = 8;   // waves

// what leaves the products: Y = sums (+ bias);  H = act(gate) * value, and the two (C2);  G = the two's gradients from dh
enum class RowsOut { Y, H, G };

// MB: blocks of 16 rows
template <RowsOut OUT, bool BKS, int MB>
__global__ __launch_bounds__(64 * RW) void gemm_rows_kernel(GemmArgs g) {
  constexpr int NB = OUT == RowsOut::H ? 2 : 1, DEPTH = 16 / NB / MB;   // blocks of 32 of K in flight
  __shared__ __attribute__((aligned(16))) unsigned char tile[BKS ? RW * DEPTH * 1024 * NB : 16];
  __shared__ f32x4 sums[RW][MB * NB][64];
  const int lane = threadIdx.x & 63, l15 = lane & 15, q4 = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const unsigned per_xcd = gridDim.x / 8, id = blockIdx.x < per_xcd * 8 ? (blockIdx.x & 7) * per_xcd + (blockIdx.x >> 3) : blockIdx.x;
  const int n0 = id * 16;   // (neighbours of a line on one XCD)
  const int per = (g.K + RW * 32 - 1) / (RW * 32) * 32, k0 = wave * per, k1 = min(g.K, k0 + per);
  const bf16 *A = (const bf16*)g.A, *B = (const bf16*)g.B;
  f32x4 acc[MB][NB];
#pragma unroll
  for (int i = 0; i < MB; ++i)
#pragma unroll
    for (int b = 0; b < NB; ++b) acc[i][b] = f32x4{0.f, 0.f, 0.f, 0.f};
  for (int k = k0; k < k1; k += 32 * DEPTH) {
    bf16x8 w[DEPTH][NB], a[DEPTH][MB];
#pragma unroll
    for (int q = 0; q < DEPTH; ++q)
#pragma unroll
      for (int b = 0; b < NB; ++b) {
        w[q][b] = bf16x8{};
        if constexpr (BKS) {   // two lanes to a row of 16 columns
          const int r = k + 32 * q + lane / 2, col = n0 + lane % 2 * 8;
          if (r < k1 && col < g.N) w[q][b] = *(const bf16x8*)(B + (long)r * g.ldb + b * g.N + col);
        } else {
          const int kk = k + 32 * q + 8 * q4;
          if (kk < k1 && n0 + l15 < g.N) w[q][b] = *(const bf16x8*)(B + (long)(n0 + l15) * g.ldb + kk);
        }
      }
#pragma unroll
    for (int q = 0; q < DEPTH; ++q)
#pragma unroll
      for (int i = 0; i < MB; ++i) {
        const int kk = k + 32 * q + 8 * q4, row = 16 * i + l15;
        a[q][i] = bf16x8{};
        if (kk < k1 && row < g.M) a[q][i] = *(const bf16x8*)(A + (long)row * g.lda + kk);
      }
    __builtin_amdgcn_sched_barrier(0);   // all requests before the first use
    if constexpr (BKS) {
      bf16* const S = (bf16*)(tile + wave * DEPTH * 1024 * NB);
#pragma unroll
      for (int q = 0; q < DEPTH; ++q)
#pragma unroll
        for (int b = 0; b < NB; ++b) *(bf16x8*)(S + (q * NB + b) * 512 + lane * 8) = w[q][b];
      __builtin_amdgcn_wave_barrier();   // (private to the wave, whose LDS accesses execute in order)
      // 16 lanes read 4 rows of 16 columns; a lane receives its column of them
#pragma unroll
      for (int q = 0; q < DEPTH; ++q)
#pragma unroll
        for (int b = 0; b < NB; ++b) {
          const bf16* const p = S + (q * NB + b) * 512 + (8 * q4 + (l15 >> 2)) * 16 + (l15 & 3) * 4;
          w[q][b] = join8(lds_read_tr16(p), lds_read_tr16(p + 64));
        }
      __builtin_amdgcn_wave_barrier();
    }
#pragma unroll
    for (int q = 0; q < DEPTH; ++q)
#pragma unroll
      for (int i = 0; i < MB; ++i)
#pragma unroll
        for (int b = 0; b < NB; ++b) acc[i][b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w[q][b], a[q][i], acc[i][b], 0, 0, 0);
  }
  // acc[i][b]: row 16 i + l15, columns n0 + 4 q4 + 0..3
#pragma unroll
  for (int i = 0; i < MB; ++i)
#pragma unroll
    for (int b = 0; b < NB; ++b) sums[wave][i * NB + b][lane] = acc[i][b];
  __syncthreads();
  const int row = 16 * wave + l15, col = n0 + 4 * q4;
  if (wave >= MB || row >= g.M || col >= g.N) return;
  f32x4 t[NB];
#pragma unroll
  for (int b = 0; b < NB; ++b) {
    t[b] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int x = 0; x < RW; ++x) t[b] += sums[x][wave * NB + b][lane];
    if (OUT != RowsOut::G && (g.epi & EPI_BIAS)) {
      const bf16x4 y = *(const bf16x4*)((const bf16*)g.bias + b * g.N + col);
#pragma unroll
      for (int e = 0; e < 4; ++e) t[b][e] += (float)y[e];
    }
  }
  bf16* const C = (bf16*)g.C + (long)row * g.ldc + col;
  auto store = [](bf16* p, f32x4 v) {
    bf16x4 o;
#pragma unroll
    for (int e = 0; e < 4; ++e) o[e] = (bf16)v[e];
    *(bf16x4*)p = o;
  };
  if constexpr (OUT == RowsOut::Y) {
    store(C, t[0]);
  } else {
    const bool silu = (g.epi & EPI_SILU) != 0;
    f32x4 x, y = t[0];
    if constexpr (OUT == RowsOut::H) {
      if (g.C2) {
        bf16* const q = (bf16*)g.C2 + (long)row * g.ldaux + col;
        store(q, t[0]);
        store(q + g.N, t[NB - 1]);
      }
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        float act, dact;
        gate_act(silu, t[0][e], act, dact);
        x[e] = act * t[NB - 1][e];
      }
      store(C, x);
    } else {
      const bf16* const q = (const bf16*)g.aux + (long)row * g.ldaux + col;
      const bf16x4 gate = *(const bf16x4*)q, value = *(const bf16x4*)(q + g.N);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        float act, dact;
        gate_act(silu, (float)gate[e], act, dact);
        x[e] = t[0][e] * (float)value[e] * dact;
        y[e] = t[0][e] * act;
      }
      store(C, x);
      store(C + g.N, y);
    }
  }
}

template <RowsOut OUT, bool BKS>
static hipError_t launch(const GemmArgs& g, hipStream_t st) {
  const dim3 grid((g.N + 15) / 16), block(64 * RW);
  if constexpr (OUT != RowsOut::H)   // (gate and value: 16 rows)
    if (g.M > 16) {
      hipLaunchKernelGGL((gemm_rows_kernel<OUT, BKS, 2>), grid, block, 0, st, g);
      return hipGetLastError();
    }
  hipLaunchKernelGGL((gemm_rows_kernel<OUT, BKS, 1>), grid, block, 0, st, g);
  return hipGetLastError();
}

// Where they take less than the smallest tiles of the MFMA kernel, whose workgroups have more columns and one wave each: while each of
// the 256 units has one of these workgroups, 4096 columns; beyond that the tiles have enough workgroups and read larger pieces.
// us, tiles / these, weights out of memory:
//   k-contiguous weights, 16 rows, depth 1024, 1024 columns 5.7 / 4.5, 4096 7.2 / 5.4, 8192 7.5 / 8.6, 16384 9.4 / 14.4; depth 4096, 4096 columns
//     16.6 / 10.8, 8192 16.8 / 19.1; 1024 of depth 8192 27.5 / 17.5 (one row 6.6 / 4.5, 7.0 / 7.1 and 15.7 / 8.2, 15.6 / 13.9 for 4096, 8192 of 1024, 4096);
//     32 rows, 4096 of depth 1024 5.8 / 5.5, 1024 of 8192 19.8 / 23.3
//   the same, a depth that is no multiple of 64 (there the tiles are of 64x64): 32 rows, depth 1032, 4096 columns 10.5 / 5.9, 8192 11.0 / 9.2, 16384
//     12.9 / 15.9; depth 4104, 4096 columns 25.1 / 13.5, 8192 25.6 / 24.2
//   k-strided, 16 rows: 1024 of 4096 11.9 / 12.8, 1032 of 4104 21.0 / 11.8 (32 rows 21.3 / 14.4); with the gate and value product, depth
//     4104, 32 rows, 4096 columns 49.5 / 43.9, 8192 91 / 102
//   gate and value, 16 rows: 256 of 2048 10.2 / 8.0, 2048 of 768 7.1 / 6.5, 4096 of 1024 8.2 / 8.4, 8192 of 2048 19 / 26; 32 rows, 256 of 2048
//     10.4 / 12.1
bool gemm_rows_takes(const GemmArgs& g, bool gate) {
  const bool ragged = g.K % 64 != 0;
  if (!g.b_kstrided) return ragged ? g.M <= 32 && g.N <= 8192 : g.M <= 16 && g.N <= 4096;
  return gate ? g.M <= 16 && g.N <= 2048 : g.M <= 32 && g.N <= 4096 && ragged;
}
hipError_t launch_rows_gate_fwd(const GemmArgs& g, hipStream_t st) { return launch<RowsOut::H, true>(g, st); }
hipError_t launch_rows_gate_bwd(const GemmArgs& g, hipStream_t st) { return launch<RowsOut::G, false>(g, st); }
hipError_t launch_rows(const GemmArgs& g, hipStream_t st) {
  return g.b_kstrided ? launch<RowsOut::Y, true>(g, st) : launch<RowsOut::Y, false>(g, st);
}

}  // namespace dapple
