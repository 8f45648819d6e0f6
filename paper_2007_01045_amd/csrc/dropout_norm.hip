// The end of a block, forward and backward:
//   z = residual + m (x + bias),  y = norm(z) gamma + beta,   m = 1 / (1 - p) where an element is kept, else 0
//   layer: norm(z) = (z - mean) rstd, rstd = (mean((z - mean)^2) + eps)^-1/2;  RMS: mean = 0
//   with h = norm(z), t = dy gamma, means over a row:  g = dz + rstd (t - mean(t) - h mean(t h))  (RMS: without mean(t))
//   dresidual = g,  dx = m g,  dbias = sum of dx over the rows,  dgamma = sum of dy h,  dbeta = sum of dy
// What is normed is z as it is stored (rounded to its type), so that the backward finds the same h.
//
// The mask is never stored: eight elements share a call of Philox4x32-10 (J. Salmon, M. Moraes, R. Dror, D. Shaw, "Parallel random
// numbers: as easy as 1, 2, 3", SC 2011), 16 bits each, and the backward calls it again.  p is thereby a multiple of 2^-16, and
// 1 / (1 - p) is that multiple's, so that means are kept exactly.
//
// Bound by memory: each tensor once.  A row stays in registers between its sums and its outputs.
#include <algorithm>

#include "kernels.h"
#include "row_chunks.h"

namespace dapple {

struct Philox {
  uint32_t k0, k1, c1, c2, c3;
  __device__ __forceinline__ Philox(const uint64_t* rng, uint32_t site) {   // rng NULL: nothing is dropped
    const uint64_t seed = rng ? rng[0] : 0, step = rng ? rng[1] : 0;
    k0 = (uint32_t)seed, k1 = (uint32_t)(seed >> 32), c1 = (uint32_t)step, c2 = (uint32_t)(step >> 32), c3 = site;
  }
  __device__ __forceinline__ void words(uint32_t group, uint32_t (&w)[4]) const {
    uint32_t a = group, b = c1, c = c2, d = c3, p = k0, q = k1;
#pragma unroll
    for (int r = 0; r < 10; ++r) {
      const uint64_t x = (uint64_t)a * 0xD2511F53u, y = (uint64_t)c * 0xCD9E8D57u;
      a = (uint32_t)(y >> 32) ^ b ^ p;
      b = (uint32_t)y;
      c = (uint32_t)(x >> 32) ^ d ^ q;
      d = (uint32_t)x;
      p += 0x9E3779B9u;
      q += 0xBB67AE85u;
    }
    w[0] = a, w[1] = b, w[2] = c, w[3] = d;
  }
};

// x = m x of a group's eight elements
__device__ __forceinline__ void drop8(const Philox& gen, uint32_t group, uint32_t level, float up, float (&x)[8]) {
  uint32_t w[4];
  gen.words(group, w);
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const uint32_t u = e & 1 ? w[e >> 1] >> 16 : w[e >> 1] & 0xffffu;
    x[e] = u >= level ? x[e] * up : 0.f;
  }
}

// The sum over a row of NW waves, the same bits in all of them.  Two slots by turns: whoever writes one again has passed the other's
// barrier, before which everybody had read this one.
template <int NW, int N>
__device__ __forceinline__ void row_sums(float (&v)[N], float* red, int& turn) {
#pragma unroll
  for (int i = 0; i < N; ++i) v[i] = wave_sum(v[i]);
  if constexpr (NW > 1) {
    float* const s = red + turn * NW * N;
    turn ^= 1;
    const int wave = threadIdx.x >> 6;
    if ((threadIdx.x & 63) == 0)
#pragma unroll
      for (int i = 0; i < N; ++i) s[wave * N + i] = v[i];
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; ++i) {
      float t = 0.f;
#pragma unroll
      for (int w = 0; w < NW; ++w) t += s[w * N + i];
      v[i] = t;
    }
  }
}

// NW waves to a row, NCH chunks of a row to a lane; a workgroup has NW waves, or four with a row each
template <int NW> constexpr int row_waves() { return NW > 1 ? NW : 4; }

template <typename T, typename Z, int NORM, int NW, int NCH>
__global__ __launch_bounds__(64 * row_waves<NW>()) void dropout_norm_fwd(DropNormArgs a) {
#pragma clang fp contract(off)
  constexpr int RPB = row_waves<NW>() / NW;
  __shared__ float red[NW > 1 ? 2 * NW : 1];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int at = wave % NW, groups = (a.H + 7) / 8;
  int turn = 0;
  const Philox gen(a.rng, a.site);
  float gam[NCH][8], bet[NCH][8], bia[NCH][8];
  int col[NCH];
#pragma unroll
  for (int c = 0; c < NCH; ++c) {
    col[c] = ((c * NW + at) * 64 + lane) * 8;
#pragma unroll
    for (int e = 0; e < 8; ++e) gam[c][e] = 1.f, bet[c][e] = bia[c][e] = 0.f;
    if (col[c] >= a.H) continue;
    if (NORM && a.gamma) load8((const T*)a.gamma + col[c], a.H - col[c], gam[c]);
    if (NORM && a.beta) load8((const T*)a.beta + col[c], a.H - col[c], bet[c]);
    if (a.bias) load8((const T*)a.bias + col[c], a.H - col[c], bia[c]);
  }
  Raw8<T> xn[NCH] = {};
  Raw8<Z> rn[NCH] = {};
  auto load = [&](long row) {
#pragma unroll
    for (int c = 0; c < NCH; ++c) {
      if (col[c] >= a.H) continue;
      xn[c].load((const T*)a.x + row * a.ldx + col[c], a.H - col[c]);
      if (a.residual) rn[c].load((const Z*)a.residual + row * a.ldr + col[c], a.H - col[c]);
    }
  };
  const long step = (long)gridDim.x * RPB;
  long row = (long)blockIdx.x * RPB + wave / NW;
  if (row < a.rows) load(row);
  for (; row < a.rows; row += step) {
    float z[NCH][8], r[NCH][8];
#pragma unroll
    for (int c = 0; c < NCH; ++c)
#pragma unroll
      for (int e = 0; e < 8; ++e) z[c][e] = xn[c].get(e), r[c][e] = rn[c].get(e);
    if (row + step < a.rows) load(row + step);   // (beside this row's sums)
    float s[1] = {0.f};
#pragma unroll
    for (int c = 0; c < NCH; ++c) {
      if (col[c] >= a.H) continue;
#pragma unroll
      for (int e = 0; e < 8; ++e) z[c][e] = z[c][e] + bia[c][e];
      if (a.level) drop8(gen, (uint32_t)(row * groups + (col[c] >> 3)), a.level, a.up, z[c]);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        z[c][e] = to_f32(from_f32<Z>(z[c][e] + r[c][e]));
        if (NORM == NORM_LAYER) s[0] += col[c] + e < a.H ? z[c][e] : 0.f;
        if (NORM == NORM_RMS) s[0] += col[c] + e < a.H ? z[c][e] * z[c][e] : 0.f;
      }
      if (a.z) store8((Z*)a.z + row * a.ldz + col[c], a.H - col[c], z[c]);
    }
    if constexpr (NORM != NORM_NONE) {
      row_sums<NW>(s, red, turn);
      float mean = 0.f, sq = s[0];
      if constexpr (NORM == NORM_LAYER) {
        mean = s[0] / (float)a.H;
        float q[1] = {0.f};
#pragma unroll
        for (int c = 0; c < NCH; ++c)
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const float d = z[c][e] - mean;
            q[0] += col[c] + e < a.H ? d * d : 0.f;
          }
        row_sums<NW>(q, red, turn);
        sq = q[0];
      }
      const float rstd = 1.f / sqrtf(sq / (float)a.H + a.eps);
      if (a.stats && at == 0 && lane == 0) {
        a.stats[2 * row] = mean;
        a.stats[2 * row + 1] = rstd;
      }
#pragma unroll
      for (int c = 0; c < NCH; ++c) {
        if (col[c] >= a.H) continue;
        float y[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) y[e] = (z[c][e] - mean) * rstd * gam[c][e] + bet[c][e];
        store8((T*)a.y + row * a.ldy + col[c], a.H - col[c], y);
      }
    }
  }
}

// A workgroup's sums over its rows go to partial[blockIdx.x][3][H] (dbias, dgamma, dbeta); its rows and their order depend on the
// sizes alone, so the sums have the same bits every time
template <typename T, typename Z, int NORM, int NW, int NCH>
__global__ __launch_bounds__(64 * row_waves<NW>()) void dropout_norm_bwd(DropNormArgs a) {
  constexpr int RPB = row_waves<NW>() / NW;
  __shared__ float red[NW > 1 ? 4 * NW : 1];
  __shared__ __attribute__((aligned(16))) float joint[NW == 1 ? 4 * 512 * NCH : 4];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int at = wave % NW, groups = (a.H + 7) / 8;
  int turn = 0;
  const Philox gen(a.rng, a.site);
  // Four chunks of a lane are more than its registers hold: dgamma's and dbeta's sums are in LDS (a lane's own), only z and dy of the next row
  // come in ahead, and beside an fp32 stream gamma is loaded for every row.  Us, 4096 rows of 16384, all in registers and memory / so: layer,
  // fp32 stream 627 / 257, RMS 479 / 222; 8192 rows of bf16, layer 759 / 266 (with gamma loaded 309; beside the fp32 stream, not loaded, 306).
  constexpr bool WIDE = NORM && NCH == 4, GAMMA_AGAIN = WIDE && sizeof(Z) == 4;
  __shared__ f32x4 kept[WIDE ? 2 * NCH * 2 * 64 * NW : 1];
  auto in_lds = [&](int v, int c, int half) -> f32x4& { return kept[((v * NCH + c) * 2 + half) * 64 * NW + threadIdx.x]; };
  auto fetch = [&](int v, int c, float (&x)[8]) __attribute__((always_inline)) {
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = in_lds(v, c, e / 4)[e % 4];
  };
  auto keep = [&](int v, int c, const float (&x)[8]) __attribute__((always_inline)) {
#pragma unroll
    for (int e = 0; e < 8; e += 4) in_lds(v, c, e / 4) = f32x4{x[e], x[e + 1], x[e + 2], x[e + 3]};
  };
  float gam[NCH][8], sum[3][NCH][8];
  int col[NCH];
#pragma unroll
  for (int c = 0; c < NCH; ++c) {
    col[c] = ((c * NW + at) * 64 + lane) * 8;
#pragma unroll
    for (int e = 0; e < 8; ++e) gam[c][e] = 1.f, sum[0][c][e] = sum[1][c][e] = sum[2][c][e] = 0.f;
    if (NORM && !GAMMA_AGAIN && a.gamma && col[c] < a.H) load8((const T*)a.gamma + col[c], a.H - col[c], gam[c]);
    if (WIDE) keep(0, c, sum[0][c]), keep(1, c, sum[0][c]);
  }
  Raw8<Z> gn[NCH] = {}, hn[NCH] = {};
  Raw8<T> tn[NCH] = {};
  float mean_n = 0.f, rstd_n = 0.f;
  auto load = [&](long row) {
#pragma unroll
    for (int c = 0; c < NCH; ++c) {
      if (col[c] >= a.H) continue;
      if (!WIDE && a.dz) gn[c].load((const Z*)a.dz + row * a.lddz + col[c], a.H - col[c]);
      if (NORM) hn[c].load((const Z*)a.z + row * a.ldz + col[c], a.H - col[c]);
      if (NORM) tn[c].load((const T*)a.dy + row * a.lddy + col[c], a.H - col[c]);
    }
    if (NORM == NORM_LAYER) mean_n = a.stats[2 * row];
    if (NORM) rstd_n = a.stats[2 * row + 1];
  };
  const long step = (long)gridDim.x * RPB;
  long row = (long)blockIdx.x * RPB + wave / NW;
  if (row < a.rows) load(row);
  for (; row < a.rows; row += step) {
    float g[NCH][8], h[NCH][8], t[NCH][8];
#pragma unroll
    for (int c = 0; c < NCH; ++c) {
      if (WIDE && a.dz && col[c] < a.H) gn[c].load((const Z*)a.dz + row * a.lddz + col[c], a.H - col[c]);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        h[c][e] = hn[c].get(e), t[c][e] = tn[c].get(e);
        if (!WIDE) g[c][e] = gn[c].get(e);
      }
    }
    const float mean = mean_n, rstd = rstd_n;
    if (row + step < a.rows) load(row + step);   // (beside this row's sums)
    if constexpr (NORM != NORM_NONE) {
      float s[2] = {0.f, 0.f};
#pragma unroll
      for (int c = 0; c < NCH; ++c) {
        float again[8] = {1.f, 1.f, 1.f, 1.f, 1.f, 1.f, 1.f, 1.f};
        if (GAMMA_AGAIN && a.gamma && col[c] < a.H) load8((const T*)a.gamma + col[c], a.H - col[c], again);
        auto add = [&](float (&dgam)[8], float (&dbet)[8]) __attribute__((always_inline)) {
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            h[c][e] = (h[c][e] - mean) * rstd;     // (behind the row's end t is 0)
            dgam[e] = fmaf(t[c][e], h[c][e], dgam[e]);
            if (NORM == NORM_LAYER) dbet[e] += t[c][e];
          }
        };
        if constexpr (WIDE) {
          float x[8], y[8];
          fetch(0, c, x);
          if (NORM == NORM_LAYER) fetch(1, c, y);
          add(x, y);
          keep(0, c, x);
          if (NORM == NORM_LAYER) keep(1, c, y);
        } else {
          add(sum[1][c], sum[2][c]);
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          t[c][e] *= GAMMA_AGAIN ? again[e] : gam[c][e];
          s[0] += t[c][e];
          s[1] = fmaf(t[c][e], h[c][e], s[1]);
        }
      }
      row_sums<NW>(s, red, turn);
      const float m0 = NORM == NORM_LAYER ? s[0] / (float)a.H : 0.f, m1 = s[1] / (float)a.H;
#pragma unroll
      for (int c = 0; c < NCH; ++c)
#pragma unroll
        for (int e = 0; e < 8; ++e) g[c][e] = fmaf(rstd, fmaf(-h[c][e], m1, t[c][e] - m0), WIDE ? gn[c].get(e) : g[c][e]);
    }
#pragma unroll
    for (int c = 0; c < NCH; ++c) {
      if (col[c] >= a.H) continue;
      if (a.dr) store8((Z*)a.dr + row * a.lddr + col[c], a.H - col[c], g[c]);
      if (!a.dx && !a.dbias) continue;
      if (a.level) drop8(gen, (uint32_t)(row * groups + (col[c] >> 3)), a.level, a.up, g[c]);
      if (a.dx) store8((T*)a.dx + row * a.lddx + col[c], a.H - col[c], g[c]);
#pragma unroll
      for (int e = 0; e < 8; ++e) sum[0][c][e] += g[c][e];
    }
  }
#pragma unroll
  for (int v = 0; v < (NORM == NORM_LAYER ? 3 : NORM == NORM_RMS ? 2 : 1); ++v) {
    if (!(v == 0 ? a.dbias : v == 1 ? a.dgamma : a.dbeta)) continue;
    float* const P = a.partial + ((long)blockIdx.x * 3 + v) * a.H;
    if (WIDE && v) {
#pragma unroll
      for (int c = 0; c < NCH; ++c) fetch(v - 1, c, sum[v][c]);
    }
    if constexpr (NW == 1) {   // the four waves' sums of the same columns, in their order
      __syncthreads();
#pragma unroll
      for (int c = 0; c < NCH; ++c)
#pragma unroll
        for (int e = 0; e < 8; e += 4)
          *(f32x4*)(joint + (wave * 64 * NCH + c * 64 + lane) * 8 + e) = f32x4{sum[v][c][e], sum[v][c][e + 1], sum[v][c][e + 2], sum[v][c][e + 3]};
      __syncthreads();
      for (int i = threadIdx.x; i < a.H; i += 256)
        P[i] = ((joint[i] + joint[512 * NCH + i]) + joint[2 * 512 * NCH + i]) + joint[3 * 512 * NCH + i];
    } else {
#pragma unroll
      for (int c = 0; c < NCH; ++c)
        if (col[c] < a.H) store8(P + col[c], a.H - col[c], sum[v][c]);
    }
  }
}

// The workgroups' sums in a fixed order: 16 waves, each an equal run of the workgroups in ascending order, then the waves'
__global__ __launch_bounds__(1024) void dropout_norm_sums(DropNormArgs a, int blocks) {
  __shared__ float red[16][64];
  float* const out = blockIdx.y == 0 ? a.dbias : blockIdx.y == 1 ? a.dgamma : a.dbeta;
  if (!out) return;
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, c = blockIdx.x * 64 + lane, per = (blocks + 15) / 16;
  float t = 0.f;
  if (c < a.H) {
    const float* p = a.partial + (long)blockIdx.y * a.H + c;
    const long stride = 3L * a.H;
    const int end = min(blocks, (w + 1) * per);
    int b = w * per;
    for (; b + 7 < end; b += 8) {
      float x[8];
#pragma unroll
      for (int u = 0; u < 8; ++u) x[u] = p[(b + u) * stride];
#pragma unroll
      for (int u = 0; u < 8; ++u) t += x[u];
    }
    for (; b < end; ++b) t += p[b * stride];
  }
  red[w][lane] = t;
  __syncthreads();
  if (w == 0 && c < a.H) {
    float r = a.accumulate ? out[c] : 0.f;
    t = 0.f;
#pragma unroll
    for (int u = 0; u < 16; ++u) t += red[u][lane];
    out[c] = r + t;
  }
}

// ------------------------------------------------------------------ launchers
// f(waves to a row, chunks of a lane)
template <typename F>
static hipError_t for_width(int H, bool bwd, F&& f) {
  using std::integral_constant;
  if (H <= 512) return f(integral_constant<int, 1>{}, integral_constant<int, 1>{});
  // (us forward, a wave / two waves to a row of 1024 in bf16, fp32 stream: 256 rows 5.1 / 3.8, 2048 7.4 / 6.6, 8192 20.1 / 17.4, 32768
  // 78.0 / 77.5; 3001 rows of 1001 in fp32 11.7 / 9.8.  The gradient: 2048 12.7 / 14.8, 8192 23.4 / 24.7, 32768 79 / 84, but 256 rows 9.0 / 8.1)
  if (H <= 1024 && bwd) return f(integral_constant<int, 1>{}, integral_constant<int, 2>{});
  if (H <= 1024) return f(integral_constant<int, 2>{}, integral_constant<int, 1>{});
  if (H <= 2048) return f(integral_constant<int, 4>{}, integral_constant<int, 1>{});
  if (H <= 4096) return f(integral_constant<int, 4>{}, integral_constant<int, 2>{});
  if (H <= 8192) return f(integral_constant<int, 8>{}, integral_constant<int, 2>{});
  return f(integral_constant<int, 8>{}, integral_constant<int, 4>{});
}
// f(io type, stream's type, norm)
template <typename F>
static hipError_t for_types(Dtype dt, const DropNormArgs& a, F&& f) {
  using std::integral_constant;
  auto norm = [&](auto t, auto z) {
    if (a.norm == NORM_LAYER) return f(t, z, integral_constant<int, NORM_LAYER>{});
    if (a.norm == NORM_RMS) return f(t, z, integral_constant<int, NORM_RMS>{});
    return f(t, z, integral_constant<int, NORM_NONE>{});
  };
  if (dt != DT_BF16) return norm(0.f, 0.f);
  return a.stream32 ? norm((bf16)0.f, 0.f) : norm((bf16)0.f, (bf16)0.f);
}

// Workgroups of the backward: each leaves 12 bytes a column behind, which are written and read once more, and its rows' loads run
// ahead of their sums, so that few waves keep the memory busy.  Us with 256 / 512 of them: rows of 256, 16384 rows 21.0 / 18.5, 2048 8.5 / 8.8;
// of 1024, 8192 rows 23.6 / 23.4, 32768 79 / 82; of 2048, 1024 rows 14.0 / 16.1, 8192 43.1 / 38.0; of 4096, 32768 rows 241 / 264; of
// 8192, 16384 rows 306 / 313 (1024 of them were the slowest of all).
int dropout_norm_blocks(int rows, int H) {
  const int per = H <= 1024 ? 4 : 1;
  return std::min((rows + per - 1) / per, H <= 512 || (H > 1024 && H <= 2048 && rows >= 4096) ? 512 : 256);
}

hipError_t launch_dropout_norm_fwd(Dtype dt, const DropNormArgs& a, hipStream_t st) {
  return for_types(dt, a, [&](auto t, auto z, auto N) {
    return for_width(a.H, false, [&](auto NW, auto NCH) {
      constexpr int nw = decltype(NW)::value, per = row_waves<nw>() / nw;
      // (us with 2048 / 4096 workgroups: rows of 1024, 8192 of them 17.4 / 18.1; of 4096, 32768 204 / 199)
      const unsigned grid = (unsigned)std::min<long>(((long)a.rows + per - 1) / per, a.H > 1024 ? 4096 : 2048);
      hipLaunchKernelGGL((dropout_norm_fwd<decltype(t), decltype(z), decltype(N)::value, nw, decltype(NCH)::value>), dim3(grid),
                         dim3(64 * row_waves<nw>()), 0, st, a);
      return hipGetLastError();
    });
  });
}

hipError_t launch_dropout_norm_bwd(Dtype dt, const DropNormArgs& a, hipStream_t st) {
  const int blocks = dropout_norm_blocks(a.rows, a.H);
  hipError_t e = for_types(dt, a, [&](auto t, auto z, auto N) {
    return for_width(a.H, true, [&](auto NW, auto NCH) {
      constexpr int nw = decltype(NW)::value;
      hipLaunchKernelGGL((dropout_norm_bwd<decltype(t), decltype(z), decltype(N)::value, nw, decltype(NCH)::value>), dim3(blocks),
                         dim3(64 * row_waves<nw>()), 0, st, a);
      return hipGetLastError();
    });
  });
  if (e != hipSuccess || (!a.dbias && !a.dgamma && !a.dbeta)) return e;
  hipLaunchKernelGGL(dropout_norm_sums, dim3((a.H + 63) / 64, 3), dim3(1024), 0, st, a, blocks);
  return hipGetLastError();
}

}  // namespace dapple
