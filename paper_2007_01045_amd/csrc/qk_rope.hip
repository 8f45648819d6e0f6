// RMS norm of every query and key head and the rotation by position, in one pass over the heads, and its gradient.
//   n = x rstd gamma,  rstd = 1 / sqrt(mean of x^2 over the head + eps)      (without gammas: n = x)
//   a pair (a, b) of the first `rot` columns becomes (a c - b s, a s + b c),  (c, s) = table[position][pair];
//   pairs: columns (i, i + rot/2), or (2i, 2i + 1); the columns from rot on stay as they are.
//   backward: dn = the pair turned back, dgamma += sum of dn x rstd over rows and heads,
//             dx = rstd (dn gamma - x rstd mean(dn gamma x rstd)).
// Bound by memory: an element is read and written once (backward: two reads, one write); the table's row of a position is
// read once per wave for all heads of the row, and comes out of the L2s.
//
// A lane owns a UNIT of a head: two chunks of V consecutive columns, chosen so that both columns of every pair are the lane's
// (the chunks rot/2 apart, or neighbours in one chunk), and the rotation needs no exchange.  G lanes (a power of two) hold a head, 64 / G heads are
// done at a time; the only exchange is the sum of squares within G lanes.  A wave takes all heads of a row, so that its part
// of the table and of gamma stays in registers.
#include <type_traits>

#include "device_common.h"
#include "kernels.h"

namespace dapple {

// sum over each group of G consecutive lanes, G a power of two, in every lane of the group, as a fixed tree
__device__ __forceinline__ float group_sum(float v, int G) {
  auto dpp = [](float x, auto CTRL) {
    return x + __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), decltype(CTRL)::value, 0xF, 0xF, true));
  };
  if (G > 1) v = dpp(v, std::integral_constant<int, 0xB1>{});    // quad_perm [1,0,3,2]
  if (G > 2) v = dpp(v, std::integral_constant<int, 0x4E>{});    // quad_perm [2,3,0,1]
  if (G > 4) v = dpp(v, std::integral_constant<int, 0x141>{});   // row_half_mirror
  if (G > 8) v = dpp(v, std::integral_constant<int, 0x140>{});   // row_mirror
  if (G > 16) v += __shfl_xor(v, 16, 64);
  if (G > 32) v += __shfl_xor(v, 32, 64);
  return v;
}

template <typename T, int V>
__device__ __forceinline__ void load_chunk(const T* p, float (&o)[V]) {
  typedef T TV __attribute__((ext_vector_type(V)));
  if constexpr (V == 1) {
    o[0] = to_f32(*p);
  } else {
    const TV x = *(const TV*)p;
#pragma unroll
    for (int e = 0; e < V; ++e) o[e] = to_f32((T)x[e]);
  }
}
template <typename T, int V>
__device__ __forceinline__ void store_chunk(T* p, const float (&o)[V]) {
  typedef T TV __attribute__((ext_vector_type(V)));
  if constexpr (V == 1) {
    *p = from_f32<T>(o[0]);
  } else {
    TV x;
#pragma unroll
    for (int e = 0; e < V; ++e) x[e] = from_f32<T>(o[e]);
    *(TV*)p = x;
  }
}

// HALF: pairs (i, i + rot/2); else neighbours.  A lane's units, NU of them: where their chunks begin (-1: none) and whether they
// turn.  Chunks that need not be together are half of the columns apart, so that a load of a head's lanes is one piece.
template <int V, bool HALF, int NU>
struct Units {
  int off[NU][2];
  bool turn[NU][2];
  int pair[NU][2];   // table pair of a chunk's first (HALF: the first's, of the V pairs of both)
  __device__ __forceinline__ void init(int d, int rot, int lane_in_head, int G) {
#pragma unroll
    for (int i = 0; i < NU; ++i) {
      const int u = lane_in_head + i * G, turning = HALF ? rot / (2 * V) : 0;
      if (HALF && u < turning) {
        off[i][0] = u * V;
        off[i][1] = rot / 2 + u * V;
        turn[i][0] = turn[i][1] = true;
        pair[i][0] = pair[i][1] = u * V;
      } else {
        const int r0 = HALF ? rot : 0, chunks = (d - r0) / V, apart = (chunks + 1) / 2, w = u - turning;
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          const int n = w + k * apart, o = r0 + n * V;
          off[i][k] = w < apart && n < chunks ? o : -1;
          turn[i][k] = !HALF && off[i][k] >= 0 && o < rot;
          pair[i][k] = o / 2;
        }
      }
    }
  }
};

// c, s of the V pairs of each unit; a position outside the table makes them NaN (nothing is read there).  A chunk's pairs lie side
// by side in the table's row: two pairs to a load.
template <int V, bool HALF, int NU>
__device__ __forceinline__ void load_table(const QkRopeArgs& a, const Units<V, HALF, NU>& un, int pos, float (&c)[NU][V], float (&s)[NU][V]) {
  typedef float f4 __attribute__((ext_vector_type(4), aligned(8)));
  constexpr int Q = HALF ? V : V / 2;   // pairs that turn or do not turn together
  const bool ok = pos >= 0 && pos < a.max_pos;
  const float2* const row = (const float2*)a.table + (long)(ok ? pos : 0) * (a.rot / 2);
  const float none = ok ? 0.f : __builtin_nanf("");
#pragma unroll
  for (int i = 0; i < NU; ++i)
#pragma unroll
    for (int q = 0; q < V; q += Q) {
#pragma unroll
      for (int e = q; e < q + Q; ++e) {
        c[i][e] = 1.f;
        s[i][e] = 0.f;
      }
      if (!un.turn[i][q / Q]) continue;
      const float2* const p = row + un.pair[i][q / Q];
#pragma unroll
      for (int e = 0; e < Q; e += 2) {
        if constexpr (Q >= 2) {
          const f4 x = *(const f4*)(p + e);
          c[i][q + e] = x[0] + none;
          s[i][q + e] = x[1] + none;
          c[i][q + e + 1] = x[2] + none;
          s[i][q + e + 1] = x[3] + none;
        } else {
          c[i][q] = p->x + none;
          s[i][q] = p->y + none;
        }
      }
    }
}

// the rotation of a unit (BACK: the other way round).  A column that does not turn is not touched: it may hold an infinity.
template <int V, bool HALF, bool BACK>
__device__ __forceinline__ void turn_unit(float (&x)[2][V], const float (&c)[V], const float (&s)[V], const bool (&turn)[2]) {
  if constexpr (HALF) {
    if (turn[0]) {
#pragma unroll
      for (int e = 0; e < V; ++e) {
        const float p = x[0][e], q = x[1][e], t = BACK ? -s[e] : s[e];
        x[0][e] = p * c[e] - q * t;
        x[1][e] = p * t + q * c[e];
      }
    }
  } else {
#pragma unroll
    for (int k = 0; k < 2; ++k)
      if (turn[k]) {
#pragma unroll
        for (int e = 0; e + 1 < V; e += 2) {
          const int j = (k * V + e) / 2;
          const float p = x[k][e], q = x[k][e + 1], t = BACK ? -s[j] : s[j];
          x[k][e] = p * c[j] - q * t;
          x[k][e + 1] = p * t + q * c[j];
        }
      }
  }
}

__device__ __forceinline__ int position_of(const QkRopeArgs& a, long row) {
  return a.positions ? a.positions[row] : a.seq > 0 ? (int)row % a.seq : (int)row;
}

// one row per wave, or `split` waves for the heads of a row where there are few rows
template <typename T, int V, bool HALF, int NU>
__global__ __launch_bounds__(256) void qk_rope_fwd_kernel(QkRopeArgs a, int G, int split) {
  const int lane = threadIdx.x & 63, per = 64 / G;
  const unsigned w = blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const long row = split > 1 ? w / split : w;
  const int part = split > 1 ? w % split : 0;
  if (row >= a.rows) return;
  Units<V, HALF, NU> un;
  un.init(a.d, a.rot, lane % G, G);
  float c[NU][V], s[NU][V];
  load_table<V, HALF, NU>(a, un, position_of(a, row), c, s);
  const float inv_d = 1.0f / (float)a.d;
#pragma unroll
  for (int t = 0; t < 2; ++t) {
    const int heads = t ? a.Ak : a.A;
    if (heads == 0) continue;
    const T *X = (const T*)(t ? a.k : a.q) + row * (t ? a.ldk : a.ldq), *gam = (const T*)(t ? a.gamma_k : a.gamma_q);
    T* Y = (T*)(t ? a.yk : a.yq) + row * (t ? a.ldyk : a.ldyq);
    float g[NU][2][V];
    if (gam) {
#pragma unroll
      for (int i = 0; i < NU; ++i)
#pragma unroll
        for (int k = 0; k < 2; ++k)
          if (un.off[i][k] >= 0) load_chunk<T, V>(gam + un.off[i][k], g[i][k]);
    }
    for (int h0 = part * per; h0 < heads; h0 += split * per) {
      const int h = h0 + lane / G;
      float x[NU][2][V], q = 0.f;
#pragma unroll
      for (int i = 0; i < NU; ++i)
#pragma unroll
        for (int k = 0; k < 2; ++k) {
#pragma unroll
          for (int e = 0; e < V; ++e) x[i][k][e] = 0.f;
          if (h < heads && un.off[i][k] >= 0) load_chunk<T, V>(X + h * a.d + un.off[i][k], x[i][k]);
        }
      if (gam) {
#pragma unroll
        for (int i = 0; i < NU; ++i)
#pragma unroll
          for (int k = 0; k < 2; ++k)
#pragma unroll
            for (int e = 0; e < V; ++e) q = fmaf(x[i][k][e], x[i][k][e], q);
        const float rstd = rsqrtf(group_sum(q, G) * inv_d + a.eps);
#pragma unroll
        for (int i = 0; i < NU; ++i)
#pragma unroll
          for (int k = 0; k < 2; ++k)
            if (un.off[i][k] >= 0) {
#pragma unroll
              for (int e = 0; e < V; ++e) x[i][k][e] = x[i][k][e] * rstd * g[i][k][e];
            }
      }
#pragma unroll
      for (int i = 0; i < NU; ++i) {
        turn_unit<V, HALF, false>(x[i], c[i], s[i], un.turn[i]);
#pragma unroll
        for (int k = 0; k < 2; ++k)
          if (h < heads && un.off[i][k] >= 0) store_chunk<T, V>(Y + h * a.d + un.off[i][k], x[i][k]);
      }
    }
  }
}

// Rows w, w + waves, ... per wave, all of them for the queries, then for the keys (in one walk the two gammas' sums would stand in
// registers side by side, and three waves of a SIMD in the place of four: 249 -> 209 us for 32768 rows, 32 + 8 heads of 128).  A lane's sums for dgamma stay in registers
// over all of its rows and heads; the workgroup's lanes of one unit are added in a fixed order, partial[block][q, k][d].
// Where a wave has one row, workgroups of their own take the keys (gridDim = 2 blocks): nothing but latencies would stand between
// the two walks (3001 rows, 12 + 4 heads of 64 in fp32 14.1 -> 11.2 us).
template <typename T, int V, bool HALF, int NU>
__global__ __launch_bounds__(256, V * NU <= 4 ? 1 : 4) void qk_rope_bwd_kernel(QkRopeArgs a, int G, int blocks, float* __restrict__ partial) {
  __shared__ float red[256][NU * 2 * V + 1];
  const int lane = threadIdx.x & 63, per = 64 / G;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  Units<V, HALF, NU> un;
  un.init(a.d, a.rot, lane % G, G);
  const float inv_d = 1.0f / (float)a.d;
  const bool norm = a.gamma_q != nullptr, apart = (int)gridDim.x > blocks;
  const int block = (int)blockIdx.x < blocks ? blockIdx.x : blockIdx.x - blocks;
#pragma unroll 1
  for (int t = (int)blockIdx.x < blocks ? 0 : 1; t < 2; ++t) {
    const int heads = t ? a.Ak : a.A;
    const long ldx = t ? a.ldk : a.ldq, lddy = t ? a.lddyk : a.lddyq, lddx = t ? a.lddk : a.lddq;
    const T *X = (const T*)(t ? a.k : a.q), *DY = (const T*)(t ? a.dyk : a.dyq), *gam = (const T*)(t ? a.gamma_k : a.gamma_q);
    T* DX = (T*)(t ? a.dk : a.dq);
    float g[NU][2][V], dg[NU][2][V];
#pragma unroll
    for (int i = 0; i < NU; ++i)
#pragma unroll
      for (int k = 0; k < 2; ++k) {
#pragma unroll
        for (int e = 0; e < V; ++e) dg[i][k][e] = g[i][k][e] = 0.f;
        if (norm && heads > 0 && un.off[i][k] >= 0) load_chunk<T, V>(gam + un.off[i][k], g[i][k]);
      }
    for (long row = (long)block * 4 + wave; heads > 0 && row < a.rows; row += (long)blocks * 4) {
      float c[NU][V], s[NU][V];
      load_table<V, HALF, NU>(a, un, position_of(a, row), c, s);
      for (int h0 = 0; h0 < heads; h0 += per) {
        const int h = h0 + lane / G;
        float x[NU][2][V], y[NU][2][V];
#pragma unroll
        for (int i = 0; i < NU; ++i)
#pragma unroll
          for (int k = 0; k < 2; ++k) {
#pragma unroll
            for (int e = 0; e < V; ++e) x[i][k][e] = y[i][k][e] = 0.f;
            if (h < heads && un.off[i][k] >= 0) {
              load_chunk<T, V>(DY + row * lddy + h * a.d + un.off[i][k], y[i][k]);
              if (norm) load_chunk<T, V>(X + row * ldx + h * a.d + un.off[i][k], x[i][k]);
            }
          }
#pragma unroll
        for (int i = 0; i < NU; ++i) turn_unit<V, HALF, true>(y[i], c[i], s[i], un.turn[i]);
        if (norm) {
          float q = 0.f, p = 0.f;
#pragma unroll
          for (int i = 0; i < NU; ++i)
#pragma unroll
            for (int k = 0; k < 2; ++k)
#pragma unroll
              for (int e = 0; e < V; ++e) {
                q = fmaf(x[i][k][e], x[i][k][e], q);
                p = fmaf(x[i][k][e], y[i][k][e] * g[i][k][e], p);
              }
          // (a head behind the last has no part in dgamma: its zeros with eps = 0 would be 0 times infinity)
          const float ms = group_sum(q, G) * inv_d + a.eps, rstd = h < heads ? rsqrtf(ms) : 0.f;
          const float m = group_sum(p, G) * inv_d * rstd;   // mean of dn gamma x rstd
#pragma unroll
          for (int i = 0; i < NU; ++i)
#pragma unroll
            for (int k = 0; k < 2; ++k)
#pragma unroll
              for (int e = 0; e < V; ++e) {
                const float xh = x[i][k][e] * rstd;
                dg[i][k][e] = fmaf(y[i][k][e], xh, dg[i][k][e]);
                y[i][k][e] = rstd * (y[i][k][e] * g[i][k][e] - xh * m);
              }
        }
#pragma unroll
        for (int i = 0; i < NU; ++i)
#pragma unroll
          for (int k = 0; k < 2; ++k)
            if (h < heads && un.off[i][k] >= 0) store_chunk<T, V>(DX + row * lddx + h * a.d + un.off[i][k], y[i][k]);
      }
    }
    if (!partial) {   // (no dgamma is wanted: the whole grid)
      if (apart) return;
      continue;
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < NU; ++i)
#pragma unroll
      for (int k = 0; k < 2; ++k)
#pragma unroll
        for (int e = 0; e < V; ++e) red[threadIdx.x][(i * 2 + k) * V + e] = dg[i][k][e];
    __syncthreads();
    // thread (u, j): value j of the lanes that hold the units u, u + G of a head
    for (int n = threadIdx.x; n < G * NU * 2 * V; n += 256) {
      const int u = n / (NU * 2 * V), j = n % (NU * 2 * V), i = j / (2 * V), k = j / V % 2, e = j % V;
      Units<V, HALF, NU> other;
      other.init(a.d, a.rot, u, G);
      float sum = 0.f;
      for (int r = u; r < 256; r += G) sum += red[r][j];
      const int off = i == 0 ? (k ? other.off[0][1] : other.off[0][0]) : (k ? other.off[NU - 1][1] : other.off[NU - 1][0]);
      if (off >= 0) partial[((long)block * 2 + t) * a.d + off + e] = sum;
    }
    if (apart) return;
  }
}

// dgamma from the workgroups' sums: 16 columns per workgroup, 64 slices of the blocks (every 64th, ascending), so that all of a
// lane's requests are in flight; the slices in a fixed order: the four of a wave by twos, then the waves
__global__ __launch_bounds__(1024) void qk_rope_dgamma_kernel(const float* __restrict__ partial, int blocks, int d, float* dgq, float* dgk,
                                                              int accumulate) {
  __shared__ float red[16][16];
  const int t = threadIdx.x & 15, slice = threadIdx.x >> 4, c = blockIdx.x * 16 + t;
  float s = 0.f;
  if (c < 2 * d) {
    float x[16];   // (at most 1024 blocks: see qk_rope_blocks)
#pragma unroll
    for (int u = 0; u < 16; ++u) x[u] = slice + 64 * u < blocks ? partial[(long)(slice + 64 * u) * 2 * d + c] : 0.f;
#pragma unroll
    for (int u = 0; u < 16; ++u) s += x[u];
  }
  s += __shfl_xor(s, 16, 64);
  s += __shfl_xor(s, 32, 64);
  if ((threadIdx.x & 63) < 16) red[threadIdx.x >> 6][t] = s;
  __syncthreads();
  if (threadIdx.x < 16 && c < 2 * d) {
    float r = red[0][t];
    for (int i = 1; i < 16; ++i) r += red[i][t];
    float* const out = c < d ? dgq : dgk;
    if (out) out[c < d ? c : c - d] = accumulate ? out[c < d ? c : c - d] + r : r;
  }
}

// [max_pos][pairs] of (cos, sin) of position * freq[pair], times a factor.  In 64 bits: a far position's angle has no
// digits to spare in 32.
struct RopeFreqs {
  double f[128];
};
__global__ void rope_table_kernel(RopeFreqs fr, float2* table, long n, int pairs, double magnitude) {
  const long i = (long)blockIdx.x * blockDim.x + threadIdx.x;
  if (i >= n) return;
  double s, c;
  sincos((double)(i / pairs) * fr.f[i % pairs], &s, &c);
  table[i] = make_float2((float)(c * magnitude), (float)(s * magnitude));
}

// ------------------------------------------------------------------ launchers
int qk_rope_blocks(long rows) {
  const long b = (rows + 3) / 4;
  return (int)(b < 1024 ? b : 1024);   // four workgroups to each of the 256 units
}

// The widest chunk that the columns' structure and every address allow, as f(V, HALF)
template <typename T, typename F>
static hipError_t pick_chunk(const QkRopeArgs& a, bool bwd, F&& f) {
  auto fits = [&](int v) {
    const int r = a.rot;
    if (a.d % v || r % v || (!a.interleaved && r / 2 % v)) return false;
    const long lds[] = {a.ldq, a.ldk, bwd ? a.lddyq : a.ldyq, bwd ? a.lddyk : a.ldyk, bwd ? a.lddq : 0, bwd ? a.lddk : 0};
    for (long l : lds)
      if (l % v) return false;
    const void* ps[] = {a.q, a.k, a.gamma_q, a.gamma_k, bwd ? a.dyq : a.yq, bwd ? a.dyk : a.yk, bwd ? a.dq : nullptr, bwd ? a.dk : nullptr};
    for (const void* p : ps)
      if ((uintptr_t)p % (v * sizeof(T))) return false;
    return true;
  };
  auto with = [&](auto V) {
    constexpr int v = decltype(V)::value;
    if constexpr (v > 1)
      if (a.interleaved) return f(V, std::false_type{});
    return f(V, std::true_type{});
  };
  if constexpr (sizeof(T) == 2)
    if (fits(8)) return with(std::integral_constant<int, 8>{});
  if (fits(4)) return with(std::integral_constant<int, 4>{});
  if (fits(2)) return with(std::integral_constant<int, 2>{});
  // (single columns: a pair is the two chunks of a unit.  Neighbours need chunks of two: see qk_rope_takes)
  return with(std::integral_constant<int, 1>{});
}
bool qk_rope_takes(Dtype dt, const QkRopeArgs& a, bool bwd) {
  int chunk = 0;
  auto see = [&](auto V, auto) {
    chunk = decltype(V)::value;
    return hipSuccess;
  };
  (void)(dt == DT_BF16 ? pick_chunk<bf16>(a, bwd, see) : pick_chunk<float>(a, bwd, see));
  return chunk > 1 || !a.interleaved;
}

template <typename F>
static hipError_t pick(Dtype dt, const QkRopeArgs& a, bool bwd, F&& f) {
  auto with = [&](auto t) {
    typedef decltype(t) T;
    return pick_chunk<T>(a, bwd, [&](auto V, auto HALF) {
      constexpr int v = decltype(V)::value, nu = v == 1 ? 2 : 1;
      const int turning = decltype(HALF)::value ? a.rot : 0, units = turning / (2 * v) + (a.d - turning + 2 * v - 1) / (2 * v);
      int G = 1;
      while (G * nu < units) G *= 2;
      if (G > 64) return hipErrorInvalidValue;   // (no head of up to 256 columns)
      return f(t, V, HALF, std::integral_constant<int, nu>{}, G);
    });
  };
  return dt == DT_BF16 ? with(bf16{}) : with(float{});
}

hipError_t launch_qk_rope_fwd(Dtype dt, const QkRopeArgs& a, hipStream_t st) {
  return pick(dt, a, false, [&](auto t, auto V, auto HALF, auto NU, int G) {
    const int per = 64 / G, passes = (a.A + per - 1) / per + (a.Ak + per - 1) / per;
    // 16 waves to each of the 256 units, where there are heads for them
    const int want = 1 + 4095 / a.rows;
    const int split = (int)(want < passes ? want : passes);
    const long waves = (long)a.rows * split;
    hipLaunchKernelGGL((qk_rope_fwd_kernel<decltype(t), decltype(V)::value, decltype(HALF)::value, decltype(NU)::value>),
                       dim3((unsigned)((waves + 3) / 4)), dim3(256), 0, st, a, G, split);
    return hipGetLastError();
  });
}

hipError_t launch_qk_rope_bwd(Dtype dt, const QkRopeArgs& a, float* partial, hipStream_t st) {
  const int blocks = qk_rope_blocks(a.rows);
  const bool sums = a.dgamma_q || a.dgamma_k;
  const hipError_t e = pick(dt, a, true, [&](auto t, auto V, auto HALF, auto NU, int G) {
    hipLaunchKernelGGL((qk_rope_bwd_kernel<decltype(t), decltype(V)::value, decltype(HALF)::value, decltype(NU)::value>), dim3(a.Ak > 0 && a.rows <= 4 * blocks ? 2 * blocks : blocks),
                       dim3(256), 0, st, a, G, blocks, sums ? partial : nullptr);
    return hipGetLastError();
  });
  if (e != hipSuccess || !sums) return e;
  hipLaunchKernelGGL(qk_rope_dgamma_kernel, dim3((2 * a.d + 15) / 16), dim3(1024), 0, st, partial, blocks, a.d, a.dgamma_q, a.dgamma_k,
                     a.accumulate);
  return hipGetLastError();
}

hipError_t launch_rope_table(float* table, int max_pos, int pairs, const double* freq, double magnitude, hipStream_t st) {
  RopeFreqs fr{};
  for (int i = 0; i < pairs; ++i) fr.f[i] = freq[i];
  const long n = (long)max_pos * pairs;
  hipLaunchKernelGGL(rope_table_kernel, dim3((unsigned)((n + 255) / 256)), dim3(256), 0, st, fr, (float2*)table, n, pairs, magnitude);
  return hipGetLastError();
}

}  // namespace dapple
