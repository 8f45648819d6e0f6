// The fp32 products of a gated feed-forward block, with its activation and the activation's gradient in their epilogues.
//
// Bound by the fp32 matrix rate, 256 flops per clock and unit: a fifteenth of the bf16 one, so neither LDS (a wave of 64x64 reads
// 4 KB for 16 instructions of 64 clocks) nor memory is near its rate and what costs is a matrix pipe that waits.  Hence a ring of
// k-tiles in LDS filled by loads that write LDS directly, three tiles ahead, and the next 8 of K read from LDS between the matrix
// instructions of these 8, also across a tile's barrier.  Of the time that a unit has a tile the pipes are busy: T = 4096, H = 1024, F = 4096
// gate and value 89%, output 85, dh 71, the last gradients 91 (1270 us, 130 TFLOP/s of the library's 148); T = 1000, H = 768, F = 2040, where
// a fifth of the time is the wait for a k-tile, 81, 70, 65, 79 -- and units have one 83, 61, 76, 86% of the launch.
#include <type_traits>
#include <utility>

#include "device_common.h"
#include "gemm_epilogue.h"
#include "kernels.h"

namespace dapple {

typedef int i32x4 __attribute__((ext_vector_type(4)));

template <int N, typename F>
__device__ __forceinline__ void unrolled(F&& f) {
  [&]<int... I>(std::integer_sequence<int, I...>) __attribute__((always_inline)) { (f(std::integral_constant<int, I>{}), ...); }
  (std::make_integer_sequence<int, N>{});
}

// C[M, N] = sum over k of A(m, k) B(n, k)
struct RingProduct {
  const float *A, *B, *bias, *aux;
  float *C, *C2, *bsum;   // bsum: the sums of B over k
  int M, N, K, lda, ldb, ldc;
  bool add, silu;         // add: C and bsum are added to
};

// One operand's [R x BK] k-tile in LDS and a wave's share of the requests that fill it, 1 KB each in lane order: the swizzle lies
// in WHICH 16 bytes a lane fetches.
//   k-contiguous: rows of BK floats, their 16-byte pieces XOR-swizzled so that 16 lanes reading a piece of 16 rows meet all banks;
//   k-strided: [BK][R], the columns of every other four rows XOR 32: a fragment's two half waves read rows 4 apart.
// Rows of the matrix past its end lie behind the buffer's record count and read as zero, so do k-strided rows past K; k-contiguous
// pieces past K are sent out of range.  (Columns past the end of a k-strided operand reach no stored element.)
template <int R, bool KS, int BK, int NW>
struct RingOperand {
  static constexpr int BYTES = R * BK * 4, PER = BYTES / 1024 / NW, CH = KS ? R / 4 : BK / 4;
  static_assert(PER * 1024 * NW == BYTES && R % 64 == 0 && (BK == 16 || BK == 32), "");
  unsigned voff[PER], live;   // live: bit i: piece i lies inside the last k-tile
  uint64_t next;
  long left, step;            // bytes from there to the operand's end; of a k-tile
  static __device__ __forceinline__ int swz(int r) { return BK == 16 ? (r >> 2) & 3 : (r >> 1) & 7; }
  // rows: of the matrix from the tile's first one on; k-strided: columns of the matrix from there; pair: F if the tile's columns are
  // 32 of the gate and the same 32 of the value by turns, else 0
  __device__ __forceinline__ void init(const float* first, int ld, long rows, int K, int pair, int wave, int lane) {
    const int tail = K - (K - 1) / BK * BK;
    live = 0;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const int at = (wave * PER + i) * 64 + lane, r = at / CH, c = at % CH;
      if (KS) {
        const int col = (c * 4) ^ ((r >> 2 & 1) << 5);
        voff[i] = 4u * (unsigned)(r * ld + (pair ? (col >> 6) * 32 + (col & 31) + (col & 32 ? pair : 0) : col));
        live |= 1u << i;
      } else {
        const int piece = c ^ swz(r);
        voff[i] = 4u * (unsigned)(r * ld + piece * 4);
        live |= piece * 4 < tail ? 1u << i : 0u;
      }
    }
    next = (uint64_t)first;
    step = 4L * BK * (KS ? ld : 1);
    left = 4L * (KS ? (long)(K - 1) * ld + rows : (rows - 1) * (long)ld + K);
  }
  // request piece i of the next k-tile into the stage at byte `to`; tiles: not yet requested.  Inline assembly and waits counted by
  // hand: the compiler would wait for all of them before any read of LDS.
  __device__ __forceinline__ void request(int i, int to, int wave, int tiles) {
    i32x4 rs;
    const long n = tiles > 0 ? (left < 0x7fffffff ? left : 0x7fffffff) : 0;
    rs[0] = __builtin_amdgcn_readfirstlane((int)(uint32_t)next);
    rs[1] = __builtin_amdgcn_readfirstlane((int)(uint32_t)(next >> 32));
    rs[2] = __builtin_amdgcn_readfirstlane((int)n);
    rs[3] = 0x00020000;   // raw buffer, 32-bit data format
    const int m = __builtin_amdgcn_readfirstlane(to + (wave * PER + i) * 1024);
    const unsigned v = !KS && tiles == 1 && !(live >> i & 1) ? 0x80000000u : voff[i];
    // (five wait states between a vector instruction that writes a scalar register and a memory instruction that reads it)
    asm volatile("s_nop 4\n\ts_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"s"(m), "v"(v), "s"(rs) : "memory", "m0");
  }
  __device__ __forceinline__ void advance() {
    next += step;
    left -= step;
  }
};

// LDS addresses of a lane's fragments: rows w0 + 32 b + (lane & 31), k = 8 kk + 4 (lane >> 5) + 0..3
template <int R, bool KS, int BK, int NB>
struct RingFrag {
  int a[KS ? NB : BK / 8];
  __device__ __forceinline__ void init(int w0, int lane) {
    const int r = lane & 31, h = lane >> 5;
    if (KS) {
#pragma unroll
      for (int b = 0; b < NB; ++b) a[b] = (4 * h * R + ((w0 + 32 * b + r) ^ (h << 5))) * 4;
    } else {
#pragma unroll
      for (int kk = 0; kk < BK / 8; ++kk) a[kk] = (w0 + r) * (BK * 4) + (((2 * kk + h) ^ RingOperand<R, KS, BK, 1>::swz(r)) << 4);
    }
  }
  template <int B, int KK>
  __device__ __forceinline__ f32x4 get(const unsigned char* tile) const {
    if (!KS) return *(const f32x4*)(tile + a[KK] + B * 32 * BK * 4);
    const unsigned char* p = tile + a[B] + KK * 8 * R * 4;
    return f32x4{*(const float*)p, *(const float*)(p + R * 4), *(const float*)(p + 2 * R * 4), *(const float*)(p + 3 * R * 4)};
  }
};

// WGM x WGN waves of MI x NI blocks of 32 x 32
template <int MI_, int NI_, int WGM_, int WGN_, int BK_, int NS_>
struct RingTile {
  static constexpr int MI = MI_, NI = NI_, WGM = WGM_, WGN = WGN_, BK = BK_, NS = NS_, NW = WGM * WGN, BM = 32 * MI * WGM, BN = 32 * NI * WGN;
  static constexpr int STAGE = (BM + BN) * BK * 4, LDS = NS * STAGE;
};
typedef RingTile<2, 2, 2, 2, 16, 4> Large;       // 128 x 128
typedef RingTile<1, 1, 2, 2, 32, 5> Small;       // 64 x 64
typedef RingTile<1, 2, 4, 2, 16, 4> LargeGate;   // the same rows and twice the columns, a wave holding a gate and its value: 128 x 128
typedef RingTile<1, 2, 2, 2, 32, 3> SmallGate;   // and 64 x 128.  (All: two workgroups to a unit.)

// GATE 1: B's columns are gate and value (N = F of each), C = act(gate) * value, C2 (may be NULL) the two, in [M, 2F]; 2: aux holds
// the two, C takes their gradients, the product being that of what act(gate) * value became.  CS: with bsum
template <typename T, bool AKS, bool BKS, int GATE, bool CS>
__device__ __forceinline__ void ring_tile(const RingProduct& g, int bid) {
  constexpr int MI = T::MI, NI = T::NI, BK = T::BK, NS = T::NS, SUB = MI * NI == 1 ? 2 : 1, STEPS = BK / 8 / SUB;   // a step: 8 of K, 16 where that were four products
  typedef RingOperand<T::BM, AKS, BK, T::NW> OA;
  typedef RingOperand<T::BN, BKS, BK, T::NW> OB;
  static_assert(GATE != 1 || NI % 2 == 0, "gate and value of a column belong to one wave");
  constexpr int BNC = GATE == 1 ? T::BN / 2 : T::BN, LOADS = OA::PER + OB::PER;
  extern __shared__ __attribute__((aligned(1024))) unsigned char smem[];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l31 = lane & 31, h = lane >> 5;
  const int wm0 = wave / T::WGN * 32 * MI, wn0 = wave % T::WGN * 32 * NI;
  int tm, tn;
  tile_of(bid, (g.M + T::BM - 1) / T::BM, (g.N + BNC - 1) / BNC, T::BM, T::BN, tm, tn);
  const int m0 = tm * T::BM, n0 = tn * BNC;
  OA oa;
  OB ob;
  oa.init(g.A + (AKS ? (long)m0 : (long)m0 * g.lda), g.lda, g.M - m0, g.K, 0, wave, lane);
  ob.init(g.B + (BKS ? (long)n0 : (long)n0 * g.ldb), g.ldb, (GATE == 1 ? 2 : 1) * g.N - n0, g.K, GATE == 1 ? g.N : 0, wave, lane);
  RingFrag<T::BM, AKS, BK, MI> fa;
  RingFrag<T::BN, BKS, BK, NI> fb;
  fa.init(wm0, lane);
  fb.init(wn0, lane);
  const int tiles = (g.K + BK - 1) / BK;
  int wanted = tiles, to = 0;   // not yet requested; the stage the next one goes to, in bytes
  auto request = [&](int e) __attribute__((always_inline)) {
    if (e < OA::PER) oa.request(e, to, wave, wanted);
    else ob.request(e - OA::PER, to + OA::BYTES, wave, wanted);
  };
  auto advance = [&]() __attribute__((always_inline)) {
    oa.advance();
    ob.advance();
    --wanted;
    to = to == (NS - 1) * T::STAGE ? 0 : to + T::STAGE;
  };
  f32x16 acc[MI][NI];
  float cs[NI];
#pragma unroll
  for (int j = 0; j < NI; ++j) {
    cs[j] = 0.f;
#pragma unroll
    for (int i = 0; i < MI; ++i)
#pragma unroll
      for (int v = 0; v < 16; ++v) acc[i][j][v] = 0.f;
  }
#pragma unroll
  for (int s = 0; s < NS - 1; ++s) {
#pragma unroll
    for (int e = 0; e < LOADS; ++e) request(e);
    advance();
  }
  // (the first step multiplies zeros)
  struct Frags {
    f32x4 a[SUB][MI], b[SUB][NI];
  } f0, f1;
#pragma unroll
  for (int s = 0; s < SUB; ++s) {
#pragma unroll
    for (int i = 0; i < MI; ++i) f1.a[s][i] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int j = 0; j < NI; ++j) f1.b[s][j] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  constexpr int NM = 4 * MI * NI * SUB, NF1 = MI + NI, NFRAG = NF1 * SUB, EXTRA = LOADS + 1;
  auto product = [&](const Frags& f, auto Q, auto WCS) __attribute__((always_inline)) {
    constexpr int q = decltype(Q)::value, s = q / (4 * MI * NI), e = q / (MI * NI) % 4, i = q / NI % MI, j = q % NI;
    // B first: a lane then owns 4 consecutive columns of one row
    acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x2f32(f.b[s][j][e], f.a[s][i][e], acc[i][j], 0, 0, 0);
    if constexpr (decltype(WCS)::value && i == 0) cs[j] += f.b[s][j][e];
  };
  // the products of `use`; behind the first ones the reads of `fill`, step J of the tile in LDS (a read takes the time of two or
  // three products), then a share of the requests
  auto step = [&](const Frags& use, Frags& fill, const unsigned char* S, auto J, auto WCS) __attribute__((always_inline)) {
    constexpr int j = decltype(J)::value, e0 = j * EXTRA / STEPS, P = NFRAG + (j + 1) * EXTRA / STEPS - e0;
    static_assert(P <= NM, "a piece behind each product");
    unrolled<NM>([&](auto Q) __attribute__((always_inline)) {
      constexpr int p = decltype(Q)::value;
      product(use, Q, WCS);
      __builtin_amdgcn_sched_barrier(0);
      if constexpr (p < NFRAG) {
        constexpr int s = p / NF1, f = p % NF1, kk = j * SUB + s;
        if constexpr (f == 0) fill.a[s][0] = fa.template get<0, kk>(S);
        else if constexpr (f <= NI) fill.b[s][f - 1] = fb.template get<f - 1, kk>(S + OA::BYTES);
        else fill.a[s][f - NI] = fa.template get<f - NI, kk>(S);
      } else if constexpr (p < P) {
        if constexpr (e0 + p - NFRAG < LOADS) request(e0 + p - NFRAG);
        else advance();
      }
      if constexpr (p < P) __builtin_amdgcn_sched_barrier(0);
    });
  };
  auto loop = [&](auto WCS) __attribute__((always_inline)) {
    int at = 0;
    for (int t = tiles; t > 0; --t) {
      constexpr int N = (NS - 2) * LOADS;
      static_assert(N < 64 && STEPS % 2 == 0, "vmcnt is a 6-bit counter; two sets of fragments");
      __builtin_amdgcn_sched_barrier(0);
      __builtin_amdgcn_s_waitcnt((N & 15) | ((N >> 4) << 14) | 0x0070);   // vmcnt(N), lgkmcnt(0)
      __builtin_amdgcn_s_barrier();   // every wave's part of this tile has landed, and the tile before has been read
      asm volatile("" ::: "memory");
      unrolled<STEPS / 2>([&](auto H) __attribute__((always_inline)) {
        constexpr int kk = 2 * decltype(H)::value;
        step(f1, f0, smem + at, std::integral_constant<int, kk>{}, WCS);
        step(f0, f1, smem + at, std::integral_constant<int, kk + 1>{}, WCS);
      });
      at = at == (NS - 1) * T::STAGE ? 0 : at + T::STAGE;
    }
    unrolled<NM>([&](auto Q) __attribute__((always_inline)) { product(f1, Q, WCS); });
  };
  const bool do_cs = CS && g.bsum && tm == 0 && wm0 == 0;
  if constexpr (CS) {   // (no branch inside the loop)
    if (do_cs) loop(std::true_type{});
    else loop(std::false_type{});
  } else {
    loop(std::false_type{});
  }
  __builtin_amdgcn_s_waitcnt(0x0F70);   // vmcnt(0): what the last requests wrote, zeros, must not meet a later workgroup's LDS
  if (do_cs) {
#pragma unroll
    for (int j = 0; j < NI; ++j) {
      const float t = cs[j] + __shfl_xor(cs[j], 32, 64);
      const int col = n0 + wn0 + 32 * j + l31;
      if (h == 0 && col < g.N) g.bsum[col] = g.add ? g.bsum[col] + t : t;
    }
  }
  // a 32x32 block's reads all before its first store: behind a store the compiler leaves a load where it stands
#pragma unroll
  for (int i = 0; i < MI; ++i) {
    const long row = m0 + wm0 + 32 * i + l31;
#pragma unroll
    for (int j = 0; j < NI; j += GATE == 1 ? 2 : 1) {
      const int col0 = n0 + (GATE == 1 ? (wn0 + 32 * j) / 2 : wn0 + 32 * j) + 4 * h;
      f32x4 x[4], y[4];
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const int col = col0 + 8 * q;
        x[q] = y[q] = f32x4{0.f, 0.f, 0.f, 0.f};
        if (row >= g.M || col >= g.N) continue;
        if constexpr (GATE == 2) {
          x[q] = *(const f32x4*)(g.aux + row * g.ldc + col);
          y[q] = *(const f32x4*)(g.aux + row * g.ldc + g.N + col);
        } else {
          if (g.bias) x[q] = *(const f32x4*)(g.bias + col);
          if (GATE == 1 && g.bias) y[q] = *(const f32x4*)(g.bias + g.N + col);
          if (GATE == 0 && g.add) x[q] = *(const f32x4*)(g.C + row * g.ldc + col);
        }
      }
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const int col = col0 + 8 * q;
        if (row >= g.M || col >= g.N) continue;
        f32x4 a = {acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]};
        float* const c = g.C + row * g.ldc + col;
        if constexpr (GATE == 0) {
          *(f32x4*)c = a + x[q];
        } else {
          f32x4 b;
          if constexpr (GATE == 1) {
            a += x[q];
            b = f32x4{acc[i][j + 1][4 * q], acc[i][j + 1][4 * q + 1], acc[i][j + 1][4 * q + 2], acc[i][j + 1][4 * q + 3]} + y[q];
            if (g.C2) {
              *(f32x4*)(g.C2 + row * 2 * g.N + col) = a;
              *(f32x4*)(g.C2 + row * 2 * g.N + g.N + col) = b;
            }
          }
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            float act, dact;
            gate_act(g.silu, GATE == 1 ? a[e] : x[q][e], act, dact);
            if constexpr (GATE == 1) {
              a[e] = act * b[e];
            } else {
              b[e] = a[e] * act;
              a[e] = a[e] * y[q][e] * dact;
            }
          }
          *(f32x4*)c = a;
          if constexpr (GATE == 2) *(f32x4*)(c + g.N) = b;
        }
      }
    }
  }
}

template <typename T, bool AKS, bool BKS, int GATE>
__global__ __launch_bounds__(64 * T::NW, 2) void ring_f32_kernel(RingProduct g) {
  ring_tile<T, AKS, BKS, GATE, false>(g, blockIdx.x);
}
// dx = [dg du] [Wg Wu]^T, its tiles from dx0 on, and the weights' gradients, in one launch: neither waits for the other, and alone
// each leaves units without a tile (T = 1000, H = 768, F = 2040: 97 + 75 + 55 us as launches of gemm_f32.hip, 165 together)
// Few tiles of many rows have their depth cut into parts, whose sums go to the workspace (T = 8000, H = 256, F = 512: 96 tiles in five
// parts 239 -> 145 us for the whole backward).
struct GradTasks {
  int dx0, ndx, nin, nout;   // tiles
  int parts, chunk;          // of the weights' depth
  float* partial;            // a part: dw_in, dw_out, db_in, db_out
};
template <typename T>
__global__ __launch_bounds__(64 * T::NW, 2) void ring_f32_grads(RingProduct dx, RingProduct in, RingProduct out, GradTasks w) {
  int b = blockIdx.x;
  if (b >= w.dx0 && b < w.dx0 + w.ndx) return ring_tile<T, false, false, 0, false>(dx, b - w.dx0);
  b -= b < w.dx0 ? 0 : w.ndx;
  const int per = w.nin + w.nout;
  auto run = [&](RingProduct& g, int tile, long at, long sum_at) __attribute__((always_inline)) {
    if (w.parts > 1) {
      const int part = b / per, k0 = part * w.chunk;
      float* const P = w.partial + part * ((long)in.M * in.N + (long)out.M * out.N + in.N + out.N);
      g.A += (long)k0 * g.lda;
      g.B += (long)k0 * g.ldb;
      g.K = min(w.chunk, g.K - k0);
      g.C = P + at;
      g.ldc = g.N;
      g.bsum = g.bsum ? P + sum_at : nullptr;
      g.add = false;
    }
    ring_tile<T, true, true, 0, true>(g, tile);
  };
  const long nw = (long)in.M * in.N, no = (long)out.M * out.N;
  if (b % per < w.nin) run(in, b % per, 0, nw + no);
  else run(out, b % per - w.nin, nw, nw + no + in.N);
}

// the parts' sums, in ascending order: [0, n0) of dw_in, then dw_out, db_in, db_out (sizes multiples of four; NULL: not wanted)
struct GradSums {
  float* to[4];
  long n[4];
};
__global__ __launch_bounds__(256) void ring_f32_join(const float* __restrict__ partial, int parts, GradSums s, bool add) {
  const long all = s.n[0] + s.n[1] + s.n[2] + s.n[3], i = ((long)blockIdx.x * 256 + threadIdx.x) * 4;
  if (i >= all) return;
  float* to = nullptr;
  long first = 0;
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    if (i >= first && i < first + s.n[k] && s.to[k]) to = s.to[k] + (i - first);
    first += s.n[k];
  }
  if (!to) return;
  f32x4 t = *(const f32x4*)(partial + i);
  for (int p = 1; p < parts; ++p) t += *(const f32x4*)(partial + p * all + i);
  *(f32x4*)to = add ? *(const f32x4*)to + t : t;
}


// ------------------------------------------------------------------ host side
static long tiles(long m, long n, int bm, int bn) { return ((m + bm - 1) / bm) * ((n + bn - 1) / bn); }

// 128-wide tiles: two for each unit, the fullest unit's not more work than with 64-wide ones.  T = 4096, H = 1024, F = 4096 the
// forward 812 us (64-wide: 830), the backward 1596 (1739); T = 2560, H = 2048, F = 1024 335 (280) and 674 (563), so not there.
static bool large(long t128, long t64) { return t128 >= 512 && 40 * ((t128 + 255) / 256) <= 11 * ((t64 + 255) / 256); }
static bool large(long m, long n, int twice) { return large(tiles(m, n, 128, 128 / twice), tiles(m, n, 64, 64 / twice)); }

template <auto KERN, typename T, typename... A>
static hipError_t launch(long blocks, hipStream_t st, A... a) {
  static const hipError_t rc = hipFuncSetAttribute((const void*)KERN, hipFuncAttributeMaxDynamicSharedMemorySize, T::LDS);
  if (rc != hipSuccess) return rc;
  hipLaunchKernelGGL(KERN, dim3((unsigned)blocks), dim3(64 * T::NW), T::LDS, st, a...);
  return hipGetLastError();
}
template <typename T, bool AKS, bool BKS, int GATE>
static hipError_t launch_one(const RingProduct& g, hipStream_t st) {
  return launch<ring_f32_kernel<T, AKS, BKS, GATE>, T>(tiles(g.M, g.N, T::BM, GATE == 1 ? T::BN / 2 : T::BN), st, g);
}
static hipError_t launch_dx(const RingProduct& g, hipStream_t st) {
  return large(g.M, g.N, 1) ? launch_one<Large, false, false, 0>(g, st) : launch_one<Small, false, false, 0>(g, st);
}
template <typename T>
static hipError_t launch_grads(const RingProduct& dx, const RingProduct& in, const RingProduct& out, GradTasks w, hipStream_t st) {
  w.ndx = dx.C ? (int)tiles(dx.M, dx.N, T::BM, T::BN) : 0;
  w.nin = (int)tiles(in.M, in.N, T::BM, T::BN);
  w.nout = (int)tiles(out.M, out.N, T::BM, T::BN);
  const long dw = (long)w.parts * (w.nin + w.nout);
  w.dx0 = dx.K > w.chunk ? 0 : (int)dw;   // (the deeper tiles first)
  return launch<ring_f32_grads<T>, T>(dw + w.ndx, st, dx, in, out, w);
}
// Fewer tiles than these have their K split over the waves of small ones (gemm_f32.hip).  (A lane's offset inside a tile has 32 bits.)
static bool enough(long t64, int ld0, int ld1) { return t64 >= 160 && ld0 <= 1 << 21 && ld1 <= 1 << 21; }

// parts of the weights' gradients' depth: 512 rows at least each, of tiles that leave the 256 units without two of them
static int grad_parts(const GatedFfnArgs& a) {
  const long w = tiles(a.H, 2L * a.F, 64, 64) + tiles(a.F, a.H, 64, 64), most = a.T / 512 < 16 ? a.T / 512 : 16, want = 512 / w;
  const long n = want < most ? want : most;
  if (n < 2) return 1;
  const int chunk = ((int)((a.T + n - 1) / n) + 31) / 32 * 32;
  return (a.T + chunk - 1) / chunk;
}
static int grad_chunk(const GatedFfnArgs& a, int parts) { return parts == 1 ? a.T : ((a.T + parts - 1) / parts + 31) / 32 * 32; }
int64_t gated_ffn_f32_workspace(const GatedFfnArgs& a) {
  const int parts = grad_parts(a);
  return parts == 1 ? 16 : 4L * parts * (3L * a.H * a.F + 2 * a.F + a.H);
}

RingPlan gated_ffn_f32_plan(const GatedFfnArgs& a) {
  const long t = tiles(a.T, a.H, 64, 64), w = grad_parts(a) * (tiles(a.H, 2L * a.F, 64, 64) + tiles(a.F, a.H, 64, 64));
  const int lw = 2 * a.F > a.H ? 2 * a.F : a.H, ly = a.ldx > a.lddy ? a.ldx : a.lddy;
  RingPlan p{};
  p.in = enough(tiles(a.T, 2L * a.F, 64, 64), a.ldx, lw);
  p.out = enough(t, lw, lw);
  p.dh = enough(tiles(a.T, a.F, 64, 64), a.lddy, lw);
  p.dx = a.dx && p.out;
  p.dw = a.dw_in && enough(w + (p.dx ? t : 0), ly, lw);
  return p;
}

hipError_t launch_ring_f32_in(const GatedFfnArgs& a, hipStream_t st) {
  RingProduct g{};
  g.A = (const float*)a.x; g.lda = a.ldx; g.B = (const float*)a.w_in; g.ldb = 2 * a.F; g.C = (float*)a.h; g.ldc = a.F; g.C2 = (float*)a.gu;
  g.bias = (const float*)a.b_in; g.M = a.T; g.N = a.F; g.K = a.H; g.silu = a.silu;
  return large(a.T, a.F, 2) ? launch_one<LargeGate, false, true, 1>(g, st) : launch_one<SmallGate, false, true, 1>(g, st);
}
hipError_t launch_ring_f32_out(const GatedFfnArgs& a, hipStream_t st) {
  RingProduct g{};
  g.A = (const float*)a.h; g.lda = a.F; g.B = (const float*)a.w_out; g.ldb = a.H; g.C = (float*)a.y; g.ldc = a.ldy; g.bias = (const float*)a.b_out;
  g.M = a.T; g.N = a.H; g.K = a.F;
  return large(a.T, a.H, 1) ? launch_one<Large, false, true, 0>(g, st) : launch_one<Small, false, true, 0>(g, st);
}
hipError_t launch_ring_f32_dh(const GatedFfnArgs& a, hipStream_t st) {
  RingProduct g{};
  g.A = (const float*)a.dy; g.lda = a.lddy; g.B = (const float*)a.w_out; g.ldb = a.H; g.aux = (const float*)a.gu; g.C = (float*)a.dgu; g.ldc = 2 * a.F;
  g.M = a.T; g.N = a.F; g.K = a.H; g.silu = a.silu;
  return large(a.T, a.F, 1) ? launch_one<Large, false, false, 2>(g, st) : launch_one<Small, false, false, 2>(g, st);
}
hipError_t launch_ring_f32_grads(const GatedFfnArgs& a, const RingPlan& p, void* workspace, hipStream_t st) {
  RingProduct dx{}, in{}, out{};
  if (p.dx) {
    dx.A = (const float*)a.dgu; dx.lda = 2 * a.F; dx.B = (const float*)a.w_in; dx.ldb = 2 * a.F; dx.C = (float*)a.dx; dx.ldc = a.lddx;
    dx.M = a.T; dx.N = a.H; dx.K = 2 * a.F;
  }
  if (!p.dw) return launch_dx(dx, st);
  in.A = (const float*)a.x; in.lda = a.ldx; in.B = (const float*)a.dgu; in.ldb = 2 * a.F; in.C = (float*)a.dw_in; in.ldc = 2 * a.F;
  in.bsum = (float*)a.db_in; in.M = a.H; in.N = 2 * a.F; in.K = a.T; in.add = a.accumulate;
  out.A = (const float*)a.h; out.lda = a.F; out.B = (const float*)a.dy; out.ldb = a.lddy; out.C = (float*)a.dw_out; out.ldc = a.H;
  out.bsum = (float*)a.db_out; out.M = a.F; out.N = a.H; out.K = a.T; out.add = a.accumulate;
  GradTasks w{};
  w.parts = grad_parts(a);
  w.chunk = grad_chunk(a, w.parts);
  w.partial = (float*)workspace;
  if (w.parts > 1) {
    hipError_t e = launch_grads<Small>(dx, in, out, w, st);
    if (e != hipSuccess) return e;
    const GradSums s{{in.C, out.C, in.bsum, out.bsum}, {(long)in.M * in.N, (long)out.M * out.N, in.N, out.N}};
    const long n = s.n[0] + s.n[1] + s.n[2] + s.n[3];
    hipLaunchKernelGGL(ring_f32_join, dim3((unsigned)((n / 4 + 255) / 256)), dim3(256), 0, st, w.partial, w.parts, s, in.add);
    return hipGetLastError();
  }
  // 128-wide tiles in two rounds at least, none deeper than an even share: T = 4096, H = 1024, F = 4096 1593 us, 64-wide ones 1720;
  // T = 2048 there 923, 858
  const long tdx = p.dx ? tiles(dx.M, dx.N, 128, 128) : 0, tdw = tiles(in.M, in.N, 128, 128) + tiles(out.M, out.N, 128, 128);
  const long deepest = dx.K > a.T ? dx.K : a.T;
  if (tdx + tdw >= 1024 && tdx * dx.K + tdw * a.T >= 512 * deepest) return launch_grads<Large>(dx, in, out, w, st);
  return launch_grads<Small>(dx, in, out, w, st);
}

}  // namespace dapple
