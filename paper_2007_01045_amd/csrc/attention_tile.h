// What the attention kernels share: blocks of bf16 rows in LDS and their ring, MFMA fragments, and the way of an output tile
// to memory (attention.hip, attention_window.hip); blocks of fp32 rows (attention_f32.hip, attention_window.hip).
#pragma once
#include "device_common.h"
#include "kernels.h"

namespace dapple {

static constexpr float LOG2E = 1.4426950408889634f;

// A 64 x D bf16 block sits in LDS as 64 rows of D/8 16-byte chunks, the chunks of row r XOR-swizzled by aswz(r).
// The same block is read two ways -- 128-bit reads along a row (16 lanes = 16 rows at a time) and transpose reads
// down the rows (32 lanes = 4 rows x 64 bytes at a time) -- and LDS has 64 four-byte banks, so either group must
// cover 256 distinct bytes modulo 256.
//   D = 64:  rows of equal parity need distinct chunks (a bijection of (r>>1)&7), and rows r and r+2 must land in
//            different 64-byte halves (bit 2 of the swizzle = bit 1 of r): (r>>1)&7 rotated right by one gives both.
//   D = 128: 16 rows need 16 distinct chunks and 4 neighbouring rows four distinct 64-byte quarters: the two halves
//            of r & 15 swapped.
//   D = 32:  four rows fill 256 bytes; rows r, r+4, r+8, r+12 need distinct chunks: (r>>2)&3.
template <int D>
__device__ __forceinline__ int aswz(int r) {
  if (D == 64) {
    int x = (r >> 1) & 7;
    return ((x & 1) << 2) | (x >> 1);
  }
  if (D == 128) return ((r & 3) << 2) | ((r >> 2) & 3);
  return (r >> 2) & 3;
}

// The streamed side: blocks of 64 rows of two matrices X and Y (keys and values; queries and output gradients) go
// through a ring of NS blocks in LDS, requested NS - 1 blocks ahead with loads that write LDS directly.  (Through
// registers, one block ahead, every block waited for memory: a block's arithmetic is about 0.6 us, a request takes
// longer.)  1 KiB per wave instruction in lane order, so the swizzle is applied to WHICH chunk a lane fetches; rows
// past the end lie beyond the buffer's record count and read as zero, columns past d get an offset out of range.
// A wave owns PER consecutive instructions of one of the two matrices.  ROWS: of a block.
typedef int i32x4 __attribute__((ext_vector_type(4)));
template <int D, int NW, int NS_, bool STATS, int ROWS = 64>
struct Ring {
  static constexpr int NS = NS_, IPM = D * ROWS / 512, PER = 2 * IPM / NW; // instructions per matrix and block; per wave
  static constexpr int Y_OFF = ROWS * D * 2, S_OFF = 2 * Y_OFF;            // X, Y, then rows of 64 fp32 (STATS)
  static constexpr int SROWS = NW > 4 ? NW : 4, STAGE = S_OFF + (STATS ? SROWS * 256 : 0), BYTES = NS * STAGE;
  static constexpr int SPW = STATS ? SROWS / NW : 0;   // rows of the statistics per wave
  static constexpr int BIAS = 3 * 1024, LOADS = PER + SPW;
  static_assert(PER <= IPM && (PER == 2 || PER % 4 == 0), "a wave's share lies in one matrix");
  static_assert((NS - 2) * LOADS < 64, "vmcnt is a 6-bit counter");
  int voff[PER];
  i32x4 rs, st[SPW ? SPW : 1];   // buffer resources: the wave's matrix; its rows of the statistics
  int step, left, left0, sleft[SPW ? SPW : 1], m0w, m0s;
  uint64_t base0, stat0[SPW ? SPW : 1];
  // g: the wave's matrix (head's first column of row 0); ld in elements; stat(r): row r of the statistics, fp32 per row
  // of X and Y, or NULL (reads zero)
  template <typename F>
  __device__ __forceinline__ void init(const bf16* g, int ld, int s, int d, int wave, int lane, F&& stat) {
#pragma unroll
    for (int j = 0; j < PER; ++j) {
      const int pos = ((wave * PER + j) % IPM) * 64 + lane, r = pos / (D / 8), c = (pos % (D / 8)) ^ aswz<D>(r);
      voff[j] = c * 8 < d ? (r * ld + c * 8) * 2 + BIAS - (j % 4) * 1024 : (int)0x80000000;
    }
    set(rs, (uint64_t)g - BIAS);
    step = ROWS * ld * 2;
    left = left0 = ((s - 1) * ld + d) * 2;
    base0 = (uint64_t)g - BIAS;
    m0w = __builtin_amdgcn_readfirstlane(wave * PER * 1024);
#pragma unroll
    for (int i = 0; i < SPW; ++i) {
      const float* p = stat(wave + NW * i);
      stat0[i] = (uint64_t)p;
      set(st[i], (uint64_t)p);
      sleft[i] = p ? s * 4 : 0;
    }
    m0s = __builtin_amdgcn_readfirstlane(S_OFF + wave * 256);
  }
  static __device__ __forceinline__ void set(i32x4& r, uint64_t p) {
    r[0] = __builtin_amdgcn_readfirstlane((int)(uint32_t)p);
    r[1] = __builtin_amdgcn_readfirstlane((int)(uint32_t)(p >> 32));
    r[3] = 0x00020000;   // raw buffer, 32-bit data format
  }
  // request the next block into stage `stage`.  Inline assembly, and the waits counted by hand, for the reasons given
  // at OperandTile::load_group in gemm_mfma.h (which also has the wait states).
  __device__ __forceinline__ void request(int stage, int lane) {
    const int base = __builtin_amdgcn_readfirstlane(stage * STAGE);
    rs[2] = __builtin_amdgcn_readfirstlane(left > 0 ? left + BIAS : 0);
    const int mw = __builtin_amdgcn_readfirstlane(base + m0w);
    if constexpr (PER == 2) {
      asm volatile(
          "s_nop 4\n\ts_mov_b32 m0, %0\n\ts_nop 0\n\t"
          "buffer_load_dwordx4 %1, %3, 0 offen lds\n\t"
          "buffer_load_dwordx4 %2, %3, 0 offen offset:1024 lds"
          :
          : "s"(mw), "v"(voff[0]), "v"(voff[1]), "s"(rs)
          : "memory", "m0");
    } else {
#pragma unroll
      for (int j = 0; j < PER; j += 4)
        asm volatile(
            "s_nop 4\n\ts_add_u32 m0, %0, %1\n\ts_nop 0\n\t"
            "buffer_load_dwordx4 %2, %6, 0 offen lds\n\t"
            "buffer_load_dwordx4 %3, %6, 0 offen offset:1024 lds\n\t"
            "buffer_load_dwordx4 %4, %6, 0 offen offset:2048 lds\n\t"
            "buffer_load_dwordx4 %5, %6, 0 offen offset:3072 lds"
            :
            : "s"(mw), "s"(j * 1024), "v"(voff[j]), "v"(voff[j + 1]), "v"(voff[j + 2]), "v"(voff[j + 3]), "s"(rs)
            : "memory", "m0", "scc");
    }
#pragma unroll
    for (int i = 0; i < SPW; ++i) {
      st[i][2] = __builtin_amdgcn_readfirstlane(sleft[i] > 0 ? sleft[i] : 0);
      const int ms = __builtin_amdgcn_readfirstlane(base + m0s + i * NW * 256);
      const int off = lane * 4;
      asm volatile(
          "s_nop 4\n\ts_mov_b32 m0, %0\n\ts_nop 0\n\t"
          "buffer_load_dword %1, %2, 0 offen lds"
          :
          : "s"(ms), "v"(off), "s"(st[i])
          : "memory", "m0");
      set(st[i], (((uint64_t)(uint32_t)st[i][1] << 32) | (uint32_t)st[i][0]) + 4 * ROWS);
      sleft[i] -= 4 * ROWS;
    }
    set(rs, (((uint64_t)(uint32_t)rs[1] << 32) | (uint32_t)rs[0]) + (uint64_t)step);
    left -= step;
  }
  // the next block requested is the first one again
  __device__ __forceinline__ void rewind(int s) {
    set(rs, base0);
    left = left0;
#pragma unroll
    for (int i = 0; i < SPW; ++i) {
      set(st[i], stat0[i]);
      sleft[i] = stat0[i] ? s * 4 : 0;
    }
  }
  // the next block requested is block `block`, col_bytes to the right (another head), its statistics stat_bytes further on
  __device__ __forceinline__ void seek(int block, int s, int col_bytes, long stat_bytes) {
    set(rs, base0 + (uint64_t)((long)block * step + col_bytes));
    left = left0 - block * step;
#pragma unroll
    for (int i = 0; i < SPW; ++i) {
      set(st[i], stat0[i] + (uint64_t)(stat_bytes + block * (4L * ROWS)));
      sleft[i] = stat0[i] ? s * 4 - block * (4 * ROWS) : 0;
    }
  }
  // what is requested from here on reads nothing
  __device__ __forceinline__ void stop() {
    left = 0;
#pragma unroll
    for (int i = 0; i < SPW; ++i) sleft[i] = 0;
  }
  // every wave's part of the oldest block is in LDS, and every wave is done with the block before it.  MORE: requests of
  // this wave's besides the ring's, issued since the one that is waited for
  template <int MORE = 0>
  static __device__ __forceinline__ void wait() {
    constexpr int N = (NS - 2) * LOADS + MORE;
    static_assert(N < 64, "vmcnt is a 6-bit counter");
    __builtin_amdgcn_sched_barrier(0);
    __builtin_amdgcn_s_waitcnt((N & 15) | ((N >> 4) << 14) | 0x0070);   // vmcnt(N), lgkmcnt(0)
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
  }
};
// operand fragment, contraction index contiguous in LDS: rows r0 + (lane&31), k = 16 kk + 8 (lane>>5) + e
template <int D>
__device__ __forceinline__ bf16x8 frag_rows(const bf16* S, int r0, int kk, int lane) {
  int r = r0 + (lane & 31), kc = kk * 2 + (lane >> 5);
  return *(const bf16x8*)(S + r * D + ((kc ^ aswz<D>(r)) << 3));
}
// operand fragment, contraction index along LDS rows: column c0 + (lane&31); element e < 4 is
// LDS row k0 + 4 (lane>>5) + e, element 4 + e is LDS row k0 + 8 + 4 (lane>>5) + e -- the order
// in which a 32x32 accumulator hands its rows to a lane
template <int D>
__device__ __forceinline__ bf16x8 frag_cols(const bf16* S, int c0, int k0, int lane) {
  int i16 = lane & 15, g16 = (lane >> 4) & 1, h = lane >> 5;
  int r = k0 + 4 * h + (i16 >> 2);
  int col = c0 + 16 * g16 + 4 * (i16 & 3);
  const bf16* p0 = S + r * D + (((col >> 3) ^ aswz<D>(r)) << 3) + (col & 7);
  const bf16* p1 = S + (r + 8) * D + (((col >> 3) ^ aswz<D>(r + 8)) << 3) + (col & 7);
  return join8(lds_read_tr16(p0), lds_read_tr16(p1));
}
// global fragment of a row the wave owns: row r (or zeros), k = 16 kk + 8 (lane>>5) + e
template <bool RAG>
__device__ __forceinline__ bf16x8 frag_global(const bf16* base, long row, bool ok, int ld, int kk, int lane, int d) {
  const int k = kk * 16 + 8 * (lane >> 5);
  if (!ok || (RAG && k >= d)) {
    bf16x8 z;
#pragma unroll
    for (int e = 0; e < 8; ++e) z[e] = (bf16)0.f;
    return z;
  }
  return *(const bf16x8*)(base + row * ld + k);
}
// accumulator rows 16 ks .. 16 ks + 15 of a 32-row block, as the k-permuted operand
__device__ __forceinline__ bf16x8 acc_to_operand(const float (&p)[16], int ks) {
  bf16x8 f;
#pragma unroll
  for (int e = 0; e < 8; ++e) f[e] = (bf16)p[8 * ks + e];
  return f;
}
// two fp32 values as bf16 in one register, and what rounding left of them (the differences are exact)
typedef __attribute__((__vector_size__(2 * sizeof(float)))) float f32x2;
__device__ __forceinline__ unsigned take_bf16(float& a, float& b) {
  const unsigned u = __builtin_bit_cast(unsigned, __builtin_convertvector(f32x2{a, b}, bf16x2));
  a -= __builtin_bit_cast(float, u << 16);
  b -= __builtin_bit_cast(float, u & 0xffff0000u);
  return u;
}
// accumulator rows 16 ks .. 16 ks + 15 as a sum of three such operands.  (Pair by pair in whole registers: element by
// element the compiler converts every value once to pack it and once more to subtract it: the last of the stages above 0.673 ms.)
__device__ __forceinline__ void acc_to_operands(const float (&p)[16], int ks, bf16x8& hi, bf16x8& mid, bf16x8& lo) {
  typedef unsigned u32x4 __attribute__((__vector_size__(4 * sizeof(unsigned))));
  u32x4 h, m, l;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    float a = p[8 * ks + 2 * e], b = p[8 * ks + 2 * e + 1];
    h[e] = take_bf16(a, b);
    m[e] = take_bf16(a, b);
    l[e] = __builtin_bit_cast(unsigned, __builtin_convertvector(f32x2{a, b}, bf16x2));
  }
  hi = __builtin_bit_cast(bf16x8, h);
  mid = __builtin_bit_cast(bf16x8, m);
  lo = __builtin_bit_cast(bf16x8, l);
}

#define MFMA(a, b, c) __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0)

// max / sum of the two half waves' values (a row's 64 keys sit in lanes l and l + 32), in both; v_permlane32_swap is an
// ordinary vector instruction where a shuffle is a trip through the LDS crossbar
__device__ __forceinline__ float halves_max(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(unsigned, x), __builtin_bit_cast(unsigned, x), false, false);
  return fmaxf(__builtin_bit_cast(float, (unsigned)r[0]), __builtin_bit_cast(float, (unsigned)r[1]));
}
__device__ __forceinline__ float halves_sum(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(unsigned, x), __builtin_bit_cast(unsigned, x), false, false);
  return __builtin_bit_cast(float, (unsigned)r[0]) + __builtin_bit_cast(float, (unsigned)r[1]);
}

__device__ __forceinline__ f32x16 zero16() {
  f32x16 z;
#pragma unroll
  for (int v = 0; v < 16; ++v) z[v] = 0.f;
  return z;
}

// A wave's 32 rows x 32 NDB columns of an output (t: rows = columns of the head, column = the lane's row) times f, through a
// piece of LDS of the wave's own into whole rows: straight from the accumulators a store is 16 bytes (32 of an fp32 copy)
// of each of 32 rows, and the L2 takes every line in eight pieces.  rows: valid rows; d: columns of the head.
// C32 (may be NULL): an fp32 copy; FAR: it is not read again soon enough to be kept in a cache (see store_c in gemm_mfma.h).
template <int NDB, bool FAR = false>
struct OutTile {
  static constexpr int W = 32 * NDB, LD = W + 4, BYTES = 32 * LD * 4;
  static constexpr int RS = 64 / (W / 4);   // rows per instruction
  // Vector stores of C by a wave whose 32 rows and W columns are all valid, C32 aside.  A caller's wait may count on as many
  // behind an older request: one instruction per RS rows, and no way past it.
  static constexpr int STORES = 32 / RS;
  static __device__ __forceinline__ void store(float* S, const f32x16* t, float f, bf16* C, float* C32, long ld, int rows, int d, int lane) {
#pragma unroll
    for (int db = 0; db < NDB; ++db)
#pragma unroll
      for (int blk = 0; blk < 4; ++blk)
        *(f32x4*)(S + (lane & 31) * LD + db * 32 + 8 * blk + 4 * (lane >> 5)) =
            f32x4{t[db][4 * blk], t[db][4 * blk + 1], t[db][4 * blk + 2], t[db][4 * blk + 3]} * f;
    __builtin_amdgcn_wave_barrier();   // (private to the wave, whose LDS accesses execute in order)
    const int r = lane / (W / 4), c = lane % (W / 4) * 4;
#pragma unroll
    for (int u = 0; u < STORES; ++u) {
      const int i = u * RS;
      const f32x4 v = *(const f32x4*)(S + (i + r) * LD + c);
      if (i + r < rows && c < d) {
        bf16x4 o;
#pragma unroll
        for (int e = 0; e < 4; ++e) o[e] = (bf16)v[e];
        *(bf16x4*)(C + (i + r) * ld + c) = o;
        if (C32) {
          if (FAR) __builtin_nontemporal_store(v, (f32x4*)(C32 + (i + r) * ld + c));
          else *(f32x4*)(C32 + (i + r) * ld + c) = v;
        }
      }
    }
    __builtin_amdgcn_wave_barrier();
  }
};

// ------------------------------------------------------------------ fp32 blocks
#define MFMA4(a, b, c) __builtin_amdgcn_mfma_f32_16x16x4f32(a, b, c, 0, 0, 0)

// D: the head block's width (16, 32, 64 or 128; narrower heads are padded with zeros); blocks of 32 rows
constexpr int BR = 32;
// T: threads that move a block
template <int D, int T = 256>
struct F32Block {
  // row stride D + 8 floats: the four lane groups of a 4-byte read lie 4 rows = 32 banks (mod 64) apart
  static constexpr int LD = D + 8, CPR = D / 4, N = BR * CPR / T > 0 ? BR * CPR / T : 1;
  f32x4 c[N];
  __device__ __forceinline__ void load(const float* g, int ldg, int tid, int rows, int d) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int p = tid + T * i, r = p / CPR, k = p % CPR * 4;
      c[i] = f32x4{0.f, 0.f, 0.f, 0.f};
      if (p < BR * CPR && r < rows && k < d) c[i] = *(const f32x4*)(g + (long)r * ldg + k);
    }
  }
  __device__ __forceinline__ void store(float* S, int tid) const {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int p = tid + T * i;
      if (p < BR * CPR) *(f32x4*)(S + p / CPR * LD + p % CPR * 4) = c[i];
    }
  }
};
// row r0 + (lane & 15), k = 16 kk + 4 (lane >> 4) + 0..3
template <int D>
__device__ __forceinline__ f32x4 frow(const float* S, int r0, int kk, int lane) {
  return *(const f32x4*)(S + (r0 + (lane & 15)) * (D + 8) + 16 * kk + 4 * (lane >> 4));
}
// column c0 + (lane & 15) of row r0 + 4 (lane >> 4) + e
template <int D>
__device__ __forceinline__ float fcol(const float* S, int c0, int r0, int e, int lane) {
  return S[(r0 + 4 * (lane >> 4) + e) * (D + 8) + c0 + (lane & 15)];
}
// the row a lane owns in registers, k = 16 kk + 4 (lane >> 4) + 0..3
template <int D>
__device__ __forceinline__ void own_row(const float* row, bool ok, int d, int lane, f32x4 (&f)[D / 16]) {
#pragma unroll
  for (int kk = 0; kk < D / 16; ++kk) {
    const int k = 16 * kk + 4 * (lane >> 4);
    f[kk] = f32x4{0.f, 0.f, 0.f, 0.f};
    if (ok && k < d) f[kk] = *(const f32x4*)(row + k);
  }
}
__device__ __forceinline__ float over_groups_sum(float v) {   // the four lanes of one owned row, pairs first
  v += __shfl_xor(v, 16, 64);
  return v + __shfl_xor(v, 32, 64);
}

}  // namespace dapple
