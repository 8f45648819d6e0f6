// Embedding, forward and backward:  y[r] = scale table[id[r]],  dtable[v] = scale * sum of dy[r] over the rows r with id[r] = v, in
// an order that depends on the sizes and ids alone.  An id outside [0, V) reads nothing: its row of y is zero and it has no gradient.
//
// Forward: a copy, bound by memory.  Backward: the rows are sorted by id (stable: a row's place among those of its id is its order),
// so that an id's rows lie one behind the other, and every row of dy is read once and every row of dtable written once, without atomics
// on values.  The sort is one of least significant digits first, of at most nine bits: per digit a count and a placing, each
// workgroup a run of the rows.  Sums: a wave takes a run of the sorted rows and 512 columns; an id whose rows lie in one run is stored,
// of one that goes on in the next runs each leaves its part, and a second kernel adds the parts in ascending order.
#include <algorithm>

#include "kernels.h"
#include "row_chunks.h"

namespace dapple {

// ------------------------------------------------------------------ forward
template <typename T>
__global__ __launch_bounds__(256) void embed_fwd(EmbeddingArgs a, int chunks) {
  const long all = (long)a.rows * chunks, stride = (long)gridDim.x * 256;
  for (long i = (long)blockIdx.x * 256 + threadIdx.x; i < all; i += stride) {
    const long row = all < (1L << 31) ? (long)((uint32_t)i / (uint32_t)chunks) : i / chunks;
    const int col = (int)(i - row * chunks) * 8, id = a.ids[row];
    float v[8];
    if (id >= 0 && id < a.V) {
      load8((const T*)a.table + (long)id * a.ldt + col, a.H - col, v);
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] *= a.scale;
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = 0.f;
    }
    store8((T*)a.y + row * a.ldy + col, a.H - col, v);
  }
}

// ------------------------------------------------------------------ sort
constexpr int DIGITS = 512, SORT_T = 1024, SUM_ROWS = 16;

// key of sorted place i, V (no token's) behind the last; ids outside the table come last
__device__ __forceinline__ uint32_t key_of(int id, int V) { return id < 0 || id > V ? (uint32_t)V : (uint32_t)id; }

// counts[workgroup][digit] of the workgroups' rows.  T: the workgroups behind them clear dtable, of that type
template <typename T, bool FIRST>
__global__ __launch_bounds__(SORT_T) void embed_count(EmbeddingArgs a, EmbedPlan p, const uint32_t* keys, int shift) {
  __shared__ uint32_t hist[DIGITS];
  const int tid = threadIdx.x;
  if ((int)blockIdx.x >= p.wgs) {
    const bool dense = a.lddt == a.H;   // one row
    const long cols = dense ? (long)a.V * a.H : a.H, chunks = (cols + 7) / 8, all = dense ? chunks : a.V * chunks;
    const float zero[8] = {};
    for (long i = (long)(blockIdx.x - p.wgs) * SORT_T + tid; i < all; i += (long)(gridDim.x - p.wgs) * SORT_T) {
      const long row = dense ? 0 : i / chunks, col = (i - row * chunks) * 8;
      store8((T*)a.dtable + row * a.lddt + col, (int)min(8L, cols - col), zero);
    }
    return;
  }
  if (tid < DIGITS) hist[tid] = 0;
  __syncthreads();
  const int first = blockIdx.x * p.per, end = min(a.rows, first + p.per);
  for (int i = first + tid; i < end; i += SORT_T) {
    const uint32_t k = FIRST ? key_of(a.ids[i], a.V) : keys[i];
    atomicAdd(&hist[(k >> shift) & (DIGITS - 1) & ((1u << p.bits) - 1)], 1u);
  }
  __syncthreads();
  if (tid < DIGITS) p.counts[(long)blockIdx.x * DIGITS + tid] = hist[tid];
}

template <bool FIRST>
__global__ __launch_bounds__(SORT_T) void embed_place(EmbeddingArgs a, EmbedPlan p, const uint32_t* keys, const uint32_t* rows, uint32_t* keys_out,
                                                      uint32_t* rows_out, int shift) {
  constexpr int NWV = SORT_T / 64;
  __shared__ uint32_t base[DIGITS], part[2][2][DIGITS], run[DIGITS / 64];
  __shared__ uint16_t of_wave[NWV][DIGITS];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, digit = tid & (DIGITS - 1), half = tid >> 9;
  {   // rows of a digit in the workgroups before this one, and in all: half of the workgroups to a thread
    uint32_t before = 0, total = 0;
    const int w0 = half * ((p.wgs + 1) / 2), w1 = half ? p.wgs : (p.wgs + 1) / 2;
#pragma unroll 8
    for (int w = w0; w < w1; ++w) {
      const uint32_t c = p.counts[(long)w * DIGITS + digit];
      before += w < (int)blockIdx.x ? c : 0;
      total += c;
    }
    part[half][0][digit] = before;
    part[half][1][digit] = total;
  }
  __syncthreads();
  uint32_t total = 0, upto = 0;
  if (tid < DIGITS) {   // the digits' first places: sums of the totals before them
    total = part[0][1][tid] + part[1][1][tid];
    upto = total;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const uint32_t v = __shfl_up(upto, o, 64);
      if (lane >= o) upto += v;
    }
    if (lane == 63) run[wave] = upto;
  }
  for (int i = tid; i < NWV * DIGITS; i += SORT_T) (&of_wave[0][0])[i] = 0;
  __syncthreads();
  if (tid < DIGITS) {
    uint32_t b = upto - total + part[0][0][tid] + part[1][0][tid];
    for (int w = 0; w < wave; ++w) b += run[w];
    base[tid] = b;
  }
  __syncthreads();
  const int first = blockIdx.x * p.per, end = min(a.rows, first + p.per);
  for (int i0 = first; i0 < end; i0 += SORT_T) {
    const int i = i0 + tid;
    const bool in = i < end;
    const uint32_t k = in ? (FIRST ? key_of(a.ids[i], a.V) : keys[i]) : 0;
    const uint32_t r = FIRST ? (uint32_t)i : (in ? rows[i] : 0);
    const uint32_t d = (k >> shift) & ((1u << p.bits) - 1);
    unsigned long long same = __ballot(in);   // the wave's rows of this lane's digit
    for (int b = 0; b < p.bits; ++b) {
      const unsigned long long m = __ballot((d >> b) & 1);
      same &= (d >> b) & 1 ? m : ~m;
    }
    const int mine = __builtin_popcountll(same & ((1ull << lane) - 1));
    if (in && mine == 0) of_wave[wave][d] = (uint16_t)__builtin_popcountll(same);
    __syncthreads();
    if (in) {
      uint32_t at = base[d] + mine;
      for (int w = 0; w < wave; ++w) at += of_wave[w][d];
      keys_out[at] = k;
      rows_out[at] = r;
    }
    __syncthreads();
    if (tid < DIGITS) {
      uint32_t n = 0;
#pragma unroll
      for (int w = 0; w < NWV; ++w) {
        n += of_wave[w][tid];
        of_wave[w][tid] = 0;
      }
      base[tid] += n;
    }
    __syncthreads();
  }
}

// ------------------------------------------------------------------ sums
template <typename T>
__device__ __forceinline__ void store_sum(const EmbeddingArgs& a, uint32_t id, int col, const float (&s)[8]) {
  float o[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) o[e] = s[e] * a.scale;
  if (a.accumulate) {
    float* const D = (float*)a.dtable + (long)id * a.lddt + col;
    float v[8];
    load8(D, a.H - col, v);
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] += o[e];
    store8(D, a.H - col, v);
  } else {
    store8((T*)a.dtable + (long)id * a.lddt + col, a.H - col, o);
  }
}

// One wave: sorted rows [run p.run, ...) and 512 columns from 512 slab on.  parts[run][0]: of an id that began before the run, [1]: of one
// that begins in it and goes on behind it
template <typename T>
__global__ __launch_bounds__(64) void embed_sum(EmbeddingArgs a, EmbedPlan p, const uint32_t* keys, const uint32_t* rows) {
  const int lane = threadIdx.x;
  for (long u = blockIdx.x; u < (long)p.runs * p.slabs; u += gridDim.x) {
    const int run = (int)(u / p.slabs), col = ((int)(u % p.slabs) * 64 + lane) * 8;
    const int first = run * p.run, end = min(a.rows, first + p.run);
    if (keys[first] >= (uint32_t)a.V) continue;
    const uint32_t ahead = first ? keys[first - 1] : 0xffffffffu, behind = end < a.rows ? keys[end] : 0xffffffffu;
    bool begun = ahead == keys[first];   // the current id began before the run
    float acc[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) acc[e] = 0.f;
    auto part = [&](int which) {
      if (col < a.H) store8(p.parts + ((long)run * 2 + which) * a.H + col, a.H - col, acc);
    };
    for (int i0 = first; i0 < end; i0 += SUM_ROWS) {
      const int i = i0 + (lane & (SUM_ROWS - 1));
      const uint32_t k = i < end ? keys[i] : behind, r = i < end ? rows[i] : 0;
      const uint32_t after = i0 + SUM_ROWS < end ? keys[i0 + SUM_ROWS] : behind;
      float x[SUM_ROWS][8];
#pragma unroll
      for (int q = 0; q < SUM_ROWS; ++q) {
        const uint32_t kq = __builtin_amdgcn_readlane(k, q), rq = __builtin_amdgcn_readlane(r, q);
        if (i0 + q < end && kq < (uint32_t)a.V && col < a.H) load8((const T*)a.dy + (long)rq * a.lddy + col, a.H - col, x[q]);
      }
#pragma unroll
      for (int q = 0; q < SUM_ROWS; ++q) {
        const uint32_t kq = __builtin_amdgcn_readlane(k, q);
        if (i0 + q >= end || kq >= (uint32_t)a.V) break;
#pragma unroll
        for (int e = 0; e < 8; ++e) acc[e] += x[q][e];
        const uint32_t next = i0 + q + 1 >= end ? behind : q + 1 < SUM_ROWS ? (uint32_t)__builtin_amdgcn_readlane(k, (q + 1) & (SUM_ROWS - 1)) : after;
        if (next == kq && i0 + q + 1 < end) continue;
        if (begun) part(0);
        else if (next == kq) part(1);
        else if (col < a.H) store_sum<T>(a, kq, col, acc);
        begun = false;
#pragma unroll
        for (int e = 0; e < 8; ++e) acc[e] = 0.f;
      }
    }
  }
}

// The parts of the id that begins in a run and goes on behind it, in ascending order: four waves, an equal share of the runs each
template <typename T>
__global__ __launch_bounds__(256) void embed_join(EmbeddingArgs a, EmbedPlan p, const uint32_t* keys) {
  __shared__ float red[4][64][8];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  for (long u = blockIdx.x; u < (long)p.runs * p.slabs; u += gridDim.x) {
    const int run = (int)(u / p.slabs), col = ((int)(u % p.slabs) * 64 + lane) * 8;
    const long first = (long)run * p.run, end = first + p.run;
    if (end >= a.rows) continue;
    const uint32_t k = keys[end - 1];
    if (k >= (uint32_t)a.V || keys[end] != k) continue;
    if (keys[first] == k && first && keys[first - 1] == k) continue;   // it began in an earlier run
    int n = 1;   // runs behind this one that hold rows of it: those that begin with one
    for (;; n += 64) {
      const long at = (long)(run + n + lane) * p.run;
      const unsigned long long m = __ballot(at < a.rows && keys[at < a.rows ? at : 0] == k);
      if (~m) {
        n += __builtin_ctzll(~m);
        break;
      }
    }
    // parts 0 .. n - 1: the run's own, then the n - 1 behind it
    const int per = (n + 3) / 4, q1 = min(n, (wave + 1) * per);
    float t[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) t[e] = 0.f;
    if (col < a.H) {
#pragma unroll 8
      for (int q = wave * per; q < q1; ++q) {
        float x[8];
        load8(p.parts + ((long)(run + q) * 2 + (q == 0)) * a.H + col, a.H - col, x);
#pragma unroll
        for (int e = 0; e < 8; ++e) t[e] += x[e];
      }
    }
    __syncthreads();
#pragma unroll
    for (int e = 0; e < 8; ++e) red[wave][lane][e] = t[e];
    __syncthreads();
    if (wave == 0 && col < a.H) {
#pragma unroll
      for (int w = 1; w < 4; ++w)
#pragma unroll
        for (int e = 0; e < 8; ++e) t[e] += red[w][lane][e];
      store_sum<T>(a, k, col, t);
    }
  }
}

// ------------------------------------------------------------------ launchers
static EmbedPlan plan_of(const EmbeddingArgs& a, void* ws) {
  EmbedPlan p{};
  int bits = 1;
  while (bits < 31 && a.V >> bits) ++bits;   // keys are 0 .. V
  p.passes = (bits + 8) / 9;
  p.bits = (bits + p.passes - 1) / p.passes;
  // at most 64 workgroups: each adds up the counts of all
  p.per = std::max(1, (int)((a.rows + 64L * SORT_T - 1) / (64L * SORT_T))) * SORT_T;
  p.wgs = (a.rows + p.per - 1) / p.per;
  // at most 8192 runs: each may leave two rows of parts
  p.run = std::max(1, (int)((a.rows + 8192L * SUM_ROWS - 1) / (8192L * SUM_ROWS))) * SUM_ROWS;
  p.runs = (a.rows + p.run - 1) / p.run;
  p.slabs = (a.H + 511) / 512;
  char* at = (char*)ws;
  auto take = [&](long bytes) {
    char* const r = at;
    at += (bytes + 15) / 16 * 16;
    return r;
  };
  for (int i = 0; i < 4; ++i) p.list[i] = (uint32_t*)take(4L * a.rows);
  p.counts = (uint32_t*)take(4L * p.wgs * DIGITS);
  p.parts = (float*)take(8L * p.runs * a.H);
  p.bytes = at - (char*)ws;
  return p;
}
int64_t embedding_workspace(const EmbeddingArgs& a) { return plan_of(a, nullptr).bytes; }

hipError_t launch_embedding_fwd(Dtype dt, const EmbeddingArgs& a, hipStream_t st) {
  const int chunks = (a.H + 7) / 8;
  const unsigned grid = (unsigned)std::min<long>(((long)a.rows * chunks + 255) / 256, 1 << 20);
  if (dt == DT_BF16) hipLaunchKernelGGL(embed_fwd<bf16>, dim3(grid), dim3(256), 0, st, a, chunks);
  else hipLaunchKernelGGL(embed_fwd<float>, dim3(grid), dim3(256), 0, st, a, chunks);
  return hipGetLastError();
}

template <typename T>
static hipError_t bwd(const EmbeddingArgs& a, const EmbedPlan& p, hipStream_t st) {
  const uint32_t *keys = nullptr, *rows = nullptr;
  for (int i = 0; i < p.passes; ++i) {
    uint32_t *const ko = p.list[i & 1], *const ro = p.list[2 + (i & 1)];
    if (i == 0) {
      // (16 KiB of dtable to a workgroup's turn; two to a unit keep the memory busy)
      const long clear = a.accumulate ? 0 : std::min<long>(512, ((long)a.V * a.H * (long)sizeof(T) + 16383) / 16384);
      hipLaunchKernelGGL((embed_count<T, true>), dim3(p.wgs + (unsigned)clear), dim3(SORT_T), 0, st, a, p, keys, 0);
      hipLaunchKernelGGL(embed_place<true>, dim3(p.wgs), dim3(SORT_T), 0, st, a, p, keys, rows, ko, ro, 0);
    } else {
      hipLaunchKernelGGL((embed_count<T, false>), dim3(p.wgs), dim3(SORT_T), 0, st, a, p, keys, i * p.bits);
      hipLaunchKernelGGL(embed_place<false>, dim3(p.wgs), dim3(SORT_T), 0, st, a, p, keys, rows, ko, ro, i * p.bits);
    }
    keys = ko;
    rows = ro;
  }
  const unsigned units = (unsigned)std::min<long>((long)p.runs * p.slabs, 1 << 20);
  hipLaunchKernelGGL(embed_sum<T>, dim3(units), dim3(64), 0, st, a, p, keys, rows);
  hipLaunchKernelGGL(embed_join<T>, dim3(units), dim3(256), 0, st, a, p, keys);
  return hipGetLastError();
}
hipError_t launch_embedding_bwd(Dtype dt, const EmbeddingArgs& a, void* ws, hipStream_t st) {
  const EmbedPlan p = plan_of(a, ws);
  return dt == DT_BF16 ? bwd<bf16>(a, p, st) : bwd<float>(a, p, st);
}

}  // namespace dapple
