// Embedding, forward and backward:  y[r] = scale table[id[r]],  dtable[v] = scale * sum of dy[r] over the rows r with id[r] = v, in
// an order that depends on the sizes and ids alone.  An id outside [0, V) reads nothing: its row of y is zero and it has no gradient.
//
// Forward: a copy, bound by memory.  Backward: the rows are sorted by id (stable: a row's place among those of its id is its order),
// so that an id's rows lie one behind the other, and every row of dy is read once and every row of dtable written once, without atomics
// on values.  The sort is one of least significant digits first, of at most ten bits: per digit a count and a placing, each
// workgroup a run of the rows.  Sums: a wave takes a run of the sorted rows and 512 columns; an id whose rows lie in one run is stored,
// of one that goes on in the next runs each leaves its part, and a second kernel adds the parts in ascending order.
#include <algorithm>

#include "kernels.h"
#include "row_chunks.h"

namespace dapple {

// what is of this size and more is not kept in the memory-side cache (256 MB), to which a part of it would be no use
constexpr long FAR_BYTES = 128L << 20;

// ------------------------------------------------------------------ forward
template <typename T, bool FAR>
__global__ __launch_bounds__(256) void embed_fwd(EmbeddingArgs a, int chunks) {
  const long all = (long)a.rows * chunks, stride = (long)gridDim.x * 256;
  for (long i = (long)blockIdx.x * 256 + threadIdx.x; i < all; i += stride) {
    const long row = all < (1L << 32) ? (long)((uint32_t)i / (uint32_t)chunks) : i / chunks;
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
    store8<FAR>((T*)a.y + row * a.ldy + col, a.H - col, v);
  }
}

// ------------------------------------------------------------------ sort
constexpr int DIGITS = 1024, SORT_T = 1024, SORT_W = SORT_T / 64;

// ids outside the table come last
__device__ __forceinline__ uint32_t key_of(int id, int V) { return id < 0 || id > V ? (uint32_t)V : (uint32_t)id; }

// the lanes of the wave that hold the same digit (of those that hold one)
__device__ __forceinline__ unsigned long long same_digit(uint32_t d, bool in, int bits) {
  unsigned long long same = __ballot(in);
  for (int b = 0; b < bits; ++b) {
    const unsigned long long m = __ballot((d >> b) & 1);
    same &= (d >> b) & 1 ? m : ~m;
  }
  return same;
}

// dtable, of type T, cleared by workgroups `wg` of `wgs`
template <typename T>
__device__ __forceinline__ void clear_table(const EmbeddingArgs& a, int wg, int wgs) {
  const bool dense = a.lddt == a.H;   // one row
  const long cols = dense ? (long)a.V * a.H : a.H, chunks = (cols + 7) / 8, all = dense ? chunks : a.V * chunks;
  const float zero[8] = {};
  const bool far = (long)a.V * a.H * (long)sizeof(T) >= FAR_BYTES;
  for (long i = (long)wg * SORT_T + threadIdx.x; i < all; i += (long)wgs * SORT_T) {
    const long row = dense ? 0 : i / chunks, col = (i - row * chunks) * 8;
    T* const to = (T*)a.dtable + row * a.lddt + col;
    if (far) store8<true>(to, (int)min(8L, cols - col), zero);
    else store8(to, (int)min(8L, cols - col), zero);
  }
}

// The digits of rows first .. end - 1: add(digit, how often, row).  Once a wave and digit, for the upper digits of frequent tokens are the same in
// most lanes; the lowest ones seldom
template <bool FIRST, typename F>
__device__ __forceinline__ void count_digits(const EmbeddingArgs& a, const EmbedPlan& p, const uint32_t* keys, int shift, int first, int end, F&& add) {
  const int lane = threadIdx.x & 63;
  for (int i0 = first; i0 < end; i0 += 8 * SORT_T) {
    uint32_t k[8];
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      const int i = min(i0 + u * SORT_T + (int)threadIdx.x, end - 1);
      k[u] = FIRST ? key_of(a.ids[i], a.V) : keys[i];
    }
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      if (i0 + u * SORT_T >= end) break;
      const bool in = i0 + u * SORT_T + (int)threadIdx.x < end;
      const uint32_t d = (k[u] >> shift) & ((1u << p.bits) - 1);
      if constexpr (FIRST) {
        if (in) add(d, 1u, i0 + u * SORT_T);
      } else {
        const unsigned long long same = same_digit(d, in, p.bits);
        if (in && (same & ((1ull << lane) - 1)) == 0) add(d, (uint32_t)__builtin_popcountll(same), i0 + u * SORT_T);
      }
    }
  }
}

// counts[workgroup][digit] of the workgroups' rows (where they are many: see embed_place)
template <typename T, bool FIRST>
__global__ __launch_bounds__(SORT_T) void embed_count(EmbeddingArgs a, EmbedPlan p, const uint32_t* keys, int shift) {
  __shared__ uint32_t hist[DIGITS];
  const int tid = threadIdx.x;
  if ((int)blockIdx.x >= p.wgs) return clear_table<T>(a, blockIdx.x - p.wgs, gridDim.x - p.wgs);
  hist[tid] = 0;
  __syncthreads();
  const int first = blockIdx.x * p.per;
  count_digits<FIRST>(a, p, keys, shift, first, min(a.rows, first + p.per), [&](uint32_t d, uint32_t n, int) { atomicAdd(&hist[d], n); });
  __syncthreads();
  if (tid < 1 << p.bits) p.counts[(long)blockIdx.x * DIGITS + tid] = hist[tid];
}

// The workgroup's rows to their places by one digit.  Few rows: each workgroup counts them all itself, without a launch for it, and the
// workgroups behind those of the first digit clear dtable
template <typename T, bool FIRST, bool COUNTS>
__global__ __launch_bounds__(SORT_T) void embed_place(EmbeddingArgs a, EmbedPlan p, const uint32_t* keys, const uint32_t* rows, uint32_t* keys_out,
                                                      uint32_t* rows_out, int shift) {
  __shared__ uint32_t base[DIGITS], part[2][DIGITS], run[SORT_W];
  __shared__ uint16_t of_wave[SORT_W][DIGITS];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int first = blockIdx.x * p.per, end = min(a.rows, first + p.per);
  if (FIRST && blockIdx.x == 0 && tid < 2) p.joins[tid] = 0;
  // a thread's digit's rows in the workgroups before this one, and in all
  uint32_t before = 0, total = 0;
  if constexpr (COUNTS) {
    const int wgs = tid < 1 << p.bits ? p.wgs : 0;
#pragma unroll 16
    for (int w = 0; w < wgs; ++w) {
      const uint32_t c = p.counts[(long)w * DIGITS + tid];
      before += w < (int)blockIdx.x ? c : 0;
      total += c;
    }
  } else {
    if ((int)blockIdx.x >= p.wgs) return clear_table<T>(a, blockIdx.x - p.wgs, gridDim.x - p.wgs);
    part[0][tid] = part[1][tid] = 0;
    __syncthreads();
    count_digits<FIRST>(a, p, keys, shift, 0, a.rows, [&](uint32_t d, uint32_t n, int i0) {
      atomicAdd(&part[1][d], n);
      if (i0 < first) atomicAdd(&part[0][d], n);
    });
    __syncthreads();
    before = part[0][tid], total = part[1][tid];
  }
  // the digits' first places: sums of the totals before them
  uint32_t upto = total;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const uint32_t v = __shfl_up(upto, o, 64);
    if (lane >= o) upto += v;
  }
  if (lane == 63) run[wave] = upto;
  for (int i = tid; i < SORT_W * DIGITS / 2; i += SORT_T) ((uint32_t*)&of_wave[0][0])[i] = 0;
  __syncthreads();
  uint32_t b0 = upto - total + before;
  for (int w = 0; w < wave; ++w) b0 += run[w];
  base[tid] = b0;
  __syncthreads();
  for (int i0 = first; i0 < end; i0 += SORT_T) {
    const int i = i0 + tid;
    const bool in = i < end;
    const uint32_t k = in ? (FIRST ? key_of(a.ids[i], a.V) : keys[i]) : 0;
    const uint32_t r = FIRST ? (uint32_t)i : (in ? rows[i] : 0);
    const uint32_t d = (k >> shift) & ((1u << p.bits) - 1);
    const unsigned long long same = same_digit(d, in, p.bits);
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
    if (i0 + SORT_T < end) {
      uint32_t n = 0;
#pragma unroll
      for (int w = 0; w < SORT_W; ++w) {
        n += of_wave[w][tid];
        of_wave[w][tid] = 0;
      }
      base[tid] += n;
      __syncthreads();
    }
  }
}

// ------------------------------------------------------------------ sums
// SUM_ROWS sorted rows at once; LONG: an id of so many runs or more is joined by a workgroup, another by a wave
constexpr int SUM_ROWS = 16, LONG = 33;

// The eight columns of a lane in a slab of 512: neighbours where H is a multiple of eight (WHOLE), else 64 apart, so that a row's end
// needs no path of its own (copied for every row that is loaded, it made the code larger than the instruction cache).  Lanes behind the row's
// end load its last columns and store nothing.
template <bool WHOLE>
struct Cols {
  int col;
  __device__ __forceinline__ Cols(int slab, int lane) : col(slab * 512 + (WHOLE ? 8 * lane : lane)) {}
  template <bool FAR = false, typename T>
  __device__ __forceinline__ void load(const T* row, int H, Raw8<T>& x) const {
    if constexpr (WHOLE) {
      x.template load<FAR>(row + min(col, H - 8), 8);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const T* const p = row + min(col + 64 * e, H - 1);
        x.set(e, FAR ? __builtin_nontemporal_load(p) : *p);
      }
    }
  }
  template <typename T>
  __device__ __forceinline__ void store(T* row, int H, const float (&v)[8]) const {
    if constexpr (WHOLE) {
      if (col < H) store8(row + col, 8, v);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (col + 64 * e < H) row[col + 64 * e] = from_f32<T>(v[e]);
    }
  }
};

template <typename T, bool ADD, bool WHOLE>
__device__ __forceinline__ void store_sum(const EmbeddingArgs& a, uint32_t id, const Cols<WHOLE>& cols, const float (&s)[8], const Raw8<float>& old) {
  float o[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) o[e] = ADD ? s[e] * a.scale + old.get(e) : s[e] * a.scale;
  if (ADD) cols.store((float*)a.dtable + (long)id * a.lddt, a.H, o);
  else cols.store((T*)a.dtable + (long)id * a.lddt, a.H, o);
}

// A wave: sorted rows [run p.run, ...) and 512 columns from 512 slab on.  parts[run][0]: of an id that began before the run, [1]: of one
// that begins in it and goes on behind it.  ADD (accumulate): the rows of dtable come in with those of dy, eight at once, for registers
template <typename T, bool ADD, bool WHOLE, bool FAR>
__global__ __launch_bounds__(256) void embed_sum(EmbeddingArgs a, EmbedPlan p, const uint32_t* keys, const uint32_t* rows) {
  constexpr int N = ADD ? SUM_ROWS / 2 : SUM_ROWS;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  for (long u = (long)blockIdx.x * 4 + wave; u < (long)p.runs * p.slabs; u += (long)gridDim.x * 4) {
    const int run = (int)(u / p.slabs), slab = (int)(u % p.slabs);
    const Cols<WHOLE> cols(slab, lane);
    const int first = run * p.run, end = min(a.rows, first + p.run);
    bool begun = false;   // the current id began before the run
    float acc[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) acc[e] = 0.f;
    for (int i0 = first; i0 < end; i0 += N) {
      // lanes 0 .. N: the keys from i0 on; lane N + 1: the one before
      const int i = lane <= N ? i0 + lane : i0 - 1, at = min(max(i, 0), a.rows - 1);
      const uint32_t found = keys[at], r = rows[at], k = i == at ? found : 0xffffffffu;
      __builtin_amdgcn_sched_barrier(0);   // (both loads before either is waited for)
      const uint32_t k0 = __builtin_amdgcn_readlane(k, 0);
      if (k0 >= (uint32_t)a.V) break;
      if (i0 == first) begun = (uint32_t)__builtin_amdgcn_readlane(k, N + 1) == k0;
      Raw8<T> x[N];   // (rows that are not summed up are loaded, too: no branch stands between the loads)
      Raw8<float> old[ADD ? N : 1];
#pragma unroll
      for (int q = 0; q < N; ++q) {
        cols.template load<FAR>((const T*)a.dy + (long)__builtin_amdgcn_readlane(r, q) * a.lddy, a.H, x[q]);
        if (ADD) cols.load((const float*)a.dtable + (long)min((uint32_t)__builtin_amdgcn_readlane(k, q), (uint32_t)a.V - 1) * a.lddt, a.H, old[q]);
      }
#pragma unroll
      for (int q = 0; q < N; ++q) {
        const uint32_t kq = __builtin_amdgcn_readlane(k, q), next = __builtin_amdgcn_readlane(k, q + 1);
        if (kq >= (uint32_t)a.V) break;   // (behind the last row, too)
#pragma unroll
        for (int e = 0; e < 8; ++e) acc[e] += x[q].get(e);
        const bool on = next == kq;
        if (on && i0 + q + 1 < end) continue;
        if (begun || on) {
          cols.store(p.parts + ((long)run * 2 + (begun ? 0 : 1)) * a.H, a.H, acc);
          if (!begun && slab == 0) {   // (listed in any order: each is by itself)
            const long far = first + (long)LONG * p.run;
            const bool many = far < a.rows && keys[far] == kq;
            if (lane == 0) p.join_list[many ? p.runs - 1 - atomicAdd(p.joins + 1, 1) : atomicAdd(p.joins, 1)] = run;
          }
        } else {
          store_sum<T, ADD>(a, kq, cols, acc, old[ADD ? q : 0]);
        }
        begun = false;
#pragma unroll
        for (int e = 0; e < 8; ++e) acc[e] = 0.f;
      }
    }
  }
}

// The parts of the ids that begin in a listed run and go on behind it, in ascending order.  A wave each; ids of many runs, which stand at the
// list's end, a workgroup each, an equal share of the runs to each of its waves
template <typename T, bool ADD, bool WHOLE>
__global__ __launch_bounds__(256) void embed_join(EmbeddingArgs a, EmbedPlan p, const uint32_t* keys) {
  __shared__ float red[4][64][8];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int few = p.joins[0], many = p.joins[1];
  // runs behind `run` that hold rows of its last id: those that begin with one
  auto runs_of = [&](int run, uint32_t k) {
    for (int n = 1;; n += 64) {
      const long at = (long)(run + n + lane) * p.run;
      const unsigned long long m = __ballot(at < a.rows && keys[at < a.rows ? at : 0] == k);
      if (~m) return n + (int)__builtin_ctzll(~m);
    }
  };
  auto add = [&](int run, int q0, int q1, const Cols<WHOLE>& cols, float (&t)[8]) {
    for (int q = q0; q < q1; q += 8) {
      Raw8<float> x[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) cols.load((const float*)p.parts + ((long)(run + min(q + i, q1 - 1)) * 2 + (q + i == 0)) * a.H, a.H, x[i]);
#pragma unroll
      for (int i = 0; i < 8; ++i)
#pragma unroll
        for (int e = 0; e < 8; ++e) t[e] += q + i < q1 ? x[i].get(e) : 0.f;
    }
  };
  auto old_of = [&](uint32_t k, const Cols<WHOLE>& cols) {
    Raw8<float> old;
    if (ADD) cols.load((const float*)a.dtable + (long)k * a.lddt, a.H, old);
    return old;
  };
  for (long u = (long)blockIdx.x; u < (long)many * p.slabs; u += gridDim.x) {
    const int run = p.join_list[p.runs - 1 - u / p.slabs];
    const Cols<WHOLE> cols((int)(u % p.slabs), lane);
    const uint32_t k = keys[(long)run * p.run + p.run - 1];
    const Raw8<float> old = old_of(k, cols);
    const int n = runs_of(run, k), per = (n + 3) / 4;
    float t[8] = {};
    add(run, wave * per, min(n, (wave + 1) * per), cols, t);
    __syncthreads();
#pragma unroll
    for (int e = 0; e < 8; ++e) red[wave][lane][e] = t[e];
    __syncthreads();
    if (wave == 0) {
#pragma unroll
      for (int w = 1; w < 4; ++w)
#pragma unroll
        for (int e = 0; e < 8; ++e) t[e] += red[w][lane][e];
      store_sum<T, ADD>(a, k, cols, t, old);
    }
  }
  for (long u = (long)blockIdx.x * 4 + wave; u < (long)few * p.slabs; u += (long)gridDim.x * 4) {
    const int run = p.join_list[u / p.slabs];
    const Cols<WHOLE> cols((int)(u % p.slabs), lane);
    const uint32_t k = keys[(long)run * p.run + p.run - 1];
    const Raw8<float> old = old_of(k, cols);
    const int n = runs_of(run, k);
    float t[8] = {};
    add(run, 0, n, cols, t);
    store_sum<T, ADD>(a, k, cols, t, old);
  }
}

// ------------------------------------------------------------------ launchers
static EmbedPlan plan_of(const EmbeddingArgs& a, void* ws) {
  EmbedPlan p{};
  int bits = 1;
  while (bits < 31 && a.V >> bits) ++bits;   // keys are 0 .. V
  p.passes = (bits + 9) / 10;
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
  p.joins = (int32_t*)take(8);
  p.join_list = (int32_t*)take(4L * p.runs);
  p.parts = (float*)take(8L * p.runs * a.H);
  p.bytes = at - (char*)ws;
  return p;
}
int64_t embedding_workspace(const EmbeddingArgs& a) { return plan_of(a, nullptr).bytes; }

template <typename T>
static hipError_t fwd(const EmbeddingArgs& a, hipStream_t st) {
  const int chunks = (a.H + 7) / 8;
  const dim3 grid((unsigned)std::min<long>(((long)a.rows * chunks + 255) / 256, 1 << 20));
  if ((long)a.rows * a.H * (long)sizeof(T) >= FAR_BYTES) hipLaunchKernelGGL((embed_fwd<T, true>), grid, dim3(256), 0, st, a, chunks);
  else hipLaunchKernelGGL((embed_fwd<T, false>), grid, dim3(256), 0, st, a, chunks);
  return hipGetLastError();
}
hipError_t launch_embedding_fwd(Dtype dt, const EmbeddingArgs& a, hipStream_t st) { return dt == DT_BF16 ? fwd<bf16>(a, st) : fwd<float>(a, st); }

template <typename T>
static hipError_t bwd(const EmbeddingArgs& a, const EmbedPlan& p, hipStream_t st) {
  // (16 KiB of dtable to a workgroup's turn; two to a unit keep the memory busy)
  const unsigned clear = a.accumulate ? 0 : (unsigned)std::min<long>(512, ((long)a.V * a.H * (long)sizeof(T) + 16383) / 16384);
  // (us without / with counts from a launch of their own, rows of 256 of 30522: 2048 rows 23.4 / 27.7, 8192 31.9 / 35.2, 12288 36.7 / 38.0, 16384
  // 41.8 / 38.1, 65536 102 / 66)
  const bool few = a.rows <= 12288;
  const uint32_t *keys = nullptr, *rows = nullptr;
  for (int i = 0; i < p.passes; ++i) {
    const int shift = i * p.bits;
    uint32_t *const ko = p.list[i & 1], *const ro = p.list[2 + (i & 1)];
    auto place = [&](auto kern, unsigned more) { hipLaunchKernelGGL(kern, dim3(p.wgs + more), dim3(SORT_T), 0, st, a, p, keys, rows, ko, ro, shift); };
    auto count = [&](auto kern, unsigned more) { hipLaunchKernelGGL(kern, dim3(p.wgs + more), dim3(SORT_T), 0, st, a, p, keys, shift); };
    if (few) {
      if (i == 0) place(embed_place<T, true, false>, clear);
      else place(embed_place<T, false, false>, 0);
    } else if (i == 0) {
      count(embed_count<T, true>, clear);
      place(embed_place<T, true, true>, 0);
    } else {
      count(embed_count<T, false>, 0);
      place(embed_place<T, false, true>, 0);
    }
    keys = ko;
    rows = ro;
  }
  const unsigned units = (unsigned)std::min<long>(((long)p.runs * p.slabs + 3) / 4, 1 << 20);   // four to a workgroup
  using std::false_type;
  using std::true_type;
  auto sums = [&](auto ADD, auto WHOLE, auto FAR) {
    hipLaunchKernelGGL((embed_sum<T, decltype(ADD)::value, decltype(WHOLE)::value, decltype(FAR)::value>), dim3(units), dim3(256), 0, st, a, p, keys, rows);
    hipLaunchKernelGGL((embed_join<T, decltype(ADD)::value, decltype(WHOLE)::value>), dim3(std::min(units, 2048u)), dim3(256), 0, st, a, p, keys);
  };
  // (dy past the cache, us: 268 MB 130 / 76 without / with; 17 MB, which are still in it, 12.4 / 14.9)
  const bool far = (long)a.rows * a.H * (long)sizeof(T) >= FAR_BYTES;
  auto pick = [&](auto ADD, auto WHOLE) { far ? sums(ADD, WHOLE, true_type{}) : sums(ADD, WHOLE, false_type{}); };
  auto whole = [&](auto ADD) { a.H % 8 ? pick(ADD, false_type{}) : pick(ADD, true_type{}); };
  a.accumulate ? whole(true_type{}) : whole(false_type{});
  return hipGetLastError();
}
hipError_t launch_embedding_bwd(Dtype dt, const EmbeddingArgs& a, void* ws, hipStream_t st) {
  const EmbedPlan p = plan_of(a, ws);
  return dt == DT_BF16 ? bwd<bf16>(a, p, st) : bwd<float>(a, p, st);
}

}  // namespace dapple
