// The global norm of many gradient tensors, and clipping by it:
//   norm = grad_scale sqrt(sum of all g^2),  factor = min(1, max_norm / norm),  out = g factor.
// Bound by memory: every gradient is read once for the norm, read again and written once for the clipped copy.
// The squares are taken and added in 64 bits: gradients of 1e-25 or 1e25 neither vanish nor overflow, and the sum of
// 3e8 of them is as exact as the inputs; the arithmetic (a conversion and one fused multiply-add each) stays in the
// shadow of the loads.
//
// The tensors' addresses travel as kernel arguments, up to LIST of them per launch: no copy to the device, so that the
// calls can be captured.  A workgroup takes CHUNK consecutive elements of one tensor, found by bisection of the list's first
// workgroups; its sum goes to a slot of its own, and one workgroup adds the slots in a fixed order: the same bits whatever
// the timing, and no atomics.
#include <algorithm>
#include <type_traits>

#include "device_common.h"
#include "kernels.h"

namespace dapple {

constexpr int LIST = 128;

struct GradList {
  const void* g[LIST];
  void* out[LIST];
  long n[LIST];
  int first[LIST];   // the tensor's first workgroup
  int tensors, blocks;
};
static_assert(sizeof(GradList) + 64 <= 4096, "kernel arguments");

__device__ __forceinline__ int tensor_of(const GradList& L, int block) {
  int lo = 0, hi = L.tensors - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (L.first[mid] <= block) lo = mid;
    else hi = mid - 1;
  }
  return lo;
}

// f(vector of 16 bytes' first element, V) over the 16-byte aligned middle of [0, n), f1(element) over the rest.
// U vectors per lane in flight.
template <typename T, int U, typename F, typename F1>
__device__ __forceinline__ void chunk_walk(const T* p, int n, F&& f, F1&& f1) {
  constexpr int V = 16 / sizeof(T);
  const int head = min(n, (int)((16 - ((uintptr_t)p & 15)) & 15) / (int)sizeof(T));
  const int nv = (n - head) / V, tail = head + nv * V, t = threadIdx.x;
  if (t < head) f1(t);
  if (t < n - tail) f1(tail + t);
  int i = t;
  for (; i + (U - 1) * 256 < nv; i += U * 256) f(head + i * V, std::integral_constant<int, U>{});
  for (; i < nv; i += 256) f(head + i * V, std::integral_constant<int, 1>{});
}

template <typename T>
struct Raw;
template <>
struct Raw<float> {
  typedef f32x4 V;
};
template <>
struct Raw<bf16> {
  typedef bf16x8 V;
};

template <typename T>
__global__ __launch_bounds__(256) void grad_square_kernel(GradList L, int chunk, double* __restrict__ partial) {
  typedef typename Raw<T>::V V;
  constexpr int E = 16 / sizeof(T), U = 8;
  const int at = tensor_of(L, blockIdx.x);
  const long i0 = (long)(blockIdx.x - L.first[at]) * chunk;
  const T* const p = (const T*)L.g[at] + i0;
  double s[4] = {0., 0., 0., 0.};   // (four chains of additions)
  auto add = [&](double& t, float x) { t = fma((double)x, (double)x, t); };
  chunk_walk<T, U>(p, (int)min(L.n[at] - i0, (long)chunk),
                   [&](int i, auto N) {
                     constexpr int n = decltype(N)::value;
                     V x[n];
#pragma unroll
                     for (int u = 0; u < n; ++u) x[u] = *(const V*)(p + i + u * 256 * E);
#pragma unroll
                     for (int u = 0; u < n; ++u)
#pragma unroll
                       for (int e = 0; e < E; ++e) add(s[e & 3], to_f32(x[u][e]));
                   },
                   [&](int i) { add(s[0], to_f32(p[i])); });
  double t = (s[0] + s[1]) + (s[2] + s[3]);
  for (int x = 32; x >= 1; x >>= 1) t += __shfl_xor(t, x, 64);
  __shared__ double red[4];
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = t;
  __syncthreads();
  if (threadIdx.x == 0) partial[blockIdx.x] = (red[0] + red[1]) + (red[2] + red[3]);
}

// norm[0], norm[1] from the sums of all workgroups.  A norm that is no finite number has the factor 0.
__global__ __launch_bounds__(1024) void grad_norm_kernel(const double* __restrict__ partial, int blocks, float grad_scale, float max_norm,
                                                         float* __restrict__ norm) {
  double s = 0.;
  int i = threadIdx.x;
  for (; i + 7 * 1024 < blocks; i += 8 * 1024) {
    double x[8];
#pragma unroll
    for (int u = 0; u < 8; ++u) x[u] = partial[i + u * 1024];
#pragma unroll
    for (int u = 0; u < 8; ++u) s += x[u];
  }
  for (; i < blocks; i += 1024) s += partial[i];
  for (int x = 32; x >= 1; x >>= 1) s += __shfl_xor(s, x, 64);
  __shared__ double red[16];
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = s;
  __syncthreads();
  if (threadIdx.x == 0) {
    double t = red[0];
    for (int w = 1; w < 16; ++w) t += red[w];
    const double all = fabs((double)grad_scale) * sqrt(t);
    norm[0] = (float)all;
    norm[1] = !isfinite((float)all) ? 0.f : (all > (double)max_norm ? (float)((double)max_norm / all) : 1.f);
  }
}

// The workgroups walk the list backwards: what the norm read last is still in the cache behind the L2s.
template <typename T>
__global__ __launch_bounds__(256) void grad_clip_kernel(GradList L, int chunk, const float* __restrict__ norm) {
  typedef typename Raw<T>::V V;
  constexpr int E = 16 / sizeof(T), U = 4;
  const int block = L.blocks - 1 - blockIdx.x;
  const int at = tensor_of(L, block);
  const long i0 = (long)(block - L.first[at]) * chunk;
  const T* const p = (const T*)L.g[at] + i0;
  T* const q = (T*)L.out[at] + i0;
  const float f = norm[1];
  const bool drop = !isfinite(norm[0]);   // (0 times an infinity is no 0)
  auto one = [&](int i) { q[i] = from_f32<T>(drop ? 0.f : to_f32(p[i]) * f); };
  const int n = (int)min(L.n[at] - i0, (long)chunk);
  if (((uintptr_t)p ^ (uintptr_t)q) & 15) {   // no 16 bytes of one are 16 aligned bytes of the other
    for (int i = threadIdx.x; i < n; i += 256) one(i);
    return;
  }
  chunk_walk<T, U>(p, n,
                   [&](int i, auto N) {
                     constexpr int m = decltype(N)::value;
                     V x[m];
#pragma unroll
                     for (int u = 0; u < m; ++u) x[u] = *(const V*)(p + i + u * 256 * E);
#pragma unroll
                     for (int u = 0; u < m; ++u) {
#pragma unroll
                       for (int e = 0; e < E; ++e) x[u][e] = from_f32<T>(drop ? 0.f : to_f32(x[u][e]) * f);
                       __builtin_nontemporal_store(x[u], (V*)(q + i + u * 256 * E));
                     }
                   },
                   one);
}

// Elements per workgroup: the chip's 256 units want several workgroups each, and a workgroup a few loads per lane.
static int chunk_of(const int64_t* sizes, int n) {
  int64_t total = 0;
  for (int i = 0; i < n; ++i) total += sizes[i];
  return total < (1 << 24) ? 4096 : 16384;
}

int64_t grad_norm_blocks(const int64_t* sizes, int n) {
  const int chunk = chunk_of(sizes, n);
  int64_t b = 0;
  for (int i = 0; i < n; ++i) b += (sizes[i] + chunk - 1) / chunk;
  return b;
}

// f(list, blocks before it) for each launch
template <typename F>
static hipError_t for_lists(const void* const* g, void* const* out, const int64_t* sizes, int n, int chunk, F&& f) {
  GradList L{};
  int64_t before = 0;
  for (int i = 0; i <= n; ++i) {
    if (L.tensors && (i == n || L.tensors == LIST)) {
      const hipError_t e = f(L, before);
      if (e != hipSuccess) return e;
      before += L.blocks;
      L.tensors = L.blocks = 0;
    }
    if (i == n || sizes[i] == 0) continue;
    const int k = L.tensors++;
    L.g[k] = g[i];
    L.out[k] = out ? out[i] : nullptr;
    L.n[k] = sizes[i];
    L.first[k] = L.blocks;
    L.blocks += (int)((sizes[i] + chunk - 1) / chunk);
  }
  return hipSuccess;
}

hipError_t launch_grad_norm(Dtype dt, const void* const* g, const int64_t* sizes, int n, float grad_scale, float max_norm, float* norm,
                            double* partial, hipStream_t st) {
  const int chunk = chunk_of(sizes, n);
  const hipError_t e = for_lists(g, nullptr, sizes, n, chunk, [&](const GradList& L, int64_t before) {
    if (dt == DT_BF16) hipLaunchKernelGGL(grad_square_kernel<bf16>, dim3(L.blocks), dim3(256), 0, st, L, chunk, partial + before);
    else hipLaunchKernelGGL(grad_square_kernel<float>, dim3(L.blocks), dim3(256), 0, st, L, chunk, partial + before);
    return hipGetLastError();
  });
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(grad_norm_kernel, dim3(1), dim3(1024), 0, st, partial, (int)grad_norm_blocks(sizes, n), grad_scale, max_norm, norm);
  return hipGetLastError();
}

hipError_t launch_grad_clip(Dtype dt, const void* const* g, void* const* out, const int64_t* sizes, int n, const float* norm, hipStream_t st) {
  const int chunk = chunk_of(sizes, n);
  return for_lists(g, out, sizes, n, chunk, [&](const GradList& L, int64_t) {
    if (dt == DT_BF16) hipLaunchKernelGGL(grad_clip_kernel<bf16>, dim3(L.blocks), dim3(256), 0, st, L, chunk, norm);
    else hipLaunchKernelGGL(grad_clip_kernel<float>, dim3(L.blocks), dim3(256), 0, st, L, chunk, norm);
    return hipGetLastError();
  });
}

}  // namespace dapple
