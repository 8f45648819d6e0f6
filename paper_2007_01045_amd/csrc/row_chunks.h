// Rows in chunks of eight neighbouring elements (dropout_norm.hip, embedding.hip): 16 bytes a lane in bf16, 32 in fp32.  Rows begin at any
// multiple of the element's size (odd widths, strides and addresses): global loads and stores of 16 bytes need no other alignment,
// only a row's last chunk, if it is not whole, goes element by element.
#pragma once
#include "device_common.h"

namespace dapple {

// A chunk as it is loaded: converted where it is used, so that a row of loads waits for none of them.
// n: columns from p to the row's end, at least 1; what lies behind them reads as zero
// FAR: the element is read once and not again soon.  It is not kept in the memory-side cache then, whose lines may have to be written back for
// it: reading 268 MB behind a kernel that had written a gigabyte took 104 us, so 55.
template <typename T> struct Raw8;
typedef __attribute__((__vector_size__(4 * sizeof(float)), aligned(4))) float f32x4_any;
typedef __attribute__((__vector_size__(8 * sizeof(__bf16)), aligned(2))) __bf16 bf16x8_any;
template <> struct Raw8<bf16> {
  bf16x8 a;
  template <bool FAR = false>
  __device__ __forceinline__ void load(const bf16* p, int n) {
    if (n >= 8) {
      a = FAR ? __builtin_nontemporal_load((const bf16x8_any*)p) : *(const bf16x8_any*)p;
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) a[e] = e < n ? p[e] : (bf16)0.f;
    }
  }
  __device__ __forceinline__ float get(int e) const { return (float)a[e]; }
  __device__ __forceinline__ void set(int e, bf16 v) { a[e] = v; }
};
template <> struct Raw8<float> {
  f32x4 a, b;
  template <bool FAR = false>
  __device__ __forceinline__ void load(const float* p, int n) {
    if (n >= 8) {
      a = FAR ? __builtin_nontemporal_load((const f32x4_any*)p) : *(const f32x4_any*)p;
      b = FAR ? __builtin_nontemporal_load((const f32x4_any*)(p + 4)) : *(const f32x4_any*)(p + 4);
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        a[e] = e < n ? p[e] : 0.f;
        b[e] = 4 + e < n ? p[4 + e] : 0.f;
      }
    }
  }
  __device__ __forceinline__ float get(int e) const { return e < 4 ? a[e & 3] : b[e & 3]; }
  __device__ __forceinline__ void set(int e, float v) {
    if (e < 4) a[e & 3] = v;
    else b[e & 3] = v;
  }
};
template <typename T>
__device__ __forceinline__ void load8(const T* p, int n, float (&o)[8]) {
  Raw8<T> r;
  r.load(p, n);
#pragma unroll
  for (int e = 0; e < 8; ++e) o[e] = r.get(e);
}
template <bool FAR = false>
__device__ __forceinline__ void store8(float* p, int n, const float (&o)[8]) {
  if (n >= 8) {
    const f32x4_any a{o[0], o[1], o[2], o[3]}, b{o[4], o[5], o[6], o[7]};
    if (FAR) {
      __builtin_nontemporal_store(a, (f32x4_any*)p);
      __builtin_nontemporal_store(b, (f32x4_any*)(p + 4));
    } else {
      *(f32x4_any*)p = a;
      *(f32x4_any*)(p + 4) = b;
    }
  } else {
#pragma unroll
    for (int e = 0; e < 7; ++e)
      if (e < n) p[e] = o[e];
  }
}
template <bool FAR = false>
__device__ __forceinline__ void store8(bf16* p, int n, const float (&o)[8]) {
  bf16x8_any a;
#pragma unroll
  for (int e = 0; e < 8; ++e) a[e] = (bf16)o[e];
  if (n >= 8) {
    if (FAR) __builtin_nontemporal_store(a, (bf16x8_any*)p);
    else *(bf16x8_any*)p = a;
  } else {
#pragma unroll
    for (int e = 0; e < 7; ++e)
      if (e < n) p[e] = a[e];
  }
}

}  // namespace dapple
