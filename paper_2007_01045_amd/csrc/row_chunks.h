// Rows in chunks of eight neighbouring elements (dropout_norm.hip, embedding.hip): 16 bytes a lane in bf16, 32 in fp32.  Rows begin at any
// multiple of the element's size (odd widths, strides and addresses): global loads and stores of 16 bytes need no other alignment,
// only a row's last chunk, if it is not whole, goes element by element.
#pragma once
#include "device_common.h"

namespace dapple {

// n: columns from p to the row's end, at least 1; what lies behind them reads as zero
__device__ __forceinline__ void load8(const float* p, int n, float (&o)[8]) {
  if (n >= 8) {
    f32x4 a, b;
    __builtin_memcpy(&a, p, 16);
    __builtin_memcpy(&b, p + 4, 16);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      o[e] = a[e];
      o[4 + e] = b[e];
    }
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) o[e] = e < n ? p[e] : 0.f;
  }
}
__device__ __forceinline__ void load8(const bf16* p, int n, float (&o)[8]) {
  bf16x8 a;
  if (n >= 8) {
    __builtin_memcpy(&a, p, 16);
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) a[e] = e < n ? p[e] : (bf16)0.f;
  }
#pragma unroll
  for (int e = 0; e < 8; ++e) o[e] = (float)a[e];
}
__device__ __forceinline__ void store8(float* p, int n, const float (&o)[8]) {
  if (n >= 8) {
    const f32x4 a{o[0], o[1], o[2], o[3]}, b{o[4], o[5], o[6], o[7]};
    __builtin_memcpy(p, &a, 16);
    __builtin_memcpy(p + 4, &b, 16);
  } else {
#pragma unroll
    for (int e = 0; e < 7; ++e)
      if (e < n) p[e] = o[e];
  }
}
__device__ __forceinline__ void store8(bf16* p, int n, const float (&o)[8]) {
  bf16x8 a;
#pragma unroll
  for (int e = 0; e < 8; ++e) a[e] = (bf16)o[e];
  if (n >= 8) {
    __builtin_memcpy(p, &a, 16);
  } else {
#pragma unroll
    for (int e = 0; e < 7; ++e)
      if (e < n) p[e] = a[e];
  }
}

}  // namespace dapple
