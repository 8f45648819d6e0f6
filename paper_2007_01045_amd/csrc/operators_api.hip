// C ABI of the operators in the second part of dapple_kernels.h: argument checks on the host, and forwarding to the
// launchers.
#include <hip/hip_runtime.h>

#include <cmath>

#include "../../include/dapple_kernels.h"
#include "../../include/dapple_stage.h"
#include "kernels.h"

using namespace dapple;

static bool bad_dtype(int dt) { return dt != STAGE_DTYPE_F32 && dt != STAGE_DTYPE_BF16; }
static Dtype type_of(int dt) { return dt == STAGE_DTYPE_BF16 ? DT_BF16 : DT_F32; }
static bool aligned_to(const void* p, size_t a) { return (uintptr_t)p % a == 0; }
static int rc_of(hipError_t e) {
  return e == hipSuccess ? STAGE_OK : set_error(STAGE_E_DEVICE, "a launch failed: %s", hipGetErrorString(e));
}

// ------------------------------------------------------------------ gradient norm
static int check_sizes(const int64_t* sizes, int n) {
  if (n < 0) return set_error(STAGE_E_CONFIG, "%d tensors", n);
  if (n > 0 && !sizes) return set_error(STAGE_E_NULL, "sizes must not be NULL");
  int64_t total = 0;
  for (int i = 0; i < n; ++i) {
    if (sizes[i] < 0) return set_error(STAGE_E_CONFIG, "tensor %d has %lld elements", i, (long long)sizes[i]);
    if (sizes[i] > (1LL << 40) || (total += sizes[i]) > (1LL << 40)) return set_error(STAGE_E_CONFIG, "more than 2^40 elements");
  }
  return STAGE_OK;
}

static int check_tensors(int dtype, const void* const* t, const int64_t* sizes, int n, const char* what) {
  if (n > 0 && !t) return set_error(STAGE_E_NULL, "%s must not be NULL", what);
  const size_t es = dtype == STAGE_DTYPE_BF16 ? 2 : 4;
  for (int i = 0; i < n; ++i) {
    if (sizes[i] == 0) continue;
    if (!t[i]) return set_error(STAGE_E_NULL, "%s[%d] is NULL", what, i);
    if (!aligned_to(t[i], es)) return set_error(STAGE_E_CONFIG, "%s[%d] is not aligned to its elements", what, i);
  }
  return STAGE_OK;
}

extern "C" {

int64_t dapple_grad_norm_workspace(const int64_t* sizes, int n) {
  const int rc = check_sizes(sizes, n);
  if (rc != STAGE_OK) return rc;
  const int64_t b = grad_norm_blocks(sizes, n);
  return 8 * (b > 0 ? b : 1);
}

int dapple_grad_norm(int dtype, const void* const* grads, const int64_t* sizes, int n, float grad_scale, float max_norm,
                     float* norm_dev, void* workspace, void* stream) {
  if (!norm_dev || !workspace) return set_error(STAGE_E_NULL, "norm_dev and workspace must not be NULL");
  if (bad_dtype(dtype)) return set_error(STAGE_E_CONFIG, "dtype %d", dtype);
  int rc = check_sizes(sizes, n);
  if (rc == STAGE_OK) rc = check_tensors(dtype, grads, sizes, n, "grads");
  if (rc != STAGE_OK) return rc;
  if (!(max_norm > 0.f)) return set_error(STAGE_E_CONFIG, "max_norm must be positive");
  if (!std::isfinite(grad_scale)) return set_error(STAGE_E_CONFIG, "grad_scale must be finite");
  if (!aligned_to(workspace, 8) || !aligned_to(norm_dev, 4)) return set_error(STAGE_E_CONFIG, "workspace or norm_dev not aligned");
  return rc_of(launch_grad_norm(type_of(dtype), grads, sizes, n, grad_scale, max_norm, norm_dev, (double*)workspace, (hipStream_t)stream));
}

int dapple_grad_clip(int dtype, const void* const* grads, void* const* outs, const int64_t* sizes, int n, const float* norm_dev,
                     void* stream) {
  if (!norm_dev) return set_error(STAGE_E_NULL, "norm_dev must not be NULL");
  if (bad_dtype(dtype)) return set_error(STAGE_E_CONFIG, "dtype %d", dtype);
  if (!aligned_to(norm_dev, 4)) return set_error(STAGE_E_CONFIG, "norm_dev not aligned");
  void* const* const to = outs ? outs : (void* const*)grads;
  int rc = check_sizes(sizes, n);
  if (rc == STAGE_OK) rc = check_tensors(dtype, grads, sizes, n, "grads");
  if (rc == STAGE_OK) rc = check_tensors(dtype, to, sizes, n, "outs");
  if (rc != STAGE_OK) return rc;
  return rc_of(launch_grad_clip(type_of(dtype), grads, to, sizes, n, norm_dev, (hipStream_t)stream));
}

}  // extern "C"
