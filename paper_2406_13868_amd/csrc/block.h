// The operators between a block's products as the kernels see them, and their
// launchers.  Arguments are validated by the C ABI before any of these is called.
#pragma once
#include <hip/hip_runtime.h>

#include <cstdint>

namespace sdq {

// Element types of activations, as in sdq.h; -1: absent.
enum : int { kF32 = 0, kBF16 = 1, kE4M3 = 2, kInt8 = 3, kNone = -1 };

struct NormArgs {
  const void *residual, *y, *gate;
  const float *weight, *bias, *post_weight, *post_bias;
  void *residual_out, *out;
  float* scales;
  int64_t residual_stride, y_stride, gate_stride, residual_out_stride;  // elements
  double eps, post_eps, per;  // per: 1 / K
  uint32_t M, K;
  int x_type, y_type, gate_type, out_type;  // residual's, y's (or kNone), ...
  bool gate_cols;                           // one gate for each element of a row, not one for the row
  bool layer;
  float scale;
};
hipError_t launch_block_norm(const NormArgs& a, hipStream_t st);

struct GluArgs {
  const void* x;
  void* out;
  float* scales;
  int64_t x_stride;  // elements
  uint32_t M, F;
  int x_type, out_type, act;
  bool gated;
};
hipError_t launch_glu_act(const GluArgs& a, hipStream_t st);

struct Int8Args {
  const int8_t *x, *w;
  const float *s_x, *s_w, *bias;
  void* y;
  int64_t x_stride, w_stride, y_stride;  // elements
  int32_t M, N, K;
  bool y_bf16;
  void* ws;  // gemm_int8_workspace_bytes bytes, or NULL: K is not divided
};
size_t gemm_int8_workspace_bytes(int64_t M, int64_t N, int64_t K);
// The form that a product takes, with or without a workspace, for the tests.
void gemm_int8_kernel_name(int64_t M, int64_t N, int64_t K, bool divide, char* out, size_t n);
hipError_t launch_gemm_int8(const Int8Args& a, hipStream_t st);

}  // namespace sdq
