// C ABI of the operators between a block's products, and of the dense int8
// product: argument validation and dispatch (see include/sdq.h).
#include <hip/hip_runtime.h>

#include <cmath>

#include "block.h"
#include "sdq.h"

using namespace sdq;

namespace {

static_assert(kF32 == SDQ_DTYPE_F32 && kBF16 == SDQ_DTYPE_BF16 && kE4M3 == SDQ_DTYPE_E4M3 && kInt8 == SDQ_DTYPE_INT8, "");

constexpr int64_t kMostRows = (int64_t(1) << 22) - 1;    // of up to 1024 threads: a launch counts its threads in 32 bits
constexpr int64_t kMostStride = int64_t(1) << 40;

bool aligned16(const void* p) { return reinterpret_cast<uintptr_t>(p) % 16 == 0; }
bool activations(int32_t t) { return t == SDQ_DTYPE_F32 || t == SDQ_DTYPE_BF16; }
bool codes(int32_t t) { return t == SDQ_DTYPE_INT8 || t == SDQ_DTYPE_E4M3; }
int64_t bytes_of(int32_t t) { return t == SDQ_DTYPE_F32 ? 4 : t == SDQ_DTYPE_BF16 ? 2 : 1; }

// Rows of n elements, `stride` apart, that start at multiples of 16 bytes.
bool rows_fit(const void* p, int32_t type, int64_t stride, int64_t n) {
  return aligned16(p) && stride >= n && stride <= kMostStride && stride * bytes_of(type) % 16 == 0;
}

// An error that an earlier HIP call on this thread left pending is not this
// call's: it is read before the launches.
void drop_pending_error() { (void)hipGetLastError(); }

}  // namespace

extern "C" sdq_status sdq_block_norm(const sdq_norm_args* t, void* stream) {
  if (!t) return SDQ_ERR_NULL;
  const bool joins = t->y != nullptr, norms = t->weight != nullptr;
  if (!activations(t->residual_dtype) || (joins && !activations(t->y_dtype)) || (t->gate && !activations(t->gate_dtype)) ||
      (norms && !activations(t->out_dtype) && !codes(t->out_dtype)) || (t->layer != 0 && t->layer != 1) ||
      (t->gate && t->gate_per_row != 0 && t->gate_per_row != 1))
    return SDQ_ERR_CONFIG;
  // what belongs to a part that is absent
  if (!joins && !norms) return SDQ_ERR_NULL;
  if ((!joins && (t->gate || t->post_weight || t->residual_out)) || (t->post_bias && !t->post_weight) ||
      (!norms && (t->bias || t->out)) || (!t->layer && (t->bias || t->post_bias)))
    return SDQ_ERR_CONFIG;
  if ((norms && !(t->eps >= 0 && std::isfinite(t->eps))) || (t->post_weight && !(t->post_eps >= 0 && std::isfinite(t->post_eps))) ||
      (joins && !std::isfinite(t->scale)))
    return SDQ_ERR_VALUE;
  const int64_t M = t->M, K = t->K;
  if (M < 0 || M > kMostRows || K < 8 || K > (int64_t(1) << 22) || K % 8) return SDQ_ERR_SHAPE;
  if (M == 0) return SDQ_OK;
  if (!t->residual || (joins && !t->residual_out) || (norms && !t->out) || (norms && codes(t->out_dtype) && !t->scales))
    return SDQ_ERR_NULL;
  if (!rows_fit(t->residual, t->residual_dtype, t->residual_stride, K) ||
      (joins && (!rows_fit(t->y, t->y_dtype, t->y_stride, K) ||
                 !rows_fit(t->residual_out, t->residual_dtype, t->residual_out_stride, K))) ||
      (joins && t->residual_out == t->residual && t->residual_out_stride != t->residual_stride) ||
      !aligned16(t->out) || !aligned16(t->weight) || !aligned16(t->bias) || !aligned16(t->post_weight) || !aligned16(t->post_bias))
    return SDQ_ERR_SHAPE;
  if (t->gate) {
    if (t->gate_stride < 0 || t->gate_stride > kMostStride) return SDQ_ERR_SHAPE;
    if (!t->gate_per_row && (!aligned16(t->gate) || t->gate_stride * bytes_of(t->gate_dtype) % 16 ||
                             (t->gate_stride != 0 && t->gate_stride < K)))
      return SDQ_ERR_SHAPE;
  }
  NormArgs a;
  a.residual = t->residual;
  a.y = t->y;
  a.gate = t->gate;
  a.weight = t->weight;
  a.bias = t->bias;
  a.post_weight = t->post_weight;
  a.post_bias = t->post_bias;
  a.residual_out = t->residual_out;
  a.out = t->out;
  a.scales = t->scales;
  a.residual_stride = t->residual_stride;
  a.y_stride = t->y_stride;
  a.gate_stride = t->gate_stride;
  a.residual_out_stride = t->residual_out_stride;
  a.eps = t->eps;
  a.post_eps = t->post_eps;
  a.per = 1.0 / double(K);
  a.M = uint32_t(M);
  a.K = uint32_t(K);
  a.x_type = t->residual_dtype;
  a.y_type = joins ? t->y_dtype : int(kNone);
  a.gate_type = t->gate_dtype;
  a.out_type = t->out_dtype;
  a.gate_cols = !t->gate_per_row;
  a.layer = t->layer != 0;
  a.scale = t->scale;
  drop_pending_error();
  return launch_block_norm(a, static_cast<hipStream_t>(stream)) == hipSuccess ? SDQ_OK : SDQ_ERR_HIP;
}

extern "C" sdq_status sdq_glu_act(const sdq_glu_args* t, void* stream) {
  if (!t) return SDQ_ERR_NULL;
  if (!activations(t->x_dtype) || (!activations(t->out_dtype) && !codes(t->out_dtype)) ||
      (t->act != SDQ_ACT_SILU && t->act != SDQ_ACT_GELU && t->act != SDQ_ACT_RELU) || (t->gated != 0 && t->gated != 1))
    return SDQ_ERR_CONFIG;
  const int64_t M = t->M, F = t->F;
  if (M < 0 || M > kMostRows || F < 8 || F > (int64_t(1) << 22) || F % 8 || M > (int64_t(1) << 34) / F) return SDQ_ERR_SHAPE;
  if (M == 0) return SDQ_OK;
  if (!t->x || !t->out || (codes(t->out_dtype) && !t->scales)) return SDQ_ERR_NULL;
  // the up part of a gated row starts F elements on
  if (!rows_fit(t->x, t->x_dtype, t->x_stride, t->gated ? 2 * F : F) || !aligned16(t->out)) return SDQ_ERR_SHAPE;
  GluArgs a;
  a.x = t->x;
  a.out = t->out;
  a.scales = t->scales;
  a.x_stride = t->x_stride;
  a.M = uint32_t(M);
  a.F = uint32_t(F);
  a.x_type = t->x_dtype;
  a.out_type = t->out_dtype;
  a.act = t->act;
  a.gated = t->gated != 0;
  drop_pending_error();
  return launch_glu_act(a, static_cast<hipStream_t>(stream)) == hipSuccess ? SDQ_OK : SDQ_ERR_HIP;
}

namespace {
// The bounds keep int32 sums exact and every offset within a tile below 2^32.
bool int8_fits(int64_t M, int64_t N, int64_t K) {
  return M >= 0 && M <= (int64_t(1) << 24) && N >= 1 && N <= (int64_t(1) << 21) && K >= 16 && K % 16 == 0 && K < (int64_t(1) << 17) &&
         M <= (int64_t(1) << 34) / N;
}
}  // namespace

extern "C" sdq_status sdq_gemm_int8_workspace_size(int64_t M, int64_t N, int64_t K, size_t* bytes) {
  if (!bytes) return SDQ_ERR_NULL;
  if (!int8_fits(M, N, K)) return SDQ_ERR_SHAPE;
  *bytes = M ? gemm_int8_workspace_bytes(M, N, K) : 0;
  return SDQ_OK;
}

// Not part of the C ABI (no declaration in sdq.h): the form of a product for the tests.
extern "C" sdq_status sdq_gemm_int8_kernel_name(int64_t M, int64_t N, int64_t K, int32_t divide, char* out, size_t bytes) {
  if (!out) return SDQ_ERR_NULL;
  if (M < 1 || !int8_fits(M, N, K)) return SDQ_ERR_SHAPE;
  gemm_int8_kernel_name(M, N, K, divide != 0, out, bytes);
  return SDQ_OK;
}

extern "C" sdq_status sdq_gemm_int8(const sdq_int8_args* t, void* stream) {
  if (!t) return SDQ_ERR_NULL;
  if (!activations(t->y_dtype)) return SDQ_ERR_CONFIG;
  const int64_t M = t->M, N = t->N, K = t->K;
  if (!int8_fits(M, N, K)) return SDQ_ERR_SHAPE;
  if (M == 0) return SDQ_OK;
  if (!t->xq || !t->wq || !t->s_x || !t->s_w || !t->y) return SDQ_ERR_NULL;
  const int64_t lim = int64_t(1) << 22;
  if (!rows_fit(t->xq, SDQ_DTYPE_INT8, t->x_stride, K) || !rows_fit(t->wq, SDQ_DTYPE_INT8, t->w_stride, K) || t->x_stride > lim ||
      t->w_stride > lim || t->y_stride < N || t->y_stride > (int64_t(1) << 21) ||
      reinterpret_cast<uintptr_t>(t->y) % size_t(bytes_of(t->y_dtype)) || !aligned16(t->workspace))
    return SDQ_ERR_SHAPE;
  if (t->workspace && t->ws_bytes < gemm_int8_workspace_bytes(M, N, K)) return SDQ_ERR_BUFFER_TOO_SMALL;
  Int8Args a;
  a.x = static_cast<const int8_t*>(t->xq);
  a.w = static_cast<const int8_t*>(t->wq);
  a.s_x = t->s_x;
  a.s_w = t->s_w;
  a.bias = t->bias;
  a.y = t->y;
  a.x_stride = t->x_stride;
  a.w_stride = t->w_stride;
  a.y_stride = t->y_stride;
  a.M = int32_t(M);
  a.N = int32_t(N);
  a.K = int32_t(K);
  a.y_bf16 = t->y_dtype == SDQ_DTYPE_BF16;
  a.ws = t->workspace;
  drop_pending_error();
  return launch_gemm_int8(a, static_cast<hipStream_t>(stream)) == hipSuccess ? SDQ_OK : SDQ_ERR_HIP;
}
