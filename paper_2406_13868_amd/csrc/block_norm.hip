// The norms around a block's products, with the residual stream between them:
//
//   u = y, or norm(y; post_weight, post_bias)
//   r' = r + (u * gate) * scale                    (written in r's type)
//   n = norm(r'; weight, bias)                     (of r' before that rounding)
//   norm(v) = d * (1 / sqrt(mean d^2 + eps)) * w + b,  d = v (rms) or v - mean v (layer)
//
// n leaves as activations or as 8-bit codes with a scale per row (row_ops.h).
// Sums over a row and the reciprocal root are in fp64, everything else is one
// fp32 operation after the other: what the order of a sum could change is lost in
// the rounding of the root, so that the codes of a row are the same however many
// threads share it.  (Their cost hides behind the loads.)
//
// A row is held in registers by a wave or a workgroup, in pieces of eight
// elements, and read and written once: 8192 x 4096, bf16 with post-norm, gates and int8
// codes, takes 47.6 us among other calls, 4.9 TB/s, the rate of a large copy (51 to 53
// captured and back to back); a single row 2.8 us, the latency of a load and of each
// sum.  Rows of more than kMostHeld elements are read again for each sum instead
// (1024 x 24576, bf16, post-norm, gates, int8 codes: 87 us, layer norm 125; a copy's
// rate would be 35).
#include <hip/hip_runtime.h>

#include <algorithm>

#include "row_ops.h"

#pragma clang fp contract(off)

namespace sdq {
namespace {

constexpr uint32_t kMostHeld = 16384;

// What a row needs of the arguments, its pointers' types decided at run time:
// the branches are uniform.
struct Row {
  const NormArgs& a;
  int64_t m;
  float gate_of_row;
  __device__ __forceinline__ Row(const NormArgs& args, int64_t row) : a(args), m(row), gate_of_row(1.f) {
    if (a.gate && !a.gate_cols)
      gate_of_row = a.gate_type == kF32 ? static_cast<const float*>(a.gate)[m * a.gate_stride]
                                        : __uint_as_float(uint32_t(static_cast<const uint16_t*>(a.gate)[m * a.gate_stride]) << 16);
  }
  // r += (u * gate) * scale for the eight elements from k; a product by one changes nothing
  __device__ __forceinline__ void join(int64_t k, float (&u)[8], float (&r)[8]) const {
    if (a.gate && a.gate_cols) {
      float g[8];
      load8(a.gate_type, a.gate, m * a.gate_stride + k, g);
#pragma unroll
      for (int i = 0; i < 8; ++i) u[i] = u[i] * g[i];
    } else if (a.gate) {
#pragma unroll
      for (int i = 0; i < 8; ++i) u[i] = u[i] * gate_of_row;
    }
    if (a.scale != 1.f) {
#pragma unroll
      for (int i = 0; i < 8; ++i) u[i] = u[i] * a.scale;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) r[i] = r[i] + u[i];
  }
};

// v = d * rstd * w + b for the eight elements from k, d = v - mean
__device__ __forceinline__ void apply(float (&v)[8], bool layer, double mean, float rstd, const float* w, const float* b, int64_t k) {
  float g[8];
  load8<true>(w, k, g);
  if (layer) {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = float(double(v[i]) - mean);
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = v[i] * rstd * g[i];
  if (b) {
    load8<true>(b, k, g);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = v[i] + g[i];
  }
}

// sum / K with the rounding of a division: the product by the rounded 1 / K, and the
// rest that it leaves times 1 / K.  (The product alone is a step off for some K: the
// mean of K = 392 ones was not 1, and what it left of the row was normed.)
__device__ __forceinline__ double mean_of(double sum, double K, double per) {
  const double q = sum * per;
  return __builtin_fma(__builtin_fma(-q, K, sum), per, q);
}

// 1 / sqrt(sum / K + eps): the reciprocal root instruction is 2^-24 off or better,
// two steps of Newton's leave fp64's own roundings.  (The division and the root that
// the compiler makes are 150 instructions for every thread.)
__device__ __forceinline__ float root(double sum, double per, double eps) {
  const double x = __builtin_fma(sum, per, eps);
  double y = __builtin_amdgcn_rsq(x);
#pragma unroll
  for (int i = 0; i < 2; ++i) y = __builtin_fma(0.5 * y, __builtin_fma(-x * y, y, 1.0), y);
  return x == __builtin_huge_val() ? 0.f : float(y);
}

// Mean (layer only) and reciprocal root of a held row, whose places past its end are 0.
template <bool LAYER, int NT, int CH>
__device__ __forceinline__ void stats(const float (&v)[CH][8], uint32_t t, uint32_t P, double per, double eps, double* red, double& mean,
                                      float& rstd) {
  mean = 0.0;
  double s = 0.0;
  if constexpr (LAYER) {
#pragma unroll
    for (int c = 0; c < CH; ++c)
#pragma unroll
      for (int i = 0; i < 8; ++i) s += double(v[c][i]);
    mean = mean_of(row_sum<NT>(s, red), 8.0 * P, per);
    s = 0.0;
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      const double mu = t + c * NT < P ? mean : 0.0;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const double d = double(v[c][i]) - mu;
        s = __builtin_fma(d, d, s);
      }
    }
  } else {
#pragma unroll
    for (int c = 0; c < CH; ++c)
#pragma unroll
      for (int i = 0; i < 8; ++i) s = __builtin_fma(double(v[c][i]), double(v[c][i]), s);
  }
  rstd = root(row_sum<NT>(s, red + NT / 64), per, eps);
}

// The weights (and biases) of a thread's pieces.
template <bool LAYER, int CH>
struct Weights {
  Raw8<true> w[CH], b[LAYER ? CH : 1];
  __device__ __forceinline__ void load(const float* weight, const float* bias, uint32_t K, uint32_t t, int nt) {
    const RowBuf<true> wr(weight, 0, K);
#pragma unroll
    for (int c = 0; c < CH; ++c) w[c].load(wr, t + c * nt);
    if constexpr (LAYER)
      if (bias) {
        const RowBuf<true> br(bias, 0, K);
#pragma unroll
        for (int c = 0; c < CH; ++c) b[c].load(br, t + c * nt);
      }
  }
  // v = d * rstd * w + b, d = v - mean.  Places past the row's P pieces, which take part in
  // the maximum and the sums that follow, become 0 with any mean of finite numbers, which is
  // a finite fp32 too; with any other the whole row is NaN.
  __device__ __forceinline__ void apply(float (&v)[CH][8], uint32_t t, int nt, uint32_t P, double mean, float rstd, bool bias) const {
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      const float by = t + c * nt < P ? rstd : 0.f;
      float g[8];
      w[c].widen(g);
      if constexpr (LAYER) {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[c][i] = float(double(v[c][i]) - mean);
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) v[c][i] = v[c][i] * by * g[i];
      if constexpr (LAYER)
        if (bias) {
          b[c].widen(g);
#pragma unroll
          for (int i = 0; i < 8; ++i) v[c][i] = v[c][i] + g[i];
        }
    }
  }
};

// YT: y's type, or kNone.  NT threads a row, in pieces of eight elements, CH each; a
// wave's rows are four to a workgroup.  A workgroup takes rows one after the other:
// what all rows share (weights, a row of gates) is loaded once, and the next row is on
// its way while one is worked on.
template <bool XF32, int YT, bool LAYER, int NT, int CH>
__global__ __launch_bounds__(NT == 64 ? 256 : NT) void block_norm_kernel(NormArgs a) {
  constexpr bool YF32 = YT == kF32, kAhead = CH <= 2;  // more pieces leave no registers for a second row
  constexpr uint32_t kRows = NT == 64 ? 4 : 1;
  __shared__ double red[2][4 * (NT / 64)];
  __shared__ uint32_t top[2][NT / 64];
  const uint32_t t = NT == 64 ? threadIdx.x & 63 : threadIdx.x, P = a.K / 8, K = a.K;
  uint32_t m = NT == 64 ? blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) : blockIdx.x;
  if (m >= a.M) return;  // whole waves, and none that others wait for
  Raw8<XF32> x[CH];
  Raw8<YF32> y[CH], g[CH];
  const auto request = [&](uint32_t row) {
    const RowBuf<XF32> xr(a.residual, int64_t(row) * a.residual_stride, K);
#pragma unroll
    for (int c = 0; c < CH; ++c) x[c].load(xr, t + c * NT);
    if constexpr (YT != kNone) {
      const RowBuf<YF32> yr(a.y, int64_t(row) * a.y_stride, K);
#pragma unroll
      for (int c = 0; c < CH; ++c) y[c].load(yr, t + c * NT);
    }
  };
  // a gate of y's own type, as a rule: of the other it is asked for when it is used
  const bool cols = YT != kNone && a.gate && a.gate_cols, ready = cols && (a.gate_type == kF32) == YF32;
  const auto request_gate = [&](uint32_t row) {
    const RowBuf<YF32> gr(a.gate, int64_t(row) * a.gate_stride, K);
#pragma unroll
    for (int c = 0; c < CH; ++c) g[c].load(gr, t + c * NT);
  };
  request(m);
  Weights<LAYER, CH> w, pw;
  if (YT != kNone && a.post_weight) pw.load(a.post_weight, a.post_bias, K, t, NT);
  if (ready) request_gate(m);
  if (a.weight) w.load(a.weight, a.bias, K, t, NT);
  for (uint32_t turn = 0;; turn ^= 1) {
    float r[CH][8], u[CH][8];
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      x[c].widen(r[c]);
      if constexpr (YT != kNone) y[c].widen(u[c]);
    }
    const uint32_t next = m + gridDim.x * kRows;
    if (kAhead && next < a.M) request(next);
    if constexpr (YT != kNone) {
      const Row row(a, m);
      if (a.post_weight) {
        double mean;
        float rstd;
        stats<LAYER, NT, CH>(u, t, P, a.per, a.post_eps, red[turn], mean, rstd);
        pw.apply(u, t, NT, P, mean, rstd, a.post_bias != nullptr);
      }
      if (cols) {
#pragma unroll
        for (int c = 0; c < CH; ++c) {
          float f[8];
          if (ready) {
            g[c].widen(f);
          } else {
            Raw8<!YF32> other;
            other.load(RowBuf<!YF32>(a.gate, int64_t(m) * a.gate_stride, K), t + c * NT);
            other.widen(f);
          }
#pragma unroll
          for (int i = 0; i < 8; ++i) u[c][i] = u[c][i] * f[i];
        }
        if (ready && a.gate_stride && next < a.M) request_gate(next);
      } else if (a.gate) {
#pragma unroll
        for (int c = 0; c < CH; ++c)
#pragma unroll
          for (int i = 0; i < 8; ++i) u[c][i] = u[c][i] * row.gate_of_row;
      }
      if (a.scale != 1.f) {  // a product by one changes nothing
#pragma unroll
        for (int c = 0; c < CH; ++c)
#pragma unroll
          for (int i = 0; i < 8; ++i) u[c][i] = u[c][i] * a.scale;
      }
      const RowBuf<XF32> to(a.residual_out, int64_t(m) * a.residual_out_stride, K);
#pragma unroll
      for (int c = 0; c < CH; ++c) {
#pragma unroll
        for (int i = 0; i < 8; ++i) r[c][i] = r[c][i] + u[c][i];
        store8(to, t + c * NT, r[c]);
      }
    }
    if (a.weight) {
      double mean;
      float rstd;
      stats<LAYER, NT, CH>(r, t, P, a.per, a.eps, red[turn] + 2 * (NT / 64), mean, rstd);
      w.apply(r, t, NT, P, mean, rstd, a.bias != nullptr);
      const int64_t to = int64_t(m) * K;
      if (a.out_type == kF32) {
#pragma unroll
        for (int c = 0; c < CH; ++c) store8(RowBuf<true>(a.out, to, K), t + c * NT, r[c]);
      } else if (a.out_type == kBF16) {
#pragma unroll
        for (int c = 0; c < CH; ++c) store8(RowBuf<false>(a.out, to, K), t + c * NT, r[c]);
      } else {
        float most = 0.f;
#pragma unroll
        for (int c = 0; c < CH; ++c)
#pragma unroll
          for (int i = 0; i < 8; ++i) most = abs_max(most, r[c][i]);
        const bool e4m3 = a.out_type == kE4M3;
        const RowCode code(row_umax<NT>(abs_bits(most), top[turn]), e4m3);
        if (t == 0) a.scales[m] = code.scale();
#pragma unroll
        for (int c = 0; c < CH; ++c)
          if (t + c * NT < P)
            *reinterpret_cast<uint2*>(static_cast<uint8_t*>(a.out) + to + (t + c * NT) * 8) = codes8(r[c], code, e4m3);
      }
    }
    if (next >= a.M) break;
    m = next;
    if (!kAhead) request(m);
  }
}

// Rows of any width: each sum reads the row again.  The stream is written in the
// last pass, which reads an element before it writes it, so it may be in place.
__global__ __launch_bounds__(1024) void block_norm_wide(NormArgs a) {
  constexpr int NT = 1024;
  __shared__ double red[4][NT / 64];
  __shared__ uint32_t top[NT / 64];
  const int64_t m = blockIdx.x, K = a.K;
  const Row row(a, m);
  double post_mean = 0.0, mean = 0.0;
  float post_rstd = 1.f, rstd = 1.f;
  auto block_out = [&](int64_t k, float (&u)[8]) { load8(a.y_type, a.y, m * a.y_stride + k, u); };
  auto stream = [&](int64_t k, float (&r)[8]) {
    load8(a.x_type, a.residual, m * a.residual_stride + k, r);
    if (a.y_type == kNone) return;
    float u[8];
    block_out(k, u);
    if (a.post_weight) apply(u, a.layer, post_mean, post_rstd, a.post_weight, a.post_bias, k);
    row.join(k, u, r);
  };
  auto sums = [&](auto&& values, double eps, double* red0, double* red1, double& mu, float& root_of) {
    if (a.layer) {
      double s = 0.0;
      for (int64_t k = threadIdx.x * 8; k < K; k += NT * 8) {
        float v[8];
        values(k, v);
#pragma unroll
        for (int i = 0; i < 8; ++i) s += double(v[i]);
      }
      mu = mean_of(row_sum<NT>(s, red0), double(a.K), a.per);
    }
    double s = 0.0;
    for (int64_t k = threadIdx.x * 8; k < K; k += NT * 8) {
      float v[8];
      values(k, v);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const double d = double(v[i]) - mu;
        s = __builtin_fma(d, d, s);
      }
    }
    root_of = root(row_sum<NT>(s, red1), a.per, eps);
  };
  if (a.y_type != kNone && a.post_weight) sums(block_out, a.post_eps, red[0], red[1], post_mean, post_rstd);
  const bool coded = a.weight && (a.out_type == kInt8 || a.out_type == kE4M3), e4m3 = a.out_type == kE4M3;
  float most = 0.f;
  if (a.weight) {
    sums(stream, a.eps, red[2], red[3], mean, rstd);
    if (coded)
      for (int64_t k = threadIdx.x * 8; k < K; k += NT * 8) {
        float v[8];
        stream(k, v);
        apply(v, a.layer, mean, rstd, a.weight, a.bias, k);
#pragma unroll
        for (int i = 0; i < 8; ++i) most = abs_max(most, v[i]);
      }
  }
  const RowCode code(coded ? row_umax<NT>(abs_bits(most), top) : 0u, e4m3);
  if (coded && threadIdx.x == 0) a.scales[m] = code.scale();
  for (int64_t k = threadIdx.x * 8; k < K; k += NT * 8) {
    float v[8];
    stream(k, v);
    if (a.y_type != kNone) store8(a.x_type == kF32, a.residual_out, m * a.residual_out_stride + k, v);
    if (!a.weight) continue;
    apply(v, a.layer, mean, rstd, a.weight, a.bias, k);
    if (coded) *reinterpret_cast<uint2*>(static_cast<uint8_t*>(a.out) + m * K + k) = codes8(v, code, e4m3);
    else store8(a.out_type == kF32, a.out, m * K + k, v);
  }
}

// Workgroups of 256 compute units' worth of waves, each taking rows in turn.
constexpr uint32_t kWaves = 256 * 16;

template <bool XF32, int YT, bool LAYER, int NT, int CH>
void launch_rows(const NormArgs& a, hipStream_t st) {
  constexpr uint32_t kThreads = NT == 64 ? 256 : NT, kRows = NT == 64 ? 4 : 1;
  const dim3 grid(std::min((a.M + kRows - 1) / kRows, kWaves / (kThreads / 64))), block(kThreads);
  hipLaunchKernelGGL((block_norm_kernel<XF32, YT, LAYER, NT, CH>), grid, block, 0, st, a);
}
template <bool XF32, int YT, int NT, int CH>
void launch(const NormArgs& a, hipStream_t st) {
  // 1024 threads have 128 registers each: a layer norm's weights and biases, or an fp32
  // block's rows, would leave them (rms, 1024 x 16384, fp32: 68 us; 60 with 512 threads).
  // A layer norm's do not fit the 256 of 512 threads either: it spills 10 (bf16 both) to
  // 103 (fp32 both) and takes 88 and 145 us for 2048 x 16384, at a copy's rate 47 and 87.
  constexpr bool kMost = NT == 1024;
  if (a.layer) launch_rows<XF32, YT, true, kMost ? 512 : NT, kMost ? 2 * CH : CH>(a, st);
  else launch_rows<XF32, YT, false, kMost && YT == kF32 ? 512 : NT, kMost && YT == kF32 ? 2 * CH : CH>(a, st);
}
template <int NT, int CH>
void launch(const NormArgs& a, hipStream_t st) {
  if (a.x_type == kF32) {
    if (a.y_type == kF32) launch<true, kF32, NT, CH>(a, st);
    else if (a.y_type == kBF16) launch<true, kBF16, NT, CH>(a, st);
    else launch<true, kNone, NT, CH>(a, st);
  } else {
    if (a.y_type == kF32) launch<false, kF32, NT, CH>(a, st);
    else if (a.y_type == kBF16) launch<false, kBF16, NT, CH>(a, st);
    else launch<false, kNone, NT, CH>(a, st);
  }
}

}  // namespace

hipError_t launch_block_norm(const NormArgs& a, hipStream_t st) {
  // The fewest registers a thread that hold a row, so that few rows end soonest; of many
  // rows two pieces a thread, where half as many threads meet for a row's sums.  Measured
  // captured and back to back (us; bf16, rms, post-norm, gates, int8 codes):
  //   1024 wide, one piece a thread and two: 64 rows 3.1, 3.3;  512 rows 3.7, 3.5;  8192 rows 15.9, 14.5
  //   2048: 64 rows 3.3, 3.6;  512 rows 4.1, 4.6;  1024 rows 6.1, 5.9;  8192 rows 30.5, 28.3
  //   4096: 64 rows 3.7, 3.8;  512 rows 6.2, 6.2;  1024 rows 10.5, 9.6;  8192 rows 56.4, 51.5
  // and wider rows, the form taken and the other:
  //   64 x 8192: 4.7 (512 threads of two pieces), 5.0 (1024 of one);  4096 x 8192: 53.2, 61.2
  //   64 x 16384: 6.6 (1024 of two), 6.5 (512 of four);  2048 x 16384: 57.4, 67.3
  const uint32_t P = a.K / 8;
  const bool many = a.M >= 512;
  if (P <= 64) launch<64, 1>(a, st);
  else if (P <= 128) many ? launch<64, 2>(a, st) : launch<128, 1>(a, st);
  else if (P <= 256) many ? launch<128, 2>(a, st) : launch<256, 1>(a, st);
  else if (P <= 512) many ? launch<256, 2>(a, st) : launch<512, 1>(a, st);
  else if (P <= 1024) launch<512, 2>(a, st);
  else if (a.K <= kMostHeld) launch<1024, 2>(a, st);
  else hipLaunchKernelGGL(block_norm_wide, dim3(a.M), dim3(1024), 0, st, a);
  return hipGetLastError();
}

}  // namespace sdq
