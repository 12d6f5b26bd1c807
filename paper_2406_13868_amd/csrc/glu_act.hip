// The activation between the projections of a feed-forward block:
//
//   h = act(g) * u (gated: x's rows are g, then u)  or  act(g)
//   silu: g / (1 + exp(-g));  relu: max(g, 0)
//   gelu: g / (1 + exp(-2 sqrt(2 / pi) (g + 0.044715 g^3))), the tanh form
//
// h leaves as activations or as 8-bit codes with a scale per row (row_ops.h).  It
// is evaluated in fp64 and rounded to fp32 once: two evaluations of exp that
// differ in an fp32's last bit would give other codes now and then.  That makes the
// vector units the bound, 39 instructions an element, two thirds of them fp64:
// 4096 x 11008, gated silu to int8 codes, takes 58 us among other calls (82% busy; 64 to 69
// back to back, where the clock falls), its bytes alone 45.
#include <hip/hip_runtime.h>

#include <type_traits>

#include "row_ops.h"
#include "sdq.h"

#pragma clang fp contract(off)

namespace sdq {
namespace {

constexpr uint32_t kMostHeld = 32768;

// exp(t) within 4.3e-14 of itself for |t| <= 700: t = n ln 2 + r with |r| <= ln 2 / 2,
// exp(r) by the polynomial of degree 9 that meets it at the ten Chebyshev nodes of
// that range (1.9e-14 off at most), times 2^n, whose n is the low word of
// t / ln 2 + 1.5 * 2^52.  (n ln 2 is off by n times the 2.3e-17 that ln 2 loses in one
// word: 2.3e-14 where |n| is 1010, and 3e-15 up to |t| = 88, where fp32's range ends.)
__device__ __forceinline__ double exp64(double t) {
  const double shifted = __builtin_fma(t, 1.4426950408889634, 0x1.8p52);
  const double r = __builtin_fma(shifted - 0x1.8p52, -0.6931471805599453, t);
  double p = 2.7632640675430236e-06;
  p = __builtin_fma(p, r, 2.4884459751751116e-05);
  p = __builtin_fma(p, r, 0.0001984119064754424);
  p = __builtin_fma(p, r, 0.0013888801749656543);
  p = __builtin_fma(p, r, 0.008333333367311603);
  p = __builtin_fma(p, r, 0.04166666704055191);
  p = __builtin_fma(p, r, 0.16666666666615648);
  p = __builtin_fma(p, r, 0.4999999999943859);
  p = __builtin_fma(p, r, 1.0000000000000013);
  p = __builtin_fma(p, r, 1.0000000000000135);
  const uint64_t bits = __builtin_bit_cast(uint64_t, p), n = __builtin_bit_cast(uint64_t, shifted);
  return __builtin_bit_cast(double, uint64_t(uint32_t(bits >> 32) + (uint32_t(n) << 20)) << 32 | uint32_t(bits));
}

// g / (1 + exp(t)): the reciprocal instruction is 2^-24 off, after a step of
// Newton's 2^-48.  HELD: t is held to where exp is finite; at the upper end the
// quotient is below fp32's least number, at the lower it is g.
template <bool HELD>
__device__ __forceinline__ double gate64(double g, double t) {
  if constexpr (HELD) t = fmin(fmax(t, -700.0), 700.0);
  const double q = 1.0 + exp64(t);
  const double x = __builtin_amdgcn_rcp(q);
  return g * __builtin_fma(x, __builtin_fma(-q, x, 1.0), x);
}

// Up to this magnitude of g, t stays where exp is finite.
template <int ACT>
constexpr float kFree = ACT == SDQ_ACT_SILU ? 700.f : 20.f;
template <int ACT, bool HELD>
__device__ __forceinline__ double act64(double g) {
  if constexpr (ACT == SDQ_ACT_SILU) return gate64<HELD>(g, -g);
  return gate64<HELD>(g, -1.5957691216057308 * (g + 0.044715 * (g * g * g)));
}

// h of eight elements
template <int ACT, bool GATED>
__device__ __forceinline__ void activate(const float (&g)[8], const float (&u)[8], float (&h)[8]) {
  if constexpr (ACT == SDQ_ACT_RELU) {  // one product of fp32 numbers: rounded once in fp32 too
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      h[i] = g[i] > 0.f || g[i] != g[i] ? g[i] : 0.f;
      if constexpr (GATED) h[i] = h[i] * u[i];
    }
    return;
  }
  float most = 0.f;
#pragma unroll
  for (int i = 0; i < 8; ++i) most = abs_max(most, g[i]);
  const auto all = [&](auto held) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      double v = act64<ACT, decltype(held)::value>(double(g[i]));
      if constexpr (GATED) v = v * double(u[i]);
      h[i] = float(v);
    }
  };
  if (__any(!(most <= kFree<ACT>))) all(std::true_type());  // NaN too
  else all(std::false_type());
}

// h of the eight elements from k of a row
template <int ACT, bool XF32, bool GATED>
__device__ __forceinline__ void values(const GluArgs& a, int64_t row, int64_t k, float (&h)[8]) {
  float g[8], u[8] = {};
  load8<XF32>(a.x, row + k, g);
  if constexpr (GATED) load8<XF32>(a.x, row + a.F + k, u);
  activate<ACT, GATED>(g, u, h);
}

// NT threads a row, in pieces of eight elements, CH each; a wave's rows are four to a
// workgroup.  (Workgroups that take row after row, the next on its way, are slower:
// the fp64 units are the bound, and the registers it takes leave fewer waves for them;
// 4096 x 11008: 78 us.)
template <int ACT, bool XF32, bool GATED, int NT, int CH>
__global__ __launch_bounds__(NT == 64 ? 256 : NT) void glu_code_kernel(GluArgs a) {
  __shared__ uint32_t top[NT / 64];
  const uint32_t t = NT == 64 ? threadIdx.x & 63 : threadIdx.x, P = a.F / 8;
  const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), first = NT == 64 ? 0 : wave * 64;  // its first piece
  const uint32_t m = NT == 64 ? blockIdx.x * 4 + wave : blockIdx.x;
  if (m >= a.M) return;  // whole waves, and none that others wait for
  const int64_t from = int64_t(m) * a.x_stride;
  const bool e4m3 = a.out_type == kE4M3;
  const RowBuf<XF32> gr(a.x, from, a.F), ur(a.x, GATED ? from + a.F : from, a.F);
  Raw8<XF32> gq[CH], uq[CH];
#pragma unroll
  for (int c = 0; c < CH; ++c) {
    gq[c].load(gr, t + c * NT);
    if constexpr (GATED) uq[c].load(ur, t + c * NT);
  }
  float h[CH][8], most = 0.f;
#pragma unroll
  for (int c = 0; c < CH; ++c) {
    if (c > 0 && first + c * NT >= P) {  // the whole wave is past the row
#pragma unroll
      for (int i = 0; i < 8; ++i) h[c][i] = 0.f;
      continue;
    }
    float g[8], u[8] = {};
    gq[c].widen(g);
    if constexpr (GATED) uq[c].widen(u);
    activate<ACT, GATED>(g, u, h[c]);  // 0 past the row
#pragma unroll
    for (int i = 0; i < 8; ++i) most = abs_max(most, h[c][i]);
  }
  const RowCode code(row_umax<NT>(abs_bits(most), top), e4m3);
  if (t == 0) a.scales[m] = code.scale();
#pragma unroll
  for (int c = 0; c < CH; ++c)
    if (t + c * NT < P)
      *reinterpret_cast<uint2*>(static_cast<uint8_t*>(a.out) + int64_t(m) * a.F + (t + c * NT) * 8) = codes8(h[c], code, e4m3);
}

// Rows of any width: the activation is evaluated for the maximum and again for
// the codes.
template <int ACT, bool XF32, bool GATED>
__global__ __launch_bounds__(1024) void glu_code_wide(GluArgs a) {
  constexpr int NT = 1024;
  __shared__ uint32_t top[NT / 64];
  const int64_t m = blockIdx.x, from = m * a.x_stride;
  const bool e4m3 = a.out_type == kE4M3;
  float most = 0.f;
  for (int64_t k = threadIdx.x * 8; k < a.F; k += NT * 8) {
    float h[8];
    values<ACT, XF32, GATED>(a, from, k, h);
#pragma unroll
    for (int i = 0; i < 8; ++i) most = abs_max(most, h[i]);
  }
  const RowCode code(row_umax<NT>(abs_bits(most), top), e4m3);
  if (threadIdx.x == 0) a.scales[m] = code.scale();
  for (int64_t k = threadIdx.x * 8; k < a.F; k += NT * 8) {
    float h[8];
    values<ACT, XF32, GATED>(a, from, k, h);
    *reinterpret_cast<uint2*>(static_cast<uint8_t*>(a.out) + m * a.F + k) = codes8(h, code, e4m3);
  }
}

// Activations: no row has to wait for its maximum, so a thread takes the piece
// that its index names.
template <int ACT, bool XF32, bool GATED>
__global__ __launch_bounds__(256) void glu_act_kernel(GluArgs a) {
  const uint32_t P = a.F / 8;
  const uint64_t at = uint64_t(blockIdx.x) * 256 + threadIdx.x;
  const uint32_t m = uint32_t(at / P), p = uint32_t(at - uint64_t(m) * P);
  if (m >= a.M) return;
  float h[8];
  values<ACT, XF32, GATED>(a, int64_t(m) * a.x_stride, int64_t(p) * 8, h);
  store8(a.out_type == kF32, a.out, int64_t(m) * a.F + int64_t(p) * 8, h);
}

template <int ACT, bool XF32, bool GATED, int NT, int CH>
void rows(const GluArgs& a, hipStream_t st) {
  const dim3 grid(NT == 64 ? (a.M + 3) / 4 : a.M), block(NT == 64 ? 256 : NT);
  hipLaunchKernelGGL((glu_code_kernel<ACT, XF32, GATED, NT, CH>), grid, block, 0, st, a);
}

template <int ACT, bool XF32, bool GATED>
void launch(const GluArgs& a, hipStream_t st) {
  // Few rows end soonest on many threads, as long as no wave waits for many others; many
  // rows keep the fp64 units busiest with few threads, of which some workgroups load
  // while others compute.  Measured captured and back to back (us; bf16, gated silu, int8
  // codes), the form for few rows and the one for many:
  //   1024 wide: 64 rows 2.9, 3.2;  512 rows 4.0, 3.4;  4096 rows 10.5, 8.1
  //   2048: 64 rows 2.9, 4.7;  512 rows 4.1, 5.0;  1024 rows 6.1, 5.3;  4096 rows 17.9, 13.7
  //   8192: 64 rows 4.3, 4.9;  512 rows 8.0, 9.0;  1024 rows 12.8, 13.8;  4096 rows 47.4, 47.3
  //   11008: 64 rows 5.0, 6.7;  512 rows 11.6, 12.0;  1024 rows 20.4, 18.2;  4096 rows 77.7, 64.4
  // and 1 x 4096: 3.1 (256 threads of two pieces), 3.4 (512 of one);  8192 x 4096: 46.4, 74.9.
  // Rows past kMostHeld are evaluated twice (1024 x 40960: 111 us, at a copy's rate 42).
  const uint32_t P = a.F / 8;
  const bool many = a.M >= 512;
  if (a.out_type == kF32 || a.out_type == kBF16) {
    const uint64_t pieces = uint64_t(a.M) * P;
    hipLaunchKernelGGL((glu_act_kernel<ACT, XF32, GATED>), dim3(uint32_t((pieces + 255) / 256)), dim3(256), 0, st, a);
  } else if (P <= 64) {
    rows<ACT, XF32, GATED, 64, 1>(a, st);
  } else if (P <= 128) {
    many ? rows<ACT, XF32, GATED, 64, 2>(a, st) : rows<ACT, XF32, GATED, 128, 1>(a, st);
  } else if (P <= 256) {
    many ? rows<ACT, XF32, GATED, 64, 4>(a, st) : rows<ACT, XF32, GATED, 256, 1>(a, st);
  } else if (P <= 512) {
    rows<ACT, XF32, GATED, 256, 2>(a, st);
  } else if (P <= 1024) {
    many ? rows<ACT, XF32, GATED, 256, 4>(a, st) : rows<ACT, XF32, GATED, 512, 2>(a, st);
  } else if (P <= 2048) {
    many ? rows<ACT, XF32, GATED, 256, 8>(a, st) : rows<ACT, XF32, GATED, 1024, 2>(a, st);
  } else if (a.F <= kMostHeld) {
    rows<ACT, XF32, GATED, 1024, 4>(a, st);
  } else {
    hipLaunchKernelGGL((glu_code_wide<ACT, XF32, GATED>), dim3(a.M), dim3(1024), 0, st, a);
  }
}

template <int ACT>
void launch_act(const GluArgs& a, hipStream_t st) {
  const bool f32 = a.x_type == kF32;
  if (f32 && a.gated) launch<ACT, true, true>(a, st);
  else if (f32) launch<ACT, true, false>(a, st);
  else if (a.gated) launch<ACT, false, true>(a, st);
  else launch<ACT, false, false>(a, st);
}

}  // namespace

hipError_t launch_glu_act(const GluArgs& a, hipStream_t st) {
  if (a.act == SDQ_ACT_SILU) launch_act<SDQ_ACT_SILU>(a, st);
  else if (a.act == SDQ_ACT_GELU) launch_act<SDQ_ACT_GELU>(a, st);
  else launch_act<SDQ_ACT_RELU>(a, st);
  return hipGetLastError();
}

}  // namespace sdq
