// What the kernels that work on rows of activations share: pieces of eight
// elements, sums and maxima over a row's threads, and the 8-bit codes of a row.
//
// Every step is one operation rounded to fp32 (or done in fp64), never a fused
// one, so that codes are the same wherever the row's values are.
#pragma once
#include <hip/hip_runtime.h>

#include <cstdint>

#include "block.h"
#include "tile_out.h"

#pragma clang fp contract(off)

namespace sdq {

// Eight neighbouring elements, widened to fp32; at: the element's index.
template <bool F32>
__device__ __forceinline__ void load8(const void* p, int64_t at, float (&v)[8]) {
  if constexpr (F32) {
    const float4* q = reinterpret_cast<const float4*>(static_cast<const float*>(p) + at);
    const float4 a = q[0], b = q[1];
    v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w;
    v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
  } else {
    const uint4 q = *reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(p) + at);
    const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      v[2 * i] = __uint_as_float(w[i] << 16);
      v[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
    }
  }
}
__device__ __forceinline__ void load8(int type, const void* p, int64_t at, float (&v)[8]) {
  if (type == kF32) load8<true>(p, at, v);
  else load8<false>(p, at, v);
}

// A row as a buffer: pieces past its end read as zeros and are not written, so that
// no load has a branch around it and all of a row's are on their way together.
template <bool F32>
struct RowBuf {
  __amdgpu_buffer_rsrc_t r;
  __device__ __forceinline__ RowBuf(const void* p, int64_t at, uint32_t n)
      : r(buffer_rsrc(static_cast<const uint8_t*>(p) + at * (F32 ? 4 : 2), n * (F32 ? 4 : 2))) {}
};
// Eight elements as they lie in memory.
template <bool F32>
struct Raw8 {
  typedef int vec __attribute__((ext_vector_type(4)));
  vec q[F32 ? 2 : 1];
  __device__ __forceinline__ void load(const RowBuf<F32>& row, uint32_t piece) {
#pragma unroll
    for (int i = 0; i < (F32 ? 2 : 1); ++i) q[i] = __builtin_amdgcn_raw_buffer_load_b128(row.r, piece * (F32 ? 32 : 16), i * 16, 0);
  }
  __device__ __forceinline__ void widen(float (&v)[8]) const {
    if constexpr (F32) {
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = __int_as_float(q[i / 4][i % 4]);
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        v[2 * i] = __uint_as_float(uint32_t(q[0][i]) << 16);
        v[2 * i + 1] = __uint_as_float(uint32_t(q[0][i]) & 0xFFFF0000u);
      }
    }
  }
};

__device__ __forceinline__ uint32_t bf16_pair(float a, float b) {
  return uint32_t(__builtin_bit_cast(uint16_t, static_cast<__bf16>(a))) |
         uint32_t(__builtin_bit_cast(uint16_t, static_cast<__bf16>(b))) << 16;
}
// Eight activations, as fp32 or rounded to bf16.
__device__ __forceinline__ void store8(bool f32, void* p, int64_t at, const float (&v)[8]) {
  if (f32) {
    float4* q = reinterpret_cast<float4*>(static_cast<float*>(p) + at);
    q[0] = make_float4(v[0], v[1], v[2], v[3]);
    q[1] = make_float4(v[4], v[5], v[6], v[7]);
  } else {
    *reinterpret_cast<uint4*>(static_cast<uint16_t*>(p) + at) =
        make_uint4(bf16_pair(v[0], v[1]), bf16_pair(v[2], v[3]), bf16_pair(v[4], v[5]), bf16_pair(v[6], v[7]));
  }
}

// The same through a row's buffer.
template <bool F32>
__device__ __forceinline__ void store8(const RowBuf<F32>& row, uint32_t piece, const float (&v)[8]) {
  typedef int vec __attribute__((ext_vector_type(4)));
  if constexpr (F32) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const vec q = {__float_as_int(v[4 * i]), __float_as_int(v[4 * i + 1]), __float_as_int(v[4 * i + 2]), __float_as_int(v[4 * i + 3])};
      __builtin_amdgcn_raw_buffer_store_b128(q, row.r, piece * 32, i * 16, 0);
    }
  } else {
    const vec q = {int(bf16_pair(v[0], v[1])), int(bf16_pair(v[2], v[3])), int(bf16_pair(v[4], v[5])), int(bf16_pair(v[6], v[7]))};
    __builtin_amdgcn_raw_buffer_store_b128(q, row.r, piece * 16, 0, 0);
  }
}

// A value of each lane, moved within the rows of 16 lanes.
template <int CTRL>
__device__ __forceinline__ uint32_t dpp(uint32_t v) {
  return uint32_t(__builtin_amdgcn_update_dpp(int(v), int(v), CTRL, 0xF, 0xF, false));
}
template <int CTRL>
__device__ __forceinline__ double dpp(double v) {
  const uint64_t b = __builtin_bit_cast(uint64_t, v);
  return __builtin_bit_cast(double, uint64_t(dpp<CTRL>(uint32_t(b >> 32))) << 32 | dpp<CTRL>(uint32_t(b)));
}

// Sum over the wave: rotations by 8, 4, 2 and 1 within rows of 16 lanes, then
// the rows.  Every lane adds the same pairs, so all get the same bits.
__device__ __forceinline__ double wave_sum(double v) {
  v += dpp<0x128>(v);
  v += dpp<0x124>(v);
  v += dpp<0x122>(v);
  v += dpp<0x121>(v);
  uint64_t b = __builtin_bit_cast(uint64_t, v);
  const auto l16 = __builtin_amdgcn_permlane16_swap(uint32_t(b), uint32_t(b), false, false);
  const auto h16 = __builtin_amdgcn_permlane16_swap(uint32_t(b >> 32), uint32_t(b >> 32), false, false);
  v = __builtin_bit_cast(double, uint64_t(h16[0]) << 32 | l16[0]) + __builtin_bit_cast(double, uint64_t(h16[1]) << 32 | l16[1]);
  b = __builtin_bit_cast(uint64_t, v);
  const auto l32 = __builtin_amdgcn_permlane32_swap(uint32_t(b), uint32_t(b), false, false);
  const auto h32 = __builtin_amdgcn_permlane32_swap(uint32_t(b >> 32), uint32_t(b >> 32), false, false);
  return __builtin_bit_cast(double, uint64_t(h32[0]) << 32 | l32[0]) + __builtin_bit_cast(double, uint64_t(h32[1]) << 32 | l32[1]);
}
__device__ __forceinline__ uint32_t wave_umax(uint32_t v) {
  v = max(v, dpp<0x128>(v));
  v = max(v, dpp<0x124>(v));
  v = max(v, dpp<0x122>(v));
  v = max(v, dpp<0x121>(v));
  const auto a = __builtin_amdgcn_permlane16_swap(v, v, false, false);
  v = max(a[0], a[1]);
  const auto b = __builtin_amdgcn_permlane32_swap(v, v, false, false);
  return max(b[0], b[1]);
}

// The NT threads of a row (one wave, or a workgroup) put their values together.
// red: NT / 64 slots of shared memory that no other call of the kernel uses.
template <int NT>
__device__ __forceinline__ double row_sum(double v, double* red) {
  v = wave_sum(v);
  if constexpr (NT == 64) return v;
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
  __syncthreads();
  double s = red[0];
#pragma unroll
  for (int i = 1; i < NT / 64; ++i) s += red[i];
  return s;
}
template <int NT>
__device__ __forceinline__ uint32_t row_umax(uint32_t v, uint32_t* red) {
  v = wave_umax(v);
  if constexpr (NT == 64) return v;
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
  __syncthreads();
  uint32_t s = red[0];
#pragma unroll
  for (int i = 1; i < NT / 64; ++i) s = max(s, red[i]);
  return s;
}

// The larger magnitude; a NaN stays one.
__device__ __forceinline__ float abs_max(float most, float v) { return __builtin_elementwise_maximum(most, fabsf(v)); }
// The bits of a magnitude: as whole numbers they are ordered as the magnitudes are,
// with infinity above them and NaN above that.
__device__ __forceinline__ uint32_t abs_bits(float v) { return __float_as_uint(v) & 0x7FFFFFFFu; }

// How the rows of 8-bit codes are scaled: s = amax / qmax and code = v * pre * inv
// to the nearest with inv = (1 / amax) * qmax.  Where inv would pass fp32's range,
// pre = 2^60 and the codes are those of the row times 2^60; a row that holds an
// infinity or a NaN has a scale that is not finite, and zero codes.
struct RowCode {
  float amax, qmax, inv, pre;
  __device__ __forceinline__ float scale() const { return amax / qmax; }
  __device__ __forceinline__ RowCode(uint32_t amax_bits, bool e4m3) : amax(__uint_as_float(amax_bits)), qmax(e4m3 ? 448.f : 127.f) {
    float a = amax;
    const bool tiny = a > 0.f && a < 0x1p-118f;  // 448 / 2^-118 is below 2^127
    pre = tiny ? 0x1p60f : 1.f;
    a *= pre;
    inv = a > 0.f && amax_bits < 0x7F800000u ? 1.f / a * qmax : 0.f;
  }
};

// Four whole numbers, each in the low byte of a word, as one word.
__device__ __forceinline__ uint32_t bytes4(float a, float b, float c, float d) {
  const uint32_t ab = __builtin_amdgcn_perm(__float_as_uint(b), __float_as_uint(a), 0x0C0C0400);
  const uint32_t cd = __builtin_amdgcn_perm(__float_as_uint(d), __float_as_uint(c), 0x0C0C0400);
  return __builtin_amdgcn_perm(cd, ab, 0x05040100);
}

// The codes of eight values, as two words.  |v * inv| is qmax at most, up to its
// roundings, which neither type's last code is left by.  int8: t + 1.5 * 2^23 is t to
// the nearest whole number, ties to even, with its two's complement in the low bits.
__device__ __forceinline__ uint2 codes8(const float (&v)[8], const RowCode& c, bool e4m3) {
  if (c.inv == 0.f) return make_uint2(0, 0);  // zero rows, and rows with values that are not finite
  float t[8];
  if (c.pre == 1.f) {
#pragma unroll
    for (int i = 0; i < 8; ++i) t[i] = v[i] * c.inv;
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) t[i] = v[i] * c.pre * c.inv;
  }
  if (e4m3) {
    uint32_t lo = __builtin_amdgcn_cvt_pk_fp8_f32(t[0], t[1], 0, false);  // to nearest even
    lo = __builtin_amdgcn_cvt_pk_fp8_f32(t[2], t[3], lo, true);
    uint32_t hi = __builtin_amdgcn_cvt_pk_fp8_f32(t[4], t[5], 0, false);
    hi = __builtin_amdgcn_cvt_pk_fp8_f32(t[6], t[7], hi, true);
    return make_uint2(lo, hi);
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) t[i] = t[i] + 0x1.8p23f;
  return make_uint2(bytes4(t[0], t[1], t[2], t[3]), bytes4(t[4], t[5], t[6], t[7]));
}

}  // namespace sdq
