// Norm of every query and key head, position rotation, and the write of new
// keys and values into the paged cache: what lies between the stacked q/k/v
// projection and attention, in one pass over the projection's output.
//
// For token m and head h of x = qkv[m]:
//   queries and keys:  y = x * w / sqrt(mean(x^2) + eps)     (with norm weights)
//                      (y_a, y_b) <- (y_a c - y_b s, y_b c + y_a s)
//                      for the rot / 2 pairs of the first rot dimensions
//   values:            y = x
// Queries go to q_out, keys and values to the token's slot: as bf16, or as
// e4m3 codes under one fp32 scale per row, s = amax / 448.
//
// Each head is taken by 8, 16 or 32 lanes with 8 elements each, so that every
// access is 16 bytes or more and a head's reductions stay in a part of a wave.
// The partner of a rotated element (rot / 2 elements away) is read again from
// global memory, along with its own: a second hit in the vector cache under
// the same latency, where a lane exchange would follow it.
//
// What bounds it: bytes.  8192 tokens of 96 heads of 128, bf16 (200 MB read, 200
// written): 85 us, 4.75 TB/s, where a plain copy reaches 4.9 to 5.4.  One token 2.6
// us on the GPU, a launch and three dependent loads.
#include <hip/hip_runtime.h>

#include "kv_cache.h"

namespace sdq {
namespace {

template <bool F32>
__device__ __forceinline__ void load8(const void* p, int64_t at, float (&v)[8]) {
  if constexpr (F32) {
    const float4 a = *reinterpret_cast<const float4*>(static_cast<const float*>(p) + at);
    const float4 b = *reinterpret_cast<const float4*>(static_cast<const float*>(p) + at + 4);
    v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w;
    v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
  } else {
    const uint4 raw = *reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(p) + at);
    const uint32_t w[4] = {raw.x, raw.y, raw.z, raw.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      v[2 * i] = __uint_as_float(w[i] << 16);
      v[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
    }
  }
}
template <bool F32>
__device__ __forceinline__ float load1(const void* p, int64_t at) {
  if constexpr (F32) return static_cast<const float*>(p)[at];
  else return __uint_as_float(uint32_t(static_cast<const uint16_t*>(p)[at]) << 16);
}

// Two values as bf16, nearest even, the first in the low half.
__device__ __forceinline__ uint32_t bf16_pair(float a, float b) {
  typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
  const bf16x2 r = {static_cast<__bf16>(a), static_cast<__bf16>(b)};
  return __builtin_bit_cast(uint32_t, r);
}
typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;
typedef __attribute__((ext_vector_type(2))) uint32_t u32x2;
// Results are written past the caches (8192 tokens: 87.3 us, through them 90.0;
// 64 tokens 3.86 and 3.86).
template <class T>
__device__ __forceinline__ void put(T* p, T v) {
  __builtin_nontemporal_store(v, p);
}
template <bool F32>
__device__ __forceinline__ void store8(void* p, int64_t at, const float (&v)[8]) {
  if constexpr (F32) {
    u32x4* d = reinterpret_cast<u32x4*>(static_cast<float*>(p) + at);
    put(d, u32x4{__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3])});
    put(d + 1, u32x4{__float_as_uint(v[4]), __float_as_uint(v[5]), __float_as_uint(v[6]), __float_as_uint(v[7])});
  } else {
    put(reinterpret_cast<u32x4*>(static_cast<uint16_t*>(p) + at),
             u32x4{bf16_pair(v[0], v[1]), bf16_pair(v[2], v[3]), bf16_pair(v[4], v[5]), bf16_pair(v[6], v[7])});
  }
}

// LPH lanes per head; EVEN: rot is a multiple of 16, so that a lane's eight
// elements are all rotated or none, on one side of the pairs, with 16-byte
// aligned partners and angles.
template <bool XF32, bool QF32, bool E4M3, int LPH, bool EVEN>
__global__ __launch_bounds__(256) void qkv_append_kernel(AppendArgs a, FastDiv by_heads) {
  const uint32_t unit = blockIdx.x * (256 / LPH) + threadIdx.x / LPH;
  const uint32_t m = by_heads.div(unit), h = unit - m * by_heads.d;
  if (m >= a.M) return;
  const uint32_t lane = threadIdx.x % LPH, D = a.kv.dim, d0 = lane * 8;
  const bool live = d0 < D;
  const bool is_q = h < a.heads_q, is_v = h >= a.heads_q + a.kv.heads;
  const int64_t row = int64_t(m) * a.row_stride + int64_t(h) * D;

  float x[8] = {};
  if (live) load8<XF32>(a.qkv, row + d0, x);
  bool bad = false;  // the position lies outside the table of angles
  if (!is_v) {
    const float* w = is_q ? a.q_weight : a.k_weight;
    const uint32_t rot = a.rot, half = rot / 2;
    float r = 1.f;
    if (w) {
      float ss = 0.f;
#pragma unroll
      for (int i = 0; i < 8; ++i) ss = fmaf(x[i], x[i], ss);
#pragma unroll
      for (int s = LPH / 2; s; s >>= 1) ss += __shfl_xor(ss, s, LPH);
      r = 1.f / sqrtf(ss / float(D) + a.eps);
      if (live) {
        float g[8];
        load8<true>(w, d0, g);
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] *= r * g[i];
      }
    }
    if (rot) {
      const int32_t p = a.pos[m];
      bad = p < 0 || p >= a.positions;
      const float* cs = a.cos_sin + int64_t(bad ? 0 : p) * rot;
      if (live && d0 < rot) {
        if constexpr (EVEN) {
          if (a.interleaved) {
            const float4 c = *reinterpret_cast<const float4*>(cs + d0 / 2);
            const float4 s = *reinterpret_cast<const float4*>(cs + half + d0 / 2);
            const float cc[4] = {c.x, c.y, c.z, c.w}, ssn[4] = {s.x, s.y, s.z, s.w};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const float u = x[2 * i], v = x[2 * i + 1];
              x[2 * i] = u * cc[i] - v * ssn[i];
              x[2 * i + 1] = v * cc[i] + u * ssn[i];
            }
          } else {
            const bool first = d0 < half;
            const uint32_t other = first ? d0 + half : d0 - half, j = first ? d0 : other;
            float y[8], c[8], s[8];
            load8<XF32>(a.qkv, row + other, y);
            load8<true>(cs, j, c);
            load8<true>(cs, half + j, s);
            if (w) {
              float g[8];
              load8<true>(w, other, g);
#pragma unroll
              for (int i = 0; i < 8; ++i) y[i] *= r * g[i];
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = x[i] * c[i] + (first ? -y[i] : y[i]) * s[i];
          }
        } else {
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const uint32_t e = d0 + i;
            if (e < rot) {
              const uint32_t j = a.interleaved ? e / 2 : e < half ? e : e - half;
              const bool first = a.interleaved ? !(e & 1) : e < half;
              const uint32_t other = a.interleaved ? e ^ 1 : first ? e + half : e - half;
              float y = load1<XF32>(a.qkv, row + other);
              if (w) y *= r * w[other];
              x[i] = x[i] * cs[j] + (first ? -y : y) * cs[half + j];
            }
          }
        }
      }
    }
  }
  if (is_q) {
    if (bad) {
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = __uint_as_float(0x7FC00000u);
    }
    if (live) store8<QF32>(a.q_out, (int64_t(m) * a.heads_q + h) * D + d0, x);
    return;
  }
  const int64_t slot = a.slot[m];
  if (slot < 0 || slot >= int64_t(a.kv.pages) * a.kv.page_size) return;
  if (is_v && a.rot) {
    const int32_t p = a.pos[m];
    bad = p < 0 || p >= a.positions;
  }
  if (bad) return;
  const uint32_t page = a.kv.per_page.div(uint32_t(slot)), off = uint32_t(slot) - page * a.kv.page_size;
  const uint32_t hk = h - a.heads_q - (is_v ? a.kv.heads : 0);
  uint8_t* dst = (is_v ? a.kv.v : a.kv.k) + page * a.kv.page_stride + hk * a.kv.head_stride + off * a.kv.slot_stride;
  const int64_t at = (int64_t(page) * a.kv.heads + hk) * a.kv.page_size + off;
  if constexpr (E4M3) {
    // the largest magnitude by its bits, so that a NaN is the largest of all
    // and shows in the scale
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) top = max(top, __float_as_uint(x[i]) & 0x7FFFFFFFu);
#pragma unroll
    for (int s = LPH / 2; s; s >>= 1) top = max(top, uint32_t(__shfl_xor(int(top), s, LPH)));
    // 448 / amax is past fp32's range below 1.3e-36: a tiny row is taken times a
    // power of two, which is exact and does not change the codes of others
    const float amax = __uint_as_float(top), up = amax < 0x1p-90f ? 0x1p60f : 1.f;
    const float inv = amax > 0.f ? 448.f / (amax * up) : 0.f;
    if (live) {
      float t[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) t[i] = fminf(fmaxf(x[i] * up * inv, -448.f), 448.f);
      uint32_t lo = 0, hi = 0;
      lo = __builtin_amdgcn_cvt_pk_fp8_f32(t[0], t[1], lo, false);
      lo = __builtin_amdgcn_cvt_pk_fp8_f32(t[2], t[3], lo, true);
      hi = __builtin_amdgcn_cvt_pk_fp8_f32(t[4], t[5], hi, false);
      hi = __builtin_amdgcn_cvt_pk_fp8_f32(t[6], t[7], hi, true);
      put(reinterpret_cast<u32x2*>(dst + d0), u32x2{lo, hi});
    }
    if (lane == 0) (is_v ? a.kv.v_scale : a.kv.k_scale)[at] = amax / 448.f;
  } else {
    if (live) store8<false>(dst, d0, x);
  }
  if (!is_v && lane == 0) {
    if (a.kv.position) a.kv.position[at] = a.pos[m];
    if (a.kv.weight) a.kv.weight[at] = 0.f;
  }
}

template <bool XF32, bool QF32, bool E4M3, int LPH>
void launch_lph(const AppendArgs& a, hipStream_t st) {
  const uint32_t heads = a.heads_q + 2 * a.kv.heads, per = 256 / LPH;
  const dim3 grid(uint32_t((uint64_t(a.M) * heads + per - 1) / per));
  if (a.rot % 16 == 0) qkv_append_kernel<XF32, QF32, E4M3, LPH, true><<<grid, 256, 0, st>>>(a, FastDiv(heads));
  else qkv_append_kernel<XF32, QF32, E4M3, LPH, false><<<grid, 256, 0, st>>>(a, FastDiv(heads));
}
template <bool XF32, bool QF32, bool E4M3>
void launch_types(const AppendArgs& a, hipStream_t st) {
  if (a.kv.dim <= 64) launch_lph<XF32, QF32, E4M3, 8>(a, st);
  else if (a.kv.dim <= 128) launch_lph<XF32, QF32, E4M3, 16>(a, st);
  else launch_lph<XF32, QF32, E4M3, 32>(a, st);
}

}  // namespace

hipError_t launch_qkv_append(const AppendArgs& a, bool x_f32, bool q_f32, hipStream_t st) {
  const int n = (x_f32 ? 4 : 0) + (q_f32 ? 2 : 0) + (a.kv.e4m3 ? 1 : 0);
  switch (n) {
    case 0: launch_types<false, false, false>(a, st); break;
    case 1: launch_types<false, false, true>(a, st); break;
    case 2: launch_types<false, true, false>(a, st); break;
    case 3: launch_types<false, true, true>(a, st); break;
    case 4: launch_types<true, false, false>(a, st); break;
    case 5: launch_types<true, false, true>(a, st); break;
    case 6: launch_types<true, true, false>(a, st); break;
    default: launch_types<true, true, true>(a, st); break;
  }
  return hipGetLastError();
}

}  // namespace sdq
