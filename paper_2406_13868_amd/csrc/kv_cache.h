// The paged key-value cache as the kernels see it, and the launchers of the
// operators on it.  Arguments are validated by the C ABI before any of these
// is called.
#pragma once
#include <hip/hip_runtime.h>

#include <cstdint>

namespace sdq {

// n / d for 0 <= n < 2^31 by a multiplication with a reciprocal that is rounded up
// (Granlund and Montgomery, "Division by Invariant Integers using Multiplication",
// 1994): with l = ceil(log2 d) and
// m = floor(2^32 (2^l - d) / d) + 1, n / d = (umulhi(m, n) + n) >> l.
struct FastDiv {
  uint32_t d, m, l;
  FastDiv() = default;
  explicit FastDiv(uint32_t div) : d(div), l(0) {
    while ((uint64_t(1) << l) < d) ++l;
    m = uint32_t(((uint64_t(1) << 32) * ((uint64_t(1) << l) - d)) / d + 1);
  }
  __device__ __forceinline__ uint32_t div(uint32_t n) const { return (__umulhi(m, n) + n) >> l; }
};

// Strides in bytes; k and v share them.  k_scale and v_scale (e4m3 only),
// position and weight (tracked caches only) are [pages][heads][page_size].
struct KV {
  uint8_t *k, *v;
  float *k_scale, *v_scale;
  int32_t* position;
  float* weight;
  int64_t page_stride, head_stride, slot_stride;
  uint32_t pages, heads, page_size, dim;
  FastDiv per_page;  // by page_size
  bool e4m3;
};

// The pages of the sequences: slot t of sequence b lies on page
// table[b * stride + t / page_size].  A sequence's length is clamped to
// [0, cap], and a page outside [0, pages) counts as absent.
struct Seqs {
  const int32_t* table;
  const int32_t* lens;
  int64_t stride;
  int32_t B, cap;
};
__device__ __forceinline__ int seq_len(const Seqs& s, int b) { return min(max(s.lens[b], 0), s.cap); }

// Inclusive prefix sum over the wave.
__device__ __forceinline__ int wave_scan(int v) {
  v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xF, 0xF, false);  // row_shr:1
  v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xF, 0xF, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xF, 0xF, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xF, 0xF, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xA, 0xF, false);  // row_bcast:15
  v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xC, 0xF, false);  // row_bcast:31
  return v;
}

struct AppendArgs {
  KV kv;
  const void* qkv;
  int64_t row_stride;  // elements
  const int32_t* pos;
  const int64_t* slot;
  const float *q_weight, *k_weight, *cos_sin;
  void* q_out;
  int64_t positions;
  uint32_t M, heads_q, rot;
  float eps;
  bool interleaved;
};
hipError_t launch_qkv_append(const AppendArgs& a, bool x_f32, bool q_f32, hipStream_t st);

struct AttnArgs {
  KV kv;
  Seqs seqs;
  const void* q;
  int64_t q_stride;  // elements per sequence
  uint32_t heads_q, group;  // group: query heads per key head
  float scale;
  void* out;
  float* lse;               // [B][heads_q] or NULL
  const float* weight_in;   // [pages][heads][page_size], with weight_out
  float* weight_out;        // or NULL: not tracked
  float* ws;
};
size_t attn_decode_workspace_bytes(uint32_t heads_kv, uint32_t dim, uint32_t heads_q, int64_t B, int64_t cap, bool track);
hipError_t launch_attn_decode(const AttnArgs& a, bool f32, hipStream_t st);

struct EvictArgs {
  KV kv;
  Seqs seqs;
  int32_t budget, recent;
  int32_t* lens_out;
  int32_t* position_out;
  float* weight_out;
  int32_t* ws;
};
size_t cache_evict_workspace_bytes(uint32_t heads_kv, int64_t B, int64_t cap, int64_t budget);
hipError_t launch_cache_evict(const EvictArgs& a, hipStream_t st);

}  // namespace sdq
