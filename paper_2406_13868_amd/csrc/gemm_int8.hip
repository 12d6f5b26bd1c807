// The dense product of 8-bit integers, with a scale per token and one per output
// channel:
//   Y[m, n] = float(sum_k Xq[m, k] Wq[n, k]) * s_x[m] * s_w[n] + bias[n]
// The sum is exact in int32 (K below 2^17 products of at most 2^14), so it does
// not depend on how K is divided.
#include <hip/hip_runtime.h>

#include "block.h"
#include "kernels.h"
#include "tile_out.h"

#pragma clang fp contract(off)

namespace sdq {
namespace {

typedef int i4 __attribute__((ext_vector_type(4)));
typedef int i16v __attribute__((ext_vector_type(16)));

constexpr int kChunk = 128;  // bytes of K per row and stage: whole cache lines

// 16 bytes per lane to shared memory, lane i's at `to` + 16 i.
__device__ __forceinline__ void request_1k(__amdgpu_buffer_rsrc_t from, uint8_t* to, uint32_t at, uint32_t base) {
  __builtin_amdgcn_raw_ptr_buffer_load_lds(from, (__attribute__((address_space(3))) void*)to, 16, at, base, 0, 0);
}

// A workgroup owns BM tokens x BN outputs, each wave WM x WN of them in tiles of
// 32 x 32.  Chunks of 128 bytes of K go to shared memory directly, the next one
// while this one is used; each stage is an array of its own, so that the compiler
// can tell a read of one from the requests into the other.  Rows past the end are
// the last row again (their results are not stored), and the pieces of 16 past the
// end of K are the last piece again, with zeros in their place on the tokens' side.
//
// In a stage, row r's piece p (16 bytes) lies at r * 128 + 16 * (p ^ (r / 2 & 7)):
// the 16 lanes that read a piece of 16 rows together touch every bank once.
template <int BM, int BN, int WM, int WN, bool YB>
__global__ __launch_bounds__((BM / WM) * (BN / WN) * 64) void gemm_int8_tile(Int8Args a, int m_blocks) {
  constexpr int kWaves = (BM / WM) * (BN / WN), MS = WM / 32, NS = WN / 32;
  constexpr int kA = BM / 8 / kWaves, kB = BN / 8 / kWaves;  // requests per wave and stage
  __shared__ __align__(1024) uint8_t s0[(BM + BN) * kChunk], s1[(BM + BN) * kChunk];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int col = lane & 31, h = lane >> 5;
  int group, mblock;
  square_work(blockIdx.x, gridDim.x / m_blocks, m_blocks, group, mblock);
  const int m0 = mblock * BM, n0 = group * BN;
  const int rows = min(a.M - m0, BM), outs = min(a.N - n0, BN);
  const int chunks = (a.K + kChunk - 1) / kChunk, last = chunks - 1;
  const int left = a.K - last * kChunk;  // bytes of the last chunk

  const __amdgpu_buffer_rsrc_t xr = buffer_rsrc(a.x + m0 * a.x_stride, uint32_t((rows - 1) * a.x_stride + a.K));
  const __amdgpu_buffer_rsrc_t wr = buffer_rsrc(a.w + n0 * a.w_stride, uint32_t((outs - 1) * a.w_stride + a.K));
  uint32_t at[kA + kB];
  const auto piece = [&](int i) { const int r = (i * kWaves + wave) * 8 + (lane >> 3); return ((lane & 7) ^ (r >> 1 & 7)) * 16; };
#pragma unroll
  for (int i = 0; i < kA + kB; ++i) {
    const int j = i < kA ? i : i - kA, r = (j * kWaves + wave) * 8 + (lane >> 3);
    at[i] = (i < kA ? uint32_t(min(r, rows - 1)) * uint32_t(a.x_stride) : uint32_t(min(r, outs - 1)) * uint32_t(a.w_stride)) + piece(j);
  }
  const auto request = [&](int c, uint8_t* s) {
    if (c > last) return;
#pragma unroll
    for (int i = 0; i < kA + kB; ++i) {
      const int j = i < kA ? i : i - kA;
      uint32_t v = at[i];
      if (c == last) {
        const int p = piece(j);
        v += min(p, left - 16) - p;
      }
      request_1k(i < kA ? xr : wr, s + (i < kA ? 0 : BM * kChunk) + (j * kWaves + wave) * 1024, v, uint32_t(c) * kChunk);
    }
  };

  i16v acc[MS][NS];
#pragma unroll
  for (int i = 0; i < MS; ++i)
#pragma unroll
    for (int j = 0; j < NS; ++j)
#pragma unroll
      for (int e = 0; e < 16; ++e) acc[i][j][e] = 0;
  const int wm = (wave % (BM / WM)) * WM, wn = (wave / (BM / WM)) * WN;
  uint32_t from[4];  // of the lane's piece in its row, for each step of 32 bytes of K
#pragma unroll
  for (int s = 0; s < 4; ++s) from[s] = col * kChunk + (((2 * s + h) ^ (col >> 1 & 7)) << 4);

  const auto step = [&](int c, const uint8_t* s, uint8_t* next) {
    __builtin_amdgcn_s_waitcnt(0x0F70);  // vmcnt(0): this wave's requests of chunk c
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_barrier();  // every wave's; and the other stage has been read
    asm volatile("" ::: "memory");
    request(c + 1, next);
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      i4 A[MS], B[NS];
#pragma unroll
      for (int i = 0; i < MS; ++i) {
        A[i] = *reinterpret_cast<const i4*>(s + (wm + i * 32) * kChunk + from[t]);
        if (c == last && (2 * t + h) * 16 >= left) A[i] = i4{0, 0, 0, 0};
      }
#pragma unroll
      for (int j = 0; j < NS; ++j) B[j] = *reinterpret_cast<const i4*>(s + (BM + wn + j * 32) * kChunk + from[t]);
#pragma unroll
      for (int i = 0; i < MS; ++i)
#pragma unroll
        for (int j = 0; j < NS; ++j) acc[i][j] = __builtin_amdgcn_mfma_i32_32x32x32_i8(A[i], B[j], acc[i][j], 0, 0, 0);
    }
  };
  request(0, s0);
  for (int c = 0; c < chunks; c += 2) {
    step(c, s0, s1);
    if (c + 1 < chunks) step(c + 1, s1, s0);
  }

  const RowScales<MS> rs = load_row_scales<MS>(a.s_x, a.M, m0 + wm, h);
  const uint32_t es = YB ? 2 : 4;
  const int have = min(a.M - m0 - wm, WM);
  if (have <= 0) return;
  const __amdgpu_buffer_rsrc_t yr =
      buffer_rsrc(static_cast<uint8_t*>(a.y) + ((m0 + wm) * a.y_stride) * es, uint32_t((have - 1) * a.y_stride + a.N) * es);
#pragma unroll
  for (int j = 0; j < NS; ++j) {
    const int n = n0 + wn + j * 32 + col;
    if (n >= a.N) continue;
    const float sw = a.s_w[n], b = a.bias ? a.bias[n] : 0.f;
#pragma unroll
    for (int i = 0; i < MS; ++i)
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        float v = float(acc[i][j][e]) * rs.v[i][e] * sw;
        if (a.bias) v += b;
        const uint32_t idx = uint32_t(i * 32 + tile_row(e, h)) * uint32_t(a.y_stride) + uint32_t(n);
        if constexpr (YB) __builtin_amdgcn_raw_buffer_store_b16(bf16_bits(v), yr, idx * 2u, 0, 0);
        else __builtin_amdgcn_raw_buffer_store_b32(__float_as_uint(v), yr, idx * 4u, 0, 0);
      }
  }
}

template <int BM, int BN, int WM, int WN>
hipError_t tile(const Int8Args& a, hipStream_t st) {
  const int mb = (a.M + BM - 1) / BM, nb = (a.N + BN - 1) / BN;
  const dim3 grid(unsigned(mb) * unsigned(nb)), block((BM / WM) * (BN / WN) * 64);
  if (a.y_bf16) hipLaunchKernelGGL((gemm_int8_tile<BM, BN, WM, WN, true>), grid, block, 0, st, a, mb);
  else hipLaunchKernelGGL((gemm_int8_tile<BM, BN, WM, WN, false>), grid, block, 0, st, a, mb);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_gemm_int8(const Int8Args& a, hipStream_t st) { return tile<128, 128, 64, 64>(a, st); }

}  // namespace sdq
