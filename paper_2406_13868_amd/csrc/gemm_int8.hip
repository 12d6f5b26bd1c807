// The dense product of 8-bit integers, with a scale per token and one per output
// channel:
//   Y[m, n] = float(sum_k Xq[m, k] Wq[n, k]) * s_x[m] * s_w[n] + bias[n]
// The sum is exact in int32 (K below 2^17 products of at most 2^14), so it does
// not depend on how K is divided.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>
#include <cstdio>

#include "block.h"
#include "kernels.h"
#include "tile_out.h"

#pragma clang fp contract(off)

namespace sdq {
namespace {

typedef int i4 __attribute__((ext_vector_type(4)));
typedef int i16v __attribute__((ext_vector_type(16)));

constexpr int kChunk = 128;  // bytes of K per row and stage: whole cache lines

// Weights that are read once pass the caches by.
constexpr int kStream = 2;

// 16 bytes per lane to shared memory, lane i's at `to` + 16 i.  In assembly, and
// awaited by the kernels themselves: a read of shared memory waits for every request
// that the compiler knows of and cannot tell from it, and it loses count where a loop
// closes (256 x 4096 x 4096: 13.0 us that way, 10.5 this).  The instruction returns
// nothing to registers.  m0 is a register that the compiler keeps no value in (it takes
// no clobber of it), and it writes it for no other instruction of these kernels.
template <int HINT = 0>
__device__ __forceinline__ void request_1k(__amdgpu_buffer_rsrc_t from, uint8_t* to, uint32_t at, uint32_t base) {
  const uint32_t where = uint32_t(reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) void*)to));
  if constexpr (HINT == kStream)
    asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tbuffer_load_dwordx4 %0, %1, %3 offen nt lds" ::"v"(at), "s"(from), "s"(where), "s"(base) : "memory");
  else
    asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tbuffer_load_dwordx4 %0, %1, %3 offen lds" ::"v"(at), "s"(from), "s"(where), "s"(base) : "memory");
}

// s_waitcnt's operand: at most n vector memory operations on their way, and no
// operation on shared memory.
constexpr int wait_vm(int n) { return (n & 15) | (n >> 4) << 14 | 0x0070; }

// An offset outside every buffer here: such a load reads nothing.
constexpr uint32_t kNowhere = 0x80000000u;

// What no kernel writes while this one runs, for scalar loads.
__device__ __forceinline__ const __attribute__((address_space(4))) float* constant(const float* p) {
  return (const __attribute__((address_space(4))) float*)(p);
}

// All waves' operations on shared memory are done; requests from memory go on.
__device__ __forceinline__ void barrier_lds() {
  __builtin_amdgcn_s_waitcnt(0xC07F);  // lgkmcnt(0)
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

constexpr int kSums = 4;  // beside kF32 and kBF16: int32 sums, not scaled yet

// ---- tiles -----------------------------------------------------------------
// BM tokens from m0 x BN outputs from n0 by a workgroup, each wave WM x WN of them in
// tiles of 32 x 32.  Chunks of 128 bytes of K go to shared memory directly, up to
// STAGES - 1 of them while one is used.  Rows past the end are the last row again
// (their results are not stored), and the pieces of 16 past the end of K are the last
// piece again, with zeros in their place on the tokens' side.
//
// What bounds a large product is how far its requests and its matrix instructions run
// beside each other: of 4096 x 22016 x 4096 the requests alone are 262 us (327 in tiles of
// 256 x 256), the matrix instructions alone 220 to 250, at the clock that random codes
// leave them.  256 x 384 is the largest tile whose sums, operands and two chunks fit: it
// asks for a sixth less, and the whole is 328 to 332 us, 2.2 POP/s (256 x 256: 369; the
// library's product of the codes: 339 to 355).
// Deeper stages of half chunks, and four waves of 128 x 128: no faster.
//
// In a stage, row r's piece p (16 bytes) lies at r * 128 + 16 * (p ^ (r / 2 & 7)):
// the 16 lanes that read a piece of 16 rows together touch every bank once.
template <int BM, int BN, int STAGES>
constexpr int kTileBytes = STAGES * (BM + BN) * kChunk;
template <int BM, int BN, int WM, int WN, int STAGES, int OUT>
__device__ __forceinline__ void tile_product(const Int8Args& a, int m0, int n0, uint8_t* mem) {
  constexpr int kWaves = (BM / WM) * (BN / WN), MS = WM / 32, NS = WN / 32;
  constexpr int kA = BM / 8 / kWaves, kB = BN / 8 / kWaves;  // requests per wave and stage
  constexpr int kStage = (BM + BN) * kChunk;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int col = lane & 31, h = lane >> 5;
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
  // the requests [lo, hi) of chunk c, without a branch around them: as many are on their way at every wait
  const auto request = [&](int c, uint8_t* s, int lo, int hi) {
#pragma unroll
    for (int i = 0; i < kA + kB; ++i) {
      if (i < lo || i >= hi) continue;
      const int j = i < kA ? i : i - kA;
      const uint32_t v = c > last ? kNowhere : at[i] + (c == last ? min(piece(j), left - 16) - piece(j) : 0);
      request_1k(i < kA ? xr : wr, s + (i < kA ? 0 : BM * kChunk) + (j * kWaves + wave) * 1024, v, uint32_t(min(c, last)) * kChunk);
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

  // Chunk c, requested into s, has arrived there for every wave; and every wave has
  // read what it reads of the chunk before.
  const auto arrive = [&](int c, uint8_t* s) {
    __builtin_amdgcn_s_waitcnt(wait_vm((STAGES - 2) * (kA + kB)));  // the chunks behind it may be on their way
    if (c == last && left < kChunk) {
#pragma unroll
      for (int i = 0; i < kA; ++i)
        if (piece(i) >= left) *reinterpret_cast<i4*>(s + (i * kWaves + wave) * 1024 + lane * 16) = i4{0, 0, 0, 0};
    }
    barrier_lds();
  };
  constexpr int kReq = kA + kB;
  const auto read_a = [&](const uint8_t* s, int t, int i) { return *reinterpret_cast<const i4*>(s + (wm + i * 32) * kChunk + from[t]); };
  const auto read_b = [&](const uint8_t* s, int t, int j) { return *reinterpret_cast<const i4*>(s + (BM + wn + j * 32) * kChunk + from[t]); };
  const auto multiply = [&](const i4& x, const i4& w, i16v& to) { to = __builtin_amdgcn_mfma_i32_32x32x32_i8(x, w, to, 0, 0, 0); };
#pragma unroll
  for (int i = 0; i < STAGES - 1; ++i) request(i, mem + i * kStage, 0, kReq);
  arrive(0, mem);
  if constexpr (MS * NS < 8) {
    // Each step's operands are read while the step before is multiplied, and the next
    // chunk is awaited before the last step, so that a chunk begins on operands in
    // registers.
    i4 xa[2][MS], xb[2][NS];
    const auto read = [&](const uint8_t* s, int t, int to) {
#pragma unroll
      for (int j = 0; j < NS; ++j) xb[to][j] = read_b(s, t, j);
#pragma unroll
      for (int i = 0; i < MS; ++i) xa[to][i] = read_a(s, t, i);
    };
    request(STAGES - 1, mem + (STAGES - 1) * kStage, 0, kReq);
    read(mem, 0, 0);
    for (int c = 0;;) {
#pragma unroll
      for (int i = 0; i < STAGES; ++i) {  // the stage's place is a constant of the reads
        uint8_t *const s = mem + i * kStage, *const next = mem + (i + 1) % STAGES * kStage;
#pragma unroll
        for (int t = 0; t < 4; ++t) {
          if (t == 3) {
            arrive(c + 1, next);
            request(c + STAGES, s, 0, kReq);
          }
          read(t < 3 ? s : next, (t + 1) & 3, (t + 1) & 1);
          __builtin_amdgcn_sched_barrier(0);
#pragma unroll
          for (int k = 0; k < MS * NS; ++k) multiply(xa[t & 1][k / NS], xb[t & 1][k % NS], acc[k / NS][k % NS]);
          __builtin_amdgcn_sched_barrier(0);
        }
        if (++c == chunks) goto multiplied;
      }
    }
  } else {
    // Between a step's products, one operand of the next step is read or one piece of a
    // chunk requested at a time: all at once they would wait for each other with the
    // matrix cores idle.  The weights' operands have two places in registers; a token
    // operand's is read into when its last product is on its way, the last one's at the
    // beginning of its own step.  The next chunk is awaited within the last step.
    constexpr int kProducts = MS * NS, kHalf = kReq / 2, kJoin = 2;
    i4 xa[MS], xb[2][NS];
    request(STAGES - 1, mem + (STAGES - 1) * kStage, 0, kHalf);
#pragma unroll
    for (int j = 0; j < NS; ++j) xb[0][j] = read_b(mem, 0, j);
#pragma unroll
    for (int i = 0; i < MS - 1; ++i) xa[i] = read_a(mem, 0, i);
    for (int c = 0;;) {
#pragma unroll
      for (int i = 0; i < STAGES; ++i) {
        uint8_t *const s = mem + i * kStage, *const next = mem + (i + 1) % STAGES * kStage, *const before = mem + (i + STAGES - 1) % STAGES * kStage;
#pragma unroll
        for (int t = 0; t < 4; ++t) {
          // addresses anew at each step: kept, they would take a register for each step and 64 KB
          uint32_t at0 = from[0] ^ t * 32, at1 = from[0] ^ ((t + 1) & 3) * 32;
          asm volatile("" : "+v"(at0), "+v"(at1));
          xa[MS - 1] = *reinterpret_cast<const i4*>(s + (wm + (MS - 1) * 32) * kChunk + at0);
          __builtin_amdgcn_sched_barrier(0);
          // the step's first products come before the next chunk is awaited
          const int first = t == 3 ? kJoin : 0;
          const uint8_t* const from_next = t == 3 ? next : s;
#pragma unroll
          for (int k = 0; k < kProducts; ++k) {
            if (t == 3 && k == kJoin) arrive(c + 1, next);
            multiply(xa[k / NS], xb[t & 1][k % NS], acc[k / NS][k % NS]);
            const int slot = k - first;
            if (slot >= 0 && slot < NS) xb[(t + 1) & 1][slot] = *reinterpret_cast<const i4*>(from_next + (BM + wn + slot * 32) * kChunk + at1);
#pragma unroll
            for (int r = 0; r < MS - 1; ++r)
              if (k == (r * NS + NS - 1 > first + NS - 1 + r ? r * NS + NS - 1 : first + NS - 1 + r)) xa[r] = *reinterpret_cast<const i4*>(from_next + (wm + r * 32) * kChunk + at1);
            if (t == 3 && slot >= 0) request(c + STAGES, s, slot * kHalf / (kProducts - kJoin), (slot + 1) * kHalf / (kProducts - kJoin));
            if (t == 0) request(c + STAGES - 1, before, kHalf + k * (kReq - kHalf) / kProducts, kHalf + (k + 1) * (kReq - kHalf) / kProducts);
            __builtin_amdgcn_sched_barrier(0);
          }
        }
        if (++c == chunks) goto multiplied;
      }
    }
  }
multiplied:
  __builtin_amdgcn_s_waitcnt(wait_vm(0));  // no request into shared memory outlives the workgroup

  const uint32_t es = OUT == kBF16 ? 2 : 4;
  const int have = min(a.M - m0 - wm, WM);
  if (have <= 0) return;
  const __amdgpu_buffer_rsrc_t yr =
      buffer_rsrc(static_cast<uint8_t*>(a.y) + ((m0 + wm) * a.y_stride) * es, uint32_t((have - 1) * a.y_stride + a.N) * es);
  float sw[NS], bias[NS];
#pragma unroll
  for (int j = 0; j < NS; ++j) {
    const int n = min(n0 + wn + j * 32 + col, a.N - 1);
    sw[j] = OUT == kSums ? 0.f : a.s_w[n];
    bias[j] = OUT != kSums && a.bias ? a.bias[n] : 0.f;
  }
#pragma unroll
  for (int i = 0; i < MS; ++i) {
    if (m0 + wm + i * 32 >= a.M) break;
    RowScales<1> rs;
    if constexpr (OUT != kSums) rs = load_row_scales<1>(a.s_x, a.M, m0 + wm + i * 32, h);
#pragma unroll
    for (int j = 0; j < NS; ++j) {
      const int n = n0 + wn + j * 32 + col;
      if (n >= a.N) continue;
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const uint32_t idx = uint32_t(i * 32 + tile_row(e, h)) * uint32_t(a.y_stride) + uint32_t(n);
        if constexpr (OUT == kSums) {
          __builtin_amdgcn_raw_buffer_store_b32(uint32_t(acc[i][j][e]), yr, idx * 4u, 0, 0);
        } else {
          float v = float(acc[i][j][e]) * rs.v[0][e] * sw[j];
          if (a.bias) v += bias[j];
          if constexpr (OUT == kBF16) __builtin_amdgcn_raw_buffer_store_b16(bf16_bits(v), yr, idx * 2u, 0, 0);
          else __builtin_amdgcn_raw_buffer_store_b32(__float_as_uint(v), yr, idx * 4u, 0, 0);
        }
      }
    }
  }
}

// part: chunks of K that a workgroup multiplies.  With OUT = kSums the sums of part p
// go to a.y, an int32 [parts][M][N].
template <int BM, int BN, int WM, int WN, int STAGES, int OUT>
__global__ __launch_bounds__((BM / WM) * (BN / WN) * 64) void gemm_int8_tile(Int8Args a, int m_blocks, int groups, int part) {
  __shared__ __align__(1024) uint8_t mem[kTileBytes<BM, BN, STAGES>];
  int group, mblock, b = blockIdx.x;
  if constexpr (OUT == kSums) {
    const int p = b / (m_blocks * groups);
    b -= p * (m_blocks * groups);
    a.x += int64_t(p) * part * kChunk;
    a.w += int64_t(p) * part * kChunk;
    a.y = static_cast<int32_t*>(a.y) + int64_t(p) * a.M * a.N;
    a.K = min(a.K - p * part * kChunk, part * kChunk);
  }
  square_work(b, groups, m_blocks, group, mblock);
  tile_product<BM, BN, WM, WN, STAGES, OUT>(a, mblock * BM, group * BN, mem);
}

// The sums of the parts, scaled: V neighbouring outputs a thread.
template <int V, bool YB>
__global__ __launch_bounds__(256) void gemm_int8_join(Int8Args a, const int32_t* sums, int parts) {
  const uint32_t per = uint32_t(a.N) / V;
  const uint64_t i = uint64_t(blockIdx.x) * 256 + threadIdx.x;
  const uint32_t m = uint32_t(i / per), n = uint32_t(i - uint64_t(m) * per) * V;
  if (m >= uint32_t(a.M)) return;
  typedef int vec __attribute__((ext_vector_type(V)));
  const int64_t all = int64_t(a.M) * a.N;
  const int32_t* p = sums + int64_t(m) * a.N + n;
  vec s = *reinterpret_cast<const vec*>(p);
  for (int k = 1; k < parts; ++k) s += *reinterpret_cast<const vec*>(p + k * all);
  const float sx = a.s_x[m];
#pragma unroll
  for (int e = 0; e < V; ++e) {
    float y = float(s[e]) * sx * a.s_w[n + e];
    if (a.bias) y += a.bias[n + e];
    store_y(a.y, YB, m * a.y_stride + n + e, y);
  }
}

// ---- few tokens ------------------------------------------------------------
// Up to 32 tokens, whose time is that of the weights' bytes.  A workgroup takes one
// tile of outputs and all tokens after the other; its waves take a tile's 128-byte
// units of K in turn.  Each wave has a ring of three units in shared memory, of which
// two are on their way while one is multiplied, the next tile's among them: it waits
// for the others only where a tile ends, and their sums are added up in shared memory
// by integer atomics.  Whole lines of rows are requested, in the order that spreads
// them over the banks.  (In the operands' own order, straight to registers, lanes
// that follow each other take four rows, which costs the address units three times as
// much: 2.9 TB/s with 16 tokens.)  16 x 22016 x 4096: 17.8 us among other calls, 5.1
// TB/s; 1 x 4096 x 4096: 5.8, of which 3 are the bytes.
//
// 16x16x64: A = 16 rows of W, B = 16 tokens, 16 bytes of K a lane (lane l: row or
// token l & 15, bytes 16 (l >> 4)); the sums leave a lane four outputs of a token.
// XG: groups of 8 tokens.
template <int XG, int NT, int WAVES, bool YB>
__global__ __launch_bounds__(WAVES * 64) void gemm_int8_few(Int8Args a) {
  constexpr int MT = (XG + 1) / 2, NR = NT * 16, kRows = NR + MT * 16;  // rows of a unit in shared memory, weights first
  constexpr int kUnit = (2 * NT + XG) * 1024;  // what a unit requests: the half of a tile of 16 tokens that is not there stays what it was
  constexpr int kRing = WAVES * kUnit + (kRows * kChunk - kUnit);
  __shared__ __align__(1024) uint8_t ring[3 * kRing];
  __shared__ int sums[MT * NT * 4 * 64];  // of all waves: whole numbers, whose order does not matter
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int i16 = lane & 15, g = lane >> 4;
  const int units = (a.K + kChunk - 1) / kChunk, left = a.K - (units - 1) * kChunk;
  const int tiles = (a.N + NR - 1) / NR;
  // this wave's units of a tile: one at least, which past the end of K counts for nothing
  const int per = max((units - wave + WAVES - 1) / WAVES, 1);
  const int mine = per * ((tiles - int(blockIdx.x) + int(gridDim.x) - 1) / int(gridDim.x));

  // Row r's piece p (16 bytes) lies at r * 128 + 16 * (p ^ (r / 2 & 7)); the lanes
  // write their pieces side by side, so they load them in that order.
  const auto piece = [&](int r) { return ((lane & 7) ^ (r >> 1 & 7)) * 16; };
  // the pieces past the end of K are the last piece again
  const auto inside = [&](int unit, uint32_t at, int r) { return unit < units - 1 ? at : at + min(piece(r), left - 16) - piece(r); };

  // the next unit to request, and the lane's place in its tile's rows
  int next_tile = blockIdx.x, next_unit = wave, next_count = 0;
  __amdgpu_buffer_rsrc_t wr;
  uint32_t w_at[2 * NT], x_at[XG];
  const auto w_rows = [&] {
    // rows past the end are the last one again; their results are not stored
    const int outs = min(a.N - next_tile * NR, NR);
    wr = buffer_rsrc(a.w + next_tile * NR * a.w_stride, uint32_t((outs - 1) * a.w_stride + a.K));
#pragma unroll
    for (int i = 0; i < 2 * NT; ++i) w_at[i] = uint32_t(min(i * 8 + (lane >> 3), outs - 1)) * uint32_t(a.w_stride) + piece(i * 8 + (lane >> 3));
  };
  const __amdgpu_buffer_rsrc_t xr = buffer_rsrc(a.x, uint32_t((a.M - 1) * a.x_stride + a.K));
#pragma unroll
  for (int i = 0; i < XG; ++i) x_at[i] = uint32_t(min(i * 8 + (lane >> 3), a.M - 1)) * uint32_t(a.x_stride) + piece(i * 8 + (lane >> 3));
  // Requests have no branch around them, so that as many are on their way at every
  // wait; those past the last unit lie outside the buffer and read nothing.
  const auto request = [&](int j, uint8_t* to) {
    const int unit = min(next_unit, units - 1);
    const uint32_t base = uint32_t(unit) * kChunk;
    to += wave * kUnit;
#pragma unroll
    for (int i = 0; i < 2 * NT; ++i)
      request_1k<kStream>(wr, to + i * 1024, j < mine ? inside(unit, w_at[i], i * 8 + (lane >> 3)) : kNowhere, base);
#pragma unroll
    for (int i = 0; i < XG; ++i)
      request_1k(xr, to + (2 * NT + i) * 1024, j < mine ? inside(unit, x_at[i], i * 8 + (lane >> 3)) : kNowhere, base);
    next_unit += WAVES;
    if (++next_count == per) {
      next_count = 0;
      next_unit = wave;
      if (j + 1 < mine) {
        next_tile += gridDim.x;
        w_rows();
      }
    }
  };

  i4 acc[MT * NT];
#pragma unroll
  for (int t = 0; t < MT * NT; ++t) acc[t] = i4{0, 0, 0, 0};
  uint32_t from[2];
#pragma unroll
  for (int s = 0; s < 2; ++s) from[s] = i16 * kChunk + (((4 * s + g) ^ (i16 >> 1 & 7)) << 4);

  // a wave finishes every WAVES-th tile of 16 outputs by 16 tokens
  int tile = blockIdx.x, unit = wave, count = 0;
  constexpr int kSums = (MT * NT + WAVES - 1) / WAVES;
  float sx[kSums];
#pragma unroll
  for (int i = 0; i < kSums; ++i) {
    const int m = (wave + i * WAVES) / NT * 16 + i16;
    sx[i] = m < a.M ? a.s_x[m] : 0.f;
  }
  // The four values of the lane's outputs, by scalar loads: a vector load would
  // wait for the requests before it.
  const auto of_lane = [&](const float* p, int nt, float (&v)[4]) {
    const __attribute__((address_space(4))) float* q = constant(p);
    float all[16];
    const int first = tile * NR + nt * 16;
    if (first + 16 <= a.N) {
#pragma unroll
      for (int i = 0; i < 16; ++i) all[i] = q[first + i];
    } else {
#pragma unroll
      for (int i = 0; i < 16; ++i) all[i] = q[min(first + i, a.N - 1)];
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = g < 2 ? (g == 0 ? all[e] : all[4 + e]) : (g == 2 ? all[8 + e] : all[12 + e]);
  };
  const auto finish = [&] {
#pragma unroll
    for (int t = 0; t < MT * NT; ++t)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        __hip_atomic_fetch_add(&sums[(t * 4 + e) * 64 + lane], acc[t][e], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
        acc[t][e] = 0;
      }
    barrier_lds();
#pragma unroll
    for (int i = 0; i < kSums; ++i) {
      const int p = wave + i * WAVES, nt = p % NT, m = p / NT * 16 + i16;
      if (p >= MT * NT) break;
      int s[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        s[e] = sums[(p * 4 + e) * 64 + lane];
        sums[(p * 4 + e) * 64 + lane] = 0;
      }
      const int n = tile * NR + nt * 16 + 4 * g;
      float sw[4], bias[4] = {};
      of_lane(a.s_w, nt, sw);
      if (a.bias) of_lane(a.bias, nt, bias);
      if (m < a.M) {
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (n + e < a.N) {
            float y = float(s[e]) * sx[i] * sw[e];
            if (a.bias) y += bias[e];
            store_y(a.y, YB, m * a.y_stride + n + e, y);
          }
      }
    }
    barrier_lds();
    tile += gridDim.x;
    unit = wave;
    count = 0;
  };

  for (int i = threadIdx.x; i < MT * NT * 4 * 64; i += WAVES * 64) sums[i] = 0;
  barrier_lds();
  w_rows();
  request(0, ring);
  request(1, ring + kRing);
  uint8_t *now = ring, *free = ring + 2 * kRing;  // unit j, and where unit j - 1 was
  for (int j = 0; j < mine; ++j) {
    __builtin_amdgcn_s_waitcnt(wait_vm(2 * NT + XG));  // unit j + 1 may be on its way
    __builtin_amdgcn_sched_barrier(0);
    request(j + 2, free);
    __builtin_amdgcn_sched_barrier(0);
    const uint8_t* mem = now + wave * kUnit;
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      i4 b[NT], v[MT];
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        b[t] = *reinterpret_cast<const i4*>(mem + t * 16 * kChunk + from[s]);
        if (unit >= units - 1 && (unit >= units || s * 64 + g * 16 >= left)) b[t] = i4{0, 0, 0, 0};
      }
#pragma unroll
      for (int t = 0; t < MT; ++t) v[t] = *reinterpret_cast<const i4*>(mem + (NT + t) * 16 * kChunk + from[s]);
#pragma unroll
      for (int t = 0; t < MT; ++t)
#pragma unroll
        for (int r = 0; r < NT; ++r) acc[t * NT + r] = __builtin_amdgcn_mfma_i32_16x16x64_i8(b[r], v[t], acc[t * NT + r], 0, 0, 0);
    }
    __builtin_amdgcn_sched_barrier(0);
    free = now;
    now = now + kRing < ring + 3 * kRing ? now + kRing : ring;
    unit += WAVES;
    if (++count == per) finish();
  }
  __builtin_amdgcn_s_waitcnt(wait_vm(0));  // no request into shared memory outlives the workgroup
}

// As many workgroups, up to one a compute unit, as share the tiles evenly.
template <int XG, int NT, int WAVES>
hipError_t few(const Int8Args& a, hipStream_t st) {
  const int tiles = (a.N + 16 * NT - 1) / (16 * NT), turns = (tiles + 255) / 256;
  const dim3 grid(unsigned((tiles + turns - 1) / turns)), block(WAVES * 64);
  if (a.y_bf16) hipLaunchKernelGGL((gemm_int8_few<XG, NT, WAVES, true>), grid, block, 0, st, a);
  else hipLaunchKernelGGL((gemm_int8_few<XG, NT, WAVES, false>), grid, block, 0, st, a);
  return hipGetLastError();
}
// Tiles of 16 to 64 outputs: those that give the busiest compute unit the fewest, and
// of these the widest, which read the tokens the least often.  Captured and back to back
// (the first of these 2.5 us more than among other calls): 16 x 22016 x 4096: 20.1 us
// with 48, 20.8 with 32, 21.0 with 64; 16 x 11008 x 4096: 11.8 with 48, 14.2 with 16;
// 16 x 16384 x 4096: 16.4 with 64, 17.8 with 32; 1 x 4096 x 4096: 5.9 with 16, 7.3 with 32.
int few_width(int64_t N) {
  int wide = 1;
  int64_t least = int64_t(1) << 30;
  for (int nt = 1; nt <= 4; ++nt) {
    const int64_t most = ((N + 16 * nt - 1) / (16 * nt) + 255) / 256 * nt;
    if (most <= least) {
      least = most;
      wide = nt;
    }
  }
  return wide;
}
template <int XG>
hipError_t few_rows(const Int8Args& a, hipStream_t st) {
  switch (few_width(a.N)) {
    case 1: return few<XG, 1, 8>(a, st);
    case 2: return few<XG, 2, 4>(a, st);
    case 3: return few<XG, 3, 4>(a, st);
    default: return few<XG, 4, 4>(a, st);
  }
}

template <int BM, int BN, int WM, int WN, int STAGES>
hipError_t tile(const Int8Args& a, int parts, hipStream_t st) {
  const int mb = (a.M + BM - 1) / BM, nb = (a.N + BN - 1) / BN;
  const dim3 block((BM / WM) * (BN / WN) * 64);
  const auto launch = [&](auto kernel, const Int8Args& args, int k, int part) {
    hipLaunchKernelGGL(kernel, dim3(unsigned(mb) * unsigned(nb) * unsigned(k)), block, 0, st, args, mb, nb, part);
    return hipGetLastError();
  };
  if (parts == 1)
    return a.y_bf16 ? launch(gemm_int8_tile<BM, BN, WM, WN, STAGES, kBF16>, a, 1, 0) : launch(gemm_int8_tile<BM, BN, WM, WN, STAGES, kF32>, a, 1, 0);
  Int8Args sums = a;
  sums.y = a.ws;
  sums.y_stride = a.N;
  const int chunks = (a.K + kChunk - 1) / kChunk, part = (chunks + parts - 1) / parts;
  return launch(gemm_int8_tile<BM, BN, WM, WN, STAGES, kSums>, sums, parts, part);
}

template <int V>
hipError_t join(const Int8Args& a, int parts, hipStream_t st) {
  const dim3 grid(unsigned((int64_t(a.M) * (a.N / V) + 255) / 256)), block(256);
  const int32_t* sums = static_cast<const int32_t*>(a.ws);
  if (a.y_bf16) hipLaunchKernelGGL((gemm_int8_join<V, true>), grid, block, 0, st, a, sums, parts);
  else hipLaunchKernelGGL((gemm_int8_join<V, false>), grid, block, 0, st, a, sums, parts);
  return hipGetLastError();
}

// The forms of tiles, and their times in microseconds: in every round of 256 compute
// units, or twice as many workgroups where two fit, `one` (`two`) a chunk of K and 2
// for its beginning and end.  Measured at 256 to 4096 tokens by 4096 outputs (the wide
// forms: 256 to 16384 by 4096 to 22016), K = 4096 and, where rows are not whole cache
// lines and a chunk of each takes two, 4112.  It counts no weights' bytes from memory: where those
// bound a call, as of 17 to 64 tokens by many outputs, the forms are ranked by their
// chunks alone.  The form taken and the nearest other, calls from Python in a row, at
// K = 4096: 256 x 22016: 35.5 us (256 x 128), 46.3 (two of 128 x 128); 512 x 22016: 56.6
// (256 x 192), 61.9 (128 x 384, dropped); 4096 x 4096: 67 (256 x 256), 77 (256 x 128);
// 2048 x 11008: 84 (256 x 384), 106 (256 x 256); 1024 x 4096: 26 (128 x 128), 32
// (256 x 128).
struct Form { int bm, bn; double one, two, one_odd, two_odd; };
constexpr Form kForms[] = {{64, 64, .22, .46, .30, .63},
                           {64, 128, .42, .80, .53, 1.0},
                           {128, 128, .72, 0, .80, 0},
                           {128, 128, .87, 1.18, 1.04, 1.46},
                           {256, 128, 1.15, 0, 1.3, 0},
                           {256, 192, 1.62, 0, 1.85, 0},
                           {256, 256, 1.85, 0, 2.1, 0},
                           {256, 384, 2.5, 0, 2.9, 0}};

struct Choice { int form, parts; };

// K divided over `parts` workgroups costs a second launch and the sums' way through
// memory: 3 microseconds, and 4 TB/s of them written and read; and it never takes
// less than the host needs for a call of two launches, 9.  (64 x 4096 x 16384:
// 26.6 us undivided, 17.0 in 4 parts; 37 x 51 x 3712, called from Python: 11.2 in
// 4 parts with a workspace of the call's own, 8.5 undivided.)
Choice choose(int64_t M, int64_t N, int64_t K, bool divide) {
  const int chunks = int((K + kChunk - 1) / kChunk);
  Choice best{0, 1};
  double least = 1e30;
  for (int f = 0; f < int(sizeof(kForms) / sizeof(kForms[0])); ++f) {
    const Form& m = kForms[f];
    const int64_t tiles = ((M + m.bm - 1) / m.bm) * ((N + m.bn - 1) / m.bn), round = m.two > 0 ? 512 : 256;
    const double one = K % kChunk ? m.one_odd : m.one, two = round == 256 ? one : K % kChunk ? m.two_odd : m.two;
    for (int parts = 1; parts <= (divide && tiles < 512 ? 16 : 1); ++parts) {
      const int part = (chunks + parts - 1) / parts;
      if (parts > 1 && (part < 4 || (parts - 1) * part >= chunks || tiles * parts > 2 * round)) continue;
      const int64_t all = tiles * parts, rest = all % round;
      const double whole = part * two + 2, some = part * one + 2;
      double t = double(all / round) * whole + (rest == 0 ? 0 : rest <= 256 ? some : whole);
      if (parts > 1) t = std::max(1.1 * (t + 3 + double(M) * double(N) * (8 * parts + 4) / 4e6), 9.0);
      if (t < least) {
        least = t;
        best = {f, parts};
      }
    }
  }
  return best;
}

// Up to 4096 outputs each of 256 compute units has one tile of 16 at most.  Measured
// captured and back to back, K = 4096, this form and tiles: 20 x 512: 6.5 us, 7.3;
// 17 x 4096: 7.2, 9.0;  32 x 4096: 7.8, 10.0;  17 x 5120: 10.3, 9.6;  32 x 5120: 11.4, 9.4;
// 32 x 8192: 12.7, 9.8.
bool few_tokens(int64_t M, int64_t N) { return M <= 16 || (M <= 32 && N <= 4096); }

}  // namespace

size_t gemm_int8_workspace_bytes(int64_t M, int64_t N, int64_t K) {
  if (few_tokens(M, N)) return 0;
  const int parts = choose(M, N, K, true).parts;
  return parts == 1 ? 0 : size_t(M) * size_t(N) * size_t(parts) * 4;
}

void gemm_int8_kernel_name(int64_t M, int64_t N, int64_t K, bool divide, char* out, size_t n) {
  if (few_tokens(M, N)) {
    std::snprintf(out, n, "few %dx%d", M <= 8 ? 8 : M <= 16 ? 16 : 32, M <= 16 ? 16 * few_width(N) : 16);
    return;
  }
  const Choice c = choose(M, N, K, divide);
  const Form& f = kForms[c.form];
  std::snprintf(out, n, "tile %dx%d%s (%d part%s)", f.bm, f.bn, f.two > 0 ? " in pairs" : "", c.parts, c.parts == 1 ? "" : "s");
}

hipError_t launch_gemm_int8(const Int8Args& a, hipStream_t st) {
  if (a.M <= 8) return few_rows<1>(a, st);
  if (a.M <= 16) return few_rows<2>(a, st);
  if (few_tokens(a.M, a.N)) return few<4, 1, 8>(a, st);
  const Choice c = choose(a.M, a.N, a.K, a.ws != nullptr);
  hipError_t e;
  switch (c.form) {
    case 0: e = tile<64, 64, 32, 32, 4>(a, c.parts, st); break;
    case 1: e = tile<64, 128, 32, 32, 3>(a, c.parts, st); break;
    case 2: e = tile<128, 128, 64, 32, 4>(a, c.parts, st); break;
    case 3: e = tile<128, 128, 64, 64, 2>(a, c.parts, st); break;
    case 4: e = tile<256, 128, 128, 64, 3>(a, c.parts, st); break;
    case 5: e = tile<256, 192, 64, 96, 2>(a, c.parts, st); break;
    case 6: e = tile<256, 256, 128, 64, 2>(a, c.parts, st); break;
    default: e = tile<256, 384, 128, 96, 2>(a, c.parts, st); break;
  }
  if (e != hipSuccess || c.parts == 1) return e;
  return a.N % 4 == 0 ? join<4>(a, c.parts, st) : join<1>(a, c.parts, st);
}

}  // namespace sdq
