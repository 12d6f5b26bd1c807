// Eviction from the paged cache by accumulated attention weight.
//
// For every sequence longer than the budget and every key head, the budget
// slots that stay are, in this order: the recent ones (position > newest -
// recent), then those of the largest weight; equal weights go to the lowest
// slot.  (If more than the budget are recent, the same order holds among
// them.)  A NaN weight counts as the lowest.
// Slots below the budget that stay are not moved.  The i-th freed slot below
// the budget takes the i-th slot above it that stays, so that the least
// possible is copied and no copy's source is another's destination.
//
// One workgroup selects for one key head of one sequence: a radix selection
// over the weights' bits (three digits, counted in shared memory), then one
// pass in slot order that settles ties and lists what moves by prefix sums.
// Up to 32768 slots are read once and kept in registers (1 to 32 per thread,
// the fewest that hold max_len); beyond, every pass reads them again from the L2.
// A second kernel moves the rows, 16 bytes per lane.
#include <hip/hip_runtime.h>

#include "kv_cache.h"

namespace sdq {
namespace {

constexpr int kSelect = 1024;  // threads of a selecting workgroup
constexpr int kDigits = 2048;  // values of an 11-bit digit

// Bits that order as the weights do, NaN lowest.
__device__ __forceinline__ uint32_t order_bits(float w) {
  if (w != w) return 0;
  w += 0.f;  // -0 and 0 are equal
  const uint32_t u = __float_as_uint(w);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}

struct Slot {
  int64_t at;  // index into [pages][heads][page_size]; -1 for an absent page
  __device__ __forceinline__ Slot(const KV& kv, const Seqs& s, int b, uint32_t h, uint32_t t) {
    const uint32_t pi = kv.per_page.div(t), page = uint32_t(s.table[b * s.stride + pi]);
    at = page < kv.pages ? (int64_t(page) * kv.heads + h) * kv.page_size + (t - pi * kv.page_size) : -1;
  }
};

// Inclusive prefix sum of v over the workgroup; `all` is the total.  Two
// barriers; the scratch may be used again after the next barrier.
__device__ __forceinline__ uint32_t block_scan(uint32_t v, uint32_t* waves, uint32_t& all) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
  for (int k = 1; k < 64; k <<= 1) {
    const uint32_t u = __shfl_up(v, k);
    if (lane >= k) v += u;
  }
  __syncthreads();
  if (lane == 63) waves[wave] = v;
  __syncthreads();
  uint32_t before = 0, sum = 0;
#pragma unroll
  for (int k = 0; k < kSelect / 64; ++k) {
    const uint32_t x = waves[k];
    if (k < wave) before += x;
    sum += x;
  }
  all = sum;
  return v + before;
}

__device__ __forceinline__ int block_max(int v, int* waves) {
#pragma unroll
  for (int k = 32; k; k >>= 1) v = max(v, __shfl_xor(v, k));
  __syncthreads();
  if ((threadIdx.x & 63) == 0) waves[threadIdx.x >> 6] = v;
  __syncthreads();
  int r = waves[0];
#pragma unroll
  for (int k = 1; k < kSelect / 64; ++k) r = max(r, waves[k]);
  return r;
}

// What selection needs of a slot.
struct Slots {
  const EvictArgs& a;
  int b, n;
  uint32_t h;
  __device__ __forceinline__ int64_t at(int t) const { return Slot(a.kv, a.seqs, b, h, t).at; }
  __device__ __forceinline__ int position(int t) const {
    const int64_t i = t < n ? at(t) : -1;
    return i >= 0 ? a.kv.position[i] : INT32_MIN;
  }
  __device__ __forceinline__ uint32_t key(int t) const {
    const int64_t i = t < n ? at(t) : -1;
    return i >= 0 ? order_bits(a.kv.weight[i]) : 0;
  }
};

constexpr int kWaves = kSelect / 64;
constexpr int kBatch = 32;  // steps of kSelect slots that are ranked together

// Exclusive prefix sums of table[0 .. steps * kWaves) in place, plus `seen`,
// which grows by their sum.
__device__ __forceinline__ void scan_table(uint32_t* table, int steps, uint32_t* waves, uint32_t& seen) {
  __syncthreads();
  const int tid = threadIdx.x;
  const uint32_t v = tid < steps * kWaves ? table[tid] : 0;
  uint32_t all;
  const uint32_t incl = block_scan(v, waves, all);
  if (tid < steps * kWaves) table[tid] = seen + incl - v;
  seen += all;
  __syncthreads();
}

// lists: per row the number of moves, the new length, `most` destinations and
// `most` sources.  The new lengths reach lens_out from the second kernel: it may
// be seq_lens, which the workgroups of the other heads still read here.
// KEEP: slots per thread kept in registers; 0: read again in every pass.
// Up to 8 the registers leave room for two workgroups on a compute unit.
template <int KEEP>
__global__ __launch_bounds__(kSelect, KEEP && KEEP <= 8 ? 8 : 4) void evict_select_kernel(EvictArgs a, int32_t* lists, int most) {
  __shared__ uint32_t hist[kDigits];
  __shared__ uint32_t table[kBatch * kWaves];
  __shared__ uint32_t waves[kWaves];
  __shared__ uint32_t pick[2];
  const int row = blockIdx.x, b = row / int(a.kv.heads), tid = threadIdx.x, wave = tid >> 6;
  const uint32_t h = row - b * int(a.kv.heads);
  const int n = seq_len(a.seqs, b), keep = min(n, a.budget);
  const Slots slots{a, b, n, h};
  int32_t* list = lists + int64_t(row) * (2 + 2 * most);
  const bool in_place = a.weight_out == a.kv.weight;
  if (tid == 0) list[1] = keep;
  if (n <= keep) {
    if (tid == 0) list[0] = 0;
    if (!in_place)
      for (int t = tid; t < n; t += kSelect) {
        const int64_t at = slots.at(t);
        if (at >= 0) {
          a.weight_out[at] = a.kv.weight[at];
          a.position_out[at] = a.kv.position[at];
        }
      }
    return;
  }

  const int steps = KEEP ? KEEP : (n + kSelect - 1) / kSelect;
  constexpr int kRegs = KEEP ? KEEP : 1;
  uint32_t key[kRegs];
  uint32_t recent_bits = 0;  // of the thread's slots
  int newest = -1;
  // a slot is recent if position > edge; 64 bits, since positions are the caller's
  int64_t edge;
  uint32_t recents = 0;
  if constexpr (KEEP > 0) {
    int pos[KEEP];
#pragma unroll
    for (int k = 0; k < KEEP; ++k) {
      pos[k] = slots.position(k * kSelect + tid);
      key[k] = slots.key(k * kSelect + tid);
    }
#pragma unroll
    for (int k = 0; k < KEEP; ++k) newest = max(newest, pos[k]);
    newest = block_max(newest, reinterpret_cast<int*>(waves));
    edge = int64_t(newest) - a.recent;
#pragma unroll
    for (int k = 0; k < KEEP; ++k) recent_bits |= uint32_t(k * kSelect + tid < n && pos[k] > edge) << k;
    recents = __popc(recent_bits);
  } else {
    for (int k = 0; k < steps; ++k) newest = max(newest, slots.position(k * kSelect + tid));
    newest = block_max(newest, reinterpret_cast<int*>(waves));
    edge = int64_t(newest) - a.recent;
    for (int k = 0; k < steps; ++k) recents += k * kSelect + tid < n && slots.position(k * kSelect + tid) > edge;
  }
  const auto key_of = [&](int k) { return KEEP ? key[KEEP ? k : 0] : slots.key(k * kSelect + tid); };
  const auto is_recent = [&](int k) {
    if constexpr (KEEP > 0) return bool(recent_bits >> k & 1);
    else return k * kSelect + tid < n && slots.position(k * kSelect + tid) > edge;
  };
  uint32_t total;
  block_scan(recents, waves, total);
  // the class that is only partly kept, and how many of it
  const bool among_recent = total >= uint32_t(keep);
  uint32_t want = among_recent ? keep : keep - total;

  // radix selection of the want-th largest weight of that class
  uint32_t prefix = 0, equal = 0;
  for (int pass = 0; pass < 3; ++pass) {
    const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0, bits = pass == 2 ? 10 : 11;
    for (int i = tid; i < kDigits; i += kSelect) hist[i] = 0;
    __syncthreads();
#pragma unroll kRegs
    for (int k = 0; k < (KEEP ? KEEP : steps); ++k) {
      if (k * kSelect + tid >= n || is_recent(k) != among_recent) continue;
      const uint32_t x = key_of(k);
      if (pass == 0 || x >> (shift + bits) == prefix) atomicAdd(&hist[x >> shift & ((1u << bits) - 1)], 1u);
    }
    __syncthreads();
    // digits from the largest down, two per thread
    const uint32_t d0 = kDigits - 1 - 2 * tid, c0 = hist[d0], c1 = hist[d0 - 1];
    uint32_t all;
    const uint32_t incl = block_scan(c0 + c1, waves, all), before = incl - c0 - c1;
    if (before < want && incl >= want) {
      const bool second = before + c0 < want;
      pick[0] = second ? d0 - 1 : d0;
      pick[1] = second ? before + c0 : before;
    }
    __syncthreads();
    prefix = prefix << bits | pick[0];
    want -= pick[1];
    equal = hist[pick[0]];
    __syncthreads();
  }

  // in slot order: what stays, and what moves
  const bool ties = equal > want;
  const uint64_t below = (uint64_t(1) << (tid & 63)) - 1;
  uint32_t eq_seen = 0, moved = 0, n_holes = 0, n_movers = 0;
  for (int base = 0; base < steps; base += kBatch) {
    const int in_batch = min(kBatch, steps - base);
    if (ties) {
#pragma unroll kRegs
      for (int j = 0; j < (KEEP ? KEEP : in_batch); ++j) {
        const int k = KEEP ? j : base + j;
        const bool eq = k * kSelect + tid < n && is_recent(k) == among_recent && key_of(k) == prefix;
        const uint64_t m = __ballot(eq);
        if ((tid & 63) == 0) table[j * kWaves + wave] = __popcll(m);
      }
      scan_table(table, in_batch, waves, eq_seen);
    }
    uint32_t stay_bits = 0;  // of this batch's slots
#pragma unroll kRegs
    for (int j = 0; j < (KEEP ? KEEP : in_batch); ++j) {
      const int k = KEEP ? j : base + j, t = k * kSelect + tid;
      const bool recent = is_recent(k), cls = t < n && recent == among_recent;
      const uint32_t x = cls ? key_of(k) : 0;
      const bool eq = cls && x == prefix;
      bool stays = cls ? x > prefix || eq : t < n && recent;
      if (ties) {
        const uint64_t m = __ballot(eq);
        if (eq) stays = table[j * kWaves + wave] + __popcll(m & below) < want;
      }
      stay_bits |= uint32_t(stays) << j;
    }
    __syncthreads();
#pragma unroll kRegs
    for (int j = 0; j < (KEEP ? KEEP : in_batch); ++j) {
      const int t = (KEEP ? j : base + j) * kSelect + tid;
      const bool stays = stay_bits >> j & 1;
      const uint64_t holes = __ballot(t < keep && !stays), movers = __ballot(t >= keep && stays);
      if ((tid & 63) == 0) table[j * kWaves + wave] = uint32_t(__popcll(holes)) | uint32_t(__popcll(movers)) << 16;
    }
    moved = 0;
    scan_table(table, in_batch, waves, moved);
#pragma unroll kRegs
    for (int j = 0; j < (KEEP ? KEEP : in_batch); ++j) {
      const int t = (KEEP ? j : base + j) * kSelect + tid;
      const bool stays = stay_bits >> j & 1, hole = t < keep && !stays, mover = t >= keep && stays;
      const uint64_t holes = __ballot(hole), movers = __ballot(mover);
      const uint32_t first = table[j * kWaves + wave];
      if (hole) list[2 + n_holes + (first & 0xFFFF) + __popcll(holes & below)] = t;
      if (mover) list[2 + most + n_movers + (first >> 16) + __popcll(movers & below)] = t;
    }
    n_holes += moved & 0xFFFF;
    n_movers += moved >> 16;
    if (!in_place) {
      for (int j = 0; j < in_batch; ++j) {
        const int t = (base + j) * kSelect + tid;
        const int64_t at = t < keep && (stay_bits >> j & 1) ? slots.at(t) : -1;
        if (at >= 0) {
          a.weight_out[at] = a.kv.weight[at];
          a.position_out[at] = a.kv.position[at];
        }
      }
    }
  }
  if (tid == 0) list[0] = int32_t(n_holes);
  __syncthreads();
  for (uint32_t i = tid; i < n_holes; i += kSelect) {
    const int64_t to = slots.at(list[2 + i]), of = slots.at(list[2 + most + i]);
    if (to >= 0 && of >= 0) {
      a.weight_out[to] = a.kv.weight[of];
      a.position_out[to] = a.kv.position[of];
    }
  }
  __syncthreads();
  for (int t = keep + tid; t < n; t += kSelect) {
    const int64_t at = slots.at(t);
    if (at >= 0) {
      a.weight_out[at] = 0.f;
      a.position_out[at] = -1;
    }
  }
}

// Moves of a row: LPR lanes of 16 bytes per key and value.
template <int LPR>
__global__ __launch_bounds__(256) void evict_move_kernel(EvictArgs a, const int32_t* lists, int most, int per_row) {
  const int row = blockIdx.x / per_row, part = blockIdx.x - row * per_row;
  const int32_t* list = lists + int64_t(row) * (2 + 2 * most);
  const int count = list[0], b = row / int(a.kv.heads), lane = threadIdx.x % LPR;
  const uint32_t h = row - b * int(a.kv.heads), bytes = a.kv.dim * (a.kv.e4m3 ? 1 : 2);
  if (h == 0 && part == 0 && threadIdx.x == 0) a.lens_out[b] = list[1];
  for (int i = part * (256 / LPR) + threadIdx.x / LPR; i < count; i += per_row * (256 / LPR)) {
    const int32_t to = list[2 + i], of = list[2 + most + i];
    const int32_t* table = a.seqs.table + b * a.seqs.stride;
    const uint32_t tp = a.kv.per_page.div(to), fp = a.kv.per_page.div(of);
    const uint32_t tpage = uint32_t(table[tp]), fpage = uint32_t(table[fp]);
    if (tpage >= a.kv.pages || fpage >= a.kv.pages) continue;
    const uint32_t toff = to - tp * a.kv.page_size, foff = of - fp * a.kv.page_size;
    const int64_t dst = tpage * a.kv.page_stride + h * a.kv.head_stride + toff * a.kv.slot_stride;
    const int64_t src = fpage * a.kv.page_stride + h * a.kv.head_stride + foff * a.kv.slot_stride;
    if (lane * 16u < bytes) {
      const uint4 k = *reinterpret_cast<const uint4*>(a.kv.k + src + lane * 16);
      const uint4 v = *reinterpret_cast<const uint4*>(a.kv.v + src + lane * 16);
      *reinterpret_cast<uint4*>(a.kv.k + dst + lane * 16) = k;
      *reinterpret_cast<uint4*>(a.kv.v + dst + lane * 16) = v;
    }
    if (a.kv.e4m3 && lane == 0) {
      const int64_t ts = (int64_t(tpage) * a.kv.heads + h) * a.kv.page_size + toff;
      const int64_t fs = (int64_t(fpage) * a.kv.heads + h) * a.kv.page_size + foff;
      a.kv.k_scale[ts] = a.kv.k_scale[fs];
      a.kv.v_scale[ts] = a.kv.v_scale[fs];
    }
  }
}

// Moves of one row, at most.
int64_t most_moves(int64_t cap, int64_t budget) {
  const int64_t above = cap - budget;
  return above <= 0 ? 0 : above < budget ? above : budget;
}

}  // namespace

size_t cache_evict_workspace_bytes(uint32_t heads_kv, int64_t B, int64_t cap, int64_t budget) {
  return size_t(B) * heads_kv * size_t(2 + 2 * most_moves(cap, budget)) * sizeof(int32_t);
}

hipError_t launch_cache_evict(const EvictArgs& a, hipStream_t st) {
  const int most = int(most_moves(a.seqs.cap, a.budget)), rows = a.seqs.B * int(a.kv.heads);
  if (a.seqs.cap <= kSelect) evict_select_kernel<1><<<rows, kSelect, 0, st>>>(a, a.ws, most);
  else if (a.seqs.cap <= 4 * kSelect) evict_select_kernel<4><<<rows, kSelect, 0, st>>>(a, a.ws, most);
  else if (a.seqs.cap <= 8 * kSelect) evict_select_kernel<8><<<rows, kSelect, 0, st>>>(a, a.ws, most);
  else if (a.seqs.cap <= 32 * kSelect) evict_select_kernel<32><<<rows, kSelect, 0, st>>>(a, a.ws, most);
  else evict_select_kernel<0><<<rows, kSelect, 0, st>>>(a, a.ws, most);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const uint32_t bytes = a.kv.dim * (a.kv.e4m3 ? 1 : 2);
  const int lpr = bytes <= 128 ? 8 : bytes <= 256 ? 16 : 32, per_block = 256 / lpr;
  int per_row = most > 0 ? (most + per_block - 1) / per_block : 1;
  // rows enough to fill the GPU take fewer workgroups each
  const int fill = (256 * 16 + rows - 1) / rows;
  if (per_row > fill) per_row = fill;
  const dim3 grid(uint32_t(rows) * per_row);
  if (lpr == 8) evict_move_kernel<8><<<grid, 256, 0, st>>>(a, a.ws, most, per_row);
  else if (lpr == 16) evict_move_kernel<16><<<grid, 256, 0, st>>>(a, a.ws, most, per_row);
  else evict_move_kernel<32><<<grid, 256, 0, st>>>(a, a.ws, most, per_row);
  return hipGetLastError();
}

}  // namespace sdq
