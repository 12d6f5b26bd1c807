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

// lists: per row the number of moves, the new length, `most` destinations and
// `most` sources.  The new lengths reach lens_out from the second kernel: it may
// be seq_lens, which the workgroups of the other heads still read here.
__global__ __launch_bounds__(kSelect) void evict_select_kernel(EvictArgs a, int32_t* lists, int most) {
  __shared__ uint32_t hist[kDigits];
  __shared__ uint32_t waves[kSelect / 64];
  __shared__ uint32_t pick[2];
  const int row = blockIdx.x, b = row / int(a.kv.heads), tid = threadIdx.x;
  const uint32_t h = row - b * int(a.kv.heads);
  const int n = seq_len(a.seqs, b), keep = min(n, a.budget);
  int32_t* list = lists + int64_t(row) * (2 + 2 * most);
  const bool in_place = a.weight_out == a.kv.weight;
  if (tid == 0) list[1] = keep;
  if (n <= keep) {
    if (tid == 0) list[0] = 0;
    if (!in_place)
      for (int t = tid; t < n; t += kSelect) {
        const Slot s(a.kv, a.seqs, b, h, t);
        if (s.at >= 0) {
          a.weight_out[s.at] = a.kv.weight[s.at];
          a.position_out[s.at] = a.kv.position[s.at];
        }
      }
    return;
  }

  int newest = -1;
  for (int t = tid; t < n; t += kSelect) {
    const Slot s(a.kv, a.seqs, b, h, t);
    if (s.at >= 0) newest = max(newest, a.kv.position[s.at]);
  }
  newest = block_max(newest, reinterpret_cast<int*>(waves));
  // a slot is recent if position > newest - recent; 64 bits, since positions are the caller's
  const int64_t edge = int64_t(newest) - a.recent;
  uint32_t recents = 0;
  for (int t = tid; t < n; t += kSelect) {
    const Slot s(a.kv, a.seqs, b, h, t);
    if (s.at >= 0 && a.kv.position[s.at] > edge) ++recents;
  }
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
    for (int t = tid; t < n; t += kSelect) {
      const Slot s(a.kv, a.seqs, b, h, t);
      const bool recent = s.at >= 0 && a.kv.position[s.at] > edge;
      if (recent != among_recent) continue;
      const uint32_t key = s.at >= 0 ? order_bits(a.kv.weight[s.at]) : 0;
      if (pass == 0 || key >> (shift + bits) == prefix) atomicAdd(&hist[key >> shift & ((1u << bits) - 1)], 1u);
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
  uint32_t eq_seen = 0, holes = 0, movers = 0;
  for (int base = 0; base < n; base += kSelect) {
    const int t = base + tid;
    bool stays = false, is_eq = false;
    int64_t at = -1;
    if (t < n) {
      const Slot s(a.kv, a.seqs, b, h, t);
      at = s.at;
      const bool recent = at >= 0 && a.kv.position[at] > edge;
      if (recent == among_recent) {
        const uint32_t key = at >= 0 ? order_bits(a.kv.weight[at]) : 0;
        is_eq = key == prefix;
        stays = key > prefix || is_eq;
      } else {
        stays = recent;
      }
    }
    if (ties) {
      uint32_t all;
      const uint32_t rank = eq_seen + block_scan(is_eq, waves, all);
      if (is_eq) stays = rank <= want;
      eq_seen += all;
    }
    const bool hole = t < keep && !stays, mover = t >= keep && stays;
    uint32_t all;
    const uint32_t rank = block_scan(uint32_t(hole) | uint32_t(mover) << 16, waves, all);
    if (hole) list[2 + holes + (rank & 0xFFFF) - 1] = t;
    if (mover) list[2 + most + movers + (rank >> 16) - 1] = t;
    holes += all & 0xFFFF;
    movers += all >> 16;
    if (!in_place && t < keep && stays && at >= 0) {
      a.weight_out[at] = a.kv.weight[at];
      a.position_out[at] = a.kv.position[at];
    }
  }
  if (tid == 0) list[0] = int32_t(holes);
  __syncthreads();
  for (uint32_t i = tid; i < holes; i += kSelect) {
    const Slot to(a.kv, a.seqs, b, h, list[2 + i]), of(a.kv, a.seqs, b, h, list[2 + most + i]);
    if (to.at >= 0 && of.at >= 0) {
      a.weight_out[to.at] = a.kv.weight[of.at];
      a.position_out[to.at] = a.kv.position[of.at];
    }
  }
  __syncthreads();
  for (int t = keep + tid; t < n; t += kSelect) {
    const Slot s(a.kv, a.seqs, b, h, t);
    if (s.at >= 0) {
      a.weight_out[s.at] = 0.f;
      a.position_out[s.at] = -1;
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
  evict_select_kernel<<<rows, kSelect, 0, st>>>(a, a.ws, most);
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
