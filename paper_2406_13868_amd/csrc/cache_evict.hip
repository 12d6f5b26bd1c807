// Eviction from the paged cache by accumulated attention weight.
//
// For every sequence longer than the budget and every key head, the budget
// slots that stay are, in this order: the recent ones (position > newest -
// recent), then those of the largest weight; equal weights go to the lowest
// slot.  (If more than the budget are recent, the same order holds among
// them.)  A NaN weight counts as the lowest.  Slots on absent pages take no part:
// they are never kept, and those below the budget are no places, so that as many
// slots stay as there are present ones below the budget.
// Slots below the budget that stay are not moved.  The i-th freed slot below
// the budget takes the i-th slot above it that stays, so that the least
// possible is copied and no copy's source is another's destination.
//
// One workgroup selects for one key head of one sequence: a radix selection
// over the weights' bits (three digits, counted in shared memory), then one
// pass in slot order that settles ties and lists what moves by prefix sums.
// Up to 16384 slots are read once and kept in registers (1, 4, 8 or 16 per thread,
// the fewest that hold max_len), up to 32768 in shared memory (one sequence of
// 31853 slots, 4 key heads: 70 us, read again 106); beyond, every pass reads them
// again from the L2, eight per thread at a time (40000 slots: 129 us).
// It moves the rows too where that is the faster way; otherwise a second kernel
// does, 16 bytes per lane.
//
// What bounds it: the moved bytes at the rate of a copy where many rows move (32
// sequences x 32 heads of 8192 slots halved, 2.1 GB read and written: 430 us, 5.0
// TB/s, beside a selection of 70 that overlaps it, 485 in all); the selection's
// chain of loads, counts and barriers where few do (641 slots: 7.6 us, of which 1.3
// until the weights are there, 1.4 for two digits, 0.7 to list the moves, 0.6 to
// write weights and positions, 2.1 to move rows; 16 x 8 rows of up to 4099 slots
// 15, and 11 in the second kernel).
#include <hip/hip_runtime.h>

#include "kv_cache.h"

namespace sdq {
namespace {

constexpr int kSelect = 1024;  // threads of a selecting workgroup
constexpr int kDigits = 2048;  // values of an 11-bit digit

// Bits that order as the weights do, NaN lowest; 0 is left for absent slots.
__device__ __forceinline__ uint32_t order_bits(float w) {
  if (w != w) return 1;
  w += 0.f;  // -0 and 0 are equal
  const uint32_t u = __float_as_uint(w);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}

constexpr int kWaves = kSelect / 64;

// Inclusive prefix sum of v over the workgroup; `all` is the total.  One
// barrier: the scratch (kWaves words) is free again after the next one.
__device__ __forceinline__ uint32_t block_scan(uint32_t v, uint32_t* waves, uint32_t& all) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  v = wave_scan(v);
  if (lane == 63) waves[wave] = v;
  __syncthreads();
  uint32_t before = 0, sum = 0;
#pragma unroll
  for (int k = 0; k < kWaves; ++k) {
    const uint32_t x = waves[k];
    if (k < wave) before += x;
    sum += x;
  }
  all = sum;
  return v + before;
}

__device__ __forceinline__ int block_max(int v, uint32_t* waves) {
  v = max(v, __builtin_amdgcn_update_dpp(v, v, 0x111, 0xF, 0xF, false));  // row_shr:1
  v = max(v, __builtin_amdgcn_update_dpp(v, v, 0x112, 0xF, 0xF, false));
  v = max(v, __builtin_amdgcn_update_dpp(v, v, 0x114, 0xF, 0xF, false));
  v = max(v, __builtin_amdgcn_update_dpp(v, v, 0x118, 0xF, 0xF, false));
  v = max(v, __builtin_amdgcn_update_dpp(v, v, 0x142, 0xA, 0xF, false));  // row_bcast:15
  v = max(v, __builtin_amdgcn_update_dpp(v, v, 0x143, 0xC, 0xF, false));  // row_bcast:31
  if ((threadIdx.x & 63) == 63) waves[threadIdx.x >> 6] = uint32_t(v);
  __syncthreads();
  int r = int(waves[0]);
#pragma unroll
  for (int k = 1; k < kWaves; ++k) r = max(r, int(waves[k]));
  return r;
}

// Where a sequence's slots lie: index into [pages][heads][page_size], -1 for an
// absent page; `place`: page * page_size + offset, also -1 then.
struct Slots {
  const KV& kv;
  const int32_t* table;
  uint32_t h;
  __device__ __forceinline__ int64_t at(uint32_t t, int32_t& place) const {
    const uint32_t pi = kv.per_page.div(t), page = uint32_t(table[pi]), off = t - pi * kv.page_size;
    const bool there = page < kv.pages;
    place = there ? int32_t(page * kv.page_size + off) : -1;
    return there ? (int64_t(page) * kv.heads + h) * kv.page_size + off : -1;
  }
  __device__ __forceinline__ int64_t at(uint32_t t) const {
    int32_t place;
    return at(t, place);
  }
};

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

typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;

// Rows pass through once: loads and stores leave the caches to others (32 x 8192
// slots 515 us, without the hint 525).
__device__ __forceinline__ u32x4 stream_load(const uint8_t* p) {
  return __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(p));
}
__device__ __forceinline__ void stream_store(uint8_t* p, u32x4 v) {
  __builtin_nontemporal_store(v, reinterpret_cast<u32x4*>(p));
}

// Moves first + i, first + i + step, ... of the list, i being the thread's index
// over 2^lpr_log.
__device__ __forceinline__ void move_rows(const EvictArgs& a, const int2* list, int count, uint32_t h, int lpr_log, int first,
                                          int step) {
  const int lane = threadIdx.x & ((1 << lpr_log) - 1);
  const uint32_t bytes = a.kv.dim * (a.kv.e4m3 ? 1 : 2);
  for (int i = first + int(threadIdx.x >> lpr_log); i < count; i += step) {
    const int2 move = list[i];
    if (move.x < 0 || move.y < 0) continue;
    const uint32_t tpage = a.kv.per_page.div(move.x), fpage = a.kv.per_page.div(move.y);
    const uint32_t toff = move.x - tpage * a.kv.page_size, foff = move.y - fpage * a.kv.page_size;
    const int64_t dst = tpage * a.kv.page_stride + h * a.kv.head_stride + toff * a.kv.slot_stride;
    const int64_t src = fpage * a.kv.page_stride + h * a.kv.head_stride + foff * a.kv.slot_stride;
    if (lane * 16u < bytes) {
      const u32x4 k = stream_load(a.kv.k + src + lane * 16);
      const u32x4 v = stream_load(a.kv.v + src + lane * 16);
      stream_store(a.kv.k + dst + lane * 16, k);
      stream_store(a.kv.v + dst + lane * 16, v);
    }
    if (a.kv.e4m3 && lane == 0) {
      const int64_t ts = (int64_t(tpage) * a.kv.heads + h) * a.kv.page_size + toff;
      const int64_t fs = (int64_t(fpage) * a.kv.heads + h) * a.kv.page_size + foff;
      a.kv.k_scale[ts] = a.kv.k_scale[fs];
      a.kv.v_scale[ts] = a.kv.v_scale[fs];
    }
  }
}

// lists: per row the number of moves, the new length, and `most` pairs of the
// places of a destination and a source: the mover need not wait for the table.  `alone`: the workgroup moves its rows itself and
// writes the new length.  Otherwise both are the second kernel's, which is also
// where lens_out overlaps seq_lens: other workgroups still read it here.
// KEEP: slots per thread kept in registers, up to 8 of which leave room for two
// workgroups on a compute unit.  kShared: 32 of them, the keys in shared memory
// (in registers they spill).  0: read again in every pass.
constexpr int kShared = 32;
template <int SLOTS>
__global__ __launch_bounds__(kSelect, SLOTS && SLOTS <= 8 ? 8 : 4) void evict_select_kernel(EvictArgs a, int2* lists, int most, bool alone, int lpr_log) {
  constexpr int KEEP = SLOTS == kShared ? 0 : SLOTS;
  __shared__ uint32_t key_of[SLOTS == kShared ? kShared : 1][kSelect];  // each thread's own
  __shared__ uint32_t hist[3][kDigits];
  __shared__ uint32_t table[(KEEP ? KEEP : 8) * kWaves];
  __shared__ uint32_t waves[7][kWaves];
  __shared__ uint32_t pick[3][3];
  __shared__ int32_t hole_slot[KEEP ? KEEP * kSelect / 2 : 1];  // at most half the slots move
  const int row = blockIdx.x, b = row / int(a.kv.heads), tid = threadIdx.x, wave = tid >> 6;
  const int n = seq_len(a.seqs, b), keep = min(n, a.budget);
  const Slots slots{a.kv, a.seqs.table + b * a.seqs.stride, uint32_t(row - b * int(a.kv.heads))};
  int2* list = lists + int64_t(row) * (1 + most);
  const bool in_place = a.weight_out == a.kv.weight;
  if (alone && tid == 0 && slots.h == 0) a.lens_out[b] = keep;
  if (n <= keep) {
    if (tid == 0) list[0] = make_int2(0, keep);
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

  // the thread's slots are k * kSelect + tid; those on absent pages have the key 0
  // and are not recent
  const int steps = KEEP ? KEEP : (n + kSelect - 1) / kSelect;
  constexpr int kRegs = KEEP ? KEEP : 8;
  constexpr int kNone = INT32_MIN;
  uint32_t keys[kRegs];
  uint32_t recent_bits = 0, recent_all = 0;
  uint32_t lost = 0;  // of the thread's slots below the budget: those on absent pages
  int edge = kNone;   // a slot is recent if position > edge
  const auto load = [&](int base, int (&p)[kRegs], bool with_keys) {
#pragma unroll
    for (int k = 0; k < kRegs; ++k) {
      const int t = (base + k) * kSelect + tid;
      const int64_t at = t < n ? slots.at(t) : -1, of = at >= 0 ? at : 0;
      p[k] = a.kv.position[of];
      if (with_keys) keys[k] = order_bits(a.kv.weight[of]);
      if (at < 0) p[k] = kNone, keys[k] = 0;
      lost += at < 0 && t < keep;
    }
  };
  const auto set_recent = [&](const int (&p)[kRegs]) {
    recent_bits = 0;
#pragma unroll
    for (int k = 0; k < kRegs; ++k) recent_bits |= uint32_t(p[k] > edge) << k;
  };
  // f(base) for every kRegs of the thread's slots, with their keys and recency
  const auto each = [&](auto f) {
    if constexpr (KEEP > 0) {
      f(0);
    } else {
      for (int base = 0; base < steps; base += kRegs) {
        if constexpr (SLOTS == kShared) {
#pragma unroll
          for (int k = 0; k < kRegs; ++k) keys[k] = key_of[base + k][tid];
          recent_bits = recent_all >> base;
        } else {
          int p[kRegs];
          load(base, p, true);
          set_recent(p);
        }
        f(base);
      }
    }
  };

  for (int i = tid; i < 3 * kDigits; i += kSelect) hist[0][i] = 0;
  if (tid < 9) pick[tid / 3][tid % 3] = 0;  // what it stays where no slot has a place
  int newest = -1;
  uint32_t recents = 0, absent, total, all_absent;
  if constexpr (SLOTS == kShared) {
    int p[kShared / kRegs][kRegs];
#pragma unroll
    for (int g = 0; g < kShared / kRegs; ++g) {
      load(g * kRegs, p[g], true);
#pragma unroll
      for (int k = 0; k < kRegs; ++k) {
        key_of[g * kRegs + k][tid] = keys[k];
        newest = max(newest, p[g][k]);
      }
    }
    newest = block_max(newest, waves[0]);
    edge = int(max(int64_t(newest) - a.recent, int64_t(kNone)));
#pragma unroll
    for (int g = 0; g < kShared / kRegs; ++g) {
      set_recent(p[g]);
      recent_all |= recent_bits << (g * kRegs);
    }
    recents = __popc(recent_all);
    absent = lost;
  } else {
    int p[kRegs];
    for (int base = 0; base < steps; base += kRegs) {
      load(base, p, KEEP > 0);
#pragma unroll
      for (int k = 0; k < kRegs; ++k) newest = max(newest, p[k]);
    }
    absent = lost;  // later passes load the same slots again
    newest = block_max(newest, waves[0]);
    edge = int(max(int64_t(newest) - a.recent, int64_t(kNone)));
    if constexpr (KEEP > 0) {
      set_recent(p);
      recents = __popc(recent_bits);
    } else {
      for (int base = 0; base < steps; base += kRegs) {
        load(base, p, false);
        set_recent(p);
        recents += __popc(recent_bits);
      }
    }
  }
  if constexpr (SLOTS > 0) {  // up to 32768 slots: both counts in one word
    block_scan(recents | absent << 16, waves[1], total);
    all_absent = total >> 16;
    total &= 0xFFFF;
  } else {
    block_scan(recents, waves[1], total);
    block_scan(absent, waves[6], all_absent);
  }
  // how many stay, the class that is only partly kept, and how many of it
  const uint32_t places = uint32_t(keep) - all_absent;
  const bool among_recent = total >= places;
  uint32_t want = among_recent ? places : places - total;

  // radix selection of the want-th largest weight of that class
  uint32_t prefix = 0, equal = 0;
#pragma unroll
  for (int pass = 0; pass < 3; ++pass) {
    const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0, bits = pass == 2 ? 10 : 11;
    // all of the digit's class stay: no need to look further (a third of the
    // passes with weights that differ)
    if (pass > 0 && equal == want) {
      prefix <<= bits;
      continue;
    }
    each([&](int base) {
#pragma unroll
      for (int k = 0; k < kRegs; ++k) {
        if ((base + k) * kSelect + tid >= n || bool(recent_bits >> k & 1) != among_recent) continue;
        if (pass == 0 || keys[k] >> (shift + bits) == prefix) atomicAdd(&hist[pass][keys[k] >> shift & ((1u << bits) - 1)], 1u);
      }
    });
    __syncthreads();
    // digits from the largest down, two per thread
    const uint32_t d0 = kDigits - 1 - 2 * tid, c0 = hist[pass][d0], c1 = hist[pass][d0 - 1];
    uint32_t all;
    const uint32_t incl = block_scan(c0 + c1, waves[2 + pass], all), before = incl - c0 - c1;
    if (before < want && incl >= want) {
      const bool second = before + c0 < want;
      pick[pass][0] = second ? d0 - 1 : d0;
      pick[pass][1] = second ? before + c0 : before;
      pick[pass][2] = second ? c1 : c0;
    }
    __syncthreads();
    prefix = prefix << bits | pick[pass][0];
    want -= pick[pass][1];
    equal = pick[pass][2];
  }

  if (places == 0) prefix = ~0u;  // above every key

  // in slot order, kRegs steps of the workgroup at a time: what stays, and what moves
  const bool ties = equal > want;
  const uint64_t below = (uint64_t(1) << (tid & 63)) - 1;
  uint32_t eq_seen = 0, n_moves = 0, n_sources = 0;
  each([&](int base) {
    uint32_t eq_bits = 0, stay_bits = 0;
#pragma unroll
    for (int k = 0; k < kRegs; ++k) {
      const bool live = (base + k) * kSelect + tid < n, recent = recent_bits >> k & 1;
      if (recent == among_recent) {
        eq_bits |= uint32_t(live && keys[k] == prefix) << k;
        stay_bits |= uint32_t(live && keys[k] >= prefix) << k;
      } else {
        stay_bits |= uint32_t(live && recent) << k;
      }
    }
    if (ties) {
#pragma unroll
      for (int k = 0; k < kRegs; ++k) {
        const uint64_t m = __ballot(eq_bits >> k & 1);
        if ((tid & 63) == 0) table[k * kWaves + wave] = __popcll(m);
      }
      scan_table(table, kRegs, waves[5], eq_seen);
#pragma unroll
      for (int k = 0; k < kRegs; ++k) {
        const uint64_t m = __ballot(eq_bits >> k & 1);
        if ((eq_bits >> k & 1) && table[k * kWaves + wave] + __popcll(m & below) >= want) stay_bits &= ~(1u << k);
      }
      __syncthreads();
    }
    if (all_absent) {  // those below the budget are no holes
#pragma unroll
      for (int k = 0; k < kRegs; ++k) stay_bits |= uint32_t(keys[k] == 0 && (base + k) * kSelect + tid < keep) << k;
    }
#pragma unroll
    for (int k = 0; k < kRegs; ++k) {
      const int t = (base + k) * kSelect + tid;
      const bool stays = stay_bits >> k & 1;
      const uint64_t holes = __ballot(t < keep && !stays), sources = __ballot(t >= keep && stays);
      if ((tid & 63) == 0) table[k * kWaves + wave] = uint32_t(__popcll(holes)) | uint32_t(__popcll(sources)) << 16;
    }
    uint32_t counts = 0;
    scan_table(table, kRegs, waves[6], counts);
#pragma unroll
    for (int k = 0; k < kRegs; ++k) {
      const int t = (base + k) * kSelect + tid;
      const bool hole = t < keep && !(stay_bits >> k & 1);
      const uint64_t holes = __ballot(hole);
      const uint32_t i = n_moves + (table[k * kWaves + wave] & 0xFFFF) + __popcll(holes & below);
      if (hole) {
        if constexpr (KEEP > 0) hole_slot[i] = t;
        else list[1 + i].x = t;  // until its source is found
      }
    }
    __syncthreads();
    // Positions and weights: to the slot that stays or takes this one, and the
    // lowest value to what is given up.  Every slot is read by its own thread
    // before it is written, but for the freed ones, which are not read.  Four
    // slots at a time: all are requested before the first is written.
    constexpr int kFour = KEEP == 1 ? 1 : 4;
#pragma unroll
    for (int k0 = 0; k0 < kRegs; k0 += kFour) {
      int64_t at[kFour], to[kFour];
      float w[kFour];
      int p[kFour];
#pragma unroll
      for (int q = 0; q < kFour; ++q) {
        const int k = k0 + q, t = (base + k) * kSelect + tid;
        const bool stays = stay_bits >> k & 1, source = t >= keep && stays;
        const uint64_t sources = __ballot(source);
        const uint32_t i = n_sources + (table[k * kWaves + wave] >> 16) + __popcll(sources & below);
        int2 move = make_int2(-1, -1);
        at[q] = t < n ? slots.at(t, move.y) : -1;
        to[q] = t < keep && stays && !in_place ? at[q] : -1;
        if (source) {
          to[q] = slots.at(KEEP ? hole_slot[KEEP ? i : 0] : list[1 + i].x, move.x);
          list[1 + i] = move;
        }
        const int64_t of = at[q] >= 0 && to[q] >= 0 ? at[q] : 0;
        w[q] = a.kv.weight[of];
        p[q] = a.kv.position[of];
      }
#pragma unroll
      for (int q = 0; q < kFour; ++q) {
        if (at[q] < 0) continue;
        if (to[q] >= 0) {
          a.weight_out[to[q]] = w[q];
          a.position_out[to[q]] = p[q];
        }
        if ((base + k0 + q) * kSelect + tid >= keep) {
          a.weight_out[at[q]] = 0.f;
          a.position_out[at[q]] = -1;
        }
      }
    }
    n_moves += counts & 0xFFFF;
    n_sources += counts >> 16;
    if constexpr (KEEP == 0) __syncthreads();  // the next steps write the table
  });
  if (tid == 0) list[0] = make_int2(int(n_moves), keep);
  if (alone) {
    __syncthreads();
    move_rows(a, list + 1, int(n_moves), slots.h, lpr_log, 0, kSelect >> lpr_log);
  }
}

// 2^lpr_log lanes of 16 bytes per key and value: the smallest that hold a row.
__global__ __launch_bounds__(256) void evict_move_kernel(EvictArgs a, const int2* lists, int most, int per_row, int lpr_log) {
  const int row = blockIdx.x / per_row, part = blockIdx.x - row * per_row, b = row / int(a.kv.heads);
  const uint32_t h = row - b * int(a.kv.heads);
  const int2* list = lists + int64_t(row) * (1 + most);
  const int2 head = list[0];
  if (h == 0 && part == 0 && threadIdx.x == 0) a.lens_out[b] = head.y;
  const int per_block = 256 >> lpr_log;
  move_rows(a, list + 1, head.x, h, lpr_log, part * per_block, per_row * per_block);
}

// Moves of one row, at most.
int64_t most_moves(int64_t cap, int64_t budget) {
  const int64_t above = cap - budget;
  return above <= 0 ? 0 : above < budget ? above : budget;
}

}  // namespace

size_t cache_evict_workspace_bytes(uint32_t heads_kv, int64_t B, int64_t cap, int64_t budget) {
  return size_t(B) * heads_kv * size_t(1 + most_moves(cap, budget)) * sizeof(int2);
}

hipError_t launch_cache_evict(const EvictArgs& a, hipStream_t st) {
  int2* const ws = reinterpret_cast<int2*>(a.ws);
  const int most = int(most_moves(a.seqs.cap, a.budget)), rows = a.seqs.B * int(a.kv.heads);
  const uint32_t bytes = a.kv.dim * (a.kv.e4m3 ? 1 : 2);
  const int lpr_log = bytes <= 128 ? 3 : bytes <= 256 ? 4 : 5, per_block = 256 >> lpr_log;
  // The selecting workgroup moves its own rows where few do, which costs less than
  // a second launch (us, with one in brackets; dim 128, bf16): at most 256 moves,
  // 1 row 8.2 (8.6), 64 rows 10.7 (11.4), 256 rows 16.6 (19.3); of 384 moves 1 row
  // 11.6 (11.0), 64 rows 16.3 (15.4), 112 rows 18.2 (18.2), 128 rows 18.4 (18.5), 160
  // rows 19.4 (21.4); of 512 moves 96 rows 21.2 (19.4), 128 rows 22.2 (21.9), 160 rows
  // 24.0 (24.0), 192 rows 25.4 (27.4).
  // With more moves it is a matter of the rows alone: 128 keep half of the compute
  // units, 192 and more enough of them, and some rows are selected while others
  // move.  Up to 4000 slots, 2000 moves: 128 rows 41.4 (40.1), 160 rows
  // 46.0 (47.7), 192 rows 52.1 (54.6), 256 rows 66.3 (69.0); 8000 slots, 4000 moves:
  // 78.0 (73.8), 87.3 (87.8), 99.8 (102.8), 130 (133), and 1024 rows 490 (507); 16000
  // slots, 8000 moves: 153 (144), 173 (171), 196 (201), 250 (256); 24000 slots, dim 64,
  // 256 rows 227 (229).  e4m3, 8000 slots: 160 rows 62.0 (58.5), 192 rows 66.0 (66.0),
  // 224 rows 70.5 (74.3).
  // It writes lens_out while other workgroups read seq_lens: not where they overlap.
  const bool apart = a.lens_out + a.seqs.B <= a.seqs.lens || a.seqs.lens + a.seqs.B <= a.lens_out;
  const bool alone = (most <= (rows >= 128 ? 512 : 256) || rows >= 192) && apart;
  if (a.seqs.cap <= kSelect) evict_select_kernel<1><<<rows, kSelect, 0, st>>>(a, ws, most, alone, lpr_log);
  else if (a.seqs.cap <= 4 * kSelect) evict_select_kernel<4><<<rows, kSelect, 0, st>>>(a, ws, most, alone, lpr_log);
  else if (a.seqs.cap <= 8 * kSelect) evict_select_kernel<8><<<rows, kSelect, 0, st>>>(a, ws, most, alone, lpr_log);
  else if (a.seqs.cap <= 16 * kSelect) evict_select_kernel<16><<<rows, kSelect, 0, st>>>(a, ws, most, alone, lpr_log);
  else if (a.seqs.cap <= kShared * kSelect) evict_select_kernel<kShared><<<rows, kSelect, 0, st>>>(a, ws, most, alone, lpr_log);
  else evict_select_kernel<0><<<rows, kSelect, 0, st>>>(a, ws, most, alone, lpr_log);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || alone) return e;
  int per_row = most > 0 ? (most + per_block - 1) / per_block : 1;
  // rows enough to fill the GPU take fewer workgroups each
  const int fill = (256 * 16 + rows - 1) / rows;
  if (per_row > fill) per_row = fill;
  evict_move_kernel<<<uint32_t(rows) * per_row, 256, 0, st>>>(a, ws, most, per_row, lpr_log);
  return hipGetLastError();
}

}  // namespace sdq
