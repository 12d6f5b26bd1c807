// Attention of one new token per sequence over the paged cache.
//
// For sequence b, query head h (of key head h / group) and its slots t < len:
//   z_t = scale * q . k_t,  p_t = exp(z_t - max z) / sum,  out = sum_t p_t v_t
//   lse = log sum_t exp z_t,   weight_out[t] = weight_in[t] + sum over the
//   key head's query heads of p_t
// A row without a slot gives zeros and lse = -inf.
//
// Work.  The unit is a chunk of 128 or 256 slots of one row (a tile of 32 or 64
// for each of four waves), a row being a key head of a sequence with up to 16
// of its query heads.  The chunks of all rows, in order, are divided evenly over
// the workgroups, so ragged lengths leave none idle and a single long row uses
// all of them.  A workgroup walks its range row by row; a row that lies wholly in
// the range is finished there, of any other a partial result (maximum, sum and
// unnormalized output of each head) goes to the workspace, and a second kernel
// joins the partials of each row in the order of their workgroups, so that
// results do not depend on timing.  (Joined by the last workgroup of a row to
// finish instead, the write-back and invalidation of the L2s that such a
// handover takes cost more than the launch: one sequence of 4000 slots, 32/8
// heads, 54 us against 12.)
//
// Matrix instructions (16x16x32 bf16).  Scores: A = 16 keys, B = the row's query
// heads.  The score of 16 keys x 16 heads leaves each lane 4 keys of one head,
// and two such tiles give the 8 keys per lane that the second product's B
// operand wants, in the key order (g * 4 .. + 3, 16 + g * 4 .. + 3) for lane
// group g.  Values: a lane loads, for the 8 keys of its group, VPL dimensions
// (value_dim); pairs of keys are put together with byte permutes, and VPL
// products follow, one for each dimension of a lane.  The operations are a part
// of what the compute units do in the time the cache takes to arrive (with e4m3,
// 270 vector and 24 matrix instructions per 8 KiB: vector units 39% busy, matrix
// cores 12%), also with one query head in 16 columns, so one kernel serves every
// head layout.
//
// What bounds it: the cache's bytes.  A plain streaming read reaches 6.9 TB/s.
// 64 ragged sequences of up to 8192 e4m3 slots, 32 heads (2.2 GB): 329 us, 6.7
// TB/s; one sequence of 131071 slots, 32/8 heads, bf16 (537 MB): 82 us, 6.6, and
// 4.6 in the second kernel.  Short calls are launches and latency: 100 slots 5.6
// us, of which 0.9 pass until the lengths are there, 0.6 until the page numbers
// and 1.4 until the first keys.
//
// Precision.  e4m3 codes are exact in bf16; their scales are applied in fp32 to
// the scores and to p.  bf16 queries are exact; fp32 queries are three bf16
// terms (24 bits).  p is the sum of two bf16 terms (17 bits, for outputs that
// are rounded to bf16) or three (fp32).  Products accumulate in fp32; maximum,
// sum and joins are fp32.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <type_traits>

#include "kv_cache.h"
#include "tile_out.h"

namespace sdq {
namespace {

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;
typedef __attribute__((ext_vector_type(2))) uint32_t u32x2;

constexpr int kMostGroups = 512;    // workgroups, at most, where rows are split
constexpr int kWholeGroups = 4096;  // and where they are not
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr float kNegInf = -__builtin_huge_valf();

struct Plan {
  uint32_t rows;      // rows per sequence: heads * row groups
  uint32_t hgroups;   // row groups per key head: ceil(group / 16)
  uint32_t gh;        // query heads per row, at most (the stride of the partials)
  uint32_t groups;    // workgroups launched
  uint32_t chunk_log; // log2 of the slots per chunk
  uint32_t head;      // what a row costs beside its chunks, in chunks
  bool whole;         // rows are not split
  bool weigh;         // tracked, and a row's workgroup adds its attention weights itself
  int64_t score_ld;   // floats between the scores of two query heads
  uint32_t part_ld;   // floats per partial result: o[gh][dim], m[gh], l[gh], in whole cache lines
  float* part;        // [groups][2][part_ld]
  float* lse2;        // [B][heads_q]: log2 of the sum, for the rows finished in one workgroup
  float* scores;      // [B][heads_q][score_ld], log2 units; tracked calls only
};

// Slots per wave and tile, and waves per SIMD that the registers are held to.
constexpr int tile_slots(int dp, bool f32) { return dp == 64 && !f32 ? 64 : 32; }
constexpr int occupancy(int dp, bool f32, bool p16) { return dp > 128 ? 1 : f32 || !p16 ? 2 : 3; }

__host__ __device__ __forceinline__ int chunks_of(int len, int chunk_log) {
  const int n = (len + (1 << chunk_log) - 1) >> chunk_log;
  return n > 1 ? n : 1;
}

// The chunks of the rows of all sequences, sequences in order: `rows` rows each,
// and `head` units before the chunks of each row.
// A wave's lanes hold 64 sequences at a time; the first 64 stay in registers.
struct Chunks {
  const Seqs& s;
  int cl, rows, head, lane, mine, upto, total;
  __device__ __forceinline__ int of(int b) const { return b < s.B ? (head + chunks_of(seq_len(s, b), cl)) * rows : 0; }
  __device__ __forceinline__ Chunks(const Seqs& seqs, const Plan& p, int l)
      : s(seqs), cl(p.chunk_log), rows(p.rows), head(p.head), lane(l) {
    mine = of(lane);
    upto = wave_scan(mine);
    total = __builtin_amdgcn_readlane(upto, 63);
    for (int base = 64; base < s.B; base += 64) total += __builtin_amdgcn_readlane(wave_scan(of(base + lane)), 63);
  }
  // The sequence that chunk c < total belongs to, and its first chunk.
  __device__ __forceinline__ void find(int c, int& b, int& first) const {
    int before = 0, v = mine, incl = upto;
    for (int base = 0;;) {
      const uint64_t past = __ballot(before + incl > c);
      if (past) {
        const int l = __builtin_ctzll(past);
        b = base + l;
        first = before + __builtin_amdgcn_readlane(incl - v, l);
        return;
      }
      before += __builtin_amdgcn_readlane(incl, 63);
      base += 64;
      if (base >= s.B) {  // not reached: the total covers c
        b = s.B - 1;
        first = before - __builtin_amdgcn_readlane(v, (s.B - 1) & 63);
        return;
      }
      v = of(base + lane);
      incl = wave_scan(v);
    }
  }
  // The first chunk of sequence b.
  __device__ __forceinline__ int first_of(int b) const {
    int before = 0, v = mine, incl = upto;
    for (int base = 0; base + 64 <= b; base += 64) {
      before += __builtin_amdgcn_readlane(incl, 63);
      v = of(base + 64 + lane);
      incl = wave_scan(v);
    }
    return before + __builtin_amdgcn_readlane(incl - v, b & 63);
  }
};

// Chunk ranges of the workgroups: n = min(groups, total) of them take part,
// and the first total % n take one chunk more.
struct Ranges {
  int n, q, r;
  __device__ __forceinline__ Ranges(int total, int groups) : n(total), q(1), r(0) {
    if (total > groups) {
      n = groups;
      q = uint32_t(total) / uint32_t(n);
      r = total - q * n;
    }
  }
  __device__ __forceinline__ int start(int w) const { return w * q + min(w, r); }
  __device__ __forceinline__ int owner(int c) const {
    if (q == 1 && r == 0) return c;
    const int wide = r * (q + 1);
    return c < wide ? uint32_t(c) / uint32_t(q + 1) : r + uint32_t(c - wide) / uint32_t(q);
  }
};

// Eight floats as TERMS bf16 vectors whose sum they are.
template <int TERMS>
__device__ __forceinline__ void split8(const float (&v)[8], bf16x8 (&t)[TERMS]) {
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    float rest = v[i];
#pragma unroll
    for (int k = 0; k < TERMS; ++k) {
      t[k][i] = static_cast<__bf16>(rest);
      if (k + 1 < TERMS) rest -= static_cast<float>(t[k][i]);
    }
  }
}

// Eight e4m3 codes (two words) as bf16.
__device__ __forceinline__ u32x4 widen8(uint32_t lo, uint32_t hi) {
  u32x4 r;
  r[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.f, false));
  r[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.f, true));
  r[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.f, false));
  r[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.f, true));
  return r;
}

__device__ __forceinline__ int64_t shfl64(int64_t v, int from) {
  const uint32_t lo = __shfl(uint32_t(v), from), hi = __shfl(uint32_t(uint64_t(v) >> 32), from);
  return int64_t(uint64_t(hi) << 32 | lo);
}

// Keys and values are read once: without a place in the caches for them the
// same loads run at 6.9 TB/s instead of 6.1 (2 GB, plain streaming read).
constexpr int kStream = 2;  // the same hint of a buffer load
template <class T>
__device__ __forceinline__ T stream_load(const T* p) {
  return __builtin_nontemporal_load(p);
}

// 16 bytes per lane from the buffer to shared memory: lane i's to to + 16 i.
__device__ __forceinline__ void request_1k(__amdgpu_buffer_rsrc_t from, uint8_t* to, uint32_t at) {
  __builtin_amdgcn_raw_ptr_buffer_load_lds(from, (__attribute__((address_space(3))) void*)to, 16, at, 0, 0, kStream);
}

__device__ __forceinline__ f32x4 mfma(bf16x8 a, bf16x8 b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}

// Where the partials of a row lie: those of workgroups w0 to w1, in order.
struct RowParts {
  int w0, w1, row_first;
  // first: of the row's chunks
  __device__ __forceinline__ RowParts(const Ranges& ranges, int first, int chunks)
      : w0(ranges.owner(first)), w1(ranges.owner(first + chunks - 1)), row_first(first) {}
  __device__ __forceinline__ static RowParts of(const Chunks& all, const Ranges& ranges, int b, int row) {
    const int chunks = chunks_of(seq_len(all.s, b), all.cl);
    return RowParts(ranges, all.first_of(b) + row * (all.head + chunks) + all.head, chunks);
  }
  __device__ __forceinline__ const float* part(const Plan& p, const Ranges& ranges, int w) const {
    return p.part + (int64_t(w) * 2 + (row_first >= ranges.start(w) ? 1 : 0)) * p.part_ld;
  }
};

// Maximum and sum of a head of a split row, by one wave: each lane joins its
// parts as they arrive, then the lanes meet.
__device__ __forceinline__ void head_stats(const AttnArgs& a, const Plan& p, const Ranges& ranges, const RowParts& rp,
                                           int h, int lane, float& top, float& sum) {
  float m = kNegInf, l = 0.f;
  for (int w = rp.w0 + lane; w <= rp.w1; w += 64) {
    const float* part = rp.part(p, ranges, w) + p.gh * a.kv.dim;
    const float pm = part[h], pl = part[p.gh + h], t = fmaxf(m, pm), ref = t == kNegInf ? 0.f : t;
    l = l * __builtin_amdgcn_exp2f(m - ref) + pl * __builtin_amdgcn_exp2f(pm - ref);
    m = t;
  }
  top = m;
#pragma unroll
  for (int k = 32; k; k >>= 1) top = fmaxf(top, __shfl_xor(top, k));
  sum = l * __builtin_amdgcn_exp2f(m - (top == kNegInf ? 0.f : top));
#pragma unroll
  for (int k = 32; k; k >>= 1) sum += __shfl_xor(sum, k);
}

// Output of query head qh (head h of its row) from the parts of the row, by the
// whole workgroup.  dim / 4 threads per set of parts; each set joins its own as
// they arrive, four requested at a time, and the sets meet in shared memory (sm:
// 1024 floats, sm_ml: 128).
template <bool F32>
__device__ __forceinline__ void join_head(const AttnArgs& a, const Plan& p, const Ranges& ranges, const RowParts& rp, int64_t qh, int h,
                                          float* sm, float* sm_ml) {
  const uint32_t D = a.kv.dim;
  const int per = int(D) / 4, sets = 256 / per, set = threadIdx.x / per, d = (threadIdx.x - set * per) * 4;
  const bool mine = set < sets;
  float top = kNegInf, sum = 0.f, r[4] = {0.f, 0.f, 0.f, 0.f};
  if (mine)
    for (int w = rp.w0 + set; w <= rp.w1; w += 4 * sets) {
      float pm[4], pl[4];
      float4 po[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const bool in = w + k * sets <= rp.w1;
        const float* part = rp.part(p, ranges, in ? w + k * sets : w);
        pm[k] = in ? part[p.gh * D + h] : kNegInf;
        pl[k] = part[p.gh * D + p.gh + h];
        po[k] = *reinterpret_cast<const float4*>(part + h * D + d);
      }
      const float t = fmaxf(fmaxf(fmaxf(pm[0], pm[1]), fmaxf(pm[2], pm[3])), top), ref = t == kNegInf ? 0.f : t;
      const float old = __builtin_amdgcn_exp2f(top - ref);
      sum *= old;
#pragma unroll
      for (int x = 0; x < 4; ++x) r[x] *= old;
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const float f = __builtin_amdgcn_exp2f(pm[k] - ref);
        sum += f * pl[k];
        r[0] += f * po[k].x;
        r[1] += f * po[k].y;
        r[2] += f * po[k].z;
        r[3] += f * po[k].w;
      }
      top = t;
    }
  *reinterpret_cast<float4*>(&sm[threadIdx.x * 4]) = make_float4(r[0], r[1], r[2], r[3]);
  if (d == 0 && mine) {
    sm_ml[set] = top;
    sm_ml[64 + set] = sum;
  }
  __syncthreads();
  const int x = threadIdx.x;
  if (x >= int(D)) return;
  float most = kNegInf;
  for (int k = 0; k < sets; ++k) most = fmaxf(most, sm_ml[k]);
  const float ref = most == kNegInf ? 0.f : most;
  float total = 0.f, y = 0.f;
  for (int k = 0; k < sets; ++k) {
    const float f = __builtin_amdgcn_exp2f(sm_ml[k] - ref);
    total += f * sm_ml[64 + k];
    y += f * sm[k * int(D) + x];
  }
  y *= total == 0.f ? 0.f : 1.f / total;
  if constexpr (F32) static_cast<float*>(a.out)[qh * D + x] = y;
  else static_cast<__bf16*>(a.out)[qh * D + x] = static_cast<__bf16>(y);
  if (x == 0 && a.lse) a.lse[qh] = (most + __log2f(total)) * kLn2;
}

// The dimension of value product j in row c: VPL = DP / 16 neighbouring ones per
// lane, in two halves where they take two loads, so that each load of a slot's
// lanes is contiguous.
template <int DP, bool E4M3>
__device__ __forceinline__ constexpr int value_dim(int c, int j) {
  return !E4M3 && DP == 256 ? (j >> 3) * 128 + c * 8 + (j & 7) : c * (DP / 16) + j;
}

// DP: dim padded to 64, 128 or 256.  FULL: dim == DP.  P16: page_size is a
// multiple of 16, so that the 16 slots of a key operand lie on one page: they are
// a buffer of their own (its base in scalar registers, offsets that no tile
// changes), and the scales of a lane's four neighbouring slots are one load.
// Keys go to shared memory row by row and are read from there in the operand's
// order: requested in that order they would be 64-byte pieces of 16 rows, which
// arrive at 5.9 TB/s where whole rows arrive at 6.9 (2 GB in random 16 KiB
// pieces).  Otherwise each slot's address is found by a lane of its own and passed
// on by lane exchanges, and keys go to registers.
//
// A wave's loads run one tile ahead: the next tile's keys are requested as soon
// as the scores of this one are formed, its values once this one's are used up,
// into the same registers, and its page numbers a tile before that.  The loads
// past the last tile have no branch around them: where paths with and without
// requests meet, every wait would be one for all loads in flight.
template <int DP, bool E4M3, bool F32, bool FULL, bool P16>
__global__ __launch_bounds__(256, occupancy(DP, F32, P16)) void attn_decode_kernel(AttnArgs a, Plan p) {
  constexpr int KS = DP / 32, VPL = DP / 16, QT = F32 ? 3 : 1, PT = F32 ? 3 : 2, ELT = E4M3 ? 1 : 2;
  constexpr int KL = E4M3 ? KS / 2 : KS;        // 16-byte key loads per key
  constexpr int VW = VPL * ELT / 4;             // words per value load
  constexpr int NS = tile_slots(DP, F32) / 32;  // 32-slot parts of a tile
  constexpr int kTile = NS * 32, kChunk = 4 * kTile;
  // P16: keys of 32 * NS slots per wave.  Row r of a wave holds its 16-byte
  // segments in the order s ^ swizzle(r), so that 8 rows' equal segments lie in
  // different banks
  constexpr int kRow = DP * ELT, kSegs = kRow / 16, kKeys = NS * 32 * kRow;
  constexpr int kFloats = 4 * 16 * (DP + 4);
  __shared__ float sm_m[4][16], sm_l[4][16], sm_lse[16];
  __shared__ __attribute__((aligned(1024))) uint8_t lds[P16 && 4 * kKeys > 4 * kFloats ? 4 * kKeys : 4 * kFloats];
  float(*const sm_o)[16][DP + 4] = reinterpret_cast<float(*)[16][DP + 4]>(lds);  // the join's, once the keys are used up

  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), c = lane & 15, g = lane >> 4;
  const uint32_t D = a.kv.dim;
  const Chunks all(a.seqs, p, lane);
  const Ranges ranges(all.total, p.groups);
  const int w = blockIdx.x;
  if (w >= ranges.n) return;
  const int begin = ranges.start(w), end = ranges.start(w + 1);
  int b, first;
  all.find(begin, b, first);

  for (int at = begin; at < end;) {
    int len = seq_len(a.seqs, b), chunks = chunks_of(len, all.cl), units = all.head + chunks;
    while (at >= first + int(p.rows) * units) {
      first += int(p.rows) * units;
      ++b;
      len = seq_len(a.seqs, b);
      chunks = chunks_of(len, all.cl);
      units = all.head + chunks;
    }
    const int row = uint32_t(at - first) / uint32_t(units), row_at = first + row * units, row_end = row_at + units;
    // the chunks of this row that lie in the range; unsplit rows belong to the
    // workgroup that has their first unit
    int c0 = max(at - row_at - all.head, 0), nc = min(end, row_end) - row_at - all.head - c0;
    if (p.whole) nc = at == row_at ? chunks : 0;
    if (nc <= 0) {
      at = row_end;
      continue;
    }
    const int hk = p.hgroups == 1 ? row : uint32_t(row) / p.hgroups, gi = row - hk * int(p.hgroups);
    const int heads = min(16, int(a.group) - gi * 16);        // of this row
    const int head0 = hk * int(a.group) + gi * 16;            // its first query head
    const int stop = min(len, (c0 + nc) * kChunk);
    const uint8_t* kbase = a.kv.k + hk * a.kv.head_stride;
    const uint8_t* vbase = a.kv.v + hk * a.kv.head_stride;
    const int32_t* table = a.seqs.table + int64_t(b) * a.seqs.stride;

    u32x4 kr[P16 ? 1 : 2 * NS][KL];
    uint8_t* const keys = lds + wave * kKeys;
    const auto swizzle = [](int r) { return (kSegs == 4 ? r >> 1 : r) & (kSegs < 8 ? kSegs - 1 : 7); };
    uint32_t vr[8 * NS][VW];
    f32x4 ks[2 * NS], vs[2 * NS];  // scales of slots u * 16 + g * 4 .. + 3
    uint32_t page[NS];             // lanes i and i + 32: the page of slot i of each part of a tile
    // P16: the live slots of each 16, this tile's and the next one's, and where their values lie
    int live[2 * NS], live_next[2 * NS];
    __amdgpu_buffer_rsrc_t vpage[2 * NS];
    const float* vscale[2 * NS];
    // otherwise: the live slots of each 32 as bits, each lane's slot's offset and scale
    uint32_t mask[NS], mask_next[NS];
    int64_t off[NS];
    float v1[NS];
    // parts of the addresses that no tile changes.  P16: dimensions past the
    // head's are out of the buffer's range; otherwise they read the row's start
    const uint32_t kd = E4M3 ? g * 16 : g * 8, slot_bytes = uint32_t(a.kv.slot_stride);
    const uint32_t vslot = P16 ? g * 4 * slot_bytes : 0;
    const auto byte_of = [&](uint32_t d, uint32_t slots) {
      return FULL || d < D ? slots + d * ELT : P16 ? 0x80000000u : 0u;
    };
    const auto key_byte = [&](int i) { return byte_of(kd + i * (E4M3 ? 64 : 32), 0); };
    // P16: request i of a part's 16 keys fills 1 KiB of the wave's rows in lane order
    const auto key_part = [&](int i) {
      const int r = i * (64 / kSegs) + lane / kSegs;
      return byte_of(((lane % kSegs) ^ swizzle(r)) * 16 / ELT, r * slot_bytes);
    };
    const auto value_byte = [&](int i, int j) { return byte_of(value_dim<DP, E4M3>(c, j), vslot + (P16 ? i * slot_bytes : 0)); };

    const auto load_pages = [&](int t0) {
#pragma unroll
      for (int x = 0; x < NS; ++x) {
        const int t = t0 + x * 32 + (lane & 31);
        page[x] = uint32_t(table[a.kv.per_page.div(t < stop ? t : 0)]);
      }
    };
    const auto load_keys = [&](int t0) {
#pragma unroll
      for (int x = 0; x < NS; ++x) {
        if constexpr (P16) {
#pragma unroll
          for (int u = 0; u < 2; ++u) {
            const int t = t0 + x * 32 + u * 16;
            const uint32_t pg = __builtin_amdgcn_readlane(page[x], u * 16), po = t - a.kv.per_page.div(t) * a.kv.page_size;
            const int n = pg < a.kv.pages ? max(min(stop - t, 16), 0) : 0;
            live_next[x * 2 + u] = n;
            // a buffer that ends with the last live slot: what lies past it
            // reads as zero, and costs no memory access
            const int64_t at_slots = n ? pg * a.kv.page_stride + po * a.kv.slot_stride : 0;
            const uint32_t bytes = n ? (n - 1) * slot_bytes + D * ELT : 0;
            const __amdgpu_buffer_rsrc_t kpage = buffer_rsrc(kbase + at_slots, bytes);
            vpage[x * 2 + u] = buffer_rsrc(vbase + at_slots, bytes);
            if constexpr (E4M3) {
              const int64_t so = n ? (int64_t(pg) * a.kv.heads + hk) * a.kv.page_size + po : 0;
              ks[x * 2 + u] = reinterpret_cast<const f32x4*>(a.kv.k_scale + so)[g];
              vscale[x * 2 + u] = a.kv.v_scale + so;
            }
#pragma unroll
            for (int i = 0; i < kRow / 64; ++i)
              request_1k(kpage, keys + (x * 2 + u) * 16 * kRow + i * 1024, key_part(i));
          }
        } else {
          const int t = t0 + x * 32 + (lane & 31);
          const uint32_t po = t - a.kv.per_page.div(t) * a.kv.page_size;
          const bool ok = t < stop && page[x] < a.kv.pages;
          mask_next[x] = uint32_t(__ballot(ok));
          // past the end: the same row again
          off[x] = ok ? page[x] * a.kv.page_stride + po * a.kv.slot_stride : off[x];
          if constexpr (E4M3) {
            const int64_t so = ok ? (int64_t(page[x]) * a.kv.heads + hk) * a.kv.page_size + po : 0;
            const float k1 = a.kv.k_scale[so];
            v1[x] = a.kv.v_scale[so];
#pragma unroll
            for (int i = 0; i < 8; ++i) ks[x * 2 + (i >> 2)][i & 3] = __shfl(k1, (i >> 2) * 16 + g * 4 + (i & 3));
          }
#pragma unroll
          for (int u = 0; u < 2; ++u) {
            const uint8_t* src = kbase + shfl64(off[x], u * 16 + c);
#pragma unroll
            for (int i = 0; i < KL; ++i) kr[x * 2 + u][i] = stream_load(reinterpret_cast<const u32x4*>(src + key_byte(i)));
          }
        }
      }
    };
    const auto load_values = [&] {
#pragma unroll
      for (int x = 0; x < NS; ++x) {
        if constexpr (E4M3) {
          if constexpr (P16) {
#pragma unroll
            for (int u = 0; u < 2; ++u) vs[x * 2 + u] = reinterpret_cast<const f32x4*>(vscale[x * 2 + u])[g];
          } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) vs[x * 2 + (i >> 2)][i & 3] = __shfl(v1[x], (i >> 2) * 16 + g * 4 + (i & 3));
          }
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          uint32_t* dst = vr[x * 8 + i];
          const uint8_t* src = P16 ? nullptr : vbase + shfl64(off[x], (i >> 2) * 16 + g * 4 + (i & 3));
          const __amdgpu_buffer_rsrc_t from = vpage[x * 2 + (i >> 2)];
          if constexpr (VW % 4 == 0) {
#pragma unroll
            for (int y = 0; y < VW / 4; ++y) {
              const uint32_t at = value_byte(i & 3, y * 16 / ELT);
              u32x4 r;
              if constexpr (P16) r = __builtin_amdgcn_raw_buffer_load_b128(from, at, 0, kStream);
              else r = stream_load(reinterpret_cast<const u32x4*>(src + at));
#pragma unroll
              for (int z = 0; z < 4; ++z) dst[y * 4 + z] = r[z];
            }
          } else if constexpr (VW == 2) {
            const uint32_t at = value_byte(i & 3, 0);
            u32x2 r;
            if constexpr (P16) r = __builtin_amdgcn_raw_buffer_load_b64(from, at, 0, kStream);
            else r = stream_load(reinterpret_cast<const u32x2*>(src + at));
            dst[0] = r[0];
            dst[1] = r[1];
          } else {
            const uint32_t at = value_byte(i & 3, 0);
            if constexpr (P16) dst[0] = __builtin_amdgcn_raw_buffer_load_b32(from, at, 0, kStream);
            else dst[0] = stream_load(reinterpret_cast<const uint32_t*>(src + at));
          }
        }
      }
    };

    f32x4 o[VPL];
#pragma unroll
    for (int j = 0; j < VPL; ++j) o[j] = f32x4{0, 0, 0, 0};
    float m = kNegInf, l = 0.f;
    const float scale2 = a.scale * kLog2e;
    bf16x8 q[QT][KS];

    const auto tile = [&](int t0) {
#pragma unroll
      for (int x = 0; x < 2 * NS; ++x) {
        if constexpr (P16) live[x] = live_next[x];
        else mask[x >> 1] = mask_next[x >> 1];
      }
      // whether slot u * 16 + g * 4 + i of part x is live
      const auto in = [&](int x, int u, int i) {
        return P16 ? g * 4 + i < live[x * 2 + u] : bool(mask[x] >> (u * 16 + g * 4 + i) & 1);
      };
      // scores of the tile's slots x 16 heads, in log2 units
      float s[NS][8];
#pragma unroll
      for (int x = 0; x < NS; ++x)
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          f32x4 acc = {0, 0, 0, 0};
#pragma unroll
          for (int i = 0; i < KS; ++i) {
            u32x4 r;
            if constexpr (P16) {
              const int row = (x * 2 + u) * 16 + c, seg = (E4M3 ? i >> 1 : i) * 4 + g;
              r = *reinterpret_cast<const u32x4*>(keys + row * kRow + (seg ^ swizzle(c)) * 16);
            } else {
              r = kr[x * 2 + u][E4M3 ? i >> 1 : i];
            }
            if (!FULL && kd + (E4M3 ? (i >> 1) * 64 : i * 32) >= D) r = u32x4{0, 0, 0, 0};
            if constexpr (E4M3) r = widen8(r[(i & 1) * 2], r[(i & 1) * 2 + 1]);
#pragma unroll
            for (int k = QT - 1; k >= 0; --k) acc = mfma(__builtin_bit_cast(bf16x8, r), q[k][i], acc);
          }
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            float z = acc[i] * scale2;
            if constexpr (E4M3) z *= ks[x * 2 + u][i];
            s[x][u * 4 + i] = in(x, u, i) ? z : kNegInf;
          }
        }
      __builtin_amdgcn_sched_barrier(0);  // every key has been read
      load_keys(t0 + kChunk);
      load_pages(t0 + 2 * kChunk);
      __builtin_amdgcn_sched_barrier(0);

      if (p.scores && c < heads) {
        float* dst = p.scores + (int64_t(b) * a.heads_q + head0 + c) * p.score_ld + t0 + g * 4;
#pragma unroll
        for (int x = 0; x < NS; ++x) {
          *reinterpret_cast<float4*>(dst + x * 32) = make_float4(s[x][0], s[x][1], s[x][2], s[x][3]);
          *reinterpret_cast<float4*>(dst + x * 32 + 16) = make_float4(s[x][4], s[x][5], s[x][6], s[x][7]);
        }
      }
      float top = s[0][0];
#pragma unroll
      for (int i = 1; i < 8 * NS; ++i) top = fmaxf(top, s[i >> 3][i & 7]);
      top = fmaxf(top, __shfl_xor(top, 16));
      top = fmaxf(top, __shfl_xor(top, 32));
      const float m_new = fmaxf(m, top), ref = m_new == kNegInf ? 0.f : m_new;
      const float alpha = __builtin_amdgcn_exp2f(m - ref);
      m = m_new;
      l *= alpha;
#pragma unroll
      for (int j = 0; j < VPL; ++j) o[j] *= alpha;
      bf16x8 pf[NS][PT];
#pragma unroll
      for (int x = 0; x < NS; ++x) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          s[x][i] = __builtin_amdgcn_exp2f(s[x][i] - ref);
          l += s[x][i];
          // a scale past the end may be NaN
          if constexpr (E4M3)
            s[x][i] = in(x, i >> 2, i & 3) ? s[x][i] * vs[x * 2 + (i >> 2)][i & 3] : 0.f;
        }
        split8<PT>(s[x], pf[x]);
      }

#pragma unroll
      for (int x = 0; x < NS; ++x) {
        // what lies in slots past the end may be NaN and takes no part
        if (!P16 && mask[x] != 0xFFFFFFFFu) {
#pragma unroll
          for (int i = 0; i < 8; ++i)
#pragma unroll
            for (int y = 0; y < VW; ++y) vr[x * 8 + i][y] = in(x, i >> 2, i & 3) ? vr[x * 8 + i][y] : 0;
        }
#pragma unroll
        for (int y = 0; y < VPL / 2; ++y) {
          uint32_t pair[8];  // bf16 of dimensions 2 y and 2 y + 1 of the lane's eight slots
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            if constexpr (E4M3)
              pair[i] = __builtin_bit_cast(
                  uint32_t, y & 1 ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(vr[x * 8 + i][y >> 1], 1.f, true)
                                  : __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(vr[x * 8 + i][y >> 1], 1.f, false));
            else
              pair[i] = vr[x * 8 + i][y];
          }
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            u32x4 f;
#pragma unroll
            for (int z = 0; z < 4; ++z) f[z] = __builtin_amdgcn_perm(pair[2 * z + 1], pair[2 * z], j ? 0x07060302u : 0x05040100u);
#pragma unroll
            for (int k = PT - 1; k >= 0; --k)
              o[2 * y + j] = mfma(__builtin_bit_cast(bf16x8, f), pf[x][k], o[2 * y + j]);
          }
        }
      }
      load_values();
      __builtin_amdgcn_sched_barrier(0);
    };
    int t0 = c0 * kChunk + wave * kTile;
    if (t0 < stop) {
#pragma unroll
      for (int x = 0; x < NS; ++x) off[x] = 0;
      load_pages(t0);
      load_keys(t0);
      load_pages(t0 + kChunk);
      load_values();
      // in the order of the loop, or its waits would be longer than they need be
      __builtin_amdgcn_sched_barrier(0);
      // the queries of the row; columns past its heads are zero
#pragma unroll
      for (int s = 0; s < KS; ++s) {
        const uint32_t d = E4M3 ? (s >> 1) * 64 + g * 16 + (s & 1) * 8 : s * 32 + g * 8;
        const bool in = c < heads && (FULL || d < D);
        const int64_t at_q = int64_t(b) * a.q_stride + int64_t(head0 + (in ? c : 0)) * D + (in ? d : 0);
        if constexpr (F32) {
          const f32x4* src = reinterpret_cast<const f32x4*>(static_cast<const float*>(a.q) + at_q);
          const f32x4 lo = src[0], hi = src[1];
          float v[8];
#pragma unroll
          for (int i = 0; i < 8; ++i) v[i] = in ? (i < 4 ? lo[i & 3] : hi[i & 3]) : 0.f;
          bf16x8 t[3];
          split8<3>(v, t);
#pragma unroll
          for (int k = 0; k < 3; ++k) q[k][s] = t[k];
        } else {
          u32x4 v = *reinterpret_cast<const u32x4*>(static_cast<const uint16_t*>(a.q) + at_q);
          if (!in) v = u32x4{0, 0, 0, 0};
          q[0][s] = __builtin_bit_cast(bf16x8, v);
        }
      }
      for (; t0 < stop; t0 += kChunk) tile(t0);
    }

    // join the four waves, where their keys were: none is still on its way
    if constexpr (P16) {
      __builtin_amdgcn_s_waitcnt(0x0F70);  // vmcnt(0)
      __syncthreads();
    }
    l += __shfl_xor(l, 16);
    l += __shfl_xor(l, 32);
    if (g == 0) {
      sm_m[wave][c] = m;
      sm_l[wave][c] = l;
    }
    if (c < heads) {
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < VPL; j += 4)
          *reinterpret_cast<float4*>(&sm_o[wave][c][value_dim<DP, E4M3>(g * 4 + i, j)]) =
              make_float4(o[j][i], o[j + 1][i], o[j + 2][i], o[j + 3][i]);
    }
    __syncthreads();
    const bool whole = nc == chunks;
    float* part = p.part + (int64_t(w) * 2 + (row_at + all.head >= begin ? 1 : 0)) * p.part_ld;
    const int per = int(D) / 4;
    for (int i = threadIdx.x; i < heads * per; i += 256) {
      const int h = i / per, d = (i - h * per) * 4;
      float top = sm_m[0][h];
#pragma unroll
      for (int k = 1; k < 4; ++k) top = fmaxf(top, sm_m[k][h]);
      const float ref = top == kNegInf ? 0.f : top;
      float sum = 0.f, r[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const float f = __builtin_amdgcn_exp2f(sm_m[k][h] - ref);
        sum += f * sm_l[k][h];
#pragma unroll
        for (int x = 0; x < 4; ++x) r[x] += f * sm_o[k][h][d + x];
      }
      if (whole) {
        const int64_t qh = int64_t(b) * a.heads_q + head0 + h;
        const float inv = sum == 0.f ? 0.f : 1.f / sum;
        if constexpr (F32) {
          *reinterpret_cast<float4*>(static_cast<float*>(a.out) + qh * D + d) =
              make_float4(r[0] * inv, r[1] * inv, r[2] * inv, r[3] * inv);
        } else {
          const bf16x2 lo = {static_cast<__bf16>(r[0] * inv), static_cast<__bf16>(r[1] * inv)};
          const bf16x2 hi = {static_cast<__bf16>(r[2] * inv), static_cast<__bf16>(r[3] * inv)};
          *reinterpret_cast<uint2*>(static_cast<uint16_t*>(a.out) + qh * D + d) =
              make_uint2(__builtin_bit_cast(uint32_t, lo), __builtin_bit_cast(uint32_t, hi));
        }
        if (d == 0) {
          const float lse2 = top + __log2f(sum);
          p.lse2[qh] = lse2;
          if (a.lse) a.lse[qh] = lse2 * kLn2;
          if (p.weigh) sm_lse[h] = lse2;
        }
      } else {
        if (d == 0) {
          part[p.gh * D + h] = top;
          part[p.gh * D + p.gh + h] = sum;
        }
        *reinterpret_cast<float4*>(part + h * D + d) = make_float4(r[0], r[1], r[2], r[3]);
      }
    }
    __syncthreads();
    if (p.weigh) {  // the row is whole and has all query heads of its key head
      const float* scores = p.scores + (int64_t(b) * a.heads_q + head0) * p.score_ld;
      // so many slots of a thread, from t0, and four heads are requested at a time
      const auto weigh = [&](auto slots, int t0) {
        constexpr int kSlots = decltype(slots)::value, kHeads = 4;
        int64_t to[kSlots];
        float old[kSlots], sum[kSlots] = {};
#pragma unroll
        for (int k = 0; k < kSlots; ++k) {
          const int t = min(t0 + k * 256, len - 1);
          const uint32_t pi = a.kv.per_page.div(t), pg = uint32_t(table[pi]);
          to[k] = pg < a.kv.pages ? (int64_t(pg) * a.kv.heads + hk) * a.kv.page_size + (t - pi * a.kv.page_size) : -1;
        }
        for (int h0 = 0; h0 < heads; h0 += kHeads) {
          float z[kHeads][kSlots];
#pragma unroll
          for (int h = 0; h < kHeads; ++h)
#pragma unroll
            for (int k = 0; k < kSlots; ++k) z[h][k] = scores[min(h0 + h, heads - 1) * p.score_ld + min(t0 + k * 256, len - 1)];
          if (h0 == 0) {
#pragma unroll
            for (int k = 0; k < kSlots; ++k) old[k] = a.weight_in[max(to[k], int64_t(0))];
          }
#pragma unroll
          for (int h = 0; h < kHeads; ++h) {
            const float lse2 = sm_lse[min(h0 + h, heads - 1)];
            if (h0 + h < heads && lse2 != kNegInf) {
#pragma unroll
              for (int k = 0; k < kSlots; ++k) sum[k] += __builtin_amdgcn_exp2f(z[h][k] - lse2);
            }
          }
        }
#pragma unroll
        for (int k = 0; k < kSlots; ++k)
          if (t0 + k * 256 < len && to[k] >= 0) a.weight_out[to[k]] = old[k] + sum[k];
      };
      for (int t0 = threadIdx.x; t0 - int(threadIdx.x) < len; t0 += 512) {
        if (t0 - int(threadIdx.x) + 256 < len) weigh(std::integral_constant<int, 2>(), t0);
        else weigh(std::integral_constant<int, 1>(), t0);
      }
      __syncthreads();
    }
    at = row_end;
  }
}

constexpr int kSlotBlock = 1024;  // slots whose weights a workgroup sums

// Workgroups below `joins` (one per query head, or none where no row is split):
// the output of one head of a split row.  The rest (tracked calls whose rows did
// not add theirs): the attention weights of 1024 slots of one key head.
template <bool F32>
__global__ __launch_bounds__(256) void attn_join_kernel(AttnArgs a, Plan p, int joins, int slot_blocks) {
  __shared__ __attribute__((aligned(16))) float sm[256 * 4];
  __shared__ float sm_ml[128];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const Chunks all(a.seqs, p, lane);
  const Ranges ranges(all.total, p.groups);
  int id = blockIdx.x;
  if (id < joins) {
    const int b = id / int(a.heads_q), hq = id - b * int(a.heads_q), hk = hq / int(a.group), gi = (hq - hk * int(a.group)) / 16;
    const int h = hq - hk * int(a.group) - gi * 16;
    const RowParts rp = RowParts::of(all, ranges, b, hk * int(p.hgroups) + gi);
    if (rp.w0 == rp.w1) return;  // the row was finished in one workgroup
    join_head<F32>(a, p, ranges, rp, int64_t(b) * a.heads_q + hq, h, sm, sm_ml);
    return;
  }
  id -= joins;
  const int b = id / (int(a.kv.heads) * slot_blocks), rest = id - b * int(a.kv.heads) * slot_blocks;
  const int hk = rest / slot_blocks, t0 = (rest - hk * slot_blocks) * kSlotBlock;
  const int len = seq_len(a.seqs, b);
  if (t0 >= len) return;
  constexpr int kPer = kSlotBlock / 256, kHeads = 4;
  // what does not wait for the sums is requested before them
  int64_t at[kPer];
  float old[kPer], w[kPer] = {};
#pragma unroll
  for (int k = 0; k < kPer; ++k) {
    const int t = min(t0 + k * 256 + int(threadIdx.x), len - 1);
    const uint32_t pi = a.kv.per_page.div(t), page = uint32_t(a.seqs.table[int64_t(b) * a.seqs.stride + pi]);
    at[k] = page < a.kv.pages ? (int64_t(page) * a.kv.heads + hk) * a.kv.page_size + (t - pi * a.kv.page_size) : -1;
  }
  for (int gi = 0; gi < int(p.hgroups); ++gi) {
    const RowParts rp = RowParts::of(all, ranges, b, hk * int(p.hgroups) + gi);
    const int heads = min(16, int(a.group) - gi * 16);
    const int64_t qh = int64_t(b) * a.heads_q + hk * a.group + gi * 16;
    for (int h0 = 0; h0 < heads; h0 += kHeads) {
      float s[kHeads][kPer];
#pragma unroll
      for (int h = 0; h < kHeads; ++h)
#pragma unroll
        for (int k = 0; k < kPer; ++k)
          s[h][k] = p.scores[(qh + min(h0 + h, heads - 1)) * p.score_ld + min(t0 + k * 256 + int(threadIdx.x), len - 1)];
      if (h0 == 0) {
        if (gi == 0) {
#pragma unroll
          for (int k = 0; k < kPer; ++k) old[k] = a.weight_in[max(at[k], int64_t(0))];
        }
        // one wave per head finds the logarithm of its sum
        __syncthreads();
        for (int h = wave; h < heads; h += 4) {
          float lse2;
          if (p.whole || rp.w0 == rp.w1) {
            lse2 = p.lse2[qh + h];
          } else {
            float top, sum;
            head_stats(a, p, ranges, rp, h, lane, top, sum);
            lse2 = top + __log2f(sum);
          }
          if (lane == 0) sm[h] = lse2;
        }
        __syncthreads();
      }
#pragma unroll
      for (int h = 0; h < kHeads; ++h) {
        const float lse2 = sm[min(h0 + h, heads - 1)];
        if (h0 + h < heads && lse2 != kNegInf) {
#pragma unroll
          for (int k = 0; k < kPer; ++k) w[k] += __builtin_amdgcn_exp2f(s[h][k] - lse2);
        }
      }
    }
  }
#pragma unroll
  for (int k = 0; k < kPer; ++k)
    if (t0 + k * 256 + int(threadIdx.x) < len && at[k] >= 0) a.weight_out[at[k]] = old[k] + w[k];
}

struct Sizes {
  uint32_t hgroups, gh;
  int64_t score_ld;
  uint32_t part_ld;
  size_t part, lse2, scores;  // floats
};
Sizes sizes_of(uint32_t heads_kv, uint32_t dim, uint32_t heads_q, int64_t B, int64_t cap, bool track) {
  Sizes s;
  const uint32_t group = heads_q / heads_kv;
  s.hgroups = (group + 15) / 16;
  s.gh = group < 16 ? group : 16;
  s.score_ld = (cap + 63) / 64 * 64;  // whole tiles
  const auto up = [](size_t n) { return (n + 3) / 4 * 4; };
  s.part_ld = (s.gh * (dim + 2) + 31) / 32 * 32;  // whole cache lines
  s.part = size_t(kMostGroups) * 2 * s.part_ld;
  s.lse2 = up(size_t(B) * heads_q);
  s.scores = track ? size_t(B) * heads_q * size_t(s.score_ld) : 0;
  return s;
}

template <int DP, bool E4M3, bool F32>
void launch(const AttnArgs& a, const Plan& p, hipStream_t st) {
  // 16 slots from a 32-bit offset, and scales of 4 slots in 16 bytes
  const bool p16 = a.kv.page_size % 16 == 0 && a.kv.slot_stride < (int64_t(1) << 27) &&
                   (reinterpret_cast<uintptr_t>(a.kv.k_scale) | reinterpret_cast<uintptr_t>(a.kv.v_scale)) % 16 == 0;
  if (a.kv.dim == DP) {
    if (p16) attn_decode_kernel<DP, E4M3, F32, true, true><<<p.groups, 256, 0, st>>>(a, p);
    else attn_decode_kernel<DP, E4M3, F32, true, false><<<p.groups, 256, 0, st>>>(a, p);
  } else {
    if (p16) attn_decode_kernel<DP, E4M3, F32, false, true><<<p.groups, 256, 0, st>>>(a, p);
    else attn_decode_kernel<DP, E4M3, F32, false, false><<<p.groups, 256, 0, st>>>(a, p);
  }
}
template <bool E4M3, bool F32>
void launch_dim(const AttnArgs& a, const Plan& p, hipStream_t st) {
  if (a.kv.dim <= 64) launch<64, E4M3, F32>(a, p, st);
  else if (a.kv.dim <= 128) launch<128, E4M3, F32>(a, p, st);
  else launch<256, E4M3, F32>(a, p, st);
}
int dim_padded(uint32_t dim) { return dim <= 64 ? 64 : dim <= 128 ? 128 : 256; }

}  // namespace

size_t attn_decode_workspace_bytes(uint32_t heads_kv, uint32_t dim, uint32_t heads_q, int64_t B, int64_t cap, bool track) {
  const Sizes s = sizes_of(heads_kv, dim, heads_q, B, cap, track);
  return (s.part + s.lse2 + s.scores) * sizeof(float);
}

hipError_t launch_attn_decode(const AttnArgs& a, bool f32, hipStream_t st) {
  const bool track = a.weight_out != nullptr;
  const Sizes s = sizes_of(a.kv.heads, a.kv.dim, a.heads_q, a.seqs.B, a.seqs.cap, track);
  Plan p;
  p.rows = a.kv.heads * s.hgroups;
  p.hgroups = s.hgroups;
  p.gh = s.gh;
  p.chunk_log = tile_slots(dim_padded(a.kv.dim), f32) == 64 ? 8 : 7;
  const int64_t rows = int64_t(a.seqs.B) * p.rows, most = chunks_of(a.seqs.cap, int(p.chunk_log));
  const int row_bytes = dim_padded(a.kv.dim) * (a.kv.e4m3 ? 1 : 2);
  // Short rows are not split: a further chunk takes 1.2 us (twice that at 512
  // bytes per slot), the second kernel 4 (one sequence of 512 slots, 32 heads of
  // 128, bf16: 10.0 us, split 10.3; of 256 7.4 and 9.5; of 700 not split 11.9, 10.7;
  // 8 heads of 256, 256 slots 10.3 and 11.7, 400 not split 12.7, 11.6).  Nor are
  // somewhat longer ones where they fill the GPU as they are.  Rows of 1000 slots,
  // heads of 128, e4m3 (us, split in brackets): 64 rows 14.7 (12.4), 128 rows 15.1
  // (14.9), 192 rows 15.4 (18.2), 256 rows 16.1 (20.7), 300 rows 22.4 (25.8), 512 rows
  // 25.3 (29.0); and of 1300 slots 128 rows 18.3 (16.8), 320 rows 27.2 (28.9).  With
  // lengths spread evenly below 1000 it takes more rows, which the host cannot know:
  // 128 rows 20.7 (13.7), 240 rows 17.4 (16.5), 256 rows 18.8 (17.6), 512 rows 23.9
  // (25.6), 2048 rows 60.6 (73.7).  Rows of 512 bytes per slot, one workgroup to a
  // compute unit: 256 rows of 1000 43.1 (44.8), 300 rows 66.5 (56.0), 512 rows 83.7
  // (86.4).
  p.whole = most <= (row_bytes > 256 ? 2 : 4) || (rows >= kMostGroups / 2 && most <= 8);
  // The first loads' latency and the join of the waves take the time of about
  // two chunks; counted, workgroups with many short rows are not the last to
  // finish (64 ragged sequences of up to 8192 e4m3 slots: 351 us, uncounted
  // 390).  The rows of one sequence are of one length.
  p.head = a.seqs.B > 1 ? 2 : 0;
  // A tile of four waves requests 64 KiB where a row has 256 bytes, which is
  // what a compute unit needs in flight: one workgroup each, and fewer partial
  // results (32 sequences of 1000 slots, 32/8 heads of 128, bf16: 26.0 us, 512
  // workgroups 29.8).  Smaller rows take two (64 sequences of 4096 e4m3 slots:
  // 359 us, 256 workgroups 378).
  // Whole rows go to a workgroup each, up to 4096 (128 sequences of up to 300
  // slots, 16 heads of 64: 26.5 us, 512 workgroups 33.5).
  int64_t groups = p.whole ? kWholeGroups : row_bytes >= 256 ? kMostGroups / 2 : kMostGroups;
  // no more than there are rows or chunks, or neighbours would be idle
  groups = std::min(groups, p.whole ? rows : rows * (p.head + most));
  p.groups = uint32_t(groups);
  // A whole row's workgroup adds its attention weights itself: no second launch
  // (one sequence of 300 slots, 32 heads 9.4 us, with one 12.1; 32 of 100 16.1 and
  // 20.0, of 500 46.9 and 48.1; 64 of 500, 8 key heads, 23.4 and 26.7).  It is as
  // fast where many query heads share 1000 slots (128 sequences of 1000 e4m3 slots,
  // 32/8 heads: 67.3 and 65.9; of bf16, 8 heads, 91.9 and 91.9), which is not told
  // apart.  Where a key head's query heads are several rows, the second kernel sums
  // over them.
  p.weigh = track && p.whole && s.hgroups == 1;
  p.score_ld = s.score_ld;
  p.part = a.ws;
  p.lse2 = p.part + s.part;
  p.scores = track ? p.lse2 + s.lse2 : nullptr;
  p.part_ld = s.part_ld;
  if (a.kv.e4m3) {
    if (f32) launch_dim<true, true>(a, p, st);
    else launch_dim<true, false>(a, p, st);
  } else {
    if (f32) launch_dim<false, true>(a, p, st);
    else launch_dim<false, false>(a, p, st);
  }
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const int slot_blocks = track && !p.weigh ? (a.seqs.cap + kSlotBlock - 1) / kSlotBlock : 0;
  const int joins = p.whole ? 0 : a.seqs.B * int(a.heads_q);
  const uint32_t grid = uint32_t(joins + int64_t(a.seqs.B) * a.kv.heads * slot_blocks);
  if (grid == 0) return e;
  if (f32) attn_join_kernel<true><<<grid, 256, 0, st>>>(a, p, joins, slot_blocks);
  else attn_join_kernel<false><<<grid, 256, 0, st>>>(a, p, joins, slot_blocks);
  return hipGetLastError();
}

}  // namespace sdq
