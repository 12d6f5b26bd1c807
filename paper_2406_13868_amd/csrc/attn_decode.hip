// Attention of one new token per sequence over the paged cache.
//
// For sequence b, query head h (of key head h / group) and its slots t < len:
//   z_t = scale * q . k_t,  p_t = exp(z_t - max z) / sum,  out = sum_t p_t v_t
//   lse = log sum_t exp z_t,   weight_out[t] = weight_in[t] + sum over the
//   key head's query heads of p_t
// A row without a slot gives zeros and lse = -inf.
//
// Work.  The unit is a chunk of 128 slots of one row, a row being a key head
// of a sequence with up to 16 of its query heads.  The chunks of all rows, in
// order, are divided evenly over the workgroups, so ragged lengths leave none
// idle and a single long row uses all of them.  A workgroup walks its range
// row by row; a row that lies wholly in the range is finished there, of any
// other a partial result (maximum, sum and unnormalized output of each head)
// goes to the workspace, and a second kernel joins the partials of each row
// in the order of their workgroups, so that results do not depend on timing.
//
// Matrix instructions (16x16x32 bf16) take keys and values straight from
// global memory in registers, without shared memory.  Scores: A = 16 keys, B =
// the row's query heads.  The score of 16 keys x 16 heads leaves each lane 4
// keys of one head, and two such tiles give the 8 keys per lane that the
// second product's B operand wants, in the key order (g * 4 .. + 3, 16 + g * 4
// .. + 3) for lane group g.  Values: a lane loads, for the 8 keys of its
// group, VPL neighbouring dimensions; pairs of keys are put together with
// byte permutes, and VPL products follow, product j giving the dimensions c *
// VPL + j.  The operation count is a small part of what the matrix cores do
// in the time the cache takes to arrive, also with one query head in 16
// columns, so one kernel serves every head layout.
//
// Precision.  e4m3 codes are exact in bf16; their scales are applied in fp32 to
// the scores and to p.  bf16 queries are exact; fp32 queries are three bf16
// terms (24 bits).  p is the sum of two bf16 terms (17 bits, for outputs that
// are rounded to bf16) or three (fp32).  Products accumulate in fp32; maximum,
// sum and joins are fp32.
#include <hip/hip_runtime.h>

#include "kv_cache.h"

namespace sdq {
namespace {

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;

constexpr int kChunk = 128;       // slots per chunk: four waves of one 32-slot tile
constexpr int kMostGroups = 512;  // workgroups: two per compute unit
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr float kNegInf = -__builtin_huge_valf();

struct Plan {
  uint32_t rows;      // rows per sequence: heads * row groups
  uint32_t hgroups;   // row groups per key head: ceil(group / 16)
  uint32_t gh;        // query heads per row, at most (the stride of the partials)
  uint32_t groups;    // workgroups launched
  int64_t score_ld;   // floats between the scores of two query heads
  float* part;        // [groups][2][gh * (dim + 2)]: m[gh], l[gh], o[gh][dim]
  float* lse2;        // [B][heads_q]: log2 of the sum, for the rows finished in one workgroup
  float* scores;      // [B][heads_q][score_ld], log2 units; tracked calls only
};

__device__ __forceinline__ int chunks_of(int len) { return max(1, (len + kChunk - 1) / kChunk); }

// Sum of the chunks of one row of every sequence.
__device__ __forceinline__ int sum_chunks(const Seqs& s, int lane) {
  int n = 0;
  for (int b = lane; b < s.B; b += 64) n += chunks_of(seq_len(s, b));
#pragma unroll
  for (int k = 32; k; k >>= 1) n += __shfl_xor(n, k);
  return n;
}

// Chunk ranges of the workgroups: n = min(groups, total) of them take part,
// and the first total % n take one chunk more.
struct Ranges {
  int n, q, r;
  __device__ __forceinline__ Ranges(int total, int groups) {
    n = min(groups, total);
    q = total / n;
    r = total - q * n;
  }
  __device__ __forceinline__ int start(int w) const { return w * q + min(w, r); }
  __device__ __forceinline__ int owner(int c) const {
    const int wide = r * (q + 1);
    return c < wide ? c / (q + 1) : r + (c - wide) / q;
  }
};

// The sequence that chunk c (of all rows) belongs to, and its first chunk.
__device__ __forceinline__ void find_seq(const Seqs& s, int rows, int c, int lane, int& b, int& first) {
  int before = 0;
  for (int base = 0;; base += 64) {
    const int v = base + lane < s.B ? chunks_of(seq_len(s, base + lane)) * rows : 0;
    int incl = v;
#pragma unroll
    for (int k = 1; k < 64; k <<= 1) {
      const int u = __shfl_up(incl, k);
      if (lane >= k) incl += u;
    }
    const uint64_t past = __ballot(before + incl > c);
    if (past || base + 64 >= s.B) {
      const int l = past ? __builtin_ctzll(past) : 63;
      b = base + l;
      first = before + __shfl(incl - v, l);
      return;
    }
    before += __shfl(incl, 63);
  }
}

// Chunks of all rows of the sequences before b.
__device__ __forceinline__ int first_chunk(const Seqs& s, int rows, int b, int lane) {
  int n = 0;
  for (int i = lane; i < b; i += 64) n += chunks_of(seq_len(s, i));
#pragma unroll
  for (int k = 32; k; k >>= 1) n += __shfl_xor(n, k);
  return n * rows;
}

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

__device__ __forceinline__ f32x4 mfma(bf16x8 a, bf16x8 b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}

// DP: dim padded to 64, 128 or 256; FULL: dim == DP.
template <int DP, bool E4M3, bool F32, bool FULL>
__global__ __launch_bounds__(256) void attn_decode_kernel(AttnArgs a, Plan p) {
  constexpr int KS = DP / 32, VPL = DP / 16, QT = F32 ? 3 : 1, PT = F32 ? 3 : 2;
  constexpr int KL = E4M3 ? KS / 2 : KS;             // 16-byte key loads per key
  constexpr int VB = VPL * (E4M3 ? 1 : 2), VW = VB / 4;  // bytes and words per value load
  __shared__ float sm_m[4][16], sm_l[4][16];
  __shared__ __attribute__((aligned(16))) float sm_o[4][16][DP + 4];

  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, c = lane & 15, g = lane >> 4;
  const uint32_t D = a.kv.dim;
  const int total = sum_chunks(a.seqs, lane) * int(p.rows);
  const Ranges ranges(total, p.groups);
  const int w = blockIdx.x;
  if (w >= ranges.n) return;
  const int begin = ranges.start(w), end = ranges.start(w + 1);
  int b, first;
  find_seq(a.seqs, p.rows, begin, lane, b, first);
  b = __builtin_amdgcn_readfirstlane(b);
  first = __builtin_amdgcn_readfirstlane(first);

  for (int at = begin; at < end;) {
    int len = seq_len(a.seqs, b), chunks = chunks_of(len);
    while (at >= first + int(p.rows) * chunks) {
      first += int(p.rows) * chunks;
      ++b;
      len = seq_len(a.seqs, b);
      chunks = chunks_of(len);
    }
    const int row = (at - first) / chunks, c0 = (at - first) - row * chunks, nc = min(end - at, chunks - c0);
    const int hk = row / int(p.hgroups), gi = row - hk * int(p.hgroups);
    const int heads = min(16, int(a.group) - gi * 16);        // of this row
    const int head0 = hk * int(a.group) + gi * 16;            // its first query head
    const int stop = min(len, (c0 + nc) * kChunk);

    // the queries of the row; columns past its heads are zero
    bf16x8 q[QT][KS];
#pragma unroll
    for (int s = 0; s < KS; ++s) {
      const uint32_t d = E4M3 ? (s >> 1) * 64 + g * 16 + (s & 1) * 8 : s * 32 + g * 8;
      const bool in = c < heads && (FULL || d < D);
      const int64_t off = int64_t(b) * a.q_stride + int64_t(head0 + (in ? c : 0)) * D + (in ? d : 0);
      if constexpr (F32) {
        const float* src = static_cast<const float*>(a.q) + off;
        float v[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = in ? src[i] : 0.f;
        bf16x8 t[3];
        split8<3>(v, t);
#pragma unroll
        for (int k = 0; k < 3; ++k) q[k][s] = t[k];
      } else {
        u32x4 v = *reinterpret_cast<const u32x4*>(static_cast<const uint16_t*>(a.q) + off);
        if (!in) v = u32x4{0, 0, 0, 0};
        q[0][s] = __builtin_bit_cast(bf16x8, v);
      }
    }

    f32x4 o[VPL];
#pragma unroll
    for (int j = 0; j < VPL; ++j) o[j] = f32x4{0, 0, 0, 0};
    float m = kNegInf, l = 0.f;
    const float scale2 = a.scale * kLog2e;
    const uint8_t* kbase = a.kv.k + hk * a.kv.head_stride;
    const uint8_t* vbase = a.kv.v + hk * a.kv.head_stride;
    const int32_t* table = a.seqs.table + int64_t(b) * a.seqs.stride;

    for (int t0 = c0 * kChunk + wave * 32; t0 < stop; t0 += kChunk) {
      // lane i and lane i + 32 find slot t0 + i
      const int t = t0 + (lane & 31);
      const uint32_t pi = a.kv.per_page.div(t < stop ? t : 0), po = (t < stop ? t : 0) - pi * a.kv.page_size;
      const uint32_t page = uint32_t(table[pi]);
      const bool ok = t < stop && page < a.kv.pages;
      const uint32_t mask = uint32_t(__ballot(ok));
      const int64_t off = ok ? page * a.kv.page_stride + po * a.kv.slot_stride : 0;
      float ks = 1.f, vs = 1.f;
      if constexpr (E4M3) {
        const int64_t so = ok ? (int64_t(page) * a.kv.heads + hk) * a.kv.page_size + po : 0;
        ks = a.kv.k_scale[so];
        vs = a.kv.v_scale[so];
      }

      u32x4 kr[2][KL];
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const uint8_t* src = kbase + shfl64(off, u * 16 + c);
#pragma unroll
        for (int i = 0; i < KL; ++i) {
          const uint32_t d = E4M3 ? i * 64 + g * 16 : i * 32 + g * 8;
          const bool in = FULL || d < D;
          kr[u][i] = *reinterpret_cast<const u32x4*>(src + (in ? d * (E4M3 ? 1 : 2) : 0));
          if (!in) kr[u][i] = u32x4{0, 0, 0, 0};
        }
      }
      uint32_t vr[8][VW];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const uint32_t d = c * VPL;
        const uint8_t* src = vbase + shfl64(off, (i >> 2) * 16 + g * 4 + (i & 3)) + (FULL || d < D ? d * (E4M3 ? 1 : 2) : 0);
        if constexpr (VW % 4 == 0) {
#pragma unroll
          for (int x = 0; x < VW / 4; ++x) {
            const u32x4 r = reinterpret_cast<const u32x4*>(src)[x];
#pragma unroll
            for (int y = 0; y < 4; ++y) vr[i][x * 4 + y] = r[y];
          }
        } else if constexpr (VW == 2) {
          const uint2 r = *reinterpret_cast<const uint2*>(src);
          vr[i][0] = r.x;
          vr[i][1] = r.y;
        } else {
          vr[i][0] = *reinterpret_cast<const uint32_t*>(src);
        }
      }

      // scores of 32 slots x 16 heads, in log2 units
      float s[8];
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        f32x4 acc = {0, 0, 0, 0};
#pragma unroll
        for (int i = 0; i < KS; ++i) {
          bf16x8 kf;
          if constexpr (E4M3) {
            const u32x4 r = kr[u][i >> 1];
            kf = __builtin_bit_cast(bf16x8, widen8(r[(i & 1) * 2], r[(i & 1) * 2 + 1]));
          } else {
            kf = __builtin_bit_cast(bf16x8, kr[u][i]);
          }
#pragma unroll
          for (int k = QT - 1; k >= 0; --k) acc = mfma(kf, q[k][i], acc);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int tok = u * 16 + g * 4 + i;
          float z = acc[i] * scale2;
          if constexpr (E4M3) z *= __shfl(ks, tok);
          s[u * 4 + i] = mask >> tok & 1 ? z : kNegInf;
        }
      }
      if (p.scores && c < heads) {
        float* dst = p.scores + (int64_t(b) * a.heads_q + head0 + c) * p.score_ld + t0 + g * 4;
        *reinterpret_cast<float4*>(dst) = make_float4(s[0], s[1], s[2], s[3]);
        *reinterpret_cast<float4*>(dst + 16) = make_float4(s[4], s[5], s[6], s[7]);
      }

      float top = s[0];
#pragma unroll
      for (int i = 1; i < 8; ++i) top = fmaxf(top, s[i]);
      top = fmaxf(top, __shfl_xor(top, 16));
      top = fmaxf(top, __shfl_xor(top, 32));
      const float m_new = fmaxf(m, top), ref = m_new == kNegInf ? 0.f : m_new;
      const float alpha = __builtin_amdgcn_exp2f(m - ref);
      m = m_new;
      l *= alpha;
#pragma unroll
      for (int j = 0; j < VPL; ++j) o[j] *= alpha;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        s[i] = __builtin_amdgcn_exp2f(s[i] - ref);
        l += s[i];
        if constexpr (E4M3) {
          const int tok = (i >> 2) * 16 + g * 4 + (i & 3);
          const float y = __shfl(vs, tok);
          s[i] = mask >> tok & 1 ? s[i] * y : 0.f;
        }
      }
      bf16x8 pf[PT];
      split8<PT>(s, pf);

      // what lies in slots past the end may be NaN and takes no part
      if (mask != 0xFFFFFFFFu) {
#pragma unroll
        for (int i = 0; i < 8; ++i)
          if (!(mask >> ((i >> 2) * 16 + g * 4 + (i & 3)) & 1))
#pragma unroll
            for (int x = 0; x < VW; ++x) vr[i][x] = 0;
      }
      uint32_t vb[8][VPL / 2];  // bf16 pairs of neighbouring dimensions
#pragma unroll
      for (int i = 0; i < 8; ++i)
#pragma unroll
        for (int x = 0; x < VPL / 2; ++x) {
          if constexpr (E4M3)
            vb[i][x] = __builtin_bit_cast(
                uint32_t, x & 1 ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(vr[i][x >> 1], 1.f, true)
                                : __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(vr[i][x >> 1], 1.f, false));
          else
            vb[i][x] = vr[i][x];
        }
#pragma unroll
      for (int j = 0; j < VPL; ++j) {
        u32x4 f;
#pragma unroll
        for (int x = 0; x < 4; ++x)
          f[x] = __builtin_amdgcn_perm(vb[2 * x + 1][j >> 1], vb[2 * x][j >> 1], j & 1 ? 0x07060302u : 0x05040100u);
#pragma unroll
        for (int k = PT - 1; k >= 0; --k) o[j] = mfma(__builtin_bit_cast(bf16x8, f), pf[k], o[j]);
      }
    }

    // join the four waves
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
          *reinterpret_cast<float4*>(&sm_o[wave][c][(g * 4 + i) * VPL + j]) =
              make_float4(o[j][i], o[j + 1][i], o[j + 2][i], o[j + 3][i]);
    }
    __syncthreads();
    const bool whole = nc == chunks;
    float* part = p.part + (int64_t(w) * 2 + (at - c0 >= begin ? 1 : 0)) * (p.gh * (D + 2));
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
        }
      } else {
        if (d == 0) {
          part[h] = top;
          part[p.gh + h] = sum;
        }
        float* po = part + 2 * p.gh + h * D + d;
#pragma unroll
        for (int x = 0; x < 4; ++x) po[x] = r[x];
      }
    }
    __syncthreads();
    at += nc;
  }
}

// Where the partials of a row lie: those of workgroups w0 to w1, in order.
struct RowParts {
  int w0, w1, row_first;
  __device__ __forceinline__ RowParts(const AttnArgs& a, const Plan& p, const Ranges& ranges, int b, int row, int lane) {
    const int chunks = chunks_of(seq_len(a.seqs, b));
    row_first = first_chunk(a.seqs, p.rows, b, lane) + row * chunks;
    w0 = ranges.owner(row_first);
    w1 = ranges.owner(row_first + chunks - 1);
  }
  __device__ __forceinline__ const float* part(const AttnArgs& a, const Plan& p, const Ranges& ranges, int w) const {
    return p.part + (int64_t(w) * 2 + (row_first >= ranges.start(w) ? 1 : 0)) * (p.gh * (a.kv.dim + 2));
  }
};

// Maximum and sum of a head of a split row, by one wave.
__device__ __forceinline__ void head_stats(const AttnArgs& a, const Plan& p, const Ranges& ranges, const RowParts& rp,
                                           int h, int lane, float& top, float& sum) {
  top = kNegInf;
  for (int w = rp.w0 + lane; w <= rp.w1; w += 64) top = fmaxf(top, rp.part(a, p, ranges, w)[h]);
#pragma unroll
  for (int k = 32; k; k >>= 1) top = fmaxf(top, __shfl_xor(top, k));
  const float ref = top == kNegInf ? 0.f : top;
  sum = 0.f;
  for (int w = rp.w0 + lane; w <= rp.w1; w += 64) {
    const float* part = rp.part(a, p, ranges, w);
    sum += __builtin_amdgcn_exp2f(part[h] - ref) * part[p.gh + h];
  }
#pragma unroll
  for (int k = 32; k; k >>= 1) sum += __shfl_xor(sum, k);
}

// Workgroups below B * heads_q: the output of one head of a split row.  The
// rest (tracked calls): the attention weights of 256 slots of one key head.
template <bool F32>
__global__ __launch_bounds__(256) void attn_join_kernel(AttnArgs a, Plan p, int slot_blocks) {
  __shared__ __attribute__((aligned(16))) float sm[256 * 4];
  const int lane = threadIdx.x & 63;
  const uint32_t D = a.kv.dim;
  const Ranges ranges(sum_chunks(a.seqs, lane) * int(p.rows), p.groups);
  int id = blockIdx.x;
  if (id < a.seqs.B * int(a.heads_q)) {
    const int b = id / int(a.heads_q), hq = id - b * int(a.heads_q), hk = hq / int(a.group), gi = (hq - hk * int(a.group)) / 16;
    const int h = hq - hk * int(a.group) - gi * 16;
    const RowParts rp(a, p, ranges, b, hk * int(p.hgroups) + gi, lane);
    if (rp.w0 == rp.w1) return;  // the row was finished in one workgroup
    float top, sum;
    head_stats(a, p, ranges, rp, h, lane, top, sum);
    const float ref = top == kNegInf ? 0.f : top;
    // dim / 4 threads per partial, as many partials at a time as fit
    const int per = int(D) / 4, sets = 256 / per, set = threadIdx.x / per, d = (threadIdx.x - set * per) * 4;
    float r[4] = {0.f, 0.f, 0.f, 0.f};
    if (set < sets)
      for (int w = rp.w0 + set; w <= rp.w1; w += sets) {
        const float* part = rp.part(a, p, ranges, w);
        const float f = __builtin_amdgcn_exp2f(part[h] - ref);
        const float* po = part + 2 * p.gh + h * D + d;
#pragma unroll
        for (int x = 0; x < 4; ++x) r[x] += f * po[x];
      }
    *reinterpret_cast<float4*>(&sm[threadIdx.x * 4]) = make_float4(r[0], r[1], r[2], r[3]);
    __syncthreads();
    const int64_t qh = int64_t(b) * a.heads_q + hq;
    const float inv = sum == 0.f ? 0.f : 1.f / sum;
    for (int x = threadIdx.x; x < int(D); x += 256) {
      float y = 0.f;
      for (int k = 0; k < sets; ++k) y += sm[k * int(D) + x];
      y *= inv;
      if constexpr (F32) static_cast<float*>(a.out)[qh * D + x] = y;
      else static_cast<__bf16*>(a.out)[qh * D + x] = static_cast<__bf16>(y);
    }
    if (threadIdx.x == 0 && a.lse) a.lse[qh] = (top + __log2f(sum)) * kLn2;
    return;
  }
  id -= a.seqs.B * int(a.heads_q);
  const int b = id / (int(a.kv.heads) * slot_blocks), rest = id - b * int(a.kv.heads) * slot_blocks;
  const int hk = rest / slot_blocks, t = (rest - hk * slot_blocks) * 256 + threadIdx.x;
  const int len = seq_len(a.seqs, b);
  if (t - int(threadIdx.x) >= len) return;
  float w = 0.f;
  for (int gi = 0; gi < int(p.hgroups); ++gi) {
    const RowParts rp(a, p, ranges, b, hk * int(p.hgroups) + gi, lane);
    for (int h = 0; h < min(16, int(a.group) - gi * 16); ++h) {
      const int64_t qh = int64_t(b) * a.heads_q + hk * a.group + gi * 16 + h;
      float lse2;
      if (rp.w0 == rp.w1) {
        lse2 = p.lse2[qh];
      } else {
        float top, sum;
        head_stats(a, p, ranges, rp, h, lane, top, sum);
        lse2 = top + __log2f(sum);
      }
      if (t < len) {
        const float s = p.scores[qh * p.score_ld + t];
        if (lse2 != kNegInf) w += __builtin_amdgcn_exp2f(s - lse2);
      }
    }
  }
  if (t >= len) return;
  const uint32_t pi = a.kv.per_page.div(t), page = uint32_t(a.seqs.table[int64_t(b) * a.seqs.stride + pi]);
  if (page >= a.kv.pages) return;
  const int64_t at = (int64_t(page) * a.kv.heads + hk) * a.kv.page_size + (t - pi * a.kv.page_size);
  a.weight_out[at] = a.weight_in[at] + w;
}

struct Sizes {
  uint32_t hgroups, gh;
  int64_t score_ld;
  size_t part, lse2, scores;  // floats
};
Sizes sizes_of(uint32_t heads_kv, uint32_t dim, uint32_t heads_q, int64_t B, int64_t cap, bool track) {
  Sizes s;
  const uint32_t group = heads_q / heads_kv;
  s.hgroups = (group + 15) / 16;
  s.gh = group < 16 ? group : 16;
  s.score_ld = (cap + 31) / 32 * 32;
  const auto up = [](size_t n) { return (n + 3) / 4 * 4; };
  s.part = up(size_t(kMostGroups) * 2 * s.gh * (dim + 2));
  s.lse2 = up(size_t(B) * heads_q);
  s.scores = track ? size_t(B) * heads_q * size_t(s.score_ld) : 0;
  return s;
}

template <int DP, bool E4M3, bool F32>
void launch(const AttnArgs& a, const Plan& p, hipStream_t st) {
  if (a.kv.dim == DP) attn_decode_kernel<DP, E4M3, F32, true><<<p.groups, 256, 0, st>>>(a, p);
  else attn_decode_kernel<DP, E4M3, F32, false><<<p.groups, 256, 0, st>>>(a, p);
}
template <bool E4M3, bool F32>
void launch_dim(const AttnArgs& a, const Plan& p, hipStream_t st) {
  if (a.kv.dim <= 64) launch<64, E4M3, F32>(a, p, st);
  else if (a.kv.dim <= 128) launch<128, E4M3, F32>(a, p, st);
  else launch<256, E4M3, F32>(a, p, st);
}

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
  const int64_t most = int64_t(a.seqs.B) * p.rows * ((a.seqs.cap + kChunk - 1) / kChunk > 0 ? (a.seqs.cap + kChunk - 1) / kChunk : 1);
  p.groups = uint32_t(most < kMostGroups ? most : kMostGroups);
  p.score_ld = s.score_ld;
  p.part = a.ws;
  p.lse2 = p.part + s.part;
  p.scores = track ? p.lse2 + s.lse2 : nullptr;
  if (a.kv.e4m3) {
    if (f32) launch_dim<true, true>(a, p, st);
    else launch_dim<true, false>(a, p, st);
  } else {
    if (f32) launch_dim<false, true>(a, p, st);
    else launch_dim<false, false>(a, p, st);
  }
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const int slot_blocks = track ? (a.seqs.cap + 255) / 256 : 0;
  const uint32_t grid = uint32_t(int64_t(a.seqs.B) * a.heads_q + int64_t(a.seqs.B) * a.kv.heads * slot_blocks);
  if (f32) attn_join_kernel<true><<<grid, 256, 0, st>>>(a, p, slot_blocks);
  else attn_join_kernel<false><<<grid, 256, 0, st>>>(a, p, slot_blocks);
  return hipGetLastError();
}

}  // namespace sdq
