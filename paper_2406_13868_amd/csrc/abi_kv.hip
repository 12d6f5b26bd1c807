// C ABI of the operators on the paged cache: argument validation and dispatch
// (see include/sdq.h).
#include <hip/hip_runtime.h>

#include <cmath>

#include "kv_cache.h"
#include "sdq.h"

using namespace sdq;

namespace {

bool aligned16(const void* p) { return reinterpret_cast<uintptr_t>(p) % 16 == 0; }

// Validates a cache; fills `out` on success.
sdq_status check_cache(const sdq_kv_cache* c, KV* out) {
  if (!c) return SDQ_ERR_NULL;
  if (c->dtype != SDQ_DTYPE_BF16 && c->dtype != SDQ_DTYPE_E4M3) return SDQ_ERR_CONFIG;
  const bool e4m3 = c->dtype == SDQ_DTYPE_E4M3;
  if (c->heads < 1 || c->heads > 1024 || c->dim < 16 || c->dim > 256 || c->dim % 16 || c->page_size < 1 ||
      c->page_size > (1 << 20) || c->pages < 1 || c->pages >= (int64_t(1) << 31) / c->page_size)
    return SDQ_ERR_SHAPE;
  if (!c->k || !c->v || (e4m3 && (!c->k_scale || !c->v_scale))) return SDQ_ERR_NULL;
  const int64_t elt = e4m3 ? 1 : 2;
  const int64_t strides[3] = {c->page_stride, c->head_stride, c->slot_stride};
  for (const int64_t s : strides)
    if (s < 0 || s > (int64_t(1) << 40) || s * elt % 16) return SDQ_ERR_SHAPE;
  if (!aligned16(c->k) || !aligned16(c->v)) return SDQ_ERR_SHAPE;
  if (out) {
    out->k = static_cast<uint8_t*>(c->k);
    out->v = static_cast<uint8_t*>(c->v);
    out->k_scale = e4m3 ? c->k_scale : nullptr;
    out->v_scale = e4m3 ? c->v_scale : nullptr;
    out->position = c->position;
    out->weight = c->weight;
    out->page_stride = c->page_stride * elt;
    out->head_stride = c->head_stride * elt;
    out->slot_stride = c->slot_stride * elt;
    out->pages = uint32_t(c->pages);
    out->heads = uint32_t(c->heads);
    out->page_size = uint32_t(c->page_size);
    out->dim = uint32_t(c->dim);
    out->per_page = FastDiv(uint32_t(c->page_size));
    out->e4m3 = e4m3;
  }
  return SDQ_OK;
}

// Validates B sequences of up to max_len slots; fills `out` on success.
sdq_status check_seqs(const sdq_kv_cache* c, int64_t B, const int32_t* table, int64_t stride, int64_t max_pages,
                      const int32_t* lens, int64_t max_len, Seqs* out) {
  if (B < 0 || B > (int64_t(1) << 20) || max_len < 0 || max_pages < 0 || stride < 0 || stride > (int64_t(1) << 40) ||
      max_pages >= (int64_t(1) << 31))
    return SDQ_ERR_SHAPE;
  int64_t cap = max_pages * c->page_size;
  if (max_len < cap) cap = max_len;
  if (cap >= (int64_t(1) << 31) - 4096) return SDQ_ERR_SHAPE;
  if (B > 0 && (!lens || (cap > 0 && !table))) return SDQ_ERR_NULL;
  out->table = table;
  out->lens = lens;
  out->stride = stride;
  out->B = int32_t(B);
  out->cap = int32_t(cap);
  return SDQ_OK;
}

bool heads_fit(const sdq_kv_cache* c, int32_t heads_q) {
  return heads_q >= 1 && heads_q <= 1024 && heads_q % c->heads == 0;
}

// Whether the chunk, workgroup and score counts of an attention call fit the
// kernels' 32-bit indexes.
bool attn_fits(const sdq_kv_cache* c, int64_t B, int32_t heads_q, int64_t cap) {
  const int64_t rows = int64_t(c->heads) * ((heads_q / c->heads + 15) / 16), lim = int64_t(1) << 31;
  const int64_t chunks = (cap + 127) / 128 + 8, blocks = (cap + 255) / 256;
  return B * rows < lim / chunks && B * (heads_q + c->heads * blocks) < lim / 2;
}

// An error that an earlier HIP call on this thread left pending is not this
// call's: it is read before the launches.
void drop_pending_error() { (void)hipGetLastError(); }

}  // namespace

extern "C" sdq_status sdq_qkv_append(const sdq_kv_cache* cache, const sdq_qk_transform* t, const void* qkv,
                                     int32_t x_dtype, int64_t M, int64_t row_stride, const int32_t* pos,
                                     const int64_t* slot, void* q_out, int32_t q_dtype, void* stream) {
  AppendArgs a;
  const sdq_status s = check_cache(cache, &a.kv);
  if (s != SDQ_OK) return s;
  if (!t) return SDQ_ERR_NULL;
  if ((x_dtype != SDQ_DTYPE_F32 && x_dtype != SDQ_DTYPE_BF16) || (q_dtype != SDQ_DTYPE_F32 && q_dtype != SDQ_DTYPE_BF16))
    return SDQ_ERR_CONFIG;
  if (t->rot_dim < 0 || t->rot_dim > cache->dim || t->rot_dim % 2 || (t->interleaved != 0 && t->interleaved != 1) ||
      !t->q_weight != !t->k_weight || (t->q_weight && !(t->eps >= 0.f && std::isfinite(t->eps))))
    return SDQ_ERR_CONFIG;
  const int64_t heads = int64_t(t->heads_q) + 2 * cache->heads;
  if (!heads_fit(cache, t->heads_q) || M < 0 || M > ((int64_t(1) << 26) - 1) / heads || t->positions < 0 ||
      t->positions >= (int64_t(1) << 31))
    return SDQ_ERR_SHAPE;
  const int64_t elt = x_dtype == SDQ_DTYPE_F32 ? 4 : 2;
  if (row_stride < heads * cache->dim || row_stride > (int64_t(1) << 40) || row_stride * elt % 16) return SDQ_ERR_SHAPE;
  if (M == 0) return SDQ_OK;
  if (!qkv || !slot || !q_out || (t->rot_dim && !t->cos_sin) || ((t->rot_dim || cache->position) && !pos))
    return SDQ_ERR_NULL;
  if (!aligned16(qkv) || !aligned16(q_out) || !aligned16(t->q_weight) || !aligned16(t->k_weight) || !aligned16(t->cos_sin))
    return SDQ_ERR_SHAPE;
  a.qkv = qkv;
  a.row_stride = row_stride;
  a.pos = pos;
  a.slot = slot;
  a.q_weight = t->q_weight;
  a.k_weight = t->k_weight;
  a.cos_sin = t->cos_sin;
  a.q_out = q_out;
  a.positions = t->positions;
  a.M = uint32_t(M);
  a.heads_q = uint32_t(t->heads_q);
  a.rot = uint32_t(t->rot_dim);
  a.eps = t->eps;
  a.interleaved = t->interleaved != 0;
  drop_pending_error();
  const hipError_t e =
      launch_qkv_append(a, x_dtype == SDQ_DTYPE_F32, q_dtype == SDQ_DTYPE_F32, static_cast<hipStream_t>(stream));
  return e == hipSuccess ? SDQ_OK : SDQ_ERR_HIP;
}

extern "C" sdq_status sdq_attn_decode_workspace_size(const sdq_kv_cache* cache, int64_t B, int32_t heads_q,
                                                     int64_t max_len, int32_t track, size_t* bytes) {
  const sdq_status s = check_cache(cache, nullptr);
  if (s != SDQ_OK) return s;
  if (!bytes) return SDQ_ERR_NULL;
  if (B < 0 || B > (int64_t(1) << 20) || max_len < 0 || max_len >= (int64_t(1) << 31) - 4096 || !heads_fit(cache, heads_q) ||
      !attn_fits(cache, B, heads_q, max_len))
    return SDQ_ERR_SHAPE;
  *bytes = attn_decode_workspace_bytes(cache->heads, cache->dim, heads_q, B, max_len, track != 0);
  return SDQ_OK;
}

extern "C" sdq_status sdq_attn_decode(const sdq_kv_cache* cache, const void* q, int32_t dtype, int64_t B,
                                      int32_t heads_q, int64_t q_stride, const int32_t* page_table,
                                      int64_t table_stride, int64_t max_pages, const int32_t* seq_lens,
                                      int64_t max_len, float scale, void* out, float* lse, float* weight_out,
                                      void* workspace, size_t ws_bytes, void* stream) {
  AttnArgs a;
  sdq_status s = check_cache(cache, &a.kv);
  if (s != SDQ_OK) return s;
  if (dtype != SDQ_DTYPE_F32 && dtype != SDQ_DTYPE_BF16) return SDQ_ERR_CONFIG;
  s = check_seqs(cache, B, page_table, table_stride, max_pages, seq_lens, max_len, &a.seqs);
  if (s != SDQ_OK) return s;
  if (!std::isfinite(scale)) return SDQ_ERR_VALUE;
  if (weight_out && !cache->weight) return SDQ_ERR_NULL;
  const int64_t elt = dtype == SDQ_DTYPE_F32 ? 4 : 2;
  if (!heads_fit(cache, heads_q) || !attn_fits(cache, B, heads_q, a.seqs.cap) ||
      q_stride < int64_t(heads_q) * cache->dim || q_stride > (int64_t(1) << 40) || q_stride * elt % 16)
    return SDQ_ERR_SHAPE;
  if (B == 0) return SDQ_OK;
  if (!q || !out || !workspace) return SDQ_ERR_NULL;
  if (!aligned16(q) || !aligned16(out) || !aligned16(workspace)) return SDQ_ERR_SHAPE;
  if (ws_bytes < attn_decode_workspace_bytes(cache->heads, cache->dim, heads_q, B, a.seqs.cap, weight_out != nullptr))
    return SDQ_ERR_BUFFER_TOO_SMALL;
  a.q = q;
  a.q_stride = q_stride;
  a.heads_q = uint32_t(heads_q);
  a.group = uint32_t(heads_q / cache->heads);
  a.scale = scale;
  a.out = out;
  a.lse = lse;
  a.weight_in = cache->weight;
  a.weight_out = weight_out;
  a.ws = static_cast<float*>(workspace);
  drop_pending_error();
  const hipError_t e = launch_attn_decode(a, dtype == SDQ_DTYPE_F32, static_cast<hipStream_t>(stream));
  return e == hipSuccess ? SDQ_OK : SDQ_ERR_HIP;
}

extern "C" sdq_status sdq_cache_evict_workspace_size(const sdq_kv_cache* cache, int64_t B, int64_t max_len,
                                                     int64_t budget, size_t* bytes) {
  const sdq_status s = check_cache(cache, nullptr);
  if (s != SDQ_OK) return s;
  if (!bytes) return SDQ_ERR_NULL;
  if (B < 0 || B > (int64_t(1) << 20) || max_len < 0 || max_len >= (int64_t(1) << 31) - 4096 || budget < 1)
    return SDQ_ERR_SHAPE;
  *bytes = cache_evict_workspace_bytes(cache->heads, B, max_len, budget);
  return SDQ_OK;
}

extern "C" sdq_status sdq_cache_evict(const sdq_kv_cache* cache, int64_t B, const int32_t* page_table,
                                      int64_t table_stride, int64_t max_pages, const int32_t* seq_lens,
                                      int64_t max_len, int64_t budget, int64_t recent, int32_t* lens_out,
                                      int32_t* position_out, float* weight_out, void* workspace, size_t ws_bytes,
                                      void* stream) {
  EvictArgs a;
  sdq_status s = check_cache(cache, &a.kv);
  if (s != SDQ_OK) return s;
  if (!cache->position || !cache->weight) return SDQ_ERR_NULL;
  s = check_seqs(cache, B, page_table, table_stride, max_pages, seq_lens, max_len, &a.seqs);
  if (s != SDQ_OK) return s;
  if (budget < 1 || recent < 0 || recent > budget || B * cache->heads >= (int64_t(1) << 28)) return SDQ_ERR_SHAPE;
  if (B == 0) return SDQ_OK;
  if (!lens_out || !position_out || !weight_out || !workspace) return SDQ_ERR_NULL;
  if ((position_out == cache->position) != (weight_out == cache->weight)) return SDQ_ERR_CONFIG;
  if (!aligned16(workspace)) return SDQ_ERR_SHAPE;
  if (ws_bytes < cache_evict_workspace_bytes(cache->heads, B, a.seqs.cap, budget)) return SDQ_ERR_BUFFER_TOO_SMALL;
  // no sequence is longer than the cap
  a.budget = int32_t(budget < a.seqs.cap ? budget : a.seqs.cap);
  a.recent = int32_t(recent < a.seqs.cap ? recent : a.seqs.cap);
  a.lens_out = lens_out;
  a.position_out = position_out;
  a.weight_out = weight_out;
  a.ws = static_cast<int32_t*>(workspace);
  drop_pending_error();
  const hipError_t e = launch_cache_evict(a, static_cast<hipStream_t>(stream));
  return e == hipSuccess ? SDQ_OK : SDQ_ERR_HIP;
}
