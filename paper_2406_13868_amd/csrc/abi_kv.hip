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

// Workgroups of 256 or 1024 threads: the threads of a launch are counted in 32 bits.
constexpr int64_t kMostBlocks256 = (int64_t(1) << 24) - 1, kMostBlocks1024 = (int64_t(1) << 22) - 1;

// Whether the chunk and workgroup counts of an attention call fit.
bool attn_fits(const sdq_kv_cache* c, int64_t B, int32_t heads_q, int64_t cap, bool track) {
  const int64_t rows = int64_t(c->heads) * ((heads_q / c->heads + 15) / 16), lim = int64_t(1) << 31;
  const int64_t chunks = (cap + 127) / 128 + 8, blocks = track ? (cap + 1023) / 1024 : 0;
  return B * rows < lim / chunks && B * (heads_q + c->heads * blocks) <= kMostBlocks256;
}

// An error that an earlier HIP call on this thread left pending is not this
// call's: it is read before the launches.
void drop_pending_error() { (void)hipGetLastError(); }

}  // namespace

extern "C" sdq_status sdq_qkv_append(const sdq_kv_cache* cache, const sdq_append_args* t, void* stream) {
  AppendArgs a;
  const sdq_status s = check_cache(cache, &a.kv);
  if (s != SDQ_OK) return s;
  if (!t) return SDQ_ERR_NULL;
  if ((t->x_dtype != SDQ_DTYPE_F32 && t->x_dtype != SDQ_DTYPE_BF16) ||
      (t->q_dtype != SDQ_DTYPE_F32 && t->q_dtype != SDQ_DTYPE_BF16))
    return SDQ_ERR_CONFIG;
  if (t->rot_dim < 0 || t->rot_dim > cache->dim || t->rot_dim % 2 || (t->interleaved != 0 && t->interleaved != 1) ||
      !t->q_weight != !t->k_weight || (t->q_weight && !(t->eps >= 0.f && std::isfinite(t->eps))))
    return SDQ_ERR_CONFIG;
  const int64_t heads = int64_t(t->heads_q) + 2 * cache->heads, M = t->M;
  if (!heads_fit(cache, t->heads_q) || M < 0 || M > ((int64_t(1) << 26) - 1) / heads || t->positions < 0 ||
      t->positions >= (int64_t(1) << 31))
    return SDQ_ERR_SHAPE;
  const int64_t elt = t->x_dtype == SDQ_DTYPE_F32 ? 4 : 2;
  if (t->row_stride < heads * cache->dim || t->row_stride > (int64_t(1) << 40) || t->row_stride * elt % 16)
    return SDQ_ERR_SHAPE;
  if (M == 0) return SDQ_OK;
  if (!t->qkv || !t->slot || !t->q_out || (t->rot_dim && !t->cos_sin) || ((t->rot_dim || cache->position) && !t->pos))
    return SDQ_ERR_NULL;
  if (t->rot_dim && t->positions == 0) return SDQ_ERR_SHAPE;  // the kernel reads row 0 for a position outside the table
  if (!aligned16(t->qkv) || !aligned16(t->q_out) || !aligned16(t->q_weight) || !aligned16(t->k_weight) ||
      !aligned16(t->cos_sin))
    return SDQ_ERR_SHAPE;
  a.qkv = t->qkv;
  a.row_stride = t->row_stride;
  a.pos = t->pos;
  a.slot = t->slot;
  a.q_weight = t->q_weight;
  a.k_weight = t->k_weight;
  a.cos_sin = t->cos_sin;
  a.q_out = t->q_out;
  a.positions = t->positions;
  a.M = uint32_t(M);
  a.heads_q = uint32_t(t->heads_q);
  a.rot = uint32_t(t->rot_dim);
  a.eps = t->eps;
  a.interleaved = t->interleaved != 0;
  drop_pending_error();
  const hipError_t e =
      launch_qkv_append(a, t->x_dtype == SDQ_DTYPE_F32, t->q_dtype == SDQ_DTYPE_F32, static_cast<hipStream_t>(stream));
  return e == hipSuccess ? SDQ_OK : SDQ_ERR_HIP;
}

extern "C" sdq_status sdq_attn_decode_workspace_size(const sdq_kv_cache* cache, int64_t B, int32_t heads_q,
                                                     int64_t max_len, int32_t track, size_t* bytes) {
  const sdq_status s = check_cache(cache, nullptr);
  if (s != SDQ_OK) return s;
  if (!bytes) return SDQ_ERR_NULL;
  if (B < 0 || B > (int64_t(1) << 20) || max_len < 0 || max_len >= (int64_t(1) << 31) - 4096 || !heads_fit(cache, heads_q) ||
      !attn_fits(cache, B, heads_q, max_len, track != 0))
    return SDQ_ERR_SHAPE;
  *bytes = attn_decode_workspace_bytes(cache->heads, cache->dim, heads_q, B, max_len, track != 0);
  return SDQ_OK;
}

extern "C" sdq_status sdq_attn_decode(const sdq_kv_cache* cache, const sdq_attn_args* t, void* stream) {
  AttnArgs a;
  sdq_status s = check_cache(cache, &a.kv);
  if (s != SDQ_OK) return s;
  if (!t) return SDQ_ERR_NULL;
  if (t->dtype != SDQ_DTYPE_F32 && t->dtype != SDQ_DTYPE_BF16) return SDQ_ERR_CONFIG;
  s = check_seqs(cache, t->B, t->page_table, t->table_stride, t->max_pages, t->seq_lens, t->max_len, &a.seqs);
  if (s != SDQ_OK) return s;
  if (!std::isfinite(t->scale)) return SDQ_ERR_VALUE;
  if (t->weight_out && !cache->weight) return SDQ_ERR_NULL;
  const int64_t elt = t->dtype == SDQ_DTYPE_F32 ? 4 : 2;
  if (!heads_fit(cache, t->heads_q) || !attn_fits(cache, t->B, t->heads_q, a.seqs.cap, t->weight_out != nullptr) ||
      t->q_stride < int64_t(t->heads_q) * cache->dim || t->q_stride > (int64_t(1) << 40) || t->q_stride * elt % 16)
    return SDQ_ERR_SHAPE;
  if (t->B == 0) return SDQ_OK;
  if (!t->q || !t->out || !t->workspace) return SDQ_ERR_NULL;
  if (!aligned16(t->q) || !aligned16(t->out) || !aligned16(t->workspace)) return SDQ_ERR_SHAPE;
  if (t->ws_bytes <
      attn_decode_workspace_bytes(cache->heads, cache->dim, t->heads_q, t->B, a.seqs.cap, t->weight_out != nullptr))
    return SDQ_ERR_BUFFER_TOO_SMALL;
  a.q = t->q;
  a.q_stride = t->q_stride;
  a.heads_q = uint32_t(t->heads_q);
  a.group = uint32_t(t->heads_q / cache->heads);
  a.scale = t->scale;
  a.out = t->out;
  a.lse = t->lse;
  a.weight_in = cache->weight;
  a.weight_out = t->weight_out;
  a.ws = static_cast<float*>(t->workspace);
  drop_pending_error();
  const hipError_t e = launch_attn_decode(a, t->dtype == SDQ_DTYPE_F32, static_cast<hipStream_t>(stream));
  return e == hipSuccess ? SDQ_OK : SDQ_ERR_HIP;
}

extern "C" sdq_status sdq_cache_evict_workspace_size(const sdq_kv_cache* cache, int64_t B, int64_t max_len,
                                                     int64_t budget, size_t* bytes) {
  const sdq_status s = check_cache(cache, nullptr);
  if (s != SDQ_OK) return s;
  if (!bytes) return SDQ_ERR_NULL;
  if (B < 0 || B > (int64_t(1) << 20) || max_len < 0 || max_len >= (int64_t(1) << 31) - 4096 || budget < 1 ||
      B * cache->heads > kMostBlocks1024)
    return SDQ_ERR_SHAPE;
  *bytes = cache_evict_workspace_bytes(cache->heads, B, max_len, budget);
  return SDQ_OK;
}

extern "C" sdq_status sdq_cache_evict(const sdq_kv_cache* cache, const sdq_evict_args* t, void* stream) {
  EvictArgs a;
  sdq_status s = check_cache(cache, &a.kv);
  if (s != SDQ_OK) return s;
  if (!t || !cache->position || !cache->weight) return SDQ_ERR_NULL;
  s = check_seqs(cache, t->B, t->page_table, t->table_stride, t->max_pages, t->seq_lens, t->max_len, &a.seqs);
  if (s != SDQ_OK) return s;
  if (t->budget < 1 || t->recent < 0 || t->recent > t->budget || t->B * cache->heads > kMostBlocks1024)
    return SDQ_ERR_SHAPE;
  if (t->B == 0) return SDQ_OK;
  if (!t->lens_out || !t->position_out || !t->weight_out || !t->workspace) return SDQ_ERR_NULL;
  if ((t->position_out == cache->position) != (t->weight_out == cache->weight)) return SDQ_ERR_CONFIG;
  if (!aligned16(t->workspace)) return SDQ_ERR_SHAPE;
  if (t->ws_bytes < cache_evict_workspace_bytes(cache->heads, t->B, a.seqs.cap, t->budget)) return SDQ_ERR_BUFFER_TOO_SMALL;
  // no sequence is longer than the cap
  a.budget = int32_t(t->budget < a.seqs.cap ? t->budget : a.seqs.cap);
  a.recent = int32_t(t->recent < a.seqs.cap ? t->recent : a.seqs.cap);
  a.lens_out = t->lens_out;
  a.position_out = t->position_out;
  a.weight_out = t->weight_out;
  a.ws = static_cast<int32_t*>(t->workspace);
  drop_pending_error();
  const hipError_t e = launch_cache_evict(a, static_cast<hipStream_t>(stream));
  return e == hipSuccess ? SDQ_OK : SDQ_ERR_HIP;
}
