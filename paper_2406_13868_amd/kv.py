"""The decode step between the projections: a paged key-value cache and the
operators on it (sdq_qkv_append, sdq_attn_decode and sdq_cache_evict of
include/sdq.h).  As in the rest of the binding, arguments are checked and
marshalled here and all work is done by the library's kernels.

    cache = KVCache.empty(pages, heads, page_size, dim, "e4m3", track=True)
    q = qkv_append(qkv, pos, slot, cache, heads_q, cos_sin)       # norm, rotation, append
    o = attn_decode(q, cache, page_table, seq_lens, weight_out=cache.weight)
    seq_lens = cache_evict(cache, page_table, seq_lens, budget=4096, recent=256)
"""
from __future__ import annotations

import ctypes as C

from . import _dev, _lib, _need, _need_bytes, _same_device, _stream, _torch, _workspace, _x_dtype


class KVCache:
    """Keys and values in pages: k and v are [pages, heads, page_size, dim]
    tensors of bfloat16 or float8_e4m3fn (any strides that keep a row of dim
    elements together and 16-byte aligned, the same for both), k_scale and
    v_scale the fp32 [pages, heads, page_size] scales of e4m3 rows, position
    (int32) and weight (fp32) of the same shape what an evicted cache keeps of
    every slot.  The object holds the tensors; it owns no other memory."""

    __slots__ = ("k", "v", "k_scale", "v_scale", "position", "weight", "pages", "heads", "page_size", "dim", "device",
                 "_c", "_ref")

    def __init__(self, k, v, k_scale=None, v_scale=None, position=None, weight=None):
        torch = _torch()
        for t, what in ((k, "k"), (v, "v")):
            if not isinstance(t, torch.Tensor) or t.dim() != 4:
                raise ValueError(f"{what} must be a [pages, heads, page_size, dim] tensor")
        if k.dtype not in (torch.bfloat16, torch.float8_e4m3fn):
            raise ValueError("k must be bfloat16 or float8_e4m3fn")
        _need(v, k.shape, k.dtype, "v")
        if v.stride() != k.stride():
            raise ValueError("k and v must have the same strides")
        shape, stride = tuple(k.shape), k.stride()
        if min(shape) < 1:
            raise ValueError("a cache has at least one page, head, slot and dimension")
        if stride[3] != 1:
            raise ValueError("the elements of a row of k and v must be contiguous")
        _no_overlap(shape, stride)
        e4m3 = k.dtype == torch.float8_e4m3fn
        if e4m3 != (k_scale is not None) or e4m3 != (v_scale is not None):
            raise ValueError("k_scale and v_scale belong to an e4m3 cache")
        for t, dt, what in ((k_scale, torch.float32, "k_scale"), (v_scale, torch.float32, "v_scale"),
                            (position, torch.int32, "position"), (weight, torch.float32, "weight")):
            if t is not None:
                _need(t, shape[:3], dt, what)
        _same_device(k, v, k_scale, v_scale, position, weight)
        self.k, self.v, self.k_scale, self.v_scale, self.position, self.weight = k, v, k_scale, v_scale, position, weight
        self.pages, self.heads, self.page_size, self.dim = shape
        self.device = k.device
        for t, what in ((k, "k"), (v, "v")):
            if not t.is_cuda:
                raise ValueError(f"{what} must be a CUDA (HIP) tensor")
        opt = lambda t, what: None if t is None else _dev(t, what)  # noqa: E731
        self._c = _lib.sdq_kv_cache(
            k.data_ptr(), v.data_ptr(), opt(k_scale, "k_scale"), opt(v_scale, "v_scale"), opt(position, "position"),
            opt(weight, "weight"), shape[0], *(0 if n == 1 else s for n, s in zip(shape, stride[:3])),
            _lib.DTYPE_E4M3 if e4m3 else _lib.DTYPE_BF16, *shape[1:])
        self._ref = C.byref(self._c)

    @classmethod
    def empty(cls, pages: int, heads: int, page_size: int, dim: int, dtype: str = "bf16", track: bool = False,
              device="cuda"):
        """A cache over new tensors; dtype "bf16" or "e4m3", track: with position and weight."""
        torch = _torch()
        if dtype not in ("bf16", "e4m3"):
            raise ValueError("dtype must be 'bf16' or 'e4m3'")
        dt = torch.bfloat16 if dtype == "bf16" else torch.float8_e4m3fn
        new = lambda d, *more: torch.zeros((pages, heads, page_size, *more), dtype=d, device=device)  # noqa: E731
        scales = (new(torch.float32), new(torch.float32)) if dtype == "e4m3" else (None, None)
        state = (new(torch.int32).fill_(-1), new(torch.float32)) if track else (None, None)
        return cls(new(dt, dim), new(dt, dim), *scales, *state)

    def with_state(self, position, weight):
        """A cache over the same keys and values with other positions and weights."""
        return KVCache(self.k, self.v, self.k_scale, self.v_scale, position, weight)


def _no_overlap(shape, stride):
    """Rows written at different indexes must not share memory."""
    at = 1
    for n, s in sorted(((n, s) for n, s in zip(shape, stride) if n > 1), key=lambda x: x[1]):
        if s < at:
            raise ValueError("the elements of k and v overlap")
        at = s * n


def _seqs(cache, page_table, seq_lens):
    """B, and the page table's row stride."""
    torch = _torch()
    if not isinstance(page_table, torch.Tensor) or page_table.dim() != 2 or page_table.dtype != torch.int32:
        raise ValueError("page_table must be [sequences, pages] int32")
    B, width = page_table.shape
    _need(seq_lens, (B,), torch.int32, "seq_lens")
    if width > 1 and page_table.stride(1) != 1:
        raise ValueError("the rows of page_table must be contiguous")
    if not page_table.is_cuda:
        raise ValueError("page_table must be a CUDA (HIP) tensor")
    return B, width, page_table.stride(0) if B > 1 else width


def qkv_append(qkv, pos, slot, cache: KVCache, heads_q: int, cos_sin=None, interleaved: bool = False, q_weight=None,
               k_weight=None, eps: float = 1e-6, out=None, out_dtype=None, stream=None):
    """Norm (with q_weight and k_weight), position rotation (with cos_sin) and
    append of new tokens, in one pass: returns the queries [M, heads_q, dim].

    qkv is [M, (heads_q + 2 heads) * dim], fp32 or bf16, the output of a stacked
    projection (rows may be strided); pos int32 [M]; slot int64 [M], page *
    page_size + offset, negative for a row that is only padding; cos_sin fp32
    [positions, rot_dim], cosines then sines.  Queries have out_dtype, by
    default qkv's."""
    torch = _torch()
    if not isinstance(qkv, torch.Tensor) or qkv.dim() != 2:
        raise ValueError("qkv must be [M, (heads_q + 2 heads) * dim]")
    M, width = qkv.shape
    dim = cache.dim
    if heads_q < 1 or width != (heads_q + 2 * cache.heads) * dim:
        raise ValueError(f"qkv must be [M, {(heads_q + 2 * cache.heads) * dim}], got {list(qkv.shape)}")
    if qkv.stride(1) != 1 or not qkv.is_cuda:
        raise ValueError("qkv must be a CUDA (HIP) tensor with contiguous rows")
    dt = _x_dtype(qkv)
    _need(slot, (M,), torch.int64, "slot")
    if pos is not None:
        _need(pos, (M,), torch.int32, "pos")
    elif cos_sin is not None or cache.position is not None:
        raise ValueError("pos is needed for the rotation and for a cache that keeps positions")
    rot, positions = 0, 0
    if cos_sin is not None:
        if cos_sin.dim() != 2 or cos_sin.dtype != torch.float32:
            raise ValueError("cos_sin must be [positions, rot_dim] float32")
        positions, rot = cos_sin.shape
    if (q_weight is None) != (k_weight is None):
        raise ValueError("q_weight and k_weight go together")
    if q_weight is not None:
        _need(q_weight, (dim,), torch.float32, "q_weight")
        _need(k_weight, (dim,), torch.float32, "k_weight")
    if out is None:
        out = torch.empty((M, heads_q, dim), dtype=out_dtype or qkv.dtype, device=qkv.device)
    else:
        _need(out, (M, heads_q, dim), out_dtype or out.dtype, "out")
    _same_device(qkv, pos, slot, cache.k, cos_sin, q_weight, k_weight, out)
    t = _lib.sdq_qk_transform(None if q_weight is None else _dev(q_weight, "q_weight"),
                              None if k_weight is None else _dev(k_weight, "k_weight"),
                              _dev(cos_sin, "cos_sin") if rot else None, positions, heads_q, rot, interleaved, eps)
    _lib.check(_lib.lib().sdq_qkv_append(cache._ref, C.byref(t), qkv.data_ptr(), dt, M,
                                         qkv.stride(0) if M > 1 else width, None if pos is None else _dev(pos, "pos"),
                                         _dev(slot, "slot"), _dev(out, "out"), _x_dtype(out), _stream(stream)),
               "sdq_qkv_append")
    return out


def attn_decode_workspace_size(cache: KVCache, B: int, heads_q: int, max_len: int, track: bool = False) -> int:
    """Device workspace bytes of attn_decode for these sizes (track: with weight_out)."""
    n = C.c_size_t()
    _lib.check(_lib.lib().sdq_attn_decode_workspace_size(cache._ref, B, heads_q, max_len, track, C.byref(n)),
               "sdq_attn_decode_workspace_size")
    return n.value


def attn_decode(q, cache: KVCache, page_table, seq_lens, max_len=None, scale=None, out=None, lse=None, weight_out=None,
                workspace=None, stream=None):
    """Attention of one new token per sequence over the cache: returns [B, heads_q, dim] of q's dtype.

    q is [B, heads_q, dim], fp32 or bf16 (sequences may be strided), page_table
    int32 [B, pages], seq_lens int32 [B]; max_len is an upper bound of the
    lengths (default: what the page table holds), scale defaults to dim ** -0.5.
    lse (fp32 [B, heads_q]) receives the logarithm of the softmax sums.
    weight_out (cache.weight itself, or a tensor like it) receives cache.weight
    plus each slot's attention weight, summed over the query heads of its key
    head.  workspace: a uint8 tensor of attn_decode_workspace_size bytes, or a
    fresh one is made."""
    torch = _torch()
    B, width, ld = _seqs(cache, page_table, seq_lens)
    if not isinstance(q, torch.Tensor) or q.dim() != 3 or q.shape[0] != B or q.shape[2] != cache.dim:
        raise ValueError(f"q must be [{B}, heads_q, {cache.dim}]")
    heads_q = q.shape[1]
    dt = _x_dtype(q)
    if not q.is_cuda or q.stride(2) != 1 or (heads_q > 1 and q.stride(1) != cache.dim):
        raise ValueError("q must be a CUDA (HIP) tensor whose sequences are contiguous")
    if out is None:
        out = torch.empty((B, heads_q, cache.dim), dtype=q.dtype, device=q.device)
    else:
        _need(out, q.shape, q.dtype, "out")
    if lse is not None:
        _need(lse, (B, heads_q), torch.float32, "lse")
    if weight_out is not None:
        if cache.weight is None:
            raise ValueError("weight_out needs a cache that keeps weights")
        _need(weight_out, cache.weight.shape, torch.float32, "weight_out")
    cap = width * cache.page_size
    if max_len is not None and max_len < cap:
        cap = max_len
    _same_device(q, cache.k, page_table, seq_lens, out, lse, weight_out, workspace)
    track = weight_out is not None
    if workspace is None:
        need = attn_decode_workspace_size(cache, B, heads_q, cap, track)
        workspace = _workspace(need, q.device, stream)
    rc = _lib.lib().sdq_attn_decode(
        cache._ref, q.data_ptr(), dt, B, heads_q, q.stride(0) if B > 1 else heads_q * cache.dim, page_table.data_ptr(),
        ld, width, _dev(seq_lens, "seq_lens"), cap, cache.dim ** -0.5 if scale is None else scale, _dev(out, "out"),
        None if lse is None else _dev(lse, "lse"), _dev(weight_out, "weight_out") if track else None,
        _dev(workspace, "workspace"), workspace.nbytes, _stream(stream))
    if rc == _lib.ERR_BUFFER_TOO_SMALL:
        _need_bytes(workspace, attn_decode_workspace_size(cache, B, heads_q, cap, track), "workspace")
    _lib.check(rc, "sdq_attn_decode")
    return out


def cache_evict_workspace_size(cache: KVCache, B: int, max_len: int, budget: int) -> int:
    """Device workspace bytes of cache_evict for these sizes."""
    n = C.c_size_t()
    _lib.check(_lib.lib().sdq_cache_evict_workspace_size(cache._ref, B, max_len, budget, C.byref(n)),
               "sdq_cache_evict_workspace_size")
    return n.value


def cache_evict(cache: KVCache, page_table, seq_lens, budget: int, recent: int = 0, max_len=None, lens_out=None,
                weight_out=None, position_out=None, workspace=None, stream=None):
    """Keep `budget` slots of every longer sequence, per key head: the recent
    ones, then those of the largest weight.  Returns the new lengths, in lens_out
    (which may be seq_lens) or a new tensor.

    Keys, values and scales move in place.  Positions and weights are updated in
    place too, or written to position_out and weight_out (both, and not the
    cache's own)."""
    torch = _torch()
    B, width, ld = _seqs(cache, page_table, seq_lens)
    if cache.position is None or cache.weight is None:
        raise ValueError("eviction needs a cache that keeps positions and weights")
    if (weight_out is None) != (position_out is None):
        raise ValueError("weight_out and position_out go together")
    if weight_out is None:
        weight_out, position_out = cache.weight, cache.position
    _need(weight_out, cache.weight.shape, torch.float32, "weight_out")
    _need(position_out, cache.weight.shape, torch.int32, "position_out")
    if lens_out is None:
        lens_out = torch.empty_like(seq_lens)
    else:
        _need(lens_out, (B,), torch.int32, "lens_out")
    cap = width * cache.page_size
    if max_len is not None and max_len < cap:
        cap = max_len
    _same_device(cache.k, page_table, seq_lens, lens_out, weight_out, position_out, workspace)
    if workspace is None:
        need = cache_evict_workspace_size(cache, B, cap, budget)
        workspace = _workspace(need, cache.device, stream)
    rc = _lib.lib().sdq_cache_evict(
        cache._ref, B, page_table.data_ptr(), ld, width, _dev(seq_lens, "seq_lens"), cap, budget, recent,
        _dev(lens_out, "lens_out"), _dev(position_out, "position_out"), _dev(weight_out, "weight_out"),
        _dev(workspace, "workspace"), workspace.nbytes, _stream(stream))
    if rc == _lib.ERR_BUFFER_TOO_SMALL:
        _need_bytes(workspace, cache_evict_workspace_size(cache, B, cap, budget), "workspace")
    _lib.check(rc, "sdq_cache_evict")
    return lens_out
