"""The decode step between the projections: a paged key-value cache and the
operators on it (sdq_qkv_append, sdq_attn_decode and sdq_cache_evict of
include/sdq.h).  As in the rest of the binding, arguments are checked and
marshalled here and all work is done by the library's kernels.

    cache = KVCache.empty(pages, heads, page_size, dim, "e4m3", track=True)
    q = qkv_append(qkv, pos, slot, cache, heads_q, cos_sin)       # norm, rotation, append
    o = attn_decode(q, cache, page_table, seq_lens, max_len=longest, weight_out=cache.weight)
    seq_lens = cache_evict(cache, page_table, seq_lens, budget=4096, recent=256, max_len=longest)
"""
from __future__ import annotations

import ctypes as C
import struct

from . import _dev, _empty, _lib, _need, _need_bytes, _same_device, _torch, _workspace, _x_dtype

# The argument structures as bytes: packing one takes a fraction of the time
# that filling a ctypes structure, or passing as many arguments, does.
_APPEND = struct.Struct("@7P3q5if")
_ATTN = struct.Struct("@7PN5q2if0q")
_EVICT = struct.Struct("@6PN6q")
assert _APPEND.size == C.sizeof(_lib.sdq_append_args)
assert _ATTN.size == C.sizeof(_lib.sdq_attn_args)
assert _EVICT.size == C.sizeof(_lib.sdq_evict_args)


def _current_stream(torch, device):
    """A function that gives the device index's current stream, without a Stream object around it where torch has one."""
    try:
        return torch._C._cuda_getCurrentRawStream
    except AttributeError:
        return lambda _: torch.cuda.current_stream(device).cuda_stream


def _ptr(t, shape, dtype, cache, what):
    """The address of a contiguous tensor of this shape and type on the cache's
    device: one cheap comparison each, and the named error where one fails."""
    try:
        if t.shape == shape and t.dtype is dtype and t.get_device() == cache._index and t.is_contiguous():
            return t.data_ptr()
    except AttributeError:
        pass
    _dev(_need(t, shape, dtype, what), what)
    _same_device(cache.k, t)
    raise ValueError(f"{what} does not fit")


class KVCache:
    """Keys and values in pages: k and v are [pages, heads, page_size, dim]
    tensors of bfloat16 or float8_e4m3fn (any strides that keep a row of dim
    elements together and 16-byte aligned, the same for both), k_scale and
    v_scale the fp32 [pages, heads, page_size] scales of e4m3 rows, position
    (int32) and weight (fp32) of the same shape what an evicted cache keeps of
    every slot.  The object holds the tensors; it owns no other memory.  Calls
    hand their addresses to the library, which are taken here once: none of them
    can be replaced (with_state() makes a cache with others), what they hold can."""

    __slots__ = ("k", "v", "k_scale", "v_scale", "position", "weight", "pages", "heads", "page_size", "dim", "device",
                 "_c", "_ref", "_index", "_current")

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
        for t, what in ((k, "k"), (v, "v")):
            if not t.is_cuda:
                raise ValueError(f"{what} must be a CUDA (HIP) tensor")
        opt = lambda t, what: None if t is None else _dev(t, what)  # noqa: E731
        c = _lib.sdq_kv_cache(
            k.data_ptr(), v.data_ptr(), opt(k_scale, "k_scale"), opt(v_scale, "v_scale"), opt(position, "position"),
            opt(weight, "weight"), shape[0], *(0 if n == 1 else s for n, s in zip(shape, stride[:3])),
            _lib.DTYPE_E4M3 if e4m3 else _lib.DTYPE_BF16, *shape[1:])
        for name, value in zip(KVCache.__slots__, (k, v, k_scale, v_scale, position, weight, *shape, k.device, c, C.byref(c),
                                                   k.get_device(), _current_stream(torch, k.device))):
            object.__setattr__(self, name, value)

    def __setattr__(self, name, value):
        if name in KVCache.__slots__:
            raise AttributeError(f"{name} of a cache is fixed: its address or size is the library's already; with_state() makes a "
                                 "cache with other positions and weights, KVCache() one with other tensors")
        object.__setattr__(self, name, value)

    def __delattr__(self, name):
        if name in KVCache.__slots__:
            raise AttributeError(f"{name} of a cache is fixed: with_state() or KVCache() makes another cache")
        object.__delattr__(self, name)

    def __reduce__(self):  # a copy takes the addresses of its own tensors
        return type(self), (self.k, self.v, self.k_scale, self.v_scale, self.position, self.weight)

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


def _seqs(cache, page_table, seq_lens, torch):
    """Of the page table: B, its width, its row stride and its address; the address of seq_lens."""
    if not isinstance(page_table, torch.Tensor) or page_table.dtype is not torch.int32 or len(shape := page_table.shape) != 2:
        raise ValueError("page_table must be [sequences, pages] int32")
    B, width = shape
    lens = _ptr(seq_lens, (B,), torch.int32, cache, "seq_lens")
    ld, step = page_table.stride()
    if step != 1 and width > 1:
        raise ValueError("the rows of page_table must be contiguous")
    if page_table.get_device() != cache._index:
        _same_device(cache.k, page_table)
    return B, width, ld if B > 1 else width, page_table.data_ptr(), lens


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
    if not isinstance(qkv, torch.Tensor) or len(shape := qkv.shape) != 2:
        raise ValueError("qkv must be [M, (heads_q + 2 heads) * dim]")
    M, width = shape
    dim = cache.dim
    if heads_q < 1 or width != (heads_q + 2 * cache.heads) * dim:
        raise ValueError(f"qkv must be [M, {(heads_q + 2 * cache.heads) * dim}], got {list(qkv.shape)}")
    ld, step = qkv.stride()
    if step != 1 or not qkv.is_cuda:
        raise ValueError("qkv must be a CUDA (HIP) tensor with contiguous rows")
    if qkv.get_device() != cache._index:
        _same_device(cache.k, qkv)
    dt = _lib.DTYPE_BF16 if qkv.dtype is torch.bfloat16 else _x_dtype(qkv)
    at = _ptr(slot, (M,), torch.int64, cache, "slot")
    where = qw = kw = angles = rot = positions = 0
    if pos is not None:
        where = _ptr(pos, (M,), torch.int32, cache, "pos")
    elif cos_sin is not None or cache.position is not None:
        raise ValueError("pos is needed for the rotation and for a cache that keeps positions")
    if cos_sin is not None:
        if not isinstance(cos_sin, torch.Tensor) or cos_sin.dim() != 2:
            raise ValueError("cos_sin must be [positions, rot_dim] float32")
        positions, rot = cos_sin.shape
        angles = _ptr(cos_sin, (positions, rot), torch.float32, cache, "cos_sin")
    if q_weight is not None and k_weight is not None:
        qw = _ptr(q_weight, (dim,), torch.float32, cache, "q_weight")
        kw = _ptr(k_weight, (dim,), torch.float32, cache, "k_weight")
    elif q_weight is not None or k_weight is not None:
        raise ValueError("q_weight and k_weight go together")
    if out is None:
        out = _empty((M, heads_q, dim), out_dtype or qkv.dtype, qkv.device, stream)
    to = _ptr(out, (M, heads_q, dim), out_dtype or out.dtype, cache, "out")
    rc = (_lib._lib or _lib.lib()).sdq_qkv_append(cache._ref, _APPEND.pack(
        qkv.data_ptr(), where, at, to, qw, kw, angles if rot else 0, M, ld if M > 1 else width, positions, dt,
        dt if out.dtype is qkv.dtype else _x_dtype(out), heads_q, rot, interleaved, eps),
        stream.cuda_stream if stream is not None else cache._current(cache._index))
    if rc:
        _lib.check(rc, "sdq_qkv_append")
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
    lengths (default: what the page table holds).  It should be given where the
    table has room for far longer sequences: it sizes the launches and the
    workspace (with weight_out 4 bytes per query head and slot of max_len) and
    picks the kernels' form.  scale defaults to dim ** -0.5.
    lse (fp32 [B, heads_q]) receives the logarithm of the softmax sums.
    weight_out (cache.weight itself, or a tensor like it) receives cache.weight
    plus each slot's attention weight, summed over the query heads of its key
    head.  workspace: a uint8 tensor of attn_decode_workspace_size bytes, or a
    fresh one is made."""
    torch = _torch()
    B, width, ld, table, lens = _seqs(cache, page_table, seq_lens, torch)
    dim = cache.dim
    if not isinstance(q, torch.Tensor) or len(shape := q.shape) != 3 or shape[0] != B or shape[2] != dim:
        raise ValueError(f"q must be [{B}, heads_q, {dim}]")
    heads_q = shape[1]
    dt = _lib.DTYPE_BF16 if q.dtype is torch.bfloat16 else _x_dtype(q)
    q_ld, head_ld, step = q.stride()
    if not q.is_cuda or step != 1 or (heads_q > 1 and head_ld != dim):
        raise ValueError("q must be a CUDA (HIP) tensor whose sequences are contiguous")
    if q.get_device() != cache._index:
        _same_device(cache.k, q)
    if out is None:
        out = _empty((B, heads_q, dim), q.dtype, q.device, stream)
    to = _ptr(out, shape, q.dtype, cache, "out")
    log = 0 if lse is None else _ptr(lse, (B, heads_q), torch.float32, cache, "lse")
    weights = 0
    if weight_out is not None:
        if cache.weight is None:
            raise ValueError("weight_out needs a cache that keeps weights")
        weights = _ptr(weight_out, cache.weight.shape, torch.float32, cache, "weight_out")
    cap = width * cache.page_size
    if max_len is not None and max_len < cap:
        cap = max_len
    if workspace is None:
        workspace = _workspace(attn_decode_workspace_size(cache, B, heads_q, cap, weights != 0), q.device, stream)
    elif workspace.get_device() != cache._index or not workspace.is_contiguous():
        _dev(workspace, "workspace")
        _same_device(cache.k, workspace)
    rc = (_lib._lib or _lib.lib()).sdq_attn_decode(cache._ref, _ATTN.pack(
        q.data_ptr(), table, lens, to, log, weights, workspace.data_ptr(), workspace.nbytes, B,
        q_ld if B > 1 else heads_q * dim, ld, width, cap, dt, heads_q, dim ** -0.5 if scale is None else scale),
        stream.cuda_stream if stream is not None else cache._current(cache._index))
    if rc:
        if rc == _lib.ERR_BUFFER_TOO_SMALL:
            _need_bytes(workspace, attn_decode_workspace_size(cache, B, heads_q, cap, weights != 0), "workspace")
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
    (which may be seq_lens) or a new tensor.  max_len: as in attn_decode.

    Keys, values and scales move in place.  Positions and weights are updated in
    place too, or written to position_out and weight_out (both, and not the
    cache's own)."""
    torch = _torch()
    B, width, ld, table, lens = _seqs(cache, page_table, seq_lens, torch)
    if cache.position is None or cache.weight is None:
        raise ValueError("eviction needs a cache that keeps positions and weights")
    if (weight_out is None) != (position_out is None):
        raise ValueError("weight_out and position_out go together")
    if weight_out is None:
        weight_out, position_out = cache.weight, cache.position
    shape = cache.weight.shape
    weights = _ptr(weight_out, shape, torch.float32, cache, "weight_out")
    positions = _ptr(position_out, shape, torch.int32, cache, "position_out")
    if lens_out is None:
        lens_out = _empty((B,), seq_lens.dtype, cache.device, stream)
    new = _ptr(lens_out, (B,), torch.int32, cache, "lens_out")
    cap = width * cache.page_size
    if max_len is not None and max_len < cap:
        cap = max_len
    if workspace is None:
        workspace = _workspace(cache_evict_workspace_size(cache, B, cap, budget), cache.device, stream)
    elif workspace.get_device() != cache._index or not workspace.is_contiguous():
        _dev(workspace, "workspace")
        _same_device(cache.k, workspace)
    rc = (_lib._lib or _lib.lib()).sdq_cache_evict(cache._ref, _EVICT.pack(
        table, lens, new, positions, weights, workspace.data_ptr(), workspace.nbytes, B, ld, width, cap, budget, recent),
        stream.cuda_stream if stream is not None else cache._current(cache._index))
    if rc:
        if rc == _lib.ERR_BUFFER_TOO_SMALL:
            _need_bytes(workspace, cache_evict_workspace_size(cache, B, cap, budget), "workspace")
        _lib.check(rc, "sdq_cache_evict")
    return lens_out
