"""What a transformer block computes between its products, and the dense int8
product (sdq_block_norm, sdq_glu_act and sdq_gemm_int8 of include/sdq.h).  As in
the rest of the binding, arguments are checked and marshalled here and all work
is done by the library's kernels.

    r, xq, s = block_norm(r, y, weight, out_dtype="int8", residual_out=r)   # join the stream, norm, codes
    gu = gemm_int8(xq, s, wq, s_w, out_dtype=torch.bfloat16)                # or gemm(xq, s, packed, N, K, cfg)
    hq, s_h = glu_act(gu, "silu", out_dtype="int8")
"""
from __future__ import annotations

import ctypes as C
import functools
import struct

from . import _dev, _empty, _lib, _need, _need_bytes, _torch, _workspace

# The argument structures as bytes, as in kv.py.
_NORM = struct.Struct("@10P6q2d6if0q")
_GLU = struct.Struct("@3P3q4i0q")
_INT8 = struct.Struct("@7PN6qi0q")

# A call's host time is its floor at decode sizes, and most of it is spent on
# asking tensors what they are: each is asked once and in place, and what does not
# fit is named by the functions below, off the straight path.
_OUT = {}   # out_dtype, as a name or a torch dtype: the dtype of the tensor and the library's type for it
_KIND = {}  # torch dtype of activations: the library's type
_f32 = _i8 = _u8 = _stream_of = _device_now = _norm = _glu = _int8 = None
_CODES = _lib.DTYPE_E4M3  # the library's types from here on are codes


def _prepare():
    """What the calls need of torch and the library, looked up once."""
    global _f32, _i8, _u8, _stream_of, _device_now, _norm, _glu, _int8
    torch, lib = _torch(), _lib.lib()
    _norm, _glu, _int8 = lib.sdq_block_norm, lib.sdq_glu_act, lib.sdq_gemm_int8
    _i8, _u8 = torch.int8, torch.uint8
    _KIND.update({torch.float32: _lib.DTYPE_F32, torch.bfloat16: _lib.DTYPE_BF16})
    _OUT.update({"int8": (_u8, _lib.DTYPE_INT8), "e4m3": (_u8, _lib.DTYPE_E4M3)})
    for name, dt in (("f32", torch.float32), ("bf16", torch.bfloat16)):
        _OUT[name] = _OUT[dt] = (dt, _KIND[dt])
    _device_now = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)
    _stream_of = getattr(torch._C, "_cuda_getCurrentRawStream", lambda i: torch.cuda.current_stream(i).cuda_stream)
    _f32 = torch.float32  # last: it says that all of them are there


def _run(fn, packed, index, stream, name):
    """The library's call on the given stream, or the current one of the tensors' device, with that device current."""
    if _device_now() != index:
        with _torch().cuda.device(index):
            rc = fn(packed, _stream_of(index) if stream is None else stream.cuda_stream)
    else:
        rc = fn(packed, _stream_of(index) if stream is None else stream.cuda_stream)
    if rc:
        _lib.check(rc, name)


def _wrong(t, what, M=None, K=None, index=None, kinds="float32 or bfloat16"):
    """Raises what is wrong with a tensor that should have rows [M, K] on a GPU."""
    torch = _torch()
    if not isinstance(t, torch.Tensor) or t.dim() != 2:
        raise ValueError(f"{what} must be a two-dimensional tensor")
    if M is not None and t.shape != (M, K):
        raise ValueError(f"{what} must be [{M}, {K}], got {list(t.shape)}")
    if not t.is_cuda or (t.stride(1) != 1 and t.shape[1] > 1):
        raise ValueError(f"{what} must be a CUDA (HIP) tensor with contiguous rows")
    if index is not None and t.get_device() != index:
        raise ValueError(f"{what} is on another device: {t.device}")
    raise ValueError(f"{what} must be {kinds}, got {t.dtype}")


def _first(t, what):
    """The tensor that the others go by: its shape, row stride, address and device index."""
    try:
        shape = t.shape
        M, K = shape
        ld, step = t.stride()
        index = t.get_device()
    except (AttributeError, ValueError):
        _wrong(t, what)
    if index < 0 or (step != 1 and K > 1):
        _wrong(t, what)
    if _f32 is None:
        _prepare()
    return shape, M, K, ld if M > 1 else K, t.data_ptr(), index


def _like(t, shape, what, index):
    """Row stride and address of a tensor of a shape on a device."""
    try:
        if t.shape == shape and t.get_device() == index:
            ld, step = t.stride()
            if step == 1 or shape[1] == 1:
                return ld if shape[0] > 1 else shape[1], t.data_ptr()
    except AttributeError:
        pass
    _wrong(t, what, *shape, index=index)


def _vec(t, n, what, index):
    """The address of an fp32 vector of n elements."""
    try:
        if t.dtype is _f32 and t.shape == n and t.get_device() == index and t.is_contiguous():
            return t.data_ptr()
    except AttributeError:
        pass
    _dev(_need(t, n, _f32, what), what)
    raise ValueError(f"{what} is on another device: {t.device}")


def _kind(t, what):
    try:
        return _KIND[t.dtype]
    except KeyError:
        raise ValueError(f"{what} must be float32 or bfloat16") from None


def _result(out, scales, out_dtype, shape, rows, like, index, stream):
    """The output of a call: the tensor, the library's type for it, and for codes the scales and their address."""
    if out is not None and not hasattr(out, "get_device"):
        raise ValueError("out must be a torch tensor")
    if out_dtype is None:
        out_dtype = like.dtype if out is None else out.dtype
    try:
        want, code = _OUT[out_dtype]
    except (KeyError, TypeError):
        raise ValueError("out_dtype must be 'int8', 'e4m3', 'bf16', 'f32' or a torch dtype of the last two") from None
    at = 0
    if code >= _CODES:
        if scales is None:
            scales = _empty(rows, _f32, like.device, stream)
        at = _vec(scales, rows, "scales", index)
    elif scales is not None:
        raise ValueError("scales belong to codes")
    if out is None:
        out = _empty(shape, want, like.device, stream)
    elif out.dtype is not want or out.shape != shape or out.get_device() != index or not out.is_contiguous():
        _dev(_need(out, shape, want, "out"), "out")
        raise ValueError(f"out is on another device: {out.device}")
    return out, code, scales, at


def block_norm(residual, y=None, weight=None, bias=None, eps: float = 1e-6, layer: bool = False, post_weight=None,
               post_bias=None, post_eps=None, gate=None, scale: float = 1.0, out_dtype=None, residual_out=None, out=None,
               scales=None, stream=None):
    """The norms around a block and the residual stream between them, in one pass:
    returns (r', n, scales).

        u = y, or norm(y; post_weight, post_bias, post_eps)
        r' = residual + (u * gate) * scale
        n = norm(r'; weight, bias, eps)

    norm is the rms norm, or with layer=True the layer norm, which may have a bias.
    residual and y are [M, K], fp32 or bf16 each (rows may be strided); weights and
    biases fp32 [K]; gate fp32 or bf16, [K] or [1, K], [M, 1], or [M, K].  Without y
    the stream stays as it is and r' is residual; without weight there is no n.
    r' goes to residual_out (residual itself for in place) or a new tensor.
    n has out_dtype: 'bf16', 'f32' (default: residual's type), or 'int8' and 'e4m3'
    for uint8 codes and their scales, the Xq and s_a of the products; scales is
    None otherwise.  post_eps defaults to eps."""
    shape, M, K, ld, at, index = _first(residual, "residual")
    cols, kind = (K,), _kind(residual, "residual")
    y_at = y_ld = y_kind = to = to_ld = 0
    gate_at = gate_ld = gate_kind = per_row = 0
    if y is not None:
        y_ld, y_at = _like(y, shape, "y", index)
        y_kind = _kind(y, "y")
        if residual_out is None:
            residual_out = _empty(shape, residual.dtype, residual.device, stream)
        to_ld, to = _like(residual_out, shape, "residual_out", index)
        if residual_out.dtype is not residual.dtype:
            _wrong(residual_out, "residual_out", kinds=residual.dtype)
        if gate is not None:
            gate_at, gate_ld, gate_kind, per_row = _gate(gate, M, K, index)
    elif gate is not None or post_weight is not None or post_bias is not None or residual_out is not None:
        raise ValueError("gate, post_weight, post_bias and residual_out belong to y")
    if weight is not None:
        out, code, scales, scales_at = _result(out, scales, out_dtype, shape, (M,), residual, index, stream)
        out_at, weight_at = out.data_ptr(), _vec(weight, cols, "weight", index)
    elif y is None or out is not None or bias is not None or scales is not None or out_dtype is not None:
        raise ValueError("out, out_dtype, scales and bias belong to weight, and without y there must be one")
    else:
        code = scales_at = out_at = weight_at = 0
    bias_at = post_at = post_bias_at = 0
    if bias is not None:
        bias_at = _vec(bias, cols, "bias", index)
    if post_weight is not None:
        post_at = _vec(post_weight, cols, "post_weight", index)
        if post_bias is not None:
            post_bias_at = _vec(post_bias, cols, "post_bias", index)
        if post_eps is None:
            post_eps = eps
    elif post_bias is not None:
        raise ValueError("post_bias belongs to post_weight")
    if M:
        _run(_norm, _NORM.pack(at, y_at, gate_at, weight_at, bias_at, post_at, post_bias_at, to, out_at, scales_at, M, K, ld, y_ld,
                               gate_ld, to_ld, eps, post_eps or 0.0, kind, y_kind, gate_kind, code, per_row, layer, scale),
             index, stream, "sdq_block_norm")
    return residual if y is None else residual_out, out, scales


def _gate(gate, M, K, index):
    """Address, row stride, the library's type of a gate, and whether it is one number per row."""
    try:
        shape, stride = gate.shape, gate.stride()
    except AttributeError:
        raise ValueError("gate must be a torch tensor") from None
    kind = _kind(gate, "gate")
    if gate.get_device() != index:
        raise ValueError(f"gate is on another device: {gate.device}")
    ld = per_row = 0
    if shape == (M, K):
        ld = stride[0] if M > 1 else 0
    elif shape == (M, 1):
        ld, per_row = stride[0] if M > 1 else 0, 1
    elif shape != (K,) and shape != (1, K):
        raise ValueError(f"gate must be [{K}], [1, {K}], [{M}, 1] or [{M}, {K}], got {list(shape)}")
    if not per_row and stride[-1] != 1:
        raise ValueError("the rows of gate must be contiguous")
    return gate.data_ptr(), ld, kind, per_row


def glu_act(x, act: str = "silu", gated: bool = True, out_dtype=None, out=None, scales=None, stream=None):
    """The activation of a feed-forward block: act(g) * u for rows [g, u] of x
    (gated), or act(x).  Returns (out, scales).

    x is [M, 2 F] (gated) or [M, F], fp32 or bf16, as a stacked gate/up projection
    writes it (rows may be strided); act 'silu', 'gelu' (the tanh form) or 'relu';
    out_dtype as in block_norm."""
    shape, M, F, ld, at, index = _first(x, "x")
    if gated:
        if F % 2:
            raise ValueError("the rows of x must be two parts of the same width")
        F //= 2
        shape = (M, F)
    code = _lib.ACT.get(act)
    if code is None:
        raise ValueError("act must be 'silu', 'gelu' or 'relu'")
    kind = _kind(x, "x")
    out, to, scales, scales_at = _result(out, scales, out_dtype, shape, (M,), x, index, stream)
    if M:
        _run(_glu, _GLU.pack(at, out.data_ptr(), scales_at, M, F, ld, kind, to, code, gated), index, stream, "sdq_glu_act")
    return out, scales


def _product_type(out_dtype):
    """The torch dtype of a product's output, given as such or by its name."""
    try:
        want, code = _OUT[out_dtype]
    except (KeyError, TypeError):
        code = _CODES
    if code >= _CODES:
        raise ValueError("out_dtype must be float32 or bfloat16, as 'f32', 'bf16' or a torch dtype")
    return want


@functools.lru_cache(maxsize=4096)
def gemm_int8_workspace_size(M: int, N: int, K: int) -> int:
    """Device workspace bytes that gemm_int8 takes for these sizes (0: none)."""
    n = C.c_size_t()
    _lib.check(_lib.lib().sdq_gemm_int8_workspace_size(M, N, K, C.byref(n)), "sdq_gemm_int8_workspace_size")
    return n.value


def gemm_int8(xq, s_x, wq, s_w, bias=None, out=None, out_dtype=None, workspace=None, stream=None):
    """The dense product of int8 codes, Y = s_x * (xq @ wq^T) * s_w + bias: returns Y [M, N].

    xq [M, K] and wq [N, K] are codes as int8, or as the uint8 that quantize_act,
    block_norm and glu_act write (rows may be strided); s_x fp32 [M], s_w fp32 [N],
    bias fp32 [N].  The codes and scales of a weight are quantize_act(W, cfg) with
    int8 activations, once.  out: [M, N], fp32 or bf16, rows may be strided; or
    out_dtype, 'f32' (the default), 'bf16' or a torch dtype.  workspace: a uint8 tensor of gemm_int8_workspace_size
    bytes, or a fresh one is made where that is not 0."""
    _, M, K, x_ld, x_at, index = _first(xq, "xq")
    _, N, depth, w_ld, w_at, where = _first(wq, "wq")
    if depth != K or where != index:
        _wrong(wq, "wq", N, K, index=index)
    dt = xq.dtype
    if dt is not _i8 and dt is not _u8:
        _wrong(xq, "xq", kinds="int8 codes (int8 or uint8)")
    dt = wq.dtype
    if dt is not _i8 and dt is not _u8:
        _wrong(wq, "wq", kinds="int8 codes (int8 or uint8)")
    if out_dtype is not None:
        out_dtype = _product_type(out_dtype)
    if out is None:
        out = _empty((M, N), out_dtype or _f32, xq.device, stream)
    elif out_dtype is not None and getattr(out, "dtype", None) is not out_dtype:
        raise ValueError(f"out must be a tensor of {out_dtype}")
    y_ld, y_at = _like(out, (M, N), "out", index)
    need = gemm_int8_workspace_size(M, N, K)
    ws = ws_bytes = 0
    if need:
        if workspace is None:
            workspace = _workspace(need, xq.device, stream)
        elif _need_bytes(workspace, need, "workspace").get_device() != index:
            raise ValueError(f"workspace is on another device: {workspace.device}")
        ws, ws_bytes = workspace.data_ptr(), workspace.nbytes
    bias_at = 0 if bias is None else _vec(bias, (N,), "bias", index)
    packed = _INT8.pack(x_at, w_at, _vec(s_x, (M,), "s_x", index), _vec(s_w, (N,), "s_w", index), bias_at, y_at, ws, ws_bytes, M, N, K,
                        x_ld, w_ld, y_ld, _kind(out, "out"))
    if M:
        _run(_int8, packed, index, stream, "sdq_gemm_int8")
    return out
