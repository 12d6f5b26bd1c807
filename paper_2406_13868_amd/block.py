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

from . import _dev, _empty, _lib, _need, _need_bytes, _stream, _torch, _workspace

# The argument structures as bytes, as in kv.py.
_NORM = struct.Struct("@10P6q2d6if0q")
_GLU = struct.Struct("@3P3q4i0q")
_INT8 = struct.Struct("@7PN6qi0q")
_CODES = {"int8": _lib.DTYPE_INT8, "e4m3": _lib.DTYPE_E4M3}


def _run(name, M, packed, index, stream):
    """The library's call on the given stream, or the current one of the tensors' device, with that device current."""
    torch = _torch()
    if M == 0:
        return
    fn = getattr(_lib._lib or _lib.lib(), name)
    if torch._C._cuda_getDevice() != index:
        with torch.cuda.device(index):
            rc = fn(packed, _stream(stream))
    else:
        rc = fn(packed, _stream(stream))
    if rc:
        _lib.check(rc, name)


def _rows(t, what, M=None, K=None, index=None):
    """A [M, K] GPU tensor whose rows are contiguous: its type, row stride and address."""
    torch = _torch()
    if not isinstance(t, torch.Tensor) or len(shape := t.shape) != 2:
        raise ValueError(f"{what} must be a two-dimensional tensor")
    if M is not None and (shape[0] != M or shape[1] != K):
        raise ValueError(f"{what} must be [{M}, {K}], got {list(shape)}")
    ld, step = t.stride()
    if not t.is_cuda or (step != 1 and shape[1] > 1):
        raise ValueError(f"{what} must be a CUDA (HIP) tensor with contiguous rows")
    if index is not None and t.get_device() != index:
        raise ValueError(f"{what} is on another device: {t.device}")
    return ld if shape[0] > 1 else shape[1], t.data_ptr()


def _type(t, what):
    torch = _torch()
    dt = t.dtype
    if dt is torch.bfloat16:
        return _lib.DTYPE_BF16
    if dt is torch.float32:
        return _lib.DTYPE_F32
    raise ValueError(f"{what} must be float32 or bfloat16")


def _vec(t, n, what, index):
    """The address of an fp32 vector of n elements; 0 for None."""
    if t is None:
        return 0
    torch = _torch()
    try:
        if t.shape == (n,) and t.dtype is torch.float32 and t.get_device() == index and t.is_contiguous():
            return t.data_ptr()
    except AttributeError:
        pass
    _dev(_need(t, (n,), torch.float32, what), what)
    raise ValueError(f"{what} is on another device: {t.device}")


def _result(out, scales, out_dtype, M, K, default, device, index, stream):
    """The output of a call: the tensor and its type, and for codes the scales and their address."""
    torch = _torch()
    if out_dtype is None:
        out_dtype = default if out is None or out.dtype is torch.uint8 else out.dtype
    code = _CODES.get(out_dtype) if isinstance(out_dtype, str) else None
    if code is None:
        if isinstance(out_dtype, str):
            out_dtype = {"f32": torch.float32, "bf16": torch.bfloat16}.get(out_dtype)
        if out_dtype is not torch.float32 and out_dtype is not torch.bfloat16:
            raise ValueError("out_dtype must be 'int8', 'e4m3', 'bf16', 'f32' or a torch dtype of the last two")
        if scales is not None:
            raise ValueError("scales belong to codes")
        want, code = out_dtype, _lib.DTYPE_F32 if out_dtype is torch.float32 else _lib.DTYPE_BF16
    else:
        want = torch.uint8
        if scales is None:
            scales = _empty((M,), torch.float32, device, stream)
    if out is None:
        out = _empty((M, K), want, device, stream)
    elif out.shape != (M, K) or out.dtype is not want or out.get_device() != index or not out.is_contiguous():
        _dev(_need(out, (M, K), want, "out"), "out")
        raise ValueError(f"out is on another device: {out.device}")
    return out, code, scales, _vec(scales, M, "scales", index)


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
    torch = _torch()
    ld, at = _rows(residual, "residual")
    M, K = residual.shape
    index, device = residual.get_device(), residual.device
    kind = _type(residual, "residual")
    y_at = y_ld = y_kind = to = to_ld = 0
    gate_at = gate_ld = gate_kind = per_row = 0
    if y is not None:
        y_ld, y_at = _rows(y, "y", M, K, index)
        y_kind = _type(y, "y")
        if residual_out is None:
            residual_out = _empty((M, K), residual.dtype, device, stream)
            to_ld, to = K, residual_out.data_ptr()
        else:
            to_ld, to = _rows(residual_out, "residual_out", M, K, index)
            if residual_out.dtype is not residual.dtype:
                raise ValueError(f"residual_out must be {residual.dtype}")
        if gate is not None:
            gate_kind, shape = _type(gate, "gate"), gate.shape
            if gate.get_device() != index:
                raise ValueError(f"gate is on another device: {gate.device}")
            gate_at = gate.data_ptr()
            if shape == (K,) or shape == (1, K):
                ok = gate.stride(-1) == 1
            elif shape == (M, K):
                gate_ld, step = gate.stride()
                ok, gate_ld = step == 1, gate_ld if M > 1 else 0
            elif shape == (M, 1):
                gate_ld, per_row, ok = gate.stride(0) if M > 1 else 0, 1, True
            else:
                raise ValueError(f"gate must be [{K}], [1, {K}], [{M}, 1] or [{M}, {K}], got {list(shape)}")
            if not ok:
                raise ValueError("the rows of gate must be contiguous")
    elif gate is not None or post_weight is not None or post_bias is not None or residual_out is not None:
        raise ValueError("gate, post_weight, post_bias and residual_out belong to y")
    if weight is not None:
        out, code, scales, scales_at = _result(out, scales, out_dtype, M, K, residual.dtype, device, index, stream)
        out_at = out.data_ptr()
    elif y is None or out is not None or bias is not None or scales is not None or out_dtype is not None:
        raise ValueError("out, out_dtype, scales and bias belong to weight, and without y there must be one")
    else:
        code = scales_at = out_at = 0
    _run("sdq_block_norm", M, _NORM.pack(
        at, y_at, gate_at, _vec(weight, K, "weight", index), _vec(bias, K, "bias", index),
        _vec(post_weight, K, "post_weight", index), _vec(post_bias, K, "post_bias", index), to, out_at, scales_at, M, K, ld, y_ld,
        gate_ld, to_ld, eps, eps if post_eps is None else post_eps, kind, y_kind, gate_kind, code, per_row, layer, scale),
        index, stream)
    return residual if y is None else residual_out, out, scales


def glu_act(x, act: str = "silu", gated: bool = True, out_dtype=None, out=None, scales=None, stream=None):
    """The activation of a feed-forward block: act(g) * u for rows [g, u] of x
    (gated), or act(x).  Returns (out, scales).

    x is [M, 2 F] (gated) or [M, F], fp32 or bf16, as a stacked gate/up projection
    writes it (rows may be strided); act 'silu', 'gelu' (the tanh form) or 'relu';
    out_dtype as in block_norm."""
    ld, at = _rows(x, "x")
    M, F = x.shape
    if gated:
        if F % 2:
            raise ValueError("the rows of x must be two parts of the same width")
        F //= 2
    code = _lib.ACT.get(act)
    if code is None:
        raise ValueError("act must be 'silu', 'gelu' or 'relu'")
    index = x.get_device()
    kind = _type(x, "x")
    out, to, scales, scales_at = _result(out, scales, out_dtype, M, F, x.dtype, x.device, index, stream)
    _run("sdq_glu_act", M, _GLU.pack(at, out.data_ptr(), scales_at, M, F, ld, kind, to, code, gated), index, stream)
    return out, scales


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
    out_dtype (default fp32).  workspace: a uint8 tensor of gemm_int8_workspace_size
    bytes, or a fresh one is made where that is not 0."""
    torch = _torch()
    x_ld, x_at = _rows(xq, "xq")
    M, K = xq.shape
    index = xq.get_device()
    w_ld, w_at = _rows(wq, "wq", index=index)
    N = wq.shape[0]
    for t, what in ((xq, "xq"), (wq, "wq")):
        if t.dtype is not torch.int8 and t.dtype is not torch.uint8:
            raise ValueError(f"{what} must be int8 codes (int8 or uint8)")
    if wq.shape[1] != K:
        raise ValueError(f"wq must be [N, {K}], got {list(wq.shape)}")
    if out is None:
        out = _empty((M, N), torch.float32 if out_dtype is None else out_dtype, xq.device, stream)
    elif out_dtype is not None and out.dtype is not out_dtype:
        raise ValueError(f"out must be {out_dtype}")
    y_ld, y_at = _rows(out, "out", M, N, index)
    need = gemm_int8_workspace_size(M, N, K)
    ws = ws_bytes = 0
    if need:
        if workspace is None:
            workspace = _workspace(need, xq.device, stream)
        elif _need_bytes(workspace, need, "workspace").get_device() != index:
            raise ValueError(f"workspace is on another device: {workspace.device}")
        ws, ws_bytes = workspace.data_ptr(), workspace.nbytes
    _run("sdq_gemm_int8", M, _INT8.pack(
        x_at, w_at, _vec(s_x, M, "s_x", index), _vec(s_w, N, "s_w", index), _vec(bias, N, "bias", index), y_at, ws, ws_bytes, M, N, K, x_ld, w_ld,
        y_ld, _type(out, "out")), index, stream)
    return out
