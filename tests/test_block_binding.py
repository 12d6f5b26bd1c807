"""Refusals of the operators between a block's products (no GPU): the C ABI's own
before any launch, and the binding's before a pointer is taken."""
import ctypes as C

import pytest

torch = pytest.importorskip("torch")

import paper_2406_13868_amd as sdq  # noqa: E402
from paper_2406_13868_amd import _lib, block  # noqa: E402

P = 1 << 20  # stands for a device pointer in calls that are refused before it is used
OK, NULL, SHAPE, CONFIG, SMALL, VALUE = 0, -1, -2, -3, -4, -7
NAN, INF = float("nan"), float("inf")


def _norm(**kw):
    f = dict(residual=P, y=2 * P, gate=None, weight=P, bias=None, post_weight=None, post_bias=None, residual_out=3 * P, out=P, scales=P, M=3,
             K=64, residual_stride=64, y_stride=64, gate_stride=0, residual_out_stride=64, eps=1e-6, post_eps=1e-6, residual_dtype=0,
             y_dtype=1, gate_dtype=0, out_dtype=3, gate_per_row=0, layer=0, scale=1.0)
    return _lib.lib().sdq_block_norm(C.byref(_lib.sdq_norm_args(**(f | kw))), None)


def _glu(**kw):
    f = dict(x=P, out=P, scales=P, M=3, F=64, x_stride=128, x_dtype=1, out_dtype=3, act=0, gated=1)
    return _lib.lib().sdq_glu_act(C.byref(_lib.sdq_glu_args(**(f | kw))), None)


def _gemm(**kw):
    f = dict(xq=P, wq=P, s_x=P, s_w=P, bias=None, y=P, M=3, N=5, K=64, x_stride=64, w_stride=64, y_stride=5, y_dtype=0)
    return _lib.lib().sdq_gemm_int8(C.byref(_lib.sdq_int8_args(**(f | kw))), None)


def test_the_packed_structures_are_those_of_the_interface():
    assert block._NORM.size == C.sizeof(_lib.sdq_norm_args)
    assert block._GLU.size == C.sizeof(_lib.sdq_glu_args)
    assert block._INT8.size == C.sizeof(_lib.sdq_int8_args)


def test_null_arguments():
    L = _lib.lib()
    assert L.sdq_block_norm(None, None) == L.sdq_glu_act(None, None) == L.sdq_gemm_int8(None, None) == NULL


@pytest.mark.parametrize("kw, status", [
    (dict(residual_dtype=2), CONFIG), (dict(y_dtype=3), CONFIG), (dict(gate=P, gate_dtype=2), CONFIG), (dict(out_dtype=4), CONFIG),
    (dict(layer=2), CONFIG), (dict(gate=P, gate_per_row=2), CONFIG), (dict(bias=P), CONFIG), (dict(post_weight=P, post_bias=P), CONFIG),
    (dict(post_bias=P, layer=1), CONFIG), (dict(y=None), CONFIG), (dict(y=None, residual_out=None, gate=P), CONFIG),
    (dict(y=None, residual_out=None, post_weight=P), CONFIG), (dict(weight=None), CONFIG), (dict(weight=None, out=None, bias=P, layer=1), CONFIG),
    (dict(y=None, residual_out=None, weight=None, out=None), NULL),
    (dict(eps=-1.0), VALUE), (dict(eps=NAN), VALUE), (dict(eps=INF), VALUE), (dict(post_weight=P, post_eps=NAN), VALUE), (dict(scale=INF), VALUE),
    (dict(M=-1), SHAPE), (dict(M=1 << 22), SHAPE), (dict(K=0), SHAPE), (dict(K=60), SHAPE), (dict(K=(1 << 22) + 8), SHAPE),
    (dict(residual=None), NULL), (dict(residual_out=None), NULL), (dict(out=None), NULL), (dict(scales=None), NULL),
    (dict(residual=P + 8), SHAPE), (dict(y=P + 8), SHAPE), (dict(residual_out=P + 8), SHAPE), (dict(out=P + 8), SHAPE), (dict(weight=P + 4), SHAPE),
    (dict(layer=1, bias=P + 4), SHAPE), (dict(post_weight=P + 4), SHAPE), (dict(layer=1, post_weight=P, post_bias=P + 4), SHAPE),
    (dict(residual_stride=56), SHAPE), (dict(residual_stride=66), SHAPE), (dict(y_stride=68), SHAPE), (dict(residual_out_stride=60), SHAPE),
    (dict(residual_out=P, residual_out_stride=128), SHAPE), (dict(gate=P + 4), SHAPE), (dict(gate=P, gate_stride=32), SHAPE),
    (dict(gate=P, gate_stride=66), SHAPE), (dict(gate=P, gate_stride=-64), SHAPE), (dict(gate=P, gate_per_row=1, gate_stride=-1), SHAPE),
    (dict(M=0, residual=None, out=None), OK),
])
def test_norm(kw, status):
    assert _norm(**kw) == status


@pytest.mark.parametrize("kw, status", [
    (dict(x_dtype=2), CONFIG), (dict(out_dtype=4), CONFIG), (dict(act=3), CONFIG), (dict(act=-1), CONFIG), (dict(gated=2), CONFIG),
    (dict(M=-1), SHAPE), (dict(M=1 << 22), SHAPE), (dict(F=0), SHAPE), (dict(F=60), SHAPE), (dict(F=1 << 23), SHAPE),
    (dict(M=1 << 20, F=1 << 15), SHAPE), (dict(x=None), NULL), (dict(out=None), NULL), (dict(scales=None), NULL), (dict(x=P + 8), SHAPE),
    (dict(out=P + 8), SHAPE), (dict(x_stride=120), SHAPE), (dict(x_stride=132), SHAPE), (dict(gated=0, x_stride=56), SHAPE),
    (dict(M=0, x=None, out=None), OK),
])
def test_glu(kw, status):
    assert _glu(**kw) == status


@pytest.mark.parametrize("kw, status", [
    (dict(y_dtype=2), CONFIG), (dict(M=-1), SHAPE), (dict(M=(1 << 24) + 1), SHAPE), (dict(N=0), SHAPE), (dict(N=(1 << 21) + 1), SHAPE),
    (dict(K=0), SHAPE), (dict(K=24), SHAPE), (dict(K=1 << 17), SHAPE), (dict(M=1 << 20, N=1 << 15), SHAPE), (dict(xq=None), NULL),
    (dict(wq=None), NULL), (dict(s_x=None), NULL), (dict(s_w=None), NULL), (dict(y=None), NULL), (dict(xq=P + 8), SHAPE), (dict(wq=P + 8), SHAPE),
    (dict(x_stride=48), SHAPE), (dict(x_stride=72), SHAPE), (dict(w_stride=72), SHAPE), (dict(w_stride=(1 << 22) + 16), SHAPE),
    (dict(y_stride=4), SHAPE), (dict(y_stride=(1 << 21) + 1), SHAPE), (dict(y=P + 2), SHAPE), (dict(y=P + 1, y_dtype=1), SHAPE),
    (dict(M=0, xq=None, y=None), OK),
])
def test_gemm(kw, status):
    assert _gemm(**kw) == status


def test_workspaces_of_products():
    n = C.c_size_t()
    size = _lib.lib().sdq_gemm_int8_workspace_size
    assert size(64, 4096, 16384, C.byref(n)) == OK and n.value % (64 * 4096 * 4) == 0 and n.value > 64 * 4096 * 4
    need = n.value
    big = dict(M=64, N=4096, K=16384, x_stride=16384, w_stride=16384, y_stride=4096)
    assert _gemm(workspace=P, ws_bytes=need - 1, **big) == SMALL
    assert _gemm(workspace=P + 4, ws_bytes=need, **big) == SHAPE
    assert size(64, 4096, 16384, None) == NULL and size(64, 0, 16, C.byref(n)) == SHAPE and size(64, 5, 24, C.byref(n)) == SHAPE
    for M in (0, 1, 16, 4096):
        assert size(M, 4096, 4096, C.byref(n)) == OK and n.value == 0
    assert sdq.gemm_int8_workspace_size(64, 4096, 16384) == need


def _raises(fn, match):
    with pytest.raises(ValueError, match=match):
        fn()


def test_the_binding_checks_the_calls():
    r, w = torch.zeros((3, 64)), torch.ones(64)
    _raises(lambda: sdq.block_norm(r[0], r, w), "residual must be")
    _raises(lambda: sdq.block_norm(r, r, w), "CUDA")
    _raises(lambda: sdq.block_norm(None, r, w), "residual must be")
    _raises(lambda: sdq.glu_act(r[0]), "x must be")
    _raises(lambda: sdq.glu_act(r), "CUDA")
    q = torch.zeros((3, 64), dtype=torch.int8)
    _raises(lambda: sdq.gemm_int8(q[0], r[:, 0], q, r[:, 0]), "xq must be")
    _raises(lambda: sdq.gemm_int8(q, r[:, 0], q, r[:, 0]), "CUDA")


def test_the_shapes_that_a_gate_may_have():
    """The address, row stride, type and kind of each form; tensors here lie on no GPU, whose index is -1."""
    block._prepare()
    K = 16
    for M in (0, 1, 3):
        for t, ld, per_row in ((torch.zeros(K), 0, 0), (torch.zeros(1, K), 0, 0), (torch.zeros(M, K), K if M > 1 else 0, 0),
                               (torch.zeros(M, 1), 1 if M > 1 else 0, 1), (torch.zeros(M, K + 8)[:, :K], K + 8 if M > 1 else 0, 0),
                               (torch.zeros(1, K).expand(M, K), 0, 0)):
            assert block._gate(t, M, K, -1) == (t.data_ptr(), ld, _lib.DTYPE_F32, per_row)
    for t in (torch.zeros(3, K + 8), torch.zeros(2, K), torch.zeros(2, 1), torch.zeros(8)):
        _raises(lambda: block._gate(t, 3, K, -1), "gate must be")
    _raises(lambda: block._gate(torch.zeros(3, 2 * K)[:, ::2], 3, K, -1), "contiguous")
    _raises(lambda: block._gate([1.0], 3, K, -1), "torch tensor")
    _raises(lambda: block._gate(torch.zeros(K), 3, K, 0), "another device")


def test_outputs_that_are_no_tensors():
    block._prepare()
    like = torch.zeros(3, 16)
    for out_dtype in (None, "int8", "bf16"):
        scales = torch.zeros(3) if out_dtype == "int8" else None
        _raises(lambda: block._result([1.0], scales, out_dtype, (3, 16), (3,), like, -1, None), "out must be a torch tensor")


def test_the_types_of_a_products_output():
    block._prepare()
    for dt in (torch.float32, torch.bfloat16):
        assert block._product_type(dt) is dt
    assert block._product_type("f32") is torch.float32 and block._product_type("bf16") is torch.bfloat16
    for out_dtype in ("int8", "e4m3", "f16", torch.float16, 3, [torch.float32]):
        _raises(lambda: block._product_type(out_dtype), "float32 or bfloat16")
