"""A rotation without a table of angles is refused before any launch (no GPU)."""
import ctypes as C

import pytest

from paper_2406_13868_amd import _lib

P, SHAPE = 1 << 20, -2  # P stands for a device pointer in calls that are refused before it is used


def _append(**kw):
    cache = _lib.sdq_kv_cache(k=P, v=P, pages=10, page_stride=8 * 16 * 64, head_stride=16 * 64, slot_stride=64, dtype=_lib.DTYPE_BF16,
                              heads=8, page_size=16, dim=64)
    f = dict(qkv=P, pos=P, slot=P, q_out=P, cos_sin=P, M=1, row_stride=24 * 64, positions=0, x_dtype=0, q_dtype=0, heads_q=8, rot_dim=64,
             interleaved=0, eps=1e-6)
    return _lib.lib().sdq_qkv_append(C.byref(cache), C.byref(_lib.sdq_append_args(**(f | kw))), None)


@pytest.mark.parametrize("rot", [2, 20, 64])
def test_no_positions(rot):
    assert _append(rot_dim=rot) == SHAPE


def test_no_tokens_need_no_angles():
    assert _append(M=0) == 0 and _append(M=0, cos_sin=None, positions=0) == 0
