"""Which form a dense int8 product takes (no GPU): the sizes of the tests of the forms stand for the forms that they
name, and all forms are among them."""
import pytest

pytest.importorskip("torch")

import paper_2406_13868_amd as sdq  # noqa: E402
import test_gpu_gemm_int8_forms as forms  # noqa: E402
from paper_2406_13868_amd import _lib  # noqa: E402
from test_gpu_gemm_int8 import DIVIDED  # noqa: E402

TILES = ["64x64 in pairs", "64x128 in pairs", "128x128", "128x128 in pairs", "256x128", "256x192", "256x256", "256x384"]


def form(name):
    return name[: name.index(" (")] if " (" in name else name


def test_divided_products():
    for (M, N, K), (name, parts) in forms.DIVIDED.items():
        assert _lib.int8_kernel_name(M, N, K) == f"{name} ({parts} parts)", (M, N, K)
        assert sdq.gemm_int8_workspace_size(M, N, K) == 4 * M * N * parts
        assert _lib.int8_kernel_name(M, N, K, workspace=False).endswith("(1 part)")
    taken = {form(_lib.int8_kernel_name(*s)) for s in list(forms.DIVIDED) + DIVIDED}
    assert taken == {"tile " + t for t in TILES}
    for t in TILES:  # depths that are whole chunks of 128 bytes, and others
        assert {K % 128 == 0 for (_, _, K), (name, _) in forms.DIVIDED.items() if name == "tile " + t} == {False, True}


def test_undivided_products():
    for (M, N, K), name in forms.UNDIVIDED.items():
        assert _lib.int8_kernel_name(M, N, K) == name + " (1 part)", (M, N, K)
        assert sdq.gemm_int8_workspace_size(M, N, K) == 0
    # with the sizes of the largest tiles' own test and of the smallest products
    others = [(M, N, K) for M, N in ((1025, 18003), (700, 30005), (3900, 4090), (255, 33000), (2040, 4005)) for K in (16, 144, 528)]
    taken = {form(_lib.int8_kernel_name(*s)) for s in list(forms.UNDIVIDED) + others + [(40, 65, 256)]}
    assert taken == {"tile " + t for t in TILES}


def test_few_tokens():
    assert [_lib.int8_kernel_name(M, 4096, 4096) for M in (1, 8, 9, 16, 17, 32)] == ["few 8x16"] * 2 + ["few 16x16"] * 2 + ["few 32x16"] * 2
    assert [_lib.int8_kernel_name(16, N, 4096) for N in (8192, 11001, 16370, 33001)] == ["few 16x32", "few 16x48", "few 16x64", "few 16x48"]
    assert _lib.int8_kernel_name(17, 4097, 4096).startswith("tile") and _lib.int8_kernel_name(33, 4096, 4096).startswith("tile")


def test_names_that_are_refused():
    for size in ((0, 64, 64), (3, 0, 64), (3, 64, 24)):
        with pytest.raises(sdq.SDQError, match="SHAPE"):
            _lib.int8_kernel_name(*size)
