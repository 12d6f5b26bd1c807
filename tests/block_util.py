"""Shared helpers of the tests of a block's operators: tensors with known host values, and how far a result may be off."""
import numpy as np

from oracle import block as O
from oracle import formats as F


def placed(torch, a, dtype, gap=0):
    """a [M, K] on the GPU in a type, its rows `gap` elements apart with NaN between them; and its values as fp32."""
    t = torch.from_numpy(np.ascontiguousarray(a, np.float32)).to(dtype)
    big = torch.full((a.shape[0], a.shape[1] + gap), float("nan"), dtype=dtype)
    big[:, : a.shape[1]] = t
    return big.cuda()[:, : a.shape[1]], t.float().numpy()


def equal(got, want):
    """The same bits, a NaN for a NaN."""
    return np.array_equal(np.asarray(got), np.asarray(want), equal_nan=np.asarray(want).dtype.kind == "f")


def rounded(torch, a, dtype):
    return torch.from_numpy(np.ascontiguousarray(a, np.float32)).to(dtype).float().numpy()


def codes_near(codes, scales, h64, kind, rel):
    """Codes and scales of rows that are h64 to within rel of each element (and of
    its row's largest): a code is the nearest to a quotient that is off by that,
    by the scale's own and by three roundings of fp32."""
    a = np.abs(h64).max(-1)
    assert (np.abs(scales - a / (127 if kind == "int8" else 448)) <= (rel + 1.1 * O.U) * a / (127 if kind == "int8" else 448)).all()
    with np.errstate(divide="ignore", invalid="ignore"):
        q = np.where(a[:, None] > 0, h64 * ((127 if kind == "int8" else 448) / a[:, None]), 0.0)
    off = np.abs(q) * (2 * rel + 3.1 * O.U)
    if kind == "int8":
        assert (np.abs(codes.view(np.int8).astype(np.float64) - q) <= 0.5 + off).all()
    else:  # half a step: 2^-4 of the value, or of the least normal number below it
        assert (np.abs(F.e4m3_decode(codes) - q) <= np.maximum(np.abs(q), 2.0 ** -6) * 2.0 ** -4 * (1 + 1e-6) + off).all()
