"""Pins of the oracle of a block's operators: closed forms, and its stepwise forms against the definitions in 64 bits."""
import numpy as np
import pytest

from oracle import block as O
from oracle import formats as F


def test_norms_of_rows_that_are_known():
    v = np.array([[3.0, 4.0, 0.0, 0.0]])
    assert np.allclose(O.norm64(v, np.ones(4), None, 0.0, False), v / 2.5, rtol=1e-15)
    assert np.allclose(O.norm64(v + 7, np.ones(4), np.full(4, 0.5), 0.0, True), (v - 1.75) / np.sqrt(np.mean((v - 1.75) ** 2)) + 0.5, rtol=1e-14)
    assert (O.norm64(np.zeros((1, 4)), np.ones(4), None, 1e-6, True) == 0).all()
    assert np.allclose(O.stream64(v, 2 * v, np.array([[1, 0, 1, 1]]), 0.5), [[6, 4, 0, 0]])


@pytest.mark.parametrize("layer", [False, True])
@pytest.mark.parametrize("K", [8, 120, 4096])
def test_steps_stay_near_the_definition(K, layer):
    rng = np.random.default_rng(K + layer)
    r, y = (rng.standard_normal((5, K)).astype(np.float32) for _ in range(2))
    w, pw, b, pb, g = (rng.uniform(0.5, 1.5, K).astype(np.float32) for _ in range(5))
    if not layer:
        b = pb = None
    # u: d, root and two products, one sum with the bias; then gate, scale and the sum: 5, then 3 roundings
    u = np.abs(O.norm64(y, pw, None, 1e-6, layer)) + (0 if pb is None else pb)
    r64, r32 = O.stream64(r, y, g, 0.3, pw, pb, 1e-6, layer), O.stream_steps(r, y, g, 0.3, pw, pb, 1e-6, layer)
    err_r = O.U * (np.abs(r64) + 1.01 * 8 * u * g * 0.3)
    assert (np.abs(r32 - r64) <= err_r).all()
    # n: the same four roundings and the bias's; the stream's errors enter by themselves, by the mean and by the root
    n64, n32 = O.norm64(r64, w, b, 1e-6, layer), O.norm_steps(r32, w, b, 1e-6, layer)
    d = r64 - (r64.mean(-1, keepdims=True) if layer else 0)
    root = 1 / np.sqrt(np.mean(d * d, -1, keepdims=True) + 1e-6)
    moved = err_r + err_r.mean(-1, keepdims=True) + np.abs(d) * root * np.sqrt(np.mean((2 * err_r) ** 2, -1, keepdims=True))
    assert (np.abs(n32 - n64) <= 1.01 * (w * root * (moved + 4 * O.U * np.abs(d)) + O.U * np.abs(n64))).all()


def test_codes_of_rows_that_are_known():
    rows = np.array([[127.0, -63.5, 0.5, 1.5], [0, 0, 0, 0], [1, np.nan, 0, 0], [np.inf, 1, -np.inf, 0], [1e-40, -1e-40, 0, 5e-41]], np.float32)
    q, s = O.codes_steps(rows, "int8")
    assert (q.view(np.int8)[0] == [127, -64, 0, 2]).all() and s[0] == 1
    assert (q[1:4] == 0).all() and s[1] == 0 and np.isnan(s[2]) and np.isinf(s[3])
    assert (q.view(np.int8)[4] == [127, -127, 0, 64]).all() and s[4] > 0
    q, s = O.codes_steps(rows, "e4m3")
    assert (F.e4m3_decode(q[0]) == [448, -224, 1.75, 5.5]).all() and s[0] == np.float32(127) / np.float32(448)


def test_activations_of_numbers_that_are_known():
    x = np.array([[0.0, 1.0, -1.0, 40.0, -40.0, -800.0]])
    e = 1 / (1 + np.exp(-1.0))
    assert np.allclose(O.activation64(x, "silu", False), [[0, e, e - 1, 40, -40 * np.exp(-40.0), 0]], rtol=1e-14, atol=0)
    assert np.allclose(O.activation64(x, "relu", False), [[0, 1, 0, 40, 0, 0]])
    gelu = O.activation64(x, "gelu", False)
    assert abs(gelu[0, 1] - 0.8411919906082768) < 1e-15 and abs(gelu[0, 1] - gelu[0, 2] * -1 - (1 - 2 * 0.15880800939172324)) < 1e-15
    g = np.linspace(-2, 9, 50)[None]
    assert np.allclose(O.activation64(g, "gelu", False), 0.5 * g * (1 + np.tanh(np.sqrt(2 / np.pi) * (g + 0.044715 * g ** 3))), rtol=1e-13)
    assert np.allclose(O.activation64(np.array([[1.0, 3.0]]), "silu", True), [[3 * e]])


def test_products_are_sums_of_codes():
    rng = np.random.default_rng(3)
    x, w = rng.integers(-128, 128, (3, 16)), rng.integers(-128, 128, (2, 16))
    sx, sw, b = rng.random(3), rng.random(2), rng.random(2)
    y, total = O.product64(x, sx, w, sw, b)
    for m in range(3):
        for n in range(2):
            t = sum(int(x[m, k]) * int(w[n, k]) for k in range(16))
            assert total[m, n] == t and np.isclose(y[m, n], t * sx[m] * sw[n] + b[n], rtol=1e-15)
