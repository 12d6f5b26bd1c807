"""Pins of the decode-step oracle against closed forms and invariants."""
import math

import numpy as np
import pytest

from oracle import decode as O
from oracle import formats as F


def test_rotation_keeps_lengths_and_turns_by_the_position():
    rng = np.random.default_rng(0)
    x = rng.standard_normal(12)
    for inter in (False, True):
        ang = rng.uniform(-3, 3, 4)
        y, _ = O.transform(x, None, 0, np.concatenate([np.cos(ang), np.sin(ang)]), inter)
        assert np.allclose(np.linalg.norm(y), np.linalg.norm(x)) and np.array_equal(y[8:], x[8:])
        a, b = (0, 1) if inter else (0, 4)
        assert np.isclose(math.atan2(y[b], y[a]) - math.atan2(x[b], x[a]), ang[0]) or np.isclose(
            abs(math.atan2(y[b], y[a]) - math.atan2(x[b], x[a]) - ang[0]), 2 * math.pi)


def test_dot_products_of_rotated_heads_depend_on_the_distance_alone():
    rng = np.random.default_rng(1)
    q, k, f = rng.standard_normal(8), rng.standard_normal(8), rng.uniform(0.1, 1, 4)
    turn = lambda x, p: O.transform(x, None, 0, np.concatenate([np.cos(f * p), np.sin(f * p)]), False)[0]  # noqa: E731
    assert np.isclose(turn(q, 7) @ turn(k, 3), turn(q, 104) @ turn(k, 100))


def test_norm_gives_unit_mean_square():
    x = np.random.default_rng(2).standard_normal(32) * 5
    y, _ = O.transform(x, np.ones(32), 0.0, None, False)
    assert np.isclose(np.mean(y * y), 1)


def test_quantized_rows():
    codes, s = O.quantize_row(np.array([448.0, -1.0, 0.0, 2.0], np.float32))
    assert s == 1 and np.array_equal(F.e4m3_decode(codes), [448, -1, 0, 2])
    codes, s = O.quantize_row(np.zeros(4, np.float32))
    assert s == 0 and not codes.any()


def test_attention_of_equal_keys_is_the_mean_and_of_none_is_zero():
    v = np.random.default_rng(3).standard_normal((5, 4))
    r = O.attend(np.ones((2, 4)), np.ones((5, 4)), v, 0.5)
    assert np.allclose(r["out"], v.mean(0)) and np.allclose(r["lse"], 2 + math.log(5)) and np.allclose(r["p"], 0.2)
    r = O.attend(np.ones((2, 4)), np.ones((0, 4)), np.ones((0, 4)), 0.5)
    assert not r["out"].any() and np.all(r["lse"] == -np.inf)


@pytest.mark.parametrize("recent", [0, 2, 4])
def test_eviction_keeps_the_best_and_moves_the_least(recent):
    rng = np.random.default_rng(recent)
    w, pos = rng.permutation(11).astype(np.float32), rng.permutation(11).astype(np.int32)
    of, to, w2, p2 = O.evict(w, pos, 4, recent)
    kept = set(p2[:4])
    assert len(of) == len(to) and np.all(to < 4) and np.all(of >= 4) and np.all(w2[4:] == 0) and np.all(p2[4:] == -1)
    assert {p for p in pos if p > 10 - recent} <= kept
    others = sorted((float(x) for x, p in zip(w, pos) if p <= 10 - recent), reverse=True)[:4 - recent]
    assert sorted(float(x) for x, p in zip(w, pos) if p in kept and p <= 10 - recent) == sorted(others)
    stay = [t for t in range(4) if t not in to]
    assert np.array_equal(w2[stay], w[stay])


def test_eviction_ties_go_to_the_lowest_slot_and_nan_is_lowest():
    w = np.array([1, np.nan, 1, 1, 0, 1], np.float32)
    of, to, w2, p2 = O.evict(w, np.arange(6, dtype=np.int32), 3, 0)
    assert list(to) == [1] and list(of) == [3] and list(p2) == [0, 3, 2, -1, -1, -1]


def test_eviction_keeps_minus_infinity_before_nan():
    of, to, w2, p2 = O.evict(np.array([np.nan, -np.inf, 1], np.float32), np.arange(3, dtype=np.int32), 2, 0)
    assert list(to) == [0] and list(of) == [2] and list(p2) == [2, 1, -1]
