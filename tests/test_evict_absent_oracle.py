"""The oracle's eviction where some pages are absent: what stays, where it goes."""
import numpy as np
import pytest

from oracle import decode as O


@pytest.mark.parametrize("recent", [0, 2, 5])
@pytest.mark.parametrize("seed", range(6))
def test_present_slots_fill_the_present_places(seed, recent):
    rng = np.random.default_rng(seed)
    n, budget = 17, 6
    w, pos = rng.permutation(n).astype(np.float32), rng.permutation(n).astype(np.int32)
    there = rng.random(n) < 0.6
    of, to, w2, p2 = O.evict(w, pos, budget, recent, there)
    places = there[:budget].sum()
    newest = max([-1] + list(pos[there]))
    assert len(of) == len(to) and there[of].all() and there[to].all() and np.all(to < budget) and np.all(of >= budget)
    kept = set(p2[:budget][there[:budget]])
    assert len(kept) == places
    class_of = lambda t: (not pos[t] > newest - recent, -w[t])  # noqa: E731
    best = sorted(np.flatnonzero(there), key=class_of)[:places]
    assert kept == {pos[t] for t in best}
    # absent slots are left alone, present ones past the budget are given up
    assert np.array_equal(w2[~there], w[~there]) and np.array_equal(p2[~there], pos[~there])
    assert not w2[budget:][there[budget:]].any() and np.all(p2[budget:][there[budget:]] == -1)


def test_all_present_is_the_plain_rule_and_none_is_nothing():
    rng = np.random.default_rng(9)
    w, pos = rng.permutation(12).astype(np.float32), rng.permutation(12).astype(np.int32)
    for a, b in zip(O.evict(w, pos, 5, 2), O.evict(w, pos, 5, 2, np.ones(12, bool))):
        assert np.array_equal(a, b)
    of, to, w2, p2 = O.evict(w, pos, 5, 2, np.zeros(12, bool))
    assert not len(of) and not len(to) and np.array_equal(w2, w) and np.array_equal(p2, pos)
