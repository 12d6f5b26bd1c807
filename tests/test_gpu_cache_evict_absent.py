"""GPU: eviction of sequences some of whose pages are absent, against the oracle:
kept slots only move to places that exist, and nothing is lost to one that does not."""
import numpy as np
import pytest

from gpu_util import say, torch_cuda
from kv_util import Pool
from oracle import decode as O

pytestmark = pytest.mark.gpu

CASES = [
    # lens, heads, D, page_size, kv, budget, recent, weights, share of pages that are absent
    ([12], 1, 16, 4, "bf16", 6, 1, "spread", 0.4),
    ([64, 65, 200, 0], 2, 64, 16, "bf16", 64, 10, "spread", 0.3),
    ([200, 333], 2, 32, 16, "e4m3", 100, 100, "odd", 0.5),
    ([900, 1000], 3, 96, 24, "e4m3", 700, 60, "few", 0.2),
    ([3000, 2047], 2, 32, 64, "bf16", 1500, 100, "odd", 0.3),
    ([7000], 2, 16, 33, "bf16", 500, 20, "spread", 0.6),
    ([15000, 9000], 1, 16, 256, "e4m3", 8000, 50, "few", 0.3),
    ([20000], 2, 16, 128, "bf16", 15000, 4000, "odd", 0.25),
    ([33000], 1, 16, 128, "bf16", 20000, 7, "odd", 0.25),
    ([300] * 4, 32, 16, 16, "bf16", 150, 7, "spread", 0.3),  # 128 rows
]


def _weights(rng, kind, shape):
    if kind == "few":
        return rng.choice(np.array([0.0, -0.0, 0.5, 2.0], np.float32), shape)
    w = np.exp(3 * rng.standard_normal(shape)).astype(np.float32)
    if kind == "odd":  # NaN and the lowest values among them: an absent slot comes after these
        w[rng.random(shape) < 0.5] = np.nan
        w[rng.random(shape) < 0.2] = -np.inf
        w[rng.random(shape) < 0.2] *= -1
    return w


@pytest.mark.parametrize("form", ["in place", "in place, lengths too", "apart"])
@pytest.mark.parametrize("case", CASES, ids=lambda c: "-".join(str(x) if not isinstance(x, list) else f"B{len(x)}x{max(x)}" for x in c))
def test_absent_pages(case, form):
    torch = torch_cuda()
    import paper_2406_13868_amd as sdq

    lens, heads, D, ps, kvt, budget, recent, kind, share = case
    say("evict, absent pages", case, form)
    rng = np.random.default_rng(budget + D)
    pool = Pool(torch, sdq, rng, lens, heads, ps, D, kvt, track=True, poison=False)
    pool.weight = _weights(rng, kind, pool.weight.shape)
    for b, n in enumerate(lens):
        t = np.arange(n)
        for h in range(heads):
            pool.position[pool.table[b][t // ps], h, t % ps] = rng.permutation(n)
    cache = pool.cache
    cache.weight.copy_(torch.from_numpy(pool.weight))
    cache.position.copy_(torch.from_numpy(pool.position))
    table = pool.table.copy()
    gone = rng.random(table.shape) < share
    gone[0, 0] = True  # a place below the budget
    table[gone] = np.where(rng.random(table.shape) < 0.5, -1, pool.pages + 5)[gone]
    raw = lambda t: t.contiguous().view(torch.uint8 if pool.e4m3 else torch.int16).cpu().numpy().copy()  # noqa: E731
    kv = [raw(cache.k), raw(cache.v)] + ([] if pool.ks is None else [pool.ks.numpy().copy(), pool.vs.numpy().copy()])
    want_w, want_p = pool.weight.copy(), pool.position.copy()
    table_gpu = torch.from_numpy(table).cuda()
    if form == "apart":
        want_w, want_p = np.full_like(want_w, 7), np.full_like(want_p, 7)
        w_out, p_out = torch.full_like(cache.weight, 7), torch.full_like(cache.position, 7)
        got = sdq.cache_evict(cache, table_gpu, pool.lens_gpu, budget, recent, weight_out=w_out, position_out=p_out)
    else:
        w_out, p_out = cache.weight, cache.position
        got = sdq.cache_evict(cache, table_gpu, pool.lens_gpu, budget, recent, lens_out=pool.lens_gpu if "lengths" in form else None)
    torch.cuda.synchronize()
    assert got.tolist() == [min(n, budget) for n in lens]
    for b, n in enumerate(lens):
        t = np.arange(n)
        there = ~gone[b][t // ps]
        for h in range(heads):
            at = lambda t: (pool.table[b][t // ps], h, t % ps)  # noqa: E731
            of, to, w, p = O.evict(pool.weight[at(t)], pool.position[at(t)], budget, recent, there)
            seen = t[there]
            want_w[at(seen)], want_p[at(seen)] = w[there], p[there]
            for x in kv:
                x[at(to)] = x[at(of)]
    assert np.array_equal(p_out.cpu().numpy(), want_p)
    assert np.array_equal(w_out.cpu().numpy().view(np.int32), want_w.view(np.int32))
    for got, want in zip((cache.k, cache.v), kv):
        assert np.array_equal(raw(got), want)
    for got, want in zip((cache.k_scale, cache.v_scale), kv[2:]):
        assert np.array_equal(got.cpu().numpy(), want)
