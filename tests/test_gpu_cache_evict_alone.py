"""GPU: eviction in place with new lengths of their own (the call of the README),
at sizes whose moves the selecting workgroups do themselves."""
import numpy as np
import pytest

from gpu_util import say, torch_cuda
from kv_util import Pool
from oracle import decode as O

pytestmark = pytest.mark.gpu

CASES = [
    # lens, heads, D, page_size, kv, budget, recent
    ([3000, 2900, 2801, 10], 4, 64, 16, "bf16", 2800, 100),
    ([9000], 2, 32, 33, "e4m3", 8800, 0),
    ([16385, 16384], 1, 16, 128, "bf16", 16200, 60),
    ([33000], 2, 16, 128, "e4m3", 32800, 500),
    ([300, 800], 64, 16, 16, "bf16", 290, 20),   # 128 rows of up to 510 moves
    ([90] * 31 + [700], 32, 16, 32, "e4m3", 60, 9),  # 1024 rows
    ([2000, 1700] * 12, 8, 16, 64, "bf16", 900, 30),  # 192 rows, of up to 900 moves
    ([1500] + [70] * 7, 128, 16, 48, "bf16", 700, 9),  # 1024 rows, of up to 700 moves
]


@pytest.mark.parametrize("case", CASES, ids=lambda c: "-".join(str(x) if not isinstance(x, list) else f"B{len(x)}x{max(x)}" for x in c))
def test_in_place(case):
    torch = torch_cuda()
    import paper_2406_13868_amd as sdq

    lens, heads, D, ps, kvt, budget, recent = case
    say("evict in place", case)
    rng = np.random.default_rng(budget)
    pool = Pool(torch, sdq, rng, lens, heads, ps, D, kvt, track=True, poison=False)
    for b, n in enumerate(lens):
        t = np.arange(n)
        for h in range(heads):
            pool.position[pool.table[b][t // ps], h, t % ps] = rng.permutation(n)
    cache = pool.cache
    cache.position.copy_(torch.from_numpy(pool.position))
    raw = lambda t: t.contiguous().view(torch.uint8 if pool.e4m3 else torch.int16).cpu().numpy().copy()  # noqa: E731
    kv = [raw(cache.k), raw(cache.v)] + ([] if pool.ks is None else [pool.ks.numpy().copy(), pool.vs.numpy().copy()])
    want_w, want_p = pool.weight.copy(), pool.position.copy()
    new = sdq.cache_evict(cache, pool.table_gpu, pool.lens_gpu, budget, recent)
    torch.cuda.synchronize()
    assert new.tolist() == [min(n, budget) for n in lens] and pool.lens_gpu.tolist() == lens
    for b, n in enumerate(lens):
        t = np.arange(n)
        for h in range(heads):
            at = lambda t: (pool.table[b][t // ps], h, t % ps)  # noqa: E731
            of, to, want_w[at(t)], want_p[at(t)] = O.evict(pool.weight[at(t)], pool.position[at(t)], budget, recent)
            for x in kv:
                x[at(to)] = x[at(of)]
    assert np.array_equal(cache.weight.cpu().numpy(), want_w) and np.array_equal(cache.position.cpu().numpy(), want_p)
    for got, want in zip((raw(cache.k), raw(cache.v)), kv):
        assert np.array_equal(got, want)
    for got, want in zip((cache.k_scale, cache.v_scale), kv[2:]):
        assert np.array_equal(got.cpu().numpy(), want)
