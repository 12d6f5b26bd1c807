"""GPU: eviction whose new lengths lie over the old ones, in place or shifted."""
import numpy as np
import pytest

from gpu_util import say, torch_cuda
from kv_util import Pool

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("shift", [-3, -1, 0, 1, 40])
def test_overlapping_lengths(shift):
    torch = torch_cuda()
    import paper_2406_13868_amd as sdq

    say("evict, lengths overlap", shift)
    rng = np.random.default_rng(4)
    lens = [int(n) for n in rng.integers(0, 300, 40)]
    budget, recent = 120, 9
    got = []
    for overlap in (False, True):
        pool = Pool(torch, sdq, np.random.default_rng(5), lens, 4, 16, 32, track=True, poison=False)
        if overlap:
            at = max(0, -shift)
            buf = torch.full((40 + abs(shift),), -7, dtype=torch.int32, device="cuda")
            seq_lens, lens_out = buf[at:at + 40], buf[at + shift:at + shift + 40]
            seq_lens.copy_(pool.lens_gpu)
        else:
            seq_lens, lens_out = pool.lens_gpu, torch.empty_like(pool.lens_gpu)
        sdq.cache_evict(pool.cache, pool.table_gpu, seq_lens, budget, recent, lens_out=lens_out)
        torch.cuda.synchronize()
        assert lens_out.tolist() == [min(n, budget) for n in lens]
        c = pool.cache
        got.append([t.view(torch.int16) if t.dtype == torch.bfloat16 else t for t in (c.k, c.v, c.weight, c.position)])
    assert all(torch.equal(a, b) for a, b in zip(*got))
