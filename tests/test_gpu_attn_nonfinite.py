"""GPU: NaN and infinities in a live slot's key, value or scale reach the query
heads that read it, and nothing else."""
import numpy as np
import pytest

from gpu_util import say, torch_cuda
from kv_util import Pool

pytestmark = pytest.mark.gpu

SHAPES = [
    # lens, heads, group, D, page_size, kv, x
    ([70, 300], 2, 2, 64, 16, "bf16", "f32"),
    ([70, 300], 2, 2, 96, 24, "bf16", "bf16"),
    ([2000, 90, 1500], 2, 3, 128, 16, "e4m3", "bf16"),
    ([2000, 90, 1500], 3, 1, 80, 7, "e4m3", "f32"),
    ([1900, 5], 2, 17, 256, 32, "bf16", "bf16"),
]


PARTS = {"bf16": ["k nan", "k inf", "k -inf", "v nan", "v inf"],
         "e4m3": ["k nan", "v nan", "k_scale nan", "k_scale inf", "v_scale nan", "v_scale inf"]}


@pytest.mark.parametrize("shape, what", [(s, w) for s in SHAPES for w in PARTS[s[5]]],
                         ids=lambda c: c if isinstance(c, str) else "-".join(str(x) if not isinstance(x, list) else f"B{len(x)}x{max(x)}" for x in c))
def test_only_their_own_heads(shape, what):
    torch = torch_cuda()
    import paper_2406_13868_amd as sdq

    lens, heads, g, D, ps, kvt, xt = shape
    name, kind = what.split()
    say("not finite", shape, what)
    rng = np.random.default_rng(D)
    pool = Pool(torch, sdq, rng, lens, heads, ps, D, kvt, track=True)
    q = torch.from_numpy(rng.standard_normal((len(lens), heads * g, D)).astype(np.float32)).cuda()
    q = q.to(torch.bfloat16) if xt == "bf16" else q

    def call():
        lse, w = torch.empty(q.shape[:2], device="cuda"), torch.zeros_like(pool.cache.weight)
        out = sdq.attn_decode(q, pool.cache, pool.table_gpu, pool.lens_gpu, lse=lse, weight_out=w)
        return [out.float(), lse, w]

    clean = call()
    assert all(torch.isfinite(t).all() for t in clean)
    b, h, t, d = 0, 1, lens[0] - 3, 5
    page, off = int(pool.table[b, t // ps]), t % ps
    part, bad = getattr(pool.cache, name), float(kind)
    if name.endswith("scale"):
        part[page, h, off] = bad
    elif kvt == "e4m3":
        part.view(torch.uint8)[page, h, off, d] = 0x7F
    else:
        part[page, h, off, d] = bad
    got = call()
    mine = slice(h * g, (h + 1) * g)
    own = torch.zeros(clean[2].shape, dtype=torch.bool)
    slots = np.arange(lens[b])
    own[torch.from_numpy(pool.table[b][slots // ps]).long(), h, torch.from_numpy(slots % ps)] = True
    own = own.cuda()
    if name.startswith("k"):
        if kind == "nan":  # every probability of these heads
            assert torch.isnan(got[0][b, mine]).all() and torch.isnan(got[1][b, mine]).all() and torch.isnan(got[2][own]).all()
        got[0][b, mine], got[1][b, mine] = clean[0][b, mine], clean[1][b, mine]
        got[2][own] = clean[2][own]
    else:
        dims = slice(None) if name == "v_scale" else d
        seen = got[0][b, mine, dims]
        assert (torch.isnan(seen) if kind == "nan" else ~torch.isfinite(seen)).all()
        got[0][b, mine, dims] = clean[0][b, mine, dims]
    assert all(torch.equal(x, y) for x, y in zip(got, clean))
