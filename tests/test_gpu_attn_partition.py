"""GPU: every live slot takes part in attention once, however the rows are divided.

All keys are zero, so every slot of a row has the same weight.  Values tell the
slot's number by its remainders: each call of a case has a modulus, dim or one
below it, and gives slot t a one in the dimension t % modulus.  An output times
the length is then the count of the slots with that remainder: one slot lost or
taken twice moves the counts of every call by one, and two such faults cancel in
all of them only if they are the same slot, as the moduli have no common divisors
and a product above the length.
Terms, sums and joins of these calls are exact: ones, whole numbers below 2^24,
exp2(0).  What is left is the reciprocal of the length and a product (fp32), and
the rounding to bf16."""
import math

import numpy as np
import pytest

from gpu_util import say, torch_cuda
from kv_util import BF16_U, make_table

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


def _ragged(B, most, seed):
    n = np.random.default_rng(seed).integers(0, most + 1, B)
    n[:4] = [most, 0, 1, most - 1]
    return [int(x) for x in n]


CASES = [
    # lens, heads, group, D, page_size, kv, x
    # rows split over workgroups, more sequences than a wave has lanes
    (_ragged(65, 3000, 0), 1, 1, 128, 16, "bf16", "f32"),
    (_ragged(65, 3000, 1), 1, 4, 112, 24, "bf16", "f32"),
    (_ragged(129, 3001, 2), 1, 3, 64, 16, "e4m3", "bf16"),
    (_ragged(129, 2047, 3), 2, 1, 96, 7, "e4m3", "f32"),
    (_ragged(130, 1500, 4), 1, 17, 256, 32, "bf16", "f32"),
    (_ragged(200, 1300, 5), 1, 2, 128, 64, "e4m3", "f32"),
    (_ragged(129, 1100, 6), 1, 1, 80, 1, "bf16", "bf16"),
    # long rows, few or one
    ([9001], 1, 3, 112, 5, "bf16", "f32"),
    ([9001], 2, 8, 128, 16, "bf16", "bf16"),
    ([9001, 4097, 4096], 2, 1, 64, 48, "e4m3", "f32"),
    ([131071], 1, 4, 64, 128, "e4m3", "f32"),
    ([40000, 7], 2, 2, 256, 64, "bf16", "f32"),
    # rows that are not split
    (list(range(0, 1000, 9)), 4, 1, 128, 16, "bf16", "f32"),
    (_ragged(300, 130, 7), 4, 5, 32, 8, "bf16", "f32"),
    (_ragged(70, 500, 8), 2, 1, 192, 16, "e4m3", "bf16"),
]


@pytest.mark.parametrize("track", [False, True])
@pytest.mark.parametrize("case", CASES, ids=lambda c: "-".join(str(x) if not isinstance(x, list) else f"B{len(x)}x{max(x)}" for x in c))
def test_every_slot_counts_once(case, track):
    torch = torch_cuda()
    import paper_2406_13868_amd as sdq

    lens, heads, g, D, ps, kvt, xt = case
    say("partition", len(lens), max(lens), case[1:], track)
    rng = np.random.default_rng(D)
    table, pages = make_table(rng, lens, ps)
    slot_of = np.full((pages, ps), -1)  # the slot that lies there
    owner = np.zeros((pages, ps), int)
    for b, n in enumerate(lens):
        t = np.arange(n)
        slot_of[table[b][t // ps], t % ps], owner[table[b][t // ps], t % ps] = t, b
    slot_of_gpu = torch.from_numpy(slot_of).cuda()
    used = (slot_of_gpu >= 0)[:, None, :].expand(pages, heads, ps)
    dt = torch.bfloat16 if kvt == "bf16" else torch.float8_e4m3fn
    k = torch.zeros((pages, heads, ps, D), device="cuda").masked_fill(~used[..., None], float("nan")).to(dt)
    v = torch.empty((pages, heads, ps, D), dtype=dt, device="cuda")
    scales = (None, None)
    if kvt == "e4m3":  # powers of two, undone by the codes
        vs = torch.from_numpy(2.0 ** rng.integers(-2, 3, (pages, heads, ps))).float().cuda()
        ks = torch.from_numpy(rng.uniform(0.5, 2, (pages, heads, ps)).astype(np.float32)).cuda()
        scales = tuple(s.masked_fill(~used, float("nan")) for s in (ks, vs))
    weight = torch.zeros((pages, heads, ps), device="cuda") if track else None
    cache = sdq.KVCache(k, v, *scales, weight=weight)
    w_out = torch.full((pages, heads, ps), -3.0, device="cuda") if track else None
    q = torch.from_numpy(rng.standard_normal((len(lens), heads * g, D)).astype(np.float32)).cuda()
    q = q.to(torch.bfloat16) if xt == "bf16" else q
    lse = torch.empty((len(lens), heads * g), device="cuda")
    table_gpu, lens_gpu = torch.from_numpy(table).cuda(), torch.tensor(lens, dtype=torch.int32).cuda()
    moduli = [D]
    while math.prod(moduli) <= max(lens):
        moduli.append(next(m for m in range(moduli[-1] - 1, 1, -1) if all(math.gcd(m, x) == 1 for x in moduli)))
    for modulus in moduli:
        one = ((slot_of_gpu % modulus)[..., None] == torch.arange(D, device="cuda"))[:, None].expand(pages, heads, ps, D).float()
        if kvt == "e4m3":
            one = one / vs[..., None]
        v.copy_(one.masked_fill(~used[..., None], float("nan")).to(dt))
        out = sdq.attn_decode(q, cache, table_gpu, lens_gpu, max_len=max(lens), lse=lse, weight_out=w_out).double().cpu().numpy()
        for b, n in enumerate(lens):
            count = np.bincount(np.arange(n) % modulus, minlength=D).astype(float)
            off = np.abs(out[b] * n - count)
            assert np.all(off <= count * (4 * U + (BF16_U if xt == "bf16" else 0))), f"sequence {b} of {n} slots, modulo {modulus}: off by {off.max()}"
            if xt == "bf16":
                assert count.max() * 2 * BF16_U < 1, "a slot shows in the rounded output"
    got = lse.double().cpu().numpy()
    for b, n in enumerate(lens):  # log2 of the count and its conversion
        assert np.all(got[b] == -np.inf) if n == 0 else np.all(np.abs(got[b] - math.log(n)) <= 8 * U * max(1, math.log(n))), (b, n)
    if track:
        w = w_out.double().cpu().numpy()
        live = slot_of >= 0
        want = np.where(live, g / np.maximum(np.array(lens)[owner], 1), 0)[:, None, :].repeat(heads, 1)
        # log2 of the sum moves an exponent by up to 2^-23 of it, a weight by that
        # times ln 2; the exponential; the sum over the heads
        tol = (2 * math.log2(max(lens) + 1) + 4 + g) * U
        live = live[:, None, :].repeat(heads, 1)
        assert np.all(np.abs(w - want)[live] <= tol * want[live]) and np.all(w[~live] == -3)


@pytest.mark.parametrize("lens", [[300, 5], [3000, 1, 0, 2047]], ids=str)
@pytest.mark.parametrize("dim", [64, 128, 256])
def test_scales_that_are_aligned_to_their_type_only(lens, dim):
    """e4m3 scales four bytes past a 16-byte boundary: another path to the same exact results."""
    torch = torch_cuda()
    import paper_2406_13868_amd as sdq

    say("scales off alignment", lens, dim)
    rng = np.random.default_rng(dim)
    table, pages = make_table(rng, lens, 32)
    shape = (pages, 2, 32)
    code = torch.from_numpy(2.0 ** rng.integers(-2, 3, (*shape, dim))).float().cuda()
    k, v = torch.zeros_like(code).to(torch.float8_e4m3fn), code.to(torch.float8_e4m3fn)
    vs = torch.from_numpy(2.0 ** rng.integers(-2, 3, shape)).float().cuda()
    q = torch.from_numpy(rng.standard_normal((len(lens), 6, dim)).astype(np.float32)).cuda()
    table_gpu, lens_gpu = torch.from_numpy(table).cuda(), torch.tensor(lens, dtype=torch.int32).cuda()

    def moved(t):
        buf = torch.empty(t.numel() + 1, device="cuda")
        buf[1:] = t.flatten()
        return buf[1:].view(t.shape)

    near, off = (sdq.KVCache(k, v, a, b) for a, b in ((vs, vs), (moved(vs), moved(vs))))
    assert near.v_scale.data_ptr() % 16 == 0 and off.v_scale.data_ptr() % 16 == 4
    want, got = (sdq.attn_decode(q, c, table_gpu, lens_gpu, max_len=max(lens)) for c in (near, off))
    assert torch.equal(got, want)
    page, at = table[0][np.arange(lens[0]) // 32], np.arange(lens[0]) % 32
    mean = (code * vs[..., None]).double()[page, :, at].mean(0)
    assert torch.all((got[0].double().view(2, 3, dim) - mean[:, None]).abs() <= 4 * U * mean[:, None])
