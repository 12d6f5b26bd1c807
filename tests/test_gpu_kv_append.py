"""GPU: norm, rotation and append against the fp64 oracle."""
import numpy as np
import pytest

from gpu_util import say, torch_cuda
from kv_util import BF16_U, E4M3_U, F32_U
from oracle import decode as O
from oracle import formats as F

pytestmark = pytest.mark.gpu

# fp32 arithmetic of a rotated, normalized element, in half steps of the sum of
# the magnitudes it is added up from: the mean square (8 additions in a lane, 5
# across lanes, halved by the root), root, division and eps (3), the two norm
# products on each side of the pair (2) and the two rotation products and their
# sum (3), on values that are exact on entry: 6.5 + 3 + 2 + 3 < 16.
ARITH = 16 * F32_U

CASES = [
    # M, heads_q, heads, D, page_size, rot, interleaved, norm, x, kv
    (1, 32, 32, 128, 64, 128, False, False, "bf16", "bf16"),
    (1, 4, 1, 16, 1, 16, False, True, "f32", "e4m3"),
    (5, 8, 2, 64, 16, 64, True, True, "bf16", "e4m3"),
    (33, 6, 3, 96, 24, 48, True, True, "f32", "bf16"),
    (33, 6, 3, 80, 7, 20, False, False, "bf16", "e4m3"),   # pairs that straddle a lane's eight elements
    (33, 6, 3, 80, 7, 20, True, True, "f32", "bf16"),
    (17, 5, 5, 192, 32, 192, False, True, "bf16", "bf16"),
    (9, 16, 1, 256, 128, 128, False, True, "f32", "e4m3"),
    (9, 2, 1, 256, 128, 0, False, False, "bf16", "bf16"),
    (300, 7, 7, 48, 64, 2, False, True, "bf16", "e4m3"),
    (3, 2, 2, 112, 5, 112, True, False, "bf16", "e4m3"),
]


def _inputs(rng, M, hq, hkv, D, rot, norm, slots, positions=97):
    x = rng.standard_normal((M, hq + 2 * hkv, D)).astype(np.float32)
    x[:, :, ::11] *= 6
    pos = rng.integers(0, positions, M).astype(np.int32)
    slot = rng.permutation(slots)[:M].astype(np.int64)
    ang = rng.uniform(-np.pi, np.pi, (positions, rot // 2))
    cs = np.concatenate([np.cos(ang), np.sin(ang)], 1).astype(np.float32)
    w = [(1 + 0.3 * rng.standard_normal(D)).astype(np.float32) for _ in range(2)] if norm else [None, None]
    return x, pos, slot, cs, w


def _check(got, want, size, kind, what):
    tol = ARITH * size + (BF16_U * np.abs(want) if kind == "bf16" else 0) + 1e-37
    err = np.abs(got - want)
    assert np.all(err <= tol), f"{what}: {np.max(err / tol):.3g} of the bound"


@pytest.mark.parametrize("case", CASES, ids=lambda c: "-".join(map(str, c)))
@pytest.mark.parametrize("layout", ["hnd", "nhd"])
def test_append(case, layout):
    torch = torch_cuda()
    import paper_2406_13868_amd as sdq

    M, hq, hkv, D, ps, rot, inter, norm, xt, kvt = case
    say("append", case, layout)
    rng = np.random.default_rng(M + D + rot)
    pages = -(-2 * M // ps) + 1
    x, pos, slot, cs, w = _inputs(rng, M, hq, hkv, D, rot, norm, pages * ps)
    if M > 4:
        slot[1], slot[3] = -1, pages * ps  # padding rows: outside the cache on either side
    tx = torch.from_numpy(x.reshape(M, -1)).to(torch.bfloat16 if xt == "bf16" else torch.float32)
    x = tx.float().numpy().reshape(x.shape)
    cache = sdq.KVCache.empty(pages, hkv, ps, D, kvt, track=True)
    if layout == "nhd":
        k, v = (torch.zeros((pages, ps, hkv, D), dtype=cache.k.dtype, device="cuda").permute(0, 2, 1, 3) for _ in range(2))
        cache = sdq.KVCache(k, v, cache.k_scale, cache.v_scale, cache.position, cache.weight)
    cache.weight.fill_(7)
    wide = torch.full((M, tx.shape[1] + 16), float("nan"), dtype=tx.dtype, device="cuda")
    wide[:, :-16] = tx.cuda()
    dev = lambda a: None if a is None else torch.from_numpy(a).cuda()  # noqa: E731
    q = sdq.qkv_append(wide[:, :-16], dev(pos), dev(slot), cache, hq, dev(cs) if rot else None, inter, dev(w[0]), dev(w[1]), 1e-5)
    torch.cuda.synchronize()
    assert q.dtype == tx.dtype
    q = q.float().cpu().numpy().astype(np.float64)
    K, V = (t.float().cpu().numpy().astype(np.float64) for t in (cache.k, cache.v))
    KS, VS = (None if t is None else t.cpu().numpy() for t in (cache.k_scale, cache.v_scale))
    P, W = cache.position.cpu().numpy(), cache.weight.cpu().numpy()
    written = np.zeros((pages, ps), bool)
    for m in range(M):
        ang = cs[pos[m]].astype(np.float64) if rot else None
        for h in range(hq):
            y, size = O.transform(x[m, h], w[0], 1e-5, ang, inter)
            _check(q[m, h], y, size, xt, f"query {m} {h}")
        if not 0 <= slot[m] < pages * ps:
            continue
        at = (slot[m] // ps, slot[m] % ps)
        written[at] = True
        for h in range(hkv):
            y, size = O.transform(x[m, hq + h], w[1], 1e-5, ang, inter)
            i = (at[0], h, at[1])
            assert P[i] == pos[m] and W[i] == 0
            raw = x[m, hq + hkv + h]
            if kvt == "bf16":
                _check(K[i], y, size, "bf16", f"key {m} {h}")
                assert np.array_equal(V[i], torch.from_numpy(raw).to(torch.bfloat16).float().numpy())
                continue
            codes, s = O.quantize_row(raw)
            assert VS[i] == s and np.array_equal(V[i], F.e4m3_decode(codes)), "values are the library's row rule, bit for bit"
            a = np.abs(y).max()
            assert abs(KS[i] - a / 448) <= (ARITH * size.max() + 2 * F32_U * a) / 448 + 1e-37
            # a code is off by half a step of its size, and by what its fp32 quotient is off
            tol = np.maximum(E4M3_U * np.abs(y), 2.0 ** -10 * KS[i]) + 2 * ARITH * size.max() + 4 * F32_U * np.abs(y)
            assert np.all(np.abs(K[i] * float(KS[i]) - y) <= tol)
    rest = ~written[:, None, :].repeat(hkv, 1)
    assert not np.any(K[rest]) and not np.any(V[rest]) and np.all(P[rest] == -1) and np.all(W[rest] == 7)


def test_positions_outside_the_table_give_nan_and_append_nothing():
    torch = torch_cuda()
    import paper_2406_13868_amd as sdq

    cache = sdq.KVCache.empty(2, 1, 4, 32, track=True)
    qkv = torch.ones((3, 3 * 32), device="cuda")
    pos = torch.tensor([-1, 5, 4], dtype=torch.int32, device="cuda")
    q = sdq.qkv_append(qkv, pos, torch.arange(3, device="cuda"), cache, 1, torch.ones((5, 32), device="cuda"))
    assert torch.isnan(q[:2]).all() and torch.isfinite(q[2]).all()
    assert not cache.k[0, 0, :2].any() and not cache.v[0, 0, :2].any() and cache.v[0, 0, 2].all()
    assert cache.position[0, 0, :3].tolist() == [-1, -1, 4]


def test_rows_that_are_not_finite_show_in_the_scale_and_zero_rows_are_zero():
    torch = torch_cuda()
    import paper_2406_13868_amd as sdq

    cache = sdq.KVCache.empty(1, 1, 4, 32, "e4m3")
    qkv = torch.ones((4, 3 * 32), device="cuda")
    qkv[0, 40], qkv[1, 70], qkv[2, 32:] = float("nan"), float("inf"), 0
    qkv[3, 32:] = 1e-39  # a subnormal row
    sdq.qkv_append(qkv, None, torch.arange(4, device="cuda"), cache, 1)
    ks, vs = cache.k_scale[0, 0], cache.v_scale[0, 0]
    assert torch.isnan(ks[0]) and torch.isinf(vs[1]) and ks[2] == 0 and vs[2] == 0 and vs[0] == 1 / torch.tensor(448.0)
    assert torch.isfinite(cache.k[0, 0, 2:].float() * ks[2:, None]).all() and not cache.k[0, 0, 2].float().any()


def test_no_tokens_and_q_dtypes():
    torch = torch_cuda()
    import paper_2406_13868_amd as sdq

    cache = sdq.KVCache.empty(1, 1, 4, 32)
    none = torch.empty((0, 96), device="cuda")
    assert sdq.qkv_append(none, None, torch.empty(0, dtype=torch.int64, device="cuda"), cache, 1).shape == (0, 1, 32)
    qkv = torch.randn((2, 96), device="cuda")
    slot = torch.arange(2, device="cuda")
    full = sdq.qkv_append(qkv, None, slot, cache, 1)
    half = sdq.qkv_append(qkv, None, slot, cache, 1, out_dtype=torch.bfloat16)
    assert torch.equal(full, qkv[:, :32].unsqueeze(1)) and torch.equal(half, full.to(torch.bfloat16))
