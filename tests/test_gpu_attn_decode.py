"""GPU: attention over the paged cache against the fp64 oracle."""
import numpy as np
import pytest

from gpu_util import say, torch_cuda
from kv_util import BF16_U, F32_U, Pool, attn_tolerance
from oracle import decode as O

pytestmark = pytest.mark.gpu

CASES = [
    # lens, heads, group, D, page_size, kv, x, layout
    ([1], 1, 1, 16, 1, "bf16", "f32", "hnd"),
    ([0, 1, 2, 31, 32, 33, 0], 2, 1, 64, 16, "bf16", "bf16", "hnd"),
    ([127, 128, 129, 255, 256, 257], 2, 4, 128, 64, "bf16", "bf16", "hnd"),
    ([127, 128, 129, 255, 256, 257], 2, 4, 128, 64, "e4m3", "f32", "nhd"),
    ([5, 100, 1000], 3, 5, 96, 24, "bf16", "f32", "wide"),
    ([5, 100, 1000], 3, 5, 80, 7, "e4m3", "bf16", "wide"),
    ([700, 0, 3], 1, 16, 256, 32, "bf16", "bf16", "hnd"),
    ([700, 0, 3], 1, 17, 192, 48, "e4m3", "f32", "hnd"),
    ([300, 41], 1, 40, 128, 128, "bf16", "f32", "nhd"),
    ([2000, 1, 4000], 4, 2, 64, 1, "e4m3", "bf16", "hnd"),
    ([9001], 2, 8, 128, 16, "bf16", "bf16", "hnd"),
    ([9001], 1, 3, 112, 5, "bf16", "f32", "nhd"),
    (list(range(0, 140, 2)) + [600], 2, 1, 48, 16, "e4m3", "bf16", "hnd"),  # more sequences than a wave has lanes
    ([40] * 300, 8, 1, 32, 8, "bf16", "bf16", "hnd"),  # more rows than workgroups
]


def _run(torch, sdq, pool, q, track, scale=None, **kw):
    B, hq = q.shape[:2]
    lse = torch.empty((B, hq), device="cuda")
    w = pool.cache.weight.clone() if track else None
    out = sdq.attn_decode(q, pool.cache, pool.table_gpu, pool.lens_gpu, scale=scale, lse=lse, weight_out=w, **kw)
    torch.cuda.synchronize()
    return out, lse, w


@pytest.mark.parametrize("track", [False, True])
@pytest.mark.parametrize("case", CASES, ids=lambda c: "-".join(str(x) if not isinstance(x, list) else f"B{len(x)}x{max(x)}" for x in c))
def test_attention(case, track):
    torch = torch_cuda()
    import paper_2406_13868_amd as sdq

    lens, heads, g, D, ps, kvt, xt, layout = case
    say("attend", case[1:], len(lens), max(lens), track)
    rng = np.random.default_rng(len(lens) * 7 + D + ps)
    pool = Pool(torch, sdq, rng, lens, heads, ps, D, kvt, layout, track)
    scale = 0.11 if g == 5 else None
    tq = torch.from_numpy((1.5 * rng.standard_normal((len(lens), heads * g, D))).astype(np.float32))
    tq = tq.to(torch.bfloat16 if xt == "bf16" else torch.float32)
    # sequences with a gap between them
    wide = torch.zeros((len(lens), heads * g + 1, D), dtype=tq.dtype, device="cuda")
    wide[:, :-1] = tq.cuda()
    out, lse, w = _run(torch, sdq, pool, wide[:, :-1], track, scale)
    assert out.dtype == tq.dtype
    q = tq.float().numpy().astype(np.float64)
    got, lse = out.float().cpu().numpy().astype(np.float64), lse.cpu().numpy().astype(np.float64)
    w = w.cpu().numpy() if track else None
    out_u, split_u = (BF16_U, 2.0 ** -17) if xt == "bf16" else (F32_U, 3 * F32_U)
    touched = None if w is None else np.zeros(w.shape, bool)
    for b, n in enumerate(lens):
        for h in range(heads):
            sel = slice(h * g, (h + 1) * g)
            ref = O.attend(q[b, sel], pool.rows(O, "k", b, h), pool.rows(O, "v", b, h), D ** -0.5 if scale is None else scale)
            tol, tol_lse, tol_p = attn_tolerance(ref, n, D, out_u, split_u)
            assert np.all(np.abs(got[b, sel] - ref["out"]) <= tol), f"sequence {b} head {h}: {np.max(np.abs(got[b, sel] - ref['out']) / tol):.3g} of the bound"
            if n == 0:
                assert np.all(lse[b, sel] == -np.inf) and not got[b, sel].any()
                continue
            assert np.all(np.abs(lse[b, sel] - ref["lse"]) <= tol_lse)
            if track:
                t = np.arange(n)
                i = (pool.table[b][t // ps], h, t % ps)
                touched[i] = True
                want = pool.weight[i].astype(np.float64) + ref["p"].sum(0)
                tol_w = tol_p.sum(0) + (g + 2) * F32_U * np.abs(want)
                assert np.all(np.abs(w[i] - want) <= tol_w), f"weights of sequence {b} head {h}"
    if track:
        assert np.array_equal(w[~touched], pool.weight[~touched]), "slots of no sequence are not written"
        again = pool.cache.weight.clone()
        pool.cache.weight.copy_(torch.from_numpy(pool.weight))
        sdq.attn_decode(wide[:, :-1], pool.cache, pool.table_gpu, pool.lens_gpu, scale=scale, weight_out=pool.cache.weight)
        assert torch.equal(pool.cache.weight.cpu(), torch.from_numpy(w)), "in place"
        del again


def _small(torch, sdq, lens=(70, 300), heads=2, g=2, D=64, ps=16, seed=3, **kw):
    rng = np.random.default_rng(seed)
    pool = Pool(torch, sdq, rng, list(lens), heads, ps, D, **kw)
    q = torch.from_numpy(rng.standard_normal((len(lens), heads * g, D)).astype(np.float32)).cuda()
    return pool, q


def test_the_bound_on_the_lengths_does_not_change_results_it_covers():
    torch = torch_cuda()
    import paper_2406_13868_amd as sdq

    pool, q = _small(torch, sdq)
    want = sdq.attn_decode(q, pool.cache, pool.table_gpu, pool.lens_gpu)
    assert torch.equal(sdq.attn_decode(q, pool.cache, pool.table_gpu, pool.lens_gpu, max_len=300), want)
    # a bound below a length cuts it, and a negative length is none
    cut = sdq.attn_decode(q, pool.cache, pool.table_gpu, pool.lens_gpu, max_len=70)
    short = sdq.attn_decode(q, pool.cache, pool.table_gpu, torch.tensor([70, 70], dtype=torch.int32).cuda())
    assert torch.equal(cut, short) and torch.equal(cut[0], want[0])
    none = sdq.attn_decode(q, pool.cache, pool.table_gpu, torch.tensor([-5, 300], dtype=torch.int32).cuda())
    assert not none[0].any() and torch.allclose(none[1], want[1], rtol=1e-5, atol=1e-6)


def test_pages_that_are_absent_are_masked():
    torch = torch_cuda()
    import paper_2406_13868_amd as sdq

    pool, q = _small(torch, sdq, lens=(64,), ps=16)
    table = pool.table_gpu.clone()
    table[0, 1], table[0, 2] = -1, pool.pages
    got = sdq.attn_decode(q, pool.cache, table, pool.lens_gpu)
    packed = pool.table_gpu[:, [0, 3]].contiguous()
    want = sdq.attn_decode(q, pool.cache, packed, torch.tensor([32], dtype=torch.int32).cuda())
    assert torch.allclose(got, want, rtol=1e-5, atol=1e-6)


def test_all_pages_absent_is_an_empty_row():
    torch = torch_cuda()
    import paper_2406_13868_amd as sdq

    pool, q = _small(torch, sdq)
    lse = torch.zeros(q.shape[:2], device="cuda")
    out = sdq.attn_decode(q, pool.cache, torch.full_like(pool.table_gpu, -1), pool.lens_gpu, lse=lse)
    assert not out.any() and torch.isneginf(lse).all()


def test_infinities_and_nan_in_live_slots_reach_their_own_heads_only():
    torch = torch_cuda()
    import paper_2406_13868_amd as sdq

    pool, q = _small(torch, sdq)
    clean = sdq.attn_decode(q, pool.cache, pool.table_gpu, pool.lens_gpu)
    page = int(pool.table[0, 1])
    pool.cache.v[page, 1, 3, 5] = float("nan")
    got = sdq.attn_decode(q, pool.cache, pool.table_gpu, pool.lens_gpu)
    assert torch.isnan(got[0, 2:, 5]).all()
    got[0, 2:, 5] = clean[0, 2:, 5]
    assert torch.equal(got, clean)


def test_extreme_scores_do_not_overflow():
    torch = torch_cuda()
    import paper_2406_13868_amd as sdq

    pool, q = _small(torch, sdq)
    out = sdq.attn_decode(q * 1000, pool.cache, pool.table_gpu, pool.lens_gpu)
    assert torch.isfinite(out).all()
    for b in range(2):  # the row of the largest score alone
        for h in range(4):
            k, v = (torch.from_numpy(pool.rows(O, x, b, h // 2)) for x in "kv")
            best = int((k @ q[b, h].cpu().double()).argmax())
            assert torch.allclose(out[b, h].cpu().double(), v[best], atol=1e-6)


def test_offsets_past_32_bits():
    torch = torch_cuda()
    import paper_2406_13868_amd as sdq

    heads, ps, D = 8, 64, 128  # 128 KiB per page: page 40000 lies past 4 GiB
    k, v = (torch.empty((40003, heads, ps, D), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    ids = torch.tensor([[40001, 7, 40002, 32768]], dtype=torch.int32, device="cuda")
    near = sdq.KVCache.empty(4, heads, ps, D)
    g = torch.Generator(device="cuda").manual_seed(0)
    for i, p in enumerate(ids[0].tolist()):
        for far, t in ((k, near.k), (v, near.v)):
            t[i] = torch.randn((heads, ps, D), generator=g, device="cuda").to(torch.bfloat16)
            far[p] = t[i]
    q = torch.randn((1, 16, D), generator=g, device="cuda").to(torch.bfloat16)
    lens = torch.tensor([230], dtype=torch.int32, device="cuda")
    far = sdq.KVCache(k, v)
    got = sdq.attn_decode(q, far, ids, lens)
    want = sdq.attn_decode(q, near, torch.arange(4, dtype=torch.int32, device="cuda")[None], lens)
    assert torch.equal(got, want)
    # the appended row lands there too
    qkv = torch.randn((1, 32 * D), generator=g, device="cuda").to(torch.bfloat16)
    sdq.qkv_append(qkv, None, torch.tensor([40002 * ps + 37], device="cuda"), far, 16)
    assert torch.equal(far.v[40002, :, 37].flatten(), qkv[0, -heads * D:])


def test_repeated_calls_agree_and_a_graph_replays_them():
    torch = torch_cuda()
    import paper_2406_13868_amd as sdq

    rng = np.random.default_rng(5)
    pool = Pool(torch, sdq, rng, [3000, 17, 1200], 2, 16, 128, track=True, poison=False)
    q = torch.from_numpy(rng.standard_normal((3, 8, 128)).astype(np.float32)).cuda()
    ws = torch.empty(sdq.attn_decode_workspace_size(pool.cache, 3, 8, 3008, True), dtype=torch.uint8, device="cuda")
    out, lse, w = torch.empty_like(q), torch.empty((3, 8), device="cuda"), torch.zeros_like(pool.cache.weight)
    call = lambda: sdq.attn_decode(q, pool.cache, pool.table_gpu, pool.lens_gpu, max_len=3008, out=out, lse=lse, weight_out=w, workspace=ws)  # noqa: E731
    call()
    first = [t.clone() for t in (out, lse, w)]
    for _ in range(3):
        ws.random_()  # what the workspace holds does not matter
        call()
        assert all(torch.equal(a, b) for a, b in zip(first, (out, lse, w)))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            call()
    for i in range(4):
        q.copy_(torch.from_numpy(np.random.default_rng(i).standard_normal(q.shape).astype(np.float32)))
        pool.lens_gpu.copy_(torch.tensor([3000 - 700 * i, 17 * i, 1200], dtype=torch.int32))
        w.zero_()
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (out, lse, w)]
        w.zero_()
        call()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, (out, lse, w))), f"replay {i}"


def test_another_stream_than_the_current_one():
    torch = torch_cuda()
    import paper_2406_13868_amd as sdq

    pool, q = _small(torch, sdq, lens=(2000, 5))
    want = sdq.attn_decode(q, pool.cache, pool.table_gpu, pool.lens_gpu)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    got = sdq.attn_decode(q, pool.cache, pool.table_gpu, pool.lens_gpu, stream=side)
    side.synchronize()
    assert torch.equal(got, want)


def test_no_sequences():
    torch = torch_cuda()
    import paper_2406_13868_amd as sdq

    pool, q = _small(torch, sdq)
    out = sdq.attn_decode(q[:0], pool.cache, pool.table_gpu[:0], pool.lens_gpu[:0])
    assert out.shape == (0, 4, 64)
