"""GPU: the operators between a block's products run together, as a feed-forward block
runs them: eagerly, captured and replayed, on other streams, and far into memory."""
import ctypes

import numpy as np
import pytest

from block_util import codes_near, equal, rounded
from gpu_util import say, torch_cuda
from oracle import block as O

pytestmark = pytest.mark.gpu


class Block:
    """norm -> gate/up product -> activation -> down product -> the stream, through every kernel's own buffers."""

    def __init__(self, torch, sdq, M, width, hidden, seed=0, act="silu", given=True):
        self.torch, self.sdq, self.M, self.width, self.hidden, self.act = torch, sdq, M, width, hidden, act
        rng = np.random.default_rng(seed)
        dev = lambda a: torch.from_numpy(np.ascontiguousarray(a, np.float32)).cuda()  # noqa: E731
        cfg = sdq.Config.int_family()
        self.W1, self.W2 = dev(rng.standard_normal((2 * hidden, width)) / np.sqrt(width)), dev(rng.standard_normal((width, hidden)) / np.sqrt(hidden))
        self.w1, self.s1 = sdq.quantize_act(self.W1, cfg)
        self.w2, self.s2 = sdq.quantize_act(self.W2, cfg)
        self.pre, self.post, self.last = (dev(rng.uniform(0.5, 1.5, width)) for _ in range(3))
        self.gate, self.bias = dev(rng.uniform(0.5, 1.5, (1, width))), dev(0.1 * rng.standard_normal(width))
        self.x = dev(rng.standard_normal((M, width))).bfloat16()
        b = lambda n, dt: torch.empty((M, n), dtype=dt, device="cuda") if given else None  # noqa: E731
        v = lambda: torch.empty(M, device="cuda") if given else None  # noqa: E731
        self.n, self.sn, self.gu, self.h, self.sh = b(width, torch.uint8), v(), b(2 * hidden, torch.bfloat16), b(hidden, torch.uint8), v()
        self.y, self.r, self.q, self.sq = b(width, torch.float32), b(width, torch.bfloat16), b(width, torch.uint8), v()

    def __call__(self, stream=None):
        sdq = self.sdq
        _, n, sn = sdq.block_norm(self.x, weight=self.pre, out_dtype="int8", out=self.n, scales=self.sn, stream=stream)
        gu = sdq.gemm_int8(n, sn, self.w1, self.s1, out=self.gu, out_dtype=self.torch.bfloat16, stream=stream)
        h, sh = sdq.glu_act(gu, self.act, out_dtype="int8", out=self.h, scales=self.sh, stream=stream)
        y = sdq.gemm_int8(h, sh, self.w2, self.s2, bias=self.bias, out=self.y, out_dtype=self.torch.float32, stream=stream)
        r, q, sq = sdq.block_norm(self.x, y, self.last, post_weight=self.post, gate=self.gate, scale=0.5, out_dtype="e4m3", out=self.q,
                                  scales=self.sq, residual_out=self.r, stream=stream)
        return dict(n=n, sn=sn, gu=gu, h=h, sh=sh, y=y, r=r, q=q, sq=sq)


def _check(b, got):
    """Every step against the oracle on what the step before gave."""
    torch, g = b.torch, {k: t.cpu() for k, t in got.items()}
    host = lambda t: t.float().cpu().numpy()  # noqa: E731
    i8 = lambda t: t.cpu().view(torch.int8).numpy()  # noqa: E731
    codes, scales = O.codes_steps(O.norm_steps(host(b.x), host(b.pre), None, 1e-6, False), "int8")
    assert equal(g["n"].numpy(), codes) and equal(g["sn"].numpy(), scales)
    _, total = O.product64(i8(g["n"]), host(g["sn"]), i8(b.w1), host(b.s1))
    assert equal(host(g["gu"]), rounded(torch, total.astype(np.float32) * host(g["sn"])[:, None] * host(b.s1), torch.bfloat16))
    codes_near(g["h"].numpy(), g["sh"].numpy(), O.activation64(host(g["gu"]), b.act, True), "int8", O.U * (1 + 1e-6))
    _, total = O.product64(i8(g["h"]), host(g["sh"]), i8(b.w2), host(b.s2))
    assert equal(host(g["y"]), total.astype(np.float32) * host(g["sh"])[:, None] * host(b.s2) + host(b.bias))
    r = O.stream_steps(host(b.x), host(g["y"]), host(b.gate), 0.5, host(b.post))
    assert equal(host(g["r"]), rounded(torch, r, torch.bfloat16))
    codes, scales = O.codes_steps(O.norm_steps(r, host(b.last), None, 1e-6, False), "e4m3")
    assert equal(g["q"].numpy(), codes) and equal(g["sq"].numpy(), scales)


@pytest.mark.parametrize("M,width,hidden,act", [(1, 512, 1376, "silu"), (5, 1024, 2752, "gelu"), (40, 512, 1056, "silu"), (200, 768, 2048, "relu")])
def test_a_feed_forward_block(M, width, hidden, act):
    torch = torch_cuda()
    import paper_2406_13868_amd as sdq
    say(M, width, hidden, act)
    b = Block(torch, sdq, M, width, hidden, M, act)
    got = b()
    _check(b, got)
    # and near the block in 64 bits with its weights as they were: a code of a normal row of largest 3.5 to 4 is off by
    # 4 / 127 / sqrt(12) = 0.9% of its size in the mean, on both sides of two products 1.8%; the largest of a row may be twice that
    x, W1, W2 = (t.double().cpu().numpy() for t in (b.x, b.W1, b.W2))
    host = lambda t: t.double().cpu().numpy()  # noqa: E731
    y = O.activation64(O.norm64(x, host(b.pre), None, 1e-6, False) @ W1.T, act, True) @ W2.T + host(b.bias)
    off = np.linalg.norm(host(got["y"]) - y) / np.linalg.norm(y)
    assert off < 0.05, off


def test_the_codes_are_what_the_decomposed_products_read():
    torch = torch_cuda()
    import paper_2406_13868_amd as sdq
    import synth
    M, N, K = 9, 96, 512
    rng = np.random.default_rng(0)
    x = torch.from_numpy(rng.standard_normal((M, K)).astype(np.float32)).cuda()
    w = torch.from_numpy(rng.uniform(0.5, 1.5, K).astype(np.float32)).cuda()
    _, n, _ = sdq.block_norm(x, weight=w)
    W = synth.make_w(3, 0, N, K)
    for cfg, kind in ((sdq.Config.int_family(), "int8"), (sdq.Config.mx_family(), "e4m3")):
        say(kind)
        blob = torch.from_numpy(sdq.pack(W, cfg)).cuda()
        _, q, s = sdq.block_norm(x, weight=w, out_dtype=kind)
        want_q, want_s = sdq.quantize_act(n, cfg)
        # the factor is one rounding apart, which no code of these rows is near enough a tie to show
        assert torch.equal(q, want_q) and torch.equal(s, want_s)
        assert torch.equal(sdq.gemm(q, s, blob, N, K, cfg), sdq.gemm(want_q, want_s, blob, N, K, cfg))


@pytest.mark.parametrize("M,width,hidden", [(1, 1024, 2752), (64, 4096, 4096), (300, 512, 1376)])
@pytest.mark.parametrize("given", [False, True])
def test_a_captured_block_replays(M, width, hidden, given):
    """Replayed with new inputs between eager calls of the same program; M = 64 divides a product over its depth."""
    torch = torch_cuda()
    import paper_2406_13868_amd as sdq
    say(M, width, hidden, given)
    b = Block(torch, sdq, M, width, hidden, 1, given=given)
    if M == 64:
        assert sdq.gemm_int8_workspace_size(M, 4096, 16384) > 0
    b()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = b()
    for k in range(4):
        b.x.copy_(torch.from_numpy(np.random.default_rng(k).standard_normal((M, width)).astype(np.float32)) * (k + 1))
        graph.replay()
        torch.cuda.synchronize()
        replayed = {n: t.clone() for n, t in held.items()}
        eager = {n: t.clone() for n, t in b().items()}
        torch.cuda.synchronize()
        assert all(torch.equal(replayed[n], eager[n]) for n in eager), k


def test_captured_products_that_share_a_workspace():
    torch = torch_cuda()
    import paper_2406_13868_amd as sdq
    M, N, K = 64, 512, 16384
    need = sdq.gemm_int8_workspace_size(M, N, K)
    assert need > 0
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    gen = torch.Generator(device="cuda").manual_seed(0)
    x, w = (torch.randint(-127, 128, s, generator=gen, device="cuda", dtype=torch.int8) for s in ((2, M, K), (2, N, K)))
    s1, s2 = torch.rand(M, device="cuda"), torch.rand(N, device="cuda")
    want = [sdq.gemm_int8(x[i], s1, w[i], s2) for i in range(2)]
    out = [torch.zeros((M, N), device="cuda") for _ in range(2)]
    graphs = []
    for i in range(2):
        sdq.gemm_int8(x[i], s1, w[i], s2, out=out[i], workspace=ws)
        torch.cuda.synchronize()
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[i]):
            sdq.gemm_int8(x[i], s1, w[i], s2, out=out[i], workspace=ws)
    for order in ((0, 1), (1, 0), (0, 0)):
        for o in out:
            o.zero_()
        ws.fill_(0xFF)
        for i in order:
            graphs[i].replay()
        torch.cuda.synchronize()
        assert all(torch.equal(out[i], want[i]) for i in set(order))


def test_two_streams_at_once():
    torch = torch_cuda()
    import paper_2406_13868_amd as sdq
    blocks = [Block(torch, sdq, 64, 512, 8192, k) for k in range(2)]
    want = [{n: t.clone() for n, t in b().items()} for b in blocks]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in blocks]
    for _ in range(5):
        for b, s in zip(blocks, streams):
            b(stream=s)
    torch.cuda.synchronize()
    for b, w in zip(blocks, want):
        assert torch.equal(b.y, w["y"]) and torch.equal(b.q, w["q"]) and torch.equal(b.r, w["r"])


def test_fresh_memory_is_the_streams_own(monkeypatch):
    torch = torch_cuda()
    import paper_2406_13868_amd as sdq
    b = Block(torch, sdq, 64, 512, 8192, given=False)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    on, empty = [], torch.empty

    def record(*a, **k):
        on.append(torch.cuda.current_stream().cuda_stream)
        return empty(*a, **k)

    monkeypatch.setattr(torch, "empty", record)
    got = b(stream=side)
    assert len(on) >= 9 and set(on) == {side.cuda_stream}
    torch.cuda.synchronize()
    on.clear()
    want = b()
    assert set(on) == {torch.cuda.current_stream().cuda_stream}
    monkeypatch.undo()
    torch.cuda.synchronize()
    assert all(torch.equal(got[n], want[n]) for n in want)


def test_a_pending_error_is_not_the_calls_own():
    torch = torch_cuda()
    import paper_2406_13868_amd as sdq
    sdq._lib.lib()
    hip = ctypes.CDLL(next(iter(sdq._lib._hip_runtimes())))
    b = Block(torch, sdq, 3, 64, 128)
    calls = [lambda: sdq.block_norm(b.x, weight=b.pre, out_dtype="int8", out=b.n, scales=b.sn)[1],
             lambda: sdq.gemm_int8(b.n, b.sn, b.w1, b.s1, out=b.gu), lambda: sdq.glu_act(b.gu, out_dtype="int8", out=b.h, scales=b.sh)[0]]
    for call in calls:
        want = call().clone()
        torch.cuda.synchronize()
        hip.hipGetLastError()
        assert hip.hipSetDevice(ctypes.c_int(1 << 20)) != 0 and hip.hipPeekAtLastError() != 0
        got = call()
        assert hip.hipPeekAtLastError() == 0
        torch.cuda.synchronize()
        assert torch.equal(got, want)


def test_offsets_that_pass_32_bits():
    """Rows far apart: the last ones lie past 2^32 bytes."""
    torch = torch_cuda()
    import paper_2406_13868_amd as sdq
    rng = np.random.default_rng(4)
    M, N, K = 1100, 300, 64
    x, w = (torch.from_numpy(rng.integers(-127, 128, (n, K)).astype(np.int8)).cuda() for n in (M, N))
    sx, sw = (torch.from_numpy(rng.uniform(0.5, 2, n).astype(np.float32)).cuda() for n in (M, N))
    want = sdq.gemm_int8(x, sx, w, sw)
    far = torch.empty((M, 1 << 22), dtype=torch.int8, device="cuda")[:, :K]
    far.copy_(x)
    y = torch.empty((M, 1 << 21), device="cuda")[:, :N]
    say("product", far.stride(), y.stride())
    for m in (M, 7):
        rows = slice(M - m, M)
        sdq.gemm_int8(far[rows], sx[rows], w, sw, out=y[rows])
        assert torch.equal(y[rows], want[rows])
        got = sdq.gemm_int8(w[: m % 50 + 1], sw[: m % 50 + 1], far, sx)
        assert torch.equal(got, sdq.gemm_int8(w[: m % 50 + 1], sw[: m % 50 + 1], x, sx))
    del far, y
    r = torch.from_numpy(rng.standard_normal((M, K)).astype(np.float32)).cuda()
    weight = torch.ones(K, device="cuda")
    want = sdq.block_norm(r, r, weight, out_dtype="int8")
    far = torch.empty((M, 1 << 20), device="cuda")[:, :K]
    far.copy_(r)
    say("norm", far.stride())
    got = sdq.block_norm(far, far, weight, out_dtype="int8", residual_out=far)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]) and torch.equal(got[2], want[2])
    far.copy_(r)
    say("activation", far.stride())
    for out in ("int8", "f32"):
        assert torch.equal(sdq.glu_act(far, out_dtype=out)[0], sdq.glu_act(r, out_dtype=out)[0])
