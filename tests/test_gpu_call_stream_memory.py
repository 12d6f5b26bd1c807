"""GPU: what a call with `stream` makes itself (outputs, workspaces) is not memory
of the current stream, where it could be a block that was freed while work
queued there still reads it; and an output's memory is not given out again while
the current stream may still read it."""
import numpy as np
import pytest

import synth
from gpu_util import say, torch_cuda

pytestmark = pytest.mark.gpu


def _calls(torch, sdq):
    """name -> a call that makes everything itself, on the given stream."""
    rng = np.random.default_rng(0)
    cache = sdq.KVCache.empty(80, 2, 16, 64, track=True)
    qkv = torch.from_numpy(rng.standard_normal((33, 8 * 64)).astype(np.float32)).cuda()
    pos, slot = torch.arange(33, dtype=torch.int32, device="cuda"), torch.arange(33, device="cuda")
    table = torch.arange(80, dtype=torch.int32, device="cuda").view(1, 80)
    lens = torch.tensor([1200], dtype=torch.int32, device="cuda")
    q = torch.from_numpy(rng.standard_normal((1, 4, 64)).astype(np.float32)).cuda()
    w, p = torch.zeros_like(cache.weight), torch.zeros_like(cache.position)
    INT, MX, DUAL = sdq.Config.int_family(), sdq.Config.mx_family(), sdq.Config.dual_family()
    M, N, K = 33, 96, 8192
    X = torch.from_numpy(synth.make_x(2, M, K)).cuda()
    blob, mx, dual = (torch.from_numpy(sdq.pack(synth.make_w(2, 0, N, K), c)).cuda() for c in (INT, MX, DUAL))
    Xq, s_a = sdq.quantize_act(X, INT)
    D = sdq.quantize_act_dual(X, DUAL)
    assert sdq.gemm_workspace_size(INT, M, N, K) > 0
    return {
        "qkv_append": lambda st: sdq.qkv_append(qkv, pos, slot, cache, 4, stream=st),
        "attn_decode": lambda st: sdq.attn_decode(q, cache, table, lens, weight_out=w, stream=st),
        "cache_evict": lambda st: sdq.cache_evict(cache, table, lens, 5000, stream=st, weight_out=w, position_out=p),
        "quantize_act": lambda st: sdq.quantize_act(X, INT, stream=st),
        "gemm": lambda st: sdq.gemm(Xq, s_a, blob, N, K, INT, stream=st),
        "linear": lambda st: sdq.linear(X, blob, N, K, INT, stream=st),
        "dual": lambda st: sdq.gemm_dual(*D, dual, N, K, DUAL, stream=st),
        "quantize_act_dual": lambda st: sdq.quantize_act_dual(X, DUAL, stream=st),
        "unpack_weights": lambda st: sdq.unpack_weights(mx, N, K, MX, stream=st),
    }


CALLS = ["qkv_append", "attn_decode", "cache_evict", "quantize_act", "gemm", "linear", "dual", "quantize_act_dual", "unpack_weights"]


def _flat(x):
    return list(x) if isinstance(x, tuple) else [x]


@pytest.mark.parametrize("name", CALLS)
@pytest.mark.parametrize("foreign", [False, True])
def test_fresh_memory_is_the_streams_own(name, foreign, monkeypatch):
    torch = torch_cuda()
    import paper_2406_13868_amd as sdq

    say("memory of a call on another stream", name)
    call = _calls(torch, sdq)[name]
    torch.cuda.synchronize()
    side = torch.cuda.Stream()

    class Handle:  # another library's stream
        cuda_stream = side.cuda_stream

    on, empty = [], torch.empty

    def record(*a, **k):
        on.append(torch.cuda.current_stream().cuda_stream)
        return empty(*a, **k)

    monkeypatch.setattr(torch, "empty", record)
    got = call(Handle() if foreign else side)
    assert on and set(on) == {side.cuda_stream}
    torch.cuda.synchronize()
    on.clear()
    want = call(None)
    assert on and set(on) == {torch.cuda.current_stream().cuda_stream}
    on.clear()
    call(torch.cuda.current_stream())
    assert on and set(on) == {torch.cuda.current_stream().cuda_stream}
    monkeypatch.undo()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(_flat(got), _flat(want)))


def test_an_output_outlives_what_the_current_stream_still_reads():
    torch = torch_cuda()
    import paper_2406_13868_amd as sdq

    say("output of a call on another stream")
    X = torch.from_numpy(synth.make_x(2, 64, 4096)).cuda()
    cfg = sdq.Config.int_family()
    want = sdq.quantize_act(X, cfg)[0].clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got, scales = sdq.quantize_act(X, cfg, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    ptr = got.data_ptr()
    torch.cuda._sleep(100_000_000)  # cycles; the copy waits behind it
    copy = got.clone()
    del got
    with torch.cuda.stream(side):
        other = torch.full((64, 4096), 77, dtype=torch.uint8, device="cuda")
    assert not torch.cuda.current_stream().query(), "the current stream should still be asleep"
    assert other.data_ptr() != ptr
    torch.cuda.synchronize()
    assert torch.equal(copy, want)
