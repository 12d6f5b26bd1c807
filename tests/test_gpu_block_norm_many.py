"""GPU: block_norm of many rows, bit for bit against the stepwise oracle: the forms that 512 rows and more take, and
workgroups that take one row after the other, the next one on its way."""
import pytest

from block_util import equal
from gpu_util import say, torch_cuda
from oracle import block as O
from test_gpu_block_norm import call, case, check

pytestmark = pytest.mark.gpu

# residual, y, gate and its type (None: y's own), norm of y, layer norm, output, in place, elements between rows
KINDS = [
    ("bf16", "bf16", "channel", None, True, False, "int8", True, 0),
    ("f32", "bf16", "full", None, True, True, "f32", False, 0),
    ("bf16", "f32", "full", "bf16", True, False, "e4m3", False, 24),
    ("f32", "f32", "token", None, False, True, "bf16", True, 8),
    ("f32", None, None, None, False, True, "int8", False, 0),
    ("bf16", "bf16", "channel", "f32", True, True, "e4m3", True, 16),
    ("bf16", "f32", "full", None, False, False, "int8", True, 0),
]


def run(torch, sdq, M, K, kind):
    x, y, gate, gate_type, post, layer, out, in_place, gap = kind
    say(M, K, *kind)
    c = case(torch, M + K, M, K, x, y, gate, post, layer, gap)
    if gate_type:
        c["gate"] = c["gate"].to({"f32": torch.float32, "bf16": torch.bfloat16}[gate_type])
        c["gate_h"] = c["gate"].float().cpu().numpy()
    kw = dict(residual_out=c["residual"]) if in_place else {}
    check(torch, c, call(sdq, c, out_dtype=out, **kw), out)


# Rows that the workgroups take at once: 4096 of a wave each, 4096 by waves of a row where more share it; three turns of
# some here.  At 8200 and more the rms norm's rows go to 1024 threads, the layer norm's and those of an fp32 block to 512.
@pytest.mark.parametrize("M,K", [(8195, 72), (8195, 520), (4099, 1032), (2051, 2056), (1027, 4104), (1027, 8200)])
@pytest.mark.parametrize("kind", KINDS, ids=range(len(KINDS)))
def test_rows_in_turn(M, K, kind):
    torch = torch_cuda()
    import paper_2406_13868_amd as sdq
    run(torch, sdq, M, K, kind)


# Widths that fill their threads.
@pytest.mark.parametrize("M,K", [(4099, 512), (4099, 1024), (2053, 2048), (1029, 4096), (517, 8192), (517, 16384), (259, 16384)])
def test_whole_widths(M, K):
    torch = torch_cuda()
    import paper_2406_13868_amd as sdq
    for kind in KINDS[:2]:
        run(torch, sdq, M, K, kind)


# Both sides of 512 rows, from where on fewer threads share a row.
@pytest.mark.parametrize("M", [511, 512])
@pytest.mark.parametrize("K", [512, 520, 1032, 2056, 4104, 8200, 16392])
def test_both_sides_of_many(M, K):
    torch = torch_cuda()
    import paper_2406_13868_amd as sdq
    run(torch, sdq, M, K, KINDS[(K // 8 + M) % len(KINDS)])


@pytest.mark.parametrize("M,K", [(8195, 520), (2051, 2056), (515, 8200)])
def test_only_the_stream_in_turn(M, K):
    """Without n: no sum at all between the rows, or one."""
    torch = torch_cuda()
    import paper_2406_13868_amd as sdq
    for post in (False, True):
        say(M, K, post)
        c = case(torch, K, M, K, "bf16", "bf16", "full", post)
        r, n, s = sdq.block_norm(c["residual"], c["y"], post_weight=c["post_weight"], gate=c["gate"], residual_out=c["residual"])
        assert n is None and s is None
        want = O.stream_steps(c["residual_h"], c["y_h"], c["gate_h"], 1.0, c["post_weight_h"])
        assert equal(r.float().cpu().numpy(), torch.from_numpy(want).bfloat16().float().numpy())


def test_rows_in_turn_replayed_on_another_stream():
    """Captured, and replayed beside eager calls."""
    torch = torch_cuda()
    import paper_2406_13868_amd as sdq
    M, K = 2051, 2056
    say(M, K)
    c = case(torch, 3, M, K, "bf16", "bf16", "full", True)
    out, scales, r = torch.empty((M, K), dtype=torch.uint8, device="cuda"), torch.empty(M, device="cuda"), torch.empty_like(c["residual"])
    kw = dict(out_dtype="int8", out=out, scales=scales, residual_out=r)
    call(sdq, c, **kw)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(sdq, c, **kw)
    side = torch.cuda.Stream()
    for k in range(3):
        c["y"].mul_(0.5)
        want = call(sdq, c, out_dtype="int8", residual_out=torch.empty_like(r))
        for t in (out, scales, r):
            t.zero_()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            graph.replay()
        torch.cuda.current_stream().wait_stream(side)
        assert all(torch.equal(a, b) for a, b in zip((r, out, scales), want)), k
    c["y_h"] = c["y"].float().cpu().numpy()
    check(torch, c, (r, out, scales), "int8")
