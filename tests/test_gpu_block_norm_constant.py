"""GPU: layer norms of rows that are all one number, whose differences from their mean are zero: bit for bit
against the stepwise oracle, where the definition leaves the bias alone, zero codes and a scale of zero."""
import numpy as np
import pytest

from block_util import equal, rounded
from gpu_util import say, torch_cuda
from oracle import block as O

pytestmark = pytest.mark.gpu

OUTS = ["int8", "e4m3", "f32", "bf16"]


def check(torch, got, rows, want_r, weight, bias, eps, out):
    r, n, s = got
    if want_r is not None:
        assert equal(r.float().cpu().numpy(), rounded(torch, want_r, r.dtype)), "stream"
    want = O.norm_steps(rows if want_r is None else want_r, weight, bias, eps, True)
    if out in ("int8", "e4m3"):
        codes, scales = O.codes_steps(want, out)
        assert equal(n.cpu().numpy(), codes) and equal(s.cpu().numpy(), scales), (out, s, scales)
    else:
        assert equal(n.float().cpu().numpy(), rounded(torch, want, n.dtype)), out


def values(rng, K, top):
    """Rows of one number each, large ones among them, beside ordinary rows."""
    rows = rng.standard_normal((6, K)).astype(np.float32)
    rows[0], rows[2], rows[3], rows[5] = top, -top / 3, 1.0, 0.1
    return rows


# On both sides of the widths that fill a row's threads: places past a row's end must not take part.
@pytest.mark.parametrize("K", [8, 64, 504, 512, 520, 1016, 1024, 1560, 3000, 4096, 6400, 8192, 8200, 12000, 16384, 16392])
@pytest.mark.parametrize("top", [1e36, 3e38])
def test_large_constant_rows(K, top):
    torch = torch_cuda()
    import paper_2406_13868_amd as sdq
    rng = np.random.default_rng(K)
    rows, (w, b, pw, pb) = values(rng, K, top), rng.uniform(0.5, 1.5, (4, K)).astype(np.float32)
    x, W, B, PW, PB = (torch.from_numpy(t).cuda() for t in (rows, w, b, pw, pb))
    other = rng.standard_normal((6, K)).astype(np.float32)
    res = torch.from_numpy(other).cuda()
    for out in OUTS:
        say(K, top, out)
        check(torch, sdq.block_norm(x, weight=W, layer=True, out_dtype=out), rows, None, w, None, 1e-6, out)
        check(torch, sdq.block_norm(x, weight=W, bias=B, layer=True, out_dtype=out), rows, None, w, b, 1e-6, out)
        # the block's output normed before it joins the stream
        got = sdq.block_norm(res, x, W, B, layer=True, post_weight=PW, post_bias=PB, scale=0.5, out_dtype=out)
        check(torch, got, None, O.stream_steps(other, rows, None, 0.5, pw, pb, 1e-6, True), w, b, 1e-6, out)


# Widths whose reciprocal in 64 bits times the width is not 1, in every form of the kernel, and some where it is.
@pytest.mark.parametrize("K", [64, 392, 784, 1288, 1568, 2576, 4488, 8976, 17720, 40960])
@pytest.mark.parametrize("eps", [1e-6, 1e-30])
def test_the_mean_of_a_constant_row_is_that_constant(K, eps):
    torch = torch_cuda()
    import paper_2406_13868_amd as sdq
    rows = np.repeat(np.array([1.0, -3.3, 0.1, 7e-5, 1e3, 123456.7], np.float32)[:, None], K, 1)
    w = np.ones(K, np.float32)
    x, W = torch.from_numpy(rows).cuda(), torch.from_numpy(w).cuda()
    for out in OUTS:
        say(K, eps, out)
        _, n, s = got = sdq.block_norm(x, weight=W, layer=True, eps=eps, out_dtype=out)
        assert (n == 0).all() and (s is None or (s == 0).all())
        check(torch, got, rows, None, w, None, eps, out)
        got = sdq.block_norm(torch.zeros_like(x), x, W, layer=True, post_weight=W, eps=eps, out_dtype=out)
        check(torch, got, None, O.stream_steps(np.zeros_like(rows), rows, None, 1.0, w, None, eps, True), w, None, eps, out)
