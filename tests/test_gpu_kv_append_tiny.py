"""GPU: e4m3 rows so small that 448 / amax is past fp32's range keep their size."""
import numpy as np
import pytest

from gpu_util import say, torch_cuda
from kv_util import E4M3_U
from oracle import decode as O
from oracle import formats as F

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("x", ["f32", "bf16"])
@pytest.mark.parametrize("D", [16, 128, 256])
def test_tiny_rows(D, x):
    torch = torch_cuda()
    import paper_2406_13868_amd as sdq

    say("tiny rows", D, x)
    rng = np.random.default_rng(D)
    sizes = [1e-25, 2.0 ** -90, 2.0 ** -91, 1e-30, 1.4e-36, 1.3e-36, 1e-37, 3e-38, 1e-38, 1e-39, 1e-41, 1e-45, 0.0]
    rows = rng.uniform(-1, 1, (len(sizes), 2, D)) * np.array(sizes)[:, None, None]
    rows[:, :, 3], rows[:, :, 5] = 0, np.array(sizes)[:, None]  # a zero, and the largest
    q = np.ones((len(sizes), D))
    t = torch.from_numpy(np.concatenate([q, rows.reshape(len(sizes), -1)], 1).astype(np.float32))
    t = t.to(torch.bfloat16) if x == "bf16" else t
    rows = t.float().numpy()[:, D:].reshape(len(sizes), 2, D)
    cache = sdq.KVCache.empty(1, 1, len(sizes), D, "e4m3")
    sdq.qkv_append(t.cuda(), None, torch.arange(len(sizes), device="cuda"), cache, 1)
    for which, (codes, scales) in enumerate(((cache.k, cache.k_scale), (cache.v, cache.v_scale))):
        codes, scales = codes[0, 0].float().cpu().numpy().astype(np.float64), scales[0, 0].cpu().numpy()
        for m, size in enumerate(sizes):
            y = rows[m, which]
            want, s = O.quantize_row(y)
            assert scales[m] == s and np.array_equal(codes[m], F.e4m3_decode(want)), (size, which)
            assert codes[m, 3] == 0
            # half a step of a code, or of the smallest ones, and the scale's own
            # rounding, which is absolute among subnormal numbers
            tol = E4M3_U * np.abs(y.astype(np.float64)) * 1.001 + 2.0 ** -10 * float(s) + 448 * 2.0 ** -150
            assert np.all(np.abs(codes[m] * float(s) - y) <= tol), (size, which)
