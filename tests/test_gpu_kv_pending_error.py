"""GPU: an error that an earlier HIP call left pending is not reported by the
cache operators, as for the library's other device entry points."""
import ctypes

import pytest

from gpu_util import torch_cuda

pytestmark = pytest.mark.gpu


def test_a_pending_error_is_not_the_calls_own():
    torch = torch_cuda()
    import paper_2406_13868_amd as sdq

    sdq._lib.lib()
    hip = ctypes.CDLL(next(iter(sdq._lib._hip_runtimes())))
    cache = sdq.KVCache.empty(4, 2, 16, 64, track=True)
    qkv = torch.randn((3, 6 * 64), device="cuda")
    table = torch.tensor([[0, 1], [2, 3]], dtype=torch.int32, device="cuda")
    lens = torch.tensor([30, 3], dtype=torch.int32, device="cuda")
    pos, slot = torch.arange(3, dtype=torch.int32, device="cuda"), torch.tensor([5, 20, 40], device="cuda")
    q, out = torch.randn((2, 2, 64), device="cuda"), torch.empty((2, 2, 64), device="cuda")
    q_new, new = torch.empty((3, 2, 64), device="cuda"), torch.empty_like(lens)
    ws = torch.empty(sdq.attn_decode_workspace_size(cache, 2, 2, 32) + sdq.cache_evict_workspace_size(cache, 2, 32, 8),
                     dtype=torch.uint8, device="cuda")
    # nothing but the library's launches between the error and the check
    calls = [lambda: sdq.qkv_append(qkv, pos, slot, cache, 2, out=q_new),
             lambda: sdq.attn_decode(q, cache, table, lens, out=out, workspace=ws),
             lambda: sdq.cache_evict(cache, table, lens, 8, lens_out=new, workspace=ws)]
    for call in calls:
        want = call().clone()
        torch.cuda.synchronize()
        hip.hipGetLastError()
        assert hip.hipSetDevice(ctypes.c_int(1 << 20)) != 0 and hip.hipPeekAtLastError() != 0
        got = call()
        assert hip.hipPeekAtLastError() == 0
        torch.cuda.synchronize()
        assert torch.equal(got, want)
