"""GPU: a feed-forward block whose second product divides its depth, with a workspace that the binding makes itself,
captured and replayed."""
import numpy as np
import pytest

from gpu_util import say, torch_cuda
from test_gpu_block_run import Block, _check

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("M,width,hidden", [(64, 512, 8192), (40, 320, 6176)])
@pytest.mark.parametrize("given", [False, True])
def test_a_captured_block_with_a_divided_product(M, width, hidden, given):
    torch = torch_cuda()
    import paper_2406_13868_amd as sdq
    say(M, width, hidden, given)
    b = Block(torch, sdq, M, width, hidden, 1, given=given)
    assert sdq.gemm_int8_workspace_size(M, width, hidden) > 0
    _check(b, b())
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = b()
    for k in range(4):
        b.x.copy_(torch.from_numpy(np.random.default_rng(k).standard_normal((M, width)).astype(np.float32)) * (k + 1))
        for t in held.values():
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        replayed = {n: t.clone() for n, t in held.items()}
        eager = {n: t.clone() for n, t in b().items()}
        torch.cuda.synchronize()
        assert all(torch.equal(replayed[n], eager[n]) for n in eager), k
