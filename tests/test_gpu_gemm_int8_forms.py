"""GPU: every form of the dense int8 product, undivided and with K divided over workgroups, against exact sums.
tests/test_block_dispatch.py holds each size to the form that it is here for."""
import pytest

from gpu_util import say, torch_cuda

pytestmark = pytest.mark.gpu

# (M, N, K): the form and the parts of K.  Depths end on a chunk of 128 bytes, 16 past one and 16 short of one; a last
# part is as long as the others, shorter, and one or two chunks; rows and outputs end inside a tile.
UNDIVIDED = {
    (258, 17201, 128): "tile 128x128 in pairs", (262, 16613, 144): "tile 128x128 in pairs", (300, 17300, 2032): "tile 128x128 in pairs",
    (2316, 3208, 2048): "tile 128x128 in pairs", (72, 16393, 256): "tile 128x128", (68, 16856, 1040): "tile 128x128",
    (18, 16406, 384): "tile 64x128 in pairs", (19, 16485, 1136): "tile 64x128 in pairs",
}
DIVIDED = {
    (33, 33, 12816): ("tile 64x64 in pairs", 11), (40, 32, 21760): ("tile 64x64 in pairs", 13),
    (2752, 65, 6016): ("tile 64x128 in pairs", 5), (36, 2353, 20112): ("tile 64x128 in pairs", 13), (67, 2889, 4272): ("tile 64x128 in pairs", 5),
    (65, 2744, 15360): ("tile 128x128", 11), (65, 3570, 8224): ("tile 128x128", 9), (68, 2717, 9152): ("tile 128x128", 11),
    (71, 8434, 9728): ("tile 128x128 in pairs", 7), (67, 8561, 9664): ("tile 128x128 in pairs", 7), (66, 8314, 8912): ("tile 128x128 in pairs", 7),
    (3646, 65, 28032): ("tile 256x128", 16), (2693, 130, 15856): ("tile 256x128", 11), (133, 5847, 6976): ("tile 256x128", 5),
    (3794, 133, 30976): ("tile 256x192", 16), (3856, 159, 28912): ("tile 256x192", 16), (3782, 135, 21712): ("tile 256x192", 16),
    (130, 5568, 20736): ("tile 256x256", 11), (130, 6668, 14608): ("tile 256x256", 9),
    (129, 13539, 15872): ("tile 256x384", 7), (132, 11039, 17392): ("tile 256x384", 8), (131, 13246, 17264): ("tile 256x384", 7),
}


def data(torch, seed, M, N, K):
    """Codes with others between the rows, where N is odd; scales and a bias."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    gap = 16 * (N % 2)
    x, w = (torch.randint(-128, 128, (n, K + gap), generator=g, device="cuda", dtype=torch.int8)[:, :K] for n in (M, N))
    sx, sw, b = (torch.rand(n, generator=g, device="cuda") / 100 + 0.005 for n in (M, N, N))
    return x, sx, w, sw, b * 3e4


def expected(x, sx, w, sw, b, dt):
    """Sums of products of codes are exact in fp64 (below 2^31), and each later step is one fp32 operation."""
    return ((x.double() @ w.double().t()).float() * sx[:, None] * sw + b).to(dt)


@pytest.mark.parametrize("M,N,K", list(UNDIVIDED))
def test_undivided(M, N, K):
    torch = torch_cuda()
    import paper_2406_13868_amd as sdq
    for dt in (torch.float32, torch.bfloat16):
        say(M, N, K, UNDIVIDED[M, N, K], dt)
        x, sx, w, sw, b = data(torch, K, M, N, K)
        big = torch.full((M + 1, N + 3), 7.0, dtype=dt, device="cuda")
        y = sdq.gemm_int8(x, sx, w, sw, bias=b, out=big[:M, :N])
        assert torch.equal(y, expected(x, sx, w, sw, b, dt))
        assert (big[M:] == 7).all() and (big[:, N:] == 7).all()


@pytest.mark.parametrize("M,N,K", list(DIVIDED))
def test_divided(M, N, K):
    """The workspace holds NaN bits before and nothing behind it is touched."""
    torch = torch_cuda()
    import paper_2406_13868_amd as sdq
    name, parts = DIVIDED[M, N, K]
    need = sdq.gemm_int8_workspace_size(M, N, K)
    x, sx, w, sw, b = data(torch, K, M, N, K)
    for dt in (torch.float32, torch.bfloat16):
        say(M, N, K, name, parts, dt)
        ws = torch.full((need + 64,), 0xFF, dtype=torch.uint8, device="cuda")
        big = torch.full((M + 1, N + 3), 7.0, dtype=dt, device="cuda")
        y = sdq.gemm_int8(x, sx, w, sw, bias=b, out=big[:M, :N], workspace=ws[:need])
        assert torch.equal(y, expected(x, sx, w, sw, b, dt))
        assert (ws[need:] == 0xFF).all() and (big[M:] == 7).all() and (big[:, N:] == 7).all()
