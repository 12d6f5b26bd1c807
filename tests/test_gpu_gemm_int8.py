"""GPU: the dense int8 product against exact integer sums."""
import numpy as np
import pytest

from block_util import equal, rounded
from gpu_util import say, torch_cuda
from oracle import block as O

pytestmark = pytest.mark.gpu


def make(torch, seed, M, N, K, x_gap=0, w_gap=0, least=-127, bias=True):
    """Codes with other codes between the rows, scales and a bias, on the GPU and the host."""
    rng = np.random.default_rng(seed)
    x, w = rng.integers(least, 128, (M, K + x_gap)).astype(np.int8), rng.integers(least, 128, (N, K + w_gap)).astype(np.int8)
    sx, sw, b = (rng.uniform(0.5, 2, n).astype(np.float32) / 100 for n in (M, N, N))
    b = b * 1000 if bias else None
    g = [torch.from_numpy(t).cuda() for t in (x, sx, w, sw)]
    return (g[0][:, :K], g[1], g[2][:, :K], g[3]), None if b is None else torch.from_numpy(b).cuda(), (x[:, :K], sx, w[:, :K], sw), b


def steps(host, b):
    """fp32(sum) * s_x * s_w + bias, an fp32 operation each: the result's every bit."""
    _, total = O.product64(*host)
    y = total.astype(np.float32) * host[1][:, None] * host[3]
    return y if b is None else y + b


def check(torch, sdq, seed, M, N, K, dtype=None, **kw):
    say(M, N, K, dtype, kw)
    args, bias, host, b = make(torch, seed, M, N, K, **kw)
    y = sdq.gemm_int8(*args, bias=bias, out_dtype=dtype)
    want = steps(host, b)
    assert y.shape == (M, N) and equal(y.float().cpu().numpy(), rounded(torch, want, y.dtype)), (M, N, K)
    y64, _ = O.product64(*host, b)
    size = np.abs(y64 - (0 if b is None else b)) * 3 + np.abs(y64)  # the sum's rounding and two products', and the bias's
    assert (np.abs(want - y64) <= 1.01 * O.U * size).all()


@pytest.mark.parametrize("M", [1, 2, 3, 4, 5, 7, 8, 9, 15, 16, 17, 31, 32, 33, 48, 63, 64, 65, 96, 127, 128, 129, 191, 256, 257, 300])
def test_every_number_of_tokens(M):
    torch = torch_cuda()
    import paper_2406_13868_amd as sdq
    check(torch, sdq, M, M, 200, 400)
    check(torch, sdq, M, M, 77, 1104, torch.bfloat16, x_gap=16, w_gap=32)


@pytest.mark.parametrize("K", [16, 32, 48, 64, 112, 128, 144, 240, 256, 272, 368, 512, 528, 1008, 1024, 1040, 2032, 2048, 2064, 4080, 4096, 4112, 8208])
def test_every_kind_of_depth(K):
    torch = torch_cuda()
    import paper_2406_13868_amd as sdq
    for M, N in ((1, 33), (3, 64), (9, 130), (40, 65), (140, 257)):
        check(torch, sdq, K, M, N, K, [torch.bfloat16, torch.float32][K // 16 % 2], bias=M % 2 == 0)


@pytest.mark.parametrize("N", [1, 2, 3, 4, 5, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 255, 256, 257, 1000, 1023])
def test_every_number_of_outputs(N):
    torch = torch_cuda()
    import paper_2406_13868_amd as sdq
    for M in (1, 6, 20, 70, 260):
        check(torch, sdq, N, M, N, 272, [torch.bfloat16, torch.float32][M % 2])


@pytest.mark.parametrize("M,N,K", [(1, 4096, 4096), (4, 4096, 4096), (16, 4096, 4096), (64, 4096, 4096), (200, 4096, 4096), (517, 5003, 1104),
                                   (1024, 2048, 4096), (2100, 1300, 272)])
def test_sizes_that_fill_the_gpu(M, N, K):
    torch = torch_cuda()
    import paper_2406_13868_amd as sdq
    check(torch, sdq, 11, M, N, K, torch.bfloat16)


@pytest.mark.parametrize("M", [1, 8, 24, 130])
def test_the_largest_sums_are_exact(M):
    """All codes -128 over the longest K: 2^14 times it, just below 2^31; and sums past 2^24, which fp32 rounds."""
    torch = torch_cuda()
    import paper_2406_13868_amd as sdq
    K = (1 << 17) - 16
    say(M, K)
    for a, b in ((-128, -128), (-128, 127), (127, 127)):
        x = torch.full((M, K), a, dtype=torch.int8, device="cuda")
        w = torch.full((35, K), b, dtype=torch.int8, device="cuda")
        x[:, 5] += 1 if a < 0 else -1
        y = sdq.gemm_int8(x, torch.ones(M, device="cuda"), w, torch.ones(35, device="cuda"))
        total = K * a * b + (b if a < 0 else -b)
        assert (y.cpu().numpy() == np.float32(total)).all() and abs(total) < 2 ** 31


def check_on_gpu(torch, M, N, K):
    """The sums are exact in fp64 too, and each later step is one fp32 operation."""
    import paper_2406_13868_amd as sdq
    dt = [torch.bfloat16, torch.float32][K // 16 % 2]
    say(M, N, K, dt)
    (x, sx, w, sw), bias, _, _ = make(torch, K, M, N, K, x_gap=16 * (N % 2), bias=K % 128 != 0)
    y = sdq.gemm_int8(x, sx, w, sw, bias=bias, out_dtype=dt)
    want = (x.double() @ w.double().t()).float() * sx[:, None] * sw
    if bias is not None:
        want = want + bias
    assert torch.equal(y, want.to(dt))


@pytest.mark.parametrize("K", [16, 112, 128, 144, 256, 272, 384, 400, 528, 1296])
@pytest.mark.parametrize("M,N", [(1025, 18003), (700, 30005), (3900, 4090), (255, 33000), (2040, 4005)])
def test_the_largest_tiles(M, N, K):
    """256 tokens by 128 to 384 outputs a workgroup, with rows, outputs and depths that end inside a tile."""
    check_on_gpu(torch_cuda(), M, N, K)


@pytest.mark.parametrize("K", [16, 144, 640, 1040, 1168])
@pytest.mark.parametrize("N", [4096, 4097, 5003, 8192, 11001, 12288, 12289, 16370, 22013, 33001])
def test_few_tokens_by_many_outputs(N, K):
    """Tiles of 16 to 64 outputs, one or several a workgroup, the last one short."""
    for M in (1, 8, 9, 16, 30):
        check_on_gpu(torch_cuda(), M, N, K)


DIVIDED = [(64, 4096, 16384), (100, 300, 8208), (40, 37, 13456), (130, 1000, 8192), (33, 4, 4096), (600, 601, 6000)]


@pytest.mark.parametrize("M,N,K", DIVIDED)
def test_products_divided_over_their_depth(M, N, K):
    """With a workspace, which holds NaN bits before; without one the same bits."""
    torch = torch_cuda()
    import paper_2406_13868_amd as sdq
    from paper_2406_13868_amd import _lib, block
    need = sdq.gemm_int8_workspace_size(M, N, K)
    parts = need // (4 * M * N)
    assert parts > 1 and need == 4 * M * N * parts
    for dt in (torch.float32, torch.bfloat16):
        say(M, N, K, parts, dt)
        args, bias, host, b = make(torch, M, M, N, K, x_gap=16 * (N % 2))
        ws = torch.full((need + 64,), 0xFF, dtype=torch.uint8, device="cuda")
        big = torch.full((M + 1, N + 5), 7.0, dtype=dt, device="cuda")
        y = sdq.gemm_int8(*args, bias=bias, out=big[:M, :N], workspace=ws[:need])
        assert equal(y.float().cpu().numpy(), rounded(torch, steps(host, b), dt))
        assert (ws[need:] == 0xFF).all() and (big[M:] == 7).all() and (big[:, N:] == 7).all()
        assert torch.equal(sdq.gemm_int8(*args, bias=bias, out_dtype=dt), y)
        if not args[0].is_contiguous():
            continue
        z = torch.empty((M, N), dtype=dt, device="cuda")
        call = _lib.sdq_int8_args(xq=args[0].data_ptr(), wq=args[2].data_ptr(), s_x=args[1].data_ptr(), s_w=args[3].data_ptr(),
                                  bias=bias.data_ptr(), y=z.data_ptr(), M=M, N=N, K=K, x_stride=K, w_stride=K, y_stride=N,
                                  y_dtype=int(dt is torch.bfloat16))
        block._run(_lib.lib().sdq_gemm_int8, bytes(call), 0, None, "sdq_gemm_int8")
        assert torch.equal(z, y)
    with pytest.raises(ValueError, match="workspace holds"):
        sdq.gemm_int8(*args, workspace=ws[: need - 16])


def test_strided_outputs_and_what_lies_beside_them():
    torch = torch_cuda()
    import paper_2406_13868_amd as sdq
    for M, N in ((1, 37), (5, 64), (30, 100), (150, 300)):
        for dt in (torch.float32, torch.bfloat16):
            say(M, N, dt)
            args, bias, host, b = make(torch, M, M, N, 160)
            big = torch.full((M + 2, N + 11), 7.0, dtype=dt, device="cuda")
            y = sdq.gemm_int8(*args, bias=bias, out=big[:M, 3:3 + N])
            assert y.data_ptr() == big[:, 3:].data_ptr()
            assert equal(y.float().cpu().numpy(), rounded(torch, steps(host, b), dt))
            big[:M, 3:3 + N] = 7
            assert (big == 7).all()


def test_codes_of_the_other_operators_and_the_scales_of_bad_rows():
    """uint8 codes as quantize_act writes them; a scale that is not finite reaches its row's outputs."""
    torch = torch_cuda()
    import paper_2406_13868_amd as sdq
    cfg = sdq.Config.int_family()
    X, W = torch.randn((9, 96), device="cuda"), torch.randn((50, 96), device="cuda")
    xq, sx = sdq.quantize_act(X, cfg)
    wq, sw = sdq.quantize_act(W, cfg)
    y = sdq.gemm_int8(xq, sx, wq, sw)
    host = [t.cpu().numpy() for t in (xq.view(torch.int8), sx, wq.view(torch.int8), sw)]
    assert equal(y.cpu().numpy(), steps(host, None))
    for M in (3, 40, 200):
        sx = torch.ones(M, device="cuda")
        sx[1] = float("nan")
        x = torch.zeros((M, 96), dtype=torch.uint8, device="cuda")
        y = sdq.gemm_int8(x, sx, wq, sw)
        assert y[1].isnan().all() and (y[[0] + list(range(2, M))] == 0).all()


def test_calls_without_rows_and_calls_that_are_refused():
    torch = torch_cuda()
    import paper_2406_13868_amd as sdq
    x, w = torch.zeros((3, 64), dtype=torch.int8, device="cuda"), torch.zeros((5, 64), dtype=torch.int8, device="cuda")
    s3, s5 = torch.ones(3, device="cuda"), torch.ones(5, device="cuda")
    assert sdq.gemm_int8(x[:0], s3[:0], w, s5).shape == (0, 5)

    def refused(match, *a, **kw):
        with pytest.raises((ValueError, sdq.SDQError), match=match):
            sdq.gemm_int8(*a, **kw)

    refused("int8 codes", x.float(), s3, w, s5)
    refused("int8 codes", x, s3, w.short(), s5)
    refused("wq must be", x, s3, w[:, :48], s5)
    refused("s_x must be", x, s5, w, s5)
    refused("s_w must be", x, s3, w, s3)
    refused("bias must be", x, s3, w, s5, bias=s3)
    refused("bias must be", x, s3, w, s5, bias=s5.double())
    refused("out must be", x, s3, w, s5, out=torch.zeros((3, 4), device="cuda"))
    refused("float32 or bfloat16", x, s3, w, s5, out_dtype=torch.float16)
    refused("SHAPE", x[:, :40], s3, w[:, :40], s5)
    refused("SHAPE", x[:, 1:49], s3, w[:, :48], s5)
    refused("contiguous", x.t().contiguous().t(), s3, w, s5)


def test_the_names_of_output_types_and_outputs_that_are_no_tensors():
    torch = torch_cuda()
    import paper_2406_13868_amd as sdq
    (x, sx, w, sw), bias, _, _ = make(torch, 1, 5, 40, 64)
    for name, dt in (("f32", torch.float32), ("bf16", torch.bfloat16)):
        y = sdq.gemm_int8(x, sx, w, sw, bias=bias, out_dtype=name)
        assert y.dtype is dt and torch.equal(y, sdq.gemm_int8(x, sx, w, sw, bias=bias, out_dtype=dt))
        assert sdq.gemm_int8(x, sx, w, sw, out=y, out_dtype=name) is y
    for out_dtype in ("int8", "e4m3", "f16", torch.float16, 3, [torch.float32]):
        with pytest.raises(ValueError, match="float32 or bfloat16"):
            sdq.gemm_int8(x, sx, w, sw, out_dtype=out_dtype)
    for out in ([1.0], x.cpu().numpy(), torch.empty((5, 40), dtype=torch.float64, device="cuda")):
        for out_dtype in (None, "bf16", torch.float32):
            with pytest.raises(ValueError, match="out must be"):
                sdq.gemm_int8(x, sx, w, sw, out=out, out_dtype=out_dtype)
