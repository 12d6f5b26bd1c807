"""GPU: glu_act against its definition in 64 bits."""
import numpy as np
import pytest

from block_util import codes_near, equal, placed
from gpu_util import say, torch_cuda
from oracle import block as O

pytestmark = pytest.mark.gpu

# h is evaluated within 1e-13 of itself and rounded to fp32 once (or to zero below its least number)
REL, ABS = O.U * (1 + 1e-6), 2.0 ** -149


def check(torch, x_h, act, gated, got, out):
    n, s = got
    h = O.activation64(x_h, act, gated)
    if out in ("int8", "e4m3"):
        codes_near(n.cpu().numpy(), s.cpu().numpy(), h, out, REL)
        return
    assert s is None

    bound = (2.0 ** -8 if out == "bf16" else 0) * np.abs(h) + REL * np.abs(h) + (2.0 ** -133 if out == "bf16" else ABS)
    assert (np.abs(n.double().cpu().numpy() - h) <= bound).all()


@pytest.mark.parametrize("F", [8, 16, 1032, 2048, 2056, 4096, 4104, 8192, 11008, 16392, 32768, 32776, 41000])
def test_every_width(F):
    torch = torch_cuda()
    import paper_2406_13868_amd as sdq
    for i, (M, out) in enumerate(((1, "int8"), (3, "e4m3"), (2, "f32"), (5, "int8"), (2, "bf16"))):
        act, gated, dt = ["silu", "gelu", "relu"][(i + F // 8) % 3], i % 2 == 0, [torch.float32, torch.bfloat16][(i + F // 8) % 2]
        say(F, M, out, act, gated, dt)
        rng = np.random.default_rng(F + i)
        x, x_h = placed(torch, rng.standard_normal((M, 2 * F if gated else F)) * 2, dt, gap=8 * (i % 3))
        check(torch, x_h, act, gated, sdq.glu_act(x, act, gated=gated, out_dtype=out), out)


@pytest.mark.parametrize("act", ["silu", "gelu", "relu"])
@pytest.mark.parametrize("out", ["int8", "e4m3", "f32", "bf16"])
@pytest.mark.parametrize("x", ["f32", "bf16"])
@pytest.mark.parametrize("gated", [False, True])
def test_every_kind(act, out, x, gated):
    torch = torch_cuda()
    import paper_2406_13868_amd as sdq
    say(act, out, x, gated)
    rng = np.random.default_rng(9)
    x, x_h = placed(torch, rng.standard_normal((131, 328 * (1 + gated))) * 3, {"f32": torch.float32, "bf16": torch.bfloat16}[x], gap=40)
    check(torch, x_h, act, gated, sdq.glu_act(x, act, gated=gated, out_dtype=out), out)


@pytest.mark.parametrize("act", ["silu", "gelu", "relu"])
def test_the_whole_range_of_arguments(act):
    """From the least numbers to where exp leaves fp64's range."""
    torch = torch_cuda()
    import paper_2406_13868_amd as sdq
    rng = np.random.default_rng(2)
    size = np.concatenate([10.0 ** rng.uniform(-44, 38, 4000), rng.uniform(0, 120, 8000), rng.uniform(600, 800, 200), [0.0, 88.7, 709.8, 3e38, 1.0, 104, 0, 0]])
    v = (size * np.where(rng.random(size.size) < 0.5, -1, 1)).astype(np.float32)[None, : size.size // 8 * 8]
    x, x_h = placed(torch, v, torch.float32)
    got, _ = sdq.glu_act(x, act, gated=False, out_dtype="f32")
    h = O.activation64(x_h, act, False)
    off = np.abs(got.double().cpu().numpy() - h)
    assert (off <= REL * np.abs(h) + ABS).all(), (x_h[0][np.argmax(off - REL * np.abs(h))], off.max())


def test_values_that_are_not_finite():
    torch = torch_cuda()
    import paper_2406_13868_amd as sdq
    for F in (64, 40960):
        x = torch.ones((4, 2 * F), device="cuda")
        x[0, 3], x[1, 5], x[2, F + 7] = float("nan"), float("inf"), float("-inf")
        for act in ("silu", "gelu", "relu"):
            for out in ("int8", "e4m3"):
                q, s = sdq.glu_act(x, act, out_dtype=out)
                assert not s[:3].isfinite().any() and s[3].isfinite() and (q[:3] == 0).all() and (q[3] != 0).all()
            h, _ = sdq.glu_act(x, act, out_dtype="f32")
            assert h[0, 3].isnan() and h[1, 5] == float("inf") and h[2, 7] == float("-inf") and int((~h.isfinite()).sum()) == 3
    z, s = sdq.glu_act(torch.zeros((2, 128), device="cuda"), "silu", out_dtype="int8")
    assert (z == 0).all() and (s == 0).all()


def test_given_outputs_and_calls_that_are_refused():
    torch = torch_cuda()
    import paper_2406_13868_amd as sdq
    x = torch.randn((3, 128), device="cuda")
    q, s = torch.full((5, 64), 77, dtype=torch.uint8, device="cuda"), torch.full((5,), -1.0, device="cuda")
    got = sdq.glu_act(x, out_dtype="int8", out=q[:3], scales=s[:3])
    check(torch, x.cpu().numpy(), "silu", True, got, "int8")
    assert (q[3:] == 77).all() and (s[3:] == -1).all() and got[0].data_ptr() == q.data_ptr()
    y = torch.full((5, 64), 9.0, device="cuda")
    sdq.glu_act(x, out=y[:3])
    check(torch, x.cpu().numpy(), "silu", True, (y[:3], None), "f32")
    assert (y[3:] == 9).all()
    e, s0 = sdq.glu_act(x[:0], out_dtype="int8")
    assert e.shape == (0, 64) and s0.shape == (0,)

    def refused(match, *a, **kw):
        with pytest.raises((ValueError, sdq.SDQError), match=match):
            sdq.glu_act(*a, **kw)

    refused("act must be", x, "swish")
    refused("two parts", x[:, :127])
    refused("float32 or bfloat16", x.half())
    refused("SHAPE", x[:, :120])
    refused("SHAPE", x[:, 1:], gated=False)
    refused("contiguous", x.t())
    refused("out must be", x, out_dtype="int8", out=q)
    refused("scales must be", x, out_dtype="int8", scales=s)
    refused("scales belong", x, scales=s[:3])
    assert equal(q.cpu().numpy()[3:], np.full((2, 64), 77, np.uint8))
