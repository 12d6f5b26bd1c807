"""GPU: glu_act of many rows to codes, in the forms that 512 rows and more take, against its definition in 64 bits."""
import numpy as np
import pytest

from block_util import placed
from gpu_util import say, torch_cuda
from test_gpu_glu_act import check

pytestmark = pytest.mark.gpu


# On both sides of the widths that the forms end at, which fill their threads.
@pytest.mark.parametrize("F", [512, 520, 1024, 1032, 2048, 2056, 4096, 4104, 8192, 8200, 16384, 16392, 32776])
@pytest.mark.parametrize("gated", [False, True])
def test_many_rows(F, gated):
    torch = torch_cuda()
    import paper_2406_13868_amd as sdq
    for i, M in enumerate((511, 512, 515)):
        act, out, dt = ["silu", "gelu", "relu"][(i + F // 8) % 3], ["int8", "e4m3"][(i + F // 8 + gated) % 2], [torch.bfloat16, torch.float32][(i + gated) % 2]
        say(M, F, gated, act, out, dt)
        rng = np.random.default_rng(F + M)
        x, x_h = placed(torch, rng.standard_normal((M, F * (1 + gated)), np.float32) * 2, dt, gap=8 * i)
        q, s = torch.full((M + 1, F), 77, dtype=torch.uint8, device="cuda"), torch.full((M + 1,), -1.0, device="cuda")
        check(torch, x_h, act, gated, sdq.glu_act(x, act, gated=gated, out_dtype=out, out=q[:M], scales=s[:M]), out)
        assert (q[M:] == 77).all() and (s[M:] == -1).all()


@pytest.mark.parametrize("F", [520, 1544, 4104, 8200])
def test_a_row_does_not_hang_on_the_others(F):
    """Each row's codes are those of a call of its own, which takes another form."""
    torch = torch_cuda()
    import paper_2406_13868_amd as sdq
    say(F)
    x = torch.randn((600, 2 * F), generator=torch.Generator(device="cuda").manual_seed(F), device="cuda").bfloat16()
    x[7, 3], x[599, F + 1], x[5] = float("nan"), float("inf"), 0
    for out in ("int8", "e4m3"):
        q, s = sdq.glu_act(x, "silu", out_dtype=out)
        for m in (0, 1, 2, 3, 4, 5, 7, 300, 598, 599):
            q1, s1 = sdq.glu_act(x[m : m + 1], "silu", out_dtype=out)
            assert torch.equal(q[m : m + 1], q1) and torch.equal(s[m : m + 1].nan_to_num(7.0, 8.0), s1.nan_to_num(7.0, 8.0))
