"""GPU: the decode example runs the projections, the append, attention and eviction
together; its attention is held to the oracle over the slots that the cache says
it holds."""
import dataclasses
import os
import sys

import numpy as np
import pytest

from gpu_util import say, torch_cuda
from kv_util import BF16_U, E4M3_U
from oracle import decode as O

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kv, budget, recent", [("bf16", 0, 0), ("e4m3", 0, 0), ("bf16", 20, 6), ("e4m3", 17, 17)])
def test_steps(kv, budget, recent):
    torch = torch_cuda()
    import decode_attention as example
    import paper_2406_13868_amd as sdq
    import synth

    say("example", kv, budget, recent)
    width, hq, hkv, D, B, tokens = 256, 8, 4, 64, 3, 40
    cfg = dataclasses.replace(sdq.Config.of(synth.INT_1x8_E4M3_3x8), y_dtype="bf16")
    block = example.Attention(cfg, width, hq, hkv, D, B, tokens, page_size=16, kv=kv, budget=budget, recent=recent)
    angles = block.cos_sin.cpu().numpy()
    rng = np.random.default_rng(budget)
    history = []
    kv_u = BF16_U if kv == "bf16" else E4M3_U
    for step in range(tokens):
        held = [block.cache.position.cpu().numpy() if budget else None, [list(p) for p in block.pages.held], list(block.lens)]
        x = torch.from_numpy(rng.standard_normal((B, width)).astype(np.float32)).to("cuda")
        got = block.step(x)
        torch.cuda.synchronize()
        qkv = got["qkv"].float().cpu().numpy().reshape(B, hq + 2 * hkv, D)
        history.append(qkv)
        q, out = (got[n].float().cpu().numpy().astype(np.float64) for n in ("q", "attention"))
        for b in range(B):
            for h in range(hkv):
                if budget:  # what the cache held before the step, and the step's own token
                    t = np.arange(held[2][b])
                    pages = np.array(held[1][b] + [0])[t // 16]
                    at = list(held[0][pages, h, t % 16]) + [step]
                else:
                    at = list(range(step + 1))
                assert len(set(at)) == len(at) and max(at) == step
                if budget and step >= recent:
                    assert set(range(step - recent + 1, step + 1)) <= set(at)
                k = np.stack([O.transform(history[p][b, hq + h], None, 0, angles[p], False)[0] for p in at])
                v = np.stack([history[p][b, hq + hkv + h] for p in at])
                g = hq // hkv
                ref = O.attend(q[b, h * g:(h + 1) * g], k, v, D ** -0.5)
                # the cache's rounding of keys moves a score by its share of sum |q k|, a
                # probability by twice that; values and outputs are rounded once
                # (1.1: second order, fp32, and codes below the smallest normal one)
                tol = 1.1 * ((2 * kv_u * ref["score_size"] + kv_u)[:, None] * ref["out_size"] + BF16_U * np.abs(ref["out"])) + 1e-6
                if kv == "e4m3":
                    tol = tol + 2.0 ** -9 / 448 * np.abs(v).max()
                assert np.all(np.abs(out[b, h * g:(h + 1) * g] - ref["out"]) <= tol), (step, b, h)
        want = min(step + 1, budget) if budget else step + 1
        assert block.lens == [want] * B and block.lens_gpu.tolist() == block.lens
        assert [len(p) for p in block.pages.held] == [-(-want // 16)] * B
        assert torch.isfinite(got["y"].float()).all()


def test_the_command_runs(capsys):
    torch_cuda()
    import decode_attention as example

    example.main(["--width", "256", "--heads", "4", "--heads-kv", "2", "--dim", "64", "--sequences", "2", "--tokens", "20", "--kv", "e4m3",
                  "--budget", "16", "--recent", "4"])
    assert "slots held [16, 16]" in capsys.readouterr().out
