"""The attention half of a transformer block answering, one token per sequence at a time.

Every step runs what a served model runs between its norms: the stacked q/k/v
projection (a decomposed product, quantized per token), the rotation and the
write of the new keys and values into a paged cache, attention over the cache,
and the output projection.  Where a budget is given, attention also tracks how
much weight every cached slot receives, and a sequence that grows past the
budget is cut back to its recent and its most attended slots.

    python examples/decode_attention.py                        # LLaMA-7B's heads and width, 8 sequences, 64 tokens each
    python examples/decode_attention.py --heads-kv 8 --kv e4m3 --budget 48 --recent 16
"""
from __future__ import annotations

import argparse
import dataclasses
import os
import sys
import time

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_2406_13868_amd as sdq  # noqa: E402
import synth  # noqa: E402


def rotary_angles(positions: int, dim: int, base: float = 10000.0, device="cuda") -> torch.Tensor:
    """[positions, dim] fp32: the cosines, then the sines of the pairs' angles."""
    rate = base ** (-torch.arange(0, dim, 2, dtype=torch.float64, device=device) / dim)
    angle = torch.arange(positions, dtype=torch.float64, device=device)[:, None] * rate
    return torch.cat([angle.cos(), angle.sin()], 1).float()


class Pages:
    """Which pages each sequence holds; the page table on the GPU follows."""

    def __init__(self, sequences: int, pages: int, most: int, page_size: int, device="cuda"):
        self.free, self.page_size = list(range(pages))[::-1], page_size
        self.held = [[] for _ in range(sequences)]
        self.table = torch.full((sequences, most), -1, dtype=torch.int32, device=device)

    def resize(self, b: int, slots: int) -> None:
        held, need = self.held[b], -(-slots // self.page_size)
        while len(held) < need:
            held.append(self.free.pop())
            self.table[b, len(held) - 1] = held[-1]
        while len(held) > need:
            self.free.append(held.pop())
            self.table[b, len(held)] = -1


class Attention:
    """One block's attention: packed projections, a cache, and a step for a token of every sequence."""

    def __init__(self, cfg, width, heads_q, heads_kv, dim, sequences, max_len, page_size=64, kv="bf16", budget=0, recent=0,
                 seed=0, device="cuda"):
        self.cfg, self.width, self.heads_q, self.heads_kv, self.dim = cfg, width, heads_q, heads_kv, dim
        self.budget, self.recent, self.B = budget, recent, sequences
        self.n_qkv = (heads_q + 2 * heads_kv) * dim
        pack = lambda tensor, n, k: torch.from_numpy(sdq.pack(synth.make_w(5, tensor, n, k, seed=seed), cfg)).to(device)  # noqa: E731
        self.w_qkv, self.w_out = pack(0, self.n_qkv, width), pack(1, width, heads_q * dim)
        self.cos_sin = rotary_angles(max_len, dim, device=device)
        cap = min(max_len, budget + 1) if budget else max_len  # slots a sequence holds at once
        per = -(-cap // page_size)
        self.cap = per * page_size
        self.cache = sdq.KVCache.empty(sequences * per, heads_kv, page_size, dim, kv, track=budget > 0, device=device)
        self.pages = Pages(sequences, sequences * per, per, page_size, device)
        self.lens = [0] * sequences
        self.lens_gpu = torch.zeros(sequences, dtype=torch.int32, device=device)
        self.position = 0
        size = sdq.attn_decode_workspace_size(self.cache, sequences, heads_q, self.cap, track=budget > 0)
        if budget:
            size = max(size, sdq.cache_evict_workspace_size(self.cache, sequences, self.cap, budget))
        self.workspace = torch.empty(size, dtype=torch.uint8, device=device)

    def step(self, x: torch.Tensor) -> dict:
        """x [sequences, width]: the block's input for one new token each.  Returns the output and what led to it."""
        qkv, _, _ = sdq.linear(x, self.w_qkv, self.n_qkv, self.width, self.cfg)
        slots = []
        for b in range(self.B):
            self.pages.resize(b, self.lens[b] + 1)
            slots.append(self.pages.held[b][self.lens[b] // self.pages.page_size] * self.pages.page_size
                         + self.lens[b] % self.pages.page_size)
            self.lens[b] += 1
        slot = torch.tensor(slots, device=x.device)
        pos = torch.full((self.B,), self.position, dtype=torch.int32, device=x.device)
        q = sdq.qkv_append(qkv, pos, slot, self.cache, self.heads_q, self.cos_sin)
        self.lens_gpu += 1
        o = sdq.attn_decode(q, self.cache, self.pages.table, self.lens_gpu, weight_out=self.cache.weight if self.budget else None,
                            workspace=self.workspace)
        y, _, _ = sdq.linear(o.view(self.B, -1), self.w_out, self.width, self.heads_q * self.dim, self.cfg)
        if self.budget and max(self.lens) > self.budget:
            sdq.cache_evict(self.cache, self.pages.table, self.lens_gpu, self.budget, self.recent, lens_out=self.lens_gpu,
                            workspace=self.workspace)
            for b in range(self.B):
                self.lens[b] = min(self.lens[b], self.budget)
                self.pages.resize(b, self.lens[b])
        self.position += 1
        return dict(y=y, qkv=qkv, q=q, attention=o)


def main(argv=None) -> None:
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--width", type=int, default=4096)
    ap.add_argument("--heads", type=int, default=32)
    ap.add_argument("--heads-kv", type=int, default=32)
    ap.add_argument("--dim", type=int, default=128)
    ap.add_argument("--sequences", type=int, default=8)
    ap.add_argument("--tokens", type=int, default=64)
    ap.add_argument("--kv", choices=("bf16", "e4m3"), default="bf16")
    ap.add_argument("--budget", type=int, default=0, help="slots a sequence may keep (0: all)")
    ap.add_argument("--recent", type=int, default=0, help="of them, the newest that are kept in any case")
    a = ap.parse_args(argv)
    cfg = dataclasses.replace(sdq.Config.of(synth.INT_1x8_E4M3_3x8), y_dtype="bf16")
    block = Attention(cfg, a.width, a.heads, a.heads_kv, a.dim, a.sequences, a.tokens, kv=a.kv, budget=a.budget, recent=a.recent)
    x = torch.from_numpy(synth.make_x(5, a.sequences, a.width)).to("cuda").to(torch.bfloat16)
    block.step(x)
    torch.cuda.synchronize()
    began = time.perf_counter()
    for _ in range(a.tokens - 1):
        x = x + block.step(x)["y"].to(torch.bfloat16)
        x = x / x.float().square().mean(-1, keepdim=True).sqrt().to(torch.bfloat16)  # keeps the walk bounded, as a norm would
    torch.cuda.synchronize()
    took = time.perf_counter() - began
    print(f"{a.sequences} sequences x {a.tokens} tokens, slots held {block.lens}, "
          f"{1e6 * took / max(1, a.tokens - 1):.0f} us per step, output rms {float(x.float().square().mean().sqrt()):.3f}")
    assert bool(torch.isfinite(x.float()).all()) and np.isfinite(took)


if __name__ == "__main__":
    main()
