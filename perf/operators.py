"""The decode step between the projections of a transformer block, as cases that can be timed and checked.

The linear layers of a block are this library's decomposed products; what lies between the stacked q/k/v projection and
the output projection when a model answers is three operators on a paged key-value cache:

  append  the norm of every query and key head (where the model has one), the position rotation, and the write of the
          new keys and values into the cache, bf16 or quantized to e4m3 with a scale per row
  attend  attention of one new token per sequence over the cache; with `track` it also adds every slot's attention
          weight, summed over the query heads of a key head, to a running total
  evict   where a sequence is longer than its budget: keep the most recent slots and those of the largest running
          total, and close the holes

The cache is pages of [heads, page_size, dim]; a sequence's slots are the pages of its row of the page table.  Pools
hold one page more than the cache uses: the plain forms, which have no predicated stores, send there what is masked.
Entries of a page table past a sequence's end are -1, the index of that page.
"""
import math

import numpy as np
import torch

own = False


# ------------------------------------------------------------------ the cases
def _append(name, M, hq, hkv, D, page=64, kv="bf16", x="bf16", norm=False, rot=None, inter=False, track=False, pad=0):
    c = dict(op="append", M=M, hq=hq, hkv=hkv, D=D, page=page, kv=kv, x=x, norm=norm, rot=D if rot is None else rot,
             inter=inter, track=track, pad=pad)
    return dict(c, name=name) if name else c


def _attend(name, B, L, hq, hkv, D, page=64, kv="bf16", x="bf16", ragged=False, track=False, empty=0):
    c = dict(op="attend", B=B, L=L, hq=hq, hkv=hkv, D=D, page=page, kv=kv, x=x, ragged=ragged, track=track, empty=empty)
    return dict(c, name=name) if name else c


def _evict(name, B, L, hkv, D, budget, recent, page=64, kv="bf16", ragged=False, worn=False):
    c = dict(op="evict", B=B, L=L, hkv=hkv, D=D, budget=budget, recent=recent, page=page, kv=kv, ragged=ragged, worn=worn)
    return dict(c, name=name) if name else c


def listed():
    return [
        # one token of decode, 32 heads of 128 (the heads of LLaMA-7B and OPT-6.7B): the smallest call, latency
        _append("append_m1", 1, 32, 32, 128),
        # 64 sequences decoded together, grouped heads with norms, quantized and tracked cache, some rows only padding
        _append("append_m64_gqa_e4m3", 64, 32, 8, 128, kv="e4m3", norm=True, track=True, pad=3),
        # a prompt of odd length, fp32 projections, odd heads, half of each head rotated in neighbouring pairs
        _append("append_m333_odd", 333, 28, 4, 96, page=24, x="f32", norm=True, rot=48, inter=True),
        # a batch of long prompts: the largest write of keys and values
        _append("append_m8192", 8192, 32, 32, 128, page=128),
        # one short conversation: the smallest call, latency
        _attend("attend_b1_short", 1, 100, 32, 32, 128),
        # one very long document, grouped heads: few rows, the work lies along the length
        _attend("attend_b1_131071", 1, 131071, 32, 8, 128),
        # a few sequences of odd lengths with an empty one, odd heads and pages, fp32, tracked
        _attend("attend_b7_odd_track", 7, 3001, 20, 4, 96, page=24, x="f32", ragged=True, track=True, empty=1),
        # an ordinary serving batch, grouped heads, tracked for eviction
        _attend("attend_b32_gqa_track", 32, 4096, 32, 8, 128, ragged=True, track=True),
        # a large serving batch, every head its own keys, quantized cache: the most bytes
        _attend("attend_b64_e4m3", 64, 8192, 32, 32, 128, kv="e4m3", ragged=True),
        # one conversation that has just passed its budget: the smallest call, latency
        _evict("evict_b1_641", 1, 641, 32, 128, 512, 64),
        # a batch of ragged, often evicted, quantized sequences of odd page size
        _evict("evict_b16_e4m3", 16, 4099, 8, 128, 1000, 100, page=48, kv="e4m3", ragged=True, worn=True),
        # a large batch halved at once: the most rows moved
        _evict("evict_b32_8192", 32, 8192, 32, 128, 4096, 256, worn=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["append", "attend", "attend", "evict"])
    D = rng.choice([64, 80, 96, 128, 128, 128, 192, 256])
    hkv = rng.choice([1, 2, 4, 5, 8, 8, 16, 32])
    hq = hkv * rng.choice([g for g in (1, 1, 2, 3, 4, 5, 7, 8, 16) if g * hkv <= 64])
    page, kv = rng.choice([1, 16, 16, 24, 32, 48, 64, 64, 128, 256]), rng.choice(["bf16", "bf16", "e4m3"])
    x = rng.choice(["bf16", "bf16", "f32"])
    if op == "append":
        while True:
            M = _log(rng, 1, 8192)
            if M * (hq + 2 * hkv) * D <= 8192 * 96 * 128:
                break
        rot = rng.choice([D, D, D // 2, 0])
        return _append(None, M, hq, hkv, D, page=page, kv=kv, x=x, norm=rng.random() < 0.5, rot=rot,
                       inter=rng.random() < 0.5, track=rng.random() < 0.5, pad=rng.randrange(0, M) // 8)
    if op == "attend":
        while True:
            B, L = _log(rng, 1, 128), _log(rng, 1, 131071)
            if B * L * hkv * D <= 32 * 8192 * 32 * 128 and B * L <= 1 << 20:
                break
        return _attend(None, B, L, hq, hkv, D, page=page, kv=kv, x=x, ragged=B > 1 and rng.random() < 0.7,
                       track=rng.random() < 0.4, empty=int(B > 3 and rng.random() < 0.3))
    while True:
        B, L = _log(rng, 1, 64), _log(rng, 16, 40000)
        budget = max(1, int(L * rng.uniform(0.2, 0.98)))
        if B * budget * hkv * D <= 32 * 4096 * 32 * 128 and B * L * hkv <= 32 * 8192 * 32:
            break
    return _evict(None, B, L, hkv, D, budget, rng.randrange(0, budget + 1) // 4, page=page, kv=kv,
                  ragged=B > 1 and rng.random() < 0.7, worn=rng.random() < 0.6)


# ------------------------------------------------------------------ the inputs
def _lens(c):
    """The sequences' lengths: L, or spread evenly below it; with `empty` the last ones have no slot yet."""
    B, L = c["B"], c["L"]
    n = [max(1, int(L * (1 - (i * 0.6180339887498949) % 1.0))) for i in range(B)] if c["ragged"] else [L] * B
    k = c.get("empty", 0)
    return n[: B - k] + [0] * k


def _gen(dev, seed):
    return torch.Generator(device=dev).manual_seed(1000003 * int(seed) + 29)


def _kv_pool(c, pages, g, dev, zero=False):
    """Keys and values of the whole pool and one page more; loud channels in the keys, as trained models have them.
    e4m3: codes and one fp32 scale per row."""
    shape = (pages + 1, c["hkv"], c["page"], c["D"])
    dt = torch.bfloat16 if c["kv"] == "bf16" else torch.float8_e4m3fn
    s = {}
    for name in ("k", "v"):
        t = torch.zeros(shape, dtype=dt, device=dev)
        if not zero:
            step = max(1, (1 << 28) // (shape[1] * shape[2] * shape[3]))
            for i in range(0, shape[0], step):
                r = torch.randn((min(step, shape[0] - i),) + shape[1:], generator=g, device=dev, dtype=torch.bfloat16)
                if name == "k":
                    r[..., :: max(1, c["D"] // 4)] *= 3
                t[i : i + step] = (r.float() * 60).clamp(-448, 448).to(dt) if c["kv"] == "e4m3" else r
        s[name] = t
        if c["kv"] == "e4m3":
            s[name + "_scale"] = torch.zeros(shape[:3], device=dev) if zero else (torch.rand(shape[:3], generator=g, device=dev) + 0.5) / 60
        else:
            s[name + "_scale"] = None
    return s


def _tables(c, g, dev):
    """Page table, lengths and page count: the pages of the sequences in random order, -1 past each end."""
    page, lens = c["page"], _lens(c)
    n = [-(-x // page) for x in lens]
    spare = 3
    ids = torch.randperm(sum(n) + spare, generator=g, device=dev)
    width = max(1, max(n))
    col = torch.arange(width, device=dev)
    n_t = torch.tensor(n, device=dev)
    first = torch.cumsum(n_t, 0) - n_t
    order = torch.randperm(len(n), generator=g, device=dev)
    table = torch.where(col < n_t[:, None], ids[(first[:, None] + col).clamp(max=sum(n) + spare - 1)], -1)
    return table[order].to(torch.int32).contiguous(), torch.tensor(lens, device=dev)[order].to(torch.int32).contiguous(), sum(n) + spare


def _slot_index(table, page, width):
    """Pool page and offset of the first `width` slots of every sequence: [B, width] each."""
    t = torch.arange(width, device=table.device)
    return table.long()[:, t // page], (t % page).expand(table.shape[0], width)


def prepare(case, seed):
    c, dev = case, torch.device("cuda")
    g = _gen(dev, seed)
    x_dt = torch.bfloat16 if c.get("x") == "bf16" else torch.float32
    s = dict(c=c, op=c["op"])
    if c["op"] == "append":
        M, hq, hkv, D, page = c["M"], c["hq"], c["hkv"], c["D"], c["page"]
        pages = -(-2 * M // page) + 1
        s |= _kv_pool(c, pages, g, dev, zero=True)
        s["qkv"] = torch.randn((M, (hq + 2 * hkv) * D), generator=g, device=dev).to(x_dt)
        slot = torch.randperm(pages * page, generator=g, device=dev)[:M]
        if c["pad"]:
            slot[-c["pad"] :] = -1  # the rows of a fixed-size batch that hold no token
        s["slot"] = slot
        positions = 4096
        s["pos"] = torch.randint(0, positions, (M,), generator=g, device=dev, dtype=torch.int32)
        half = c["rot"] // 2
        angle = torch.arange(positions, device=dev, dtype=torch.float64)[:, None] * 10000.0 ** (-torch.arange(half, device=dev, dtype=torch.float64) / max(half, 1))
        s["cos_sin"] = torch.cat([angle.cos(), angle.sin()], 1).float() if c["rot"] else None
        for n in ("q_norm", "k_norm"):
            s[n] = 1 + 0.2 * torch.randn(D, generator=g, device=dev) if c["norm"] else None
        s["out"] = torch.zeros((M, hq, D), dtype=x_dt, device=dev)
        s["position"] = torch.full((pages + 1, hkv, page), -1, dtype=torch.int32, device=dev) if c["track"] else None
        s["weight"] = torch.ones((pages + 1, hkv, page), device=dev) if c["track"] else None
    else:
        s["table"], s["lens"], pages = _tables(c, g, dev)
        s |= _kv_pool(c, pages, g, dev)
        hkv, page = c["hkv"], c["page"]
        shape = (pages + 1, hkv, page)
        s["position"] = s["weight"] = None
        if c["op"] == "attend":
            B, hq, D = c["B"], c["hq"], c["D"]
            s["q"] = (torch.randn((B, hq, D), generator=g, device=dev) * 1.5).to(x_dt)
            s["out"] = torch.zeros((B, hq, D), dtype=x_dt, device=dev)
            s["lse"] = torch.zeros((B, hq), device=dev)
            if c["track"]:
                s["weight"] = torch.zeros(shape, device=dev)
                s["weight_out"] = torch.zeros(shape, device=dev)
        else:
            s["weight"] = torch.zeros(shape, device=dev)
            s["weight_out"] = torch.zeros(shape, device=dev)
            s["position"] = torch.full(shape, -1, dtype=torch.int32, device=dev)
            s["position_out"] = torch.full(shape, -1, dtype=torch.int32, device=dev)
            s["lens_out"] = torch.zeros(c["B"], dtype=torch.int32, device=dev)
        if s["weight"] is not None:
            B, width = c["B"], max(1, c["L"])
            at, off = _slot_index(s["table"], page, width)
            live = torch.arange(width, device=dev) < s["lens"][:, None]
            # accumulated weights spread over orders of magnitude; one slot in 64 has had none yet
            w = torch.exp(2 * torch.randn((B, width, hkv), generator=g, device=dev))
            w *= torch.rand((B, width, hkv), generator=g, device=dev) > 1 / 64
            at = torch.where(live, at, -1)
            s["weight"][at, :, off] = w * live[..., None]
            s["weight"][-1] = 0
            if s["position"] is not None:
                if c["worn"]:  # often evicted: slots in any order of position, gaps between the positions
                    p = torch.rand((B, width, hkv), generator=g, device=dev).masked_fill(~live[..., None], 2.0).argsort(1).argsort(1) * 3 + 1
                else:
                    p = torch.arange(width, device=dev)[None, :, None].expand(B, width, hkv)
                s["position"][at, :, off] = p.to(torch.int32)
                s["position"][-1] = -1
    s["pages"] = pages
    if own:
        _handles(s)
    return s


def _handles(s):
    """What a serving program keeps: the cache object over its pools, and a workspace."""
    import paper_2406_13868_amd as sdq

    n, c = s["pages"], s["c"]

    def part(name):
        return None if s.get(name) is None else s[name][:n]

    s["cache"] = sdq.KVCache(part("k"), part("v"), part("k_scale"), part("v_scale"), part("position"), part("weight"))
    size = 0
    if c["op"] == "attend":
        size = sdq.attn_decode_workspace_size(s["cache"], c["B"], c["hq"], max(1, c["L"]), track=c["track"])
    elif c["op"] == "evict":
        size = sdq.cache_evict_workspace_size(s["cache"], c["B"], c["L"], c["budget"])
    s["workspace"] = torch.zeros(max(16, size), dtype=torch.uint8, device=s["k"].device)
    for name in ("weight_out", "position_out"):
        s["own_" + name] = part(name)


# ------------------------------------------------------------------ one pass
def run(state):
    return (_own if own else _plain)[state["op"]](state)


def _own_append(s):
    import paper_2406_13868_amd as sdq

    c = s["c"]
    sdq.qkv_append(s["qkv"], s["pos"], s["slot"], s["cache"], c["hq"], cos_sin=s["cos_sin"], interleaved=c["inter"],
                   q_weight=s["q_norm"], k_weight=s["k_norm"], eps=1e-6, out=s["out"])
    return _append_outputs(s)


def _own_attend(s):
    import paper_2406_13868_amd as sdq

    c = s["c"]
    sdq.attn_decode(s["q"], s["cache"], s["table"], s["lens"], max_len=max(1, c["L"]), out=s["out"], lse=s["lse"],
                    weight_out=s.get("own_weight_out"), workspace=s["workspace"])
    return _attend_outputs(s)


def _own_evict(s):
    import paper_2406_13868_amd as sdq

    c = s["c"]
    sdq.cache_evict(s["cache"], s["table"], s["lens"], c["budget"], recent=c["recent"], max_len=c["L"],
                    lens_out=s["lens_out"], weight_out=s["own_weight_out"], position_out=s["own_position_out"],
                    workspace=s["workspace"])
    return _evict_outputs(s)


_own = dict(append=_own_append, attend=_own_attend, evict=_own_evict)


def _pool_outputs(s, names):
    return {n: s[n][: s["pages"]] for n in names if s.get(n) is not None}


def _append_outputs(s):
    return dict(_pool_outputs(s, ("k", "v", "k_scale", "v_scale", "position", "weight")), q=s["out"])


def _attend_outputs(s):
    return dict(_pool_outputs(s, ("weight_out",)), out=s["out"], lse=s["lse"])


def _evict_outputs(s):
    return dict(_pool_outputs(s, ("k", "v", "k_scale", "v_scale", "weight_out", "position_out")), lens=s["lens_out"])


# ------------------------------------------------------------------ the plain forms
def _raw(t):
    """A pool as elements that can be indexed: e4m3 codes as bytes."""
    return t.view(torch.uint8) if t.dtype == torch.float8_e4m3fn else t


def _rotate(x, cs, inter):
    """x [M, h, D] fp32, cs [M, rot] (cosines, then sines): the first rot dimensions turned by pairs."""
    half = cs.shape[1] // 2
    cos, sin = cs[:, None, :half], cs[:, None, half:]
    head, rest = x[..., : 2 * half], x[..., 2 * half :]
    if inter:
        a, b = head[..., 0::2], head[..., 1::2]
        turned = torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
    else:
        a, b = head[..., :half], head[..., half:]
        turned = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
    return torch.cat([turned, rest], -1)


def _head_norm(x, w):
    return x * torch.rsqrt((x * x).mean(-1, keepdim=True) + 1e-6) * w


def _plain_append(s):
    c = s["c"]
    M, hq, hkv, D = c["M"], c["hq"], c["hkv"], c["D"]
    x = s["qkv"].float().view(M, hq + 2 * hkv, D)
    q, k, v = x[:, :hq], x[:, hq : hq + hkv], x[:, hq + hkv :]
    if c["norm"]:
        q, k = _head_norm(q, s["q_norm"]), _head_norm(k, s["k_norm"])
    if c["rot"]:
        cs = s["cos_sin"][s["pos"].long()]
        q, k = _rotate(q, cs, c["inter"]), _rotate(k, cs, c["inter"])
    s["out"].copy_(q)
    page = torch.where(s["slot"] < 0, -1, s["slot"] // c["page"])
    off = s["slot"] % c["page"]
    for name, t in (("k", k), ("v", v)):
        if c["kv"] == "e4m3":
            a = t.abs().amax(-1)
            inv = torch.where(a > 0, 448.0 / a, torch.zeros_like(a))
            _raw(s[name])[page, :, off] = _raw((t * inv[..., None]).clamp(-448, 448).to(torch.float8_e4m3fn))
            s[name + "_scale"][page, :, off] = a / 448.0
        else:
            s[name][page, :, off] = t.to(torch.bfloat16)
    if c["track"]:
        s["position"][page, :, off] = s["pos"][:, None].expand(M, hkv)
        s["weight"][page, :, off] = torch.zeros((), device=x.device)
    return _append_outputs(s)


def _gathered(s, name):
    """The slots of every sequence in fp32: [B, hkv, width, D], scaled."""
    table = s["table"].long()
    t = _raw(s[name])[table].view(s[name].dtype).float()
    if s[name + "_scale"] is not None:
        t = t * s[name + "_scale"][table][..., None]
    return t.transpose(1, 2).flatten(2, 3)


def _plain_attend(s):
    c = s["c"]
    B, hq, hkv, D = c["B"], c["hq"], c["hkv"], c["D"]
    q = s["q"].float().view(B, hkv, hq // hkv, D)
    score = torch.matmul(q, _gathered(s, "k").transpose(2, 3).contiguous()) * D**-0.5
    width = score.shape[-1]
    live = (torch.arange(width, device=q.device) < s["lens"][:, None])[:, None, None]
    score = score.masked_fill(~live, -math.inf)
    top = score.amax(-1, keepdim=True)
    e = torch.exp(score - top.masked_fill(top == -math.inf, 0.0))
    total = e.sum(-1, keepdim=True)
    p = e / total.masked_fill(total == 0, 1.0)
    v = _gathered(s, "v").masked_fill(~live.squeeze(2)[..., None], 0.0)
    s["out"].copy_(torch.matmul(p, v).view(B, hq, D))
    s["lse"].copy_((top + total.log()).view(B, hq))
    if c["track"]:
        table, page = s["table"].long(), c["page"]
        new = p.sum(2).view(B, hkv, -1, page).transpose(1, 2)
        s["weight_out"][table] = s["weight"][table] + new
    return _attend_outputs(s)


def _plain_evict(s):
    c = s["c"]
    hkv, page, budget, recent = c["hkv"], c["page"], c["budget"], c["recent"]
    table, lens = s["table"], s["lens"].long()
    dev, B = table.device, c["B"]
    at, off = _slot_index(table, page, c["L"])
    w, p = (s[n][at, :, off].transpose(1, 2) for n in ("weight", "position"))  # [B, hkv, width]
    t = torch.arange(c["L"], device=dev)
    live = (t < lens[:, None])[:, None].expand_as(w)
    n_new = lens.clamp(max=budget)[:, None, None]
    newest = p.masked_fill(~live, -1).amax(-1, keepdim=True)
    rank = (live.int() + (live & (p > newest - recent)).int())
    by_weight = torch.sort(w.masked_fill(~live, -1.0), dim=-1, descending=True, stable=True).indices
    by_class = torch.sort(rank.gather(-1, by_weight), dim=-1, descending=True, stable=True).indices
    order = by_weight.gather(-1, by_class)
    kept = torch.zeros_like(live).scatter(-1, order, (t < n_new).expand_as(live))
    hole, mover = ~kept & (t < n_new), kept & (t >= n_new)
    count = hole.sum(-1, keepdim=True)
    most = max(1, min(budget, c["L"] - budget) if c["L"] > budget else 1)
    to = torch.sort(hole.int(), dim=-1, descending=True, stable=True).indices[..., :most]
    of = torch.sort(mover.int(), dim=-1, descending=True, stable=True).indices[..., :most]
    moves = t[:most] < count
    h = torch.arange(hkv, device=dev)[None, :, None]
    b = torch.arange(B, device=dev)[:, None, None]
    of_page, of_off = table.long()[b, of // page], of % page
    to_page, to_off = torch.where(moves, table.long()[b, to // page], -1), to % page
    for name in ("k", "v", "k_scale", "v_scale"):
        if s[name] is not None:
            pool = _raw(s[name])
            pool[to_page, h, to_off] = pool[of_page, h, of_off]
    source = t.expand_as(w).clone().scatter(-1, torch.where(moves, to, c["L"] - 1), torch.where(moves, of, c["L"] - 1)) if c["L"] > budget else t.expand_as(w)
    inside = t < n_new
    at_live = torch.where(live, at[:, None], -1)
    where = (at_live, h, off[:, None].expand_as(w))
    s["weight_out"][where] = torch.where(inside, w.gather(-1, source), 0.0)
    s["position_out"][where] = torch.where(inside, p.gather(-1, source), -1)
    s["lens_out"].copy_(lens.clamp(max=budget))
    return _evict_outputs(s)


_plain = dict(append=_plain_append, attend=_plain_attend, evict=_plain_evict)


# ------------------------------------------------------------------ the work
def work(case):
    c = case
    elt = 2 if c["kv"] == "bf16" else 1
    row = c["D"] * elt + (4 if c["kv"] == "e4m3" else 0)  # one key or value of one head in the cache
    if c["op"] == "append":
        M, hq, hkv, D = c["M"], c["hq"], c["hkv"], c["D"]
        x, kept = (2 if c["x"] == "bf16" else 4), M - c["pad"]
        b = M * (hq + 2 * hkv) * D * x + M * hq * D * x + kept * 2 * hkv * row + M * (4 + 8) + min(M, 4096) * c["rot"] * 4
        return {"bytes": b + (kept * hkv * 8 if c["track"] else 0), "flops": M * (hq + hkv) * D * (3 + (4 if c["norm"] else 0))}
    lens = _lens(c)
    total, pages = sum(lens), sum(-(-n // c["page"]) for n in lens)
    if c["op"] == "attend":
        x = 2 if c["x"] == "bf16" else 4
        b = total * c["hkv"] * (2 * row + (8 if c["track"] else 0)) + 2 * c["B"] * c["hq"] * c["D"] * x + c["B"] * (c["hq"] * 4 + 4) + pages * 4
        return {"bytes": b, "flops": 4 * total * c["hq"] * c["D"] + 4 * total * c["hq"]}
    moves = 0.0
    for n in lens:  # slots below the budget that lose their place: as many rows move into them
        if n > c["budget"]:
            if c["worn"]:
                moves += c["budget"] * (1 - c["budget"] / n)
            else:
                r = min(c["recent"], c["budget"])
                moves += min(c["budget"], n - r) * (1 - (c["budget"] - r) / max(1, n - r))
    return {"bytes": total * c["hkv"] * 16 + moves * c["hkv"] * 4 * row + pages * 4 + c["B"] * 8, "flops": total * c["hkv"] * 4}


# ------------------------------------------------------------------ the definitions in 64 bits
def exact(case, seed):
    c = case
    s = prepare(c, seed)
    return dict(append=_exact_append, attend=_exact_attend, evict=_exact_evict)[c["op"]](c, s)


def _exact_append(c, s):
    M, hq, hkv, D = c["M"], c["hq"], c["hkv"], c["D"]
    x = s["qkv"].double().view(M, hq + 2 * hkv, D)
    qk, v = x[:, : hq + hkv].clone(), x[:, hq + hkv :]
    if c["norm"]:
        gain = torch.cat([s["q_norm"].double().expand(hq, D), s["k_norm"].double().expand(hkv, D)])
        qk = qk / torch.sqrt(qk.square().sum(-1, keepdim=True) / D + 1e-6) * gain
    half = c["rot"] // 2
    if half:
        cs = s["cos_sin"].double()[s["pos"].long()]
        i = torch.arange(half, device=x.device)
        first, second = (2 * i, 2 * i + 1) if c["inter"] else (i, i + half)
        z = torch.complex(qk[..., first], qk[..., second]) * torch.complex(cs[:, :half], cs[:, half:])[:, None]
        qk[..., first], qk[..., second] = z.real, z.imag
    got = dict(q=qk[:, :hq])
    n = s["pages"]
    page, off = torch.where(s["slot"] < 0, n, s["slot"] // c["page"]), s["slot"] % c["page"]
    for name, t in (("k", qk[:, hq:]), ("v", v)):
        pool = torch.zeros(s[name].shape, dtype=torch.float64, device=x.device)
        if c["kv"] == "e4m3":  # the quotient that is rounded to a code, and the scale
            a = t.abs().amax(-1)
            scale = torch.zeros(s[name].shape[:3], dtype=torch.float64, device=x.device)
            scale[page, :, off] = a / 448
            got[name + "_scale"] = scale[:n]
            t = t * 448 / a[..., None]
        pool[page, :, off] = t
        got[name] = pool[:n]
    if c["track"]:
        got["weight"], got["position"] = None, None
    return got


def _exact_attend(c, s):
    B, hq, hkv, D = c["B"], c["hq"], c["hkv"], c["D"]
    out = torch.zeros((B, hq, D), dtype=torch.float64, device=s["q"].device)
    lse = torch.full((B, hq), -math.inf, dtype=torch.float64, device=s["q"].device)
    weight = s["weight"].double().zero_() if c["track"] else None
    for b, n in enumerate(s["lens"].tolist()):
        if not n:
            continue
        used = s["table"][b, : -(-n // c["page"])].long()
        k, v = (_raw(s[m])[used].view(s[m].dtype).double() * (1.0 if s[m + "_scale"] is None else s[m + "_scale"][used].double()[..., None]) for m in ("k", "v"))
        k, v = (t.permute(1, 0, 2, 3).reshape(hkv, -1, D)[:, :n] for t in (k, v))
        q = s["q"][b].double().view(hkv, -1, D)
        z = torch.bmm(q, k.transpose(1, 2).contiguous()) / math.sqrt(D)
        lse[b] = torch.logsumexp(z, -1).view(hq)
        p = torch.exp(z - lse[b].view(hkv, -1, 1))
        out[b] = torch.bmm(p, v.contiguous()).view(hq, D)
        if c["track"]:
            t = torch.arange(n, device=used.device)
            weight[used[t // c["page"]], :, t % c["page"]] = p.sum(1).T + s["weight"].double()[used[t // c["page"]], :, t % c["page"]]
    got = dict(out=out, lse=lse)
    if c["track"]:
        got["weight_out"] = weight[: s["pages"]]
    return got


def _exact_evict(c, s):
    """Row by row on the host: which slots stay, and what moves into the places that fall free."""
    page, budget, n_pages = c["page"], c["budget"], s["pages"]
    table, lens = s["table"].cpu().numpy(), s["lens"].cpu().numpy()
    pools = {n: s[n].cpu().numpy() for n in ("weight", "position", "weight_out", "position_out")}
    moved = [[], []]
    for b, n in enumerate(lens):
        t = np.arange(n)
        at, off, new = table[b][t // page], t % page, min(int(n), budget)
        for h in range(c["hkv"]):
            w, p = (pools[m][at, h, off] for m in ("weight", "position"))
            order = np.lexsort((t, -w.astype(np.float64), p <= p.max(initial=-1) - c["recent"]))
            kept = np.zeros(n, bool)
            kept[order[:new]] = True
            to, of = np.flatnonzero(~kept[:new]), new + np.flatnonzero(kept[new:])
            source = t[:new].copy()
            source[to] = of
            for m, v, none in (("weight_out", w, 0), ("position_out", p, -1)):
                pools[m][at, h, off] = np.concatenate([v[source], np.full(n - new, none, v.dtype)])
            for k, x in enumerate((of, to)):
                moved[k].append(np.stack([at[x], np.full(len(x), h), off[x]]).astype(np.int64))
    of, to = (torch.from_numpy(np.concatenate(m, 1)).to(s["k"].device) for m in moved)
    got = dict(weight_out=torch.from_numpy(pools["weight_out"][:n_pages]).double(), position_out=None, lens=None)
    for name in ("k", "v", "k_scale", "v_scale"):
        if s[name] is not None:
            pool = s[name][:n_pages].double()
            pool[tuple(to)] = pool[tuple(of)]
            got[name] = pool
    return got
