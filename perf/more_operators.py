"""What a transformer block computes around its decomposed products, as cases that can be timed and checked.

A block's projections are this library's products of 8-bit activations.  Three operators carry a model from one of them
to the next:

  norm  the block's output joins the residual stream (normed first, gated and scaled, where the model has that), and the
        stream is normed for the next projections: as activations, or as 8-bit codes with a scale per token
  glu   the activation between the projections of a feed-forward block, act(gate) * up or act(x), to the same outputs
  gemm  the product of a layer that is kept dense: 8-bit integer codes on both sides, a scale per token and one per
        output channel, a bias where the layer has one

Codes of 8 bits: s = max|v| / qmax, code = v * (qmax / max|v|) to the nearest, ties to even, with qmax 127 (int8) or 448
(e4m3).  Norms take their mean and mean square in 64 bits, and the activation is evaluated in 64 bits, so that the codes
do not hang on the order of a sum; the steps between are 32-bit operations in the order written in the plain forms.
"""
import math

import torch

own = False

QMAX = {"int8": 127.0, "e4m3": 448.0}
DTYPE = {"f32": torch.float32, "bf16": torch.bfloat16}


# ------------------------------------------------------------------ the cases
def _norm(name, M, K, x="bf16", y="bf16", out="int8", layer=False, post=False, gate="none", scale=1.0, first=False):
    c = dict(op="norm", M=M, K=K, x=x, y=y, out=out, layer=layer, post=post, gate=gate, scale=scale, first=first)
    return dict(c, name=name) if name else c


def _glu(name, M, F, act="silu", gated=True, x="bf16", out="int8"):
    c = dict(op="glu", M=M, F=F, act=act, gated=gated, x=x, out=out)
    return dict(c, name=name) if name else c


def _gemm(name, M, N, K, y="bf16", bias=False):
    c = dict(op="gemm", M=M, N=N, K=K, y=y, bias=bias)
    return dict(c, name=name) if name else c


def listed():
    return [
        # one token of decode at a width of 4096: the smallest call, latency
        _norm("norm_m1_4096", 1, 4096),
        # 64 sequences decoded together: the stream in 32 bits, the block's output normed and gated by channel, e4m3 codes
        _norm("norm_m64_sandwich_e4m3", 64, 4096, x="f32", y="f32", out="e4m3", post=True, gate="channel", scale=0.5),
        # a prompt of odd length and odd width: layer norms with biases, a gate of its own for every element
        _norm("norm_m333_layer_odd", 333, 1544, x="f32", y="bf16", out="f32", layer=True, post=True, gate="full", scale=0.7),
        # a batch of long prompts: the most bytes
        _norm("norm_m8192_4096", 8192, 4096, post=True, gate="channel"),
        # one token between the stacked gate/up and the down projection of a feed-forward block of 11008
        _glu("glu_m1_11008", 1, 11008),
        # an odd prompt through an ungated activation, odd width, 32-bit input
        _glu("glu_m517_gelu_odd", 517, 2728, act="gelu", gated=False, x="f32", out="bf16"),
        # a batch of long prompts: the most bytes
        _glu("glu_m4096_11008", 4096, 11008),
        # one token through a 4096 x 4096 layer: latency
        _gemm("gemm_m1_4096", 1, 4096, 4096),
        # 16 sequences through a stacked gate/up projection: the weights' bytes
        _gemm("gemm_m16_gateup", 16, 22016, 4096),
        # 64 sequences through the second projection of a feed-forward block of 16384, with its bias
        _gemm("gemm_m64_fc2_bias", 64, 4096, 16384, y="f32", bias=True),
        # odd sizes throughout
        _gemm("gemm_m517_odd", 517, 5003, 1104, y="f32", bias=True),
        # a batch of prompts through the stacked gate/up projection: the most operations
        _gemm("gemm_m4096_gateup", 4096, 22016, 4096),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["norm", "glu", "gemm", "gemm"])
    if op == "norm":
        while True:
            M, K = _log(rng, 1, 16384), 8 * _log(rng, 4, 2048)
            if M * K <= 8192 * 4096:
                break
        first = rng.random() < 0.15  # the first norm of a model: nothing to add yet
        return _norm(None, M, K, x=rng.choice(["bf16", "f32"]), y=rng.choice(["bf16", "f32"]),
                     out=rng.choice(["int8", "int8", "e4m3", "bf16", "f32"]), layer=rng.random() < 0.4,
                     post=not first and rng.random() < 0.5, gate="none" if first else rng.choice(["none", "channel", "token", "full"]),
                     scale=1.0 if first else rng.choice([1.0, 0.5, 0.22, -1.0]), first=first)
    if op == "glu":
        while True:
            M, F = _log(rng, 1, 16384), 8 * _log(rng, 4, 3584)
            if M * F <= 4096 * 11008:
                break
        gated = rng.random() < 0.7
        return _glu(None, M, F, act=rng.choice(["silu", "gelu", "relu"]), gated=gated, x=rng.choice(["bf16", "bf16", "f32"]),
                    out=rng.choice(["int8", "int8", "e4m3", "bf16", "f32"]))
    while True:
        M, N, K = _log(rng, 1, 8192), _log(rng, 16, 32768), 16 * _log(rng, 4, 1792)
        if M * N * K <= 4096 * 22016 * 4096 and N * K <= 22016 * 11008 and M * N <= 4096 * 22016:
            break
    return _gemm(None, M, N, K, y=rng.choice(["bf16", "f32"]), bias=rng.random() < 0.5)


# ------------------------------------------------------------------ the inputs
def _gen(dev, seed):
    return torch.Generator(device=dev).manual_seed(1000033 * int(seed) + 71)


def _codes(t):
    """int8 codes of the rows of t, and their scales: what the product's two sides hold."""
    a = t.abs().amax(-1)
    return torch.round(t * (127.0 / a)[:, None]).clamp(-127, 127).to(torch.int8), a / 127.0


def prepare(case, seed):
    c, dev = case, torch.device("cuda")
    g = _gen(dev, seed)

    def randn(*shape):
        return torch.randn(shape, generator=g, device=dev)

    s = dict(c=c)
    if c["op"] == "norm":
        M, K = c["M"], c["K"]
        loud = 1 + 9 * (torch.rand(K, generator=g, device=dev) < 1 / 64)  # a few loud channels, as trained models have them
        s["residual"] = (randn(M, K) * loud + 0.1).to(DTYPE[c["x"]])
        s["y"] = None if c["first"] else (0.5 * randn(M, K) * loud - 0.05).to(DTYPE[c["y"]])
        for n in ("weight", "post_weight"):
            s[n] = 1 + 0.2 * randn(K)
        for n in ("bias", "post_bias"):
            s[n] = 0.1 * randn(K) if c["layer"] else None
        if not c["post"]:
            s["post_weight"] = s["post_bias"] = None
        shape = {"none": None, "channel": (1, K), "token": (M, 1), "full": (M, K)}[c["gate"]]
        s["gate"] = None if shape is None else (1 + 0.5 * randn(*shape)).to(DTYPE[c["y"]])
    elif c["op"] == "glu":
        s["x"] = (1.5 * randn(c["M"], c["F"] * (2 if c["gated"] else 1))).to(DTYPE[c["x"]])
    else:
        M, N, K = c["M"], c["N"], c["K"]
        loud = 1 + 9 * (torch.rand(K, generator=g, device=dev) < 1 / 64)
        s["xq"], s["s_x"] = _codes(randn(M, K) * loud)
        s["wq"], s["s_w"] = _codes(randn(N, K) / math.sqrt(K))
        s["bias"] = randn(N) if c["bias"] else None
    if own:
        _buffers(s)
    return s


def _buffers(s):
    """What a serving program keeps: the buffers that its steps write."""
    c, dev = s["c"], torch.device("cuda")
    if c["op"] == "gemm":
        s["y"] = torch.empty((c["M"], c["N"]), dtype=DTYPE[c["y"]], device=dev)
        return
    shape = (c["M"], c["K"] if c["op"] == "norm" else c["F"])
    coded = c["out"] in QMAX
    s["out"] = torch.empty(shape, dtype=torch.uint8 if coded else DTYPE[c["out"]], device=dev)
    s["result"] = {"out": s["out"]}
    if coded:  # the codes as the numbers that they are
        s["scales"] = torch.empty(shape[0], device=dev)
        s["result"] = {"out": s["out"].view(torch.int8 if c["out"] == "int8" else torch.float8_e4m3fn), "scales": s["scales"]}
    if c["op"] == "norm" and not c["first"]:
        s["result"]["residual"] = s["residual_out"] = torch.empty_like(s["residual"])


# ------------------------------------------------------------------ one pass
def run(state):
    return (_own if own else _plain)[state["c"]["op"]](state)


def _own_norm(s):
    import paper_2406_13868_amd as sdq

    c = s["c"]
    sdq.block_norm(s["residual"], s["y"], s["weight"], bias=s["bias"], eps=1e-6, layer=c["layer"], post_weight=s["post_weight"],
                   post_bias=s["post_bias"], gate=s["gate"], scale=c["scale"], out_dtype=c["out"], out=s["out"],
                   scales=s.get("scales"), residual_out=s.get("residual_out"))
    return s["result"]


def _own_glu(s):
    import paper_2406_13868_amd as sdq

    c = s["c"]
    sdq.glu_act(s["x"], c["act"], gated=c["gated"], out_dtype=c["out"], out=s["out"], scales=s.get("scales"))
    return s["result"]


def _own_gemm(s):
    import paper_2406_13868_amd as sdq

    return sdq.gemm_int8(s["xq"], s["s_x"], s["wq"], s["s_w"], bias=s["bias"], out=s["y"])


_own = dict(norm=_own_norm, glu=_own_glu, gemm=_own_gemm)


# ------------------------------------------------------------------ the plain forms
def _coded(v, out):
    """v as activations of a type, or as 8-bit codes with a scale per row."""
    if out not in QMAX:
        return {"out": v.to(DTYPE[out])}
    a, q = v.abs().amax(-1), QMAX[out]
    t = v * torch.where(a > 0, q / a, torch.zeros_like(a))[:, None]
    codes = torch.round(t).clamp(-q, q).to(torch.int8) if out == "int8" else t.clamp(-q, q).to(torch.float8_e4m3fn)
    return {"out": codes, "scales": a / q}


def _plain_normed(v, weight, bias, layer, eps=1e-6):
    d = v.double()
    if layer:
        d = d - d.mean(-1, keepdim=True)
    t = d.float() * (1.0 / torch.sqrt(d.square().mean(-1, keepdim=True) + eps)).float() * weight
    return t if bias is None else t + bias


def _plain_norm(s):
    c = s["c"]
    r = s["residual"].float()
    if not c["first"]:
        u = s["y"].float()
        if c["post"]:
            u = _plain_normed(u, s["post_weight"], s["post_bias"], c["layer"])
        if s["gate"] is not None:
            u = u * s["gate"].float()
        r = r + u * c["scale"]
    got = _coded(_plain_normed(r, s["weight"], s["bias"], c["layer"]), c["out"])
    return got if c["first"] else dict(got, residual=r.to(DTYPE[c["x"]]))


def _plain_glu(s):
    c = s["c"]
    x = s["x"]
    g = x[:, : c["F"]].double()
    if c["act"] == "silu":
        h = g / (1.0 + torch.exp(-g))
    elif c["act"] == "gelu":
        h = g / (1.0 + torch.exp(-2.0 * math.sqrt(2.0 / math.pi) * (g + 0.044715 * (g * g * g))))
    else:
        h = torch.where(g > 0, g, torch.zeros_like(g))
    if c["gated"]:
        h = h * x[:, c["F"] :].double()
    return _coded(h.float(), c["out"])


def _plain_gemm(s):
    y = torch.matmul(s["xq"].float(), s["wq"].float().t()) * s["s_x"][:, None] * s["s_w"]
    if s["bias"] is not None:
        y = y + s["bias"]
    return y.to(DTYPE[s["c"]["y"]])


_plain = dict(norm=_plain_norm, glu=_plain_glu, gemm=_plain_gemm)


# ------------------------------------------------------------------ the work
def work(case):
    c = case
    size = dict(bf16=2, f32=4, int8=1, e4m3=1)
    if c["op"] == "gemm":
        M, N, K = c["M"], c["N"], c["K"]
        return {"bytes": M * K + N * K + M * N * size[c["y"]] + 4 * (M + N + N * c["bias"]), "flops": 2 * M * N * K}
    M = c["M"]
    scales = 4 * M if c["out"] in QMAX else 0
    if c["op"] == "glu":
        F = c["F"]
        return {"bytes": M * F * (size[c["x"]] * (2 if c["gated"] else 1) + size[c["out"]]) + scales, "flops": 12 * M * F}
    K = c["K"]
    gate = {"none": 0, "channel": K, "token": M, "full": M * K}[c["gate"]] * size[c["y"]]
    rows = 4 * K * (1 + c["post"]) * (1 + c["layer"])
    stream = M * K * size[c["x"]] if c["first"] else M * K * (2 * size[c["x"]] + size[c["y"]])
    return {"bytes": stream + gate + rows + M * K * size[c["out"]] + scales, "flops": M * K * (8 + 8 * c["post"])}


# ------------------------------------------------------------------ the definitions in 64 bits
def exact(case, seed):
    """Codes of int8 have no value but themselves; in the place of an e4m3 code stands the quotient that is rounded to it."""
    c = case
    s = prepare(c, seed)
    return dict(norm=_exact_norm, glu=_exact_glu, gemm=_exact_gemm)[c["op"]](c, s)


def _exact_codes(v, out):
    if out not in QMAX:
        return dict(out=v)
    top = torch.maximum(v.amax(1), -v.amin(1))
    return dict(out=None if out == "int8" else v * QMAX[out] / top.clamp(min=1e-300)[:, None], scales=top / QMAX[out])


def _exact_normed(v, weight, bias, layer):
    n = v.shape[1]
    if layer:
        v = v - (v.sum(1) / n)[:, None]
    v = v * weight.double() / torch.sqrt((v * v).sum(1) / n + 1e-6)[:, None]
    return v if bias is None else v + bias.double()


def _exact_norm(c, s):
    r = s["residual"].double()
    if c["first"]:
        return _exact_codes(_exact_normed(r, s["weight"], s["bias"], c["layer"]), c["out"])
    y = s["y"].double()
    if c["post"]:
        y = _exact_normed(y, s["post_weight"], s["post_bias"], c["layer"])
    if s["gate"] is not None:
        y = s["gate"].double() * y
    r = torch.add(r, y, alpha=c["scale"])
    return dict(_exact_codes(_exact_normed(r, s["weight"], s["bias"], c["layer"]), c["out"]), residual=r)


def _exact_glu(c, s):
    F = c["F"]
    gate, up = s["x"].double().split([F, s["x"].shape[1] - F], 1)
    if c["act"] == "silu":
        h = gate * torch.sigmoid(gate)
    elif c["act"] == "gelu":  # the tanh form
        h = 0.5 * gate * (1 + torch.tanh(math.sqrt(2 / math.pi) * (gate + 0.044715 * gate**3)))
    else:
        h = gate.clamp(min=0)
    return _exact_codes(h * up if c["gated"] else h, c["out"])


def _exact_gemm(c, s):
    x = s["xq"].double() * s["s_x"].double()[:, None]
    w = s["wq"].double() * s["s_w"].double()[:, None]
    y = torch.mm(x, w.t().contiguous())
    return y if s["bias"] is None else y + s["bias"].double()
