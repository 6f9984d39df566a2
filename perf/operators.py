"""The block-scaled 8-bit floating point layer and the norm and rotation of queries and keys: plain forms and timed cases.

  act      `quantize_act_fp8`: activations [rows, cin] to E4M3 codes with a scale for each block of 128 channels of a token
  weight   `quantize_weight_fp8`: a weight matrix to E4M3 codes with a scale for each block of 128 x 128
  linear   `fp8_linear`: the product of such codes with both scales, and the bias
  rope     `qk_norm_rope`: root-mean-square norm of every query and key head, then the rotation by the token's positions
           (one axis for text, height and width for images, time, height and width for video)

`run` computes them with elementary torch operations where `own` is false and calls the framework where it is true.
"""
import math

import torch

own = False

DTYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
BYTES = {"fp32": 4, "bf16": 2, "fp16": 2}
BLOCK = 128
E4M3_MAX = 448.0
SMALLEST = 2.0 ** -64            # smallest maximum that a block's scale is taken from
MAX_MACS = 16384 * 4096 * 4096   # the largest listed layer
MAX_CELLS = 16384 * 4096


def act(name, rows, cin, x, pitch=0):
    return {"name": name, "op": "act", "rows": rows, "cin": cin, "x": x, "pitch": pitch}


def weight(name, cout, cin, x):
    return {"name": name, "op": "weight", "cout": cout, "cin": cin, "x": x}


def linear(name, rows, cin, cout, y, bias=True):
    return {"name": name, "op": "linear", "rows": rows, "cin": cin, "cout": cout, "y": y, "bias": bias}


def rope(name, rows, hq, hk, dim, rot, axes, x, norm=True, adjacent=False, far=0):
    return {"name": name, "op": "rope", "rows": rows, "hq": hq, "hk": hk, "dim": dim, "rot": rot, "axes": axes, "x": x, "norm": norm,
            "adjacent": adjacent, "far": far}


def listed():
    return [
        # the benchmark's smallest layer: half a block of channels, latency
        act("act_256x64_fp32", 256, 64, "fp32"),
        # ViT-B tokens at batch 32
        act("act_vitb_bf16", 32 * 577, 768, "bf16"),
        # channels that end inside a block, odd number of rows, rows with a pitch that no wide load fits
        act("act_ragged_fp16", 4097, 1000, "fp16", pitch=1),
        # conversion of the stage-3 qkv weights: ragged blocks in both directions
        weight("weight_960x320_bf16", 960, 320, "bf16"),
        # conversion of a large matrix
        weight("weight_4096_fp32", 4096, 4096, "fp32"),
        # one token through a large layer: the weights' bytes
        linear("token_4096_bf16", 1, 4096, 4096, "bf16"),
        # qkv of stage 3 on one image
        linear("stage3_qkv_fp32", 576, 320, 960, "fp32", bias=False),
        # ViT-B qkv at batch 32
        linear("vitb_qkv_bf16", 32 * 577, 768, 2304, "bf16"),
        # the compute-bound end
        linear("tokens_16384_bf16", 16384, 4096, 4096, "bf16"),
        # one new token for each of 32 sequences, grouped heads, far positions
        rope("rope_tokens_32", 32, 32, 8, 128, 128, 1, "bf16", far=1 << 20),
        # ViT-B at batch 32: height and width, no grouping
        rope("rope_image_fp16", 32 * 576, 12, 12, 64, 64, 2, "fp16"),
        # frames of video: time, height and width, grouped heads
        rope("rope_video_bf16", 16384, 32, 8, 128, 128, 3, "bf16"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choices(["act", "weight", "linear", "rope"], [3, 2, 6, 4])[0]
    x = rng.choice(["bf16", "bf16", "fp16", "fp32"])
    while True:
        if op == "act":
            c = {"op": op, "rows": _log(rng, 1, 32768), "cin": _log(rng, 32, 8192), "x": x, "pitch": rng.choice([0, 0, 8, 1])}
            if c["rows"] * c["cin"] <= MAX_CELLS:
                return c
        elif op == "weight":
            return {"op": op, "cout": _log(rng, 32, 4096), "cin": _log(rng, 32, 4096), "x": x}
        elif op == "linear":
            c = {"op": op, "rows": _log(rng, 1, 32768), "cin": _log(rng, 64, 8192), "cout": _log(rng, 32, 16384), "y": x,
                 "bias": rng.random() < 0.5}
            if c["rows"] * c["cin"] * c["cout"] <= MAX_MACS and max(c["cin"], c["cout"]) * c["rows"] <= MAX_CELLS:
                return c
        else:
            hk = rng.choice([1, 2, 4, 8, 12])
            dim = rng.choice([32, 64, 64, 80, 96, 128, 128, 256])
            c = {"op": op, "rows": _log(rng, 1, 32768), "hq": hk * rng.choice([1, 1, 4, 5]), "hk": hk, "dim": dim,
                 "rot": dim if rng.random() < 0.7 else dim // 2, "axes": rng.randint(1, 3), "x": x, "norm": rng.random() < 0.8,
                 "adjacent": rng.random() < 0.3, "far": rng.choice([0, 0, 1 << 17, 1 << 20])}
            if c["rows"] * (c["hq"] + c["hk"]) * dim <= 2 * MAX_CELLS:
                return c


def _blocks(n):
    return (n + BLOCK - 1) // BLOCK


class _Inputs:
    """Seeded values on the GPU: heavy-tailed tokens (a tenth of them Student-t of three degrees, widths that differ between
    tokens), normal weights."""

    def __init__(self, seed):
        self.g = torch.Generator(device="cuda")
        self.g.manual_seed(seed)

    def normal(self, *shape):
        return torch.randn(shape, generator=self.g, device="cuda", dtype=torch.float32)

    def uniform(self, *shape):
        return torch.rand(shape, generator=self.g, device="cuda", dtype=torch.float32)

    def integers(self, hi, *shape):
        return torch.randint(0, hi, shape, generator=self.g, device="cuda")

    def tokens(self, rows, cin):
        x = self.normal(rows, cin)
        heavy = self.uniform(rows, 1) < 0.1
        tail = torch.sqrt((self.normal(rows, 1) ** 2 + self.normal(rows, 1) ** 2 + self.normal(rows, 1) ** 2) / 3.0)
        return torch.where(heavy, 20.0 * x / tail.clamp_min(0.05), x * torch.exp(0.5 * self.normal(rows, 1)))


def _codes(blocked, dims):
    """E4M3 codes and scales of a tensor whose blocks are the axes `dims`."""
    top = blocked.abs().amax(dim=dims, keepdim=True).clamp_min(SMALLEST)
    most = torch.full_like(top, E4M3_MAX)      # a tensor: torch divides by a number, and a number by a tensor, with a reciprocal
    codes = (blocked * (most / top)).to(torch.float8_e4m3fn)
    return codes, top / most


def _plain_act(x):
    rows, cin = x.shape
    k = _blocks(cin)
    padded = torch.zeros((rows, k * BLOCK), dtype=torch.float32, device=x.device)
    padded[:, :cin] = x
    codes, scale = _codes(padded.view(rows, k, BLOCK), (2,))
    return codes.view(rows, k * BLOCK), scale.view(rows, k)


def _plain_weight(w):
    cout, cin = w.shape
    t, k = _blocks(cout), _blocks(cin)
    padded = torch.zeros((t * BLOCK, k * BLOCK), dtype=torch.float32, device=w.device)
    padded[:cout, :cin] = w
    codes, scale = _codes(padded.view(t, BLOCK, k, BLOCK), (1, 3))
    return codes.view(t * BLOCK, k * BLOCK)[:cout].contiguous(), scale.view(t, k)


def _plain_linear(xcodes, xscale, wcodes, wscale, bias, dtype):
    x = xcodes.to(torch.float32) * xscale.repeat_interleave(BLOCK, 1)
    w = wcodes.to(torch.float32) * wscale.repeat_interleave(BLOCK, 1).repeat_interleave(BLOCK, 0)[:wcodes.shape[0]]
    y = x @ w.t()
    if bias is not None:
        y = y + bias
    return y.to(dtype)


def _plain_rope(x, weight, positions, freq, axis, eps, adjacent):
    n = x.to(torch.float32)
    if eps is not None:
        n = n * torch.rsqrt((n * n).mean(-1, keepdim=True) + eps)
        n = n * weight
    half = freq.numel()
    angle = positions[:, axis.long()].to(torch.float64) * freq
    cos, sin = torch.cos(angle).to(torch.float32)[:, None], torch.sin(angle).to(torch.float32)[:, None]
    out = n.clone()
    a, b = (slice(0, 2 * half, 2), slice(1, 2 * half, 2)) if adjacent else (slice(0, half), slice(half, 2 * half))
    out[..., a] = n[..., a] * cos - n[..., b] * sin
    out[..., b] = n[..., b] * cos + n[..., a] * sin
    return out.to(x.dtype)


def prepare(case, seed):
    inp, op = _Inputs(seed), case["op"]
    s = {"op": op}
    if op == "act":
        rows, cin = case["rows"], case["cin"]
        s["x"] = torch.zeros((rows, cin + case["pitch"]), dtype=DTYPES[case["x"]], device="cuda")[:, :cin]
        s["x"].copy_(inp.tokens(rows, cin))
        s["codes"] = torch.empty((rows, _blocks(cin) * BLOCK), dtype=torch.float8_e4m3fn, device="cuda")
        s["scale"] = torch.empty((rows, _blocks(cin)), dtype=torch.float32, device="cuda")
    elif op == "weight":
        s["x"] = (0.02 * inp.normal(case["cout"], case["cin"])).to(DTYPES[case["x"]])
    elif op == "linear":
        rows, cin, cout = case["rows"], case["cin"], case["cout"]
        s["xc"], s["xs"] = _plain_act(inp.tokens(rows, cin))
        s["wc"], s["ws"] = _plain_weight(0.02 * inp.normal(cout, cin))
        s["bias"] = 0.1 * inp.normal(cout) if case["bias"] else None
        s["dtype"] = DTYPES[case["y"]]
        s["y"] = torch.empty((rows, cout), dtype=s["dtype"], device="cuda")
        s["workspace"] = torch.zeros((256,), dtype=torch.uint8, device="cuda")
    else:
        rows, hq, hk, dim, rot, axes = (case[k] for k in ("rows", "hq", "hk", "dim", "rot", "axes"))
        # the rows of a qkv layer's output: queries, keys, values
        qkv = inp.tokens(rows, (hq + 2 * hk) * dim).to(DTYPES[case["x"]])
        s["q"] = qkv[:, :hq * dim].view(rows, hq, dim)
        s["k"] = qkv[:, hq * dim:(hq + hk) * dim].view(rows, hk, dim)
        s["qw"], s["kw"] = 1.0 + 0.1 * inp.normal(dim), 1.0 + 0.1 * inp.normal(dim)
        s["eps"] = 1e-6 if case["norm"] else None
        if axes == 1:
            s["positions"] = torch.arange(rows, device="cuda")[:, None] + inp.integers(case["far"] + 1, 1)
        else:   # a grid of 24 columns, rows of 24, then time; the last axes of it
            at = torch.arange(rows, device="cuda") + 576 * inp.integers(case["far"] // 576 + 1, 1)
            s["positions"] = torch.stack([at // 576, at // 24 % 24, at % 24][3 - axes:], 1).contiguous()
        half = rot // 2
        s["freq"] = 10000.0 ** (-2.0 * torch.arange(half, dtype=torch.float64, device="cuda") / rot)
        s["axis"] = (torch.arange(half, device="cuda") * axes // half).to(torch.int32)
        s["adjacent"] = case["adjacent"]
        s["q_out"] = torch.empty((rows, hq, dim), dtype=qkv.dtype, device="cuda")
        s["k_out"] = torch.empty((rows, hk, dim), dtype=qkv.dtype, device="cuda")
    return s


def _own(s):
    from paper_2604_16855_b200 import tdq
    if s["op"] == "act":
        return tdq.quantize_act_fp8(s["x"], codes=s["codes"], scale=s["scale"])
    if s["op"] == "weight":
        return tdq.quantize_weight_fp8(s["x"])
    if s["op"] == "linear":
        return tdq.fp8_linear(s["xc"], s["xs"], s["wc"], s["ws"], s["bias"], y=s["y"], workspace=s["workspace"])
    return tdq.qk_norm_rope(s["q"], s["k"], s["positions"], (s["freq"], s["axis"]), s["qw"] if s["eps"] else None,
                            s["kw"] if s["eps"] else None, eps=s["eps"], adjacent=s["adjacent"], q_out=s["q_out"], k_out=s["k_out"])


def run(s):
    if own:
        return _own(s)
    if s["op"] == "act":
        return _plain_act(s["x"])
    if s["op"] == "weight":
        return _plain_weight(s["x"])
    if s["op"] == "linear":
        return _plain_linear(s["xc"], s["xs"], s["wc"], s["ws"], s["bias"], s["dtype"])
    return tuple(_plain_rope(x, w, s["positions"], s["freq"], s["axis"], s["eps"], s["adjacent"])
                 for x, w in ((s["q"], s["qw"]), (s["k"], s["kw"])))


def work(case):
    op = case["op"]
    if op == "linear":
        m, i, o, k = case["rows"], _blocks(case["cin"]) * BLOCK, case["cout"], _blocks(case["cin"])
        return {"bytes": m * i + o * i + 4 * k * (m + _blocks(o)) + (4 * o if case["bias"] else 0) + m * o * BYTES[case["y"]],
                "flops": 2 * m * i * o}
    if op == "rope":
        cells = case["rows"] * (case["hq"] + case["hk"]) * case["dim"]
        return {"bytes": 2 * cells * BYTES[case["x"]] + 8 * case["rows"] * case["axes"], "flops": 6 * cells}
    rows, cin = (case["rows"] if op == "act" else case["cout"]), case["cin"]
    k = _blocks(cin)
    return {"bytes": rows * cin * BYTES[case["x"]] + rows * k * BLOCK + 4 * k * (rows if op == "act" else _blocks(rows)),
            "flops": 3 * rows * cin}


def _exact_blocks(x, rows_per):
    """Scales in 64 bits and the E4M3 value next to the binary32 product of each element with the binary32 quotient 448 / maximum,
    ties to even: rounded to a whole number of steps of 2^-3 of its power of two, of 2^-9 below 2^-6."""
    rows, cin = x.shape
    t, k = (rows + rows_per - 1) // rows_per, _blocks(cin)
    p = torch.nn.functional.pad(x.to(torch.float64), (0, k * BLOCK - cin, 0, t * rows_per - rows))
    p = p.reshape(t, rows_per, k, BLOCK)
    top = torch.maximum(p.abs().amax((1, 3)), torch.tensor(SMALLEST, dtype=torch.float64, device=x.device))
    q = p * (E4M3_MAX / top).float().double()[:, None, :, None]
    q = q.float().double()
    _, exponent = torch.frexp(q)                                         # |q| in [2^(e-1), 2^e)
    step = torch.ldexp(torch.ones_like(q), torch.clamp(exponent - 1, min=-6) - 3)
    q = torch.round(q / step) * step
    return q.reshape(t * rows_per, k * BLOCK)[:rows], top / E4M3_MAX


def exact(case, seed):
    s = prepare(case, seed)
    if s["op"] == "act":
        return _exact_blocks(s["x"], 1)
    if s["op"] == "weight":
        return _exact_blocks(s["x"], BLOCK)
    if s["op"] == "linear":
        m, o, k = s["xc"].shape[0], s["wc"].shape[0], s["xs"].shape[1]
        x = (s["xc"].double().view(m, k, BLOCK) * s["xs"].double()[:, :, None]).view(m, -1)
        ws = s["ws"].double()[torch.arange(o, device="cuda") // BLOCK]
        w = (s["wc"].double().view(o, k, BLOCK) * ws[:, :, None]).view(o, -1)
        y = torch.mm(x, w.t())
        return y if s["bias"] is None else y.add_(s["bias"].double())
    out = []
    for x, w in ((s["q"], s["qw"]), (s["k"], s["kw"])):
        n = x.double()
        if s["eps"] is not None:
            n = n / torch.sqrt(n.square().mean(-1, keepdim=True) + s["eps"]) * w.double()
        half = s["freq"].numel()
        angle = torch.gather(s["positions"].double(), 1, s["axis"].long()[None].expand(n.shape[0], half)) * s["freq"]
        turn = torch.polar(torch.ones_like(angle), angle)[:, None]
        r = n[..., :2 * half]
        if s["adjacent"]:
            z = torch.complex(r[..., 0::2], r[..., 1::2]) * turn
            r = torch.stack([z.real, z.imag], -1).reshape(r.shape)
        else:
            z = torch.complex(r[..., :half], r[..., half:]) * turn
            r = torch.cat([z.real, z.imag], -1)
        out.append(torch.cat([r, n[..., 2 * half:]], -1))
    return tuple(out)
