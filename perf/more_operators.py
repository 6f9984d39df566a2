"""What stands around an 8-bit layer when a block is served and when it is trained: plain forms and timed cases.

  norm       `layer_norm`: normalised tokens in the input's type, with their means and reciprocal deviations
  norm8      `layer_norm_fp8`: the same, straight to the E4M3 codes and block scales that `fp8_linear` takes
  norm_back  `layer_norm_backward`: gradients of the input (with the residual branch's added), the weight and the bias
  linear     `fp8_linear` with an activation, a residual and the activation's input in its epilogue
  act_back   `activation_backward_fp8`: the activation's backward pass from its input kept in 8 bits
  grad       `fp8_weight_grad`: a layer's weight and bias gradients from its input kept in 8 bits

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
EPS = 1e-5
MAX_MACS = 16384 * 1024 * 4096   # the largest listed layer
MAX_CELLS = 16384 * 4096


def norm(name, op, rows, cols, x, pitch=0, affine=True, add=False):
    return {"name": name, "op": op, "rows": rows, "cols": cols, "x": x, "pitch": pitch, "affine": affine, "add": add}


def linear(name, rows, cin, cout, y, act=None, residual=False, pre=False):
    return {"name": name, "op": "linear", "rows": rows, "cin": cin, "cout": cout, "y": y, "act": act, "residual": residual, "pre": pre}


def act_back(name, rows, cols, x, act):
    return {"name": name, "op": "act_back", "rows": rows, "cols": cols, "x": x, "act": act}


def grad(name, rows, cin, cout, x, dw, bias=True):
    return {"name": name, "op": "grad", "rows": rows, "cin": cin, "cout": cout, "x": x, "dw": dw, "bias": bias}


def listed():
    return [
        # one new token of each of four sequences: latency
        norm("norm_tokens_4_bf16", "norm", 4, 4096, "bf16"),
        # ViT-B tokens at batch 32
        norm("norm_vitb_bf16", "norm", 32 * 577, 768, "bf16"),
        # the same in front of an 8-bit layer
        norm("norm8_vitb_bf16", "norm8", 32 * 577, 768, "bf16"),
        # odd rows, channels that end inside a block, rows with a pitch that no wide load fits, no weights
        norm("norm8_ragged_fp16", "norm8", 4097, 1000, "fp16", pitch=1, affine=False),
        # training: the residual branch's gradient added on the way
        norm("norm_back_vitb_bf16", "norm_back", 32 * 577, 768, "bf16", add=True),
        # few wide tokens in full precision
        norm("norm_back_1021x2000_fp32", "norm_back", 1021, 2000, "fp32"),
        # one token through a layer, its activation, and onto the residual stream
        linear("linear_token_silu_fp16", 1, 4096, 4096, "fp16", act="silu", residual=True),
        # first layer of an MLP in training: the activation's input is kept
        linear("linear_gelu_pre_bf16", 16384, 1024, 4096, "bf16", act="gelu", pre=True),
        # backward through an MLP's activation
        act_back("act_back_gelu_bf16", 16384, 4096, "bf16", "gelu"),
        # the same on one image in full precision, stage 3 of the encoder
        act_back("act_back_silu_fp32", 577, 1280, "fp32", "silu"),
        # the largest weight gradient
        grad("grad_1024_4096_bf16", 16384, 1024, 4096, "bf16", "bf16"),
        # stage 3 of the encoder: channels that end inside a block, an odd number of tokens
        grad("grad_stage3_fp16", 8 * 577, 320, 960, "fp16", "fp32"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choices(["norm", "norm8", "norm_back", "linear", "act_back", "grad"], [3, 2, 4, 5, 2, 5])[0]
    x = rng.choice(["bf16", "bf16", "fp16", "fp32"])
    act = rng.choice(["gelu", "gelu_tanh", "silu", "relu"])
    while True:
        rows = _log(rng, 1, 32768)
        if op in ("linear", "grad"):
            c = {"op": op, "rows": rows, "cin": _log(rng, 64, 4096), "cout": _log(rng, 32, 8192)}
            if c["rows"] * c["cin"] * c["cout"] > MAX_MACS or max(c["cin"], c["cout"]) * rows > MAX_CELLS:
                continue
            if op == "grad":
                return dict(c, x=x, dw=rng.choice([x, "fp32"]), bias=rng.random() < 0.8)
            kind = rng.choice(["act", "act", "pre", "residual", "residual", "both"])
            return dict(c, y=x, act=None if kind == "residual" else act, residual=kind in ("residual", "both"), pre=kind == "pre")
        c = {"op": op, "rows": rows, "cols": _log(rng, 32, 8192), "x": x}
        if c["rows"] * c["cols"] > MAX_CELLS // 2:
            continue
        if op == "act_back":
            return dict(c, act=act)
        return dict(c, pitch=rng.choice([0, 0, 8, 1]), affine=rng.random() < 0.8, add=op == "norm_back" and rng.random() < 0.5)


def _blocks(n):
    return (n + BLOCK - 1) // BLOCK


class _Inputs:
    """Seeded values on the GPU: tokens whose widths differ and some of whose channels stand far out, as a residual stream's do;
    normal weights."""

    def __init__(self, seed):
        self.g = torch.Generator(device="cuda")
        self.g.manual_seed(seed)

    def normal(self, *shape):
        return torch.randn(shape, generator=self.g, device="cuda", dtype=torch.float32)

    def uniform(self, *shape):
        return torch.rand(shape, generator=self.g, device="cuda", dtype=torch.float32)

    def tokens(self, rows, cols):
        return self.normal(rows, cols) * torch.exp(0.5 * self.normal(rows, 1))

    def stream(self, rows, cols):
        far = torch.where(self.uniform(cols) < 0.02, 8.0 * self.normal(cols), 0.3 * self.normal(cols))
        return self.tokens(rows, cols) + far


def _codes(blocked, dims, pow2=False):
    """E4M3 codes and scales of a tensor whose blocks are the axes `dims`: the largest magnitude of a block at 448, or the scale the
    smallest power of two that keeps it there."""
    top = blocked.abs().amax(dim=dims, keepdim=True).clamp_min(SMALLEST)
    most = torch.full_like(top, E4M3_MAX)      # a tensor: torch divides by a number, and a number by a tensor, with a reciprocal
    if pow2:
        mantissa, exponent = torch.frexp(top)  # top = mantissa 2^exponent, 0.5 <= mantissa < 1;  448 = 0.875 2^9
        scale = torch.ldexp(torch.ones_like(top), exponent - 9 + (mantissa > 0.875).int())
        return (blocked * (1.0 / scale)).to(torch.float8_e4m3fn), scale
    return (blocked * (most / top)).to(torch.float8_e4m3fn), top / most


def _rows_codes(x, pow2=False):
    rows, cols = x.shape
    k = _blocks(cols)
    padded = torch.zeros((rows, k * BLOCK), dtype=torch.float32, device=x.device)
    padded[:, :cols] = x
    codes, scale = _codes(padded.view(rows, k, BLOCK), (2,), pow2)
    return codes.view(rows, k * BLOCK), scale.view(rows, k)


def _weight_codes(w):
    cout, cin = w.shape
    t, k = _blocks(cout), _blocks(cin)
    padded = torch.zeros((t * BLOCK, k * BLOCK), dtype=torch.float32, device=w.device)
    padded[:cout, :cin] = w
    codes, scale = _codes(padded.view(t, BLOCK, k, BLOCK), (1, 3))
    return codes.view(t * BLOCK, k * BLOCK)[:cout].contiguous(), scale.view(t, k)


def _restore(codes, scale, cols):
    return (codes.to(torch.float32) * scale.repeat_interleave(BLOCK, 1))[:, :cols]


def _act(name, z):
    if name == "relu":
        return torch.clamp_min(z, 0.0)
    if name == "silu":
        return z / (1.0 + torch.exp(-z))
    if name == "gelu":
        return 0.5 * z * (1.0 + torch.erf(z * math.sqrt(0.5)))
    return 0.5 * z * (1.0 + torch.tanh(math.sqrt(2.0 / math.pi) * (z + 0.044715 * z * z * z)))


def _act_slope(name, z):
    if name == "relu":
        return (z > 0).to(z.dtype)
    if name == "silu":
        s = 1.0 / (1.0 + torch.exp(-z))
        return s * (1.0 + z * (1.0 - s))
    if name == "gelu":
        return 0.5 * (1.0 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) * (1.0 / math.sqrt(2.0 * math.pi))
    a = math.sqrt(2.0 / math.pi)
    t = torch.tanh(a * (z + 0.044715 * z * z * z))
    return 0.5 * (1.0 + t) + 0.5 * z * (1.0 - t * t) * a * (1.0 + 3.0 * 0.044715 * z * z)


def _plain_norm(x, weight, bias):
    x = x.to(torch.float32)
    mean = x.mean(1, keepdim=True)
    off = x - mean
    rstd = torch.rsqrt((off * off).mean(1, keepdim=True) + EPS)
    y = off * rstd
    return y if weight is None else y * weight + bias, mean[:, 0], rstd[:, 0]


def _plain_norm_back(dy, x, mean, rstd, weight, add):
    dy32 = dy.to(torch.float32)
    hat = (x.to(torch.float32) - mean[:, None]) * rstd[:, None]
    g = dy32 if weight is None else dy32 * weight
    dx = rstd[:, None] * (g - g.mean(1, keepdim=True) - hat * (g * hat).mean(1, keepdim=True))
    if add is not None:
        dx = dx + add.to(torch.float32)
    return dx.to(x.dtype), (dy32 * hat).sum(0), dy32.sum(0)


def _plain_linear(s):
    w = s["wc"].to(torch.float32) * s["ws"].repeat_interleave(BLOCK, 1).repeat_interleave(BLOCK, 0)[:s["wc"].shape[0]]
    z = (s["xc"].to(torch.float32) * s["xs"].repeat_interleave(BLOCK, 1)) @ w.t() + s["bias"]
    y = z if s["act"] is None else _act(s["act"], z)
    if s["residual"] is not None:
        y = y + s["residual"].to(torch.float32)
    y = y.to(s["y"].dtype)
    return y if s["pre"] is None else (y, z.to(y.dtype))


def prepare(case, seed):
    inp, op, rows = _Inputs(seed), case["op"], case["rows"]
    s = {"op": op}
    if op in ("norm", "norm8", "norm_back"):
        cols, dtype = case["cols"], DTYPES[case["x"]]

        def pitched(values):
            t = torch.zeros((rows, cols + case["pitch"]), dtype=dtype, device="cuda")[:, :cols]
            t.copy_(values)
            return t

        s["x"] = pitched(inp.stream(rows, cols))
        s["weight"] = 1.0 + 0.1 * inp.normal(cols) if case["affine"] else None
        s["bias"] = 0.1 * inp.normal(cols) if case["affine"] else None
        s["mean"] = torch.empty((rows,), dtype=torch.float32, device="cuda")
        s["rstd"] = torch.empty((rows,), dtype=torch.float32, device="cuda")
        if op == "norm":
            s["y"] = torch.empty((rows, cols), dtype=dtype, device="cuda")
        elif op == "norm8":
            s["codes"] = torch.empty((rows, _blocks(cols) * BLOCK), dtype=torch.float8_e4m3fn, device="cuda")
            s["scale"] = torch.empty((rows, _blocks(cols)), dtype=torch.float32, device="cuda")
        else:
            _, s["mean"], s["rstd"] = _plain_norm(s["x"], None, None)
            s["dy"] = pitched(0.01 * inp.tokens(rows, cols))
            s["add"] = pitched(0.01 * inp.tokens(rows, cols)) if case["add"] else None
            s["dx"] = torch.empty((rows, cols), dtype=dtype, device="cuda")
            s["dweight"] = torch.empty((cols,), dtype=torch.float32, device="cuda")
            s["dbias"] = torch.empty((cols,), dtype=torch.float32, device="cuda")
    elif op == "linear":
        cin, cout, dtype = case["cin"], case["cout"], DTYPES[case["y"]]
        s["xc"], s["xs"] = _rows_codes(inp.tokens(rows, cin))
        s["wc"], s["ws"] = _weight_codes(inp.normal(cout, cin) / math.sqrt(cin))
        s["bias"] = 0.1 * inp.normal(cout)
        s["act"] = case["act"]
        s["residual"] = inp.stream(rows, cout).to(dtype) if case["residual"] else None
        s["y"] = torch.empty((rows, cout), dtype=dtype, device="cuda")
        s["pre"] = torch.empty((rows, cout), dtype=dtype, device="cuda") if case["pre"] else None
        s["workspace"] = torch.zeros((256,), dtype=torch.uint8, device="cuda")
    elif op == "act_back":
        s["act"] = case["act"]
        s["dh"] = (0.01 * inp.tokens(rows, case["cols"])).to(DTYPES[case["x"]])
        s["zc"], s["zs"] = _rows_codes(inp.tokens(rows, case["cols"]), pow2=True)
        s["dz"] = torch.empty_like(s["dh"])
    else:
        cin, cout = case["cin"], case["cout"]
        s["cin"] = cin
        s["dy"] = (0.01 * inp.tokens(rows, cout)).to(DTYPES[case["x"]])
        s["xc"], s["xs"] = _rows_codes(inp.stream(rows, cin), pow2=True)
        s["dw"] = torch.empty((cout, cin), dtype=DTYPES[case["dw"]], device="cuda")
        s["db"] = torch.empty((cout,), dtype=torch.float32, device="cuda") if case["bias"] else None
    return s


def _own(s):
    from paper_2604_16855_b200 import tdq
    op = s["op"]
    if op == "norm":
        return tdq.layer_norm(s["x"], s["weight"], s["bias"], eps=EPS, y=s["y"], mean=s["mean"], rstd=s["rstd"])
    if op == "norm8":
        return tdq.layer_norm_fp8(s["x"], s["weight"], s["bias"], eps=EPS, codes=s["codes"], scale=s["scale"], mean=s["mean"], rstd=s["rstd"])
    if op == "norm_back":
        return tdq.layer_norm_backward(s["dy"], s["x"], s["mean"], s["rstd"], s["weight"], add=s["add"], dx=s["dx"], dweight=s["dweight"],
                                       dbias=s["dbias"])
    if op == "linear":
        y = tdq.fp8_linear(s["xc"], s["xs"], s["wc"], s["ws"], s["bias"], activation=s["act"], residual=s["residual"], y=s["y"], pre=s["pre"],
                           workspace=s["workspace"])
        return y if s["pre"] is None else (y, s["pre"])
    if op == "act_back":
        return tdq.activation_backward_fp8(s["dh"], s["zc"], s["zs"], s["act"], dz=s["dz"])
    dw, db = tdq.fp8_weight_grad(s["dy"], s["xc"], s["xs"], s["cin"], dw=s["dw"], db=s["db"], bias=s["db"] is not None)
    return dw if db is None else (dw, db)


def run(s):
    if own:
        return _own(s)
    op = s["op"]
    if op == "norm":
        y, mean, rstd = _plain_norm(s["x"], s["weight"], s["bias"])
        return y.to(s["x"].dtype), mean, rstd
    if op == "norm8":
        y, mean, rstd = _plain_norm(s["x"], s["weight"], s["bias"])
        return (*_rows_codes(y), mean, rstd)
    if op == "norm_back":
        return _plain_norm_back(s["dy"], s["x"], s["mean"], s["rstd"], s["weight"], s["add"])
    if op == "linear":
        return _plain_linear(s)
    if op == "act_back":
        return (s["dh"].to(torch.float32) * _act_slope(s["act"], _restore(s["zc"], s["zs"], s["dh"].shape[1]))).to(s["dh"].dtype)
    dy = s["dy"].to(torch.float32)
    dw = (dy.t() @ _restore(s["xc"], s["xs"], s["cin"])).to(s["dw"].dtype)
    return dw if s["db"] is None else (dw, dy.sum(0))


def work(case):
    op, m = case["op"], case["rows"]
    if op == "linear":
        i, o, k = _blocks(case["cin"]) * BLOCK, case["cout"], _blocks(case["cin"])
        out = m * o * BYTES[case["y"]]
        return {"bytes": m * i + o * i + 4 * k * (m + _blocks(o)) + 4 * o + out * (1 + case["residual"] + case["pre"]), "flops": 2 * m * i * o}
    if op == "grad":
        i, o = case["cin"], case["cout"]
        kept = m * _blocks(i) * (BLOCK + 4)
        return {"bytes": kept + m * o * BYTES[case["x"]] + i * o * BYTES[case["dw"]] + (4 * o if case["bias"] else 0), "flops": 2 * m * i * o}
    n = case["cols"]
    e, kept = BYTES[case["x"]], m * _blocks(n) * (BLOCK + 4)
    affine = 8 * n if case.get("affine") else 0
    if op == "norm":
        return {"bytes": 2 * m * n * e + 8 * m + affine, "flops": 8 * m * n}
    if op == "norm8":
        return {"bytes": m * n * e + kept + 8 * m + affine, "flops": 10 * m * n}
    if op == "norm_back":
        return {"bytes": (3 + case["add"]) * m * n * e + 8 * m + affine // 2 + 8 * n, "flops": 16 * m * n}
    return {"bytes": 2 * m * n * e + kept, "flops": 12 * m * n}


def _exact_act(name, z):
    if name == "relu":
        return torch.maximum(z, torch.zeros_like(z))
    if name == "silu":
        return z * torch.special.expit(z)
    if name == "gelu":
        return z * torch.special.ndtr(z)
    return z * torch.special.expit(2.0 * math.sqrt(2.0 / math.pi) * (z + 0.044715 * z ** 3))


def _exact_values(codes, scale, cols):
    m, k = scale.shape
    return (codes.double().view(m, k, BLOCK) * scale.double()[:, :, None]).view(m, k * BLOCK)[:, :cols]


def exact(case, seed):
    s = prepare(case, seed)
    op = s["op"]
    if op in ("norm", "norm8"):
        x = s["x"].double()
        var, mean = torch.var_mean(x, 1, unbiased=False)
        rstd = 1.0 / torch.sqrt(var + EPS)
        y = (x - mean[:, None]) * rstd[:, None]
        if s["weight"] is not None:
            y = torch.addcmul(s["bias"].double(), y, s["weight"].double())
        if op == "norm":
            return y, mean, rstd
        m, n = x.shape
        k = _blocks(n)
        p = torch.nn.functional.pad(y, (0, k * BLOCK - n)).view(m, k, BLOCK)
        top = torch.maximum(p.abs().amax(2), torch.tensor(SMALLEST, dtype=torch.float64, device=p.device))
        # the E4M3 value next to each quotient: whole steps of 2^-3 of its power of two, of 2^-9 below 2^-6
        q = p * (E4M3_MAX / top)[:, :, None]
        step = torch.ldexp(torch.ones_like(q), torch.clamp(torch.frexp(q)[1] - 1, min=-6) - 3)
        return (torch.round(q / step) * step).view(m, k * BLOCK), top / E4M3_MAX, mean, rstd
    if op == "norm_back":
        # the gradient of sum(dy y) as the input moves, with y's mean and deviation held as they were given
        dy, x = s["dy"].double(), s["x"].double()
        rstd = s["rstd"].double()[:, None]
        hat = (x - s["mean"].double()[:, None]) * rstd
        g = dy if s["weight"] is None else dy * s["weight"].double()
        n = x.shape[1]
        along = torch.einsum("mc,mc->m", g, hat)[:, None] / n
        dx = rstd * (g - g.sum(1, keepdim=True) / n - hat * along)
        if s["add"] is not None:
            dx = dx + s["add"].double()
        return dx, torch.einsum("mc,mc->c", dy, hat), dy.sum(0)
    if op == "linear":
        w = s["ws"].double()[torch.arange(s["wc"].shape[0], device="cuda") // BLOCK]
        m, k = s["xs"].shape
        w = (s["wc"].double().view(-1, k, BLOCK) * w[:, :, None]).view(-1, k * BLOCK)
        z = torch.addmm(s["bias"].double(), _exact_values(s["xc"], s["xs"], k * BLOCK), w.t())
        y = z if s["act"] is None else _exact_act(s["act"], z)
        if s["residual"] is not None:
            y = y + s["residual"].double()
        return y if s["pre"] is None else (y, z)
    if op == "act_back":
        with torch.enable_grad():
            z = _exact_values(s["zc"], s["zs"], s["dh"].shape[1]).requires_grad_()
            if s["act"] == "gelu":
                slope = torch.special.ndtr(z) + z * torch.exp(-0.5 * z * z) / math.sqrt(2.0 * math.pi)
            else:
                slope, = torch.autograd.grad(_exact_act(s["act"], z).sum(), z)
            if s["act"] == "relu":
                slope = torch.where(z > 0, 1.0, 0.0).double()
        return s["dh"].double() * slope.detach()
    dw = torch.mm(s["dy"].double().t(), _exact_values(s["xc"], s["xs"], s["cin"]))
    return dw if s["db"] is None else (dw, s["dy"].double().sum(0))
