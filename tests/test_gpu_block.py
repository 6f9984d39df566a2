"""A pre-norm MLP block, forward and backward, with its activations kept in 8 bits: y = x + W2 gelu(W1 norm(x) + b1) + b2."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def tdq():
    from paper_2604_16855_b200 import tdq
    return tdq


class Block:
    """What a program keeps: weights' codes, and those of the transposed weights for the gradients of the layers' inputs."""

    def __init__(self, tdq, d, hidden, seed):
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)
        r = lambda *s: torch.randn(s, generator=g, device="cuda")  # noqa: E731
        self.tdq = tdq
        self.w1, self.w2 = r(hidden, d) / math.sqrt(d), r(d, hidden) / math.sqrt(hidden)
        self.b1, self.b2, self.gain, self.shift = 0.1 * r(hidden), 0.1 * r(d), 1 + 0.1 * r(d), 0.1 * r(d)
        self.q1, self.q2 = tdq.quantize_weight_fp8(self.w1), tdq.quantize_weight_fp8(self.w2)
        self.t1, self.t2 = tdq.quantize_weight_fp8(self.w1.t().contiguous()), tdq.quantize_weight_fp8(self.w2.t().contiguous())

    def forward(self, x):
        t = self.tdq
        a, a_scale, mean, rstd = t.layer_norm_fp8(x, self.gain, self.shift, pow2=True)
        z = torch.empty((x.shape[0], self.w1.shape[0]), dtype=x.dtype, device="cuda")
        h = t.fp8_linear(a, a_scale, *self.q1, self.b1, activation="gelu", out_dtype=x.dtype, pre=z)
        h8, z8 = t.quantize_act_fp8(h, pow2=True), t.quantize_act_fp8(z, pow2=True)
        y = t.fp8_linear(*h8, *self.q2, self.b2, residual=x, out_dtype=x.dtype)
        return y, (x, mean, rstd, (a, a_scale), z8, h8)

    def backward(self, dy, kept):
        t = self.tdq
        x, mean, rstd, a8, z8, h8 = kept
        dw2, db2 = t.fp8_weight_grad(dy, *h8, self.w2.shape[1])
        dh = t.fp8_linear(*t.quantize_act_fp8(dy), *self.t2, out_dtype=x.dtype)
        dz = t.activation_backward_fp8(dh, *z8, "gelu", dz=dh)
        dw1, db1 = t.fp8_weight_grad(dz, *a8, self.w1.shape[1])
        da = t.fp8_linear(*t.quantize_act_fp8(dz), *self.t1, out_dtype=x.dtype)
        dx, dgain, dshift = t.layer_norm_backward(da, x, mean, rstd, self.gain, add=dy)
        return {"x": dx, "w1": dw1, "b1": db1, "w2": dw2, "b2": db2, "gain": dgain, "shift": dshift}

    def exact(self, x, dy):
        """The block in 64 bits without any codes, and its gradients."""
        with torch.enable_grad():
            p = {n: getattr(self, n).double().requires_grad_() for n in ("w1", "b1", "w2", "b2", "gain", "shift")}
            xd = x.double().requires_grad_()
            mu = xd.mean(1, keepdim=True)
            a = (xd - mu) / torch.sqrt(((xd - mu) ** 2).mean(1, keepdim=True) + 1e-5) * p["gain"] + p["shift"]
            z = a @ p["w1"].t() + p["b1"]
            y = xd + 0.5 * z * torch.special.erfc(-z / math.sqrt(2.0)) @ p["w2"].t() + p["b2"]
            grads = torch.autograd.grad((y * dy.double()).sum(), [xd, *p.values()])
        return y.detach(), dict(zip(["x", *p], grads))


def _off(got, want):
    return float((got.double() - want).norm() / want.norm())


@pytest.mark.parametrize("m,d,hidden", [(577, 320, 1280), (1200, 768, 2304), (65, 200, 500), (1, 256, 512)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32, torch.float16], ids=["bf16", "fp32", "fp16"])
def test_block(tdq, m, d, hidden, dtype):
    b = Block(tdq, d, hidden, m)
    x, dy = torch.randn((m, d), device="cuda").to(dtype), torch.randn((m, d), device="cuda").to(dtype)
    y, kept = b.forward(x)
    got = b.backward(dy, kept)
    want_y, want = b.exact(x, dy)
    # a code is off by 2^-4 of its value at most, by 2^-4 / sqrt 3 = 0.036 in the mean of squares; the longest way from dy to a gradient passes seven quantized factors (dy, W2, z's slope,
    # dz, W1, a's norm, a): 0.036 sqrt 7 = 0.095 where they are independent, and twice that is allowed
    assert _off(y, want_y) < 0.19
    for name, g in got.items():
        assert bool(g.isfinite().all()) and _off(g, want[name]) < 0.19, (name, _off(g, want[name]))
    if m > 1:
        assert got["x"].dtype == dtype and _off(got["b2"], want["b2"]) < 1e-5      # no code on its way


def test_captured_step_is_the_eager_one(tdq):
    b = Block(tdq, 320, 1280, 3)
    x, dy = torch.randn((577, 320), device="cuda", dtype=torch.bfloat16), torch.randn((577, 320), device="cuda", dtype=torch.bfloat16)
    y, kept = b.forward(x)
    want = b.backward(dy, kept)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=s):
        y2, kept2 = b.forward(x)
        got = b.backward(dy, kept2)
    for _ in range(2):
        for t in (y2, *got.values()):
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y2, y) and all(torch.equal(got[n], want[n]) for n in want)


def test_steps_on_two_streams_at_once(tdq):
    b = Block(tdq, 256, 640, 4)
    xs = [torch.randn((900, 256), device="cuda", dtype=torch.bfloat16) for _ in range(2)]
    want = []
    for x in xs:
        y, kept = b.forward(x)
        want.append((y, b.backward(x, kept)))
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in xs]
    for _ in range(5):
        got = []
        for x, s in zip(xs, streams):
            with torch.cuda.stream(s):
                y, kept = b.forward(x)
                got.append((y, b.backward(x, kept)))
        torch.cuda.synchronize()
        for (y, g), (wy, wg) in zip(got, want):
            assert torch.equal(y, wy) and all(torch.equal(g[n], wg[n]) for n in wg)
