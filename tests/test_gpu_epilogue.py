"""What follows the 8-bit layer in its epilogue, and the activations' backward pass from 8 bits, against the formulas in 64 bits."""
import math

import pytest
import torch

import fp8_utils as fu

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
ACTS = ["relu", "gelu", "gelu_tanh", "silu"]


@pytest.fixture(scope="module")
def tdq():
    from paper_2604_16855_b200 import tdq
    return tdq


def value(act, z):
    if act == "relu":
        return torch.where(z > 0, z, torch.zeros_like(z))
    if act == "gelu":
        return z * 0.5 * torch.special.erfc(-z / math.sqrt(2.0))
    if act == "gelu_tanh":
        return 0.5 * z * (1 + torch.tanh(math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3)))
    if act == "silu":
        return z / (1 + torch.exp(-z))
    return z


def slope(act, z):
    if act == "relu":
        return (z > 0).double()
    if act == "gelu":
        return 0.5 * torch.special.erfc(-z / math.sqrt(2.0)) + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    if act == "gelu_tanh":
        a = math.sqrt(2 / math.pi)
        t = torch.tanh(a * (z + 0.044715 * z ** 3))
        return 0.5 * (1 + t) + 0.5 * z * (1 - t * t) * a * (1 + 3 * 0.044715 * z * z)
    if act == "silu":
        s = torch.sigmoid(z)
        return s * (1 + z * (1 - s))
    return torch.ones_like(z)


def value_tol(act, z):
    """max(|z|, 1) 2^-21: the gaussian's polynomial to 6e-8, exponentials and quotients to 2^-22 of themselves, their argument's rounding |z| 2^-24 log2(e) in
    the exponent where the result is z exp(-|z|), a few products."""
    return z.abs().clamp_min(1.0) * 2.0 ** -21 if act in ("gelu", "gelu_tanh", "silu") else torch.zeros_like(z)


def halfway(v, dtype):
    fi = torch.finfo(dtype)
    return (U if dtype == torch.float32 else fi.eps / 2) * v.abs() + fi.tiny * fi.eps / 2


def operands(tdq, m, i, o, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    r = lambda *s: torch.randn(s, generator=g, device="cuda")  # noqa: E731
    xc, xs = tdq.quantize_act_fp8(r(m, i))
    wc, ws = tdq.quantize_weight_fp8(r(o, i) / math.sqrt(i))
    return xc, xs, wc, ws, 0.3 * r(o), r


def matrix(m, n, dtype, pitch, values=None):
    whole = torch.full((m, n + pitch), 99.0, dtype=dtype, device="cuda")
    if values is not None:
        whole[:, :n] = values.to(dtype)
    return whole[:, :n], whole


# every kind of kernel: few tokens in one part and several, 128 tokens, pairs of 256 and of 128 columns; one tile a cluster and many; ragged in every direction
SHAPES = [(1, 4096, 4096), (1, 64, 1), (9, 300, 1000), (33, 639, 523), (100, 256, 1030), (591, 2561, 460), (1354, 127, 898), (1500, 640, 300), (2594, 156, 1400),
          (606, 156, 13082), (1688, 91, 2164), (5783, 256, 1369), (4096, 512, 2304)]


@pytest.mark.parametrize("m,i,o", SHAPES)
@pytest.mark.parametrize("y_type,pitch", [("fp32", 0), ("bf16", 8), ("fp16", 1), ("fp32", 3)])
def test_epilogue(tdq, m, i, o, y_type, pitch):
    dtype = TYPES[y_type]
    xc, xs, wc, ws, bias, r = operands(tdq, m, i, o, m + o)
    z = tdq.fp8_linear(xc, xs, wc, ws, bias)                     # the layer's own sums, in binary32: the same tiles, the same bits
    zd = z.double()
    res, _ = matrix(m, o, dtype, pitch, r(m, o))
    for act in ACTS + [None]:
        for residual in (None, res):
            y, whole = matrix(m, o, dtype, pitch)
            if act is None and residual is None:
                continue
            got = tdq.fp8_linear(xc, xs, wc, ws, bias, activation=act, residual=residual, y=y)
            assert got is y and bool((whole[:, o:] == 99.0).all())
            want, tol = value(act, zd), value_tol(act, zd)
            if residual is not None:
                want = want + residual.double()
                tol = tol + 2 * U * want.abs()
            err = (y.double() - want).abs()
            tol = tol + halfway(want.abs() + tol, dtype)
            assert bool((err <= tol).all()), (act, float((err / tol).max()))
        if act is not None:
            y, whole = matrix(m, o, dtype, pitch)
            pre, pwhole = matrix(m, o, dtype, pitch)
            tdq.fp8_linear(xc, xs, wc, ws, bias, activation=act, y=y, pre=pre)
            assert torch.equal(pre, z.to(dtype)) and bool((pwhole[:, o:] == 99.0).all()) and bool((whole[:, o:] == 99.0).all())
            assert torch.equal(y, tdq.fp8_linear(xc, xs, wc, ws, bias, activation=act, out_dtype=dtype))


@pytest.mark.parametrize("m,i,o", [(1, 512, 700), (64, 512, 700), (700, 130, 530), (3000, 256, 1111), (3000, 256, 1120)])
@pytest.mark.parametrize("y_type", list(TYPES))
def test_residual_in_place_and_on_other_grids(tdq, m, i, o, y_type):
    dtype = TYPES[y_type]
    xc, xs, wc, ws, bias, r = operands(tdq, m, i, o, 3 * m + o)
    stream = r(m, o).to(dtype)
    want = tdq.fp8_linear(xc, xs, wc, ws, bias, activation="silu", residual=stream, out_dtype=dtype)
    y = stream.clone()
    assert torch.equal(tdq.fp8_linear(xc, xs, wc, ws, bias, activation="silu", residual=y, y=y), want)
    for rp, yp in ((1, 0), (0, 1), (16, 5)):                     # rows of one on the grid, of the other not
        res, _ = matrix(m, o, dtype, rp, stream)
        y, whole = matrix(m, o, dtype, yp)
        assert torch.equal(tdq.fp8_linear(xc, xs, wc, ws, bias, activation="silu", residual=res, y=y), want) and bool((whole[:, o:] == 99.0).all())
        pre, _ = matrix(m, o, dtype, rp)
        tdq.fp8_linear(xc, xs, wc, ws, bias, pre=pre, y=y)
        assert torch.equal(pre, y) and torch.equal(y, tdq.fp8_linear(xc, xs, wc, ws, bias, out_dtype=dtype))


def test_activations_far_out(tdq):
    """Through a layer that passes its input on: magnitudes up to 448 2^10, zeros, infinite sums, NaN."""
    v = torch.tensor([0.0, 1e-3, 0.5, 1.0, 3.0, 5.0, 5.5, 6.5, 13.0, 20.0, 88.0, 120.0, 448.0, 4.5e5], device="cuda")
    x = torch.zeros((28, 128), device="cuda")
    x[:14, 0], x[14:, 0] = v, -v
    wc, ws = tdq.quantize_weight_fp8(torch.eye(128, device="cuda")[:16])
    xc, xs = tdq.quantize_act_fp8(x)
    z = tdq.fp8_linear(xc, xs, wc, ws).double()
    for act in ACTS:
        y = tdq.fp8_linear(xc, xs, wc, ws, activation=act)
        want = value(act, z)
        assert bool((y.isfinite()).all()) and bool(((y.double() - want).abs() <= value_tol(act, z) + halfway(want, torch.float32)).all()), act
    bias = torch.zeros((16,), device="cuda")
    bias[3], bias[4] = float("nan"), float("inf")
    for act in ACTS:
        y = tdq.fp8_linear(xc, xs, wc, ws, bias, activation=act)
        assert bool(y[:, 3].isnan().all()) and bool((y[:, 4] == float("inf")).all()) and bool(y[:, 5:].isfinite().all())


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("x_type", list(TYPES))
@pytest.mark.parametrize("m,n,pitch", [(1, 1, 0), (3, 64, 0), (577, 1280, 0), (50, 1000, 8), (33, 129, 0), (40, 300, 1), (7, 4096, 0)])
def test_activation_backward(tdq, m, n, pitch, x_type, act):
    dtype = TYPES[x_type]
    g = torch.Generator(device="cuda")
    g.manual_seed(m * n)
    z0 = 2.0 * torch.randn((m, n), generator=g, device="cuda") * torch.exp(torch.randn((m, 1), generator=g, device="cuda"))
    dh, _ = matrix(m, n, dtype, pitch, torch.randn((m, n), generator=g, device="cuda"))
    for pow2 in (True, False):
        zc, zs = tdq.quantize_act_fp8(z0, pow2=pow2)
        k = fu.blocks(n)
        z = (zc.float().view(m, k, 128) * zs[:, :, None]).view(m, -1)[:, :n].double()
        dz, whole = matrix(m, n, dtype, pitch)
        assert tdq.activation_backward_fp8(dh, zc, zs, act, dz=dz) is dz
        want = dh.double() * slope(act, z)
        # the slope to max(|z|, 1) 2^-21 as its value; behind |z| = 20 the exponentials' own z^2 is below 2^-21
        tol = dh.double().abs() * (value_tol(act, z.clamp(-20, 20)) + 2 * U) + U * want.abs()
        err = (dz.double() - want).abs()
        tol = tol + halfway(want.abs() + tol, dtype)
        assert bool((err <= tol).all()), float((err / tol).max())
        assert bool((whole[:, n:] == 99.0).all())
        mine = dh.clone()
        assert torch.equal(tdq.activation_backward_fp8(mine, zc, zs, act, dz=mine), dz)
    e = torch.zeros((0, n), device="cuda", dtype=dtype)
    assert tdq.activation_backward_fp8(e, zc[:0], zs[:0], act).shape == (0, n)


@pytest.mark.parametrize("x_type", list(TYPES))
@pytest.mark.parametrize("m,n", [(301, 128), (1, 256), (100, 384), (65, 640), (9, 72), (33, 896)])
def test_activation_backward_of_few_blocks_a_row(tdq, m, n, x_type):
    """A thread's vectors lie in several rows."""
    test_activation_backward(tdq, m, n, 0, x_type, "gelu")


@pytest.mark.parametrize("act", ACTS)
def test_slopes_are_the_values_differences(tdq, act):
    """The epilogue's values at z - d and z + d against the slope at z, both as the kernels compute them."""
    z = torch.linspace(-6, 6, 128 * 40, device="cuda").view(40, 128)
    zc, zs = tdq.quantize_act_fp8(z, pow2=True)
    zr = (zc.float() * zs.repeat_interleave(128, 1))
    s = tdq.activation_backward_fp8(torch.ones_like(zr), zc, zs, act).double()
    d = 2.0 ** -6
    lo, hi = value(act, zr.double() - d), value(act, zr.double() + d)
    smooth = zr.abs() > d if act == "relu" else torch.ones_like(zr, dtype=torch.bool)
    # third derivatives of these functions are below 2: d^2 / 6 x 2
    assert bool(((hi - lo) / (2 * d) - s).abs()[smooth].max() <= d * d / 3 + 2.0 ** -18)


def test_refusals(tdq):
    xc, xs, wc, ws, bias, r = operands(tdq, 8, 200, 40, 0)
    y = torch.zeros((8, 40), device="cuda")
    n0 = tdq.kernel_launch_count()
    for e, f in [(TypeError, lambda: tdq.fp8_linear(xc, xs, wc, ws, y=y, residual=y.half())), (ValueError, lambda: tdq.fp8_linear(xc, xs, wc, ws, y=y, residual=y[:7])),
                 (ValueError, lambda: tdq.fp8_linear(xc, xs, wc, ws, y=y, pre=y.t().contiguous().t())), (ValueError, lambda: tdq.fp8_linear(xc, xs, wc, ws, y=y, pre=y.cpu())),
                 (tdq.TdqError, lambda: tdq.fp8_linear(xc, xs, wc, ws, y=y, pre=y)), (tdq.TdqError, lambda: tdq.fp8_linear(xc, xs, wc, ws, y=y, pre=y + 1, residual=y + 2)),
                 (ValueError, lambda: tdq.activation_backward_fp8(y, xc, xs, "gelu")), (TypeError, lambda: tdq.activation_backward_fp8(y.double(), xc, xs, "gelu"))]:
        with pytest.raises(e):
            f()
    assert tdq.kernel_launch_count() == n0


def test_captured(tdq):
    xc, xs, wc, ws, bias, r = operands(tdq, 900, 512, 777, 9)
    res = r(900, 777)
    want = tdq.fp8_linear(xc, xs, wc, ws, bias, activation="gelu", residual=res)
    y, wsp = torch.zeros_like(want), tdq.fp8_linear_workspace("cuda")
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        tdq.fp8_linear(xc, xs, wc, ws, bias, activation="gelu", residual=res, y=y, workspace=wsp)
    for _ in range(3):
        y.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, want)
