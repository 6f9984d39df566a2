"""The activations' slopes far from zero, and beside the values that the 8-bit layer's epilogue computes."""
import pytest
import torch

from test_gpu_epilogue import ACTS, TYPES, U, halfway, slope, value, value_tol

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def tdq():
    from paper_2604_16855_b200 import tdq
    return tdq


FAR = [0.0, 1e-30, 19.0, 20.5, 87.0, 89.0, 127.0, 129.0, 448.0, 1e4, 1.1e13, 1.2e13, 1.3e13, 1.8e19, 2e19, 1e25, 1e30, 3e38]


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("x_type", list(TYPES))
@pytest.mark.parametrize("pitch", [0, 1])
def test_slopes_far_out(tdq, pitch, x_type, act):
    """Every finite input has a finite slope, 1 and 0 at either end.  A magnitude from 248 x 2^120 on has code x scale = 2^128 with a power of two as scale, an infinity of
    binary32: the slope there is the limit.  The tolerance is that of the slopes near zero, whose |z| stops at 20."""
    dtype = TYPES[x_type]
    z0 = torch.tensor(FAR + [3.4e38], device="cuda").view(-1, 1)
    x = torch.zeros((2 * z0.shape[0], 136), device="cuda")
    x[:, 5:6], x[:, 129:136] = torch.cat([z0, -z0]), torch.cat([-z0, z0])
    dh = torch.full((x.shape[0], 136 + pitch), -0.75, device="cuda", dtype=dtype)[:, :136]
    for pow2 in (True, False):
        zc, zs = tdq.quantize_act_fp8(x, pow2=pow2)
        z = (zc.float().view(-1, 2, 128) * zs[:, :, None]).view(-1, 256)[:, :136]
        assert not bool(z.isnan().any()) and bool(z.isinf().any()) == pow2
        z = z.double().clamp(-1e30, 1e30)
        want = dh.double() * slope(act, z)
        tol = dh.double().abs() * (value_tol(act, z.clamp(-20, 20)) + 2 * U) + U * want.abs()
        dz = tdq.activation_backward_fp8(dh, zc, zs, act)
        err = (dz.double() - want).abs()
        assert bool((err <= tol + halfway(want.abs() + tol, dtype)).all()), (act, pow2, float(err.max()))


@pytest.mark.parametrize("act", ACTS)
def test_slopes_of_what_is_no_number(tdq, act):
    x = torch.ones((3, 256), device="cuda")
    x[1, 200] = float("nan")
    zc, zs = tdq.quantize_act_fp8(x, pow2=True)
    dz = tdq.activation_backward_fp8(torch.ones_like(x), zc, zs, act)
    bad = torch.zeros_like(x, dtype=torch.bool)
    bad[1, 128:] = act != "relu"                             # NaN > 0 does not hold: RELU's slope is 0
    assert torch.equal(dz.isnan(), bad)
    assert act != "relu" or bool((dz[1, 128:] == 0).all())


@pytest.mark.parametrize("act", ACTS)
def test_slopes_are_the_epilogues_differences(tdq, act):
    """The layer's own activation(z + d) - activation(z - d), z given as the bias of a layer of zeros, against the slope that the backward pass multiplies by.

    value_tol of either value over 2 d, of the slope itself, and d^2 / 6 times the third derivative, which stays below 2 for |z| <= 6 (0.8 at most)."""
    d = 2.0 ** -6
    z = torch.linspace(-6, 6, 128 * 40, device="cuda").view(40, 128)
    zc, zs = tdq.quantize_act_fp8(z, pow2=True)
    zr = zc.float() * zs
    s = tdq.activation_backward_fp8(torch.ones_like(zr), zc, zs, act).double()
    xc, xs = tdq.quantize_act_fp8(torch.zeros((1, 128), device="cuda"))
    wc, ws = tdq.quantize_weight_fp8(torch.zeros((128 * 40, 128), device="cuda"))
    # code +- d is exact in binary32: four bits from 2^-9 2^-7 on and 2^-6
    hi, lo = (tdq.fp8_linear(xc, xs, wc, ws, (zr + e).flatten(), activation=act).view(40, 128).double() for e in (d, -d))
    smooth = zr.abs() > d if act == "relu" else torch.ones_like(zr, dtype=torch.bool)
    tol = (value_tol(act, zr.double().abs() + d) + halfway(value(act, zr.double().abs() + d), torch.float32)) / d + value_tol(act, zr.double()) + 2 * U + d * d / 3
    assert bool((((hi - lo) / (2 * d) - s).abs() <= tol)[smooth].all())
