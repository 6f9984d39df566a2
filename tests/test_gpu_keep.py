"""Activations kept in 8 bits: the quantizer with power-of-two scales, bit for bit."""
import pytest
import torch

import fp8_utils as fu

pytestmark = pytest.mark.gpu
TYPES = [torch.float32, torch.bfloat16, torch.float16]


@pytest.fixture(scope="module")
def tdq():
    from paper_2604_16855_b200 import tdq
    return tdq


def plain(x):
    m, n = x.shape
    k = fu.blocks(n)
    p = torch.nn.functional.pad(x.float(), (0, k * 128 - n)).view(m, k, 128)
    mantissa, exponent = torch.frexp(p.abs().amax(2).clamp_min(2.0 ** -64))
    scale = torch.ldexp(torch.ones_like(mantissa), exponent - 9 + (mantissa > 0.875).int())      # 448 = 0.875 2^9
    return (p / scale[:, :, None]).to(torch.float8_e4m3fn).view(m, k * 128), scale


@pytest.mark.parametrize("dtype", TYPES, ids=["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("m,n,pitch", [(1, 1, 0), (3, 64, 0), (577, 768, 0), (100, 1000, 1), (33, 300, 0), (40, 130, 3), (64, 147, 0), (5, 4096, 8)])
def test_pow2_scales(tdq, m, n, pitch, dtype):
    g = torch.Generator(device="cuda")
    g.manual_seed(m + n)
    x = torch.zeros((m, n + pitch), dtype=dtype, device="cuda")[:, :n]
    x.copy_(torch.randn((m, n), generator=g, device="cuda") * torch.exp(torch.randn((m, 1), generator=g, device="cuda")))
    x[0, 0] = 448.0                                          # at the border, and next to it on either side
    if m > 2:
        x[1], x[2] = 0.0, x[2] / x[2].abs().max() * 3.5
    codes, scale = tdq.quantize_act_fp8(x, pow2=True)
    want, ws = plain(x)
    assert torch.equal(scale, ws)
    assert torch.equal(codes.view(torch.uint8) & 0x7f, want.view(torch.uint8) & 0x7f) and torch.equal(codes.float(), want.float())


def test_borders_and_values_without_number(tdq):
    v = torch.tensor([448.0, 448.0 + 2 ** -15, 449.0, 224.0, 2.0 ** -64, 0.0, 2.0 ** -70, 1.75 * 2.0 ** -60, float("inf"), float("nan"), 1.0, 1.75, 1.76, 3e38],
                     device="cuda")
    x = torch.zeros((v.numel(), 200), device="cuda")
    x[:, 130] = v
    codes, scale = tdq.quantize_act_fp8(x, pow2=True)
    want, ws = plain(torch.where(x.isfinite(), x, torch.zeros_like(x)))
    fine = v.isfinite()
    assert torch.equal(scale[fine], ws[fine]) and torch.equal(codes[fine].float(), want[fine].float())
    assert bool(scale[~fine, 1].isnan().all()) and bool(codes[~fine, 128:].float().isnan().all()) and torch.equal(scale[~fine, 0], ws[~fine, 0])
    restored = codes[fine].float() * scale[fine].repeat_interleave(128, 1)
    bf = restored.to(torch.bfloat16).float()
    assert torch.equal(bf, restored)                         # bf16 numbers, all of them
