"""The weight gradient where launches follow each other at once, and what a float32 dy's addends are worth in the kernel for large layers."""
import pytest
import torch

from test_gpu_grad import TYPES, check, inputs, restored

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def tdq():
    from paper_2604_16855_b200 import tdq
    return tdq


# Clusters of eight blocks, lanes without channels and rows without outputs in the last ones: blocks leave while others of the next launch start.  4000 tokens are not little work:
# sixteen steps of 2600 clocks and more a block, against less than 21000 in all for the other kernel with the launch of its addends and of what adds the parts.
@pytest.mark.parametrize("m,o,i", [(4000, 65, 129), (1000, 300, 300), (257, 8, 1), (256, 130, 40)])
@pytest.mark.parametrize("dy_type", list(TYPES))
def test_launches_that_follow_at_once(tdq, m, o, i, dy_type):
    sets = [inputs(tdq, m, o, i, TYPES[dy_type], seed=s) for s in (1, 2)]
    outs = [[(torch.zeros((o, i), device="cuda"), torch.zeros((o,), device="cuda")) for _ in range(60)] for _ in sets]
    ws = tdq.fp8_weight_grad_workspace(sets[0][0], i)
    n0 = tdq.kernel_launch_count()
    for n in range(60):
        for (dy, xc, xs), out in zip(sets, outs):
            tdq.fp8_weight_grad(dy, xc, xs, i, dw=out[n][0], db=out[n][1], workspace=ws)
    assert tdq.kernel_launch_count() - n0 == (360 if m == 4000 else 120)
    assert tdq.workspace_status(ws) == (tdq.OK, 0)
    for (dy, xc, xs), out in zip(sets, outs):
        check(*out[0], dy, xc, xs, i, {"bf16": 1, "fp16": 2, "fp32": 3}[dy_type])
        assert all(torch.equal(dw, out[0][0]) and torch.equal(db, out[0][1]) for dw, db in out)


# pieces of one stage and of a few, with and without addends: the last commits and arrivals come when there is little left to do
@pytest.mark.parametrize("m,o,i", [(9217, 63, 147), (64, 5000, 2100), (4617, 960, 320), (20000, 8, 8)])
@pytest.mark.parametrize("dy_type", ["bf16", "fp32"])
def test_large_layers_that_follow_at_once(tdq, m, o, i, dy_type):
    sets = [inputs(tdq, m, o, i, TYPES[dy_type], seed=s) for s in (3, 4)]
    outs = [[(torch.zeros((o, i), device="cuda"), torch.zeros((o,), device="cuda")) for _ in range(20)] for _ in sets]
    ws = tdq.fp8_weight_grad_workspace(sets[0][0], i)
    for n in range(20):
        for (dy, xc, xs), out in zip(sets, outs):
            tdq.fp8_weight_grad(dy, xc, xs, i, dw=out[n][0], db=out[n][1], workspace=ws)
    assert tdq.workspace_status(ws) == (tdq.OK, 0)
    for (dy, xc, xs), out in zip(sets, outs):
        check(*out[0], dy, xc, xs, i, {"bf16": 1, "fp32": 3}[dy_type])
        assert all(torch.equal(dw, out[0][0]) and torch.equal(db, out[0][1]) for dw, db in out)


def launches(tdq, f):
    n0 = tdq.kernel_launch_count()
    out = f()
    return tdq.kernel_launch_count() - n0, out


# Kernels without db: the addends', the sum's and, where tiles are cut, the parts'.  Tiles cut over all clusters, long sums of two tiles, whole tiles with one stage of an addend and with several;
# O off the 16-byte grid or on it
@pytest.mark.parametrize("m,o,i,kernels", [(4096, 2048, 1024, 3), (9000, 300, 200, 3), (5003, 77, 130, 3), (64, 5000, 2100, 2), (190, 5000, 4100, 2)])
@pytest.mark.parametrize("dy_type", ["fp32", "fp16"])
def test_every_bit_of_dy_in_large_layers(tdq, m, o, i, kernels, dy_type):
    """An output has one token, of all bits that its type holds, and x is a power of two: each product, each addend's share and each sum of them is a binary32 number, so dw and
    db are exact.  Without the last addend of a float32 they would be off by 2^-16."""
    dtype = TYPES[dy_type]
    g = torch.Generator(device="cuda")
    g.manual_seed(m + o)
    at = torch.randint(0, m, (o,), generator=g, device="cuda")
    bits = 24 if dtype == torch.float32 else 11
    v = torch.randint(2 ** (bits - 1), 2 ** bits, (o,), generator=g, device="cuda") | 1
    v = (v.double() * torch.exp2(torch.randint(-3, 4, (o,), generator=g, device="cuda").double() - bits) * (1 - 2 * torch.randint(0, 2, (o,), generator=g, device="cuda"))).to(dtype)
    dy = torch.zeros((m, o), dtype=dtype, device="cuda")
    dy[at, torch.arange(o, device="cuda")] = v
    x = torch.exp2(torch.randint(-3, 4, (m, i), generator=g, device="cuda").float()) * (1 - 2 * torch.randint(0, 2, (m, i), generator=g, device="cuda"))
    xc, xs = tdq.quantize_act_fp8(x, pow2=True)
    assert torch.equal(restored(xc, xs, i), x.double())
    n, (dw, none) = launches(tdq, lambda: tdq.fp8_weight_grad(dy, xc, xs, i, bias=False))
    assert n == kernels and none is None
    assert torch.equal(dw.double(), v.double()[:, None] * x[at].double())
    dw2, db = tdq.fp8_weight_grad(dy, xc, xs, i)
    assert torch.equal(dw2, dw) and torch.equal(db, v.float())


# more tokens than the kernel for little work takes (4096)
@pytest.mark.parametrize("m,o,i,pitch", [(5000, 300, 260, 0), (4617, 960, 320, 0), (8193, 129, 640, 3)])
@pytest.mark.parametrize("dy_type", list(TYPES))
@pytest.mark.parametrize("pow2", [True, False])
def test_large_layers_in_binary32(tdq, m, o, i, pitch, dy_type, pow2):
    dy, xc, xs = inputs(tdq, m, o, i, TYPES[dy_type], pitch, seed=21, pow2=pow2)
    dw, db = tdq.fp8_weight_grad(dy, xc, xs, i)
    check(dw, db, dy, xc, xs, i, {"bf16": 1, "fp16": 2, "fp32": 3}[dy_type])


@pytest.mark.parametrize("dy_type", list(TYPES))
def test_values_without_number_in_large_layers(tdq, dy_type):
    m, o, i = 5000, 300, 260
    dy, xc, xs = inputs(tdq, m, o, i, TYPES[dy_type], seed=8)
    clean, cdb = tdq.fp8_weight_grad(dy, xc, xs, i)
    dy[37, 11], dy[4100, 40], xs[4900, 1] = float("nan"), float("-inf"), float("nan")
    xc.view(torch.uint8)[2222, 5] = 0x7f
    dw, db = tdq.fp8_weight_grad(dy, xc, xs, i)
    nan = torch.zeros_like(dw, dtype=torch.bool)
    nan[11], nan[:, 128:256], nan[:, 5] = True, True, True
    x = restored(xc, xs, i)[4100]
    nan[40] |= x == 0                                        # infinity times 0
    assert torch.equal(dw.isnan(), nan)
    rest = ~nan
    rest[40] = False
    assert torch.equal(dw[rest], clean[rest])
    assert torch.equal(dw[40][~nan[40]], -torch.sign(x[~nan[40]]).float() * float("inf"))
    assert bool(db[11].isnan()) and float(db[40]) == float("-inf")
    other = torch.ones_like(db, dtype=torch.bool)
    other[11], other[40] = False, False
    assert torch.equal(db[other], cdb[other])
