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
