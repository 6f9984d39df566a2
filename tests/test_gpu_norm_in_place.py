"""Layer norm and its gradients over their own inputs: the same bits as into other buffers, for every width of group, on the 16-byte grid and off it, many rows a block."""
import pytest
import torch

from test_gpu_norm import TYPES, _inputs

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def tdq():
    from paper_2604_16855_b200 import tdq
    return tdq


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("m,n,pitch", [(9000, 64, 0), (9000, 61, 1), (3000, 768, 0), (3000, 768, 5), (2000, 1001, 0), (1500, 2048, 0), (1200, 2489, 0), (900, 8192, 0), (700, 16384, 0),
                                       (700, 16383, 0)])
def test_over_the_inputs(tdq, m, n, pitch, dtype):
    (x, xw), w, b, (dy, dyw), (add, addw) = _inputs(m, n, dtype, pitch, n)
    y, mean, rstd = tdq.layer_norm(x, w, b)
    dx, dw, db = tdq.layer_norm_backward(dy, x, mean, rstd, w, add=add)
    z = xw.clone()
    assert torch.equal(tdq.layer_norm(z[:, :n], w, b, y=z[:, :n])[0], y)
    assert bool((z[:, n:] == 77.0).all())
    for which in range(3):
        t = [v.clone()[:, :n] for v in (dyw, xw, addw)]
        got = tdq.layer_norm_backward(t[0], t[1], mean, rstd, w, add=t[2], dx=t[which])
        assert torch.equal(got[0], dx) and torch.equal(got[1], dw) and torch.equal(got[2], db)


@pytest.mark.parametrize("n,deep", [(300, 7 + 4), (2000, 4)])
def test_column_sums_of_few_roundings(tdq, n, deep):
    """Sixteen rows of 2000 channels are a block each, and the blocks' sums are added in pairs: four roundings deep, so within 4 x 2^-24 of the sum of magnitudes.  One after
    another the ones would all be lost beside 2^24.  Of 300 channels a block has eight rows, whose sums are added one after another first: seven more."""
    dy = torch.ones((16, n), device="cuda")
    dy[torch.arange(n, device="cuda") % 16, torch.arange(n, device="cuda")] = 2.0 ** 24
    x = torch.arange(n, device="cuda", dtype=torch.float32).sin().repeat(16, 1)
    mean, rstd = torch.zeros((16,), device="cuda"), torch.ones((16,), device="cuda")
    _, dw, db = tdq.layer_norm_backward(dy, x, mean, rstd)
    total = dy.double().sum(0)
    assert bool(((db.double() - total).abs() <= deep * 2.0 ** -24 * total).all())
    # dweight: x is one number a column, whose products round once more
    assert bool(((dw.double() - total * x[0].double()).abs() <= (deep + 1) * 2.0 ** -24 * total * x[0].double().abs()).all())
