"""Weight and bias gradients from activations kept in 8 bits against the formula in 64 bits.

Products of bf16 numbers are exact in binary32.  An accumulator takes 32 instructions of 16 products (512 tokens of an addend), each of which may drop up to a step
of the accumulator's last place (2^-23 of it) for the sum so far and again for the products that it aligns; the rest are binary32 additions.  So an element is off by at most
2^-23 x (2 x 32 + 16 + additions) times the sum of its terms' magnitudes."""
import pytest
import torch

import fp8_utils as fu

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}


@pytest.fixture(scope="module")
def tdq():
    from paper_2604_16855_b200 import tdq
    return tdq


def inputs(tdq, m, o, i, dtype, pitch=0, seed=0, pow2=True):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed + m + o + i)
    r = lambda *s: torch.randn(s, generator=g, device="cuda")  # noqa: E731
    dy = torch.full((m, o + pitch), 77.0, dtype=dtype, device="cuda")[:, :o]
    dy.copy_(0.1 * r(m, o) * torch.exp(r(m, 1)))
    xc, xs = tdq.quantize_act_fp8(r(m, i) * torch.exp(0.5 * r(m, 1)) + r(1, i), pow2=pow2)
    return dy, xc, xs


def restored(xc, xs, i):
    m, k = xs.shape
    x = (xc.float().view(m, k, 128) * xs[:, :, None]).to(torch.bfloat16)
    return x.double().view(m, -1)[:, :i]


def check(dw, db, dy, xc, xs, i, parts):
    m = dy.shape[0]
    x, d = restored(xc, xs, i), dy.double()
    want, size = d.t() @ x, d.abs().t() @ x.abs()
    more = parts * m / 512 + 148
    tol = 2 * U * (64 + 16 + more) * size
    fi = torch.finfo(dw.dtype)
    if dw.dtype != torch.float32:
        tol = tol + fi.eps / 2 * (want.abs() + tol) + fi.tiny * fi.eps / 2
    err = (dw.double() - want).abs()
    assert bool((err <= tol).all()), float((err / tol.clamp_min(1e-300)).max())
    if db is not None:                                       # a thread adds every sixteenth token of its piece, a warp two, eight warps, the pieces
        err = (db.double() - d.sum(0)).abs()
        assert bool((err <= U * (parts * (m / 16 + 4) + 12 + 148) * d.abs().sum(0)).all())
    return err


# one tile and less, tiles cut over all clusters, many whole tiles; tokens below a stage, of one stage, of an accumulator's eight and around them
SIZES = [(1, 1, 1), (1, 256, 256), (3, 7, 130), (63, 200, 64), (64, 256, 128), (65, 257, 300), (511, 96, 256), (512, 128, 640), (513, 300, 257), (4617, 960, 320),
         (2000, 1000, 1000), (100, 4096, 1000), (64, 5000, 2100), (9217, 63, 147), (1500, 2304, 768), (300, 2600, 2560)]


@pytest.mark.parametrize("m,o,i", SIZES)
@pytest.mark.parametrize("dy_type,dw_type,pitch", [("bf16", "fp32", 0), ("bf16", "bf16", 8), ("bf16", "fp16", 1), ("fp16", "fp32", 3), ("fp32", "fp16", 0)])
def test_gradients(tdq, m, o, i, dy_type, dw_type, pitch):
    dy, xc, xs = inputs(tdq, m, o, i, TYPES[dy_type], pitch)
    ws = tdq.fp8_weight_grad_workspace(dy, i)
    whole = torch.full((o, i + pitch), 55.0, dtype=TYPES[dw_type], device="cuda")
    dw, db = tdq.fp8_weight_grad(dy, xc, xs, i, dw=whole[:, :i], workspace=ws)
    assert tdq.workspace_status(ws) == (tdq.OK, 0)
    check(dw, db, dy, xc, xs, i, {"bf16": 1, "fp16": 2, "fp32": 3}[dy_type])
    assert bool((whole[:, i:] == 55.0).all())
    again, none = tdq.fp8_weight_grad(dy, xc, xs, i, out_dtype=TYPES[dw_type], bias=False)
    assert none is None and torch.equal(again, dw)


def test_scales_that_are_no_powers_of_two(tdq):
    dy, xc, xs = inputs(tdq, 700, 300, 500, torch.bfloat16, pow2=False)
    dw, db = tdq.fp8_weight_grad(dy, xc, xs, 500)
    check(dw, db, dy, xc, xs, 500, 1)


def test_exact_where_sums_are(tdq):
    """Whole numbers below 2^24 in all: every addition is exact, so is the result, whatever the order."""
    g = torch.Generator(device="cuda")
    g.manual_seed(5)
    m, o, i = 3000, 520, 400
    for dtype in TYPES.values():
        dy = torch.randint(-8, 9, (m, o), generator=g, device="cuda").to(dtype)
        x = torch.randint(-16, 17, (m, i), generator=g, device="cuda").float()
        xc, xs = tdq.quantize_act_fp8(x, pow2=True)
        assert torch.equal(restored(xc, xs, i), x.double())  # up to 16 fits in four bits and a power of two
        dw, db = tdq.fp8_weight_grad(dy, xc, xs, i)
        assert torch.equal(dw.double(), dy.double().t() @ x.double()) and torch.equal(db.double(), dy.double().sum(0))


def test_full_precision_of_dy(tdq):
    """One token: a product each, so the gradient of a float32 or fp16 dy has to be right to the last place but one."""
    for dtype in (torch.float32, torch.float16):
        dy, xc, xs = inputs(tdq, 1, 777, 200, dtype, seed=3)
        dw, _ = tdq.fp8_weight_grad(dy, xc, xs, 200)
        want = dy.double().t() @ restored(xc, xs, 200)
        assert bool(((dw.double() - want).abs() <= 8 * U * want.abs()).all())


def test_values_without_number(tdq):
    dy, xc, xs = inputs(tdq, 600, 300, 260, torch.float32)
    clean, cdb = tdq.fp8_weight_grad(dy, xc, xs, 260)
    dy[37, 11] = float("nan")
    xs[500, 1] = float("nan")
    dw, db = tdq.fp8_weight_grad(dy, xc, xs, 260)
    bad = torch.zeros_like(dw, dtype=torch.bool)
    bad[11], bad[:, 128:256] = True, True
    assert torch.equal(dw.isnan(), bad) and torch.equal(dw[~bad], clean[~bad])
    assert torch.equal(db.isnan(), torch.arange(300, device="cuda") == 11)


def test_empty(tdq):
    z = torch.zeros((0, 40), device="cuda", dtype=torch.bfloat16)
    xc, xs = torch.zeros((0, 128), dtype=torch.uint8, device="cuda"), torch.zeros((0, 1), device="cuda")
    whole = torch.full((40, 100), 3.0, device="cuda")
    dw, db = tdq.fp8_weight_grad(z, xc, xs, 90, dw=whole[:, :90])
    assert bool((whole[:, :90] == 0).all()) and bool((whole[:, 90:] == 3).all()) and bool((db == 0).all())


def test_refusals(tdq):
    dy, xc, xs = inputs(tdq, 8, 40, 90, torch.bfloat16)
    n0 = tdq.kernel_launch_count()
    small = torch.zeros((16,), dtype=torch.uint8, device="cuda")
    for e, f in [(TypeError, lambda: tdq.fp8_weight_grad(dy.double(), xc, xs, 90)), (ValueError, lambda: tdq.fp8_weight_grad(dy, xc, xs, 129)),
                 (ValueError, lambda: tdq.fp8_weight_grad(dy, xc, xs, 0)), (ValueError, lambda: tdq.fp8_weight_grad(dy[:7], xc, xs, 90)),
                 (TypeError, lambda: tdq.fp8_weight_grad(dy, xc.float(), xs, 90)), (ValueError, lambda: tdq.fp8_weight_grad(dy.t(), xc, xs, 90)),
                 (ValueError, lambda: tdq.fp8_weight_grad(dy, xc, xs, 90, dw=torch.zeros((90, 40), device="cuda").t())),
                 (ValueError, lambda: tdq.fp8_weight_grad(dy, xc, xs, 90, db=torch.zeros((39,), device="cuda"))),
                 (ValueError, lambda: tdq.fp8_weight_grad(dy, xc, xs, 90, db=torch.zeros((40,), device="cuda"), bias=False)),
                 (tdq.TdqError, lambda: tdq.fp8_weight_grad(dy, xc, xs, 90, workspace=small)), (ValueError, lambda: tdq.fp8_weight_grad(dy, xc, xs.cpu(), 90))]:
        with pytest.raises(e):
            f()
    assert tdq.kernel_launch_count() == n0


def test_captured_on_another_stream(tdq):
    for dtype in (torch.bfloat16, torch.float32):
        dy, xc, xs = inputs(tdq, 1200, 700, 500, dtype)
        want = tdq.fp8_weight_grad(dy, xc, xs, 500)
        ws = tdq.fp8_weight_grad_workspace(dy, 500)
        dw, db = torch.zeros_like(want[0]), torch.zeros_like(want[1])
        s = torch.cuda.Stream()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            tdq.fp8_weight_grad(dy, xc, xs, 500, dw=dw, db=db, workspace=ws)
        for _ in range(3):
            dw.zero_(), db.zero_()
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(dw, want[0]) and torch.equal(db, want[1])


def test_both_kernels_run(tdq):
    """Little work is one launch, whatever dy's type and with db; a long or a wide sum takes the kernel for large layers, one more launch for what is cut or for db, one more
    for dy's addends."""
    for m, o, i, dtype, launches in [(64, 96, 200, torch.float32, 1), (500, 300, 500, torch.bfloat16, 1), (1, 4096, 1000, torch.float16, 1), (20000, 64, 64, torch.bfloat16, 2),
                                     (4096, 2048, 1024, torch.bfloat16, 2), (4096, 2048, 1024, torch.float16, 3)]:
        dy, xc, xs = inputs(tdq, m, o, i, dtype)
        n0 = tdq.kernel_launch_count()
        tdq.fp8_weight_grad(dy, xc, xs, i)
        assert tdq.kernel_launch_count() - n0 == launches, (m, o, i, dtype)


# every number of parts of the tokens that the kernel for little work takes, and ragged ends in each direction
@pytest.mark.parametrize("m", [1, 31, 33, 65, 97, 129, 161, 193, 225, 400, 512, 513, 1024, 2000, 4000])
@pytest.mark.parametrize("o,i", [(8, 128), (65, 129), (130, 40)])
@pytest.mark.parametrize("dy_type,pitch", [("bf16", 0), ("fp32", 8), ("fp16", 1)])
def test_little_work(tdq, m, o, i, dy_type, pitch):
    dy, xc, xs = inputs(tdq, m, o, i, TYPES[dy_type], pitch, seed=11)
    for dw_type in (torch.float32, torch.bfloat16):
        whole = torch.full((o, i + 3), 55.0, dtype=dw_type, device="cuda")
        ws = tdq.fp8_weight_grad_workspace(dy, i)
        ws.fill_(255)
        dw, db = tdq.fp8_weight_grad(dy, xc, xs, i, dw=whole[:, :i], workspace=ws)
        assert tdq.workspace_status(ws) == (tdq.OK, 0) and bool((whole[:, i:] == 55.0).all())
        check(dw, db, dy, xc, xs, i, {"bf16": 1, "fp16": 2, "fp32": 3}[dy_type])
