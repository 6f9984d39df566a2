"""Layer norm and its gradients against the formulas in 64 bits: every width of group, rows on the grid and off it, both kinds of output.

Tolerances count roundings.  A sum over a row is at most 32 additions of a thread, ten of a butterfly and a few products: DEEP of them.  A column's sum is one
addition for each row of a group, then 16 groups, then the blocks."""
import pytest
import torch

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
DEEP = 48
TYPES = [torch.float32, torch.bfloat16, torch.float16]
# warps, several warps, many of them; vectors 1 .. 4 a thread (8 for long rows of binary32, backward)
SIZES = [(1, 1), (3, 7), (5, 8), (2, 63), (33, 64), (700, 128), (3, 130), (611, 500), (601, 512), (700, 768), (4, 768), (601, 1000), (593, 1024), (3, 1024),
         (2, 1025), (600, 1500), (599, 2048), (2, 2304), (594, 4096), (3, 4096), (2, 5000), (593, 8192), (2, 8192), (1, 8200), (3, 16384), (593, 16384),
         (600, 15000), (593, 6001), (700, 192), (594, 12000)]


@pytest.fixture(scope="module")
def tdq():
    from paper_2604_16855_b200 import tdq
    return tdq


def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _pitched(values, dtype, pitch):
    """The values as a view whose rows are `pitch` elements longer; what lies between them is 77."""
    m, n = values.shape
    whole = torch.full((m, n + pitch), 77.0, dtype=dtype, device="cuda")
    whole[:, :n] = values.to(dtype)
    return whole[:, :n], whole


def _inputs(m, n, dtype, pitch, seed):
    g = _gen(seed)
    r = lambda *s: torch.randn(s, generator=g, device="cuda")  # noqa: E731
    x = (r(m, n) * torch.exp(0.5 * r(m, 1)) + 2.0 * r(1, n)).to(dtype)
    return _pitched(x, dtype, pitch), 1.0 + 0.2 * r(n), 0.2 * r(n), _pitched(r(m, n) * 0.1, dtype, pitch), _pitched(r(m, n) * 0.1, dtype, pitch)


def _exact(x, w, b, eps):
    x = x.double()
    mean = x.mean(1, keepdim=True)
    rstd = 1.0 / torch.sqrt(((x - mean) ** 2).mean(1, keepdim=True) + eps)
    hat = (x - mean) * rstd
    far = DEEP * U * x.abs().mean(1, keepdim=True)                  # of the mean
    tol_rstd = rstd * ((DEEP / 2 + 4) * U + (far * rstd) ** 2)
    wd = torch.ones_like(x[0]) if w is None else w.double()
    bd = torch.zeros_like(x[0]) if b is None else b.double()
    y = hat * wd + bd
    tol = wd.abs() * (rstd * far + hat.abs() * (tol_rstd / rstd + 4 * U)) + 2 * U * bd.abs()
    return y, tol * 1.01, mean[:, 0], (far + 2 * U * mean.abs())[:, 0], rstd[:, 0], tol_rstd[:, 0]


def _within(got, want, tol, dtype=torch.float32):
    fi = torch.finfo(dtype)
    step = 0.0 if dtype == torch.float32 else fi.eps / 2 * (want.abs() + tol) + fi.tiny * fi.eps / 2
    err = (got.double() - want).abs()
    assert bool((err <= tol + step).all()), float((err / (tol + step)).max())


@pytest.mark.parametrize("dtype", TYPES, ids=["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("pitch", [0, 8, 1])
@pytest.mark.parametrize("m,n", SIZES)
def test_forward(tdq, m, n, pitch, dtype):
    (x, _), w, b, _, _ = _inputs(m, n, dtype, pitch, m + 3 * n)
    out, whole = _pitched(torch.zeros(m, n, device="cuda"), dtype, pitch)
    y, mean, rstd = tdq.layer_norm(x, w, b, eps=1e-5, y=out)
    want, tol, mu, tmu, rs, trs = _exact(x, w, b, 1e-5)
    _within(y, want, tol, dtype)
    _within(mean, mu, tmu)
    _within(rstd, rs, trs)
    assert y is out and bool((whole[:, n:] == 77.0).all())
    y, _, _ = tdq.layer_norm(x, eps=0.5)
    want, tol = _exact(x, None, None, 0.5)[:2]
    _within(y, want, tol, dtype)
    assert y.is_contiguous()


def _half_step(v):
    """Half a step of E4M3 at |v|: 2^-4 of its power of two, 2^-10 below 2^-6."""
    _, e = torch.frexp(v.abs().clamp_max(448.0))
    return torch.ldexp(torch.ones_like(v), torch.clamp(e - 1, min=-6) - 4)


@pytest.mark.parametrize("dtype", TYPES, ids=["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("pow2", [False, True], ids=["any", "pow2"])
@pytest.mark.parametrize("m,n", SIZES)
def test_codes(tdq, m, n, pow2, dtype):
    (x, _), w, b, _, _ = _inputs(m, n, dtype, (m + n) % 3, m + 5 * n)
    codes, scale, mean, rstd = tdq.layer_norm_fp8(x, w, b, pow2=pow2)
    want, tol, mu, tmu, rs, trs = _exact(x, w, b, 1e-5)
    _within(mean, mu, tmu)
    _within(rstd, rs, trs)
    k = (n + 127) // 128
    assert codes.shape == (m, k * 128) and scale.shape == (m, k) and bool((codes[:, n:].float() == 0).all())
    pad = lambda t: torch.nn.functional.pad(t, (0, k * 128 - n)).view(m, k, 128)  # noqa: E731
    y, t = pad(want), pad(tol)
    top, far = y.abs().amax(2), t.amax(2)
    s = scale.double()
    if pow2:
        assert bool((torch.frexp(scale)[0] == 0.5).all())
        assert bool((top - far <= 448.0 * s).all()) and bool((top + far >= 224.0 * s).all())
    else:
        assert bool(((s - top / 448.0).abs() <= far / 448.0 + 2 * U * top / 448.0).all())
    value = codes.double().view(m, k, 128)
    q = y / s[:, :, None]
    near = t / s[:, :, None] + 4 * U * q.abs()
    assert bool(((value - q).abs() <= _half_step(q.abs() + near) + near).all())


@pytest.mark.parametrize("n", [128, 768, 1024, 4096, 16384])
@pytest.mark.parametrize("m", [3, 601])
def test_codes_are_the_quantizers(tdq, m, n):
    """With binary32 rows of whole blocks the two calls and the one give the same bits."""
    (x, _), w, b, _, _ = _inputs(m, n, torch.float32, 0, n)
    y, mean, rstd = tdq.layer_norm(x, w, b)
    for pow2 in (False, True):
        c, s, mu, rs = tdq.layer_norm_fp8(x, w, b, pow2=pow2)
        c2, s2 = tdq.quantize_act_fp8(y, pow2=pow2)
        assert torch.equal(c.view(torch.uint8), c2.view(torch.uint8)) and torch.equal(s, s2) and torch.equal(mu, mean) and torch.equal(rs, rstd)


@pytest.mark.parametrize("dtype", TYPES, ids=["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("pitch", [0, 8, 1])
@pytest.mark.parametrize("m,n", SIZES)
def test_backward(tdq, m, n, pitch, dtype):
    (x, _), w, _, (dy, _), (add, _) = _inputs(m, n, dtype, pitch, m + 7 * n)
    _, mean, rstd = tdq.layer_norm(x, w)
    for weight, more in ((w, None), (None, add), (w, add)):
        out, whole = _pitched(torch.zeros(m, n, device="cuda"), dtype, pitch)
        dx, dw, db = tdq.layer_norm_backward(dy, x, mean, rstd, weight, add=more, dx=out)
        d, h = dy.double(), (x.double() - mean.double()[:, None]) * rstd.double()[:, None]
        g = d if weight is None else d * w.double()
        r = rstd.double()[:, None]
        gh = (g * h).mean(1, keepdim=True)
        want = r * (g - g.mean(1, keepdim=True) - h * gh)
        tol = r * U * (6 * g.abs() + (DEEP + 6) * g.abs().mean(1, keepdim=True) + (DEEP + 10) * h.abs() * (g * h).abs().mean(1, keepdim=True))
        if more is not None:
            want = want + add.double()
            tol = tol + 2 * U * (add.double().abs() + want.abs())
        _within(dx, want, tol, dtype)
        deep = m / 148 + 16 + 10 + 16 + 8
        _within(dw, (d * h).sum(0), deep * U * (d * h).abs().sum(0))
        _within(db, d.sum(0), deep * U * d.abs().sum(0))
        assert bool((whole[:, n:] == 77.0).all())
        again = tdq.layer_norm_backward(dy, x, mean, rstd, weight, add=more)
        assert all(torch.equal(p, q) for p, q in zip(again, (dx, dw, db)))


@pytest.mark.parametrize("m,n", [(5, 24), (3, 129), (40, 768)])
def test_gradients_against_differences(tdq, m, n):
    g = _gen(n)
    r = lambda *s: torch.randn(s, generator=g, device="cuda")  # noqa: E731
    x, w, b, dy = r(m, n), 1 + 0.2 * r(n), r(n), r(m, n)
    _, mean, rstd = tdq.layer_norm(x, w, b)
    dx, dw, db = tdq.layer_norm_backward(dy, x, mean, rstd, w)

    def loss(x, w, b):
        return (_exact(x, w, b, 1e-5)[0] * dy.double()).sum()
    e = 1e-5
    for _ in range(3):
        u, v, t = r(m, n).double(), r(n).double(), r(n).double()
        diff = (loss(x.double() + e * u, w.double() + e * v, b.double() + e * t) - loss(x.double() - e * u, w.double() - e * v, b.double() - e * t)) / (2 * e)
        mine = (dx.double() * u).sum() + (dw.double() * v).sum() + (db.double() * t).sum()
        size = (dx.double() * u).abs().sum() + (dw.double() * v).abs().sum() + (db.double() * t).abs().sum()
        # binary32's gradients: DEEP roundings of each term; the difference's own error is e^2 of the third derivative, 1e-8 or so of the terms
        assert abs(float(diff - mine)) <= float(size) * (2 * DEEP * U + 1e-7)


def test_far_mean_and_constant_rows(tdq):
    """A mean 10^4 deviations away costs what the inputs' own rounding costs; a row without spread gives 0 (the bias), not NaN."""
    g = _gen(0)
    x = 1e4 + torch.randn((64, 1000), generator=g, device="cuda")
    y, mean, rstd = tdq.layer_norm(x)
    want, tol, mu, tmu, rs, trs = _exact(x, None, None, 1e-5)
    _within(y, want, tol)
    _within(rstd, rs, trs)
    b = torch.randn((1000,), generator=g, device="cuda")
    y, mean, rstd = tdq.layer_norm(torch.full((3, 1000), 2.0, device="cuda"), None, b)
    assert torch.equal(y, b.expand(3, 1000)) and bool((mean == 2.0).all())
    c, s, _, _ = tdq.layer_norm_fp8(torch.full((3, 1000), 2.0, device="cuda"))
    assert bool((c.float() == 0).all()) and bool((s == 2.0 ** -64 / 448).all())


def test_nan_stays_in_its_row(tdq):
    x = torch.randn((20, 768), device="cuda", dtype=torch.bfloat16)
    x[3, 5], x[11, 700] = float("nan"), float("inf")
    y, _, _ = tdq.layer_norm(x)
    c, s, _, _ = tdq.layer_norm_fp8(x)
    for m in range(20):
        bad = m in (3, 11)
        assert bool(y[m].isnan().all()) == bad and bool(s[m].isnan().all()) == bad and bool(c[m].float().isnan().all()) == bad


@pytest.mark.parametrize("n", [768, 1001])
def test_in_place(tdq, n):
    (x, _), w, b, (dy, _), (add, _) = _inputs(700, n, torch.bfloat16, 0, n)
    y, mean, rstd = tdq.layer_norm(x, w, b)
    dx, dw, db = tdq.layer_norm_backward(dy, x, mean, rstd, w, add=add)
    for which in range(3):
        t = [v.clone() for v in (dy, x, add)]
        got = tdq.layer_norm_backward(t[0], t[1], mean, rstd, w, add=t[2], dx=t[which])
        assert torch.equal(got[0], dx) and torch.equal(got[1], dw) and torch.equal(got[2], db)
    z = x.clone()
    assert torch.equal(tdq.layer_norm(z, w, b, y=z)[0], y)


def test_more_dimensions_empty_inputs_and_outputs_left_alone(tdq):
    x = torch.randn((2, 5, 3, 64), device="cuda")
    y, mean, rstd = tdq.layer_norm(x)
    assert y.shape == x.shape and mean.shape == (30,)
    assert torch.equal(y.view(30, 64), tdq.layer_norm(x.view(30, 64))[0])
    t = x.transpose(1, 2)                                        # rows unevenly spaced: brought together
    assert torch.equal(tdq.layer_norm(t)[0], y.transpose(1, 2))
    dx, dw, db = tdq.layer_norm_backward(x, x, mean, rstd)
    assert dx.shape == x.shape and dw.shape == db.shape == (64,)
    e = torch.zeros((0, 64), device="cuda")
    none = torch.zeros((0,), device="cuda")
    y, mean, rstd = tdq.layer_norm(e)
    assert y.shape == (0, 64) and mean.shape == (0,)
    assert [t.shape[0] for t in tdq.layer_norm_fp8(e)] == [0, 0, 0, 0]
    dx, dw, db = tdq.layer_norm_backward(e, e, none, none)
    assert dx.shape == (0, 64) and bool((dw == 0).all()) and bool((db == 0).all())


def test_refusals(tdq):
    x, w = torch.zeros((4, 64), device="cuda"), torch.ones((64,), device="cuda")
    m = torch.zeros((4,), device="cuda")
    n0 = tdq.kernel_launch_count()
    for e, f in [(TypeError, lambda: tdq.layer_norm(x.double())), (TypeError, lambda: tdq.layer_norm(x, w.half())), (ValueError, lambda: tdq.layer_norm(x, w[:32])),
                 (ValueError, lambda: tdq.layer_norm(x.t())), (TypeError, lambda: tdq.layer_norm(x, y=x.half())), (ValueError, lambda: tdq.layer_norm(x, y=x[:2])),
                 (ValueError, lambda: tdq.layer_norm(x, mean=m[:3])), (ValueError, lambda: tdq.layer_norm(x.cpu())),
                 (ValueError, lambda: tdq.layer_norm_fp8(x, codes=torch.zeros((4, 64), dtype=torch.uint8, device="cuda"))),
                 (ValueError, lambda: tdq.layer_norm_fp8(x, scale=torch.zeros((4, 2), device="cuda"))),
                 (TypeError, lambda: tdq.layer_norm_backward(x.half(), x, m, m)), (ValueError, lambda: tdq.layer_norm_backward(x[:3], x, m, m)),
                 (ValueError, lambda: tdq.layer_norm_backward(x, x, m[:3], m)), (TypeError, lambda: tdq.layer_norm_backward(x, x, m, m, add=x.half())),
                 (ValueError, lambda: tdq.layer_norm_backward(x, x, m, m, dweight=m)),
                 (tdq.TdqError, lambda: tdq.layer_norm_backward(x, x, m, m, workspace=torch.zeros((16,), dtype=torch.uint8, device="cuda"))),
                 (tdq.TdqError, lambda: tdq.layer_norm(torch.zeros((1, 16385), device="cuda"))), (tdq.TdqError, lambda: tdq.layer_norm(x, eps=-1.0))]:
        with pytest.raises(e):
            f()
    assert tdq.kernel_launch_count() == n0


def test_captured_on_another_stream(tdq):
    (x, _), w, b, (dy, _), _ = _inputs(300, 768, torch.bfloat16, 0, 1)
    y, mean, rstd = tdq.layer_norm(x, w, b)
    want = tdq.layer_norm_backward(dy, x, mean, rstd, w)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    out, dx, dw, db = torch.zeros_like(y), torch.zeros_like(y), torch.zeros_like(w), torch.zeros_like(w)
    ws = torch.zeros((148 * 2 * 768 * 4 * 2,), dtype=torch.uint8, device="cuda")
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=s):
        tdq.layer_norm(x, w, b, y=out, mean=mean, rstd=rstd)
        tdq.layer_norm_backward(dy, x, mean, rstd, w, dx=dx, dweight=dw, dbias=db, workspace=ws)
    for _ in range(3):
        out.zero_(), dx.zero_(), dw.zero_(), db.zero_(), mean.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, y) and torch.equal(dx, want[0]) and torch.equal(dw, want[1]) and torch.equal(db, want[2])
