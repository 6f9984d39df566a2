"""Refusals of what stands around the 8-bit layer, before anything is launched (no GPU needed)."""
import ctypes

import pytest
import torch

FAKE = ctypes.c_void_p(0x1000)      # never dereferenced: every call below fails its checks or has nothing to do
ODD = ctypes.c_void_p(0x1001)
OFF4 = ctypes.c_void_p(0x1004)


@pytest.fixture(scope="module")
def tdq():
    from paper_2604_16855_b200 import build
    build.build()
    from paper_2604_16855_b200 import tdq
    return tdq


@pytest.fixture(autouse=True)
def nothing_launched(tdq):
    n0 = tdq.kernel_launch_count()
    yield
    assert tdq.kernel_launch_count() == n0


def _each(f, good, changes):
    for change in changes:
        args = list(good)
        for at, value in change[:-1]:
            args[at] = value
        assert f(*args) == change[-1], change


def test_pow2_quantizer(tdq):
    inv, ali, uns = tdq.ERR_INVALID_ARG, tdq.ERR_ALIGNMENT, tdq.ERR_UNSUPPORTED
    _each(tdq.lib().tdq_quantize_act_fp8_pow2, [FAKE, 1, 2, 4, 64, 64, FAKE, FAKE, None],
          [((i, v), c) for i, v, c in [(0, None, inv), (1, 3, inv), (2, -1, inv), (3, -1, inv), (4, 0, inv), (5, 63, inv), (6, None, inv), (7, None, inv),
                                       (0, ODD, ali), (6, OFF4, ali), (7, ODD, ali), (3, 1 << 30, uns), (3, 0, tdq.OK)]])


def test_layer_norm(tdq):
    inv, ali, uns = tdq.ERR_INVALID_ARG, tdq.ERR_ALIGNMENT, tdq.ERR_UNSUPPORTED
    f = tdq.lib().tdq_layer_norm
    #       x     dt M  C   xst w     b     eps   fl y     yst codes scale mean  rstd  stream
    good = [FAKE, 1, 4, 64, 64, FAKE, FAKE, 1e-5, 0, FAKE, 64, None, None, FAKE, FAKE, None]
    one = lambda *cs: [((i, v), c) for i, v, c in cs]  # noqa: E731
    _each(f, good, one((0, None, inv), (1, 3, inv), (1, -1, inv), (2, -1, inv), (3, 0, inv), (4, 63, inv), (7, -1.0, inv), (7, float("nan"), inv), (8, 1, inv),
                       (8, 2, inv), (9, None, inv), (10, 63, inv), (11, FAKE, inv), (12, FAKE, inv), (0, ODD, ali), (5, ODD, ali), (6, ODD, ali), (9, ODD, ali),
                       (13, ODD, ali), (14, ODD, ali), (2, 1 << 31, uns), (2, 0, tdq.OK)))
    _each(f, good, [((3, 16385), (4, 16385), (10, 16385), uns)])
    codes = good[:9] + [None, 0, FAKE, FAKE, None, None, None]
    _each(f, codes, one((11, None, inv), (12, None, inv), (11, OFF4, ali), (12, ODD, ali), (8, 4, inv), (0, None, inv), (2, 0, tdq.OK)))
    _each(f, codes, [((8, 1), (2, 0), tdq.OK), ((2, 0), (11, None), (12, None), tdq.OK)])


def test_layer_norm_backward(tdq):
    inv, ali, uns = tdq.ERR_INVALID_ARG, tdq.ERR_ALIGNMENT, tdq.ERR_UNSUPPORTED
    f = tdq.lib().tdq_layer_norm_backward
    #       dy    st  x     st  dt M  C   mean  rstd  w     add   st  dx    st  dw    db    ws    bytes    stream
    good = [FAKE, 64, FAKE, 64, 1, 4, 64, FAKE, FAKE, FAKE, FAKE, 64, FAKE, 64, FAKE, FAKE, FAKE, 1 << 20, None]
    _each(f, good, [((i, v), c) for i, v, c in
                    [(i, None, inv) for i in (0, 2, 7, 8, 12)] + [(i, 63, inv) for i in (1, 3, 11, 13)] + [(i, ODD, ali) for i in (0, 2, 7, 8, 9, 10, 12, 14, 15)] +
                    [(16, OFF4, ali), (4, 3, inv), (5, -1, inv), (6, 0, inv), (5, 1 << 31, uns)]])
    big = 16385
    _each(f, good, [((6, big), (1, big), (3, big), (11, big), (13, big), uns), ((5, 0), (14, None), (15, None), tdq.OK)])
    assert int(tdq.lib().tdq_layer_norm_backward_workspace_bytes(4, 64)) == 4 * 2 * 64 * 4
    assert tdq.lib().tdq_layer_norm_backward_workspace_bytes(0, 64) == tdq.lib().tdq_layer_norm_backward_workspace_bytes(4, 16385) == 0


def test_binding_refuses_cpu_tensors(tdq):
    x, v = torch.zeros(4, 64), torch.zeros(4)
    for f in (lambda: tdq.layer_norm(x), lambda: tdq.layer_norm_fp8(x), lambda: tdq.layer_norm_backward(x, x, v, v), lambda: tdq.quantize_act_fp8(x, pow2=True)):
        with pytest.raises(ValueError):
            f()


def test_weight_grad(tdq):
    inv, ali, uns = tdq.ERR_INVALID_ARG, tdq.ERR_ALIGNMENT, tdq.ERR_UNSUPPORTED
    f, size = tdq.lib().tdq_fp8_weight_grad, tdq.lib().tdq_fp8_weight_grad_workspace_bytes
    #       dy    dt st  xc    xs    M   O   I   dw    dt st   db    ws    bytes    stream
    good = [FAKE, 1, 40, FAKE, FAKE, 64, 40, 90, FAKE, 0, 96, FAKE, FAKE, 1 << 40, None]
    _each(f, good, [((i, v), c) for i, v, c in
                    [(i, None, inv) for i in (0, 3, 4, 8)] + [(i, ODD, ali) for i in (0, 3, 4, 8, 11, 12)] +
                    [(3, OFF4, ali), (12, OFF4, ali), (1, 3, inv), (9, -1, inv), (2, 39, inv), (10, 89, inv), (5, -1, inv), (6, -1, inv), (7, 0, inv),
                     (5, 1 << 30, uns), (6, 0, tdq.OK)]])
    _each(f, good, [((6, 1 << 31), (2, 1 << 31), uns), ((7, 1 << 31), (10, 1 << 31), uns)])
    head = int(size(FAKE, 1, 40, 0, 40, 90))
    assert head == 256 and size(FAKE, 3, 40, 64, 40, 90) == size(FAKE, 1, 40, -1, 40, 90) == size(FAKE, 1, 40, 64, 40, 0) == 0
    # little work needs the status word alone
    assert size(FAKE, 1, 40, 64, 40, 90) == size(FAKE, 0, 41, 500, 40, 90) == 256
    # many whole tiles: a place for each tile's sums of dy; fp16 and rows off the grid pass through the workspace
    tiles, n, o = 16 * 148, 512, 4096
    one = 256 + (2 * 74 + tiles) * 4096
    assert size(FAKE, 1, o, n, o, 148 * 256) == one and size(ODD, 1, o, n, o, 148 * 256) == one + n * o * 2
    assert size(FAKE, 2, o, n, o, 148 * 256) == one + 2 * n * o * 2 and size(FAKE, 0, o, n - 1, o, 148 * 256) == one + 3 * n * o * 2
    # a long sum: two places for each of some clusters
    assert (size(FAKE, 1, 40, 1 << 20, 40, 90) - 256 - 4096) % (2 * 256 * (256 + 4) * 4) == 0


def test_linear_epilogue(tdq):
    inv, ali, uns = tdq.ERR_INVALID_ARG, tdq.ERR_ALIGNMENT, tdq.ERR_UNSUPPORTED
    f = tdq.lib().tdq_fp8_linear_epilogue
    n = tdq.FP8_WORKSPACE_BYTES

    def call(e=(2, None, 0, None, 0), **kw):
        a = dict(xc=FAKE, xs=FAKE, wc=FAKE, ws=FAKE, bias=None, M=4, I=256, O=8, e=0, y=FAKE, dt=0, st=8, wsp=FAKE, n=n, stream=None)
        a.update(kw)
        a["e"] = ctypes.byref(tdq.Fp8Epilogue(*e)) if e else None
        return f(*a.values())
    assert call(e=None) == inv and call(e=(-1, None, 0, None, 0)) == inv and call(e=(5, None, 0, None, 0)) == inv
    assert call(e=(0, 0x2000, 7, None, 0)) == inv and call(e=(0, None, 0, 0x2000, 7)) == inv and call(e=(0, None, 0, 0x1000, 8)) == inv
    assert call(e=(0, 0x2000, 8, 0x3000, 8)) == uns
    assert call(e=(0, 0x2001, 8, None, 0)) == ali and call(e=(0, None, 0, 0x2002, 8)) == ali
    assert call(xc=None) == inv and call(xc=OFF4) == ali and call(wsp=None) == tdq.ERR_WORKSPACE and call(M=1 << 31) == uns
    assert call(M=0) == tdq.OK


def test_activation_backward(tdq):
    inv, ali, uns = tdq.ERR_INVALID_ARG, tdq.ERR_ALIGNMENT, tdq.ERR_UNSUPPORTED
    _each(tdq.lib().tdq_activation_backward_fp8, [FAKE, 1, 4, 40, 40, FAKE, FAKE, 2, FAKE, 40, None],
          [((i, v), c) for i, v, c in [(0, None, inv), (5, None, inv), (6, None, inv), (8, None, inv), (1, 3, inv), (2, -1, inv), (3, 0, inv), (4, 39, inv),
                                       (9, 39, inv), (7, 5, inv), (7, -1, inv), (0, ODD, ali), (8, ODD, ali), (5, OFF4, ali), (6, ODD, ali), (2, 1 << 30, uns), (2, 0, tdq.OK)]])


def test_activation_names(tdq):
    x = torch.zeros(4, 64)
    for f in (lambda: tdq.fp8_linear(x, x, x, x, activation="tanh"), lambda: tdq.activation_backward_fp8(x, x, x, "tanh"), lambda: tdq.activation_backward_fp8(x, x, x, "gelu")):
        with pytest.raises(ValueError):
            f()


def test_workspace_for_gradients_of_another_type(tdq):
    with pytest.raises(TypeError, match="float64"):
        tdq.fp8_weight_grad_workspace(torch.zeros((2, 8), dtype=torch.float64), 128)
