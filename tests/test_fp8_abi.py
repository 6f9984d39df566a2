"""Refusals of the 8-bit floating point layer and of the norm and rotation, before anything is launched (no GPU needed)."""
import ctypes

import numpy as np
import pytest
import torch

import fp8_utils as fu

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


def test_plain_codes_are_the_formats(tdq):
    v = fu.e4m3_values()
    t = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(v, t, equal_nan=True)
    q = np.random.default_rng(0).normal(size=4096).astype(np.float32).astype(np.float64) * 32
    q = np.concatenate([q, (v[:126] + v[1:127]) / 2, -(v[:126] + v[1:127]) / 2, v[:127]])
    want = torch.from_numpy(q).to(torch.float32).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    assert np.array_equal(fu.nearest_code(q), want)


def _each(f, good, changes):
    for at, value, code in changes:
        args = list(good)
        args[at] = value
        assert f(*args) == code, (at, value)


def test_quantizers(tdq):
    inv, ali, uns = tdq.ERR_INVALID_ARG, tdq.ERR_ALIGNMENT, tdq.ERR_UNSUPPORTED
    f = tdq.lib().tdq_quantize_act_fp8
    _each(f, [FAKE, 1, 2, 4, 64, 64, FAKE, FAKE, None],
          [(0, None, inv), (1, 3, inv), (1, -1, inv), (2, -1, inv), (3, -1, inv), (4, 0, inv), (4, 1 << 31, inv), (5, 63, inv), (6, None, inv),
           (7, None, inv), (0, ODD, ali), (6, OFF4, ali), (7, ODD, ali), (3, 1 << 30, uns), (3, 0, tdq.OK), (2, 0, tdq.OK)])
    assert f(FAKE, 1, 1 << 33, 1 << 33, 64, 64, FAKE, FAKE, None) == inv     # the product passes 64 bits
    _each(tdq.lib().tdq_quantize_weight_fp8, [FAKE, 0, 4, 64, FAKE, FAKE, None],
          [(0, None, inv), (1, 5, inv), (2, -1, inv), (3, 0, inv), (4, None, inv), (5, None, inv), (0, ctypes.c_void_p(0x1002), ali),
           (4, OFF4, ali), (5, ODD, ali), (2, 1 << 40, uns), (3, 1 << 31, uns), (2, 0, tdq.OK)])


def test_linear(tdq):
    inv, ali, uns = tdq.ERR_INVALID_ARG, tdq.ERR_ALIGNMENT, tdq.ERR_UNSUPPORTED
    f = tdq.lib().tdq_fp8_linear
    n = int(tdq.lib().tdq_fp8_linear_workspace_bytes(4, 128, 8))
    assert n == tdq.FP8_WORKSPACE_BYTES and n % 16 == 0
    #       xc    xs    wc    ws    bias  M  I    O  y     dt yst wsp   bytes stream
    good = [FAKE, FAKE, FAKE, FAKE, None, 4, 256, 8, FAKE, 0, 8, FAKE, n, None]
    _each(f, good, [(i, None, inv) for i in (0, 1, 2, 3, 8)] +
          [(5, -1, inv), (6, 0, inv), (6, 192, inv), (7, -1, inv), (9, 3, inv), (10, 7, inv), (11, None, tdq.ERR_WORKSPACE),
           (12, n - 1, tdq.ERR_WORKSPACE), (0, OFF4, ali), (2, OFF4, ali), (11, OFF4, ali), (1, ODD, ali), (3, ODD, ali), (4, ODD, ali),
           (8, ODD, ali), (5, 1 << 31, uns), (6, 1 << 31, uns), (5, 0, tdq.OK)])
    good[7] = good[10] = 1 << 31
    assert f(*good) == uns
    good[7] = good[10] = 0
    assert f(*good) == tdq.OK


def test_rope(tdq):
    f = tdq.lib().tdq_qk_norm_rope

    def h(**kw):
        d = dict(x=0x1000, out=0x2000, weight=0x3000, heads=4, row_stride=512, head_stride=64, out_row_stride=256, out_head_stride=64)
        d.update(kw)
        return tdq.RopeHeads(*[d[n] for n, _ in tdq.RopeHeads._fields_])

    def call(q=None, k=None, dt=1, M=3, p=(64, 64, 1, 1, 1e-6), pos=FAKE, freq=FAKE, axis=FAKE):
        rp = tdq.RopeParams(*p) if p else None
        return f(ctypes.byref(q) if q else None, ctypes.byref(k) if k else None, dt, M, ctypes.byref(rp) if rp else None, pos, freq, axis, None)
    inv, ali, uns = tdq.ERR_INVALID_ARG, tdq.ERR_ALIGNMENT, tdq.ERR_UNSUPPORTED
    assert call() == inv and call(q=h(), p=None) == inv and call(q=h(), M=-1) == inv and call(q=h(), dt=3) == inv
    assert call(q=h(), M=1 << 31) == uns and call(q=h(heads=1, row_stride=1 << 17, out_row_stride=1 << 17), p=(1 << 17, 64, 1, 1, 1e-6)) == uns
    for p in [(0, 0, 1, 1, 1e-6), (64, 66, 1, 1, 1e-6), (64, -2, 1, 1, 1e-6), (64, 31, 1, 1, 1e-6), (64, 64, 0, 1, 1e-6), (64, 64, 1, 4, 1e-6),
              (64, 64, 1, 1, -1.0), (64, 64, 1, 1, float("nan"))]:
        assert call(q=h(), p=p) == inv, p
    assert call(q=h(), pos=None) == inv and call(q=h(), freq=None) == inv and call(q=h(), axis=None) == inv
    assert call(q=h(), pos=OFF4) == ali and call(q=h(), freq=OFF4) == ali and call(q=h(), axis=ODD) == ali
    for kw in [dict(x=None), dict(out=None), dict(heads=-1), dict(row_stride=-1), dict(head_stride=1 << 60), dict(out_head_stride=63),
               dict(out_row_stride=255), dict(out_row_stride=64, out_head_stride=128), dict(out_row_stride=32, out_head_stride=0),
               dict(out=0x1000), dict(out=0x1000, out_row_stride=512, out_head_stride=128)]:
        assert call(q=h(**kw)) == inv and call(q=h(), k=h(**kw)) == inv, kw
    assert call(q=h(x=0x1001)) == ali and call(q=h(out=0x2001)) == ali and call(k=h(weight=0x3002)) == ali
    assert call(q=h(heads=70000, out_row_stride=70000 * 64)) == uns
    # one tensor for both sides, written: refused unless one side has no heads
    for q, k in [(h(), h()), (h(), h(x=0x5000)), (h(), h(x=0x2000, out=0x6000)), (h(x=0x6000), h(x=0x5000, out=0x6000)),
                 (h(x=0x2000, out_row_stride=512), h(x=0x2000, out=0x6000))]:
        assert call(q=q, k=k) == inv
    assert call(q=h(), M=0) == tdq.OK and call(q=h(heads=0), k=h(heads=0)) == tdq.OK


def test_binding_refuses_cpu_tensors_and_bad_tables(tdq):
    x = torch.zeros(4, 64)
    with pytest.raises(ValueError):
        tdq.quantize_act_fp8(x)
    with pytest.raises(ValueError):
        tdq.quantize_weight_fp8(x)
    with pytest.raises(ValueError):
        tdq.fp8_linear(x, x, x, x)
    with pytest.raises(ValueError):
        tdq.qk_norm_rope(x.view(4, 1, 64), None, torch.zeros(4, dtype=torch.long), tdq.rope_table(64, device="cpu"))
    for args, kw in [((63,), {}), ((-2,), {}), ((64, [16, 15]), {}), ((64, [33, -1]), {}), ((64,), {"base": 0.0})]:
        with pytest.raises(ValueError):
            tdq.rope_table(*args, device="cpu", **kw)


def test_rope_table(tdq):
    freq, axis = tdq.rope_table(64, device="cpu")
    assert freq.dtype == torch.float64 and axis.dtype == torch.int32 and torch.equal(axis, torch.zeros(32, dtype=torch.int32))
    assert np.allclose(freq.numpy(), 10000.0 ** (-2.0 * np.arange(32) / 64), rtol=1e-14)
    freq, axis = tdq.rope_table(128, [16, 24, 24], 5e5, device="cpu")
    assert axis.tolist() == [0] * 16 + [1] * 24 + [2] * 24
    assert np.allclose(freq.numpy(), 5e5 ** (-np.arange(64) / 64.0), rtol=1e-14)
    freq, axis = tdq.rope_table(64, [16, 16], 100.0, restart=True, device="cpu")
    assert np.allclose(freq.numpy(), 100.0 ** (-np.tile(np.arange(16), 2) / 16.0), rtol=1e-14)
    freq, axis = tdq.rope_table(0, device="cpu")
    assert freq.numel() == 0 and axis.numel() == 0


def test_wait_selftest_of_the_layer(tdq):
    f = tdq.lib().tdq_selftest_wait_timeout
    assert f(3, 100000, None, None) == f(3, 10, FAKE, None) == f(3, 1 << 40, FAKE, None) == tdq.ERR_INVALID_ARG
    assert f(3, 100000, OFF4, None) == tdq.ERR_ALIGNMENT


def test_the_ways_a_layer_is_computed(tdq):
    """Every way that the estimate can choose has shapes that the GPU tests run it with."""
    for way, shapes in fu.WAYS.items():
        for M, I, O in shapes:
            assert tdq.fp8_linear_tiles(M, fu.blocks(I) * 128, O, 148) == way, (M, I, O)
    rng = np.random.default_rng(0)
    seen = {tdq.fp8_linear_tiles(*[int(v) for v in (m, 128 * k, o)], 148)
            for m, k, o in zip(np.exp(rng.uniform(0, 12, 40000)), np.exp(rng.uniform(0, 5, 40000)).astype(int), np.exp(rng.uniform(0, 11.5, 40000)))}
    assert seen <= set(fu.WAYS), seen - set(fu.WAYS)
    assert {(16, 128, s) for s in range(1, 9)} <= set(fu.WAYS) and {(n, 128, s) for n in (32, 64, 128) for s in range(2, 9)} <= set(fu.WAYS)
    assert tdq.fp8_linear_tiles(0, 128, 5, 148) == tdq.fp8_linear_tiles(5, 128, 0, 148) == (0, 0, 0)
    f, out = tdq.lib().tdq_fp8_linear_tiles, [ctypes.byref(ctypes.c_int32(0)) for _ in range(3)]
    inv, uns = tdq.ERR_INVALID_ARG, tdq.ERR_UNSUPPORTED
    _each(f, [4, 256, 8, 148] + out, [(0, -1, inv), (1, 0, inv), (1, 100, inv), (2, -1, inv), (3, 0, inv), (4, None, inv), (5, None, inv), (6, None, inv),
                                      (0, 1 << 31, uns), (1, 1 << 31, uns), (2, 1 << 31, uns), (0, 4, tdq.OK)])


@pytest.mark.parametrize("sm_count", [1, 7, 66, 132, 148, 160])
def test_a_way_exists_on_any_number_of_sms(tdq, sm_count):
    rng = np.random.default_rng(sm_count)
    for _ in range(3000):
        M, K, O = (int(np.exp(rng.uniform(0, top))) for top in (13, 5, 12))
        tokens, channels, parts = tdq.fp8_linear_tiles(M, 128 * K, O, sm_count)
        assert (tokens, channels) in {(16, 128), (32, 128), (64, 128), (128, 128), (256, 128), (256, 256)}
        assert 1 <= parts <= min(8, K) and (tokens < 256 or parts == 1)


def test_rope_table_without_pairs(tdq):
    for sections in (None, [], [0], [0, 0]):
        for restart in (False, True):
            freq, axis = tdq.rope_table(0, sections, restart=restart, device="cpu")
            assert freq.dtype == torch.float64 and axis.dtype == torch.int32 and freq.shape == axis.shape == (0,)
