"""The 8-bit floating point layer against 64-bit forms: codes and scales bit for bit, outputs within a derived tolerance."""
import numpy as np
import pytest
import torch

import fp8_utils as fu

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def tdq():
    from paper_2604_16855_b200 import tdq
    return tdq


def _tokens(M, C, seed, dtype):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn((M, C), generator=g) * torch.exp(torch.randn((M, 1), generator=g))
    x[:, ::37] *= 20.0
    return x.to(dtype)


def _same(codes, scale, x, rows_per):
    want_c, want_s = fu.quantize(x.float().cpu().numpy(), rows_per)
    assert np.array_equal(scale.cpu().numpy(), want_s, equal_nan=True)
    got = codes.view(torch.uint8).cpu().numpy()
    assert np.array_equal(got, want_c), "%d codes differ" % int((got != want_c).sum())


# ------------------------------------------------------------------------------------------------ quantizers

@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("M,C", [(1, 1), (1, 128), (3, 15), (2, 16), (5, 127), (4, 129), (33, 200), (257, 64), (65, 1000), (9, 4104)])
@pytest.mark.parametrize("pitch,offset", [(0, 0), (16, 0), (1, 0), (0, 1), (8, 8)])
def test_activations(tdq, dtype, M, C, pitch, offset):
    x = _tokens(M, C, M * 1000 + C, fu.DT[dtype])
    buf = torch.full((offset + M * (C + pitch),), float("nan"), dtype=x.dtype, device="cuda")      # what is not a channel must not be read as one
    v = buf[offset:].view(M, C + pitch)[:, :C]
    v.copy_(x)
    codes, scale = tdq.quantize_act_fp8(v)
    assert codes.dtype == torch.float8_e4m3fn and codes.shape == (M, fu.blocks(C) * 128) and scale.shape == (M, fu.blocks(C))
    _same(codes, scale, x, 1)


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("C", [1, 70, 127, 128, 129, 147, 255, 257, 300, 383, 511, 513, 639, 767, 895, 1023, 1025, 1151, 1279, 2175])
@pytest.mark.parametrize("M", [1, 5, 130])
def test_rows_off_the_grid(tdq, dtype, C, M):
    x = _tokens(M, C, M + C, fu.DT[dtype])
    pitch = 1 + C % 2                                     # odd rows, in turn on either half of a word
    buf = torch.full((1 + M * (C + pitch),), float("nan"), dtype=x.dtype, device="cuda")
    v = buf[1:].view(M, C + pitch)[:, :C]
    v.copy_(x)
    K = fu.blocks(C)
    codes, scale = torch.full((M + 2, K * 128), 77, dtype=torch.uint8, device="cuda"), torch.full((M + 2, K), 77.0, device="cuda")
    c, s = tdq.quantize_act_fp8(v, codes=codes[:M], scale=scale[:M])
    _same(c.view(torch.float8_e4m3fn), s, x, 1)
    assert (codes[M:] == 77).all() and (scale[M:] == 77).all()


def _edge_rows(C=256):
    """Rows at the edges of the formula: zeros, below the floor, denormals, the largest numbers, ties, one spike, signed zeros."""
    g = torch.Generator().manual_seed(5)
    r = [torch.zeros(C), torch.full((C,), 2.0 ** -70), torch.full((C,), 2.0 ** -64), 2.0 ** -60 * torch.randn(C, generator=g),
         1e-40 * torch.randn(C, generator=g), 3e38 * (1 - 2 * (torch.arange(C) % 2).float()), 448.0 * torch.ones(C)]
    ties = torch.from_numpy((fu.e4m3_values()[:126] + fu.e4m3_values()[1:127]) / 2).float()
    r.append(torch.cat([ties, torch.tensor([448.0, -448.0]), -ties, torch.tensor([448.0, -448.0])]))       # scale 1: ties stay ties
    r.append(r[-1] * 3)
    r.append(r[-2] * 1.2345)
    spike = 1e-3 * torch.randn(C, generator=g)
    spike[::128] = 1e4
    r += [spike, -torch.zeros(C), torch.arange(C).float() - C / 2]
    return torch.stack(r)


@pytest.mark.parametrize("pitch", [0, 1])
@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
def test_edges(tdq, dtype, pitch):
    x = _edge_rows()
    if dtype == "fp16":
        x = x.clamp(-65504, 65504)
    x = x.to(fu.DT[dtype])
    x = x[torch.isfinite(x.float()).all(1)]
    buf = torch.zeros((x.shape[0], x.shape[1] + pitch), dtype=x.dtype, device="cuda")[:, :x.shape[1]]
    buf.copy_(x)
    _same(*tdq.quantize_act_fp8(buf), x, 1)
    w = x.repeat(20, 1)[:131].contiguous()
    if pitch:
        w = w[:, :-1].contiguous()
    _same(*tdq.quantize_weight_fp8(w.cuda()), w, 128)


@pytest.mark.parametrize("value", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
def test_non_finite_blocks_are_nan_and_the_others_are_not(tdq, dtype, value):
    for C in (300, 301):                                  # both kernels of the activations
        x = _tokens(7, C, 3, fu.DT[dtype])
        x[2, 130] = value
        x[4, C - 1] = value
        _same(*tdq.quantize_act_fp8(x.cuda()), x, 1)
    w = _tokens(200, 300, 4, fu.DT[dtype])
    w[150, 7] = value
    _same(*tdq.quantize_weight_fp8(w.cuda()), w, 128)


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("O,I", [(1, 1), (2, 128), (127, 130), (128, 128), (129, 127), (300, 77), (960, 320), (260, 1032)])
def test_weights(tdq, dtype, O, I):
    w = (0.02 * _tokens(O, I, O + I, torch.float32)).to(fu.DT[dtype])
    _same(*tdq.quantize_weight_fp8(w.cuda()), w, 128)
    _same(*tdq.quantize_weight_fp8(w.cuda().t().contiguous().t()), w, 128)      # made contiguous


def test_every_bf16_quotient_of_one_block(tdq):
    """All bf16 magnitudes of eight binades against 127 block maxima: ties and their neighbours for every maximum's scale."""
    tops = torch.arange(1, 128, dtype=torch.float32) / 128 + 1                          # maxima 1 .. 2
    vals = (torch.arange(0, 127 * 16, dtype=torch.float32) % 128 / 128 + 1).view(16, 127) * 2.0 ** -torch.arange(0, 16, dtype=torch.float32)[:, None]
    x = torch.cat([vals[None].expand(127, 16, 127).minimum(tops[:, None, None]), tops[:, None, None].expand(127, 16, 1)], 2).reshape(127 * 16, 128)
    assert torch.equal(x.bfloat16().float(), x)
    _same(*tdq.quantize_act_fp8(x.bfloat16().cuda()), x, 1)


def test_given_outputs_and_empty_inputs(tdq):
    x = _tokens(9, 200, 1, torch.bfloat16).cuda()
    codes = torch.full((12, 256), 77, dtype=torch.uint8, device="cuda")
    scale = torch.full((12, 2), 7.0, device="cuda")
    c, s = tdq.quantize_act_fp8(x.view(3, 3, 200), codes=codes[:9], scale=scale[:9])
    assert c.data_ptr() == codes.data_ptr() and (codes[9:] == 77).all() and (scale[9:] == 7).all()      # rows behind stay
    _same(codes[:9], scale[:9], x, 1)
    n0 = tdq.kernel_launch_count()
    c, s = tdq.quantize_act_fp8(x[:0])
    assert c.shape == (0, 256) and s.shape == (0, 2)
    c, s = tdq.quantize_weight_fp8(x[:0])
    assert c.shape == (0, 256) and s.shape == (0, 2)
    wc, ws = torch.zeros((8, 256), dtype=torch.uint8, device="cuda"), torch.ones((1, 2), device="cuda")
    assert tdq.fp8_linear(codes[:0], scale[:0], wc, ws).shape == (0, 8)
    assert tdq.fp8_linear(codes, scale, wc[:0], ws[:0]).shape == (12, 0)
    assert tdq.kernel_launch_count() == n0


def test_rows_past_32_bits(tdq):
    """A row pitch of more than 2^31 elements."""
    far = torch.zeros((1 << 31) + 4096, dtype=torch.bfloat16, device="cuda")
    for pitch in ((1 << 31) + 8, (1 << 31) + 9):
        x = far.as_strided((2, 300), (pitch, 1))
        x.copy_(_tokens(2, 300, 8, torch.bfloat16))
        _same(*tdq.quantize_act_fp8(x), x, 1)
    xc, xs = tdq.quantize_act_fp8(_tokens(2, 128, 9, torch.float32).cuda())
    wc, ws = tdq.quantize_weight_fp8(_tokens(64, 128, 10, torch.float32).cuda())
    want = tdq.fp8_linear(xc, xs, wc, ws, out_dtype=torch.bfloat16)
    for pitch in ((1 << 31) + 8, (1 << 31) + 9):
        y = far.as_strided((2, 64), (pitch, 1))
        tdq.fp8_linear(xc, xs, wc, ws, y=y)
        assert torch.equal(y, want)
    q = far.as_strided((2, 2, 64), ((1 << 31) + 8, 64, 1))
    q.copy_(_tokens(4, 64, 11, torch.bfloat16).view(2, 2, 64))
    pos, table = torch.arange(2, device="cuda"), tdq.rope_table(64)
    want = tdq.qk_norm_rope(q.clone(), None, pos, table)[0]
    tdq.qk_norm_rope(q, None, pos, table, q_out=q)
    assert torch.equal(q, want)


# ------------------------------------------------------------------------------------------------ linear layer

def _operands(M, I, O, seed, device="cuda"):
    """Random codes of all magnitudes (no NaN) and scales over several binades, as the quantizers would not all make them."""
    g = torch.Generator().manual_seed(seed)
    K = fu.blocks(I)

    def codes(rows):
        c = torch.randint(0, 256, (rows, K * 128), generator=g, dtype=torch.int32)
        c = torch.where(c % 128 == 127, c - 1, c).to(torch.uint8)
        c[:, I:] = 0
        return c.view(torch.float8_e4m3fn).to(device)
    scale = lambda r: torch.exp(2 * torch.randn((r, K), generator=g)).to(device)  # noqa: E731
    return codes(M), scale(M), codes(O), scale(fu.blocks(O)), (100 * torch.randn((O,), generator=g)).to(device), K


def _run(tdq, M, I, O, dtype, bias, pitch=0, offset=0, seed=0):
    xc, xs, wc, ws, b, K = _operands(M, I, O, seed + M + I + O)
    if dtype == "fp16":                                   # into fp16's range
        xs, ws, b = xs * 1e-4, ws * 1e-2, b * 1e-3
    b = b if bias else None
    buf = torch.full((offset + (M + 2) * (O + pitch),), 7.0, dtype=fu.DT[dtype], device="cuda")
    rows = buf[offset:].view(M + 2, O + pitch)
    y = rows[:M, :O]
    wsp = tdq.fp8_linear_workspace("cuda")
    wsp.fill_(255)
    tdq.fp8_linear(xc, xs, wc, ws, b, y=y, workspace=wsp)
    assert tdq.workspace_status(wsp) == (tdq.OK, 0)
    ref, t = fu.linear(xc, xs, wc, ws, b)
    fu.check_linear(y, ref, t, K)
    assert (rows[M:] == 7).all() and (rows[:, O:] == 7).all() and (buf[:offset] == 7).all()     # nothing else is written
    y2 = tdq.fp8_linear(xc, xs, wc, ws, b, out_dtype=fu.DT[dtype])
    assert torch.equal(y2, y)                             # whatever way it is stored, the same bits


@pytest.mark.parametrize("M", [1, 2, 15, 16, 17, 32, 33, 63, 64, 65, 127, 128, 129, 300])
@pytest.mark.parametrize("I,O", [(1, 1), (128, 128), (129, 127), (384, 3), (640, 129), (1152, 260)])
def test_few_tokens(tdq, M, I, O):
    _run(tdq, M, I, O, "fp32", M % 2 == 0)


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("pitch,offset", [(0, 0), (16, 0), (16, 8), (1, 0), (3, 1)])
@pytest.mark.parametrize("M,O", [(5, 260), (40, 260), (130, 260), (2500, 1000), (700, 4000)])
def test_types_and_pitches(tdq, M, O, dtype, pitch, offset):
    _run(tdq, M, 300, O, dtype, True, pitch, offset)


@pytest.mark.parametrize("M,I,O", [(1, 128 * 67, 130), (20, 128 * 33, 1000), (100, 128 * 130, 64), (3000, 128 * 37, 900), (129, 128, 256 * 80)])
def test_long_contractions_and_many_tiles(tdq, M, I, O):
    _run(tdq, M, I, O, "bf16", False)


# The layer's tiles are 16, 32, 64 or 128 tokens wide, with the contraction in one part or several, or 256 x 256: shapes that take each of them.
WIDTHS = [(9, 200, 300), (31, 1030, 200), (77, 640, 5165), (20, 4096, 4095), (400, 768, 2303), (64, 4096, 4001), (48, 2048, 8190), (100, 4096, 4097),
          (127, 2048, 8191), (2742, 33 * 128, 100), (1030, 300, 1300)]


@pytest.mark.parametrize("M,I,O", WIDTHS)
@pytest.mark.parametrize("dtype,pitch", [("fp32", 1), ("bf16", 0), ("bf16", 3), ("fp16", 8)])
def test_every_width_of_tile(tdq, M, I, O, dtype, pitch):
    _run(tdq, M, I, O, dtype, pitch != 1, pitch)


# for every width of tile, one to eight parts
SPLITS = [(145, 64, 6359), (18, 1425, 6807), (1502, 690, 42), (853, 1989, 34), (924, 1747, 41), (723, 3711, 32), (622, 3208, 37),
          (540, 4951, 41), (4838, 66, 37), (2596, 390, 37), (2437, 262, 36), (1926, 970, 36), (1242, 1236, 35), (1276, 2016, 34),
          (1266, 1768, 44), (929, 2797, 32), (2959, 922, 160), (4970, 771, 40), (3335, 2330, 33), (3251, 1578, 39), (2427, 1995, 45),
          (1897, 2622, 36), (1559, 4031, 43), (5664, 65, 137), (1, 67, 34), (1, 907, 33)]


@pytest.mark.parametrize("n", range(len(SPLITS)))
def test_every_number_of_parts(tdq, n):
    _run(tdq, *SPLITS[n], ("fp32", "bf16", "fp16")[n % 3], n % 2 == 0, n % 4)


# tiles of 256 x 128: one round of them and several, fewer blocks than stages and many
NARROW = [(5227, 34, 33), (4750, 137, 33), (3259, 311, 34), (5142, 522, 33), (4756, 665, 33), (4744, 866, 36), (5075, 1097, 32), (6800, 2146, 33), (512, 4096, 4096),
          (1200, 1400, 1300), (300, 8190, 900), (9616, 32, 266), (9505, 298, 257), (9637, 552, 259), (9814, 785, 261), (9892, 2065, 280), (584, 32, 6435),
          (525, 258, 6557), (514, 533, 6468), (520, 1042, 7092)]


@pytest.mark.parametrize("M,I,O", NARROW)
@pytest.mark.parametrize("dtype,pitch", [("fp32", 0), ("bf16", 0), ("fp16", 8), ("bf16", 1), ("fp32", 2)])
def test_narrow_tiles(tdq, M, I, O, dtype, pitch):
    _run(tdq, M, I, O, dtype, pitch < 2, (-O) % 8 if pitch == 0 else pitch)


@pytest.mark.parametrize("M,O", [(9000, 1001), (9000, 998), (20000, 4093), (1200, 1301), (300, 61), (40, 999)])
def test_padded_rows_keep_what_stands_behind_the_last_column(tdq, M, O):
    """Rows on the 16-byte grid whose last column ends inside 16 bytes, for every kind of tile."""
    for dtype in ("fp32", "bf16", "fp16"):
        _run(tdq, M, 300, O, dtype, True, (-O) % 8)
        _run(tdq, M, 300, O, dtype, False, (-O) % 8 + 8, 8)


@pytest.mark.parametrize("M,I,O", [(1200, 700, 1300), (9505, 298, 257)])
def test_nan_in_narrow_tiles(tdq, M, I, O):
    xc, xs, wc, ws, b, K = _operands(M, I, O, 6)
    xc.view(torch.uint8)[1, 200] = 0x7F
    ws[1, 2] = float("nan")
    xs[M - 1, 0] = float("inf")
    y = tdq.fp8_linear(xc, xs, wc, ws, b)
    bad = torch.zeros((M, O), dtype=torch.bool, device="cuda")
    bad[1], bad[M - 1], bad[:, 128:256] = True, True, True
    assert torch.isfinite(y[~bad]).all() and not torch.isfinite(y[bad]).any()


@pytest.mark.parametrize("M,O", [(257, 256 * 37 + 1), (256 * 5 + 1, 256 * 9 - 1), (256 * 38 - 127, 100), (20000, 257)])
def test_ragged_large_tiles(tdq, M, O):
    _run(tdq, M, 256, O, "fp32", True)


@pytest.mark.parametrize("M,I,O", [(1, 256, 40000), (33, 130, 37889), (64, 256, 65537), (65, 256, 37890)])
def test_few_tokens_and_very_many_outputs(tdq, M, I, O):
    _run(tdq, M, I, O, "bf16", True)


@pytest.mark.parametrize("M,I,O", [(3, 300, 300), (100, 300, 300), (2600, 300, 1000)] + [w for w in WIDTHS if w[1] > 256 and w[2] > 258])
def test_nan_codes_and_scales_reach_their_outputs_only(tdq, M, I, O):
    xc, xs, wc, ws, b, K = _operands(M, I, O, 6)
    xc.view(torch.uint8)[1, 200] = 0x7F
    wc.view(torch.uint8)[257, 5] = 0xFF
    ws[1, 2] = float("inf")
    xs[M - 1, 0] = float("nan")
    xs[0, 1] = 0.0
    y = tdq.fp8_linear(xc, xs, wc, ws, b)
    ref, t = fu.linear(xc, xs, wc, ws, b)
    bad = ~torch.isfinite(ref)
    assert bad.any() and not bad.all()
    assert not torch.isfinite(y[bad]).any() and torch.isfinite(y[~bad]).all()
    fine = torch.where(bad, torch.zeros_like(ref), ref)
    fu.check_linear(torch.where(bad, torch.zeros_like(y), y), fine, torch.where(bad, torch.zeros_like(t), t), K)


def test_zero_scales_and_codes_give_the_bias(tdq):
    for M, O in ((4, 200), (2600, 1000)):
        xc, xs, wc, ws, b, K = _operands(M, 256, O, 2)
        assert torch.equal(tdq.fp8_linear(xc, xs * 0, wc, ws, b), b.expand(M, O))
        assert torch.equal(tdq.fp8_linear(torch.zeros_like(xc), xs, wc, ws), torch.zeros((M, O), device="cuda"))


def test_uint8_codes_and_refusals_of_the_binding(tdq):
    xc, xs, wc, ws, b, K = _operands(6, 256, 200, 1)
    y = tdq.fp8_linear(xc, xs, wc, ws, b)
    assert torch.equal(y, tdq.fp8_linear(xc.view(torch.uint8), xs, wc.view(torch.uint8), ws, b))
    n0 = tdq.kernel_launch_count()
    for args in [(xc.float(), xs, wc, ws), (xc, xs.double(), wc, ws), (xc, xs, wc.view(torch.int8), ws)]:
        with pytest.raises(TypeError):
            tdq.fp8_linear(*args)
    for args in [(xc, xs[:5], wc, ws), (xc, xs.t().contiguous(), wc, ws), (xc, xs, wc, ws[:1]), (xc, xs, wc[:, :128].contiguous(), ws),
                 (xc[:, :100].contiguous(), xs, wc, ws), (xc, xs, wc.t().contiguous().t(), ws), (xc, xs, wc, ws, b[:199]), (xc[0], xs, wc, ws)]:
        with pytest.raises(ValueError):
            tdq.fp8_linear(*args)
    for kw in [dict(y=torch.zeros((6, 201), device="cuda")), dict(y=torch.zeros((200, 6), device="cuda").t()), dict(y=torch.zeros((6, 200))),
               dict(workspace=torch.zeros(256, dtype=torch.uint8))]:
        with pytest.raises(ValueError):
            tdq.fp8_linear(xc, xs, wc, ws, **kw)
    with pytest.raises(TypeError):
        tdq.fp8_linear(xc, xs, wc, ws, y=torch.zeros((6, 200), dtype=torch.float64, device="cuda"))
    for bad in [torch.zeros(128, dtype=torch.uint8, device="cuda")]:
        with pytest.raises(tdq.TdqError) as e:
            tdq.fp8_linear(xc, xs, wc, ws, workspace=bad)
        assert e.value.code == tdq.ERR_WORKSPACE
    x = _tokens(4, 256, 0, torch.float32).cuda()
    for f, x_bad in [(tdq.quantize_act_fp8, x.t()), (tdq.quantize_weight_fp8, x[0])]:
        with pytest.raises(ValueError):
            f(x_bad)
    with pytest.raises(TypeError):
        tdq.quantize_act_fp8(x.double())
    with pytest.raises(ValueError):
        tdq.quantize_act_fp8(x, codes=torch.zeros((4, 128), dtype=torch.uint8, device="cuda"))
    with pytest.raises(tdq.TdqError):
        tdq.quantize_act_fp8(x[:1].expand(4, 256))        # rows that overlap
    assert tdq.kernel_launch_count() == n0


# ------------------------------------------------------------------------------------------------ as a program runs them

def _layer(tdq, M, C, O, seed):
    x = _tokens(M, C, seed, torch.bfloat16).cuda()
    w = (0.02 * _tokens(O, C, seed + 1, torch.float32)).cuda()
    return x, tdq.quantize_weight_fp8(w)


def test_two_streams_at_once(tdq):
    jobs = []
    for i, (M, C, O) in enumerate([(1, 2048, 2048), (50, 1024, 1500), (200, 768, 900), (3000, 512, 1100)]):
        x, (wc, ws) = _layer(tdq, M, C, O, 10 * i)
        jobs.append((x, wc, ws, tdq.fp8_linear(*tdq.quantize_act_fp8(x), wc, ws)))
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(4)]
    got = [[] for _ in jobs]
    for _ in range(5):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                for j in range(4):
                    x, wc, ws, _ = jobs[(i + j) % 4]
                    got[(i + j) % 4].append(tdq.fp8_linear(*tdq.quantize_act_fp8(x), wc, ws))
    torch.cuda.synchronize()
    for (_, _, _, want), ys in zip(jobs, got):
        assert all(torch.equal(y, want) for y in ys)


@pytest.mark.parametrize("M,C,O", [(3, 1024, 640), (2600, 384, 1000)])
def test_graph_replay_follows_its_inputs(tdq, M, C, O):
    x, (wc, ws) = _layer(tdq, M, C, O, 5)
    codes, scale = tdq.quantize_act_fp8(x)
    y = torch.zeros((M, O), dtype=torch.bfloat16, device="cuda")
    wsp = tdq.fp8_linear_workspace("cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            tdq.quantize_act_fp8(x, codes=codes, scale=scale)
            tdq.fp8_linear(codes, scale, wc, ws, y=y, workspace=wsp)
    for seed in (21, 22):
        x.copy_(_tokens(M, C, seed, torch.bfloat16))
        graph.replay()
        torch.cuda.synchronize()
        c, s = tdq.quantize_act_fp8(x.clone())
        assert torch.equal(y, tdq.fp8_linear(c, s, wc, ws, out_dtype=torch.bfloat16))
    assert tdq.workspace_status(wsp) == (tdq.OK, 0)


@pytest.mark.parametrize("M,hq,hk,D", [(1, 8, 2, 64), (1152, 5, 5, 64), (300, 8, 2, 128)])
def test_qkv_layer_then_rotation_in_place(tdq, M, hq, hk, D):
    """Quantizer, qkv layer, norm and rotation in place on views of its output: every stage against its 64-bit form."""
    C, O = 320, (hq + 2 * hk) * D
    x, (wc, ws) = _layer(tdq, M, C, O, 30)
    bias = 0.1 * torch.randn((O,), device="cuda")
    codes, scale = tdq.quantize_act_fp8(x)
    _same(codes, scale, x, 1)
    qkv = tdq.fp8_linear(codes, scale, wc, ws, bias, out_dtype=torch.bfloat16)
    ref, t = fu.linear(codes, scale, wc, ws, bias)
    fu.check_linear(qkv, ref, t, fu.blocks(C))
    before = qkv.clone()
    q, k = qkv[:, :hq * D].view(M, hq, D), qkv[:, hq * D:(hq + hk) * D].view(M, hk, D)
    at = torch.arange(M, device="cuda")
    pos = torch.stack([at // 24, at % 24], 1).contiguous()
    freq, axis = tdq.rope_table(D, [D // 4, D // 4], restart=True)
    qw, kw = 1 + 0.1 * torch.randn((D,), device="cuda"), 1 + 0.1 * torch.randn((D,), device="cuda")
    tdq.qk_norm_rope(q, k, pos, (freq, axis), qw, kw, q_out=q, k_out=k)
    for now, was, w in ((q, before[:, :hq * D].view(M, hq, D), qw), (k, before[:, hq * D:(hq + hk) * D].view(M, hk, D), kw)):
        fu.check_rope(now, *fu.rope(was, w, pos, freq, axis.long(), 1e-6, False))
    assert torch.equal(qkv[:, (hq + hk) * D:], before[:, (hq + hk) * D:])       # the values are left as they were


FIRST_IN_A_CAPTURE = """
import torch
from paper_2604_16855_b200 import tdq
x = torch.randn((%(M)d, 300), device="cuda").bfloat16()
w = torch.randn((%(O)d, 300), device="cuda")
pos, table = torch.arange(%(M)d, device="cuda"), tdq.rope_table(64)
torch.cuda.synchronize()
side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
with torch.cuda.stream(side), torch.cuda.graph(graph, stream=side):
    wc, ws = tdq.quantize_weight_fp8(w)
    y = tdq.fp8_linear(*tdq.quantize_act_fp8(x), wc, ws, out_dtype=torch.bfloat16)
    q, _ = tdq.qk_norm_rope(y[:, :128].view(-1, 2, 64), None, pos, table)
graph.replay()
torch.cuda.synchronize()
wc, ws = tdq.quantize_weight_fp8(w)
z = tdq.fp8_linear(*tdq.quantize_act_fp8(x), wc, ws, out_dtype=torch.bfloat16)
assert torch.equal(y, z) and torch.equal(q, tdq.qk_norm_rope(z[:, :128].view(-1, 2, 64), None, pos, table)[0])
"""


@pytest.mark.parametrize("M,O", [(3, 200), (2600, 1000)])
def test_first_use_inside_a_capture(M, O):
    import os
    import subprocess
    import sys
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, "-c", FIRST_IN_A_CAPTURE % dict(M=M, O=O)], cwd=root, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr[-2000:]


@pytest.mark.parametrize("way,n", [(way, n) for way, shapes in fu.WAYS.items() for n in range(len(shapes))])
def test_every_way_of_the_layer(tdq, way, n):
    """Each kind of tile with each number of parts, and the shapes are computed that way (tdq_fp8_linear_tiles; the lists above were drawn for earlier choices)."""
    M, I, O = fu.WAYS[way][n]
    assert torch.cuda.get_device_properties(0).multi_processor_count != 148 or tdq.fp8_linear_tiles(M, fu.blocks(I) * 128, O) == way
    _run(tdq, M, I, O, "fp32", n % 2 == 0, n % 3)
    _run(tdq, M, I, O, "bf16", n % 2 == 1, (-O) % 8)
    _run(tdq, M, I, O, "fp16", True, (-O) % 8 + 8, 8 * (n % 2))


TILES = """
import sys, json
import torch
from torch.profiler import ProfilerActivity, profile
from paper_2604_16855_b200 import tdq
shapes = %s
calls = []
for M, I, O in shapes:
    K = (I + 127) // 128
    calls.append((torch.zeros((M, K * 128), dtype=torch.uint8, device="cuda"), torch.ones((M, K), device="cuda"), torch.zeros((O, K * 128), dtype=torch.uint8, device="cuda"),
                  torch.ones(((O + 127) // 128, K), device="cuda")))
torch.cuda.synchronize()
with profile(activities=[ProfilerActivity.CUDA]) as p:
    for c in calls:
        tdq.fp8_linear(*c)
    torch.cuda.synchronize()
p.export_chrome_trace(sys.argv[1])
"""


def test_the_query_says_what_runs(tdq, tmp_path):
    """Kernel and grid of one layer for each way, from the profiler's record."""
    import json
    import os
    import subprocess
    import sys
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    shapes = [v[0] for v in fu.WAYS.values()]
    r = subprocess.run([sys.executable, "-c", TILES % shapes, str(tmp_path / "trace")], cwd=root, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr[-2000:]
    events = [e for e in json.load(open(tmp_path / "trace"))["traceEvents"] if e.get("cat") == "kernel" and "fp8_" in e["name"]]
    events.sort(key=lambda e: e["ts"])
    assert len(events) == len(shapes)
    sms = torch.cuda.get_device_properties(0).multi_processor_count
    for (M, I, O), e in zip(shapes, events):
        tokens, channels, parts = tdq.fp8_linear_tiles(M, fu.blocks(I) * 128, O)
        tiles = -(-M // tokens) * -(-O // channels)
        if tokens == 256:
            assert "fp8_pair_kernel<0, %d>" % channels in e["name"] and e["args"]["grid"][0] == 2 * min(tiles, sms // 2), e
        else:
            assert "fp8_split_kernel<%d>" % tokens in e["name"] and e["args"]["grid"][0] == tiles * parts, e
