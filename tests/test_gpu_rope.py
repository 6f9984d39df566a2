"""Norm and rotation of queries and keys against the 64-bit form."""
import math

import pytest
import torch

import fp8_utils as fu

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def tdq():
    from paper_2604_16855_b200 import tdq
    return tdq


def _heads(M, H, D, seed, dtype):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn((M, H, D), generator=g) * torch.exp(torch.randn((M, H, 1), generator=g))).to(dtype).cuda()


def _case(tdq, M, hq, hk, D, R, axes, dtype, eps=1e-6, adjacent=False, weights=True, far=0, views=None):
    dt = fu.DT[dtype]
    q, k = _heads(M, hq, D, 1, dt), _heads(M, hk, D, 2, dt)
    g = torch.Generator().manual_seed(3)
    qw = (1 + 0.2 * torch.randn((D,), generator=g)).cuda() if weights and eps is not None else None
    kw = (1 + 0.2 * torch.randn((D,), generator=g)).cuda() if weights and eps is not None else None
    pos = torch.randint(-far - 50, far + 50, (M, axes), generator=g).cuda()
    half = R // 2
    freq, axis = tdq.rope_table(R, [half // axes + (i < half % axes) for i in range(axes)])
    if views:
        q, k = views(q), views(k)
    qo, ko = tdq.qk_norm_rope(q, k, pos, (freq, axis), qw, kw, eps=eps, adjacent=adjacent)
    for out, x, w in ((qo, q, qw), (ko, k, kw)):
        assert out.shape == x.shape and out.dtype == dt and out.is_contiguous()
        fu.check_rope(out, *fu.rope(x, w, pos, freq, axis.long(), eps, adjacent))
    tdq.qk_norm_rope(q, k, pos, (freq, axis), qw, kw, eps=eps, adjacent=adjacent, q_out=q, k_out=k)
    assert torch.equal(q, qo) and torch.equal(k, ko)      # in place: the same bits


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("adjacent", [False, True])
@pytest.mark.parametrize("D,R", [(2, 2), (1, 0), (3, 2), (16, 16), (32, 32), (40, 40), (64, 64), (64, 32), (80, 80), (80, 40), (96, 96), (128, 128), (128, 64),
                                 (128, 0), (256, 256), (512, 512), (72, 48), (576, 64), (1030, 1030)])
def test_head_sizes(tdq, D, R, adjacent, dtype):
    _case(tdq, 7, 3, 2, D, R, 1, dtype, adjacent=adjacent)


@pytest.mark.parametrize("M,hq,hk", [(1, 1, 1), (1, 32, 8), (2, 71, 1), (5, 12, 12), (9, 200, 3), (65, 4, 4), (1000, 6, 1)])
@pytest.mark.parametrize("D", [64, 128, 72])
def test_tokens_and_heads(tdq, M, hq, hk, D):
    _case(tdq, M, hq, hk, D, D, 1, "bf16")


@pytest.mark.parametrize("axes", [1, 2, 3, 5])
@pytest.mark.parametrize("adjacent", [False, True])
def test_axes(tdq, axes, adjacent):
    _case(tdq, 33, 4, 2, 128, 128, axes, "fp32", adjacent=adjacent)


@pytest.mark.parametrize("D", [64, 72])
@pytest.mark.parametrize("far", [1 << 17, 1 << 24, 1 << 31])
def test_far_positions(tdq, far, D):
    _case(tdq, 50, 2, 2, D, D, 2, "fp32", far=far)


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("adjacent", [False, True])
@pytest.mark.parametrize("D,R", [(8, 8), (8, 0), (24, 16), (40, 8), (72, 72), (80, 40), (88, 80), (104, 104), (200, 40), (248, 248), (256, 8)])
def test_vectors_of_eight_bytes(tdq, D, R, adjacent, dtype):
    def views(x):                                         # rows and heads on the 8-byte grid only
        M, H, D = x.shape
        v = torch.full((4 + M * (H * (D + 4) + 4),), float("nan"), dtype=x.dtype, device="cuda")[4:]
        v = v.as_strided((M, H, D), (H * (D + 4) + 4, D + 4, 1))
        v.copy_(x)
        return v
    for M, hq, hk in ((1, 1, 1), (37, 9, 2), (700, 3, 3)):
        _case(tdq, M, hq, hk, D, R, 2, dtype, adjacent=adjacent)
        _case(tdq, M, hq, hk, D, R, 1, dtype, adjacent=adjacent, views=views, weights=False)


@pytest.mark.parametrize("D", [64, 72])
def test_whole_turns_and_frequencies_that_are_no_numbers(tdq, D):
    x = _heads(6, 3, D, 8, torch.float32)
    pos = torch.tensor([0, 1, -1, 1 << 31, (1 << 52) + 3, -(1 << 62)], device="cuda")
    freq, axis = tdq.rope_table(D)
    out, _ = tdq.qk_norm_rope(x, None, pos, (torch.zeros_like(freq), axis), eps=None)
    assert torch.equal(out, x)                            # no turn at any position
    freq[3], freq[5], freq[7] = float("nan"), float("inf"), -float("inf")
    out, _ = tdq.qk_norm_rope(x, None, pos, (freq, axis), eps=None)
    bad = torch.zeros(D, dtype=torch.bool, device="cuda")
    bad[[3, 5, 7]] = bad[[D // 2 + 3, D // 2 + 5, D // 2 + 7]] = True
    assert out[:, :, bad].isnan().all() and torch.isfinite(out[:, :, ~bad]).all()


@pytest.mark.parametrize("M,hq,hk,D,dtype", [(6000, 32, 8, 128, "bf16"), (702, 60, 12, 64, "bf16"), (314, 16, 4, 256, "fp32"), (2219, 48, 12, 96, "fp32"),
                                             (29386, 1, 1, 256, "bf16"), (300, 300, 1, 128, "fp16"), (40000, 1, 0, 16, "fp32"), (149, 9, 9, 512, "bf16")])
def test_blocks_of_tokens_and_groups(tdq, M, hq, hk, D, dtype):
    _case(tdq, M, hq, hk, D, D // 2, 2, dtype, far=1 << 20)


@pytest.mark.parametrize("D", [64, 72])
def test_without_norm_and_without_weights(tdq, D):
    _case(tdq, 20, 4, 2, D, D, 1, "fp16", eps=None)
    _case(tdq, 20, 4, 2, D, D, 1, "fp16", weights=False)
    _case(tdq, 20, 4, 2, D, D, 1, "fp32", eps=0.0)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("gap,shift", [(0, 0), (16, 16), (8, 0), (1, 0), (0, 1), (3, 5)])
def test_strides_and_alignment(tdq, gap, shift, dtype):
    def views(x):
        M, H, D = x.shape
        v = torch.full((shift + M * (H * (D + gap) + gap),), float("nan"), dtype=x.dtype, device="cuda")[shift:]
        v = v.as_strided((M, H, D), (H * (D + gap) + gap, D + gap, 1))
        v.copy_(x)
        return v
    _case(tdq, 11, 3, 2, 64, 64, 1, dtype, views=views)
    _case(tdq, 11, 3, 2, 64, 64, 1, dtype, views=lambda x: x.transpose(0, 1).contiguous().transpose(0, 1))      # head-major


def test_zero_heads_of_zeros_and_non_finite_ones(tdq):
    table, pos = tdq.rope_table(64), torch.arange(4, device="cuda")
    x = _heads(4, 3, 64, 5, torch.float32)
    x[1, 1] = 0
    x[2, 0, 5] = float("nan")
    x[3, 2, 63] = float("inf")
    out, none = tdq.qk_norm_rope(x, None, pos, table)
    assert none is None and (out[1, 1] == 0).all()
    bad = torch.zeros((4, 3), dtype=torch.bool, device="cuda")
    bad[2, 0] = bad[3, 2] = True
    assert torch.isfinite(out[~bad]).all() and out[2, 0].isnan().all() and not torch.isfinite(out[3, 2, [31, 63]]).any()
    o = torch.zeros((4, 0, 64), device="cuda")
    qo, ko = tdq.qk_norm_rope(x, o, pos, table)           # a side without heads
    assert ko.shape == (4, 0, 64) and torch.equal(qo.nan_to_num(), out.nan_to_num())
    n0 = tdq.kernel_launch_count()
    qo, ko = tdq.qk_norm_rope(x[:0], o[:0], pos[:0], table)
    assert qo.shape == (0, 3, 64) and tdq.kernel_launch_count() == n0


def test_an_axis_outside_the_positions_is_their_last(tdq):
    x, pos = _heads(9, 2, 64, 1, torch.float32), torch.randint(0, 99, (9, 3), device="cuda")
    freq, axis = tdq.rope_table(64, [10, 11, 11])
    want = tdq.qk_norm_rope(x, None, pos, (freq, axis))[0]
    for odd in (3, -1, 2 ** 31 - 1, -2 ** 31):
        assert torch.equal(tdq.qk_norm_rope(x, None, pos, (freq, torch.where(axis == 2, odd, axis).to(torch.int32)))[0], want)


def test_refusals_of_the_binding(tdq):
    x, pos, table = _heads(4, 2, 64, 1, torch.float32), torch.arange(4, device="cuda"), tdq.rope_table(64)
    n0 = tdq.kernel_launch_count()
    w = torch.ones(64, device="cuda")
    for args, kw in [((x[0], None, pos, table), {}), ((x, x[:3], pos, table), {}), ((x, x.half(), pos, table), {}), ((x, None, pos[:3], table), {}),
                     ((x, None, pos, tdq.rope_table(128)), {}), ((x, None, pos, table, w[:32]), {}), ((x, None, pos, table, w), {"eps": None}),
                     ((x, None, pos, table, None, w), {}), ((x, None, pos, table), {"q_out": x[:, :1]}), ((x, None, pos, table), {"q_out": x.half()}),
                     ((x.transpose(1, 2).contiguous().transpose(1, 2), None, pos, table), {}), ((x, None, pos.cpu(), table), {}),
                     ((x, None, pos, (table[0], table[1][:3])), {}), ((x, None, pos.view(1, 1, 4), table), {})]:
        with pytest.raises(ValueError):
            tdq.qk_norm_rope(*args, **kw)
    for args in [(x.double(), None, pos, table), (x, None, pos.int(), table), (x, None, pos, (table[0].float(), table[1])),
                 (x, None, pos, (table[0], table[1].long())), (x, None, pos, table, w.half())]:
        with pytest.raises(TypeError):
            tdq.qk_norm_rope(*args)
    for kw in [{"eps": -1.0}, {"q_out": x[:1].expand(4, 2, 64)}]:
        with pytest.raises(tdq.TdqError) as e:
            tdq.qk_norm_rope(x, None, pos, table, **kw)
        assert e.value.code == tdq.ERR_INVALID_ARG
    assert tdq.kernel_launch_count() == n0


@pytest.mark.parametrize("D", [64, 72])
def test_the_same_tensor_for_both_sides(tdq, D):
    x, pos, table = _heads(9, 3, D, 4, torch.bfloat16), torch.arange(9, device="cuda"), tdq.rope_table(D)
    w = torch.linspace(0.5, 1.5, D, device="cuda")
    before = x.clone()
    q, k = tdq.qk_norm_rope(x, x, pos, table, None, w)    # read twice, written to two new tensors
    assert torch.equal(x, before)
    assert torch.equal(q, tdq.qk_norm_rope(x, None, pos, table)[0]) and torch.equal(k, tdq.qk_norm_rope(x, None, pos, table, w)[0])
    e, k = tdq.qk_norm_rope(x[:, :0], x, pos, table, None, w)   # queries without heads
    assert e.shape == (9, 0, D) and torch.equal(k, tdq.qk_norm_rope(x, None, pos, table, w)[0])
    for kw in [dict(q_out=x), dict(k_out=x), dict(q_out=x, k_out=x), dict(q_out=q, k_out=q)]:
        with pytest.raises(tdq.TdqError) as error:
            tdq.qk_norm_rope(x, x, pos, table, **kw)
        assert error.value.code == tdq.ERR_INVALID_ARG
    assert torch.equal(x, before)


@pytest.mark.parametrize("D", [128, 72])
def test_graph_replay_in_place(tdq, D):
    q, k = _heads(40, 4, D, 1, torch.bfloat16), _heads(40, 2, D, 2, torch.bfloat16)
    pos, table = torch.arange(40, device="cuda"), tdq.rope_table(D)
    qo, ko = torch.empty_like(q), torch.empty_like(k)
    tdq.qk_norm_rope(q, k, pos, table, q_out=qo, k_out=ko)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            tdq.qk_norm_rope(q, k, pos, table, q_out=qo, k_out=ko)
    q.copy_(_heads(40, 4, D, 7, torch.bfloat16))
    pos.add_(1000)
    graph.replay()
    torch.cuda.synchronize()
    want = tdq.qk_norm_rope(q, k, pos, table)
    assert torch.equal(qo, want[0]) and torch.equal(ko, want[1])


def _turns_per_radian():
    """1 / 2 pi as an integer over 2^400: Machin's formula, pi = 16 arctan(1/5) - 4 arctan(1/239), in integers."""
    bits = 460

    def arctan(n):
        term, total, k = (1 << bits) // n, 0, 0
        while term:
            total += (-1) ** k * (term // (2 * k + 1))
            term //= n * n
            k += 1
        return total
    pi = 16 * arctan(5) - 4 * arctan(239)
    return (1 << (400 + bits)) // (2 * pi)


@pytest.mark.parametrize("adjacent", [False, True])
@pytest.mark.parametrize("D", [64, 70])
def test_angles_up_to_positions_of_2_to_the_40(tdq, D, adjacent):
    """Both kernels against angles reduced in integers, where a binary64 product of position and frequency has lost 2^-13 of a turn.

    The pair's fraction of a turn is off by 2^-64 a position at most and by 2^-32 where it is cut, its binary32 form by 2^-25; then two
    units of the cosine (2^-23) and two products and a sum (3 2^-24), relative to the pair's magnitudes."""
    from fractions import Fraction
    turns, half = _turns_per_radian(), D // 2
    freq, axis = tdq.rope_table(2 * half, base=5e5, device="cpu")
    odd = [1.0, math.pi, -math.pi, 2 * math.pi, 3 * math.pi, 7.5, -0.7, 1000.25, 1e6 + 0.1, 2.0 ** -30, 1e-12, 0.0]
    freq[5:5 + len(odd)] = torch.tensor(odd, dtype=torch.float64)
    far = [1 << 40, -(1 << 40), (1 << 40) - 1, (1 << 39) + 12345, (1 << 34) + 77, -(1 << 31) - 5, 1 << 28, 12345, -7, 0]
    x = _heads(len(far), 2, D, 6, torch.float32)
    out, _ = tdq.qk_norm_rope(x, None, torch.tensor(far, device="cuda"), (freq.cuda(), axis.cuda()), eps=None, adjacent=adjacent)
    angle = torch.empty((len(far), half), dtype=torch.float64)
    for i, p in enumerate(far):
        for j, f in enumerate(freq.tolist()):
            t = Fraction(f) * p * turns / (1 << 400)
            angle[i, j] = 2 * math.pi * float(t - round(t))
    c, s = torch.cos(angle).cuda()[:, None], torch.sin(angle).cuda()[:, None]
    a, b = (slice(0, D, 2), slice(1, D, 2)) if adjacent else (slice(0, half), slice(half, D))
    xa, xb = x[..., a].double(), x[..., b].double()
    off = 2.0 ** -64 * torch.tensor(far, device="cuda").abs().double()[:, None, None] + 2.0 ** -32 + 2.0 ** -25
    tol = (xa.abs() + xb.abs()) * (2 * math.pi * off + 2.0 ** -23 + 3 * 2.0 ** -24)
    for got, want in ((out[..., a], xa * c - xb * s), (out[..., b], xb * c + xa * s)):
        assert ((got.double() - want).abs() <= tol).all(), float(((got.double() - want).abs() / tol).max())


@pytest.mark.parametrize("M,hq,hk,D", [(1, 8, 2, 64), (577, 5, 5, 64), (300, 6, 2, 72)])
def test_four_bit_qkv_layer_then_rotation_in_place(tdq, M, hq, hk, D):
    """The 4-bit layer's bf16 output, its query and key channels turned where they are, each stage against its own reference."""
    import oracle
    from parity_utils import compare_y
    C, O = 320, (hq + 2 * hk) * D
    g = torch.Generator().manual_seed(M)
    x, w = torch.randn((M, C), generator=g), 0.05 * torch.randn((O, C), generator=g)
    codes, scale = tdq.quantize_act(x.cuda())
    wcodes, wscale = tdq.quantize_weight(w.cuda())
    qkv = tdq.w4a4_linear(codes, scale, wcodes, wscale, out_dtype=torch.bfloat16)
    xa, wq = oracle.quantize_act(x.numpy()), oracle.quantize_weight(w.numpy())
    # half a step of bf16, of a number that is off by the sum's bound itself
    compare_y(qkv.float().cpu().numpy(), oracle.w4a4_linear(xa["codes"], xa["scale"], wq["codes"], wq["scale"]), C // 32, out_eps=1.01 * 2.0 ** -8)
    before = qkv.clone()
    q, k = qkv[:, :hq * D].view(M, hq, D), qkv[:, hq * D:(hq + hk) * D].view(M, hk, D)
    at = torch.arange(M, device="cuda")
    pos = torch.stack([at // 24, at % 24], 1).contiguous()
    freq, axis = tdq.rope_table(D, [D // 4, D // 4], restart=True)
    qw, kw = 1 + 0.1 * torch.randn((D,), generator=g).cuda(), 1 + 0.1 * torch.randn((D,), generator=g).cuda()
    tdq.qk_norm_rope(q, k, pos, (freq, axis), qw, kw, q_out=q, k_out=k)
    for now, was, weight in ((q, before[:, :hq * D].view(M, hq, D), qw), (k, before[:, hq * D:(hq + hk) * D].view(M, hk, D), kw)):
        fu.check_rope(now, *fu.rope(was, weight, pos, freq, axis.long(), 1e-6, False))
    assert torch.equal(qkv[:, (hq + hk) * D:], before[:, (hq + hk) * D:])       # the values stay
