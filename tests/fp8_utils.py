"""Plain 64-bit forms of the 8-bit floating point layer and of the norm and rotation, and the tolerances they are compared with."""
import numpy as np
import torch

BLOCK = 128
DT = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
HALF_STEP = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}


# Layers (M, I, O) for each way that the layer is computed in on 148 SMs: (tile's tokens, tile's output channels, parts of the contraction).  Ragged in every
# direction; a block a part or less than two, a few that do not divide, more than the ring and the factors' places hold; for pairs of CTAs 1, 2, 5, 6, 9 and 33
# blocks in one round of tiles, two and three.  128 tokens in one part is never chosen.
WAYS = {
    (16, 128, 1): [(9, 2175, 17908), (23, 639, 8035), (12, 91, 937)],
    (16, 128, 2): [(12, 4223, 8598), (35, 796, 2214), (8, 219, 347)],
    (16, 128, 3): [(5, 6875, 4906), (9, 897, 4919), (2, 284, 74)],
    (16, 128, 4): [(46, 8575, 1289), (14, 6016, 4106), (23, 385, 203)],
    (16, 128, 5): [(51, 13953, 775), (206, 2139, 164), (22, 540, 55)],
    (16, 128, 6): [(356, 15132, 119), (44, 8988, 1020), (23, 731, 315)],
    (16, 128, 7): [(54, 17152, 529), (150, 4124, 101), (7, 796, 654)],
    (16, 128, 8): [(21, 17023, 67), (30, 8193, 75), (53, 987, 203)],
    (32, 128, 1): [(23, 2431, 12559), (22, 511, 19916), (26, 1, 35559)],
    (32, 128, 2): [(17, 4224, 8310), (27, 2907, 7201)],
    (32, 128, 3): [(19, 6273, 4828), (27, 895, 10621), (17, 284, 10220)],
    (32, 128, 4): [(19, 8348, 4418), (19, 4097, 4606)],
    (32, 128, 5): [(28, 10396, 3159), (846, 2176, 51)],
    (32, 128, 6): [(29, 13825, 2782), (346, 4380, 156)],
    (32, 128, 7): [(157, 15489, 460), (27, 2560, 2625)],
    (32, 128, 8): [(53, 16987, 1142), (506, 8575, 34)],
    (64, 128, 1): [(39, 2305, 15582), (46, 896, 15234), (34, 128, 39489)],
    (64, 128, 2): [(58, 4353, 7643), (147, 1883, 2577)],
    (64, 128, 3): [(46, 6529, 5010), (860, 1663, 257), (2593, 384, 118)],
    (64, 128, 4): [(54, 10241, 3740), (58, 4864, 4730)],
    (64, 128, 5): [(35, 11995, 3220), (1844, 2139, 68), (600, 513, 525)],
    (64, 128, 6): [(51, 12801, 2730), (744, 5532, 135)],
    (64, 128, 7): [(151, 17792, 855), (44, 5248, 2255)],
    (64, 128, 8): [(828, 17792, 74), (250, 4992, 410)],
    (128, 128, 2): [(441, 8923, 1766), (1592, 2561, 460)],
    (128, 128, 3): [(132, 13403, 2108), (4945, 1564, 119)],
    (128, 128, 4): [(155, 16768, 1939), (3409, 3291, 87)],
    (128, 128, 5): [(634, 15873, 612), (242, 2432, 1204)],
    (128, 128, 6): [(492, 13439, 446), (1268, 3841, 165)],
    (128, 128, 7): [(88, 3100, 1902)],
    (128, 128, 8): [(231, 16603, 726), (68, 10369, 1429)],
    (256, 128, 1): [(1354, 127, 898), (3658, 1, 1085), (2534, 1, 2235), (2594, 156, 140), (3313, 255, 1383), (1478, 156, 4055),
                    (2543, 4124, 630), (3139, 4187, 1329), (6349, 540, 41), (1750, 513, 2580), (5641, 540, 1095), (4626, 668, 155),
                    (865, 768, 4694), (6160, 668, 983), (1176, 1151, 919), (3659, 1052, 1025), (749, 1025, 8099)],
    (256, 256, 1): [(1688, 91, 2164), (3952, 128, 1779), (1612, 91, 7339), (1069, 156, 3217), (1296, 219, 5228), (606, 156, 13082),
                    (1285, 4187, 2865), (4404, 4224, 1510), (615, 513, 5015), (2082, 639, 3932), (704, 603, 16014), (1718, 731, 1850),
                    (3595, 731, 2178), (1647, 641, 5829), (4043, 1025, 674), (5783, 1025, 1369), (866, 1151, 13519)],
}


def blocks(n):
    return (n + BLOCK - 1) // BLOCK


def e4m3_values():
    """The 256 codes' values (NaN at 0x7F and 0xFF) from the format's definition: 4 exponent bits (bias 7), 3 mantissa bits."""
    b = np.arange(256)
    e, m = (b >> 3) & 15, b & 7
    v = np.where(e == 0, m * 2.0 ** -9, (8 + m) * 2.0 ** (e - 10.0))
    v = np.where((b & 0x7F) == 0x7F, np.nan, v)
    return np.where(b >= 128, -v, v)


def nearest_code(q):
    """E4M3 code next to each |q| <= 464 (float64), ties to the even mantissa, by comparing with the midpoints of the codes' values."""
    v = e4m3_values()[:127]
    mid = (v[:-1] + v[1:]) / 2                     # exact
    a = np.abs(q)
    code = np.searchsorted(mid, a, side="left")    # mid[code-1] < a <= mid[code]
    tie = (code < 126) & (a == mid[np.minimum(code, 125)])
    code = np.where(tie & (code % 2 == 1), code + 1, code)
    return np.where(np.signbit(q), code + 128, code).astype(np.uint8)


def quantize(x, rows_per):
    """Codes [M, C_pad] (uint8) and scales of x [M, C] (numpy float32, the input's values) by blocks of rows_per x 128."""
    M, C = x.shape
    K, T = blocks(C), (M + rows_per - 1) // rows_per
    p = np.zeros((T * rows_per, K * BLOCK), np.float32)
    p[:M, :C] = x
    p = p.reshape(T, rows_per, K, BLOCK)
    bad = ~np.isfinite(p).all((1, 3))
    p = np.where(np.isfinite(p), p, np.float32(0))
    a = np.maximum(np.abs(p).max((1, 3)), np.float32(2.0 ** -64))
    a = np.where(bad, np.float32(np.finfo(np.float32).max), a)
    scale, r = a / np.float32(448.0), np.float32(448.0) / a
    assert scale.dtype == r.dtype == np.float32
    codes = nearest_code((p * r[:, None, :, None]).astype(np.float64))
    codes = np.where(bad[:, None, :, None], np.uint8(0x7F), codes)
    scale = np.where(bad, np.float32(np.nan), scale)
    return codes.reshape(T * rows_per, K * BLOCK)[:M], scale


def linear(xc, xs, wc, ws, bias):
    """(y, sum of absolute terms) in float64 on the tensors' device; codes uint8 or float8."""
    val = torch.tensor(e4m3_values(), dtype=torch.float64, device=xc.device)
    idx = lambda c: val[c.view(torch.uint8).long()]  # noqa: E731
    x = idx(xc) * xs.double().repeat_interleave(BLOCK, 1)
    w = idx(wc) * ws.double().repeat_interleave(BLOCK, 1).repeat_interleave(BLOCK, 0)[:wc.shape[0]]
    y, t = x @ w.t(), x.abs() @ w.abs().t()
    return (y, t) if bias is None else (y + bias.double(), t + bias.double().abs())


def linear_tolerance(y, t, K, dtype):
    """Inside an instruction 32 exact products and the accumulator are aligned to the largest of them and cut to binary32's 24 bits
    or one more: 33 cuts of 2^-25 each, four instructions a block, relative to the terms' absolute sum.  Then per block a
    rounded factor and a rounded multiply-add, the additions of parts and the bias, half a step of binary32 each, and half a step
    of y's type (denormal fp16 outputs: half of 2^-24)."""
    return t * (4 * 33 * 2.0 ** -25 + (3 * K + 8) * 2.0 ** -24) + y.abs() * HALF_STEP[dtype] * 1.01 + (2.0 ** -25 if dtype == torch.float16 else 0.0)


def check_linear(y, ref, t, K):
    assert torch.equal(torch.isnan(y), torch.isnan(ref))
    tol = linear_tolerance(ref, t, K, y.dtype)
    if y.dtype == torch.float16:   # numbers from 65520 on, half a step of 32 above the largest, round to infinity
        sums = linear_tolerance(ref, t, K, torch.float32)
        inf = torch.isinf(y)
        assert (ref.abs() + sums)[inf].ge(65520).all() and ((ref.abs() - sums)[~inf] < 65520).all()
        assert (y[inf].double() * ref[inf] > 0).all()
        y, ref, tol = y[~inf], ref[~inf], tol[~inf]
    err = (y.double() - ref).abs()
    assert not (err > tol).any(), "%d outputs off, worst %.3g of the tolerance" % (int((err > tol).sum()), float((err / tol).nan_to_num().max()))


def rope(x, weight, pos, freq, axis, eps, adjacent):
    """(out, tolerance without the output's rounding) in float64 for x [M, H, D]; pos [M, A] int64, freq float64, axis int64."""
    D = x.shape[2]
    n = x.double()
    rel = 2.0 ** -24
    if eps is not None:
        n = n / torch.sqrt(n.square().mean(-1, keepdim=True) + eps)
        if weight is not None:
            n = n * weight.double()
        # a sum of D squares and its mean (half of it survives the root), a reciprocal root of two units, three products
        rel = (D / 2 + 2 + 4 + 4) * 2.0 ** -24
    out, tol = n.clone(), n.abs() * rel
    half = freq.numel()
    if half:
        t = pos[:, axis].double() * freq
        c, s = torch.cos(t)[:, None], torch.sin(t)[:, None]
        a, b = (slice(0, 2 * half, 2), slice(1, 2 * half, 2)) if adjacent else (slice(0, half), slice(half, 2 * half))
        na, nb = n[..., a], n[..., b]
        out[..., a], out[..., b] = na * c - nb * s, nb * c + na * s
        # the fraction of a turn to 2^-25, two units of the cosine, the angle in binary64, two products and a sum
        e = (na.abs() + nb.abs()) * (rel + 2 * np.pi * 2.0 ** -25 + 2.0 ** -23 + 3 * 2.0 ** -24 + (t.abs() * 2.0 ** -51)[:, None])
        tol[..., a] = e
        tol[..., b] = e
    return out, tol


def check_rope(y, ref, tol):
    tol = tol * (1 + HALF_STEP[y.dtype]) + ref.abs() * HALF_STEP[y.dtype] * 1.01 + (2.0 ** -25 if y.dtype == torch.float16 else 1e-38)
    err = (y.double() - ref).abs()
    assert (err <= tol).all(), "worst %.3g of the tolerance" % float((err / tol).nan_to_num(1e9).max())
