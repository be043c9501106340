"""Plain 64-bit forms of dare_k_norm_q8, dare_k_linear_q8 and dare_k_logprobs on the CPU, with bounds of what a kernel that rounds where the
operator says so may be off by (U32 = 2^-24, the largest relative error of one rounding to fp32)."""
import math

import numpy as np
import torch

from operator_util import HALF_STEP, U32, act64


def norm64(kind, x, o, gain, bias, eps):
    """(s in the type, y in 64 bits).  s: one sum in fp32 and one rounding to the type."""
    s = x if o is None else (x.float() + o.float()).to(x.dtype)
    y = s.double()
    if kind == "layer":
        y = y - y.mean(1, keepdim=True)
    if kind is not None:
        y = y / torch.sqrt((y * y).mean(1, keepdim=True) + eps) * gain.double()
    if kind == "layer" and bias is not None:
        y = y + bias.double()
    return s, y


def check_codes(y, codes, scales):
    """scales: max |y| / 127 within one rounding to fp32.  codes: the nearest whole number to y / scale, as it is for every y that is not within 1e-9 of
    the middle between two (sums of up to 2^15 terms in 64 bits are off by less than 2^-37)."""
    codes, scales = codes.cpu().double(), scales.cpu()
    want = y.abs().amax(1) / 127
    assert ((scales.double() - want).abs() <= U32 * (1 + 1e-6) * want).all()
    step = scales.double()[:, None]
    q = torch.where(step > 0, y / step.clamp(min=1e-300), torch.zeros_like(y))
    border = ((q - torch.floor(q)) - 0.5).abs() < 1e-9
    nearest = torch.round(q)
    assert torch.equal(codes[~border], nearest[~border])
    assert ((codes - q).abs() <= 0.5 + 1e-8).all()
    return int(border.sum())


def linear_q8_64(a, sa, wt, sw, bias, act, residual, dtype):
    """(value, bound).  The sum is exact; its rounding to fp32, two products and the sum with the bias are off by 4 U32 of the sizes; activations as in
    linear64 (slopes below 1.13, their own forms within 2^-20 (|z| + 1)); the sum with the residual, and the rounding to the type."""
    u = HALF_STEP[dtype]
    prod = (a.double() @ wt.double().t()) * sa.double()[:, None] * sw.double()
    z = prod if bias is None else prod + bias.double()
    err = 4 * U32 * (prod.abs() + z.abs())
    y = act64(act, z)
    if act is not None:
        err = 1.13 * err + 2.0 ** -20 * (z.abs() + 1)
    out = y if residual is None else y + residual.double()
    err = err + 2 * U32 * (y.abs() + out.abs())
    return out, err + u * (out.abs() + err)


def logprobs64(x, tokens, scale, top):
    """logprob, entropy, ids, top log-probabilities, and the bounds of the three that are computed.
    In units of 2: an exponent d = c (x - m) has the roundings of the difference, of c (two) and of the product, 4 U32 of itself; the exponential 2 U32
    more; a sum over a row goes through chains of up to vocab / 256 + 64 roundings, whatever the kernel's number of lanes, and as many where its maximum moves."""
    v = x.double()
    rows, vocab = v.shape
    finite = v > -math.inf
    m = torch.where(finite, v, torch.full_like(v, -1e300)).amax(1, keepdim=True)
    z = (v - m) * scale
    e = torch.where(finite, torch.exp(z), torch.zeros_like(v))
    total = e.sum(1)
    has = total > 0
    log_sum = torch.log(total.clamp(min=1e-300))
    dist = torch.where(e > 0, -z, torch.zeros_like(z)) / math.log(2)
    d1, d2 = (e * dist).sum(1) / total.clamp(min=1e-300), (e * dist * dist).sum(1) / total.clamp(min=1e-300)
    chain = 2 * (vocab / 256 + 64)
    err_log = U32 * (4 * d1 + 2 + chain + 4 * log_sum.abs())
    inside = (tokens >= 0) & (tokens < vocab)
    picked = z.gather(1, tokens.long().clamp(0, vocab - 1)[:, None])[:, 0]
    picked = torch.where(inside & torch.isfinite(picked) & has, picked, torch.full_like(picked, -math.inf))
    lp = torch.where(torch.isfinite(picked), picked - log_sum, picked)
    bound = err_log + 6 * U32 * picked.abs().nan_to_num(0.0, 0.0, 0.0)
    entropy = torch.where(has, log_sum + math.log(2) * d1, torch.zeros_like(d1))
    bound_h = err_log + U32 * (4 * d2 + 8 * d1 + 2 * chain * d1)
    order = np.lexsort((np.broadcast_to(np.arange(vocab), v.shape), -(v.numpy() + 0.0)), axis=1)[:, :top]
    order = torch.from_numpy(np.ascontiguousarray(order))
    tops = z.gather(1, order)
    gone = ~torch.isfinite(v.gather(1, order))
    ids = torch.where(gone, torch.full_like(order, -1), order)
    top_lp = torch.where(gone, torch.full_like(tops, -math.inf), tops - log_sum[:, None])
    top_bound = err_log[:, None] + 6 * U32 * torch.where(gone, torch.zeros_like(tops), tops.abs())
    return lp, bound, entropy, bound_h, ids, top_lp, top_bound


# dare_k_linear_q8 with bf16 outputs: (shape, rows, columns, k), every shape of its launch, ragged in rows and columns of the tile but where one row or the
# columns' multiple of 64 leaves nothing ragged
LINEAR_Q8_SHAPES = [
    ("kSkinny", 5, 448, 8704), ("k32x32", 19, 320, 8320), ("k32x32", 65, 1088, 2048), ("k64x32", 213, 1344, 768), ("k64x64", 65, 4160, 4224),
    ("k64x64", 2, 8256, 2176), ("k32x64", 1, 126464, 384), ("k32x64", 3, 50048, 128), ("k128x192", 3, 40000, 128), ("k128x192", 61, 46464, 256), ("k32x64", 32, 66624, 384), ("k64x96", 65, 8320, 2176),
    ("k64x96", 650, 1728, 384), ("k64x96", 20, 18944, 128), ("k64x128", 65, 12352, 1152), ("k64x128", 36, 26560, 384), ("k128x96", 130, 11008, 1920),
    ("k128x96", 1287, 1792, 256), ("k128x128", 130, 12352, 1408), ("k128x128", 1024, 4096, 384), ("k128x192", 258, 11008, 2048),
    ("k128x192", 777, 6144, 256), ("kQuad192", 514, 11008, 2048), ("kQuad192", 1026, 13120, 384), ("kQuad192", 877, 9856, 384),
    ("kQuad192", 259, 66624, 384), ("kQuad256", 770, 12352, 2048), ("kQuad256", 1538, 14144, 384),
    ("kQuad256", 770, 12352, 8320),      # one round of tiles, a long k
    ("kQuad256", 4617, 15424, 384),      # more than 128 MB of outputs, which are stored past the L2
]

# (columns, k, numbers of rows): calls whose common rows have the same bits although their tiles have other shapes; together every shape there is
LINEAR_Q8_ROWS = [
    (4096, 384, (5, 9, 70, 140, 260, 330, 520, 650, 1030, 1420)),
    (12352, 384, (3, 70, 140, 260, 390, 770)),
    (15424, 384, (5, 300, 4617)),        # the last one stored past the L2
    (66624, 384, (3, 40, 259)),
]
