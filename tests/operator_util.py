"""Plain 64-bit forms of dare_k_linear, dare_k_rope and dare_k_attention_packed on the CPU, each with a bound of what a kernel
that sums in fp32 and rounds where the operator says so may be off by.

u = finfo.eps / 2 of a type: the largest relative error of one rounding (bf16 2^-8, fp32 2^-24)."""
import math

import torch

U32 = 2.0 ** -24
HALF_STEP = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def rand(gen, *shape, dtype="f32", std=1.0):
    return (torch.randn(shape, generator=gen, dtype=torch.float64) * std).to(DTYPES[dtype])


def act64(act, z):
    if act is None:
        return z
    if act == "silu":
        return z / (1 + torch.exp(-z))
    if act == "gelu":
        return z * torch.special.ndtr(z)
    return 0.5 * z * (1 + torch.tanh(math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3)))


def linear64(a, wt, bias, act, residual):
    """(value, bound).  The product of k terms summed in fp32 in any order is off by at most k u32 sum |a w|; the activations
    have slopes below 1.13; their own fp32 forms are off by 2^-20 (|z| + 1) at most (exponentials of arguments up to 90 whose
    rounding is 90 u32 relative, times a few operations; the erfc formula 1.5e-7 |z|); then the sums with bias and
    residual, and the rounding to the type."""
    u = HALF_STEP[a.dtype]
    k = a.shape[1]
    prod, size = a.double() @ wt.double().t(), a.double().abs() @ wt.double().abs().t()
    z = prod if bias is None else prod + bias.double()
    err = (k + 2) * U32 * (size + (0 if bias is None else bias.double().abs()))
    y = act64(act, z)
    if act is not None:
        err = 1.13 * err + 2.0 ** -20 * (z.abs() + 1)
    out = y if residual is None else y + residual.double()
    err = err + 2 * U32 * (y.abs() + out.abs())
    return out, err + u * (out.abs() + err)


def rope64(x, pos, freqs, rot, layout, magnitude):
    """(value, bound): cos and sin times the magnitude rounded to fp32 once, two products and a sum in fp32, one rounding."""
    u = HALF_STEP[x.dtype]
    ang = pos.double()[:, None] * freqs.double()[None, :]
    cos, sin = (torch.cos(ang) * magnitude)[:, None], (torch.sin(ang) * magnitude)[:, None]
    y, err = x.double().clone(), torch.zeros(x.shape, dtype=torch.float64)
    ia = torch.arange(0, rot, 2) if layout == "pairs" else torch.arange(rot // 2)
    ib = ia + (1 if layout == "pairs" else rot // 2)
    a, b = x.double()[..., ia], x.double()[..., ib]
    y[..., ia], y[..., ib] = a * cos - b * sin, b * cos + a * sin
    slack = 4 * U32 * abs(magnitude) * (a.abs() + b.abs())
    err[..., ia], err[..., ib] = slack, slack
    err[..., :rot] += u * (y[..., :rot].abs() + err[..., :rot])
    return y, err


def limit(i, len_q, len_k, block):
    """Keys that query token i of a sequence sees."""
    pos = i + len_k - len_q
    return len_k if block == 0 else max(0, min(len_k, (pos // block + 1) * block))


def attention64(q, k, v, q_off, k_begin, k_end, block, scale):
    """(value, bound, covered): covered marks the rows of out that belong to a sequence.
    A logit is off by D u32 times the sum of its terms' sizes, its weight by that and the roundings of the exponential's argument
    (2 u32 |z|) and of the exponential (4 u32) relative; the sum of n weights by n u32; bf16 rounds the weights (u of each).
    All of it is relative to a mean of |v| under the weights."""
    u = HALF_STEP[q.dtype]
    h, d = q.shape[1:]
    g = h // k.shape[1]
    out, err = torch.zeros(q.shape, dtype=torch.float64), torch.zeros(q.shape, dtype=torch.float64)
    covered = torch.zeros(q.shape[0], dtype=torch.bool)
    kd, vd = k.double().repeat_interleave(g, 1), v.double().repeat_interleave(g, 1)
    for b in range(len(k_begin)):
        lq, lk = q_off[b + 1] - q_off[b], k_end[b] - k_begin[b]
        covered[q_off[b]:q_off[b + 1]] = True
        for i in range(lq):
            n = limit(i, lq, lk, block)
            if n == 0:
                continue
            kk, vv = kd[k_begin[b]:k_begin[b] + n], vd[k_begin[b]:k_begin[b] + n]
            qq = q[q_off[b] + i].double()
            z = torch.einsum("hd,nhd->hn", qq, kk) * scale
            size = torch.einsum("hd,nhd->hn", qq.abs(), kk.abs()) * scale
            w = torch.softmax(z, -1)
            y = torch.einsum("hn,nhd->hd", w, vv)
            mean = torch.einsum("hn,nhd->hd", w, vv.abs())
            worst = (U32 * (d * size + 2 * z.abs()).amax(-1, keepdim=True) + (n + 16) * U32)
            rel = 2 * worst + (2 * u if q.dtype == torch.bfloat16 else 0.0)
            e = rel * mean
            out[q_off[b] + i], err[q_off[b] + i] = y, e + u * (y.abs() + e)
    return out, err, covered


def worst(got, want, bound):
    """Largest error as a share of its bound; infinity where one side only is finite."""
    got = got.double().cpu()
    bad = torch.isfinite(got) != torch.isfinite(want)
    share = ((got - want).abs() / (bound + 1e-30)).nan_to_num(0.0)
    share[bad] = math.inf
    return float(share.max()) if share.numel() else 0.0


# dare_k_linear in bf16: (route, rows, columns, k), every route of its launch, ragged in rows and, but for the first three, in the columns of the tile
LINEAR_SHAPES = [
    ("kSkinny", 5, 448, 4352), ("k32x32", 19, 320, 4160), ("k64x32", 65, 1088, 1024), ("k64x64", 65, 4160, 2112), ("k64x96", 65, 8320, 1088),
    ("k64x128", 65, 12352, 576), ("k64x128", 1, 126464, 192), ("k128x96", 130, 11008, 960), ("k128x128", 130, 12352, 704),
    ("k128x192", 258, 11008, 1024), ("kPp128", 386, 8256, 2048), ("kPp192", 514, 11008, 1024), ("kPp256", 770, 12352, 1024),
    ("kQuad192", 1026, 13120, 192), ("kQuad256", 1538, 14144, 192),
    ("kQuad256", 770, 12352, 4160),      # one round of tiles, a long k
    ("kQuad256", 4617, 15424, 192),      # more than 128 MB of outputs, which are stored past the L2
]
