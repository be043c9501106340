"""dare_k_norm_q8, dare_k_linear_q8 and dare_k_logprobs against their plain 64-bit forms, and as the end of a step together."""
import math

import pytest
import torch

from paper_2605_08134_amd import binding as B
import operator_util as ou
import step8_util as su

pytestmark = pytest.mark.gpu

TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def _gen(seed):
    return torch.Generator().manual_seed(seed)


def _padded(t, pad, fill=float("nan")):
    """t on the GPU as a view of a buffer with `pad` elements of something else behind every row."""
    buf = torch.full((t.shape[0], t.shape[1] + pad), fill, dtype=t.dtype, device="cuda")
    buf[:, :t.shape[1]] = t.cuda()
    return buf[:, :t.shape[1]]


def _behind(t):
    """What lies behind the rows of a view made by _padded."""
    return t._base[:, t.shape[1]:]


# ---- normalisation into codes -------------------------------------------------------------------

def _norm(kind, x, o=None, keep=False, gain=None, bias=None, eps=1e-5, pad=0):
    codes = _padded(torch.full(x.shape, 77, dtype=torch.int8), pad, 99)
    scales = torch.full((x.shape[0],), 7.0, device="cuda")
    s = _padded(torch.zeros_like(x), pad) if keep else None
    dev = lambda t: None if t is None else t.cuda()
    B.dare_k_norm_q8(kind, _padded(x, pad), codes, scales, None if o is None else _padded(o, 2 * pad), s, dev(gain), dev(bias), eps)
    if pad:
        assert (_behind(codes) == 99).all() and (s is None or torch.isnan(_behind(s)).all())
    return codes, scales, s


@pytest.mark.parametrize("kind", [None, "layer", "rms"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,d,pad", [(1, 8, 0), (3, 64, 8), (5, 512, 0), (9, 520, 16), (7, 1544, 0), (4, 2048, 8), (3, 2056, 0), (6, 4096, 0),
                                        (2, 4104, 8), (2, 8192, 0), (3, 8200, 0), (2, 16384, 8), (3, 16392, 8), (2, 40000, 0), (1, 131008, 0)])
@pytest.mark.parametrize("extras", ["none", "sum", "sum kept"])
def test_norm_q8(kind, dtype, rows, d, pad, extras):
    g = _gen(rows * d)
    x = ou.rand(g, rows, d, dtype=dtype, std=3.0)
    o = None if extras == "none" else ou.rand(g, rows, d, dtype=dtype)
    gain = None if kind is None else (1 + 0.2 * torch.randn(d, generator=g)).to(x.dtype)
    bias = ou.rand(g, d, dtype=dtype) if kind == "layer" and extras != "none" else None
    codes, scales, s = _norm(kind, x, o, extras == "sum kept", gain, bias, 1e-5, pad)
    ws, y = su.norm64(kind, x, o, gain, bias, 1e-5)
    borders = su.check_codes(y, codes, scales)
    assert borders <= 1e-4 * y.numel()
    if s is not None:
        assert torch.equal(s.cpu(), ws)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 4096, 16392])
@pytest.mark.parametrize("place", ["x", "o"])
def test_norm_q8_sum_in_place(dtype, d, place):
    g = _gen(d)
    x, o = ou.rand(g, 5, d, dtype=dtype).cuda(), ou.rand(g, 5, d, dtype=dtype).cuda()
    gain = ou.rand(g, d, dtype=dtype).cuda()
    one = [torch.empty(5, d, dtype=torch.int8, device="cuda"), torch.empty(5, device="cuda")]
    two = [torch.empty_like(t) for t in one]
    s = torch.empty_like(x)
    for kind in ("rms", "layer", None):
        xx, oo = x.clone(), o.clone()
        B.dare_k_norm_q8(kind, x, *one, o, s, gain if kind else None)
        B.dare_k_norm_q8(kind, xx, *two, oo, xx if place == "x" else oo, gain if kind else None)
        assert torch.equal(one[0], two[0]) and torch.equal(one[1], two[1])
        assert torch.equal(s, xx if place == "x" else oo) and torch.equal(x if place == "o" else o, xx if place == "o" else oo)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 1024, 16400])
def test_norm_q8_special_rows(dtype, d):
    x = torch.randn(9, d, generator=_gen(d)).to(TYPES[dtype])
    x[0] = 0
    x[1, d - 1] = float("inf")
    x[2, 3] = float("nan")
    x[3, 5] = float("-inf")
    x[4] = 3e38                      # squares beyond fp32
    x[5] *= 1e-30                    # squares below fp32
    x[6] = 0
    x[6, 2] = 2e-45 if dtype == "f32" else 1e-40     # a scale of 0, or no normal number
    x[7] = torch.arange(d) % 255 - 127               # whole numbers: codes are the values
    gain = torch.ones(d, dtype=x.dtype)
    for kind in (None, "rms", "layer"):
        codes, scales, _ = _norm(kind, x, gain=gain if kind else None, eps=0.0 if kind == "rms" else 1e-5)
        codes, scales = codes.cpu(), scales.cpu()
        for r in (1, 2, 3):
            assert torch.isnan(scales[r]) and (codes[r] == 0).all()
        if kind != "rms":            # (eps 0: 0 / 0)
            assert scales[0] == 0 and (codes[0] == 0).all()
        else:
            assert torch.isnan(scales[0]) and (codes[0] == 0).all()
        good = [4, 5, 7, 8]
        _, y = su.norm64(kind, x, None, gain, None, 0.0 if kind == "rms" else 1e-5)
        su.check_codes(y[good], codes[good], scales[good])
        if kind is None:
            assert scales[7] == 1 and torch.equal(codes[7].double(), x[7].double())
            got = codes[6].double() * scales[6].double()    # no code beyond 127, and within a scale of the value where that is not 0
            assert scales[6] == 0 or (got - x[6].double()).abs().max() <= scales[6]
            assert codes[6].abs().max() <= 127
        # a gain that is not finite reaches the whole row, a channel that it multiplies with 0 too
        if kind:
            bad = gain.clone()
            bad[1] = float("nan")
            codes, scales, _ = _norm(kind, x[8:], gain=bad)
            assert torch.isnan(scales).all() and (codes == 0).all()


@pytest.mark.parametrize("d", [40000, 8000])
def test_norm_q8_scales_beyond_fp32(d):
    """y of up to sqrt(d) times the gain: a scale that fp32 does not hold is NaN, the largest that it holds is right."""
    x, gain = torch.zeros(2, d), torch.ones(d)
    x[0, 7], x[1] = 1.0, torch.randn(d, generator=_gen(1))
    gain[7] = 3e38
    codes, scales, _ = _norm("rms", x, gain=gain, eps=0.0)
    _, y = su.norm64("rms", x, None, gain, None, 0.0)
    if float(y[0].abs().max()) / 127 > torch.finfo(torch.float32).max:
        assert torch.isnan(scales[0]) and (codes[0] == 0).all()
    else:
        su.check_codes(y[:1], codes[:1], scales[:1])
    su.check_codes(y[1:], codes[1:], scales[1:])


def test_norm_q8_ties_go_to_the_even_code():
    """Values in the middle between two codes, with a scale that is no power of two in f32."""
    for dtype, step in (("bf16", 1.0), ("f32", 1.0), ("f32", 0.6875)):
        step = float(torch.tensor(step, dtype=torch.float32))
        x = torch.zeros(1, 256, dtype=torch.float64)
        x[0, :255] = (torch.arange(255) - 127) * (0.5 * step)
        x[0, 255] = 127 * step
        x = x.to(TYPES[dtype])
        if not torch.equal(x.double()[0, :255], (torch.arange(255) - 127) * (0.5 * step)):
            continue    # (no middles in this type)
        codes, scales, _ = _norm(None, x)
        assert scales[0] == torch.tensor(float(x[0, 255]) / 127, dtype=torch.float32)
        want = torch.round(x.double() / scales.cpu().double())
        assert torch.equal(codes.cpu().double(), want)


def test_norm_q8_of_no_rows_and_weights():
    e = torch.empty(0, 64, device="cuda")
    B.dare_k_norm_q8("rms", e, torch.empty(0, 64, dtype=torch.int8, device="cuda"), torch.empty(0, device="cuda"), gain=torch.ones(64, device="cuda"))
    w = torch.randn(256, 192, generator=_gen(1)).bfloat16()       # [k, n]
    wt = B.dare_k_pack_weight(w.cuda())
    codes, scales = torch.empty(192, 256, dtype=torch.int8, device="cuda"), torch.empty(192, device="cuda")
    B.dare_k_norm_q8(None, wt, codes, scales)
    su.check_codes(w.t().double(), codes, scales)


# ---- projection of codes ------------------------------------------------------------------------

def _codes(g, *shape):
    return torch.randint(-127, 128, shape, generator=g, dtype=torch.int8)


def _linear(a, sa, wt, sw, bias, act, res, dtype, pads=(64, 8, 16)):
    out = _padded(torch.zeros(a.shape[0], wt.shape[0], dtype=TYPES[dtype]), pads[1])
    dev = lambda t: None if t is None else t.cuda()
    B.dare_k_linear_q8(_padded(a, pads[0], 55), sa.cuda(), wt.cuda(), sw.cuda(), out, dev(bias), act,
                       None if res is None else _padded(res, pads[2]))
    assert torch.isnan(_behind(out)).all()
    return out


@pytest.mark.parametrize("act", [None, "silu", "gelu", "gelu_tanh"])
@pytest.mark.parametrize("dtype,m,n,k", [
    ("bf16", 1, 64, 128), ("bf16", 8, 128, 1024), ("bf16", 17, 192, 640), ("bf16", 33, 8192, 128), ("bf16", 2, 8256, 256),
    ("bf16", 200, 320, 384), ("bf16", 257, 1088, 896), ("f32", 1, 64, 128), ("f32", 7, 192, 8192), ("f32", 37, 192, 256), ("f32", 130, 576, 640),
])
@pytest.mark.parametrize("extras", ["none", "bias", "residual", "both"])
def test_linear_q8(act, dtype, m, n, k, extras):
    g = _gen(m * 31 + n)
    a, wt = _codes(g, m, k), _codes(g, n, k)
    sa, sw = torch.rand(m, generator=g) * 0.03, torch.rand(n, generator=g) * 0.02 / math.sqrt(k)
    bias = ou.rand(g, n, dtype=dtype) if extras in ("bias", "both") else None
    res = ou.rand(g, m, n, dtype=dtype) if extras in ("residual", "both") else None
    want, bound = su.linear_q8_64(a, sa, wt, sw, bias, act, res, TYPES[dtype])
    assert ou.worst(_linear(a, sa, wt, sw, bias, act, res, dtype), want, bound) <= 1.0


@pytest.mark.parametrize("shape,m,n,k", su.LINEAR_Q8_SHAPES)
@pytest.mark.parametrize("dtype,act,extras", [("bf16", None, False), ("bf16", "gelu", True), ("f32", "silu", True)])
def test_linear_q8_in_every_shape(shape, m, n, k, dtype, act, extras):
    g = torch.Generator(device="cuda").manual_seed(m + n)
    codes = lambda *s: torch.randint(-127, 128, s, generator=g, dtype=torch.int8, device="cuda")
    td = TYPES[dtype]
    a, wt, sa, sw = codes(m, k), codes(n, k), torch.rand(m, generator=g, device="cuda") * 0.02, torch.rand(n, generator=g, device="cuda") * 0.02
    rn = lambda *s: torch.randn(s, generator=g, device="cuda").to(td)
    bias, res = (rn(n), rn(m, n)) if extras else (None, None)
    out = torch.full((m, n), float("nan"), dtype=td, device="cuda")
    B.dare_k_linear_q8(a, sa, wt, sw, out, bias, act, res)
    rows = torch.cat([torch.arange(0, m, 97), torch.tensor([m - 1])]).unique().cuda()
    cpu = lambda t, r=None: None if t is None else (t if r is None else t[r]).cpu()
    want, bound = su.linear_q8_64(cpu(a, rows), cpu(sa, rows), cpu(wt), cpu(sw), cpu(bias), act, cpu(res, rows), td)
    assert ou.worst(out[rows], want, bound) <= 1.0
    # every row: the sums again in fp32, in which the products are exact and their sum off by k 2^-24 of their sizes
    full = (a.float() @ wt.float().t()) * sa[:, None] * sw + (bias.float() if extras else 0.0)
    full = torch.nn.functional.gelu(full) if act == "gelu" else torch.nn.functional.silu(full) if act == "silu" else full
    full = full + (res.float() if extras else 0.0)
    slack = k * 2.0 ** -24 * (127 * 127 * 0.02 * 0.02) * math.sqrt(k)
    assert torch.allclose(out.float(), full, rtol=2.0 ** -7, atol=0.02 + slack)


@pytest.mark.parametrize("dtype,m,n,k", [("bf16", 5, 256, 256), ("bf16", 700, 512, 256), ("bf16", 4200, 4096, 512), ("f32", 90, 128, 128)])
def test_linear_q8_residual_in_place(dtype, m, n, k):
    g = _gen(m)
    a, wt, sa, sw = _codes(g, m, k).cuda(), _codes(g, n, k).cuda(), torch.rand(m, generator=g).cuda() * 0.01, torch.rand(n, generator=g).cuda() * 0.01
    res = ou.rand(g, m, n, dtype=dtype).cuda()
    out = torch.empty_like(res)
    B.dare_k_linear_q8(a, sa, wt, sw, out, residual=res, act="silu")
    B.dare_k_linear_q8(a, sa, wt, sw, res, residual=res, act="silu")
    assert torch.equal(out, res)


@pytest.mark.parametrize("m", [3, 40, 300])
def test_linear_q8_largest_sums_and_scales_that_are_not_finite(m):
    """Every code -128 or 127 at the longest k; a NaN or infinite scale stays in its row or column."""
    k = (1 << 17) - 128
    a = torch.full((m, k), -128, dtype=torch.int8, device="cuda")
    a[1] = 127
    wt = torch.full((64, k), -128, dtype=torch.int8, device="cuda")
    wt[5] = 127
    sa, sw = torch.ones(m, device="cuda"), torch.ones(64, device="cuda")
    out = torch.empty(m, 64, device="cuda")
    B.dare_k_linear_q8(a, sa, wt, sw, out)
    assert out[0, 0] == 128 * 128 * k and out[0, 5] == -128 * 127 * k and out[1, 5] == float(torch.tensor(127 * 127 * k, dtype=torch.float32))
    sa[2], sw[7] = float("nan"), float("inf")
    a[0], wt[9] = 0, 0
    B.dare_k_linear_q8(a, sa, wt, sw, out)
    assert torch.isnan(out[2]).all() and torch.isnan(out[0, 7]) and torch.isinf(out[1, 7])
    keep = torch.ones(m, 64, dtype=torch.bool, device="cuda")
    keep[2], keep[:, 7] = False, False
    assert torch.isfinite(out[keep]).all() and (out[0][keep[0]] == 0).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("m", [3, 40, 1600])
def test_linear_q8_special_values_of_activations(dtype, m):
    """The identity far above 0, 0 far below, infinities of the bias (GELU of -infinity is 0, the others are NaN there), NaN in its column alone."""
    td = TYPES[dtype]
    n = 14144 if m > 1000 else 64
    a, wt = torch.zeros(m, 384, dtype=torch.int8, device="cuda"), torch.zeros(n, 384, dtype=torch.int8, device="cuda")
    one = lambda k: torch.ones(k, device="cuda")
    bias = torch.zeros(n, dtype=td, device="cuda")
    bias[:6] = torch.tensor([200.0, -200.0, 1e30, -1e30, math.inf, math.nan])
    bias[n - 1] = -math.inf
    for act in ("silu", "gelu", "gelu_tanh"):
        out = torch.empty(m, n, dtype=td, device="cuda")
        B.dare_k_linear_q8(a, one(m), wt, one(n), out, bias, act)
        assert (out[:, 0] == bias[0]).all() and (out[:, 2] == bias[2]).all() and (out[:, 4] == math.inf).all()
        assert (out[:, 1].abs() < 1e-30).all() and (out[:, 3].abs() < 1e-30).all() and torch.isnan(out[:, 5]).all()
        assert (out[:, n - 1] == 0).all() if act == "gelu" else torch.isnan(out[:, n - 1]).all()
        assert (out[:, 6:n - 1] == 0).all()


def test_linear_q8_scales_whose_product_is_no_normal_number():
    a, wt = torch.full((2, 128), 100, dtype=torch.int8, device="cuda"), torch.full((64, 128), 100, dtype=torch.int8, device="cuda")
    sa, sw = torch.full((2,), 1e-20, device="cuda"), torch.full((64,), 3e-20, device="cuda")
    out = torch.empty(2, 64, device="cuda")
    B.dare_k_linear_q8(a, sa, wt, sw, out)
    want = 128 * 1e4 * float(sa[0]) * float(sw[0])
    assert ((out.double() - want).abs() <= 2.0 ** -23 * want).all()


# ---- log-probabilities ----------------------------------------------------------------------------

def _outputs(rows, top):
    return (torch.full((rows,), 7.0, device="cuda"), torch.full((rows,), 7.0, device="cuda"),
            torch.full((rows, top), 77, dtype=torch.int32, device="cuda"), torch.full((rows, top), 7.0, device="cuda"))


def _check(x, tokens, scale, top, got):
    lp, b, h, bh, ids, tops, bt = su.logprobs64(x, tokens, scale, top)
    assert torch.equal(got[2].cpu().long(), ids)
    for mine, want, bound in ((got[0], lp, b), (got[1], h, bh), (got[3], tops, bt)):
        mine = mine.cpu().double()
        want = torch.where(want < -torch.finfo(torch.float32).max, torch.full_like(want, -math.inf), want)   # (beyond fp32)
        assert torch.equal(mine == -math.inf, want == -math.inf) and not torch.isnan(mine).any()
        fin = want > -math.inf
        assert ((mine - want).abs()[fin] <= bound[fin]).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("vocab,top", [(1, 1), (2, 2), (7, 3), (63, 32), (100, 5), (1000, 32), (2047, 17), (2055, 32), (2063, 1), (4097, 32), (16383, 8),
                                       (16384, 32), (16391, 2), (32003, 20), (126464, 32), (300001, 4)])
@pytest.mark.parametrize("pad,scale,spread,banned", [(0, 1.0, 2.0, 0), (1, 0.7, 6.0, 3), (8, 30.0, 1.0, 0.9), (3, 1.0, 0.0, 0.2)])
def test_logprobs(dtype, vocab, top, pad, scale, spread, banned):
    g = _gen(vocab + pad)
    rows = 3
    x = (torch.randn(rows, vocab, generator=g) * spread).to(TYPES[dtype])
    n = int(banned * vocab) if banned < 1 else min(banned, vocab - 1)
    if n:
        x[:, torch.randperm(vocab, generator=g)[:n]] = -math.inf
    tokens = torch.randint(0, vocab, (rows,), generator=g, dtype=torch.int32)
    tokens[0] = int(x[0].float().argmax())
    got = _outputs(rows, top)
    B.dare_k_logprobs(_padded(x, pad, float("inf")), tokens.cuda(), *got, scale=scale)
    _check(x, tokens, scale, top, got)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("vocab", [5, 1000, 40000])
def test_logprobs_special_rows(dtype, vocab):
    g = _gen(vocab)
    lowest = float(torch.finfo(TYPES[dtype]).min)
    x = torch.randn(10, vocab, generator=g).to(TYPES[dtype])
    x[0] = -math.inf                                  # nothing left
    x[1], x[1, vocab - 2] = -math.inf, 3.0            # one alternative
    x[2] = lowest                                     # the lowest value is a value
    x[3], x[3, 1] = lowest, 0.0
    x[4, 3] = math.nan
    x[5, vocab - 1] = math.inf
    x[6], x[6, 2] = 0.0, -0.0                         # the zeros are equal
    x[6, 4] = -1.0
    x[7], x[7, 0] = lowest, -lowest                   # differences beyond the type
    x[8] = -math.inf
    x[8, 4] = lowest
    top = 4
    tokens = torch.tensor([0, vocab - 2, 1, 1, 0, vocab - 1, 2, 1, 4, vocab], dtype=torch.int32)
    got = _outputs(10, top)
    B.dare_k_logprobs(x.cuda(), tokens.cuda(), *got)
    for r in (4, 5):
        assert torch.isnan(got[0][r]) and torch.isnan(got[1][r]) and (got[2][r] == -1).all() and torch.isnan(got[3][r]).all()
    keep = [0, 1, 2, 3, 6, 7, 8, 9]
    _check(x[keep], tokens[keep], 1.0, top, [t[torch.tensor(keep).cuda()] for t in got])
    tokens[:] = -1
    B.dare_k_logprobs(x.cuda(), tokens.cuda(), got[0])
    assert (got[0][torch.tensor(keep).cuda()] == -math.inf).all() and torch.isnan(got[0][4:6]).all()


@pytest.mark.parametrize("dtype,vocab,lanes", [("bf16", 1000, 64), ("f32", 1000, 64), ("bf16", 12000, 256), ("f32", 15001, 256), ("bf16", 126464, 1024), ("f32", 126464, 1024)])
@pytest.mark.parametrize("top", [1, 7, 32])
def test_logprobs_largest_logits_in_few_places(dtype, vocab, lanes, top):
    """The largest logits lie in chunks that a few lanes of a workgroup read, in equal and in different values, and more of them than a list of them holds."""
    g = _gen(vocab)
    per = 8 if dtype == "bf16" else 4
    at = torch.arange(vocab) // per % lanes
    x = torch.randn(4, vocab, generator=g).to(TYPES[dtype])
    x[0, at < lanes // 4] = 30.0
    x[1, at < lanes // 6] += 20.0
    x[2] = torch.arange(vocab) / 1000.0
    few = at < (28 if lanes == 64 else 6 * 64)
    x[3], x[3, few] = -math.inf, (torch.randn(int(few.sum()), generator=g) * 4).to(TYPES[dtype])
    tokens = torch.zeros(4, dtype=torch.int32)
    got = _outputs(4, top)
    B.dare_k_logprobs(x.cuda(), tokens.cuda(), *got)
    _check(x, tokens, 1.0, top, got)


def test_logprobs_parts_that_are_left_out_and_no_rows():
    x = torch.randn(5, 777, generator=_gen(2)).cuda()
    tokens = torch.arange(5, dtype=torch.int32, device="cuda")
    full, part = _outputs(5, 3), _outputs(5, 3)
    B.dare_k_logprobs(x, tokens, *full)
    B.dare_k_logprobs(x, tokens, part[0])
    B.dare_k_logprobs(x, entropy=part[1])
    B.dare_k_logprobs(x, top_ids=part[2], top_logprobs=part[3])
    assert all(torch.equal(a, b) for a, b in zip(full, part))
    B.dare_k_logprobs(x)
    B.dare_k_logprobs(x, tokens, part[0], part[1], part[2][:, :0].contiguous(), part[3][:, :0].contiguous())
    assert torch.equal(full[0], part[0]) and torch.equal(full[1], part[1])
    with pytest.raises(ValueError):
        B.dare_k_logprobs(x, top_ids=part[2][:, :2], top_logprobs=part[3][:, :2])
    B.dare_k_logprobs(x[:0], tokens[:0], part[0][:0], part[1][:0], part[2][:0], part[3][:0])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,vocab,pad", [(1, 126464, 0), (1, 126465, 3), (2, 33001, 1), (7, 65536, 0), (16, 131072, 0), (17, 90001, 1), (64, 70000, 8), (65, 70000, 0)])
@pytest.mark.parametrize("top", [0, 1, 8, 32])
def test_logprobs_of_few_rows_with_a_workspace(dtype, rows, vocab, pad, top):
    """A row's result does not depend on what is in the workspace, nor, but for roundings, on the parts it is cut into."""
    g = _gen(rows + vocab)
    x = (torch.randn(rows, vocab, generator=g) * 3).to(TYPES[dtype])
    x[0, :vocab // 2] = -math.inf
    x[0, vocab - 9000:] = -math.inf
    x[rows - 1, 100:5000] = 12.0
    tokens = torch.randint(0, vocab, (rows,), generator=g, dtype=torch.int32)
    got = _outputs(rows, top)
    code = B.DARE_BF16 if dtype == "bf16" else B.DARE_F32
    need = B.dare_k_logprobs_workspace(code, rows, vocab, top)
    ws = torch.full((need + 64,), 255, dtype=torch.uint8, device="cuda")
    B.dare_k_logprobs(_padded(x, pad, float("nan")), tokens.cuda(), *got, workspace=ws)
    _check(x, tokens, 1.0, top, got)
    assert (ws[need:] == 255).all()
    if top == 32:     # the same rows among many
        many = _outputs(300, top)
        big = torch.cat([x.cuda(), x[:1].cuda().expand(300 - rows, vocab)]) if 300 * vocab * x.element_size() < 1 << 28 else None
        if big is not None:
            B.dare_k_logprobs(big, tokens.repeat(300 // rows + 1)[:300].cuda(), *many)
            assert torch.equal(many[2][:rows], got[2]) and torch.allclose(many[3][:rows], got[3], rtol=0, atol=1e-4)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_logprobs_special_parts(dtype):
    """Parts without an element, with NaN or infinity, and with values at the ends of the type, beside ordinary ones."""
    vocab, top = 126464, 5
    lowest = float(torch.finfo(TYPES[dtype]).min)
    x = torch.randn(11, vocab, generator=_gen(8)).to(TYPES[dtype])
    x[0] = -math.inf
    x[1], x[1, 70000] = -math.inf, 2.0
    x[2, 126463] = math.nan
    x[3, 0] = math.inf
    x[4, :100000] = lowest
    x[5] = lowest
    x[6, 60000:] = -math.inf
    x[6, :8192] = -math.inf
    x[7, 9] = -lowest
    x[8], x[8, 50000] = lowest, -math.inf            # one value, but for a place
    x[9, 20000:], x[9, :10] = lowest, -lowest         # both ends
    x[10], x[10, 100000:100003] = -math.inf, lowest   # all of the probability on three of the lowest values
    tokens = torch.tensor([5, 70000, 1, 1, 3, 4, 9000, 9, 50000, 3, 100001], dtype=torch.int32)
    got = _outputs(11, top)
    B.dare_k_logprobs(x.cuda(), tokens.cuda(), *got)
    for r in (2, 3):
        assert torch.isnan(got[0][r]) and torch.isnan(got[1][r]) and (got[2][r] == -1).all() and torch.isnan(got[3][r]).all()
    keep = [0, 1, 4, 5, 6, 7, 8, 9, 10]
    _check(x[keep], tokens[keep], 1.0, top, [t[torch.tensor(keep).cuda()] for t in got])


def test_logprobs_many_rows_of_few_logits():
    for rows, vocab, top, dtype in ((70001, 33, 2, "bf16"), (1100, 1023, 32, "f32"), (1024, 4095, 32, "bf16"), (1030, 4001, 5, "f32")):
        x = torch.randn(rows, vocab, generator=_gen(4)).to(TYPES[dtype])
        x[3], x[4, 50:], x[5, ::3], x[6] = 1.5, -math.inf, 4.0, -math.inf      # equal ones, few, more than a list holds, none
        x[7, torch.arange(vocab) // (8 if dtype == "bf16" else 4) % 64 < 20] += 30.0
        tokens = torch.randint(0, vocab, (rows,), generator=_gen(5), dtype=torch.int32)
        got = _outputs(rows, top)
        B.dare_k_logprobs(x.cuda(), tokens.cuda(), *got)
        _check(x, tokens, 1.0, top, got)


# ---- the end of a step ------------------------------------------------------------------------------

class _End:
    """Residual sum, final norm, output embedding in 8 bits, and what the logits say about every row."""

    def __init__(self, rows, d, vocab, top, seed):
        g = _gen(seed)
        w = (torch.randn(d, vocab, generator=g) * 2 / math.sqrt(d)).bfloat16().cuda()
        self.gain = (1 + 0.1 * torch.randn(d, generator=g)).bfloat16().cuda()
        self.x, self.o = torch.randn(rows, d, generator=g).bfloat16().cuda(), torch.randn(rows, d, generator=g).bfloat16().cuda()
        self.tokens = torch.randint(0, vocab, (rows,), generator=g, dtype=torch.int32).cuda()
        packed = B.dare_k_pack_weight(w)
        self.w, self.sw = torch.empty(vocab, d, dtype=torch.int8, device="cuda"), torch.empty(vocab, device="cuda")
        B.dare_k_norm_q8(None, packed, self.w, self.sw)
        self.codes, self.scales = torch.empty(rows, d, dtype=torch.int8, device="cuda"), torch.empty(rows, device="cuda")
        self.logits = torch.empty(rows, vocab, dtype=torch.bfloat16, device="cuda")
        self.s, self.top, self.out = torch.empty_like(self.x), top, _outputs(rows, top)

    def run(self, stream=None):
        B.dare_k_norm_q8("rms", self.x, self.codes, self.scales, self.o, self.s, self.gain, stream=stream)
        B.dare_k_linear_q8(self.codes, self.scales, self.w, self.sw, self.logits, stream=stream)
        B.dare_k_logprobs(self.logits, self.tokens, *self.out, stream=stream)

    def check(self):
        s, y = su.norm64("rms", self.x.cpu(), self.o.cpu(), self.gain.cpu(), None, 1e-5)
        assert torch.equal(self.s.cpu(), s)
        su.check_codes(y, self.codes, self.scales)
        want, bound = su.linear_q8_64(self.codes.cpu(), self.scales.cpu(), self.w.cpu(), self.sw.cpu(), None, None, None, torch.bfloat16)
        assert ou.worst(self.logits, want, bound) <= 1.0
        _check(self.logits.cpu(), self.tokens.cpu(), 1.0, self.top, self.out)
        return y


def test_end_of_a_step():
    end = _End(37, 512, 4160, 4, 11)
    end.run()
    y = end.check()
    # codes of both sides are off by half a step each: the logits by that of a row's and a column's scale over sqrt(d) random terms, 6 sigma
    w = end.w.cpu().double() * end.sw.cpu().double()[:, None]
    exact = y @ w.t()
    sigma = end.scales.cpu().double()[:, None] / math.sqrt(12) * w.norm(dim=1)
    assert ((end.logits.cpu().double() - exact).abs() <= 6 * sigma + 2.0 ** -8 * exact.abs()).all()


def test_end_of_a_step_on_another_stream_and_captured():
    end = _End(9, 384, 1088, 3, 12)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    end.run(side)
    side.synchronize()
    end.check()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        end.run()
    g = _gen(13)
    for _ in range(4):
        end.x.copy_(torch.randn(end.x.shape, generator=g))
        end.tokens.copy_(torch.randint(0, 1088, (9,), generator=g))
        graph.replay()
        torch.cuda.synchronize()
        end.check()
        captured = [t.clone() for t in end.out]
        end.run()
        assert all(torch.equal(a, b) for a, b in zip(captured, end.out))


def test_logprobs_of_few_rows_captured():
    """A captured call with a workspace of its own, and two graphs that share one, replayed in turn with other logits."""
    rows, vocab, top = 2, 70001, 4
    g = _gen(21)
    x = torch.randn(rows, vocab, generator=g).bfloat16().cuda()
    tokens = torch.randint(0, vocab, (rows,), generator=g, dtype=torch.int32).cuda()
    need = B.dare_k_logprobs_workspace(B.DARE_BF16, rows, vocab, top)
    assert need > 0
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    outs, graphs = [_outputs(rows, top) for _ in range(3)], []
    B.dare_k_logprobs(x, tokens, *outs[0])
    torch.cuda.synchronize()
    for out, w in zip(outs, (None, ws, ws)):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            B.dare_k_logprobs(x, tokens, *out, workspace=w)
    for _ in range(4):
        x.copy_(torch.randn(rows, vocab, generator=g))
        for graph in graphs:
            graph.replay()
        torch.cuda.synchronize()
        eager = _outputs(rows, top)
        B.dare_k_logprobs(x, tokens, *eager)
        _check(x.cpu(), tokens.cpu(), 1.0, top, eager)
        for out in outs:
            assert all(torch.equal(a, b) for a, b in zip(out, eager))


def test_logprobs_on_two_streams_at_once():
    rows, vocab, top = 3, 90000, 5
    g = _gen(22)
    sets = []
    for i in range(2):
        x = torch.randn(rows, vocab, generator=g).bfloat16()
        tokens = torch.randint(0, vocab, (rows,), generator=g, dtype=torch.int32)
        sets.append((x, tokens, x.cuda(), tokens.cuda(), _outputs(rows, top), torch.cuda.Stream()))
    torch.cuda.synchronize()
    for _ in range(20):
        for x, tokens, xd, td, out, stream in sets:
            B.dare_k_logprobs(xd, td, *out, stream=stream)
    torch.cuda.synchronize()
    for x, tokens, xd, td, out, stream in sets:
        _check(x, tokens, 1.0, top, out)


def test_codes_through_a_layer_with_shared_key_heads():
    """Q, K and V from codes, attention of packed sequences, its output as codes into the output projection, onto the residual stream."""
    g, rows, h, kv, d = _gen(20), 41, 4, 2, 64
    hidden = h * d
    rn = lambda *s: torch.randn(s, generator=g).bfloat16().cuda()
    x, gain, bias = rn(rows, hidden), rn(hidden).mul_(0.1).add_(1), rn((h + 2 * kv) * d)

    def quantised(w):
        codes, scales = torch.empty(w.shape, dtype=torch.int8, device="cuda"), torch.empty(w.shape[0], device="cuda")
        B.dare_k_norm_q8(None, w, codes, scales)
        return codes, scales

    wqkv, wo = quantised(rn((h + 2 * kv) * d, hidden).mul_(hidden ** -0.5)), quantised(rn(hidden, hidden).mul_(hidden ** -0.5))
    codes, scales = torch.empty(rows, hidden, dtype=torch.int8, device="cuda"), torch.empty(rows, device="cuda")
    qkv, attn, out = torch.empty(rows, h + 2 * kv, d, dtype=torch.bfloat16, device="cuda"), torch.empty(rows, h, d, dtype=torch.bfloat16, device="cuda"), torch.empty_like(x)
    ints = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")
    B.dare_k_norm_q8("rms", x, codes, scales, gain=gain)
    B.dare_k_linear_q8(codes, scales, *wqkv, qkv.view(rows, -1), bias=bias)
    B.dare_k_attention_packed(qkv[:, :h], qkv[:, h:h + kv], qkv[:, h + kv:], attn, ints([0, 30, 41]), ints([0, 30]), ints([30, 41]), 30, 30, causal_block=1)
    c1 = (codes.clone(), scales.clone())
    B.dare_k_norm_q8(None, attn.view(rows, -1), codes, scales)
    B.dare_k_linear_q8(codes, scales, *wo, out, residual=x)
    _, y = su.norm64("rms", x.cpu(), None, gain.cpu(), None, 1e-5)
    su.check_codes(y, *c1)
    want, bound = su.linear_q8_64(c1[0].cpu(), c1[1].cpu(), wqkv[0].cpu(), wqkv[1].cpu(), bias.cpu(), None, None, torch.bfloat16)
    assert ou.worst(qkv.view(rows, -1), want, bound) <= 1.0
    q = qkv.cpu()
    want, bound, _ = ou.attention64(q[:, :h], q[:, h:h + kv], q[:, h + kv:], [0, 30, 41], [0, 30], [30, 41], 1, d ** -0.5)
    assert ou.worst(attn, want, bound) <= 1.0
    su.check_codes(attn.cpu().view(rows, -1).double(), codes, scales)
    want, bound = su.linear_q8_64(codes.cpu(), scales.cpu(), wo[0].cpu(), wo[1].cpu(), None, None, x.cpu(), torch.bfloat16)
    assert ou.worst(out, want, bound) <= 1.0
