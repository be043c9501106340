"""dare_k_linear, dare_k_rope and dare_k_attention_packed against their plain 64-bit forms, and as a layer together."""
import math

import pytest
import torch

from paper_2605_08134_amd import binding as B
import operator_util as ou

pytestmark = pytest.mark.gpu


def _gen(seed):
    return torch.Generator().manual_seed(seed)


def _padded(t, pad, fill=float("nan")):
    """t on the GPU as a view of a buffer with `pad` elements of something else behind every row."""
    buf = torch.full((t.shape[0], t[0].numel() + pad), fill, dtype=t.dtype, device="cuda")
    buf[:, :t[0].numel()] = t.reshape(t.shape[0], -1).cuda()
    return buf[:, :t[0].numel()].unflatten(1, t.shape[1:])


# ---- projection with epilogue ---------------------------------------------------------------

@pytest.mark.parametrize("act", [None, "silu", "gelu", "gelu_tanh"])
@pytest.mark.parametrize("dtype,m,n,k", [
    ("bf16", 1, 64, 64), ("bf16", 16, 128, 512), ("bf16", 17, 192, 320), ("bf16", 33, 8192, 64), ("bf16", 2, 8256, 128),
    ("bf16", 200, 320, 192), ("bf16", 257, 1088, 448), ("f32", 1, 64, 64), ("f32", 37, 192, 128), ("f32", 130, 576, 320),
])
@pytest.mark.parametrize("extras", ["none", "bias", "residual", "both"])
def test_linear(act, dtype, m, n, k, extras):
    g = _gen(m * 31 + n)
    a, wt = ou.rand(g, m, k, dtype=dtype), ou.rand(g, n, k, dtype=dtype, std=2.0 / math.sqrt(k))
    bias = ou.rand(g, n, dtype=dtype) if extras in ("bias", "both") else None
    res = ou.rand(g, m, n, dtype=dtype) if extras in ("residual", "both") else None
    want, bound = ou.linear64(a, wt, bias, act, res)
    out = _padded(torch.zeros(m, n, dtype=a.dtype), 8)
    B.dare_k_linear(_padded(a, 64), wt.cuda(), out, None if bias is None else bias.cuda(), act,
                    None if res is None else _padded(res, 16))
    assert ou.worst(out, want, bound) <= 1.0


# many rows, ragged in rows and columns (every tile shape: test_gpu_operators_bounds.py)
@pytest.mark.parametrize("m,n,k", [(515, 1600, 128), (777, 6144, 128), (1000, 2112, 192), (1100, 4096, 64), (1281, 8256, 256),
                                   (2047, 3136, 128), (2049, 4160, 448), (4100, 4416, 128), (9000, 1216, 64)])
@pytest.mark.parametrize("act,extras", [(None, False), ("gelu", True)])
def test_linear_many_rows(m, n, k, act, extras):
    g = torch.Generator(device="cuda").manual_seed(m)
    rn = lambda *s: torch.randn(s, device="cuda", generator=g).bfloat16()
    a, wt = rn(m, k), rn(n, k)
    bias, res = (rn(n), rn(m, n)) if extras else (None, None)
    out = torch.empty(m, n, dtype=torch.bfloat16, device="cuda")
    B.dare_k_linear(a, wt, out, bias, act, res)
    rows = torch.cat([torch.arange(0, m, 97), torch.tensor([m - 1])])
    dev = lambda t, r=None: None if t is None else (t if r is None else t[r.cuda()]).cpu()
    want, bound = ou.linear64(dev(a, rows), wt.cpu(), dev(bias), act, dev(res, rows))
    assert ou.worst(out[rows.cuda()], want, bound) <= 1.0
    full = a.float() @ wt.float().t() + (bias.float() if extras else 0.0)   # every row, roughly: none is left out
    full = torch.nn.functional.gelu(full) if act else full
    assert torch.allclose(out.float(), full + (res.float() if extras else 0.0), rtol=2.0 ** -7, atol=0.05)


@pytest.mark.parametrize("dtype,m,n,k", [("bf16", 5, 256, 128), ("bf16", 700, 512, 128), ("bf16", 4200, 4096, 256), ("f32", 90, 128, 64)])
def test_linear_residual_in_place(dtype, m, n, k):
    g = _gen(m)
    a, wt, res = ou.rand(g, m, k, dtype=dtype).cuda(), ou.rand(g, n, k, dtype=dtype).cuda(), ou.rand(g, m, n, dtype=dtype).cuda()
    out = torch.empty_like(res)
    B.dare_k_linear(a, wt, out, residual=res, act="silu")
    B.dare_k_linear(a, wt, res, residual=res, act="silu")
    assert torch.equal(out, res)


def test_linear_of_no_rows_and_special_values():
    w = torch.eye(64, dtype=torch.bfloat16, device="cuda")
    B.dare_k_linear(torch.empty(0, 64, dtype=torch.bfloat16, device="cuda"), w, torch.empty(0, 64, dtype=torch.bfloat16, device="cuda"))
    for dtype in (torch.bfloat16, torch.float32):
        x = torch.zeros(8, 64, dtype=dtype, device="cuda")
        x[0, 0], x[1, 0], x[2, 0], x[3, 0] = 200.0, -200.0, 1e30, -1e30
        x[4, 0] = float("nan")
        for act in ("silu", "gelu", "gelu_tanh"):
            out = torch.empty_like(x)
            B.dare_k_linear(x, w.to(dtype), out, act=act)
            assert out[0, 0] == x[0, 0] and out[2, 0] == x[2, 0]     # the identity far above 0, 0 far below
            assert abs(float(out[1, 0])) < 1e-30 and abs(float(out[3, 0])) < 1e-30
            assert torch.isnan(out[4, 0]) and not torch.isnan(out[5]).any()
            y = x.clone()
            y[4, 0], y[:4, 0] = float("inf"), 0.0
            B.dare_k_linear(y, torch.ones(64, 64, dtype=dtype, device="cuda"), out, act=act)
            assert (out[4] == float("inf")).all()


# ---- rotary embedding -------------------------------------------------------------------------

@pytest.mark.parametrize("layout", ["half", "pairs"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,h,kv,d,rot,pad", [
    (1, 1, 1, 8, 2, 0), (3, 5, 1, 64, 64, 0), (7, 8, 2, 128, 128, 8), (65, 4, 4, 64, 32, 0), (130, 3, 1, 256, 256, 0),
    (9, 2, 2, 128, 34, 0), (5, 3, 1, 40, 14, 0), (6, 7, 1, 128, 96, 3), (300, 28, 4, 128, 64, 0),
])
@pytest.mark.parametrize("magnitude", [1.0, 1.3])
def test_rope(layout, dtype, n, h, kv, d, rot, pad, magnitude):
    g = _gen(n * d + rot)
    q, k, v = ou.rand(g, n, h, d, dtype=dtype), ou.rand(g, n, kv, d, dtype=dtype), ou.rand(g, n, kv, d, dtype=dtype)
    pos = torch.randint(0, 1 << 20, (n,), generator=g, dtype=torch.int32)
    pos[0] = 2 ** 31 - 1 if n > 2 else 0
    freqs = torch.tensor([10000.0 ** (-2.0 * i / rot) for i in range(rot // 2)], dtype=torch.float64)
    room = 2 * n + 3
    rows = torch.randperm(room, generator=g)[:n].to(torch.int32)
    cache = ou.rand(g, room, kv, d, dtype=dtype)
    qd, kd, vd = _padded(q, pad), _padded(k, pad), _padded(v, pad)
    qo, ko, vo = _padded(torch.zeros_like(q), 0), _padded(cache, pad), _padded(cache, 2 * pad)
    B.dare_k_rope(pos.cuda(), freqs.cuda(), layout, qd, qo, kd, ko, vd, vo, rows=rows.cuda(), magnitude=magnitude)
    wq, bq = ou.rope64(q, pos, freqs, rot, layout, magnitude)
    wk, bk = ou.rope64(k, pos, freqs, rot, layout, magnitude)
    assert ou.worst(qo, wq, bq) <= 1.0
    assert ou.worst(ko.cpu()[rows.long()], wk, bk) <= 1.0
    assert torch.equal(qo.cpu()[..., rot:], q[..., rot:])
    rest = torch.ones(room, dtype=torch.bool)
    rest[rows.long()] = False
    assert torch.equal(vo.cpu()[rows.long()], v) and torch.equal(vo.cpu()[rest], cache[rest])
    assert torch.equal(ko.cpu()[rest], cache[rest])
    # in place gives the same bits
    B.dare_k_rope(pos.cuda(), freqs.cuda(), layout, qd, qd, kd, kd, magnitude=magnitude)
    assert torch.equal(qd, qo) and torch.equal(kd.cpu(), ko.cpu()[rows.long()])


def test_rope_rows_that_go_nowhere_and_parts_that_are_left_out():
    g = _gen(3)
    k, v = ou.rand(g, 6, 2, 64, dtype="bf16").cuda(), ou.rand(g, 6, 2, 64, dtype="bf16").cuda()
    q = ou.rand(g, 6, 4, 64, dtype="bf16").cuda()
    pos = torch.arange(6, dtype=torch.int32, device="cuda")
    freqs = B.dare_k_rope_freqs(64)
    rows = torch.tensor([3, -1, 9, 10, 0, -2 ** 31], dtype=torch.int32, device="cuda")
    ko, vo, qo = (torch.full((10, 2, 64), 7.0, dtype=torch.bfloat16, device="cuda") for _ in range(2)), None, torch.empty_like(q)
    ko, vo = ko
    B.dare_k_rope(pos, freqs, "half", q, qo, k, ko, v, vo, rows=rows)
    assert torch.equal(vo[3], v[0]) and torch.equal(vo[9], v[2]) and torch.equal(vo[0], v[4])
    for r in (1, 2, 4, 5, 6, 7, 8):
        assert (ko[r] == 7).all() and (vo[r] == 7).all()
    k2 = torch.empty_like(k)
    B.dare_k_rope(pos, freqs, "half", k=k, k_out=k2)          # keys alone
    assert torch.equal(k2[0], ko[3]) and torch.equal(k2[2], ko[9])
    q2 = torch.empty_like(q)
    B.dare_k_rope(pos, freqs, "half", q, q2)                  # queries alone
    assert torch.equal(q2, qo)
    v2 = torch.empty_like(v)
    B.dare_k_rope(pos, freqs, "half", v=v, v_out=v2)          # a copy
    assert torch.equal(v2, v)
    e = torch.empty(0, 4, 64, dtype=torch.bfloat16, device="cuda")
    B.dare_k_rope(pos[:0], freqs, "half", e, e)


def test_rope_leaves_infinities_of_other_channels_alone():
    """A channel that is not rotated keeps its value, whatever its neighbours in the same 16 bytes do."""
    x = torch.randn(2, 1, 64, device="cuda")
    x[0, 0, 20:] = float("inf")
    x[1, 0, 33] = float("nan")
    pos, freqs = torch.tensor([5, 9], dtype=torch.int32, device="cuda"), B.dare_k_rope_freqs(18)
    for layout in ("half", "pairs"):
        out = torch.empty_like(x)
        B.dare_k_rope(pos, freqs, layout, x, out)
        assert torch.isfinite(out[..., :18]).all()
        assert torch.equal(out[0, 0, 18:], x[0, 0, 18:]) and torch.isnan(out[1, 0, 33])
        assert torch.equal(out[1, 0, 34:], x[1, 0, 34:])


def test_rope_negative_positions_turn_back():
    x = torch.randn(5, 3, 128, device="cuda")
    pos, freqs = torch.tensor([0, 1, 77, 5000, 131071], dtype=torch.int32, device="cuda"), B.dare_k_rope_freqs(128, 500000.0)
    there, back = torch.empty_like(x), torch.empty_like(x)
    for layout in ("half", "pairs"):
        B.dare_k_rope(pos, freqs, layout, x, there)
        B.dare_k_rope(-pos, freqs, layout, there, back)
        assert torch.allclose(back, x, rtol=0, atol=20 * 2.0 ** -24 * float(x.abs().max()))


@pytest.mark.parametrize("scaling", [None, "linear", "base", "turns"])
@pytest.mark.parametrize("rot", [4, 64, 128])
def test_rope_freqs(scaling, rot):
    got = B.dare_k_rope_freqs(rot, 500000.0, scaling, 8.0, 8192, 1.0, 4.0).cpu()
    base = 500000.0 * (8.0 ** (rot / (rot - 2)) if scaling == "base" else 1.0)
    want = []
    for i in range(rot // 2):
        f = base ** (-2.0 * i / rot)
        if scaling == "linear":
            f /= 8.0
        if scaling == "turns":
            mix = min(1.0, max(0.0, (8192 * f / (2 * math.pi) - 1.0) / 3.0))
            f *= mix + (1 - mix) / 8.0
        want.append(f)
    assert torch.allclose(got, torch.tensor(want, dtype=torch.float64), rtol=1e-14, atol=0)
    if scaling == "base":      # fastest pair as it was, slowest divided by the factor
        assert got[0] == 1.0 and abs(float(got[-1]) * 8.0 / 500000.0 ** (-(rot - 2.0) / rot) - 1) < 1e-12


# ---- attention of packed sequences ----------------------------------------------------------------

def _ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def _offsets(lens):
    off = [0]
    for n in lens:
        off.append(off[-1] + n)
    return off


def _run_attention(q, k, v, off, begin, end, block, scale=None, out=None, max_q=None, max_k=None, **kw):
    out = torch.full(q.shape, 7.0, dtype=q.dtype, device="cuda") if out is None else out
    lq = [b - a for a, b in zip(off, off[1:])] or [0]
    lk = [b - a for a, b in zip(begin, end)] or [0]
    B.dare_k_attention_packed(q, k, v, out, _ints(off), _ints(begin), _ints(end), max(lq) if max_q is None else max_q,
                              max(lk) if max_k is None else max_k, causal_block=block, scale=scale, **kw)
    return out


def _check_attention(q, k, v, off, begin, end, block, scale=None, **kw):
    want, bound, covered = ou.attention64(q, k, v, off, begin, end, block, scale or q.shape[2] ** -0.5)
    out = _run_attention(q.cuda(), k.cuda(), v.cuda(), off, begin, end, block, scale, **kw)
    assert ou.worst(out[covered.cuda()], want[covered], bound[covered]) <= 1.0
    assert (out[~covered.cuda()] == 7.0).all()
    return out


LENGTHS = {
    "one": ([1], [1]),
    "single tokens": ([1, 1, 1, 1, 1], [1, 31, 33, 64, 300]),
    "idle": ([0, 1, 0, 2, 0], [5, 40, 0, 129, 0]),
    "ragged": ([3, 130, 1, 65, 17], [3, 130, 1, 65, 17]),
    "behind a cache": ([32, 7, 1, 40], [96, 200, 256, 41]),
    "more queries than keys": ([9, 40, 70, 3], [4, 0, 33, 2]),
}


@pytest.mark.parametrize("lengths", list(LENGTHS))
@pytest.mark.parametrize("block", [0, 1, 5, 32])
@pytest.mark.parametrize("dtype,h,kv,d", [("bf16", 8, 2, 128), ("bf16", 7, 1, 64), ("bf16", 2, 2, 64), ("bf16", 3, 3, 128),
                                          ("f32", 6, 2, 64), ("f32", 2, 1, 128)])
def test_attention(lengths, block, dtype, h, kv, d):
    lq, lk = LENGTHS[lengths]
    g = _gen(len(lengths) * 100 + d + h)
    off, kb = _offsets(lq), _offsets(lk)
    n, rows = off[-1] + 3, kb[-1] + 2
    q, k, v = ou.rand(g, n, h, d, dtype=dtype, std=2.0), ou.rand(g, rows, kv, d, dtype=dtype), ou.rand(g, rows, kv, d, dtype=dtype)
    _check_attention(q, k, v, off, kb[:-1], kb[1:], block)


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("bf16", 64), ("f32", 64)])
@pytest.mark.parametrize("lens", [[1, 2, 127, 128, 129], [511, 64, 700], [256, 1, 320, 33]])
@pytest.mark.parametrize("block,h,kv,pad", [(0, 4, 2, 0), (1, 4, 2, 24), (32, 4, 2, 0), (1, 7, 1, 8), (1, 2, 2, 40)])
def test_attention_of_prompts(dtype, d, lens, block, h, kv, pad):
    """Longer prompts, queries, keys and values parts of one buffer, whose rows may end in something else."""
    g = _gen(sum(lens) + d)
    off = _offsets(lens)
    qkv = ou.rand(g, off[-1], h + 2 * kv, d, dtype=dtype)
    q, k, v = qkv[:, :h], qkv[:, h:h + kv], qkv[:, h + kv:]
    want, bound, _ = ou.attention64(q, k, v, off, off[:-1], off[1:], block, d ** -0.5)
    dev = _padded(qkv, pad)
    out = _run_attention(dev[:, :h], dev[:, h:h + kv], dev[:, h + kv:], off, off[:-1], off[1:], block)
    assert ou.worst(out, want, bound) <= 1.0


@pytest.mark.parametrize("h,kv,d,lq,lk", [(8, 1, 128, 1, 5000), (4, 1, 64, 3, 9001), (16, 4, 128, 16, 2500), (8, 2, 128, 32, 4100),
                                            (8, 2, 64, 7, 3000), (14, 2, 128, 4, 2600), (6, 2, 64, 50, 2300)])
@pytest.mark.parametrize("block", [0, 1])
def test_attention_over_a_long_cache(h, kv, d, lq, lk, block):
    """Keys of a row cut over workgroups."""
    g = _gen(lk)
    lens = [lk, lk // 3, 17, lk - 1]
    off, kb = _offsets([lq] * 4), _offsets(lens)
    q, k, v = ou.rand(g, off[-1], h, d, dtype="bf16", std=2.0), ou.rand(g, kb[-1], kv, d, dtype="bf16"), ou.rand(g, kb[-1], kv, d, dtype="bf16")
    assert B.dare_k_attention_packed_workspace(B.DARE_BF16, 4, off[-1], lq, lk, h, kv, d) > 0
    out = _check_attention(q, k, v, off, kb[:-1], kb[1:], block)
    # shorter hints only cut it in another way
    want, bound, _ = ou.attention64(q, k, v, off, kb[:-1], kb[1:], block, d ** -0.5)
    again = _run_attention(q.cuda(), k.cuda(), v.cuda(), off, kb[:-1], kb[1:], block, max_q=0, max_k=lk // 2)
    assert ou.worst(again, want, bound) <= 1.0
    same = _run_attention(q.cuda(), k.cuda(), v.cuda(), off, kb[:-1], kb[1:], block)
    assert torch.equal(out, same)


@pytest.mark.parametrize("batch", [63, 64, 65, 200, 4097, 5000])
def test_attention_of_many_sequences(batch):
    """The search for a block's sequence in one, two and three rounds; empty sequences anywhere."""
    g = _gen(batch)
    lq = torch.randint(0, 4, (batch,), generator=g).tolist()
    lq[0], lq[-1] = 0, 2
    lk = [n + int(x) for n, x in zip(lq, torch.randint(0, 9, (batch,), generator=g))]
    off, kb = _offsets(lq), _offsets(lk)
    for h, kv, d, dtype in ((4, 2, 64, "bf16"), (2, 2, 64, "f32")):
        q, k, v = ou.rand(g, off[-1], h, d, dtype=dtype), ou.rand(g, kb[-1], kv, d, dtype=dtype), ou.rand(g, kb[-1], kv, d, dtype=dtype)
        _check_attention(q, k, v, off, kb[:-1], kb[1:], 1)


@pytest.mark.parametrize("batch", [70, 300])
@pytest.mark.parametrize("h,kv,d,q_most,k_most", [(4, 1, 64, 1, 3000), (4, 1, 128, 40, 1500), (2, 2, 64, 90, 90)])
def test_attention_of_many_sequences_of_many_lengths(batch, h, kv, d, q_most, k_most):
    """More than 64, and more than 256, sequences, a few of them long: keys cut with both ways of finding a block."""
    g = _gen(batch + q_most)
    lq = torch.randint(0, 3, (batch,), generator=g).clamp(max=q_most).tolist()
    lk = [n + int(x) for n, x in zip(lq, torch.randint(0, 9, (batch,), generator=g))]
    for i in (1, batch // 2, batch - 1):
        lq[i], lk[i] = q_most, k_most
    off, kb = _offsets(lq), _offsets(lk)
    q, k, v = ou.rand(g, off[-1], h, d, dtype="bf16"), ou.rand(g, kb[-1], kv, d, dtype="bf16"), ou.rand(g, kb[-1], kv, d, dtype="bf16")
    cut = B.dare_k_attention_packed_workspace(B.DARE_BF16, batch, off[-1], q_most, k_most, h, kv, d) > 0
    assert cut == (k_most > 1000)
    for block in (0, 1):
        _check_attention(q, k, v, off, kb[:-1], kb[1:], block)


@pytest.mark.parametrize("q_off,most", [([0, 6, 2, 8, 3], 1), ([0, 8, 0, 8, 0], 6), ([5, 3, 1, 0, 0], 1), ([0, 2 ** 31 - 1, -5, 9, 4], 40)])
@pytest.mark.parametrize("batch", [4, 80])
def test_attention_with_offsets_that_do_not_ascend_stays_inside(q_off, most, batch):
    """Whatever they lead to, rows that no sequence can have are left alone, and the call ends."""
    g = _gen(most)
    q_off = q_off + [q_off[-1]] * (batch - 4)
    for h, kv, d, dtype in ((4, 1, 64, "bf16"), (4, 1, 128, "bf16"), (2, 1, 64, "f32")):
        q, k, v = (ou.rand(g, n, x, d, dtype=dtype).cuda() for n, x in ((8, h), (1500, kv), (1500, kv)))
        buf = torch.full((24, h, d), 7.0, dtype=q.dtype, device="cuda")
        _run_attention(q, k, v, q_off, [0, 700, 3, 9] * (batch // 4), [1500, 1400, 1100, 1200] * (batch // 4), 1, out=buf[8:16],
                       max_q=most, max_k=1500)
        torch.cuda.synchronize()
        assert (buf[:8] == 7).all() and (buf[16:] == 7).all() and torch.isfinite(buf).all()


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("bf16", 64), ("f32", 64)])
@pytest.mark.parametrize("lq,ctx", [(1, 70), (40, 33), (300, 0)])
def test_attention_does_not_see_what_is_masked(dtype, d, lq, ctx):
    """Infinities and NaN in the rows of the cache around a sequence's keys, in keys and values behind a token's own, and in
    another sequence, change no bit."""
    g = _gen(lq + d)
    h, kv, lk = 4, 2, lq + ctx
    off, begin = [0, lq, 2 * lq], [5, lk + 40]
    end = [b + lk for b in begin]
    rows = end[1] + 50
    q, k, v = (ou.rand(g, n, x, d, dtype=dtype).cuda() for n, x in ((2 * lq, h), (rows, kv), (rows, kv)))
    for block in (0, 1, 8):
        clean = _run_attention(q, k, v, off, begin, end, block)
        k2, v2 = k.clone(), v.clone()
        inside = torch.zeros(rows, dtype=torch.bool, device="cuda")
        for b, e in zip(begin, end):
            inside[b:e] = True
        for t in (k2, v2):
            t[~inside] = float("nan")
        v2[~inside, :, ::2] = float("-inf")
        assert torch.equal(_run_attention(q, k2, v2, off, begin, end, block), clean)
        if block == 0 or lq == 1:
            continue
        # the last keys of the first sequence: seen by its last tokens only
        n_bad = 3
        k3, v3 = k.clone(), v.clone()
        k3[end[0] - n_bad:end[0], 0] = float("nan")
        v3[end[0] - n_bad:end[0], 1, 3] = float("inf")
        v3[end[0] - 1, 1, 4] = float("nan")
        got = _run_attention(q, k3, v3, off, begin, end, block)
        sees = [ou.limit(i, lq, lk, block) > lk - n_bad for i in range(lq)]
        blind = torch.tensor([not s for s in sees] + [True] * lq, device="cuda")
        assert torch.equal(got[blind], clean[blind])
        for i in range(lq):
            if not sees[i]:
                continue
            assert torch.isnan(got[i, :2]).all()                       # heads of key head 0: a NaN logit
            assert torch.isinf(got[i, 2:, 3]).all() and (got[i, 2:, 3] > 0).all()
            assert torch.isnan(got[i, 2:, 4]).all() == (ou.limit(i, lq, lk, block) == lk)
            other = [c for c in range(d) if c not in (3, 4)]
            assert torch.isfinite(got[i, 2:, other]).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attention_with_steep_and_shifted_logits(dtype):
    """Logits of thousands, rising along the keys: the reference of the exponentials has to follow."""
    g = _gen(5)
    lq, lk, h, kv, d = 40, 700, 4, 2, 128
    q = ou.rand(g, lq, h, d, dtype=dtype).abs()
    k = ou.rand(g, lk, kv, d, dtype=dtype).abs() * torch.linspace(-20, 20, lk)[:, None, None]
    k, v = k.to(q.dtype), ou.rand(g, lk, kv, d, dtype=dtype)
    for block in (0, 1, 16):
        _check_attention(q, k, v, [0, lq], [0], [lk], block, scale=1.0)
        _check_attention(q, -k, v, [0, lq], [0], [lk], block, scale=0.01)


def test_attention_reads_behind_32_bits():
    """Rows of K and V more than 2^32 bytes, and 2^31 elements, apart."""
    d, kv, h, ld, lk = 128, 1, 4, 1 << 24, 200
    buf = torch.empty(lk * ld, dtype=torch.bfloat16, device="cuda")
    g = _gen(9)
    k, v, q = ou.rand(g, lk, kv, d, dtype="bf16"), ou.rand(g, lk, kv, d, dtype="bf16"), ou.rand(g, 3, h, d, dtype="bf16")
    kd = buf.as_strided((lk, kv, d), (ld, d, 1))
    vd = buf.as_strided((lk, kv, d), (ld, d, 1), storage_offset=1 << 20)
    kd.copy_(k)
    vd.copy_(v)
    want, bound, _ = ou.attention64(q, k, v, [0, 3], [0], [lk], 1, d ** -0.5)
    assert ou.worst(_run_attention(q.cuda(), kd, vd, [0, 3], [0], [lk], 1), want, bound) <= 1.0
    want, bound, _ = ou.attention64(q, k, v, [0, 3], [150], [lk], 1, d ** -0.5)
    assert ou.worst(_run_attention(q.cuda(), kd, vd, [0, 3], [150], [lk], 1), want, bound) <= 1.0


def test_attention_takes_bad_offsets_as_the_nearest_good_ones():
    g = _gen(11)
    q, k, v = (ou.rand(g, n, x, 64, dtype="bf16").cuda() for n, x in ((10, 2), (50, 1), (50, 1)))
    bad = _run_attention(q, k, v, [0, 4, 99], [-7, 20], [30, 1000], 1, max_q=10, max_k=50)
    good = _run_attention(q, k, v, [0, 4, 10], [0, 20], [30, 50], 1, max_q=10, max_k=50)
    assert torch.equal(bad, good)
    out = _run_attention(q, k, v, [0, 4, 10], [30, 20], [10, 5], 0, max_k=50)      # an end in front of its begin: no keys
    assert (out == 0).all()


def test_attention_of_nothing():
    q = torch.empty(0, 4, 64, dtype=torch.bfloat16, device="cuda")
    k = torch.randn(5, 2, 64, device="cuda").bfloat16()
    _run_attention(q, k, k, [0, 0, 0], [0, 0], [5, 0], 1)
    _run_attention(q, k, k, [0], [], [], 1)
    q = torch.randn(6, 4, 64, device="cuda").bfloat16()
    assert (_run_attention(q, k[:0], k[:0], [0, 6], [0], [0], 0) == 0).all()


# ---- streams, graphs, a layer ---------------------------------------------------------------------

def test_calls_on_two_streams_at_once():
    """Each call has a workspace of its own."""
    g = _gen(21)
    sets = []
    for _ in range(2):
        q, k, v = (ou.rand(g, n, x, 128, dtype="bf16").cuda() for n, x in ((1, 8), (6000, 1), (6000, 1)))
        sets.append((q, k, v, _run_attention(q, k, v, [0, 1], [0], [6000], 1)))
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    outs = [[], []]
    for _ in range(20):
        for i, s in enumerate(streams):
            q, k, v, _ = sets[i]
            out = torch.empty_like(q)
            off, b, e = _ints([0, 1]), _ints([0]), _ints([6000])
            s.wait_stream(torch.cuda.current_stream())
            B.dare_k_attention_packed(q, k, v, out, off, b, e, 1, 6000, causal_block=1, stream=s)
            for t in (off, b, e, out):
                t.record_stream(s)
            outs[i].append(out)
    torch.cuda.synchronize()
    for i in range(2):
        assert all(torch.equal(o, sets[i][3]) for o in outs[i])


class Layer:
    """A decoder layer's attention over a cache made of the three operators: Q, K and V with biases, rotation and cache rows,
    attention, output projection onto the residual stream."""

    def __init__(self, seed, dtype, hidden, h, kv, d, batch, room, block):
        g = _gen(seed)
        self.h, self.kv, self.d, self.block, self.room, self.batch = h, kv, d, block, room, batch
        self.hidden, self.n = hidden, (h + 2 * kv) * d
        self.wqkv, self.bias = ou.rand(g, self.n, hidden, dtype=dtype, std=hidden ** -0.5).cuda(), ou.rand(g, self.n, dtype=dtype).cuda()
        self.wo = ou.rand(g, hidden, h * d, dtype=dtype, std=(h * d) ** -0.5).cuda()
        self.freqs = B.dare_k_rope_freqs(d, 10000.0, "turns", 4.0, 128)
        self.k, self.v = (torch.zeros(batch * room, kv, d, dtype=self.wo.dtype, device="cuda") for _ in range(2))

    def step(self, x, lens, ctx, check=False, offsets=None):
        """lens new tokens of every sequence behind ctx cached ones; x [tokens, hidden] is updated."""
        h, kv, d = self.h, self.kv, self.d
        off = _offsets(lens)
        if offsets is None:
            offsets = self.offsets(lens, ctx)
        pos, rows, q_off, begin, end = offsets
        qkv = torch.empty(x.shape[0], self.n, dtype=x.dtype, device="cuda")
        B.dare_k_linear(x, self.wqkv, qkv, bias=self.bias)
        heads = qkv.view(-1, h + 2 * kv, d)
        q, k, v = heads[:, :h], heads[:, h:h + kv], heads[:, h + kv:]
        if check:
            want, bound = ou.linear64(x.cpu(), self.wqkv.cpu(), self.bias.cpu(), None, None)
            assert ou.worst(qkv, want, bound) <= 1.0
            wq, bq = ou.rope64(q.cpu(), pos.cpu(), self.freqs.cpu(), d, "half", 1.0)
            wk, bk = ou.rope64(k.cpu(), pos.cpu(), self.freqs.cpu(), d, "half", 1.0)
        B.dare_k_rope(pos, self.freqs, "half", q, q, k, self.k, v, self.v, rows=rows)
        if check:
            assert ou.worst(q, wq, bq) <= 1.0 and ou.worst(self.k[rows.long()], wk, bk) <= 1.0
            assert torch.equal(self.v[rows.long()], v)
        o = torch.empty_like(q, memory_format=torch.contiguous_format)
        B.dare_k_attention_packed(q, self.k, self.v, o, q_off, begin, end, max(lens), max(a + b for a, b in zip(lens, ctx)),
                                  causal_block=self.block)
        if check:
            want, bound, covered = ou.attention64(q.cpu(), self.k.cpu(), self.v.cpu(), off, begin.tolist(), end.tolist(), self.block, d ** -0.5)
            assert covered.all() and ou.worst(o, want, bound) <= 1.0
            want, bound = ou.linear64(o.cpu().flatten(1), self.wo.cpu(), None, None, x.cpu())
        B.dare_k_linear(o.flatten(1), self.wo, x, residual=x)
        if check:
            assert ou.worst(x, want, bound) <= 1.0
        return x

    def offsets(self, lens, ctx):
        pos = [c + i for n, c in zip(lens, ctx) for i in range(n)]
        rows = [b * self.room + c + i for b, (n, c) in enumerate(zip(lens, ctx)) for i in range(n)]
        begin = [b * self.room for b in range(self.batch)]
        return (_ints(pos), _ints(rows), _ints(_offsets(lens)), _ints(begin), _ints([s + n + c for s, n, c in zip(begin, lens, ctx)]))


@pytest.mark.parametrize("dtype,hidden,h,kv,d,block", [("bf16", 512, 8, 2, 64, 1), ("bf16", 896, 7, 1, 128, 32), ("f32", 256, 4, 2, 64, 1)])
def test_layer_of_a_prompt_blocks_and_single_tokens(dtype, hidden, h, kv, d, block):
    layer = Layer(5, dtype, hidden, h, kv, d, 3, 200, block)
    g = _gen(8)
    ctx = [0, 0, 0]
    for lens in ([40, 96, 1], [32, 32, 32], [1, 0, 1], [1, 1, 1]):
        x = ou.rand(g, sum(lens), hidden, dtype=dtype).cuda()
        layer.step(x, lens, ctx, check=True)
        ctx = [a + b for a, b in zip(ctx, lens)]


def test_layer_captured_and_replayed_with_other_lengths():
    """One captured step over the cache, replayed as the sequences grow, with eager work between the replays."""
    make = lambda: Layer(6, "bf16", 512, 8, 2, 64, 3, 3000, 1)
    eager, cap = make(), make()
    g = _gen(9)
    fill = [ou.rand(g, 9000, 2, 64, dtype="bf16").cuda() for _ in range(2)]
    for l in (eager, cap):
        l.k.copy_(fill[0])
        l.v.copy_(fill[1])
    lens, ctx0 = [1, 1, 1], [2900, 1203, 7]
    static_x = torch.zeros(3, 512, dtype=torch.bfloat16, device="cuda")
    static_off = tuple(t.clone() for t in cap.offsets(lens, ctx0))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        cap.step(static_x.clone(), lens, [2990] * 3, offsets=static_off)      # warm-up; its cache rows are written again below
    torch.cuda.synchronize()
    cap.k.copy_(fill[0])
    cap.v.copy_(fill[1])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        y = static_x.clone()
        cap.step(y, lens, [2990] * 3, offsets=static_off)
    torch.cuda.synchronize()
    ctx = list(ctx0)
    for rep in range(5):
        x = ou.rand(g, 3, 512, dtype="bf16").cuda()
        static_x.copy_(x)
        for dst, src in zip(static_off, cap.offsets(lens, ctx)):
            dst.copy_(src)
        graph.replay()
        torch.cuda.synchronize()
        # the eager layer with the same hints, on its own cache
        want = eager.step(x.clone(), lens, [2990] * 3, offsets=eager.offsets(lens, ctx))
        assert torch.equal(y, want), rep
        assert torch.equal(cap.k, eager.k) and torch.equal(cap.v, eager.v)
        ctx = [c + 1 for c in ctx]


def test_frequencies_in_memory_that_an_earlier_kernel_still_writes():
    """Made while the stream still has work for a freed tensor whose memory they get: they come behind it."""
    want = B.dare_k_rope_freqs(128).cpu()
    busy = torch.empty(1 << 28, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for _ in range(3):
            old = torch.empty(64, dtype=torch.float64, device="cuda")
            for _ in range(20):
                busy.fill_(1.0)
            old.fill_(7.0)
            del old
            freqs = B.dare_k_rope_freqs(128)
            side.synchronize()
            assert torch.equal(freqs.cpu(), want)
            del freqs
    torch.cuda.synchronize()
