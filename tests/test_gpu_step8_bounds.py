"""dare_k_norm_q8, dare_k_linear_q8 and dare_k_logprobs where offsets pass 32 bits, and that they leave alone what lies beside their outputs."""
import pytest
import torch

from paper_2605_08134_amd import binding as B
import operator_util as ou
import step8_util as su

pytestmark = pytest.mark.gpu

FAR = 1 << 20     # elements from row to row


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _far(rows, cols, dtype, ld=FAR):
    """An empty [rows, cols] view of a buffer whose last row begins behind 2^32 bytes and, but for one-byte types, behind 2^31 elements."""
    return torch.empty(rows, ld, dtype=dtype, device="cuda")[:, :cols]


def test_norm_q8_rows_behind_32_bits():
    rows, d = 4200, 520
    g = _gen(1)
    x, s, codes = _far(rows, d, torch.bfloat16), _far(rows, d, torch.bfloat16), _far(rows, d, torch.int8)
    x.copy_(torch.randn(rows, d, generator=g, device="cuda"))
    o = torch.randn(rows, d, generator=g, device="cuda").bfloat16()
    gain = torch.ones(d, dtype=torch.bfloat16, device="cuda")
    scales = torch.empty(rows, device="cuda")
    B.dare_k_norm_q8("rms", x, codes, scales, o, s, gain)
    pick = torch.tensor([0, 1, 2047, 2048, 4095, 4096, 4199])
    cpu = lambda t: t[pick.cuda()].cpu()
    want, y = su.norm64("rms", cpu(x), cpu(o), gain.cpu(), None, 1e-5)
    assert torch.equal(cpu(s), want)
    su.check_codes(y, cpu(codes), cpu(scales))


@pytest.mark.parametrize("m", [4200, 9000])
def test_linear_q8_rows_behind_32_bits(m):
    n, k = 192, 256
    g = _gen(2)
    a, out = _far(m, k, torch.int8), _far(m, n, torch.bfloat16)
    a.copy_(torch.randint(-127, 128, (m, k), generator=g, device="cuda", dtype=torch.int8))
    wt = torch.randint(-127, 128, (n, k), generator=g, device="cuda", dtype=torch.int8)
    sa, sw = torch.rand(m, generator=g, device="cuda") * 0.02, torch.rand(n, generator=g, device="cuda") * 0.02
    B.dare_k_linear_q8(a, sa, wt, sw, out)
    pick = torch.tensor([0, 1, 2047, 2048, 4095, 4096, m - 1]).cuda()
    want, bound = su.linear_q8_64(a[pick].cpu(), sa[pick].cpu(), wt.cpu(), sw.cpu(), None, None, None, torch.bfloat16)
    assert ou.worst(out[pick], want, bound) <= 1.0


@pytest.mark.parametrize("m", [3, 70, 300])
def test_linear_q8_weights_and_outputs_behind_32_bits(m):
    """A weight of more than 2^32 codes; with 300 rows the wide tiles."""
    n, k = (1 << 19) + 128, 8320
    g = _gen(3)
    wt = torch.randint(-127, 128, (n, k), generator=g, device="cuda", dtype=torch.int8)
    a = torch.randint(-127, 128, (m, k), generator=g, device="cuda", dtype=torch.int8)
    sa, sw = torch.rand(m, generator=g, device="cuda") * 0.02, torch.rand(n, generator=g, device="cuda") * 0.002
    out = torch.empty(m, n, dtype=torch.bfloat16, device="cuda")
    B.dare_k_linear_q8(a, sa, wt, sw, out)
    cols = torch.cat([torch.arange(64), torch.arange(n - 200, n), torch.tensor([258110, 258111, 516222])]).cuda()
    want, bound = su.linear_q8_64(a.cpu(), sa.cpu(), wt[cols].cpu(), sw[cols].cpu(), None, None, None, torch.bfloat16)
    assert ou.worst(out[:, cols], want, bound) <= 1.0


@pytest.mark.parametrize("dtype,rows,vocab", [(torch.bfloat16, 4200, 333), (torch.float32, 2200, 20001)])
def test_logprobs_rows_behind_32_bits(dtype, rows, vocab):
    g = _gen(4)
    x = _far(rows, vocab, dtype)
    x.copy_(torch.randn(rows, vocab, generator=g, device="cuda") * 3)
    tokens = torch.randint(0, vocab, (rows,), generator=g, device="cuda", dtype=torch.int32)
    lp, h = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
    ids, tops = torch.empty(rows, 3, dtype=torch.int32, device="cuda"), torch.empty(rows, 3, device="cuda")
    B.dare_k_logprobs(x, tokens, lp, h, ids, tops)
    pick = torch.tensor([0, 1, 1023, 1024, 2047, 2048, rows - 1]).cuda()
    cpu = lambda t: t[pick].cpu()
    w = su.logprobs64(cpu(x), cpu(tokens), 1.0, 3)
    assert torch.equal(cpu(ids).long(), w[4])
    for got, want, bound in ((lp, w[0], w[1]), (h, w[2], w[3]), (tops, w[5], w[6])):
        assert ((cpu(got).double() - want).abs() <= bound).all()


def test_outputs_that_lie_next_to_other_tensors():
    """Every output between two guards: what is beside it stays."""
    g = _gen(5)

    def guarded(n, dtype, value):
        buf = torch.full((n + 512,), value, dtype=dtype, device="cuda")
        return buf, buf[256:256 + n]

    for rows, d in ((3, 64), (5, 200), (7, 1544), (2, 20000)):
        x = torch.randn(rows, d, generator=g, device="cuda")
        bc, codes = guarded(rows * d, torch.int8, 99)
        bs, scales = guarded(rows, torch.float32, 7.0)
        bo, s = guarded(rows * d, torch.float32, 7.0)
        B.dare_k_norm_q8(None, x, codes.view(rows, d), scales, x, s.view(rows, d))
        for b, v in ((bc, 99), (bs, 7.0), (bo, 7.0)):
            assert (b[:256] == v).all() and (b[-256:] == v).all()
    for m, n, k in ((1, 64, 128), (9, 128, 384), (33, 4160, 128), (200, 1088, 256), (777, 6144, 128), (300, 12352, 384), (1030, 13120, 384), (17, 66624, 128)):
        a = torch.randint(-127, 128, (m, k), generator=g, device="cuda", dtype=torch.int8)
        wt = torch.randint(-127, 128, (n, k), generator=g, device="cuda", dtype=torch.int8)
        bo, out = guarded(m * n, torch.bfloat16, 7.0)
        B.dare_k_linear_q8(a, torch.ones(m, device="cuda"), wt, torch.ones(n, device="cuda"), out.view(m, n))
        assert (bo[:256] == 7).all() and (bo[-256:] == 7).all()
    for rows, vocab, top in ((1, 5, 2), (3, 1000, 32), (2, 9000, 7), (4, 20000, 32), (2, 70000, 32)):
        x = torch.randn(rows, vocab, generator=g, device="cuda").bfloat16()
        tokens = torch.zeros(rows, dtype=torch.int32, device="cuda")
        bl, lp = guarded(rows, torch.float32, 7.0)
        bh, h = guarded(rows, torch.float32, 7.0)
        bi, ids = guarded(rows * top, torch.int32, 77)
        bt, tops = guarded(rows * top, torch.float32, 7.0)
        B.dare_k_logprobs(x, tokens, lp, h, ids.view(rows, top), tops.view(rows, top))
        for b, v in ((bl, 7.0), (bh, 7.0), (bi, 77), (bt, 7.0)):
            assert (b[:256] == v).all() and (b[-256:] == v).all()
        assert (ids >= 0).all() and torch.isfinite(tops).all() and torch.isfinite(lp).all()
