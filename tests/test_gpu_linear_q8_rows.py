"""A row's result of dare_k_linear_q8 has the same bits whatever the number of rows beside it, and with it the shape of the tiles."""
import pytest
import torch

from paper_2605_08134_amd import binding as B
import step8_util as su

pytestmark = pytest.mark.gpu

TYPES = {"bf16": (torch.bfloat16, torch.int16), "f32": (torch.float32, torch.int32)}


@pytest.mark.parametrize("act", [None, "silu", "gelu", "gelu_tanh"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("extras", ["none", "bias", "residual", "both"])
@pytest.mark.parametrize("n,k,rows", su.LINEAR_Q8_ROWS)
def test_rows_have_the_same_bits_in_every_shape(n, k, rows, extras, dtype, act):
    """Products of some 40 in size, so that activations end in zeros of both signs; a scale of 0 and one below it."""
    td, bits = TYPES[dtype]
    g = torch.Generator(device="cuda").manual_seed(n + k)
    most = max(rows)
    codes = lambda *s: torch.randint(-127, 128, s, generator=g, dtype=torch.int8, device="cuda")
    a, wt = codes(most, k), codes(n, k)
    sa, sw = torch.rand(most, generator=g, device="cuda") * 0.04, torch.rand(n, generator=g, device="cuda") * 0.04
    sa[1], sa[2] = 0.0, -0.02
    rn = lambda *s: torch.randn(s, generator=g, device="cuda").to(td)
    bias = rn(n) if extras in ("bias", "both") else None
    res = rn(most, n) if extras in ("residual", "both") else None
    want = None
    for m in sorted(rows, reverse=True):
        out = torch.full((m, n), float("nan"), dtype=td, device="cuda")
        B.dare_k_linear_q8(a[:m], sa[:m], wt, sw, out, bias, act, None if res is None else res[:m])
        want = out if want is None else want
        other = out.view(bits) != want[:m].view(bits)
        assert not other.any(), "%d of %d rows: %s and %s" % (m, most, out[other][:4].tolist(), want[:m][other][:4].tolist())
