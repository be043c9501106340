"""dare_k_logprobs of logits whose scaled size lies far from 0, between ordinary ones and the ends of fp32, against 64 bits.

The bounds are those of ordinary logits (step8_util.logprobs64): they go by differences from the largest logit, which fp32 holds whatever the
logits' own size.  Scales are fp32 numbers, so that both sides have the same."""
import math

import numpy as np
import pytest
import torch

from paper_2605_08134_amd import binding as B
import step8_util as su
from test_gpu_step8 import TYPES, _check, _gen, _outputs

pytestmark = pytest.mark.gpu


def _run(x, tokens, scale, top):
    scale = float(np.float32(scale))
    got = _outputs(x.shape[0], top)
    B.dare_k_logprobs(x.cuda(), tokens.cuda(), *got, scale=scale)
    _check(x, tokens, scale, top, got)


# a wave, four waves and sixteen per row, and few rows cut into parts
VOCABS = [1, 5, 1000, 12000, 40000, 126464]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("vocab", VOCABS)
@pytest.mark.parametrize("scale", [3e4, 65535.0, 65536.0, 1e5, 1e6, 1e7, 1e8, 3e8, 1e9, 1e10, 1e20, 1e30])
def test_logprobs_of_large_scales(dtype, vocab, scale):
    """Temperatures near 0: a leading logit of many sizes, several equal ones, one among -infinity."""
    g = _gen(vocab)
    lead = vocab // 3
    x = (torch.randn(14, vocab, generator=g) * 2).to(TYPES[dtype])
    for r, v in enumerate((24.25, 30.25, 30.5, 31.75, 33.5, 37.25, 38.25, 39.5)):
        x[r, lead] = v
    x[8, ::2] = 30.5                                  # equal ones: the entropy is the logarithm of their number
    x[9] = 38.25
    x[10], x[10, lead] = -math.inf, 30.25
    x[11], x[11, lead] = -math.inf, -30.25
    x[12] = -30.5
    x[13] -= 1000.0
    tokens = torch.full((14,), lead, dtype=torch.int32)
    tokens[3] = vocab - 1
    _run(x, tokens, scale, min(3, vocab))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("vocab", VOCABS)
@pytest.mark.parametrize("size", [1e5, 3e6, 6e6, 1.3e7, 1e9, 1.7e9, 1e10, 1e13, 1e15, 1e20, 1e30, 1e37])
def test_logprobs_of_large_logits(dtype, vocab, size):
    """Logits of a size at scale 1, of both signs; equal ones; neighbours in the type; one apart from the others."""
    g = _gen(vocab)
    spread = torch.randn(2, vocab, generator=g).to(TYPES[dtype])
    x = torch.empty(9, vocab, dtype=TYPES[dtype])
    x[0], x[1] = size, -size
    x[2], x[3] = spread * size
    x[4], x[4, vocab // 2] = size, size * 1.01
    x[5], x[5, vocab // 2] = -size, -size * 0.99
    x[6], x[6, ::3] = -size, 0.5
    x[7], x[7, vocab - 1] = spread[0], size
    x[8], x[8, vocab - 1] = -math.inf, -size
    tokens = torch.full((9,), vocab // 2, dtype=torch.int32)
    tokens[7:] = vocab - 1
    _run(x, tokens, 1.0, min(4, vocab))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("vocab", [1, 5, 1000, 40000, 126464])
@pytest.mark.parametrize("mask", [-1e9, -1e10, -1e15, -1e20, -1e30, -1e38, None])
@pytest.mark.parametrize("scale", [0.5, 0.6, 0.7, 1.0, 1.5])
def test_logprobs_of_masks_that_are_numbers(dtype, vocab, mask, scale):
    """Masks of a large negative number (None: the type's lowest) beside ordinary logits: a whole row, all but one, whole parts of a row, a place here and there."""
    g = _gen(vocab + 1)
    mask = float(torch.finfo(TYPES[dtype]).min) if mask is None else mask
    x = (torch.randn(8, vocab, generator=g) * 3).to(TYPES[dtype])
    x[0] = mask
    x[1], x[1, vocab // 2] = mask, 1.5
    x[2, :vocab // 2] = mask
    x[3, vocab // 4:] = mask
    x[4, ::2] = mask
    x[5], x[5, vocab - 1] = -math.inf, mask
    x[6], x[6, vocab // 3:] = mask, -math.inf
    x[7, :min(40, vocab)] = mask
    tokens = torch.full((8,), vocab // 2, dtype=torch.int32)
    tokens[2], tokens[5], tokens[6] = 0, vocab - 1, 0
    _run(x, tokens, scale, min(5, vocab))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("mask", [-6.5e6, -1e10, -1e30])
@pytest.mark.parametrize("scale", [1.0, 60000.0, 1e8])
def test_logprobs_of_masked_parts(dtype, mask, scale):
    """A row of several parts of which some hold nothing but the mask, others nothing but -infinity; NaN and infinity still reach the whole row."""
    vocab, top = 126464, 6
    x = (torch.randn(9, vocab, generator=_gen(3)) * 3).to(TYPES[dtype])
    x[0, 8000:24000] = mask
    x[1, :100000] = mask
    x[2], x[2, 126000:] = mask, -math.inf
    x[3, :60000], x[3, 60000:] = -math.inf, mask
    x[4], x[4, 50000:50003] = mask, mask / 2          # low ones, some of them less so
    x[5], x[5, 50000:50003] = mask, 2.0
    x[6, :100000], x[6, 101000] = mask, math.nan
    x[7, :100000], x[7, 99] = mask, math.inf
    x[8], x[8, 777] = mask, math.nan
    tokens = torch.full((9,), 50001, dtype=torch.int32)
    got = _outputs(9, top)
    B.dare_k_logprobs(x.cuda(), tokens.cuda(), *got, scale=scale)
    for r in (6, 7, 8):
        assert torch.isnan(got[0][r]) and torch.isnan(got[1][r]) and (got[2][r] == -1).all() and torch.isnan(got[3][r]).all()
    _check(x[:6], tokens[:6], scale, top, [t[:6] for t in got])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("vocab", [5, 1000, 40000, 126464])
@pytest.mark.parametrize("scale", [1e-31, 1e-3, 0.3, 0.49, 0.6, 0.7])
def test_logprobs_of_differences_beyond_fp32(dtype, vocab, scale):
    """A largest logit near the type's end: a lower one's distance from it is beyond fp32, times the scale it is not."""
    most = float(torch.finfo(TYPES[dtype]).max)
    x = torch.zeros(6, vocab, dtype=TYPES[dtype])
    for r, v in enumerate((-1e37, -1e36, -0.4 * most, -0.9 * most, -most, 1e37)):
        x[r], x[r, 1] = v, most
        x[r, 2::7] = -v / 3
    x[5, 3] = -most
    tokens = torch.tensor([0, 0, 0, 0, 4, 3], dtype=torch.int32)
    _run(x, tokens, scale, 5)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("vocab", [5, 1000, 12000, 40000, 126464])
@pytest.mark.parametrize("scale", [65536.0, 1e8, 1e30])
def test_logprobs_special_rows_of_large_scales(dtype, vocab, scale):
    """Nothing left, a token outside the vocabulary, zeros of both signs, the type's ends; NaN and infinity reach their row alone."""
    lowest = float(torch.finfo(TYPES[dtype]).min)
    x = torch.randn(9, vocab, generator=_gen(7)).to(TYPES[dtype])
    x[0] = -math.inf
    x[2], x[2, 3] = 0.0, -0.0
    x[2, 4] = -1.0
    x[3] = lowest
    x[4], x[4, 0] = lowest, -lowest
    x[5], x[5, 2] = -math.inf, lowest
    x[6], x[6, 1:3] = -math.inf, 1e-30
    x[7, vocab - 1], x[8, 0] = math.inf, math.nan
    tokens = torch.tensor([0, vocab, 3, 1, 0, 2, 1, 0, 1], dtype=torch.int32)
    got = _outputs(9, 4)
    B.dare_k_logprobs(x.cuda(), tokens.cuda(), *got, scale=float(np.float32(scale)))
    _check(x[:7], tokens[:7], float(np.float32(scale)), 4, [t[:7] for t in got])
    assert torch.isnan(got[0][7:]).all() and torch.isnan(got[1][7:]).all()
    assert (got[2][7:] == -1).all() and torch.isnan(got[3][7:]).all()
