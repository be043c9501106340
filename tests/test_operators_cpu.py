"""Refusals of dare_k_linear, dare_k_rope and dare_k_attention_packed, in front of any GPU work, and the plain arithmetic of
attn_packed.h: the keys that a token sees, and how the work is cut."""
import ctypes
import os
import subprocess

import pytest
import torch

from paper_2605_08134_amd import binding as B
import operator_util as ou

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
P = 0x1000      # never dereferenced: the checks come first


@pytest.fixture(scope="module")
def L():
    if not os.path.exists(B.LIB_PATH):
        from paper_2605_08134_amd import build
        build.build_library(verbose=False)
    return B.lib()


LINEAR = dict(dtype=B.DARE_BF16, a=P, lda=128, wt=P, n=64, k=128, m=3, bias=None, act=0, residual=None, ldr=0, out=2 * P, ldo=64)


@pytest.mark.parametrize("change,want", [
    (dict(dtype=5), B.DARE_ERR_INVALID_ARG), (dict(m=-1), B.DARE_ERR_INVALID_ARG), (dict(n=0), B.DARE_ERR_INVALID_ARG),
    (dict(act=4), B.DARE_ERR_INVALID_ARG), (dict(act=-1), B.DARE_ERR_INVALID_ARG), (dict(a=None), B.DARE_ERR_INVALID_ARG),
    (dict(wt=None), B.DARE_ERR_INVALID_ARG), (dict(out=None), B.DARE_ERR_INVALID_ARG), (dict(lda=120), B.DARE_ERR_INVALID_ARG),
    (dict(ldo=56), B.DARE_ERR_INVALID_ARG), (dict(residual=P, ldr=56), B.DARE_ERR_INVALID_ARG),
    (dict(lda=132), B.DARE_ERR_INVALID_ARG), (dict(a=P + 8), B.DARE_ERR_INVALID_ARG), (dict(bias=P + 2), B.DARE_ERR_INVALID_ARG),
    (dict(residual=2 * P, ldr=128), B.DARE_ERR_INVALID_ARG), (dict(n=96), B.DARE_ERR_UNSUPPORTED),
    (dict(k=96), B.DARE_ERR_UNSUPPORTED), (dict(m=(1 << 24) + 1), B.DARE_ERR_UNSUPPORTED),
    (dict(n=(1 << 20) + 64, ldo=1 << 21), B.DARE_ERR_UNSUPPORTED), (dict(lda=1 << 25), B.DARE_ERR_UNSUPPORTED),
])
def test_linear_refuses(L, change, want):
    a = dict(LINEAR, **change)
    assert L.dare_k_linear(*a.values(), None) == want
    assert L.dare_last_error(None)


def test_linear_of_no_rows_is_fine_without_tensors(L):
    assert L.dare_k_linear(*dict(LINEAR, m=0, a=None, out=None, wt=None).values(), None) == B.DARE_OK


ROPE = dict(dtype=B.DARE_BF16, layout=0, n=3, d=64, rot=64, pos=P, freqs=P, mag=1.0, q=P, ldq=256, qo=2 * P, ldqo=256, h=4,
            k=P, ldk=128, ko=2 * P, ldko=128, v=P, ldv=128, vo=2 * P, ldvo=128, kv=2, rows=P, out_rows=9)


@pytest.mark.parametrize("change,want", [
    (dict(dtype=2), B.DARE_ERR_INVALID_ARG), (dict(layout=2), B.DARE_ERR_INVALID_ARG), (dict(n=-1), B.DARE_ERR_INVALID_ARG),
    (dict(rot=0), B.DARE_ERR_INVALID_ARG), (dict(rot=7), B.DARE_ERR_INVALID_ARG), (dict(rot=66), B.DARE_ERR_INVALID_ARG),
    (dict(d=260, rot=8), B.DARE_ERR_UNSUPPORTED), (dict(d=264, rot=8), B.DARE_ERR_UNSUPPORTED), (dict(d=4, rot=2), B.DARE_ERR_UNSUPPORTED),
    (dict(pos=None), B.DARE_ERR_INVALID_ARG), (dict(freqs=None), B.DARE_ERR_INVALID_ARG), (dict(freqs=P + 4), B.DARE_ERR_INVALID_ARG),
    (dict(pos=P + 2), B.DARE_ERR_INVALID_ARG), (dict(mag=float("nan")), B.DARE_ERR_INVALID_ARG),
    (dict(mag=float("inf")), B.DARE_ERR_INVALID_ARG), (dict(qo=None), B.DARE_ERR_INVALID_ARG), (dict(k=None), B.DARE_ERR_INVALID_ARG),
    (dict(ldq=255), B.DARE_ERR_INVALID_ARG), (dict(ldvo=127), B.DARE_ERR_INVALID_ARG), (dict(h=0), B.DARE_ERR_INVALID_ARG),
    (dict(kv=0), B.DARE_ERR_INVALID_ARG), (dict(q=P + 1), B.DARE_ERR_INVALID_ARG), (dict(k=2 * P), B.DARE_ERR_INVALID_ARG),
    (dict(q=2 * P, ldq=260), B.DARE_ERR_INVALID_ARG), (dict(out_rows=0), B.DARE_ERR_INVALID_ARG),
    (dict(ldq=(1 << 24) + 1), B.DARE_ERR_UNSUPPORTED),
])
def test_rope_refuses(L, change, want):
    assert L.dare_k_rope(*dict(ROPE, **change).values(), None) == want
    assert L.dare_last_error(None)


@pytest.mark.parametrize("args,want", [
    ((None, 64, 1e4, 0, 1, 1, 0, 1), B.DARE_ERR_INVALID_ARG), ((P, 63, 1e4, 0, 1, 1, 0, 1), B.DARE_ERR_INVALID_ARG),
    ((P, 258, 1e4, 0, 1, 1, 0, 1), B.DARE_ERR_INVALID_ARG), ((P, 64, 0.0, 0, 1, 1, 0, 1), B.DARE_ERR_INVALID_ARG),
    ((P, 64, 1e4, 4, 1, 1, 0, 1), B.DARE_ERR_INVALID_ARG), ((P, 64, 1e4, 1, 0.0, 1, 0, 1), B.DARE_ERR_INVALID_ARG),
    ((P, 2, 1e4, 2, 2.0, 1, 0, 1), B.DARE_ERR_INVALID_ARG), ((P, 64, 1e4, 3, 2.0, 0.0, 0, 1), B.DARE_ERR_INVALID_ARG),
    ((P, 64, 1e4, 3, 2.0, 8192.0, 1, 1), B.DARE_ERR_INVALID_ARG), ((P, 64, float("inf"), 0, 1, 1, 0, 1), B.DARE_ERR_INVALID_ARG),
])
def test_rope_freqs_refuses(L, args, want):
    assert L.dare_k_rope_freqs(*args) == want


def _packed(**kw):
    base = dict(struct_size=ctypes.sizeof(B.DarePackedConfig), dtype=B.DARE_BF16, batch=2, total_q=5, k_rows=50, max_q=4, max_k=30,
                n_heads=4, n_kv_heads=2, head_dim=64, causal_block=1, scale=0.125, ldq=256, ldk=128, ldv=128, ldo=256)
    base.update(kw)
    return B.DarePackedConfig(**base)


@pytest.mark.parametrize("kw,want", [
    (dict(struct_size=8), B.DARE_ERR_INVALID_ARG), (dict(dtype=3), B.DARE_ERR_INVALID_ARG), (dict(batch=-1), B.DARE_ERR_INVALID_ARG),
    (dict(total_q=-1), B.DARE_ERR_INVALID_ARG), (dict(max_k=-1), B.DARE_ERR_INVALID_ARG), (dict(causal_block=-1), B.DARE_ERR_INVALID_ARG),
    (dict(n_heads=0), B.DARE_ERR_INVALID_ARG), (dict(n_kv_heads=3), B.DARE_ERR_INVALID_ARG), (dict(scale=0.0), B.DARE_ERR_INVALID_ARG),
    (dict(scale=float("nan")), B.DARE_ERR_INVALID_ARG), (dict(scale=float("inf")), B.DARE_ERR_INVALID_ARG),
    (dict(head_dim=96), B.DARE_ERR_UNSUPPORTED), (dict(ldq=248), B.DARE_ERR_INVALID_ARG), (dict(ldk=120), B.DARE_ERR_INVALID_ARG),
    (dict(ldo=1 << 25), B.DARE_ERR_UNSUPPORTED), (dict(total_q=2 ** 31 - 1), B.DARE_ERR_UNSUPPORTED),
    (dict(batch=2 ** 24), B.DARE_ERR_UNSUPPORTED),
    (dict(batch=2 ** 23, n_heads=256, n_kv_heads=256, ldq=2 ** 14, ldk=2 ** 14, ldv=2 ** 14, ldo=2 ** 14), B.DARE_ERR_UNSUPPORTED),
])
def test_attention_refuses_a_config(L, kw, want):
    cfg, need = _packed(**kw), ctypes.c_size_t(7)
    assert L.dare_k_attention_packed(ctypes.byref(cfg), P, P, P, P, P, P, P, P, 1 << 30, None) == want
    assert L.dare_last_error(None)
    assert L.dare_k_attention_packed_workspace(ctypes.byref(cfg), ctypes.byref(need)) == want and need.value == 0


def test_attention_refuses_pointers_and_workspaces(L):
    ok = [P] * 7 + [P, 1 << 30]
    call = lambda cfg, args: L.dare_k_attention_packed(ctypes.byref(cfg), *args, None)
    for i in range(7):
        assert call(_packed(), ok[:i] + [None] + ok[i + 1:]) == B.DARE_ERR_INVALID_ARG, i
    for i in range(4):
        assert call(_packed(), ok[:i] + [P + 8] + ok[i + 1:]) == B.DARE_ERR_INVALID_ARG, i
    for i in range(4, 7):
        assert call(_packed(), ok[:i] + [P + 2] + ok[i + 1:]) == B.DARE_ERR_INVALID_ARG, i
    assert call(_packed(ldk=132), ok) == B.DARE_ERR_INVALID_ARG
    long = dict(batch=1, total_q=1, max_q=1, max_k=100000, k_rows=100000)
    need = ctypes.c_size_t()
    assert L.dare_k_attention_packed_workspace(ctypes.byref(_packed(**long)), ctypes.byref(need)) == B.DARE_OK
    assert need.value > 0
    for ws in ([None, need.value], [P, need.value - 1], [P + 4, need.value]):
        assert call(_packed(**long), [P] * 7 + ws) == B.DARE_ERR_INVALID_ARG
    assert L.dare_k_attention_packed(None, *ok, None) == B.DARE_ERR_INVALID_ARG
    assert L.dare_k_attention_packed_workspace(ctypes.byref(_packed()), None) == B.DARE_ERR_INVALID_ARG
    # nothing to do: no pointers needed
    assert call(_packed(total_q=0), [None] * 8 + [0]) == B.DARE_OK and call(_packed(batch=0), [None] * 8 + [0]) == B.DARE_OK


def test_binding_refuses_what_is_not_on_the_gpu():
    x = torch.zeros(4, 2, 64)
    i = torch.zeros(4, dtype=torch.int32)
    with pytest.raises(ValueError):
        B.dare_k_linear(torch.zeros(4, 64), torch.zeros(64, 64), torch.zeros(4, 64))
    with pytest.raises(ValueError):
        B.dare_k_rope(i, torch.zeros(32, dtype=torch.float64), "half", x, x)
    with pytest.raises(ValueError):
        B.dare_k_rope(i, torch.zeros(32, dtype=torch.float64), "half")
    with pytest.raises(ValueError):
        B.dare_k_attention_packed(x, x, x, x, i, i, i, 1, 1)


def test_the_workspace_stays_small_whatever_the_batch():
    for batch, total, max_q in ((1, 1, 1), (1 << 20, 1, 1), (300, 300, 1), (64, 64, 1), (64, 2048, 32), (4096, 9000, 700), (16, 512, 32)):
        for kv in (1, 8, 64):
            for max_k in (1, 511, 4096, 1 << 20):
                need = B.dare_k_attention_packed_workspace(B.DARE_BF16, batch, total, max_q, max_k, 4 * kv, kv, 128)
                assert 0 <= need <= 300 << 20, (batch, total, kv, max_k, need)
                assert B.dare_k_attention_packed_workspace(B.DARE_F32, batch, total, max_q, max_k, 4 * kv, kv, 128) == 0


# ---- the rule ------------------------------------------------------------------------------------

PROBE = r"""
#include <cstdio>
#include <cstdlib>
#include "attn_packed.h"
int main(int n, char** a) {
  if (n == 2) {  // every token of a few sequences
    for (int lq = 1; lq < 12; ++lq)
      for (int lk = 0; lk < 14; ++lk)
        for (int block = 0; block < 9; ++block)
          for (int i = 0; i < lq; ++i) std::printf("%d ", dare::packed_limit(i, lk - lq, lk, block, dare::divider(block ? block : 1)));
    const dare::Divider most = dare::divider(2147483647);
    std::printf("%d %d", dare::packed_limit(5, 0, 10, 2147483647, most), dare::packed_limit(2147483645, 0, 2147483647, 2147483647, most));
    return 0;
  }
  if (n == 3) {  // divisions, at the ends of quotients and of the range
    long wrong = 0;
    unsigned seed = 1;
    for (int k = 0; k < 3000; ++k) {
      seed = seed * 1664525u + 1013904223u;
      const unsigned d = k < 1000 ? k + 1 : k < 1031 ? 1u << (k - 1000) : (seed >> 1 >> (seed & 31) % 31) + 1;
      if (d > 2147483647u) continue;
      const dare::Divider by = dare::divider(d);
      for (unsigned q = 0; q < 2000; ++q) {
        seed = seed * 1664525u + 1013904223u;
        const unsigned long long at = (unsigned long long)(q < 1000 ? q : seed % (2147483647u / d + 1)) * d;
        for (long j = (long)at - 1; j <= (long)at + 1; ++j)
          if (j >= 0 && j < 2147483648l) wrong += dare::divide((int)j, by) != (int)((unsigned)j / d);
      }
      wrong += dare::divide(2147483647, by) != (int)(2147483647u / d);
    }
    std::printf("%ld", wrong);
    return 0;
  }
  const dare::PackedPlan p = dare::packed_plan(atoi(a[1]), atoi(a[2]), atoi(a[3]), atoi(a[4]), atoi(a[5]), atoi(a[6]));
  std::printf("%d %d %d %d", p.rows, p.blocks, p.parts, p.part_keys);
}
"""


@pytest.fixture(scope="module")
def probe(tmp_path_factory):
    d = tmp_path_factory.mktemp("attn_packed")
    (d / "probe.cpp").write_text(PROBE)
    subprocess.run(["g++", "-std=c++17", "-I", os.path.join(ROOT, "paper_2605_08134_amd", "csrc"), str(d / "probe.cpp"),
                    "-o", str(d / "probe")], check=True)
    return lambda *args: [int(v) for v in subprocess.run([str(d / "probe")] + [str(v) for v in args], capture_output=True,
                                                         text=True, check=True).stdout.split()]


def test_keys_that_a_token_sees(probe):
    got = iter(probe("limits"))
    for lq in range(1, 12):
        for lk in range(14):
            for block in range(9):
                for i in range(lq):
                    assert next(got) == ou.limit(i, lq, lk, block), (lq, lk, block, i)
    assert list(got) == [10, 2147483646 + 1]


def test_division_by_a_product(probe):
    assert probe("divide", "all") == [0]


@pytest.mark.parametrize("batch", [1, 3, 32, 257])
@pytest.mark.parametrize("max_q", [1, 4, 33, 5000])
@pytest.mark.parametrize("max_k", [1, 300, 4096, 131072])
@pytest.mark.parametrize("group,kv", [(1, 1), (4, 8), (7, 4)])
def test_the_plan_covers_every_row_and_key(probe, batch, max_q, max_k, group, kv):
    total = batch * max_q - (batch > 1)
    rows, blocks, parts, keys = probe(batch, total, max_q, max_k, group, kv)
    # sequence b has the block numbers from floor(rows in front / BM) + b on
    off = [min(i * max_q, total) for i in range(batch + 1)]
    start = [o * group // rows + b for b, o in enumerate(off)]
    for b in range(batch):
        assert start[b + 1] - start[b] >= -(-(off[b + 1] - off[b]) * group // rows)
    assert start[batch] <= blocks
    assert 1 <= parts <= 64 and keys * parts >= max_k
    if parts > 1:
        assert keys % 64 == 0 and keys >= 128 and -(-max_k // keys) <= parts
