"""Refusals of dare_k_linear, dare_k_rope and dare_k_attention_packed, in front of any GPU work, and the plain arithmetic of
attn_packed.h: the keys that a token sees, and how the work is cut."""
import ctypes
import os
import struct
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


ROPE = dict(size=B._ROPE_CALL.size, dtype=B.DARE_BF16, layout=0, n=3, d=64, rot=64, h=4, kv=2, out_rows=9, mag=1.0, pos=P, freqs=P, rows=P,
            q=P, k=P, v=P, qo=2 * P, ko=2 * P, vo=2 * P, ldq=256, ldk=128, ldv=128, ldqo=256, ldko=128, ldvo=128)


@pytest.mark.parametrize("change,want", [
    (dict(size=8), B.DARE_ERR_INVALID_ARG), (dict(rows=P + 2), B.DARE_ERR_INVALID_ARG),
    (dict(dtype=2), B.DARE_ERR_INVALID_ARG), (dict(layout=2), B.DARE_ERR_INVALID_ARG), (dict(n=-1), B.DARE_ERR_INVALID_ARG),
    (dict(rot=0), B.DARE_ERR_INVALID_ARG), (dict(rot=7), B.DARE_ERR_INVALID_ARG), (dict(rot=66), B.DARE_ERR_INVALID_ARG),
    (dict(d=260, rot=8), B.DARE_ERR_UNSUPPORTED), (dict(d=264, rot=8), B.DARE_ERR_UNSUPPORTED), (dict(d=4, rot=2), B.DARE_ERR_UNSUPPORTED),
    (dict(pos=0), B.DARE_ERR_INVALID_ARG), (dict(freqs=0), B.DARE_ERR_INVALID_ARG), (dict(freqs=P + 4), B.DARE_ERR_INVALID_ARG),
    (dict(pos=P + 2), B.DARE_ERR_INVALID_ARG), (dict(mag=float("nan")), B.DARE_ERR_INVALID_ARG),
    (dict(mag=float("inf")), B.DARE_ERR_INVALID_ARG), (dict(qo=0), B.DARE_ERR_INVALID_ARG), (dict(k=0), B.DARE_ERR_INVALID_ARG),
    (dict(ldq=255), B.DARE_ERR_INVALID_ARG), (dict(ldvo=127), B.DARE_ERR_INVALID_ARG), (dict(h=0), B.DARE_ERR_INVALID_ARG),
    (dict(kv=0), B.DARE_ERR_INVALID_ARG), (dict(q=P + 1), B.DARE_ERR_INVALID_ARG), (dict(k=2 * P), B.DARE_ERR_INVALID_ARG),
    (dict(q=2 * P, ldq=260), B.DARE_ERR_INVALID_ARG), (dict(out_rows=0), B.DARE_ERR_INVALID_ARG),
    (dict(ldq=(1 << 24) + 1), B.DARE_ERR_UNSUPPORTED),
])
def test_rope_refuses(L, change, want):
    assert L.dare_k_rope(B._ROPE_CALL.pack(*dict(ROPE, **change).values()), None) == want
    assert L.dare_last_error(None)


def test_rope_of_no_call_and_of_no_tokens(L):
    assert L.dare_k_rope(None, None) == B.DARE_ERR_INVALID_ARG
    assert L.dare_k_rope(B._ROPE_CALL.pack(*dict(ROPE, n=0, q=0, pos=0, freqs=0).values()), None) == B.DARE_OK


@pytest.mark.parametrize("rows", [0, P])
def test_rope_without_tensors_has_nothing_to_do(L, rows):
    """q, k and v may each be left out, and so may all of them: nothing is launched."""
    none = dict(q=0, k=0, v=0, qo=0, ko=0, vo=0)
    assert L.dare_k_rope(B._ROPE_CALL.pack(*dict(ROPE, rows=rows, **none).values()), None) == B.DARE_OK


def test_structs_of_the_binding_are_those_of_the_header(tmp_path):
    """Size and the place of the last field of every group."""
    (tmp_path / "sizes.cpp").write_text(r"""
#include <cstdio>
#include <cstddef>
#include "dare_kernels.h"
#define P(t, f) std::printf("%zu ", offsetof(t, f))
int main() {
  std::printf("%zu %zu ", sizeof(dare_rope_call), sizeof(dare_packed_call));
  P(dare_rope_call, magnitude); P(dare_rope_call, pos); P(dare_rope_call, rows); P(dare_rope_call, v); P(dare_rope_call, v_out); P(dare_rope_call, ldvo);
  P(dare_packed_call, scale); P(dare_packed_call, ldo); P(dare_packed_call, out); P(dare_packed_call, k_end);
}""")
    subprocess.run(["g++", "-std=c++17", "-I", os.path.join(ROOT, "include"), str(tmp_path / "sizes.cpp"), "-o", str(tmp_path / "sizes")], check=True)
    got = [int(x) for x in subprocess.run([str(tmp_path / "sizes")], capture_output=True, text=True, check=True).stdout.split()]
    at = lambda fmt: struct.calcsize("@" + fmt)
    assert got == [B._ROPE_CALL.size, B._PACKED_CALL.size, at("I8i"), at("I8ifP") - 8, at("I8if3P") - 8, at("I8if6P") - 8, at("I8if9P") - 8,
                   B._ROPE_CALL.size - 8, at("I10i"), at("I10if4q") - 8, at("I10if4q4P") - 8, B._PACKED_CALL.size - 8]


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
    base = dict(struct_size=B._PACKED_CALL.size, dtype=B.DARE_BF16, batch=2, total_q=5, k_rows=50, max_q=4, max_k=30,
                n_heads=4, n_kv_heads=2, head_dim=64, causal_block=1, scale=0.125, ldq=256, ldk=128, ldv=128, ldo=256,
                q=P, k=P, v=P, out=P, q_off=P, k_begin=P, k_end=P)
    base.update(kw)
    return B._PACKED_CALL.pack(*base.values())


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
def test_attention_refuses_a_call(L, kw, want):
    call, need = _packed(**kw), ctypes.c_size_t(7)
    assert L.dare_k_attention_packed(call, P, 1 << 30, None) == want
    assert L.dare_last_error(None)
    assert L.dare_k_attention_packed_workspace(call, ctypes.byref(need)) == want and need.value == 0


def test_attention_refuses_pointers_and_workspaces(L):
    run = lambda ws=P, size=1 << 30, **kw: L.dare_k_attention_packed(_packed(**kw), ws, size, None)
    for name in ("q", "k", "v", "out", "q_off", "k_begin", "k_end"):
        assert run(**{name: 0}) == B.DARE_ERR_INVALID_ARG, name
        assert run(**{name: P + (8 if name in ("q", "k", "v", "out") else 2)}) == B.DARE_ERR_INVALID_ARG, name
    assert run(ldk=132) == B.DARE_ERR_INVALID_ARG
    long = dict(batch=1, total_q=1, max_q=1, max_k=100000, k_rows=100000)
    need = ctypes.c_size_t()
    assert L.dare_k_attention_packed_workspace(_packed(**long), ctypes.byref(need)) == B.DARE_OK
    assert need.value > 0
    for ws in ((None, need.value), (P, need.value - 1), (P + 4, need.value)):
        assert run(*ws, **long) == B.DARE_ERR_INVALID_ARG
    assert L.dare_k_attention_packed(None, P, 1 << 30, None) == B.DARE_ERR_INVALID_ARG
    assert L.dare_k_attention_packed_workspace(_packed(), None) == B.DARE_ERR_INVALID_ARG
    # nothing to do: no pointers needed
    nothing = dict(q=0, k=0, v=0, out=0, q_off=0, k_begin=0, k_end=0)
    assert run(None, 0, total_q=0, **nothing) == B.DARE_OK and run(None, 0, batch=0, **nothing) == B.DARE_OK


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


def test_launches_of_more_lanes_than_there_can_be_are_refused(L):
    """2^32 lanes in a launch: a workgroup of 256 per four tokens, per block of rows and key head."""
    assert L.dare_k_rope(B._ROPE_CALL.pack(*dict(ROPE, n=(1 << 25) + 1).values()), None) == B.DARE_ERR_UNSUPPORTED
    wide = dict(n_heads=8, n_kv_heads=8, ldq=512, ldk=512, ldv=512, ldo=512, batch=1, q=0)   # q=0: nothing is launched
    for dtype, max_q, rows in ((B.DARE_BF16, 1, 16), (B.DARE_BF16, 32, 32), (B.DARE_BF16, 33, 128), (B.DARE_F32, 33, 16)):
        for blocks, want in (((1 << 21) - 2, B.DARE_ERR_INVALID_ARG), (1 << 21, B.DARE_ERR_UNSUPPORTED)):
            # (2^28 - 17 tokens of 8 heads stay below the limit on rows, and are (2^28 - 17) // 128 + 1 = 2^21 blocks of 128)
            call = _packed(**dict(wide, dtype=dtype, max_q=max_q, total_q=min(blocks * rows, (1 << 28) - 17)))
            assert L.dare_k_attention_packed(call, P, 1 << 30, None) == want, (dtype, max_q, blocks)


def test_limits_that_the_header_names(L):
    """Every ld up to 2^24, heads of a rotation up to 65535; the query of the workspace does not count blocks."""
    beyond = (1 << 24) + 64
    for change in (dict(lda=beyond), dict(ldo=beyond), dict(residual=3 * P, ldr=beyond)):
        assert L.dare_k_linear(*dict(LINEAR, **change).values(), None) == B.DARE_ERR_UNSUPPORTED, change
    for name in ("ldq", "ldk", "ldv", "ldqo", "ldko", "ldvo"):
        assert L.dare_k_rope(B._ROPE_CALL.pack(*dict(ROPE, **{name: beyond}).values()), None) == B.DARE_ERR_UNSUPPORTED, name
    for change in (dict(h=65536, ldq=1 << 23, ldqo=1 << 23), dict(kv=65536, ldk=1 << 23, ldko=1 << 23)):
        assert L.dare_k_rope(B._ROPE_CALL.pack(*dict(ROPE, **change).values()), None) == B.DARE_ERR_INVALID_ARG
    need = ctypes.c_size_t(7)
    for name in ("ldq", "ldk", "ldv", "ldo"):
        call = _packed(**{name: beyond})
        assert L.dare_k_attention_packed(call, P, 1 << 30, None) == B.DARE_ERR_UNSUPPORTED, name
        assert L.dare_k_attention_packed_workspace(call, ctypes.byref(need)) == B.DARE_ERR_UNSUPPORTED and need.value == 0
    many = _packed(n_heads=8, n_kv_heads=8, ldq=512, ldk=512, ldv=512, ldo=512, batch=1 << 21, max_q=1, total_q=5)
    assert L.dare_k_attention_packed(many, P, 1 << 30, None) == B.DARE_ERR_UNSUPPORTED
    assert L.dare_k_attention_packed_workspace(many, ctypes.byref(need)) == B.DARE_OK


ROUTES = r"""
#include <cstdio>
#include <cstdlib>
#include <initializer_list>
#include "gemm_route.h"
int main(int n, char** a) {
  for (int i = 1; i + 2 < n; i += 3) std::printf("%d ", (int)dare::linear_route(atoi(a[i]), atoi(a[i + 1]), atoi(a[i + 2])));
  if (n > 1) return 0;
  bool seen[64] = {};  // what the rule ever takes
  for (int m = 1; m <= 20000; m = m < 300 ? m + 1 : m + m / 37)
    for (int c = 64; c <= 1 << 20; c = c < 16384 ? c + 64 : c + c / 640 * 64)
      for (int k : {64, 128, 192, 2048, 4096}) seen[(int)dare::linear_route(m, c, k)] = true;
  for (int r = 0; r < 64; ++r)
    if (seen[r]) std::printf("%d ", r);
}
"""


def test_every_tile_shape_of_the_projection_has_a_test(tmp_path):
    """The sizes that the GPU test runs take the routes that they are there for, those are all that the launch can take, and the rule takes no
    other."""
    import re
    csrc = os.path.join(ROOT, "paper_2605_08134_amd", "csrc")
    header, source = (open(os.path.join(csrc, f)).read() for f in ("gemm_route.h", "gemm_bf16.hip"))
    names = re.findall(r"^  (k\w+),", header[header.index("enum class GemmRoute"):header.index("};")], re.M)
    body = source[source.index("hipError_t launch_linear(const GemmArgs& g"):]
    launched = set(re.findall(r"case GemmRoute::(\w+)", body[:body.index("default:")]))
    (tmp_path / "routes.cpp").write_text(ROUTES)
    subprocess.run(["g++", "-std=c++17", "-O2", "-I", csrc, str(tmp_path / "routes.cpp"), "-o", str(tmp_path / "routes")], check=True)
    run = lambda *args: [names[int(v)] for v in subprocess.run([str(tmp_path / "routes"), *args], capture_output=True, text=True, check=True).stdout.split()]
    assert run(*[str(v) for s in ou.LINEAR_SHAPES for v in s[1:]]) == [s[0] for s in ou.LINEAR_SHAPES]
    assert {s[0] for s in ou.LINEAR_SHAPES} == launched
    assert set(run()) == launched
    assert any(s[0] == "kQuad256" and s[1] * s[2] * 2 > 128 << 20 for s in ou.LINEAR_SHAPES)
