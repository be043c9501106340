"""Refusals of dare_k_norm_q8, dare_k_linear_q8 and dare_k_logprobs, in front of any GPU work; the structs of the binding; the tile that a
projection of codes takes."""
import os
import struct
import subprocess

import pytest
import torch

from paper_2605_08134_amd import binding as B
import step8_util as su

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
P = 0x1000      # never dereferenced: the checks come first
INVALID, UNSUPPORTED = B.DARE_ERR_INVALID_ARG, B.DARE_ERR_UNSUPPORTED


@pytest.fixture(scope="module")
def L():
    if not os.path.exists(B.LIB_PATH):
        from paper_2605_08134_amd import build
        build.build_library(verbose=False)
    return B.lib()


NORM = dict(size=B._NORM_Q8_CALL.size, dtype=B.DARE_BF16, kind=2, rows=3, d=64, eps=1e-5, ldx=64, ldo=72, ldxo=64, ldc=64, x=P, o=2 * P,
            gain=P, bias=0, x_out=3 * P, codes=4 * P, scales=5 * P)


@pytest.mark.parametrize("change,want", [
    (dict(size=8), INVALID), (dict(dtype=2), INVALID), (dict(kind=3), INVALID), (dict(kind=-1), INVALID), (dict(rows=-1), INVALID),
    (dict(d=0), INVALID), (dict(eps=-1.0), INVALID), (dict(eps=float("nan")), INVALID), (dict(eps=float("inf")), INVALID), (dict(x=0), INVALID),
    (dict(codes=0), INVALID), (dict(scales=0), INVALID), (dict(gain=0), INVALID), (dict(kind=1, gain=0), INVALID), (dict(kind=0), INVALID),
    (dict(bias=P), INVALID), (dict(ldx=56), INVALID), (dict(ldo=56), INVALID), (dict(ldxo=56), INVALID), (dict(ldc=56), INVALID),
    (dict(ldx=68), INVALID), (dict(x=P + 8), INVALID), (dict(o=P + 2), INVALID), (dict(gain=P + 8), INVALID), (dict(x_out=P + 4), INVALID),
    (dict(codes=P + 4), INVALID), (dict(ldc=68), INVALID), (dict(scales=P + 2), INVALID), (dict(x_out=P, ldxo=128), INVALID),
    (dict(x_out=2 * P), INVALID), (dict(d=60), UNSUPPORTED), (dict(rows=(1 << 23) + 1), UNSUPPORTED), (dict(ldx=(1 << 24) + 8), UNSUPPORTED),
    (dict(d=(1 << 24) + 8), UNSUPPORTED), (dict(dtype=B.DARE_F32, ldx=66), INVALID),
])
def test_norm_q8_refuses(L, change, want):
    assert L.dare_k_norm_q8(B._NORM_Q8_CALL.pack(*dict(NORM, **change).values()), None) == want
    assert L.dare_last_error(None)


LINEAR = dict(size=B._LINEAR_Q8_CALL.size, dtype=B.DARE_BF16, m=3, n=64, k=128, act=0, lda=128, ldr=0, ldo=64, a=P, row_scale=P, wt=P,
              col_scale=P, bias=0, residual=0, out=2 * P)


@pytest.mark.parametrize("change,want", [
    (dict(size=8), INVALID), (dict(dtype=5), INVALID), (dict(m=-1), INVALID), (dict(n=0), INVALID), (dict(k=0), INVALID), (dict(act=4), INVALID),
    (dict(act=-1), INVALID), (dict(a=0), INVALID), (dict(wt=0), INVALID), (dict(out=0), INVALID), (dict(row_scale=0), INVALID),
    (dict(col_scale=0), INVALID), (dict(lda=112), INVALID), (dict(ldo=56), INVALID), (dict(residual=P, ldr=56), INVALID),
    (dict(lda=136), INVALID), (dict(a=P + 8), INVALID), (dict(wt=P + 8), INVALID), (dict(bias=P + 2), INVALID), (dict(col_scale=P + 4), INVALID),
    (dict(row_scale=P + 2), INVALID), (dict(residual=2 * P, ldr=128), INVALID), (dict(n=96), UNSUPPORTED), (dict(k=192, lda=192), UNSUPPORTED),
    (dict(k=1 << 17, lda=1 << 17), UNSUPPORTED), (dict(m=(1 << 24) + 1), UNSUPPORTED), (dict(n=(1 << 20) + 64, ldo=1 << 21), UNSUPPORTED),
    (dict(m=1 << 18, n=(1 << 19) + 64, ldo=1 << 20), UNSUPPORTED), (dict(lda=1 << 25), UNSUPPORTED), (dict(dtype=B.DARE_F32, ldo=66), INVALID),
])
def test_linear_q8_refuses(L, change, want):
    assert L.dare_k_linear_q8(B._LINEAR_Q8_CALL.pack(*dict(LINEAR, **change).values()), None) == want
    assert L.dare_last_error(None)


LOGPROBS = dict(size=B._LOGPROBS_CALL.size, dtype=B.DARE_F32, rows=3, vocab=100, top=2, scale=1.0, ld=100, logits=P, tokens=P, logprobs=P,
                entropy=P, top_ids=P, top_logprobs=P)


@pytest.mark.parametrize("change,want", [
    (dict(size=8), INVALID), (dict(dtype=-1), INVALID), (dict(rows=-1), INVALID), (dict(vocab=0), INVALID), (dict(top=-1), INVALID),
    (dict(vocab=1), INVALID), (dict(scale=0.0), INVALID), (dict(scale=-1.0), INVALID), (dict(scale=float("nan")), INVALID),
    (dict(scale=float("inf")), INVALID), (dict(scale=2e30), INVALID), (dict(ld=99), INVALID), (dict(logits=0), INVALID), (dict(tokens=0), INVALID),
    (dict(logprobs=0), INVALID), (dict(top_ids=0), INVALID), (dict(top_logprobs=0), INVALID), (dict(logits=P + 2), INVALID),
    (dict(entropy=P + 2), INVALID), (dict(tokens=P + 1), INVALID), (dict(dtype=B.DARE_BF16, logits=P + 1), INVALID), (dict(top=33), UNSUPPORTED),
    (dict(rows=(1 << 21) + 1), UNSUPPORTED), (dict(vocab=(1 << 28) + 1, ld=1 << 29), UNSUPPORTED), (dict(ld=(1 << 32) + 1), UNSUPPORTED),
])
def test_logprobs_refuses(L, change, want):
    assert L.dare_k_logprobs(B._LOGPROBS_CALL.pack(*dict(LOGPROBS, **change).values()), None, 0, None) == want
    assert L.dare_last_error(None)


def test_logprobs_workspace(L):
    """Few rows of many logits are cut into parts and need a workspace; a call without it, or with one too small or not aligned, is refused."""
    need = B.dare_k_logprobs_workspace(B.DARE_BF16, 1, 126464, 2)
    assert need > 0 and need % 16 == 0
    assert B.dare_k_logprobs_workspace(B.DARE_BF16, 1, 126464, 0) < need < B.dare_k_logprobs_workspace(B.DARE_BF16, 3, 126464, 2)
    for rows, vocab in ((0, 126464), (1, 1000), (300, 126464), (1 << 21, 1 << 28)):
        assert B.dare_k_logprobs_workspace(B.DARE_F32, rows, vocab, 32) == 0
    for rows in range(1, 257):
        for vocab in (16384, 40000, 126464, 1 << 28):
            assert B.dare_k_logprobs_workspace(B.DARE_F32, rows, vocab, 32) <= 256 * (16 + 8 * 32)
    few = dict(LOGPROBS, dtype=B.DARE_BF16, rows=1, vocab=126464, ld=126464)
    call = B._LOGPROBS_CALL.pack(*few.values())
    for ws, size in ((None, 0), (P, need - 1), (P + 8, need)):
        assert L.dare_k_logprobs(call, ws, size, None) == INVALID
    assert L.dare_k_logprobs_workspace(call, None) == INVALID
    with pytest.raises(B.DareError):
        B.dare_k_logprobs_workspace(B.DARE_BF16, 1, 126464, 33)


def test_no_call_and_no_rows(L):
    assert L.dare_k_norm_q8(None, None) == L.dare_k_linear_q8(None, None) == L.dare_k_logprobs(None, None, 0, None) == INVALID
    assert L.dare_k_norm_q8(B._NORM_Q8_CALL.pack(*dict(NORM, rows=0, x=0, codes=0, scales=0, gain=0).values()), None) == B.DARE_OK
    assert L.dare_k_linear_q8(B._LINEAR_Q8_CALL.pack(*dict(LINEAR, m=0, a=0, wt=0, out=0).values()), None) == B.DARE_OK
    assert L.dare_k_logprobs(B._LOGPROBS_CALL.pack(*dict(LOGPROBS, rows=0, logits=0).values()), None, 0, None) == B.DARE_OK
    nothing = dict(LOGPROBS, top=0, tokens=0, logprobs=0, entropy=0, top_ids=0, top_logprobs=0)
    assert L.dare_k_logprobs(B._LOGPROBS_CALL.pack(*nothing.values()), None, 0, None) == B.DARE_OK


def test_structs_of_the_binding_are_those_of_the_header(tmp_path):
    (tmp_path / "sizes.cpp").write_text(r"""
#include <cstdio>
#include <cstddef>
#include "dare_kernels.h"
#define P(t, f) std::printf("%zu ", offsetof(t, f))
int main() {
  std::printf("%zu %zu %zu ", sizeof(dare_norm_q8_call), sizeof(dare_linear_q8_call), sizeof(dare_logprobs_call));
  P(dare_norm_q8_call, eps); P(dare_norm_q8_call, ldc); P(dare_norm_q8_call, bias); P(dare_norm_q8_call, x_out); P(dare_norm_q8_call, scales);
  P(dare_linear_q8_call, act); P(dare_linear_q8_call, ldo); P(dare_linear_q8_call, col_scale); P(dare_linear_q8_call, out);
  P(dare_logprobs_call, scale); P(dare_logprobs_call, ld); P(dare_logprobs_call, entropy); P(dare_logprobs_call, top_logprobs);
}""")
    subprocess.run(["g++", "-std=c++17", "-I", os.path.join(ROOT, "include"), str(tmp_path / "sizes.cpp"), "-o", str(tmp_path / "sizes")], check=True)
    got = [int(x) for x in subprocess.run([str(tmp_path / "sizes")], capture_output=True, text=True, check=True).stdout.split()]
    end = lambda fmt, size: struct.calcsize("@" + fmt) - size
    n, l, p = B._NORM_Q8_CALL.size, B._LINEAR_Q8_CALL.size, B._LOGPROBS_CALL.size
    assert got == [n, l, p, end("I4id", 8), end("I4id4q", 8), end("I4id4q4P", 8), end("I4id4q5P", 8), n - 8,
                   end("I5i", 4), end("I5i3q", 8), end("I5i3q4P", 8), l - 8, end("I4if", 4), end("I4ifq", 8), end("I4ifq4P", 8), p - 8]


def test_binding_refuses_tensors_that_are_not_on_the_gpu():
    x, codes, s = torch.zeros(2, 64), torch.zeros(2, 64, dtype=torch.int8), torch.zeros(2)
    with pytest.raises(ValueError):
        B.dare_k_norm_q8(None, x, codes, s)
    with pytest.raises(ValueError):
        B.dare_k_norm_q8("batch", x, codes, s)
    with pytest.raises(ValueError):
        B.dare_k_linear_q8(codes, s, codes, s, x)
    with pytest.raises(ValueError):
        B.dare_k_logprobs(x)
    with pytest.raises(ValueError):
        B.dare_k_logprobs(x, top_ids=codes)


def test_shapes_of_a_projection_of_codes(tmp_path):
    """Every size takes a shape that its launch has: the wide ones only for bf16 outputs and three k-steps or more."""
    (tmp_path / "route.cpp").write_text(r"""
#include <cstdio>
#include "gemm_route.h"
using namespace dare;
int main() {
  const int ns[] = {64, 512, 4096, 6144, 8128, 8192, 12288, 32000, 126464}, ks[] = {64, 128, 192, 2048, 6144, 65472};
  int m = 1, bad = 0, seen = 0;
  for (; m < 40000; m += 1 + m / 7)
    for (int n : ns)
      for (int k : ks)
        for (int bf16 = 0; bf16 < 2; ++bf16) {
          const GemmRoute r = linear_q8_route(m, n, k, bf16);
          const bool wide = r == GemmRoute::kQuad192 || r == GemmRoute::kQuad256;
          if (wide && (!bf16 || k < 192)) ++bad;
          switch (r) {
            case GemmRoute::kSkinny: case GemmRoute::k32x32: case GemmRoute::k64x32: case GemmRoute::k32x64: case GemmRoute::k64x64: case GemmRoute::k64x96:
            case GemmRoute::k64x128: case GemmRoute::k128x96: case GemmRoute::k128x128: case GemmRoute::k128x192: case GemmRoute::kQuad192:
            case GemmRoute::kQuad256: seen |= 1 << (int)r; break;
            default: ++bad;
          }
        }
  std::printf("%d %d", bad, __builtin_popcount(seen));
}""")
    csrc = os.path.join(ROOT, "paper_2605_08134_amd", "csrc")
    subprocess.run(["g++", "-std=c++17", "-I", csrc, str(tmp_path / "route.cpp"), "-o", str(tmp_path / "route")], check=True)
    bad, shapes = subprocess.run([str(tmp_path / "route")], capture_output=True, text=True, check=True).stdout.split()
    assert int(bad) == 0 and int(shapes) == 12


def test_shapes_that_the_gpu_tests_name(tmp_path):
    src = '#include <cstdio>\n#include "gemm_route.h"\nusing namespace dare;\nint main() {\n'
    for shape, m, n, k in su.LINEAR_Q8_SHAPES:
        src += "  std::printf(\"%%d \", linear_q8_route(%d, %d, %d, true) == GemmRoute::%s);\n" % (m, n, k // 2, shape)
    (tmp_path / "names.cpp").write_text(src + "}\n")
    csrc = os.path.join(ROOT, "paper_2605_08134_amd", "csrc")
    subprocess.run(["g++", "-std=c++17", "-I", csrc, str(tmp_path / "names.cpp"), "-o", str(tmp_path / "names")], check=True)
    got = subprocess.run([str(tmp_path / "names")], capture_output=True, text=True, check=True).stdout.split()
    assert got == ["1"] * len(su.LINEAR_Q8_SHAPES)
    assert len({s[0] for s in su.LINEAR_Q8_SHAPES}) == 12


def test_rows_that_are_compared_are_in_every_shape(tmp_path):
    src = '#include <cstdio>\n#include "gemm_route.h"\nusing namespace dare;\nint main() {\n'
    calls = [(n, k, m) for n, k, rows in su.LINEAR_Q8_ROWS for m in rows]
    for n, k, m in calls:
        src += "  std::printf(\"%%d %%d \", (int)linear_q8_route(%d, %d, %d, true), (int)linear_q8_route(%d, %d, %d, false));\n" % (2 * (m, n, k // 2))
    (tmp_path / "rows.cpp").write_text(src + "}\n")
    csrc = os.path.join(ROOT, "paper_2605_08134_amd", "csrc")
    subprocess.run(["g++", "-std=c++17", "-I", csrc, str(tmp_path / "rows.cpp"), "-o", str(tmp_path / "rows")], check=True)
    got = subprocess.run([str(tmp_path / "rows")], capture_output=True, text=True, check=True).stdout.split()
    assert len(got) == 2 * len(calls)
    assert len(set(got[0::2])) == 12 and len(set(got[1::2])) == 10       # (two shapes are there for bf16 outputs only)
