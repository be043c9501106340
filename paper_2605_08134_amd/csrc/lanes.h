// Reductions over the 64 lanes of a wave whose result every lane gets, by the vector unit alone: an exchange through
// LDS (which a general shuffle is) takes a wave over a hundred cycles, six of them in a row for each value.
#pragma once

#include <hip/hip_runtime.h>

namespace dare {
namespace {

// Step s of 0 .. 5: the words `v` of two groups of 2^s lanes, in all lanes of both.  Within a group every lane holds
// the same result by then, so it does not matter which lane of the other group is read: neighbours, pairs, half rows
// and rows of 16 by DPP, the rest by swaps of rows.
template <int STEP>
__device__ __forceinline__ void both_halves(unsigned v, unsigned& a, unsigned& b) {
  if constexpr (STEP < 4) {
    constexpr int pattern = STEP == 0 ? 0xb1 : STEP == 1 ? 0x4e : STEP == 2 ? 0x141 : 0x140;
    a = v;
    b = __builtin_amdgcn_update_dpp(0, v, pattern, 0xf, 0xf, true);
  } else if constexpr (STEP == 4) {
    const auto s = __builtin_amdgcn_permlane16_swap(v, v, false, false);
    a = s[0];
    b = s[1];
  } else {
    const auto s = __builtin_amdgcn_permlane32_swap(v, v, false, false);
    a = s[0];
    b = s[1];
  }
}

// f(x, y) of the same bits whichever of the two comes first; T of 4-byte words.  FROM .. TO: steps, 0 and 6 for the whole wave.
template <int FROM = 0, int TO = 6, typename T, class F>
__device__ __forceinline__ T over_lanes(T v, F f) {
  if constexpr (FROM < TO) {
    constexpr int N = sizeof(T) / 4;
    static_assert(sizeof(T) % 4 == 0, "words");
    unsigned w[N], x[N], y[N];
    __builtin_memcpy(w, &v, sizeof(T));
#pragma unroll
    for (int i = 0; i < N; ++i) both_halves<FROM>(w[i], x[i], y[i]);
    T a, b;
    __builtin_memcpy(&a, x, sizeof(T));
    __builtin_memcpy(&b, y, sizeof(T));
    return over_lanes<FROM + 1, TO>(f(a, b), f);
  } else {
    return v;
  }
}

}  // namespace
}  // namespace dare
