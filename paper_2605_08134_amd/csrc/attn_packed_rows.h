// Rows of attention over packed sequences, for the kernels of both types: block numbers, sequences, keys (see
// attn_packed.hip).
#pragma once

#include "attn_packed.h"
#include "dare_common.h"

namespace dare {

struct PackedRows {
  const int32_t* q_off;
  const int32_t* k_begin;
  const int32_t* k_end;
  int batch, total_q, k_rows;
  int group;         // query heads per key head
  int causal_block;
  int n_blocks;      // row blocks launched
  Divider by_group, by_causal_block;
};

inline PackedRows packed_rows(const PackedArgs& a, int n_blocks) {
  return {a.q_off, a.k_begin, a.k_end, a.batch, a.total_q, a.k_rows, a.n_heads / a.n_kv_heads, a.causal_block, n_blocks,
          divider(a.n_heads / a.n_kv_heads), divider(a.causal_block ? a.causal_block : 1)};
}

struct Place {
  int q0, k0;        // first query token and first key of the sequence
  int len_k, shift;  // its keys; keys in front of the first query (len_k - len_q)
  int row0, rows;    // rows of the block: row0 .. row0 + rows - 1 of the sequence's
};

// Block g of BM rows; false if it is empty.  All lanes of a wave call it; the result is the same in all of them.  Whatever the
// offsets hold, rows lie in [0, total_q) and keys in [0, k_rows).
template <int BM>
__device__ __forceinline__ bool find_block(const PackedRows& p, const int g, Place& at) {
  const int lane = threadIdx.x & 63;
  auto offset = [&](int b) __attribute__((always_inline)) {
    const int o = p.q_off[b];
    return o < 0 ? 0 : o > p.total_q ? p.total_q : o;
  };
  auto number = [&](int off, int b) __attribute__((always_inline)) { return (int)((unsigned)(off * p.group) / BM) + b; };
  int lo = 0, n = p.batch;
  while (n > 64) {  // 64 candidates at a time
    const int step = (n + 63) >> 6, b = lane * step;
    const int count = __builtin_popcountll(__ballot(b < n && number(offset(lo + b), lo + b) <= g));
    if (count == 0) return false;
    lo += (count - 1) * step;
    n -= (count - 1) * step;
    n = n < step ? n : step;
  }
  // (the last round reads all that is to know of its candidates)
  const int b = lo + (lane < n ? lane : n - 1);
  const int own_first = offset(b), own_end = offset(b + 1), own_begin = p.k_begin[b], own_stop = p.k_end[b];
  const int chosen = __builtin_popcountll(__ballot(lane < n && number(own_first, b) <= g)) - 1;
  if (chosen < 0) return false;
  lo += chosen;
  const int first = __builtin_amdgcn_readlane(own_first, chosen), end = __builtin_amdgcn_readlane(own_end, chosen);
  const int len_q = end > first ? end - first : 0;
  at.q0 = first;
  at.row0 = (g - number(first, lo)) * BM;
  const int rows = len_q * p.group - at.row0;
  if (at.row0 < 0 || rows <= 0) return false;
  at.rows = rows < BM ? rows : BM;
  int begin = __builtin_amdgcn_readlane(own_begin, chosen), stop = __builtin_amdgcn_readlane(own_stop, chosen);
  begin = begin < 0 ? 0 : begin > p.k_rows ? p.k_rows : begin;
  stop = stop > p.k_rows ? p.k_rows : stop;
  at.k0 = begin;
  at.len_k = stop > begin ? stop - begin : 0;
  at.shift = at.len_k - len_q;
  return true;
}

// Keys that row j of the sequence sees
__device__ __forceinline__ int row_limit(const PackedRows& p, const Place& at, int j) {
  return packed_limit(divide(j, p.by_group), at.shift, at.len_k, p.causal_block, p.by_causal_block);
}

// All four lanes L, L ^ 16, L ^ 32 and L ^ 48, which hold the same row: maximum, sum.  (The swap's words are copied before they are taken
// for floats: __builtin_bit_cast of an element of a vector reads the first one.)
template <class Join>
__device__ __forceinline__ float row_join(float x, Join join) {
  const unsigned own = __builtin_bit_cast(unsigned, x);
  const auto rows = __builtin_amdgcn_permlane16_swap(own, own, false, false);
  const unsigned even = rows[0], odd = rows[1];
  const unsigned pair = __builtin_bit_cast(unsigned, join(__builtin_bit_cast(float, even), __builtin_bit_cast(float, odd)));
  const auto halves = __builtin_amdgcn_permlane32_swap(pair, pair, false, false);
  const unsigned low = halves[0], high = halves[1];
  return join(__builtin_bit_cast(float, low), __builtin_bit_cast(float, high));
}
__device__ __forceinline__ float row_max(float x) {
  return row_join(x, [](float a, float b) __attribute__((always_inline)) { return fmaxf(a, b); });
}
__device__ __forceinline__ float row_sum(float x) {
  return row_join(x, [](float a, float b) __attribute__((always_inline)) { return a + b; });
}

}  // namespace dare
