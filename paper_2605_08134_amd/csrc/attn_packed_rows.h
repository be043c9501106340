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

// Inclusive sum along the lanes
__device__ __forceinline__ int wave_prefix_sum(int v) {
  v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xf, 0xf, false);  // row_shr 1, 2, 4, 8: within 16 lanes
  v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xf, 0xf, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xf, 0xf, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xf, 0xf, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xa, 0xf, false);  // row_bcast 15: lane 15 to row 1, 47 to row 3
  v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xc, 0xf, false);  // row_bcast 31: lane 31 to rows 2 and 3
  return v;
}

// All sequences of a launch (64 S at most), S in each lane: their blocks of BM rows and the parts that the keys of a block (tiles of
// KEYS) are cut into, by the lengths as they are and not as the host knows them, without a number for a block or a part that is not there.
// Blocks are numbered by lane, then by sequence of the lane.
// FIT: no more parts than slots, which are at least twice the blocks.
template <int BM, int KEYS, int S, bool FIT>
struct Layout {
  int q0[S], len_q[S], k0[S], len_k[S], blocks[S], parts[S];
  int blocks_upto, units_upto;  // of the lanes up to and including this one
  int n_blocks, n_units;        // in all
  int part_tiles;

  // slots: workgroups that run at once.  A part is what makes about as many parts as there are slots (with many blocks, four for every
  // block), each block's last one half full; 4 tiles at least.
  __device__ __forceinline__ void read(const PackedRows& p, int n_kv, int slots, int max_parts) {
    const int lane = threadIdx.x & 63;
    int begin[S], stop[S];
#pragma unroll
    for (int i = 0; i < S; ++i) {
      const int b = lane + 64 * i < p.batch ? lane + 64 * i : p.batch - 1;
      q0[i] = p.q_off[b];
      len_q[i] = p.q_off[b + 1];
      begin[i] = p.k_begin[b];
      stop[i] = p.k_end[b];
    }
    auto within = [](int v, int end) __attribute__((always_inline)) { return v < 0 ? 0 : v > end ? end : v; };
    float work = 0.f;
    int own_blocks = 0;
#pragma unroll
    for (int i = 0; i < S; ++i) {
      q0[i] = within(q0[i], p.total_q);
      const int n = within(len_q[i], p.total_q) - q0[i];
      len_q[i] = lane + 64 * i < p.batch && n > 0 ? n : 0;
      k0[i] = within(begin[i], p.k_rows);
      const int m = within(stop[i], p.k_rows) - k0[i];
      len_k[i] = m > 0 ? m : 0;
      blocks[i] = (int)((unsigned)(len_q[i] * p.group + BM - 1) / BM);
      own_blocks += blocks[i];
      work += (float)blocks[i] * (float)((unsigned)len_k[i] / KEYS + 1);
    }
    blocks_upto = wave_prefix_sum(own_blocks);
    n_blocks = __builtin_amdgcn_readlane(blocks_upto, 63);
    part_tiles = 1 << 30;
    if (max_parts > 1) {
      // (cut into parts of P tiles, n blocks make less than their tiles / P + n parts)
      const float pairs = (float)n_blocks * (float)n_kv, wanted = FIT || pairs <= 0.5f * (float)slots ? (float)slots : 4.f * pairs;
      part_tiles = (int)(wave_sum(work) * (float)n_kv / (wanted - (FIT ? 1.f : 0.5f) * pairs)) + 1;
      part_tiles = __builtin_amdgcn_readfirstlane(part_tiles < 4 ? 4 : part_tiles);
    }
    int own_units = 0;
#pragma unroll
    for (int i = 0; i < S; ++i) {
      const int tiles = (int)(((unsigned)len_k[i] + KEYS - 1) / KEYS);
      const int n = (tiles + part_tiles - 1) / part_tiles;
      parts[i] = n < 1 ? 1 : n < max_parts ? n : max_parts;
      own_units += blocks[i] * parts[i];
    }
    units_upto = wave_prefix_sum(own_units);
    n_units = __builtin_amdgcn_readlane(units_upto, 63);
  }

  // Parts of a block that sees `tiles` only, of the n_parts that its sequence's keys would make
  __device__ __forceinline__ int needed(int tiles, int n_parts) const {
    const int n = (int)((unsigned)(tiles + part_tiles - 1) / (unsigned)part_tiles);
    return n < 1 ? 1 : n < n_parts ? n : n_parts;
  }
  // Place of block `local` of sequence i of lane l
  __device__ __forceinline__ void place(const PackedRows& p, int l, int i, int local, Place& at, int& n_parts) const {
#pragma unroll
    for (int j = 0; j < S; ++j)
      if (j == i) {
        at.q0 = __builtin_amdgcn_readlane(q0[j], l);
        at.k0 = __builtin_amdgcn_readlane(k0[j], l);
        at.len_k = __builtin_amdgcn_readlane(len_k[j], l);
        const int len = __builtin_amdgcn_readlane(len_q[j], l), rows = len * p.group - local * BM;
        at.shift = at.len_k - len;
        at.row0 = local * BM;
        at.rows = rows < BM ? rows : BM;
        n_parts = __builtin_amdgcn_readlane(parts[j], l);
      }
  }
  // Unit u < n_units: its place, number of the block, part
  __device__ __forceinline__ void unit(const PackedRows& p, int u, Place& at, int& block, int& part, int& n_parts) const {
    const int l = __builtin_ctzll(__ballot(units_upto > u));
    int own = 0, b = 0;
#pragma unroll
    for (int i = 0; i < S; ++i) {
      own += blocks[i] * parts[i];
      b += blocks[i];
    }
    u -= __builtin_amdgcn_readlane(units_upto - own, l);
    block = __builtin_amdgcn_readlane(blocks_upto - b, l);
    int i = 0, local = 0;
#pragma unroll
    for (int j = 0; j < S; ++j) {
      const int here = __builtin_amdgcn_readlane(blocks[j], l), cut = __builtin_amdgcn_readlane(parts[j], l);
      if (i == j) {
        if (u >= here * cut && j + 1 < S) {
          u -= here * cut;
          block += here;
          i = j + 1;
        } else {
          local = u / cut;
          part = u - local * cut;
        }
      }
    }
    block += local;
    place(p, l, i, local, at, n_parts);
  }
  // Block c < n_blocks
  __device__ __forceinline__ void block(const PackedRows& p, int c, Place& at, int& n_parts) const {
    const int l = __builtin_ctzll(__ballot(blocks_upto > c));
    int b = 0;
#pragma unroll
    for (int i = 0; i < S; ++i) b += blocks[i];
    c -= __builtin_amdgcn_readlane(blocks_upto - b, l);
    int i = 0;
#pragma unroll
    for (int j = 0; j < S; ++j) {
      const int here = __builtin_amdgcn_readlane(blocks[j], l);
      if (i == j && c >= here && j + 1 < S) {
        c -= here;
        i = j + 1;
      }
    }
    place(p, l, i, c, at, n_parts);
  }
};

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
