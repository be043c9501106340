// Which keys a token sees and how attention over packed sequences is cut, as plain arithmetic: no HIP here, so that both
// can be evaluated over their whole range without a GPU.
#pragma once

namespace dare {

// j / d for 0 <= j < 2^31 by a product: with 2^(L - 1) < d <= 2^L and mul = ceil(2^(31 + L) / d), which is below 2^32, j mul / 2^(31 +
// L) lies above j / d by less than j 2^L / (d 2^(31 + L)) < 1 / d.  (An exact division takes 40 instructions of a wave that has
// nothing else to do yet.)
struct Divider {
  unsigned mul;
  int shift;
};
constexpr Divider divider(unsigned d) {
  int log = 0;
  while ((1ull << log) < d) ++log;
  return {(unsigned)(((1ull << (31 + log)) + d - 1) / d), 31 + log};
}
constexpr __attribute__((always_inline)) int divide(int j, Divider by) {
  return (int)(((unsigned long long)(unsigned)j * by.mul) >> by.shift);
}

// Keys that token i of a sequence sees: a prefix of its len_k keys.  shift = len_k - len_q: the queries are the last
// positions.  block 0: all; else up to the end of the token's block of that many positions.  A token in front of the
// first key (negative position) sees none.
constexpr __attribute__((always_inline)) int packed_limit(int i, int shift, int len_k, int block, Divider by_block) {
  if (block == 0) return len_k;
  const int pos = i + shift;
  if (pos < 0) return 0;
  const unsigned end = ((unsigned)divide(pos, by_block) + 1u) * (unsigned)block;  // (at most pos + block < 2^32)
  return end < (unsigned)len_k ? (int)end : len_k;
}

// Partial results of a block of `rows` rows: sums [rows][head_dim], references [rows], sums of probabilities [rows]
constexpr long packed_slot_floats(int head_dim, int rows) { return (long)rows * (head_dim + 2); }

constexpr int kPackedMaxParts = 64;

struct PackedPlan {
  int rows;       // rows of a block
  int blocks;     // blocks launched (of every key head)
  int parts;      // parts of a block's keys, at most
  int part_keys;  // keys of a part, at least
};

constexpr PackedPlan packed_plan(int batch, int total_q, int max_q, int max_k, int group, int n_kv) {
  PackedPlan plan{};
  plan.rows = (long)max_q * group <= 16 ? 16 : (long)max_q * group <= 32 ? 32 : 128;
  plan.blocks = (int)((long)total_q * group / plan.rows) + batch;
  plan.parts = 1;
  plan.part_keys = 1 << 30;
  // Few rows: parts of 128 keys and more (Layout in attn_packed_rows.h takes what it needs of them), where there are 512 keys to cut
  // (8 sequences of 300 keys uncut 10.6 us, in two parts 12.0), and fewer where 16 rounds of workgroups even out by themselves.  For
  // more than 256 sequences, whose lengths a workgroup does not look through, parts of 512.
  // Many rows, whose partial results are bytes that count: as many parts as give every CU two workgroups, or, up to four, four, because
  // sequences differ and masked rows see less (with equal parts: 32 tokens each over 32 caches of 100 to 4000 keys 98 us with two,
  // 79 with four, 2000 causal ones 45 and 41, but 64 over 60000 keys 96 with 32 parts and 120 with 64; 62, 38 and 96 since the parts
  // follow the lengths, Layout); of 512 keys, or 256 where there are CUs to spare (32 tokens over 4000 keys 20.5 and 17.3, over
  // 16 caches of 256 to 2048 36 and 43).
  // (pairs: blocks that hold rows, about: at least what the rows fill, at least one of every sequence)
  const long filled = (long)total_q * group / plan.rows, some = batch < total_q ? batch : total_q;
  const long pairs = (filled > some ? filled : some > 0 ? some : 1) * n_kv;
  long room = 8192 / pairs;
  if (plan.rows == 128) room = 512 / pairs >= 4 ? 512 / pairs : 1024 / pairs < 4 ? 1024 / pairs : 4;
  const long even = max_k * pairs / 512;
  long parts = max_k / (plan.rows < 128 || even > 512 ? 512 : even > 256 ? even : 256);
  if (plan.rows < 128 && batch <= 256 && parts > 0) parts = max_k / 128;
  if (parts > room) parts = room;
  // (a slot of the workspace for every part of every block that there can be: 270 MB at most)
  const long slots = (plan.rows == 128 ? 4096 : 16384) / ((long)plan.blocks * n_kv + 1);
  if (parts > slots) parts = slots;
  if (parts > kPackedMaxParts) parts = kPackedMaxParts;
  if (parts > 1) {
    plan.parts = (int)parts;
    plan.part_keys = (int)((max_k + parts - 1) / parts + 63) / 64 * 64;
  }
  return plan;
}

}  // namespace dare
