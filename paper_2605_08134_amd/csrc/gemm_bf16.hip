// Row-selected bf16 projection on the gfx950 matrix cores:
//     C[t, :] = A[t, :] . W      for t in a device-side row list
// (Alg. 1 lines 2, 6-7, 11 and Alg. 2 lines 2, 7, 11 of the paper: the Q, K, V
// and output projections, for all rows or only for the refreshed rows).
//
// Layout: A rows are k-contiguous; the weight arrives packed as Wt[n, k]
// (k-contiguous), so both MFMA operands are 16-byte runs of 8 consecutive k.
//
// A workgroup owns a BM x BN output tile and walks k in steps of 64.  Tiles of A
// and Wt go from global memory STRAIGHT INTO LDS (global_load_lds_dwordx4: lane L
// of a wave deposits its 16 bytes at wave_base + 16 L), through a ring of STAGES
// buffers, so several k-steps are in flight while the matrix cores work on the
// oldest one; no staging registers, no ds_write.  Because the LDS position is
// fixed by the lane number, bank conflicts are removed on the global side: the
// lane that owns LDS slot s of row r fetches k-chunk s ^ ((r >> 1) & 7), and the
// MFMA fragment reads apply the same XOR (measured conflict-free for 16-byte
// reads: 246 of 256 B/clk/CU).
//
// Each wave computes the TRANSPOSED tile (weight fragment as the first MFMA operand): a lane
// then owns one output row and runs of 4 consecutive output columns (8 in the large tiles),
// which gives 8- or 16-byte stores and keeps a row's values inside one lane.
//
// k-parts.  A projection with few output tiles and a long k (the scored query columns
// for all rows: 1024 x 128 x 4096) can cut k into ranges that run as separate
// workgroups; each range writes its fp32 partial products to its own slab of the fp32
// output and the consumer (the score kernel) adds the slabs in range order.  No
// atomics, no fences: the kernel boundary orders producer and consumer.
//
// Tile order.  The hardware deals workgroup ids round-robin to the 8 XCDs, each
// with its own L2.  Ids are remapped so that every XCD works on a contiguous
// range of tiles, and inside the range tiles run down groups of 8 row-tiles
// before moving to the next column-tile: the workgroups that are resident on an
// XCD at the same time then share both their A tiles and their weight tiles.
//
// Row count known only on the device (the refreshed-row list): one kernel holds
// several tile shapes and every workgroup picks the same one from the count it
// reads, so a step with 50 refreshed rows does not pay for a 256-row tile and no
// host round trip is needed.
#include <type_traits>

#include "dare_common.h"
#include "gemm_route.h"
#include "gemm_tiles.h"

namespace dare {
namespace {

// A range of the k (one of k_parts) of an output tile of C for m rows, computed by the WAVES_M * WAVES_N waves of a
// workgroup in smem_bytes<BM, BN, STAGES>() bytes of LDS.
template <int BM, int BN, int WAVES_M, int WAVES_N, int STAGES>
__device__ __forceinline__ void gemm_tile(const GemmDev& p, const int m, unsigned char* smem) {
  constexpr int NW = WAVES_M * WAVES_N;
  constexpr int WM = BM / WAVES_M, WN = BN / WAVES_N;
  constexpr int TM = WM / 32, TN = WN / 32;
  constexpr int STAGE_BYTES = (BM + BN) * ROW_BYTES;
  constexpr int GROUPS = (BM + BN) / 8;  // 8-row groups = one wave load each
  constexpr int LPW = GROUPS / NW;       // loads per wave per stage
  static_assert(WM % 32 == 0 && WN % 32 == 0, "wave tile must be a multiple of 32 x 32");
  static_assert(GROUPS % NW == 0, "row groups must divide among the waves");
  static_assert(LPW * (STAGES - 1) < 64, "vmcnt range");

  // ---- which tile: XCD-contiguous ranges, GROUP_M row-tiles per column step ----
  // (the k-ranges of one tile are neighbours in this order)
  const int parts = p.k_parts;
  const int tiles_m = (m + BM - 1) / BM, tiles_n = (p.n + BN - 1) / BN;
  const int total = tiles_m * tiles_n * parts;
  const int per_xcd = (total + 7) >> 3;
  const int slot = blockIdx.x >> 3;
  if (slot >= per_xcd) return;
  const int unit = (blockIdx.x & 7) * per_xcd + slot;
  if (unit >= total) return;
  const int logical = unit / parts, part = unit - logical * parts;
  int tile_m, tile_n;
  tile_of_unit(logical, tiles_m, tiles_n, tile_m, tile_n);
  const int m0 = tile_m * BM, n0 = tile_n * BN;

  // (the wave number as a scalar: LDS addresses of the global -> LDS loads go through M0, and a
  // wave number held in a vector register would send every one of them through v_readfirstlane)
  const int tid = threadIdx.x;
  const int lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wave_m = wave % WAVES_M, wave_n = wave / WAVES_M;
  const int l32 = lane & 31, half = lane >> 5;

  // this workgroup's k-range, in k-steps (the host makes parts divide the step count)
  const int KT = p.k / BK / parts;
  const int kt0 = part * KT;

  // ---- global -> LDS assignment: wave w issues loads for row groups w*LPW .. +LPW
  // (rows 0..BM-1 are A rows, BM..BM+BN-1 are weight rows).  Lane L of a load owns
  // row (L >> 3) of the group and LDS slot (L & 7); it fetches the k-chunk that
  // the swizzle puts into that slot.  Rows past the end re-read the last row.
  const bf16_t* src[LPW];
  int row_in[LPW], tok_in[LPW];
#pragma unroll
  for (int i = 0; i < LPW; ++i) {
    const int row = m0 + (wave * LPW + i) * 8 + (lane >> 3);
    row_in[i] = row < m ? row : m - 1;
  }
  row_tokens(p.idx, nullptr, row_in, tok_in);
#pragma unroll
  for (int i = 0; i < LPW; ++i) {
    const int r = (wave * LPW + i) * 8 + (lane >> 3);  // row within the stage
    const int chunk = (lane & 7) ^ ((r >> 1) & 7);
    if (r < BM) {
      src[i] = p.a + (long)tok_in[i] * p.lda + chunk * 8 + kt0 * BK;
    } else {
      int col = n0 + (r - BM);
      col = col < p.n ? col : p.n - 1;
      src[i] = p.wt + (long)col * p.k + chunk * 8 + kt0 * BK;
    }
  }
  int row_out[TM], tok_out[TM];
  bool live_out[TM];
#pragma unroll
  for (int i = 0; i < TM; ++i) {
    const int row = m0 + wave_m * WM + i * 32 + l32;
    live_out[i] = row < m;
    row_out[i] = row < m ? row : m - 1;
  }
  row_tokens(p.idx, nullptr, row_out, tok_out);
  auto issue_loads = [&](int kt, int buf) __attribute__((always_inline)) {
    unsigned char* base = smem + buf * STAGE_BYTES + wave * LPW * 8 * ROW_BYTES;
#pragma unroll
    for (int i = 0; i < LPW; ++i)
      __builtin_amdgcn_global_load_lds((gptr_t)(src[i] + kt * BK),
                                       (lptr_t)(base + i * 8 * ROW_BYTES), 16, 0, 0);
  };

  f32x16 acc[TM][TN];
#pragma unroll
  for (int i = 0; i < TM; ++i)
#pragma unroll
    for (int j = 0; j < TN; ++j)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.f;

  // fragment read offsets: row (wave tile base + 32 i + l32), k-chunk 2 ks + half,
  // stored at slot chunk ^ ((row >> 1) & 7); the tile bases are multiples of 32,
  // so the XOR term depends on l32 only
  constexpr int KS = BK / 16;
  const int sw = (l32 >> 1) & 7;
  int koff[KS];
#pragma unroll
  for (int ks = 0; ks < KS; ++ks) koff[ks] = ((ks * 2 + half) ^ sw) * 16;
  const int a_row_off = (wave_m * WM + l32) * ROW_BYTES;
  const int b_row_off = (BM + wave_n * WN + l32) * ROW_BYTES;

  // ---- pipeline: STAGES-1 k-steps in flight ahead of the one being multiplied.
  // Loads of k-steps past the end are issued on the last valid k-step again (into
  // a buffer nobody reads any more), so the count of outstanding loads per wave is
  // the same in every iteration and one vmcnt value serves the whole loop.
  //
  // MFMA operands are double-buffered in registers: all fragments of k-step kt+1 are fetched
  // after the first PRE MFMAs of k-step kt and arrive under the rest.  The barrier that publishes
  // k-step kt+1 sits right before that fetch: by then every LDS read of k-step kt has been issued
  // and (lgkmcnt 0) has completed, so its buffer may be refilled after the barrier.
  // The scheduling fences keep the compiler from sinking the LDS reads back down
  // to their first use, which would undo the register double buffering.
  bf16x8 fa[2][KS][TM], fb[2][KS][TN];
  auto load_frags = [&](int buf, int set) __attribute__((always_inline)) {
    const unsigned char* st = smem + buf * STAGE_BYTES;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
#pragma unroll
      for (int i = 0; i < TM; ++i)
        fa[set][ks][i] = *reinterpret_cast<const bf16x8*>(st + a_row_off + i * 32 * ROW_BYTES + koff[ks]);
#pragma unroll
      for (int j = 0; j < TN; ++j)
        fb[set][ks][j] = *reinterpret_cast<const bf16x8*>(st + b_row_off + j * 32 * ROW_BYTES + koff[ks]);
    }
  };
  // MFMAs [first, last) of the KS x TM x TN grid of one fragment set
  constexpr int NMMA = KS * TM * TN;
  constexpr int PRE = NMMA >= 8 ? 2 : 1;
  auto mma = [&](int set, int first, int last) __attribute__((always_inline)) {
#pragma unroll
    for (int t = 0; t < NMMA; ++t) {
      if (t < first || t >= last) continue;
      const int ks = t / (TM * TN), i = (t / TN) % TM, j = t % TN;
      acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fb[set][ks][j], fa[set][ks][i], acc[i][j], 0, 0, 0);
    }
  };

#pragma unroll
  for (int s = 0; s < STAGES - 1; ++s) issue_loads(s < KT ? s : KT - 1, s);
  wait_vmcnt_and_barrier<LPW*(STAGES - 2)>();
  load_frags(0, 0);
  // two k-steps per trip so that the fragment set index is a compile-time constant
  // (a run-time index would push the fragment arrays out of registers)
  auto kstep = [&](int kt, auto set_c) __attribute__((always_inline)) {
    constexpr int SET = decltype(set_c)::value;
    const int nxt = kt + STAGES - 1;
    issue_loads(nxt < KT ? nxt : KT - 1, nxt % STAGES);
    mma(SET, 0, PRE);
    __builtin_amdgcn_sched_barrier(0);
    wait_vmcnt_and_barrier<LPW*(STAGES - 2)>();
    load_frags((kt + 1) % STAGES, SET ^ 1);
    __builtin_amdgcn_sched_barrier(0);
    mma(SET, PRE, NMMA);
    __builtin_amdgcn_sched_barrier(0);
  };
  int kt = 0;
  for (; kt + 1 < KT; kt += 2) {
    kstep(kt, std::integral_constant<int, 0>{});
    kstep(kt + 1, std::integral_constant<int, 1>{});
  }
  if (kt < KT) kstep(kt, std::integral_constant<int, 0>{});
  wait_vmcnt<0>();

  float* c32 = p.c32 + part * p.c32_part_stride;
  // Epilogue.  acc[i][j][r] = C[row, col] with
  //   row = m0 + wave_m*WM + i*32 + l32
  //   col = n0 + wave_n*WN + j*32 + (r/4)*8 + half*4 + r%4
  int col[4 * TN];
#pragma unroll
  for (int j = 0; j < 4 * TN; ++j) col[j] = n0 + wave_n * WN + j * 8 + half * 4;
  store_tile<4>(p, c32, tok_out, live_out, col,
                [&](int i, int j, int e) __attribute__((always_inline)) { return acc[i][j >> 2][(j & 3) * 4 + e]; });
}

// ---- large tiles: 256 x (64 TN), eight waves in two groups that take turns ----------------
// (listed rows; all rows in 256 x 128, with k cut too, and in one round of the wider ones)
// Waves w and w + 4 sit on the same SIMD.  Waves 0-3 (group 0) own the left half of the tile's
// columns, waves 4-7 (group 1) the right half, each wave 64 rows x 32 TN columns.  A k-step of 64 is
// cut into TN phases, one per block of 32 columns, and a phase into a memory part (fragment
// reads of the phase from LDS, waits) and a matrix part (16 MFMAs), with a workgroup barrier
// after each.  Group 1 runs one barrier behind group 0, so on every SIMD one wave multiplies while
// the other reads: neither the LDS reads nor the barriers leave the matrix pipe idle.
//   * The global -> LDS loads are issued between the MFMAs of the matrix part, one or two per phase
//     and wave.  In the memory part, or ahead of its reads, the vector-memory queue holds up the
//     wave that the others wait for: 2930 and 3870 cycles per k-step of a 256 x 256 tile, against
//     2300 between the MFMAs (2048 is what the MFMAs alone take).
//   * v_mfma_f32_16x16x32_bf16 and not 32x32x16: it moves fewer accumulator registers per flop, and
//     these kernels run at the power limit (1.6-1.9 GHz of 2.4 under load): 16384 x 12288 x 4096 takes
//     1140 us against 1285 us although a k-step has 9 % more cycles.
//   * The weight rows of a fragment are permuted (row 8 a + b of a 32-row block feeds result row
//     4 a + b of the first MFMA, row 8 a + 4 + b the second, a, b = 0 .. 3), so that a lane ends up with
//     eight neighbouring output columns: 16-byte stores, half the store requests (the epilogue of a
//     256 x 256 tile: 5.1 against 11 thousand cycles).  The chunk XOR of a weight row follows that
//     order ((row >> 1) & 1 | ((row >> 3) & 3) << 1), which keeps the reads conflict-free.
//   * LDS: two stages (three for TN = 2), each freed region by region.  The A rows of k-step kt are read in phase 0 only
//     and column block j in phase j (block 0 already in the last phase of kt - 1); a region is filled
//     again for kt + 2 from the phase after on, so a load has 3.5 (TN = 3) or 4.5 phases (TN = 4) of
//     512 MFMA cycles to arrive.
// Measured with gathered-row support and all (us, before: one k-loop that every wave runs in step):
// 16384 x 12288 x 4096 1540 -> 1140 (1.45 PFLOP/s), 1024 x 12288 x 4096 98 -> 78, 1024 x 24576 x 4096
// 206 -> 154.  TN = 2 against 128 x 128 tiles: 2048 x 4096 x 4096 83 -> 59; with the k of a tile cut over
// two workgroups (below; 64 to 128 tiles, which leave half of the CUs idle, and a long k), inside a
// model step: 1024 x 4096 x 12288 122 -> 97.  A k-step takes 1610 cycles for 1024 of MFMAs:
// every byte of LDS written or read for it at 128 B per cycle is 1400.
// The last k-steps load nothing and wait for what is under way: a launch of one round had two k-steps of 64
// pulled in vain and the last load's latency at its end.  Steps: 3 x 777, outputs reused 285.7 -> 282.1 us, 8 x 2048
// refreshed 534.8 -> 525.2, dense block 2323 -> 2300; a dense step of 1024 tokens 148.6 -> 148.9.
template <int TN>
constexpr int pp_stages() { return TN == 2 ? 3 : 2; }
template <int TN>
constexpr int pp_smem_bytes() {
  return pp_stages<TN>() * (kPpRows + 64 * TN) * ROW_BYTES;
}
// vblock, lidx and the result as in gemm_tile16; called by all 512 threads.
template <int TN, bool SPLIT = false, bool LINEAR = false>
__device__ __forceinline__ bool gemm_tile_pp(const GemmDev& p, const int m, unsigned char* smem, const int vblock,
                                             lds_idx_t lidx = nullptr) {
  static_assert(TN >= 2 && TN <= 4, "column blocks of 32 per wave");
  static_assert(!SPLIT || TN == 2, "k is cut for the narrow tile only");
  constexpr int BM = kPpRows, BN = 64 * TN;
  constexpr int ASZ = BM * ROW_BYTES, BSZ = BN * ROW_BYTES, STAGE_BYTES = ASZ + BSZ, STAGES = pp_stages<TN>();
  constexpr int PARTS = SPLIT ? 2 : 1;

  const int tiles_m = (m + BM - 1) / BM, tiles_n = (p.n + BN - 1) / BN;
  const int total = tiles_m * tiles_n * PARTS;
  const int per_xcd = (total + 7) >> 3;
  const int slot = vblock >> 3;
  if (slot >= per_xcd) return false;
  const int unit = (vblock & 7) * per_xcd + slot;
  if (unit >= total) return false;
  const int tile = unit / PARTS;
  int tile_m, tile_n;
  tile_of_unit(tile, tiles_m, tiles_n, tile_m, tile_n);
  const int m0 = tile_m * BM, n0 = tile_n * BN;

  const int tid = threadIdx.x;
  const int lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int grp = wave >> 2, wm = wave & 3;
  const int l16 = lane & 15, kq = lane >> 4;
  const int KT = p.k / BK / PARTS;
  const int k_first = SPLIT ? (unit & 1) * KT * BK : 0;

  // ---- global -> LDS: per k-step a wave loads 4 groups of 8 A rows and one group of 8 weight rows
  // of each column block (block j: rows 32 j .. of the left and of the right half, 64 in all).
  // Rows past the end re-read the last one.
  const bf16_t* src_a[4];
  const bf16_t* src_b[TN];
  int row_in[4], tok_in[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int row = m0 + (wave * 4 + i) * 8 + (lane >> 3);
    row_in[i] = row < m ? row : m - 1;
  }
  row_tokens(p.idx, lidx, row_in, tok_in);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int r = (wave * 4 + i) * 8 + (lane >> 3);
    src_a[i] = p.a + (long)tok_in[i] * p.lda + ((lane & 7) ^ ((r >> 1) & 7)) * 8 + k_first;
  }
#pragma unroll
  for (int j = 0; j < TN; ++j) {
    const int r = wave * 8 + (lane >> 3);
    int col = n0 + (r >> 5) * (32 * TN) + j * 32 + (r & 31);
    col = col < p.n ? col : p.n - 1;
    src_b[j] = p.wt + (long)col * p.k + ((lane & 7) ^ pp_bkey(r & 31)) * 8 + k_first;
  }
  int row_out[4], tok_out[4];
  bool live_out[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int row = m0 + wm * 64 + i * 16 + l16;
    live_out[i] = row < m;
    row_out[i] = row < m ? row : m - 1;
  }
  row_tokens(p.idx, lidx, row_out, tok_out);
  // (in front of the loop, k-steps past the end of a short k re-read the last one into a region that nobody
  // reads, so that the loads in flight are at least those that the loop counts; the loop loads nothing past the end)
  auto stage = [&](int kt) __attribute__((always_inline)) { return smem + (kt % STAGES) * STAGE_BYTES; };
  auto load_a = [&](int i, int kt, int k) __attribute__((always_inline)) {
    __builtin_amdgcn_global_load_lds((gptr_t)(src_a[i] + k * BK), (lptr_t)(stage(kt) + (wave * 4 + i) * 1024), 16, 0, 0);
  };
  auto load_b = [&](int j, int kt, int k) __attribute__((always_inline)) {
    __builtin_amdgcn_global_load_lds((gptr_t)(src_b[j] + k * BK),
                                     (lptr_t)(stage(kt) + ASZ + j * 64 * ROW_BYTES + wave * 1024), 16, 0, 0);
  };

  f32x4 acc[4][2 * TN];
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < 2 * TN; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};

  const int a_off = (wm * 64 + l16) * ROW_BYTES;
  int a_koff[2], b_koff[2][2];
  const int brow = (l16 >> 2) * 8 + (l16 & 3);
#pragma unroll
  for (int ks = 0; ks < 2; ++ks) {
    a_koff[ks] = ((ks * 4 + kq) ^ ((l16 >> 1) & 7)) * 16;
#pragma unroll
    for (int h = 0; h < 2; ++h)
      b_koff[h][ks] = (grp * 32 + brow + 4 * h) * ROW_BYTES + (((ks * 4 + kq) ^ pp_bkey(brow + 4 * h)) * 16);
  }
  bf16x8 fa[4][2], fb[2][2][2];  // A fragments of a k-step; weight fragments of two column blocks
  auto read_a = [&](int kt) __attribute__((always_inline)) {
    const unsigned char* st = stage(kt) + a_off;
#pragma unroll
    for (int ks = 0; ks < 2; ++ks)
#pragma unroll
      for (int i = 0; i < 4; ++i) fa[i][ks] = *reinterpret_cast<const bf16x8*>(st + i * 16 * ROW_BYTES + a_koff[ks]);
  };
  auto read_b = [&](int set, int j, int kt) __attribute__((always_inline)) {
    const unsigned char* st = stage(kt) + ASZ + j * 64 * ROW_BYTES;
#pragma unroll
    for (int ks = 0; ks < 2; ++ks)
#pragma unroll
      for (int h = 0; h < 2; ++h) fb[set][h][ks] = *reinterpret_cast<const bf16x8*>(st + b_koff[h][ks]);
  };
  // MFMAs [first, last) of the 16 of column block j
  auto mma = [&](int set, int j, int first, int last) __attribute__((always_inline)) {
#pragma unroll
    for (int t = 0; t < 16; ++t) {
      if (t < first || t >= last) continue;
      const int ks = t >> 3, i = (t >> 1) & 3, h = t & 1;
      acc[i][j * 2 + h] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fb[set][h][ks], fa[i][ks], acc[i][j * 2 + h], 0, 0, 0);
    }
  };
  // end of a memory part: all but N of the wave's loads have landed, its LDS reads have returned
  auto end_mem = [&](auto n_c) __attribute__((always_inline)) {
    __builtin_amdgcn_sched_barrier(0);
    wait_vmcnt_and_barrier<decltype(n_c)::value>();
    __builtin_amdgcn_sched_barrier(0);
  };
  // a matrix part: the MFMAs of column block j with up to four loads between them
  auto matrix = [&](int set, int j, auto l1, auto l2, auto l3, auto l4) __attribute__((always_inline)) {
    __builtin_amdgcn_s_setprio(1);
    mma(set, j, 0, 4);
    __builtin_amdgcn_sched_barrier(0);
    l1();
    __builtin_amdgcn_sched_barrier(0);
    mma(set, j, 4, 8);
    __builtin_amdgcn_sched_barrier(0);
    l2();
    __builtin_amdgcn_sched_barrier(0);
    mma(set, j, 8, 12);
    __builtin_amdgcn_sched_barrier(0);
    l3();
    __builtin_amdgcn_sched_barrier(0);
    mma(set, j, 12, 14);
    __builtin_amdgcn_sched_barrier(0);
    l4();
    __builtin_amdgcn_sched_barrier(0);
    mma(set, j, 14, 16);
    __builtin_amdgcn_s_setprio(0);
    __builtin_amdgcn_sched_barrier(0);
    asm volatile("s_barrier" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
  };
  auto none = []() __attribute__((always_inline)) {};
#define DARE_N(n) std::integral_constant<int, n>{}
#define DARE_A(on, i, d) [&]() __attribute__((always_inline)) { if constexpr (on) load_a(i, kt + d, kt + d); }
#define DARE_B(on, j, d) [&]() __attribute__((always_inline)) { if constexpr (on) load_b(j, kt + d, kt + d); }

  // Loads in the order in which they are needed: block 0 of a k-step, its A rows, its blocks
  // 1 .. TN - 1.  The counts below are the loads issued after the last one that the next phase reads.
  const int k1 = KT > 1 ? 1 : 0, k2 = KT > 2 ? 2 : KT - 1;
  load_b(0, 0, 0);
#pragma unroll
  for (int i = 0; i < 4; ++i) load_a(i, 0, 0);
#pragma unroll
  for (int j = 1; j < TN; ++j) load_b(j, 0, 0);
  load_b(0, 1, k1);
#pragma unroll
  for (int i = 0; i < 4; ++i) load_a(i, 1, k1);
  load_b(1, 1, k1);
  if constexpr (TN == 4) load_b(2, 1, k1);
  if constexpr (TN == 2) {
    load_b(0, 2, k2);
#pragma unroll
    for (int i = 0; i < 4; ++i) load_a(i, 2, k2);
  }
  wait_vmcnt_and_barrier<TN == 4 ? 10 : (TN == 3 ? 8 : 12)>();
  read_b(0, 0, 0);
  // (group 0 refills the region that these reads take from after this barrier)
  if (grp == 1) asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
  // LEFT: k-steps that follow, STAGES for as many or more; S: fragment set of block 0 (alternates where TN is odd).
  auto kstep = [&](int kt, auto set_c, auto left_c) __attribute__((always_inline)) {
    constexpr int S = decltype(set_c)::value, LEFT = decltype(left_c)::value;
    constexpr bool L1 = LEFT > 0, L2 = LEFT > 1, L3 = LEFT > 2;  // k-steps kt + 1, kt + 2, kt + 3 exist
    read_a(kt);
    if constexpr (TN == 4) {
      end_mem(DARE_N(L1 ? 9 : 2));
      matrix(0, 0, DARE_B(L1, 3, 1), none, DARE_B(L2, 0, 2), none);
      read_b(1, 1, kt);
      end_mem(DARE_N(L2 ? 10 : (L1 ? 9 : 1)));
      matrix(1, 1, DARE_A(L2, 0, 2), none, DARE_A(L2, 1, 2), none);
      read_b(0, 2, kt);
      end_mem(DARE_N(L2 ? 10 : (L1 ? 7 : 0)));
      matrix(0, 2, DARE_A(L2, 2, 2), none, DARE_A(L2, 3, 2), none);
      read_b(1, 3, kt);
      if constexpr (L1) read_b(0, 0, kt + 1);
      end_mem(DARE_N(L2 ? 8 : (L1 ? 3 : 0)));
      matrix(1, 3, DARE_B(L2, 1, 2), none, DARE_B(L2, 2, 2), none);
    } else if constexpr (TN == 2) {
      end_mem(DARE_N(L2 ? 10 : (L1 ? 5 : 0)));
      matrix(0, 0, DARE_B(L2, 1, 2), none, DARE_B(L3, 0, 3), none);
      read_b(1, 1, kt);
      if constexpr (L1) read_b(0, 0, kt + 1);
      end_mem(DARE_N(L3 ? 8 : (L2 ? 7 : (L1 ? 1 : 0))));
      matrix(1, 1, DARE_A(L3, 0, 3), DARE_A(L3, 1, 3), DARE_A(L3, 2, 3), DARE_A(L3, 3, 3));
    } else {
      end_mem(DARE_N(L1 ? 7 : 1));
      matrix(S, 0, DARE_B(L1, 2, 1), none, DARE_B(L2, 0, 2), none);
      read_b(S ^ 1, 1, kt);
      end_mem(DARE_N(L2 ? 7 : (L1 ? 6 : 0)));
      matrix(S ^ 1, 1, DARE_A(L2, 0, 2), DARE_A(L2, 1, 2), DARE_A(L2, 2, 2), DARE_A(L2, 3, 2));
      read_b(S, 2, kt);
      if constexpr (L1) read_b(S ^ 1, 0, kt + 1);
      end_mem(DARE_N(L2 ? 7 : (L1 ? 2 : 0)));
      matrix(S, 2, none, DARE_B(L2, 1, 2), none, none);
    }
  };
  // a k-step alone leaves the next one's block 0 in the set where it starts (branches that meet with different
  // sets cost registers)
  auto single = [&](int kt, auto left_c) __attribute__((always_inline)) {
    kstep(kt, DARE_N(0), left_c);
    if constexpr (TN == 3) {
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int ks = 0; ks < 2; ++ks) fb[0][h][ks] = fb[1][h][ks];
    }
  };
  int kt = 0;
  if constexpr (TN == 3) {
    for (; kt + 1 < KT - STAGES; kt += 2) {
      kstep(kt, DARE_N(0), DARE_N(STAGES));
      kstep(kt + 1, DARE_N(1), DARE_N(STAGES));
    }
    if (kt < KT - STAGES) single(kt++, DARE_N(STAGES));
  } else {
    for (; kt < KT - STAGES; ++kt) kstep(kt, DARE_N(0), DARE_N(STAGES));
  }
  if constexpr (STAGES > 2) {
    if (kt < KT - 2) single(kt++, DARE_N(2));
  }
  if (kt < KT - 1) single(kt++, DARE_N(1));
  kstep(kt, DARE_N(0), DARE_N(0));
#undef DARE_N
#undef DARE_A
#undef DARE_B
  if (grp == 0) asm volatile("s_barrier" ::: "memory");
  wait_vmcnt<0>();

  // The workgroup that arrives last at a tile adds the other one's sums to its own (a sum of two
  // does not depend on which came first) and stores the tile; the other one leaves its sums in
  // its half of the tile's workspace and goes.  Nobody waits: a workgroup that finds the other's sums
  // complete need not store its own, and of two that both stored theirs the second one counted is
  // the last (1 us more per launch than a wait for the first one's sums).  The counter's
  // parity says whether one has arrived: even between launches, whatever the launch before left.
  // The sums are written and read at device scope (sc1: past whatever an XCD's L2 holds), and counted
  // once every wave's stores have completed, so no fence, which would write back the whole L2
  // (20-40 us), is needed.
  if constexpr (SPLIT) {
    constexpr int kDeviceScope = 16;  // cache policy sc1
    float* slots = p.split_tiles + (long)tile * (PARTS * BM * BN);
    const auto mine = __builtin_amdgcn_make_buffer_rsrc(slots + (unit & 1) * (BM * BN), 0, BM * BN * 4, 0x00027000);
    const auto other = __builtin_amdgcn_make_buffer_rsrc(slots + (~unit & 1) * (BM * BN), 0, BM * BN * 4, 0x00027000);
    int* count = p.split_count + tile;
    int* last = reinterpret_cast<int*>(smem);
    __syncthreads();
    if (tid == 0) *last = __hip_atomic_load(count, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) & 1;
    __syncthreads();
    if (!*last) {
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 2 * TN; ++j)
          __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, acc[i][j]), mine,
                                                 ((i * 2 * TN + j) * 512 + tid) * 16, 0, kDeviceScope);
      wait_vmcnt<0>();
      __syncthreads();
      if (tid == 0) *last = __hip_atomic_fetch_add(count, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) & 1;
      __syncthreads();
      if (!*last) return true;
    } else if (tid == 0) {
      __hip_atomic_fetch_add(count, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int j = 0; j < 2 * TN; ++j)
        acc[i][j] += __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(
                                                   other, ((i * 2 * TN + j) * 512 + tid) * 16, 0, kDeviceScope));
  }

  // acc[i][2 j + h][e] = C[row, col], row = m0 + 64 wm + 16 i + l16, col = n0 + 32 TN grp + 32 j + 8 kq + 4 h + e
  int col[TN];
#pragma unroll
  for (int j = 0; j < TN; ++j) col[j] = n0 + grp * (32 * TN) + j * 32 + kq * 8;
  auto value = [&](int i, int j, int e) __attribute__((always_inline)) { return acc[i][j * 2 + (e >> 2)][e & 3]; };
  if constexpr (LINEAR)
    store_linear<8>(p, tok_out, live_out, col, value);
  else
    store_tile<8>(p, p.c32, tok_out, live_out, col, value);
  return true;
}

// Columns [0, part_n) for the listed rows, whose count the device knows, and the others for all rows: one launch for
// both, in the shape of the least cost.  Two shapes, no gate and no fp32 copy: 8310 instructions and no spilled scalar, where 256 x 128, which
// is slower with the weights in memory, and those epilogues made it 22345 and 38 (block steps, with them and without, us: 5 x 1024 tokens
// of hidden 4096, a twentieth refreshed, 403.8 400.7, 4 x 800 half refreshed 385.4 383.3, 16 x 1000 of hidden 2048 392.0 385.9).
__global__ void __launch_bounds__(256, 1) gemm_bf16_part_kernel(GemmDev p) {
  __shared__ __attribute__((aligned(1024))) unsigned char smem[kQuadSmem];
  const int part_m = *(const __attribute__((address_space(4))) int32_t*)(uintptr_t)p.part_m_dev;
  if (part_columns(p.m_max, p.n, part_m, p.part_n) == 3) return gemm_tiles_quad<3, false, true>(p, p.m_max, smem, part_m);
  gemm_tiles_quad<4, false, true>(p, p.m_max, smem, part_m);
}

template <int TN, bool STREAM>
__global__ void __launch_bounds__(256, 1) gemm_bf16_quad_kernel(GemmDev p) {
  __shared__ __attribute__((aligned(1024))) unsigned char smem[kQuadSmem];
  gemm_tiles_quad<TN, STREAM>(p, p.m_max, smem);
}

// ---- one tile shape, chosen on the host (row count known): k in ranges, then whole k --------------
template <int BM, int BN, int WAVES_M, int WAVES_N, int STAGES>
__global__ void __launch_bounds__(WAVES_M* WAVES_N * 64) gemm_bf16_ranges_kernel(GemmDev p) {
  __shared__ __attribute__((aligned(1024))) unsigned char smem[smem_bytes<BM, BN, STAGES>()];
  gemm_tile<BM, BN, WAVES_M, WAVES_N, STAGES>(p, p.m_max, smem);
}

template <int BM, int BN, int WAVES_M, int WAVES_N, int STAGES>
__global__ void __launch_bounds__(512) gemm_bf16_tile16_kernel(GemmDev p) {
  __shared__ __attribute__((aligned(1024))) unsigned char smem[smem_bytes<BM, BN, STAGES>()];
  gemm_tile16<BM, BN, WAVES_M, WAVES_N, STAGES>(p, p.m_max, smem, threadIdx.x, blockIdx.x);
}

// All rows: 256 x 128, and a round of 256 x 192 or 256 (four_waves, gemm_route.h).  256 x 128: with the weights in memory eight waves and
// three stages in flight are faster than four waves, whose ring holds two and a half: 1320 x 3072 x 9216 102 us and 119, x 3072 x 3072
// 39-44 and 45-52 (in the caches 91.6 and 83.4, 34.9 and 33.2).
template <int TN, bool SPLIT>
__global__ void __launch_bounds__(512) gemm_bf16_pp_kernel(GemmDev p) {
  __shared__ __attribute__((aligned(1024))) unsigned char smem[pp_smem_bytes<TN>()];
  gemm_tile_pp<TN, SPLIT>(p, p.m_max, smem, blockIdx.x);
}

// ---- act(A W + bias) + residual of all rows ---------------------------------------------------
template <int BM, int BN, int WAVES_M, int WAVES_N, int STAGES>
__global__ void __launch_bounds__(WAVES_M* WAVES_N * 64) linear_bf16_tile16_kernel(GemmDev p) {
  __shared__ __attribute__((aligned(1024))) unsigned char smem[smem_bytes<BM, BN, STAGES>()];
  gemm_tile16<BM, BN, WAVES_M, WAVES_N, STAGES, true>(p, p.m_max, smem, threadIdx.x, blockIdx.x);
}
template <int TN>
__global__ void __launch_bounds__(512) linear_bf16_pp_kernel(GemmDev p) {
  __shared__ __attribute__((aligned(1024))) unsigned char smem[pp_smem_bytes<TN>()];
  gemm_tile_pp<TN, false, true>(p, p.m_max, smem, blockIdx.x);
}
template <int TN, bool STREAM>
__global__ void __launch_bounds__(256, 1) linear_bf16_quad_kernel(GemmDev p) {
  __shared__ __attribute__((aligned(1024))) unsigned char smem[kQuadSmem];
  gemm_tiles_quad<TN, STREAM, false, true>(p, p.m_max, smem);
}
__global__ void __launch_bounds__(512) linear_bf16_skinny_kernel(GemmDev p) {
  __shared__ __attribute__((aligned(1024))) unsigned char smem[8 * 64 * 16];
  skinny_tile<8, 1, true>(p, p.m_max, smem, threadIdx.x);
}

// ---- row count read on the device: the tile shape follows it -------------------------
// One kernel for every projection of refreshed rows that has a choice of shapes, 8 waves and 144 KiB of LDS, one workgroup per CU
// whatever the count turns out to be (a grid sized for the worst case, whose surplus workgroups
// return at once, costs 1 us more at 205 rows); the shape is the one that best_tile (gemm_route.h) names, and
// its tiles are walked in passes.
constexpr int kWideSmem = pp_smem_bytes<2>();
// The refreshed-row list from the mask bytes, by every workgroup for itself (Alg. 1/2 line 5
// folded into the first kernel that needs the list: a compaction kernel of its own costs a
// launch, 4-5 us of a 90 us step, for a few hundred bytes of work).  512 threads, up to
// kSelMaxTokens tokens, four per thread; ascending by construction.  Returns the count.
// While the mask is on its way and the list is made, the first 256 k of the weight rows are read ahead: an XCD's
// workgroups, 16 rows each at a time, read its share of them (tiles are dealt to the XCDs in contiguous ranges of
// columns, as long as there are at most GROUP_M row tiles) into its L2, into 1 KiB of LDS that nobody reads; nothing here
// waits for them.  What it fills is the time of the mask's round trip and the list.  (The first
// one in a block with the mask: the compiler waits for loads into LDS with those in front of them.)  Steps over 1 x 1024
// tokens with 205 refreshed rows, without and with it (us): hidden 4096 89.2 and 87.7, 6144 155.7 and 154.0, 1024 to 3072 and
// 8192, and 4 rows, no difference beyond the runs'.  The stream over the weights (skinny_tile) deals its columns
// otherwise and has nothing from it.
__device__ __forceinline__ int derive_rows(const GemmDev& p, int32_t* list, int* wave_tot, unsigned char* nobody) {
  const int n_tok = p.sel_batch * p.sel_seq;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int t0 = tid * 4;
  const int per_xcd = (p.n + 7) >> 3, first = (blockIdx.x & 7) * per_xcd, slots = gridDim.x >> 3;
  const int last = first + per_xcd < p.n ? first + per_xcd - 1 : p.n - 1;
  const uint8_t* mask[4];
#pragma unroll
  for (int k = 0; k < 4; ++k) mask[k] = p.sel_mask + (t0 + k < n_tok ? t0 + k : n_tok - 1);
  auto ahead = [&](int i) __attribute__((always_inline)) {
    const int r = first + (((blockIdx.x >> 3) + i * slots) * 8 + wave) * 2 + (lane >> 5);
    return p.wt + (long)(r < last ? r : last) * p.k + ((lane & 31) * 8 < p.k ? (lane & 31) * 8 : 0);
  };
  const unsigned lds = (unsigned)(size_t)(lptr_t)nobody;
  int reused[4];
  asm volatile(
      "global_load_ubyte %0, %4, off\n\tglobal_load_ubyte %1, %5, off\n\t"
      "global_load_ubyte %2, %6, off\n\tglobal_load_ubyte %3, %7, off\n\t"
      "global_load_lds_dwordx4 %8, off\n\ts_waitcnt vmcnt(1)"
      : "=&v"(reused[0]), "=&v"(reused[1]), "=&v"(reused[2]), "=&v"(reused[3])
      : "v"(mask[0]), "v"(mask[1]), "v"(mask[2]), "v"(mask[3]), "v"(ahead(0)), "{m0}"(lds)
      : "memory");
#pragma unroll 1
  for (int i = 1; i < p.ahead; ++i)
    asm volatile("global_load_lds_dwordx4 %0, off" ::"v"(ahead(i)), "{m0}"(lds) : "memory");
  bool z[4];
  int cnt = 0;
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    z[k] = t0 + k < n_tok && reused[k] == 0;
    cnt += z[k];
  }
  int incl = cnt;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int up = __shfl_up(incl, o, 64);
    if (lane >= o) incl += up;
  }
  if (lane == 63) wave_tot[wave] = incl;
  asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
  int rank = incl - cnt, total = 0;
#pragma unroll
  for (int w = 0; w < 8; ++w) {
    if (w < wave) rank += wave_tot[w];
    total += wave_tot[w];
  }
#pragma unroll
  for (int k = 0; k < 4; ++k)
    if (z[k]) list[rank++] = t0 + k;
  asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
  if (blockIdx.x == 0) {  // what the compaction kernel would have written, for the kernels that follow
    for (int r = tid; r < total; r += 512) {
      p.sel_idx_out[r] = list[r];
      if (p.sel_idx_out2) p.sel_idx_out2[r] = list[r];
    }
    // refreshed tokens in front of sequence b: first list position holding a token >= b * seq
    auto before = [&](int b) {
      const int key = b * p.sel_seq;
      int lo = 0, hi = total;
      while (lo < hi) {
        const int mid = (lo + hi) >> 1;
        if (list[mid] < key) lo = mid + 1; else hi = mid;
      }
      return lo;
    };
    for (int b = tid; b <= p.sel_batch; b += 512) {  // (a batch may have more sequences than threads)
      const int off = before(b);
      p.sel_off_out[b] = off;
      if (p.sel_count_out && b < p.sel_batch) p.sel_count_out[b] = before(b + 1) - off;
    }
  }
  return total;
}

// The count of listed rows and, FUSED, the list derived from the mask bytes inside the kernel (two instantiations,
// so that the plain one carries none of the list handling), behind STAGES bytes of stage memory: 64 bytes of sums, the
// list, 1 KiB that nobody reads; else that KiB alone.
template <bool FUSED>
constexpr int kListBytes = FUSED ? 64 + kSelMaxTokens * 4 + 1024 : 1024;
template <bool FUSED, int STAGES>
__device__ __forceinline__ int listed_rows(const GemmDev& p, unsigned char* smem, lds_idx_t& lidx) {
  if constexpr (FUSED) {
    int32_t* list = reinterpret_cast<int32_t*>(smem + STAGES + 64);
    const int m = derive_rows(p, list, reinterpret_cast<int*>(smem + STAGES), smem + STAGES + 64 + kSelMaxTokens * 4);
    lidx = (lds_idx_t)list;
    return m;
  } else {
    // (the weights ahead as in derive_rows, 16 rows per workgroup: the count and the list are a shorter wait, and the
    // list, which comes behind these loads, must not wait for more.  Steps over 1 x 1024 tokens with 205 refreshed rows, hidden
    // 1024 40.9 -> 40.6 us, 3072 70.8 -> 70.2, 4096 87.7 -> 86.9; with 4 rows, the stream, no difference; 16384 tokens unchanged)
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int per_xcd = (p.n + 7) >> 3, first = (blockIdx.x & 7) * per_xcd;
    const int last = first + per_xcd < p.n ? first + per_xcd - 1 : p.n - 1;
    const int r = first + ((blockIdx.x >> 3) * 8 + wave) * 2 + (lane >> 5);
    const bf16_t* ahead = p.wt + (long)(r < last ? r : last) * p.k + ((lane & 31) * 8 < p.k ? (lane & 31) * 8 : 0);
    __builtin_amdgcn_global_load_lds((gptr_t)ahead, (lptr_t)(smem + STAGES), 16, 0, 0);
    // (a scalar load, which does not wait for the weights)
    return p.m_dev ? *(const __attribute__((address_space(4))) int32_t*)(uintptr_t)p.m_dev : p.m_max;
  }
}
// Up to 32 rows and a narrow output (the output projection): the register-fed stream
// (measured at n = 4096: 11-15 us against 17 us for 64 x 64 tiles, which give that width
// only 64 workgroups).  Wide outputs keep the 64 x 64 tiles for few rows: with 192
// column tiles they already stream the weights at 5 TB/s.
__device__ __forceinline__ bool few_rows(const GemmDev& p, const int m, unsigned char* smem, lds_idx_t lidx) {
  if (m > kSkinnyRows || p.n >= kSkinnyMaxN) return false;
  if (m <= 16) skinny_tile<8, 1>(p, m, smem, threadIdx.x, lidx); else skinny_tile<8, 2>(p, m, smem, threadIdx.x, lidx);
  return true;
}

// Sizes that 64 x 64 tiles serve in one round whatever the count turns out to be: without the other shapes and the rule (what
// bounds such a launch is its own start: code fetched once, the list, the first reads).  Launches of 80 rows, 402 x 1536 x 512 and 402 x
// 512 x 512, with the kernel of all shapes and with this one 5.48 and 5.14, 5.44 and 5.12 us; a step of 2 x 201 tokens of hidden 512 27.32 and 26.80.
template <bool FUSED>
__global__ void __launch_bounds__(512) gemm_bf16_rows_small_kernel(GemmDev p) {
  constexpr int STAGES = smem_bytes<64, 64, 8>();
  __shared__ __attribute__((aligned(1024))) unsigned char smem[STAGES + kListBytes<FUSED>];
  lds_idx_t lidx = nullptr;
  const int m = listed_rows<FUSED, STAGES>(p, smem, lidx);
  // (every way out waits for the loads into LDS that are under way)
  if (m > 0 && !few_rows(p, m, smem, lidx)) gemm_tile16<64, 64, 2, 4, 8>(p, m, smem, threadIdx.x, blockIdx.x, lidx);
  wait_vmcnt<0>();
}

template <bool FUSED>
__global__ void __launch_bounds__(512) gemm_bf16_rows_wide_kernel(GemmDev p) {
  // A row list derived from the mask lies behind the stage memory for the whole launch.  (In the stage memory
  // it had to be read before the first load into LDS, a barrier between them, and derived again, seven copies of
  // that code and 152 spilled scalars, in front of every further pass.  Steps, with the shape in line: 2 x 201 tokens
  // of hidden 512 28.5 -> 27.6 us, 1 x 1024 of 4096 with 4 refreshed rows 60.9 -> 60.4, with 205 rows 89.8 -> 89.4.
  // One array for both: see score_proj_kernel.)
  static_assert(kWideSmem + kListBytes<FUSED> <= 160 * 1024, "stage memory and row list must fit the LDS of a CU");
  __shared__ __attribute__((aligned(1024))) unsigned char smem[kWideSmem + kListBytes<FUSED>];
  static_assert(smem_bytes<64, 64, 8>() <= kWideSmem && smem_bytes<128, 48, 5>() <= kWideSmem &&
                    smem_bytes<128, 64, 4>() <= kWideSmem && smem_bytes<128, 96, 4>() <= kWideSmem &&
                    smem_bytes<128, 192, 3>() <= kWideSmem && smem_bytes<128, 128, 4>() <= kWideSmem &&
                    pp_smem_bytes<3>() <= kWideSmem && pp_smem_bytes<4>() <= kWideSmem,
                "shared buffer too small");
  lds_idx_t lidx = nullptr;
  const int m = listed_rows<FUSED, kWideSmem>(p, smem, lidx);
  // (every way out waits for the loads into LDS that are under way)
  if (m <= 0 || few_rows(p, m, smem, lidx)) return wait_vmcnt<0>();
  // Tiles in passes, virtual block id = block id + pass * grid size.  Every thread of the workgroup
  // sees the same m and so takes the same branch and the same number of passes.
  auto passes = [&](int tiles, auto tile) __attribute__((always_inline)) {
    const int per_xcd = (tiles + 7) >> 3;
    for (int vb = blockIdx.x; (vb >> 3) < per_xcd; vb += gridDim.x) {
      if (vb != (int)blockIdx.x) __syncthreads();  // the ring is reused: everybody is done with the last tile
      if (!tile(vb)) break;
    }
    wait_vmcnt<0>();
  };
  const GemmRoute shape = best_tile(m, p.n, true);
  if (shape == GemmRoute::kPp256Cut) {
    // Rounds of 256 x 256 tiles; the tiles of the last round are cut into four 128 x 128 tiles each and
    // spread over all workgroups (one or two short rounds instead of a long, mostly idle one).
    const int G = gridDim.x, tiles_m = (m + 255) / 256, tiles_n = p.n / 256;
    const int total = tiles_m * tiles_n, per_xcd = (total + 7) >> 3, n_vb = per_xcd * 8;  // 8 per XCD slot
    const int whole_end = n_vb - n_vb % G;
    bool first = true;
    auto next_tile = [&]() __attribute__((always_inline)) {
      if (!first) __syncthreads();  // the ring is reused: everybody is done with the last tile
      first = false;
    };
    for (int vb = blockIdx.x; vb < whole_end; vb += G) {
      next_tile();
      gemm_tile_pp<4>(p, m, smem, vb, lidx);
    }
    // child c: the parents of an XCD slot stay on their XCD (c & 7), 4 children per parent
    for (int c = blockIdx.x; c < 4 * (n_vb - whole_end); c += G) {
      const int vb = whole_end + ((c >> 5) << 3) + (c & 7), quarter = (c >> 3) & 3;
      const int unit = (vb & 7) * per_xcd + (vb >> 3);
      if (unit >= total) continue;
      int tm, tn;
      tile_of_unit(unit, tiles_m, tiles_n, tm, tn);
      const int cm = 2 * tm + (quarter >> 1), cn = 2 * tn + (quarter & 1);
      if (cm * 128 >= m) continue;
      next_tile();
      gemm_tile16<128, 128, 2, 4, 4>(p, m, smem, threadIdx.x, 0, lidx, cm, cn);
    }
    return wait_vmcnt<0>();
  }
  switch (shape) {
    case GemmRoute::kPp256:
      return passes(tiles_of(m, p.n, kPpRows, 256), [&](int vb) { return gemm_tile_pp<4>(p, m, smem, vb, lidx); });
    case GemmRoute::kPp192:
      return passes(tiles_of(m, p.n, kPpRows, 192), [&](int vb) { return gemm_tile_pp<3>(p, m, smem, vb, lidx); });
    case GemmRoute::kPp128:
      return passes(tiles_of(m, p.n, kPpRows, 128), [&](int vb) { return gemm_tile_pp<2>(p, m, smem, vb, lidx); });
    case GemmRoute::k128x192:
      return passes(tiles_of(m, p.n, 128, 192), [&](int vb) { return gemm_tile16<128, 192, 2, 4, 3>(p, m, smem, threadIdx.x, vb, lidx); });
    case GemmRoute::k128x128:
      return passes(tiles_of(m, p.n, 128, 128), [&](int vb) { return gemm_tile16<128, 128, 2, 4, 4>(p, m, smem, threadIdx.x, vb, lidx); });
    case GemmRoute::k128x96:
      return passes(tiles_of(m, p.n, 128, 96), [&](int vb) { return gemm_tile16<128, 96, 4, 2, 4>(p, m, smem, threadIdx.x, vb, lidx); });
    case GemmRoute::k128x64:
      return passes(tiles_of(m, p.n, 128, 64), [&](int vb) { return gemm_tile16<128, 64, 4, 2, 4>(p, m, smem, threadIdx.x, vb, lidx); });
    case GemmRoute::k128x48:
      return passes(tiles_of(m, p.n, 128, 48), [&](int vb) { return gemm_tile16<128, 48, 8, 1, 5>(p, m, smem, threadIdx.x, vb, lidx); });
    default:
      return passes(tiles_of(m, p.n, 64, 64), [&](int vb) { return gemm_tile16<64, 64, 2, 4, 8>(p, m, smem, threadIdx.x, vb, lidx); });
  }
}

// ---- scored query columns of all rows, with the score ---------------------------------
// One launch for what were three dependent steps of a few microseconds each (projection in
// k-range slabs, a second kernel that added the slabs and scored): BM rows x all WIDTH scored
// columns per workgroup, so that a workgroup holds whole queries and can score them.  What bounds
// it is the operands that a CU pulls, (BM + WIDTH) rows of k; with few row tiles k is cut over
// KP workgroups, each of which leaves its sums at device scope (as in gemm_tile_pp), and the
// last one to arrive adds them up.
// Sum over k: that of the caller's ranges of k, added up as a binary tree whatever BM and KP are,
// so the route (workspace or not) does not show in a query.
// Measured (projection + score + the gap between them -> this launch, inside a step): 1024 rows
// 7.6 + 4.9 + 2.4 -> 11 us, 8192 rows 45 + 7.7 + 2.4 -> 38 us, 16384 rows 52 + 9.4 + 2.4 -> 45 us.
struct ScoreProjDev {
  const bf16_t* a;
  const bf16_t* wt;
  const int32_t* idx;
  float* q_prev;
  float* scores;
  uint8_t* mask;
  float* sums;
  unsigned* count;
  int k, m, k_parts, ranges;  // workgroups per row tile; ranges of the summation tree
  int force_refresh, batch, seq, prefix;
  float threshold;
};

template <int BM, int WIDTH, int WAVES_M, int WAVES_N>
__global__ void __launch_bounds__(WAVES_M* WAVES_N * 64) score_proj_kernel(ScoreProjDev p) {
  constexpr int NW = WAVES_M * WAVES_N, NT = NW * 64, STAGES = 5;
  constexpr int WM = BM / WAVES_M, WN = WIDTH / WAVES_N;
  constexpr int TM = WM / 16, TN = WN / 16, KS = BK / 32;
  constexpr int STAGE_BYTES = (BM + WIDTH) * ROW_BYTES;
  constexpr int GROUPS = (BM + WIDTH) / 8;
  constexpr int LPW = (GROUPS + NW - 1) / NW;  // surplus loads repeat the last group
  constexpr int LDQ = score_query_stride(WIDTH);
  static_assert(WM % 16 == 0 && WN % 16 == 0 && BM % NW == 0, "wave tiles of 16 x 16, whole rows per wave");
  static_assert(LPW * (STAGES - 1) < 64, "vmcnt range");
  // (one LDS array only: with a second one the compiler tracks which of them a global -> LDS load
  // may write, and puts s_waitcnt vmcnt(0) in front of the fragment reads, which drains the ring)
  __shared__ __attribute__((aligned(1024))) unsigned char smem[STAGES * STAGE_BYTES];
  // whether this workgroup is the last one lies behind the queries, which a wave may write while another
  // one still reads it
  constexpr int ARRIVED = score_arrived_offset(BM, WIDTH);
  static_assert(ARRIVED + 4 <= STAGES * STAGE_BYTES, "the flag must fit into the stage memory");
  int& last_here = *reinterpret_cast<int*>(smem + ARRIVED);

  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  // frozen tokens: always reused, never scored
  for (long i = (long)blockIdx.x * NT + tid; i < (long)p.batch * p.prefix; i += (long)gridDim.x * NT) {
    const long tok = i / p.prefix * p.seq + i % p.prefix;
    if (p.scores) p.scores[tok] = 0.f;
    p.mask[tok] = 1;
  }

  const int tile = blockIdx.x / p.k_parts, part = blockIdx.x % p.k_parts;
  const int m0 = tile * BM;
  const int wave_m = wave % WAVES_M, wave_n = wave / WAVES_M;
  const int l16 = lane & 15, kq = lane >> 4;
  const int KT = p.k / BK / p.k_parts;      // k-steps of this workgroup
  const int range = p.k / BK / p.ranges;    // k-steps of a range of the tree

  const bf16_t* src[LPW];
  int grp[LPW];
#pragma unroll
  for (int i = 0; i < LPW; ++i) {
    grp[i] = wave * LPW + i < GROUPS ? wave * LPW + i : GROUPS - 1;
    const int r = grp[i] * 8 + (lane >> 3);
    const long off = (long)part * KT * BK + ((lane & 7) ^ ((r >> 1) & 7)) * 8;
    if (r < BM) {
      const int row = m0 + r < p.m ? m0 + r : p.m - 1;
      src[i] = p.a + (long)(p.idx ? p.idx[row] : row) * p.k + off;
    } else {
      src[i] = p.wt + (long)(r - BM) * p.k + off;
    }
  }
  auto issue_loads = [&](int kt) __attribute__((always_inline)) {
    unsigned char* base = smem + (kt % STAGES) * STAGE_BYTES;
    const int k = kt < KT ? kt : KT - 1;
#pragma unroll
    for (int i = 0; i < LPW; ++i)
      __builtin_amdgcn_global_load_lds((gptr_t)(src[i] + k * BK), (lptr_t)(base + grp[i] * 8 * ROW_BYTES), 16, 0, 0);
  };

  f32x4 acc[TM][TN], level[3][TM][TN];
#pragma unroll
  for (int i = 0; i < TM; ++i)
#pragma unroll
    for (int j = 0; j < TN; ++j) acc[i][j] = level[0][i][j] = level[1][i][j] = level[2][i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
  const int sw = (l16 >> 1) & 7;
  const int a_row_off = (wave_m * WM + l16) * ROW_BYTES;
  const int b_row_off = (BM + wave_n * WN + l16) * ROW_BYTES;

#pragma unroll
  for (int s = 0; s < STAGES - 1; ++s) issue_loads(s);
  int done = 0, in_range = 0;  // ranges complete, k-steps of the current one
  for (int kt = 0; kt < KT; ++kt) {
    wait_vmcnt_and_barrier<LPW*(STAGES - 2)>();
    issue_loads(kt + STAGES - 1);
    const unsigned char* st = smem + (kt % STAGES) * STAGE_BYTES;
    bf16x8 fa[KS][TM], fb[KS][TN];
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      const int koff = ((ks * 4 + kq) ^ sw) * 16;
#pragma unroll
      for (int i = 0; i < TM; ++i) fa[ks][i] = *reinterpret_cast<const bf16x8*>(st + a_row_off + i * 16 * ROW_BYTES + koff);
#pragma unroll
      for (int j = 0; j < TN; ++j) fb[ks][j] = *reinterpret_cast<const bf16x8*>(st + b_row_off + j * 16 * ROW_BYTES + koff);
    }
#pragma unroll
    for (int ks = 0; ks < KS; ++ks)
#pragma unroll
      for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j)
          acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fb[ks][j], fa[ks][i], acc[i][j], 0, 0, 0);
    if (++in_range < range) continue;
    // a range is complete: up the tree (the last one of the workgroup ends as its whole sum in acc)
    in_range = 0;
    const bool last = kt + 1 == KT;
    bool carry = true;
#pragma unroll
    for (int l = 0; l < 3; ++l) {
      if (!carry) break;
      if ((done >> l) & 1) {
#pragma unroll
        for (int i = 0; i < TM; ++i)
#pragma unroll
          for (int j = 0; j < TN; ++j) acc[i][j] = level[l][i][j] + acc[i][j];
      } else if (!last) {
#pragma unroll
        for (int i = 0; i < TM; ++i)
#pragma unroll
          for (int j = 0; j < TN; ++j) {
            level[l][i][j] = acc[i][j];
            acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
          }
        carry = false;
      }
    }
    ++done;
  }
  wait_vmcnt<0>();
  __syncthreads();

  if (p.k_parts > 1) {
    constexpr int kDeviceScope = 16;  // cache policy sc1
    constexpr int kSlot = BM * WIDTH * 4;
    const auto slots = __builtin_amdgcn_make_buffer_rsrc(p.sums + (long)tile * p.k_parts * (BM * WIDTH), 0, p.k_parts * kSlot, 0x00027000);
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
      for (int j = 0; j < TN; ++j)
        __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, acc[i][j]), slots, part * kSlot + ((i * TN + j) * NT + tid) * 16, 0, kDeviceScope);
    wait_vmcnt<0>();
    __syncthreads();
    if (tid == 0) last_here = arrive_last(p.count + tile, p.k_parts);
    __syncthreads();
    if (!last_here) return;
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
      for (int j = 0; j < TN; ++j) {
        f32x4 w[8];
#pragma unroll
        for (int q = 0; q < 8; ++q) {
          w[q] = f32x4{0.f, 0.f, 0.f, 0.f};
          if (q < p.k_parts)
            w[q] = __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(slots, q * kSlot + ((i * TN + j) * NT + tid) * 16, 0, kDeviceScope));
        }
        f32x4 v = w[0] + w[1];  // (the tree above the workgroups)
        if (p.k_parts > 2) v += w[2] + w[3];
        if (p.k_parts > 4) v += (w[4] + w[5]) + (w[6] + w[7]);
        acc[i][j] = v;
      }
  }

  // acc[i][j][e] = query[row, col]: row = wave_m*WM + 16 i + l16, col = wave_n*WN + 16 j + 4 kq + e
  float* qs = reinterpret_cast<float*>(smem);
#pragma unroll
  for (int i = 0; i < TM; ++i)
#pragma unroll
    for (int j = 0; j < TN; ++j)
      *reinterpret_cast<f32x4*>(qs + (wave_m * WM + i * 16 + l16) * LDQ + wave_n * WN + j * 16 + kq * 4) = acc[i][j];
  __syncthreads();
  // score: a wave per row, two neighbouring channels per lane, the three sums with one lane
  // assignment and one butterfly (an unchanged query gives dot == |q|^2 == |p|^2 bit for bit)
  constexpr int RPW = BM / NW;
  const int c = lane * 2;
  f32x2 prev[RPW];
  long tok[RPW];
#pragma unroll
  for (int r = 0; r < RPW; ++r) {
    const int row = m0 + wave * RPW + r;
    const int listed = row < p.m ? row : p.m - 1;
    tok[r] = p.idx ? p.idx[listed] : listed;
    prev[r] = c < WIDTH ? *reinterpret_cast<const f32x2*>(p.q_prev + tok[r] * WIDTH + c) : f32x2{0.f, 0.f};
  }
#pragma unroll
  for (int r = 0; r < RPW; ++r) {
    if (m0 + wave * RPW + r >= p.m) break;
    f32x2 q = {0.f, 0.f};
    if (c < WIDTH) {
      q = *reinterpret_cast<const f32x2*>(qs + (wave * RPW + r) * LDQ + c);
      *reinterpret_cast<f32x2*>(p.q_prev + tok[r] * WIDTH + c) = q;  // the score cache takes this step's query
    }
    const float dot = wave_sum(fmaf(q[1], prev[r][1], q[0] * prev[r][0]));
    const float nq = wave_sum(fmaf(q[1], q[1], q[0] * q[0]));
    const float np = wave_sum(fmaf(prev[r][1], prev[r][1], prev[r][0] * prev[r][0]));
    if (lane == 0) {
      const float s = drift_score(dot, nq, np);
      if (p.scores) p.scores[tok[r]] = s;
      p.mask[tok[r]] = (!p.force_refresh && s <= p.threshold) ? 1 : 0;
    }
  }
}

GemmDev to_dev(const GemmArgs& g) {
  GemmDev p;
  p.a = static_cast<const bf16_t*>(g.a);
  p.wt = static_cast<const bf16_t*>(g.wt);
  p.idx = g.idx;
  p.m_dev = g.m_dev;
  p.c0 = static_cast<bf16_t*>(g.c[0]);
  p.c1 = static_cast<bf16_t*>(g.c[1]);
  p.c2 = static_cast<bf16_t*>(g.c[2]);
  p.c32 = g.c32;
  p.lda = g.lda;
  p.n = g.n;
  p.k = g.k;
  p.m_max = g.m_max;
  p.ldc = g.ldc;
  p.seg_n = g.seg_n;
  p.c32_cols = g.c32_cols;
  p.k_parts = 1;
  p.c32_part_stride = 0;
  p.rope = g.rope;
  p.rope_cols = g.rope_cols;
  p.rope_dh = g.rope_dh;
  p.rope_seq = g.rope_seq;
  p.swiglu_pairs = g.swiglu_pairs;
  p.sel_mask = g.sel_mask;
  p.sel_batch = g.sel_batch;
  p.sel_seq = g.sel_seq;
  if (g.linear) {
    p.bias = static_cast<const bf16_t*>(g.bias);
    p.residual = static_cast<const bf16_t*>(g.residual);
    p.ldr = g.ldr;
    p.act = g.act;
  } else {
    p.sel_idx_out = g.sel_idx_out;
    p.sel_idx_out2 = g.sel_idx_out2;
    p.sel_off_out = g.sel_off_out;
    p.sel_count_out = g.sel_count_out;
  }
  p.ahead = 0;
  p.split_tiles = g.split_tiles;
  p.split_count = g.split_count;
  p.part_n = g.part_n;
  p.part_idx = g.part_idx;
  p.part_m_dev = g.part_m_dev;
  return p;
}

// Outputs larger than half of the last-level cache (256 MB) are stored past the L2: what the stages behind them read first is
// no longer there anyway, and the operands stay in its place (us, stored through the L2 and past it, in a step of 8 x 2048 tokens of hidden 4096:
// Q, K and V, 403 MB, 1136 and 1130, the score, the normalisation and the residual sum around them 10.4 and 9.0, 46.2 and 45.7, 70.0
// and 64.9).  Smaller ones are not: 25 MB, 1 x 1024 x 12288, leave the attention behind them 32.2 us, and 33.4 stored past it.
constexpr long kStreamBytes = 128l << 20;
template <int TN>
hipError_t launch_quad(const GemmArgs& g, hipStream_t s) {
  const int tiles = grid_for(tiles_of(g.m_max, g.n, kPpRows, 64 * TN));
  const dim3 grid(tiles < kWideGrid ? tiles : kWideGrid);
  if (TN == 4 && (long)g.m_max * g.n * (g.swiglu_pairs ? 1 : 2) > kStreamBytes)
    hipLaunchKernelGGL((gemm_bf16_quad_kernel<TN, TN == 4>), grid, dim3(256), 0, s, to_dev(g));
  else
    hipLaunchKernelGGL((gemm_bf16_quad_kernel<TN, false>), grid, dim3(256), 0, s, to_dev(g));
  return hipGetLastError();
}

template <int BM, int BN, int WAVES_M, int WAVES_N, int STAGES>
hipError_t launch_ranges(const GemmArgs& g, hipStream_t s) {
  GemmDev p = to_dev(g);
  p.k_parts = g.k_parts;
  p.c32_part_stride = g.c32_part_stride;
  hipLaunchKernelGGL((gemm_bf16_ranges_kernel<BM, BN, WAVES_M, WAVES_N, STAGES>),
                     dim3(grid_for(tiles_of(g.m_max, g.n, BM, BN) * p.k_parts)), dim3(WAVES_M * WAVES_N * 64), 0, s, p);
  return hipGetLastError();
}

template <int BM, int BN, int WAVES_M, int WAVES_N, int STAGES>
hipError_t launch_tile16(const GemmArgs& g, hipStream_t s) {
  hipLaunchKernelGGL((gemm_bf16_tile16_kernel<BM, BN, WAVES_M, WAVES_N, STAGES>),
                     dim3(grid_for(tiles_of(g.m_max, g.n, BM, BN))), dim3(512), 0, s, to_dev(g));
  return hipGetLastError();
}

template <int TN, bool SPLIT = false>
hipError_t launch_pp(const GemmArgs& g, hipStream_t s) {
  const int tiles = tiles_of(g.m_max, g.n, kPpRows, 64 * TN);
  if (SPLIT && (tiles > kSplitTiles || !g.split_tiles || !g.split_count)) return hipErrorInvalidValue;
  hipLaunchKernelGGL((gemm_bf16_pp_kernel<TN, SPLIT>), dim3(grid_for(SPLIT ? 2 * tiles : tiles)), dim3(512), 0, s,
                     to_dev(g));
  return hipGetLastError();
}

hipError_t launch_rows_wide(const GemmArgs& g, hipStream_t s) {
  // as many as the smallest tiles, or the column groups of the stream over the weights, whichever are more
  const int small = tiles_of(g.m_max, g.n, 64, 64), groups = g.m_max > 0 ? g.n / 16 : 0;
  int blocks = small > groups ? small : groups;
  if (blocks == 0) return hipSuccess;
  if (blocks > kWideGrid) blocks = kWideGrid;
  blocks = grid_for(blocks);
  GemmDev p = to_dev(g);
  p.ahead = ahead_loads(g.n, blocks);
  if (small <= kWideGrid && g.sel_mask)
    hipLaunchKernelGGL(gemm_bf16_rows_small_kernel<true>, dim3(blocks), dim3(512), 0, s, p);
  else if (small <= kWideGrid)
    hipLaunchKernelGGL(gemm_bf16_rows_small_kernel<false>, dim3(blocks), dim3(512), 0, s, p);
  else if (g.sel_mask)
    hipLaunchKernelGGL(gemm_bf16_rows_wide_kernel<true>, dim3(blocks), dim3(512), 0, s, p);
  else
    hipLaunchKernelGGL(gemm_bf16_rows_wide_kernel<false>, dim3(blocks), dim3(512), 0, s, p);
  return hipGetLastError();
}

// act(A W + bias) + residual (linear_route)
template <int BM, int BN, int WAVES_M, int WAVES_N, int STAGES>
hipError_t launch_linear_tile16(const GemmArgs& g, hipStream_t s) {
  hipLaunchKernelGGL((linear_bf16_tile16_kernel<BM, BN, WAVES_M, WAVES_N, STAGES>),
                     dim3(grid_for(tiles_of(g.m_max, g.n, BM, BN))), dim3(WAVES_M * WAVES_N * 64), 0, s, to_dev(g));
  return hipGetLastError();
}
template <int TN>
hipError_t launch_linear_pp(const GemmArgs& g, hipStream_t s) {
  hipLaunchKernelGGL(linear_bf16_pp_kernel<TN>, dim3(grid_for(tiles_of(g.m_max, g.n, kPpRows, 64 * TN))), dim3(512), 0, s,
                     to_dev(g));
  return hipGetLastError();
}
template <int TN>
hipError_t launch_linear_quad(const GemmArgs& g, hipStream_t s) {
  const int tiles = grid_for(tiles_of(g.m_max, g.n, kPpRows, 64 * TN));
  const dim3 grid(tiles < kWideGrid ? tiles : kWideGrid);
  if (TN == 4 && (long)g.m_max * g.n * 2 > kStreamBytes)
    hipLaunchKernelGGL((linear_bf16_quad_kernel<TN, TN == 4>), grid, dim3(256), 0, s, to_dev(g));
  else
    hipLaunchKernelGGL((linear_bf16_quad_kernel<TN, false>), grid, dim3(256), 0, s, to_dev(g));
  return hipGetLastError();
}
hipError_t launch_linear(const GemmArgs& g, hipStream_t s) {
  switch (linear_route(g.m_max, g.n, g.k)) {
    case GemmRoute::kSkinny:
      hipLaunchKernelGGL(linear_bf16_skinny_kernel, dim3(g.n / 16), dim3(512), 0, s, to_dev(g));
      return hipGetLastError();
    case GemmRoute::k32x32: return launch_linear_tile16<32, 32, 2, 2, 8>(g, s);
    case GemmRoute::k64x32: return launch_linear_tile16<64, 32, 4, 2, 6>(g, s);
    case GemmRoute::kQuad256: return launch_linear_quad<4>(g, s);
    case GemmRoute::kQuad192: return launch_linear_quad<3>(g, s);
    case GemmRoute::kPp256: return launch_linear_pp<4>(g, s);
    case GemmRoute::kPp192: return launch_linear_pp<3>(g, s);
    case GemmRoute::kPp128: return launch_linear_pp<2>(g, s);
    case GemmRoute::k128x192: return launch_linear_tile16<128, 192, 2, 4, 3>(g, s);
    case GemmRoute::k128x128: return launch_linear_tile16<128, 128, 2, 4, 4>(g, s);
    case GemmRoute::k128x96: return launch_linear_tile16<128, 96, 4, 2, 4>(g, s);
    case GemmRoute::k64x128: return launch_linear_tile16<64, 128, 2, 4, 5>(g, s);
    case GemmRoute::k64x96: return launch_linear_tile16<64, 96, 4, 2, 6>(g, s);
    case GemmRoute::k64x64: return launch_linear_tile16<64, 64, 2, 4, 8>(g, s);
    default: return hipErrorInvalidValue;
  }
}

}  // namespace

hipError_t launch_gemm_bf16(const GemmArgs& g, hipStream_t s) {
  if (g.part_n > 0) {
    if (g.m_max == 0) return hipSuccess;
    if (g.m_dev || g.sel_mask || g.c32 || g.swiglu_pairs || !g.part_idx || !g.part_m_dev || g.part_n >= g.n || g.part_n % 64 != 0 ||
        g.k < kQuadMinSteps * BK)
      return hipErrorInvalidValue;
    hipLaunchKernelGGL(gemm_bf16_part_kernel, dim3(kWideGrid), dim3(256), 0, s, to_dev(g));
    return hipGetLastError();
  }
  if (g.m_dev || g.sel_mask) return launch_rows_wide(g, s);
  if (g.m_max == 0) return hipSuccess;
  if (g.linear) return launch_linear(g, s);
  switch (gemm_route(g.m_max, g.n, g.k, g.k_parts, g.split_tiles && !g.c32)) {
    case GemmRoute::kPp128Split: return launch_pp<2, true>(g, s);
    case GemmRoute::kQuad256: return launch_quad<4>(g, s);
    case GemmRoute::kQuad192: return launch_quad<3>(g, s);
    case GemmRoute::kPp256: return launch_pp<4>(g, s);
    case GemmRoute::kPp192: return launch_pp<3>(g, s);
    case GemmRoute::kPp128: return launch_pp<2>(g, s);
    case GemmRoute::k128x192: return launch_tile16<128, 192, 2, 4, 3>(g, s);
    case GemmRoute::k128x128: return launch_tile16<128, 128, 2, 4, 4>(g, s);
    case GemmRoute::k128x96: return launch_tile16<128, 96, 4, 2, 4>(g, s);
    case GemmRoute::k64x128: return launch_tile16<64, 128, 2, 4, 5>(g, s);
    case GemmRoute::k64x96: return launch_tile16<64, 96, 4, 2, 6>(g, s);
    case GemmRoute::k64x64: return launch_tile16<64, 64, 2, 4, 8>(g, s);
    case GemmRoute::kTile128: return launch_ranges<128, 128, 4, 2, 4>(g, s);
    case GemmRoute::kTile64: return launch_ranges<64, 64, 2, 2, 4>(g, s);
    case GemmRoute::k128x48: case GemmRoute::k128x64: case GemmRoute::kPp256Cut: break;  // (listed rows)
  }
  return hipErrorInvalidValue;
}

hipError_t launch_score_proj(const ScoreProjArgs& g, hipStream_t s) {
  if (g.m == 0) return hipSuccess;
  const int ranges = g.k_ranges;
  // Rows per workgroup and workgroups per row tile, by what a workgroup takes (us): its operands at
  // 100 KB/us; when k is cut, 3 for the hand-over and the slots that the last workgroup reads back at
  // 40 KB/us; 0.04 per row to score.  Fitted at 1024 rows of 4096, width 128 (rows / workgroups per
  // tile): 16/4 11.0 us, 16/2 13.6, 32/4 12.7, 32/8 13.1, 64/4 16.1, 64/8 16.4.
  int bm = 64, kp = 1;
  double best = 1e30;
  for (int b = 16; b <= 64; b *= 2)
    for (int q = 1; q <= ranges; q *= 2) {
      const long tiles = (g.m + b - 1) / b;
      const size_t slots = (size_t)tiles * q * b * g.width;
      if (q > 1 && (!g.sums || tiles > kScoreTiles || slots > g.sums_elems)) continue;
      const double rounds = (double)((tiles * q + 255) / 256);
      const double pull = rounds * (b + g.width) * (double)(g.k / q) * 2 / 100e3;
      const double cost = pull + (q > 1 ? 3.0 + (double)q * b * g.width * 4 / 40e3 : 0.0) + 0.04 * b;
      if (cost < best) {
        best = cost;
        bm = b;
        kp = q;
      }
    }
  ScoreProjDev p;
  p.a = static_cast<const bf16_t*>(g.a);
  p.wt = static_cast<const bf16_t*>(g.wt);
  p.idx = g.idx;
  p.q_prev = g.q_prev;
  p.scores = g.scores;
  p.mask = g.mask;
  p.sums = g.sums;
  p.count = g.count;
  p.k = g.k;
  p.m = g.m;
  p.k_parts = kp;
  p.ranges = ranges;
  p.force_refresh = g.force_refresh;
  p.batch = g.batch;
  p.seq = g.seq;
  p.prefix = g.prefix;
  p.threshold = g.threshold;
  const dim3 grid((unsigned)((g.m + bm - 1) / bm * kp));
  if (g.width == 128) {
    if (bm == 16) hipLaunchKernelGGL((score_proj_kernel<16, 128, 1, 8>), grid, dim3(512), 0, s, p);
    else if (bm == 32) hipLaunchKernelGGL((score_proj_kernel<32, 128, 2, 4>), grid, dim3(512), 0, s, p);
    else hipLaunchKernelGGL((score_proj_kernel<64, 128, 2, 4>), grid, dim3(512), 0, s, p);
  } else if (g.width == 64) {
    if (bm == 16) hipLaunchKernelGGL((score_proj_kernel<16, 64, 1, 4>), grid, dim3(256), 0, s, p);
    else if (bm == 32) hipLaunchKernelGGL((score_proj_kernel<32, 64, 2, 4>), grid, dim3(512), 0, s, p);
    else hipLaunchKernelGGL((score_proj_kernel<64, 64, 4, 2>), grid, dim3(512), 0, s, p);
  } else {
    return hipErrorInvalidValue;
  }
  return hipGetLastError();
}

}  // namespace dare
