// Tiles of a projection that its bf16 and its 8-bit form share (gfx950 matrix cores): what a workgroup loads, in which order it multiplies,
// and how it stores.
//
// Both types have 128 bytes of k per row and k-step, 16 bytes of it per lane and MFMA operand, and matrix instructions of the same length
// (v_mfma_f32_16x16x32_bf16, v_mfma_i32_16x16x64_i8: 16 rows and columns, 64 bytes of k): loads, LDS layout and fragment reads know nothing
// of the type.  Sizes along k (GemmDev's k and lda, BK) count units of two bytes: one bf16, two codes of 8 bits.
#pragma once

#include <type_traits>

#include "dare_common.h"
#include "gemm_route.h"

namespace dare {
namespace {

constexpr int BK = kRouteBK;      // k per stage: one 128-byte row segment
constexpr int ROW_BYTES = BK * 2;
constexpr int GROUP_M = 8;        // row-tiles walked before the next column-tile

struct GemmDev {
  const bf16_t* a;
  const bf16_t* wt;
  const int32_t* idx;
  const int32_t* m_dev;
  bf16_t* c0;
  bf16_t* c1;
  bf16_t* c2;
  float* c32;
  int lda, n, k, m_max, ldc, seg_n, c32_cols;
  int k_parts;           // k is cut into this many ranges (1 = whole k per tile)
  long c32_part_stride;  // elements between the fp32 outputs of consecutive ranges
  const float* rope;     // rotary table, or nullptr
  int rope_cols, rope_dh, rope_seq;
  int swiglu_pairs;
  const uint8_t* sel_mask;
  int sel_batch, sel_seq;
  // What a kernel that makes its row list writes of it, or, for LINEAR forms, which have no such list, act(product + bias) + residual:
  // in one place, or the arguments of every kernel here end in one more cache line (a step of 1024 tokens 73.26 us, and 73.58).
  union {
    struct {
      int32_t* sel_idx_out;
      int32_t* sel_idx_out2;
      int32_t* sel_off_out;
      int32_t* sel_count_out;
    };
    struct {
      const bf16_t* bias;
      const bf16_t* residual;
      long ldr;
      int act;
    };
  };
  int ahead;                // loads of weights per wave while the list is made (ahead_loads)
  // two workgroups on the halves of k of one tile (gemm_tile_pp): [tiles][2] fp32 tiles and
  // [tiles] counters; nullptr = one workgroup per tile
  float* split_tiles;
  int* split_count;
  // columns [0, part_n) for the rows of a second list only (gemm_bf16_part_kernel)
  int part_n;
  const int32_t* part_idx;
  const int32_t* part_m_dev;
};

typedef const __attribute__((address_space(1))) void* gptr_t;
typedef __attribute__((address_space(3))) void* lptr_t;
typedef const __attribute__((address_space(3))) int32_t* lds_idx_t;  // a row list held in LDS

// The operands' type: bf16 with sums in fp32.
struct Bf16Op {
  typedef GemmDev Dev;
  typedef bf16x8 Frag;
  typedef f32x4 Acc;
  static constexpr bool kScaled = false;
  static __device__ __forceinline__ Acc mfma(Frag w, Frag x, Acc sum) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(w, x, sum, 0, 0, 0); }
};

// Token ids of listed rows: from the list in LDS when the kernel derived it itself, else from the
// caller's list, else the rows themselves.  (One branch around all of them: a branch per row takes
// longer than the reads.)
template <int N>
__device__ __forceinline__ void row_tokens(const int32_t* __restrict__ gidx, lds_idx_t lidx, const int (&row)[N],
                                           int (&tok)[N]) {
  if (lidx) {
#pragma unroll
    for (int i = 0; i < N; ++i) tok[i] = lidx[row[i]];
  } else if (gidx) {
#pragma unroll
    for (int i = 0; i < N; ++i) tok[i] = gidx[row[i]];
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i) tok[i] = row[i];
  }
}

// Wait until at most N of this wave's vector-memory operations are outstanding
// and all of its LDS reads have returned, then join the workgroup barrier.
// Written as one asm statement with a memory clobber: __syncthreads() would add a
// release fence, and the compiler answers a fence with vmcnt(0), which would
// drain the whole ring of in-flight k-steps.
template <int N>
__device__ __forceinline__ void wait_vmcnt_and_barrier() {
  static_assert(N >= 0 && N < 64, "vmcnt range");
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(N) : "memory");
}
template <int N>
__device__ __forceinline__ void wait_vmcnt() {
  static_assert(N >= 0 && N < 64, "vmcnt range");
  asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}

// The same where `ahead` (0 .. MAX, or more for MAX; the same in all waves) stages of LOADS each may be outstanding
template <int LOADS, int MAX>
__device__ __forceinline__ void wait_stages_and_barrier(const int ahead) {
  if constexpr (MAX > 0) {
    if (ahead < MAX) return wait_stages_and_barrier<LOADS, MAX - 1>(ahead);
  }
  wait_vmcnt_and_barrier<LOADS * MAX>();
}

template <int BM, int BN, int STAGES>
constexpr int smem_bytes() {
  return STAGES * (BM + BN) * ROW_BYTES;
}

// silu(g) = g / (1 + exp(-g)), by hand: reciprocal, product, one correction, special values by v_div_fixup.  Over all 2^32 values of g
// it has the bits of the compiler's division, which does not know that the divisor is 1 or more and takes twice as long.
// SCALED: divisors above 2^126 (g below -87.336), whose reciprocal is flushed to 0, are multiplied by a power of two; without it only
// for g of kGateLow or more.
constexpr float kGateLow = -87.0f;
template <bool SCALED = true>
__device__ __forceinline__ float silu(float g) {
  const float scale = SCALED && g < kGateLow ? 0x1p-32f : 1.0f;
  const float d = fmaf(__expf(-g), scale, scale), r = __builtin_amdgcn_rcpf(d), q = g * r;
  return __builtin_amdgcn_div_fixupf(fmaf(fmaf(-d, q, g), r, q) * scale, d, g);
}

// Activation of N values at once: what it is is settled outside the loop.  Reciprocals and exponentials by the hardware's
// instructions, 1 ulp of fp32 each, behind them a rounding to bf16.
// GELU: z Phi(z) = max(z, 0) - |z| h(|z|) e^(-z^2 / 2), h(x) = e^(x^2 / 2) erfc(x / sqrt(2)) / 2 = t (a1 + t (a2 + t (a3 + t (a4 + t a5)))), t = 1 / (1 +
// p x), in 14 instructions.  p and the a_i are a fit of our own (least largest error of h relative to min(e^(1.2 x), 400), by linear
// programming): evaluated in fp32 the result is off by 7e-7 at most and, where it falls to 0, by 4.7e-4 of itself, an eighth of the rounding to
// bf16, down to z = -13, where it ends.  (One term more: 1e-7 and 1.3e-4, but 16384 x 12288 x 4096 1225 us for 1212, x 4096 x 512 136 for 130.)
// Tanh form: z / (1 + e^-2y), y = sqrt(2 / pi) (z + 0.044715 z^3).
// MED: minimum and maximum as the middle of three, which saves the instructions that quiet a NaN in front of them (a
// NaN is in e as well): the same values, 16384 x 12288 x 4096 in 8 bits 712 -> 700 us.
template <bool MED = false, int N>
__device__ __forceinline__ void activate(const int act, float (&v)[N]) {
  if (act == DARE_ACT_SILU) {
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] *= __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(-1.44269504f * v[i]));
  } else if (act == DARE_ACT_GELU) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const float z = v[i], x = fabsf(z);
      const float t = __builtin_amdgcn_rcpf(fmaf(x, 0.35056123f, 1.f));
      float e = fmaf(t, -0.096569724f, 0.27045822f);
      e = fmaf(t, e, 0.024472961f);
      e = fmaf(t, e, 0.16388455f);
      e = fmaf(t, e, 0.13775338f) * t * __builtin_amdgcn_exp2f(-0.72134752f * x * x);
      if constexpr (MED)
        v[i] = fmaf(-__builtin_amdgcn_fmed3f(x, 0.f, 1e18f), e, __builtin_amdgcn_fmed3f(z, 0.f, INFINITY));
      else
        v[i] = fmaf(-fminf(x, 1e18f), e, fmaxf(z, 0.f));  // (infinity times 0 is none)
    }
  } else if (act == DARE_ACT_GELU_TANH) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const float z = v[i];
      v[i] = z * __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(-2.30220819f * fmaf(0.044715f * z * z, z, z)));
    }
  }
}

// The same with act(product + bias) + residual in the place of what it describes: sums, activation and residual sum in fp32, one rounding.
// The residual's rows may be the output's: a lane reads what it stores.
template <int W, int TM, int TN, class Value>
__device__ __forceinline__ void store_linear(const GemmDev& p, const int (&tok)[TM], const bool (&live)[TM],
                                             const int (&col)[TN], Value value) {
  typedef __bf16 out_t __attribute__((ext_vector_type(W)));
  const long ldc = p.ldc, ldr = p.ldr;
#pragma unroll
  for (int j = 0; j < TN; ++j) {
    const int c = col[j];
    if (c >= p.n) continue;
    out_t res[TM], bias;
    if (p.residual) {
#pragma unroll
      for (int i = 0; i < TM; ++i) res[i] = *reinterpret_cast<const out_t*>(p.residual + tok[i] * ldr + c);
    }
    if (p.bias) bias = *reinterpret_cast<const out_t*>(p.bias + c);
#pragma unroll
    for (int i = 0; i < TM; ++i) {
      float v[W];
#pragma unroll
      for (int e = 0; e < W; ++e) v[e] = value(i, j, e) + (p.bias ? (float)bias[e] : 0.f);
      activate(p.act, v);
      out_t o;
#pragma unroll
      for (int e = 0; e < W; ++e) o[e] = (bf16_t)(v[e] + (p.residual ? (float)res[i][e] : 0.f));
      if (live[i]) *reinterpret_cast<out_t*>(reinterpret_cast<bf16_t*>(p.c0) + tok[i] * ldc + c) = o;
    }
  }
}

// Epilogue of a wave tile: W (4 or 8) neighbouring output columns col[j] .. col[j] + W - 1 (col[j] a multiple
// of W; a segment, whose width is a multiple of 32, holds all of them) of tokens tok[i], live[i] or not,
// value(i, j, e) each.  Plain: the fp32 copy of the scored columns (before any rotation), then
// rotation, rounding and the store into the column's segment.  Gated: (gate, up) pairs, W / 2 outputs
// silu(gate) * up from column col / 2 on.
// What a launch asks for is settled outside the loops and what a column needs outside that over the rows: decided
// at every store, with the kernel's arguments read again and a division each for segment and
// position, the epilogue was as long as a third of the k loop (its gain is part of gemm_tile16's figures).
template <int W, int TM, int TN, class Value>
__device__ __forceinline__ void store_tile(const GemmDev& p, float* c32, const int (&tok)[TM], const bool (&live)[TM],
                                           const int (&col)[TN], Value value) {
  static_assert(W == 4 || W == 8, "columns of a store");
  typedef __bf16 out_t __attribute__((ext_vector_type(W)));
  typedef __bf16 half_t __attribute__((ext_vector_type(W / 2)));
  if (p.swiglu_pairs) {
#pragma unroll
    for (int i = 0; i < TM; ++i) {
      bf16_t* row = p.c0 + (long)tok[i] * p.ldc;
#pragma unroll
      for (int j = 0; j < TN; ++j) {
        half_t o;
#pragma unroll
        for (int e = 0; e < W / 2; ++e) {
          const float g = value(i, j, 2 * e);
          o[e] = (bf16_t)(silu(g) * value(i, j, 2 * e + 1));
        }
        if (live[i] && col[j] < p.n) *reinterpret_cast<half_t*>(row + (col[j] >> 1)) = o;
      }
    }
    return;
  }
  int pos[TM];
  if (p.rope) {
#pragma unroll
    for (int i = 0; i < TM; ++i) pos[i] = (unsigned)tok[i] % (unsigned)p.rope_seq;
  }
  const long ldc = p.ldc;
#pragma unroll
  for (int j = 0; j < TN; ++j) {
    const int c = col[j];
    if (c >= p.n) continue;
    float v[TM][W];
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
      for (int e = 0; e < W; ++e) v[i][e] = value(i, j, e);
    if (c32) {
#pragma unroll
      for (int h = 0; h < W; h += 4)
        if (c + h < p.c32_cols) {
#pragma unroll
          for (int i = 0; i < TM; ++i)
            if (live[i])
              *reinterpret_cast<f32x4*>(c32 + (long)tok[i] * p.c32_cols + c + h) =
                  f32x4{v[i][h], v[i][h + 1], v[i][h + 2], v[i][h + 3]};
        }
    }
    const int seg = (c >= p.seg_n) + (c >= 2 * p.seg_n);
    bf16_t* cbase = seg == 0 ? p.c0 : (seg == 1 ? p.c1 : p.c2);
    if (!cbase) continue;
    cbase += c - seg * p.seg_n;
    if (p.rope) {
#pragma unroll
      for (int h = 0; h < W; h += 4)
        if (c + h < p.rope_cols) {
          const float* table = p.rope + (((unsigned)(c + h) % (unsigned)p.rope_dh) >> 1) * 2;
          f32x4 cs[TM];
#pragma unroll
          for (int i = 0; i < TM; ++i) cs[i] = *reinterpret_cast<const f32x4*>(table + (long)pos[i] * p.rope_dh);
#pragma unroll
          for (int i = 0; i < TM; ++i) rope_rotate4(cs[i], v[i][h], v[i][h + 1], v[i][h + 2], v[i][h + 3]);
        }
    }
#pragma unroll
    for (int i = 0; i < TM; ++i) {
      out_t o;
#pragma unroll
      for (int e = 0; e < W; ++e) o[e] = (bf16_t)v[i][e];
      if (live[i]) *reinterpret_cast<out_t*>(cbase + tok[i] * ldc) = o;
    }
  }
}

// Tile order: GROUP_M row-tiles per column step (the tiles that run at the same time on one
// XCD then share few distinct A and W tiles).
__device__ __forceinline__ void tile_of_unit(const int unit, const int tiles_m, const int tiles_n, int& tile_m,
                                             int& tile_n) {
  const int group_size = GROUP_M * tiles_n;
  const int first_m = (unit / group_size) * GROUP_M;
  const int rows_in_group = tiles_m - first_m < GROUP_M ? tiles_m - first_m : GROUP_M;
  const int rem = unit % group_size;
  tile_m = first_m + rem % rows_in_group;
  tile_n = rem / rows_in_group;
}

// Tiles that the CUs get one of, or few: eight waves, v_mfma_f32_16x16x32_bf16 (wave tiles in units of
// 16, so that eight waves can share a 128 x 96 tile: 129-256 refreshed rows of a 12288-wide output then
// make 256 workgroups of 8 waves, where the 32-wide shape allows 192 workgroups of 128 x 128).  LDS
// layout as in gemm_tile; a fragment is 16 rows x 32 k (lane L: row L & 15, k-chunk L >> 4), a k-step
// holds two such slices, and all fragments of the next k-step are fetched under the MFMAs of the
// current one.  vblock is the workgroup's (virtual) block id: one that walks several tiles calls this
// once per pass with block id + pass * grid size; the result says whether that id held a tile.
// What bounds it is the pull of a CU: the operands come at most at 64 B per cycle, at 100 GB/s where
// lines come from beyond the L2 (1024 x 4096 x 4096: loads alone 26 us of 33, MFMAs alone 20).  So the whole ring is
// kept in flight (the stage of k-step kt is filled again for kt + STAGES as soon as the barrier says that its
// fragments are in registers) and the loads of a k-step are issued one by one between its MFMAs: in a
// row, a wave that waits for a place in the queue keeps its MFMAs waiting as well.  us, before (STAGES - 1
// stages in flight, loads in a row, 32-wide MFMAs for 128 x 128, the epilogue before store_tile) and now, weights in the
// last-level cache: all rows, 1024 x 4096 x 4096 41.3 and 36.3, 512 x 8192 41.5 and 35.3; listed rows, 205 x 12288 32.2 and
// 31.4 (weights from HBM 39.4 and 37.6), 205 x 4096 16.7 and 16.4, 512 x 8192 43.3 and 37.1, but 100 x 12288 (128 x 48) 23.1
// and 23.8.  (The order of a sum over k is that of the instruction: 128 x 128 tiles sum 32 products at a time where they
// summed 16, results differ from then by single bf16 roundings.)  The k of a k-step halved
// between two groups of four waves with twice the wave tile (half the fragment reads) is no faster.
// Some waves repeat the last group of rows (128 x 96: 32 loads for 28 groups).
template <int BM, int BN, int WAVES_M, int WAVES_N, int STAGES, bool LINEAR = false, class Op = Bf16Op>
__device__ __forceinline__ bool gemm_tile16(const typename Op::Dev& p, const int m, unsigned char* smem, const int tid,
                                            const int vblock, lds_idx_t lidx = nullptr,
                                            const int forced_tile_m = -1, const int forced_tile_n = 0) {
  constexpr int NW = WAVES_M * WAVES_N;
  constexpr int WM = BM / WAVES_M, WN = BN / WAVES_N;
  constexpr int TM = WM / 16, TN = WN / 16;
  constexpr int STAGE_BYTES = (BM + BN) * ROW_BYTES;
  constexpr int GROUPS = (BM + BN) / 8;
  constexpr int LPW = (GROUPS + NW - 1) / NW;  // surplus loads repeat the last group
  constexpr int KS = BK / 32;
  static_assert(WM % 16 == 0 && WN % 16 == 0, "wave tile must be a multiple of 16 x 16");
  static_assert(STAGES >= 3 && LPW * (STAGES - 1) < 64, "vmcnt range");

  const int tiles_m = (m + BM - 1) / BM, tiles_n = (p.n + BN - 1) / BN;
  int tile_m, tile_n;
  if (forced_tile_m >= 0) {  // the caller names the tile
    tile_m = forced_tile_m;
    tile_n = forced_tile_n;
  } else {
    const int total = tiles_m * tiles_n;
    const int per_xcd = (total + 7) >> 3;
    const int slot = vblock >> 3;
    if (slot >= per_xcd) return false;
    const int unit = (vblock & 7) * per_xcd + slot;
    if (unit >= total) return false;
    tile_of_unit(unit, tiles_m, tiles_n, tile_m, tile_n);
  }
  const int m0 = tile_m * BM, n0 = tile_n * BN;

  // (the wave number as a scalar: LDS addresses of the global -> LDS loads go through M0, and a
  // wave number held in a vector register would send every one of them through v_readfirstlane)
  const int lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wave_m = wave % WAVES_M, wave_n = wave / WAVES_M;
  const int l16 = lane & 15, kq = lane >> 4;
  const int KT = p.k / BK;

  const bf16_t* src[LPW];
  int grp[LPW], row_in[LPW], tok_in[LPW];
#pragma unroll
  for (int i = 0; i < LPW; ++i) {
    grp[i] = wave * LPW + i < GROUPS ? wave * LPW + i : GROUPS - 1;
    const int row = m0 + grp[i] * 8 + (lane >> 3);
    row_in[i] = row < m ? row : m - 1;
  }
  row_tokens(p.idx, lidx, row_in, tok_in);
#pragma unroll
  for (int i = 0; i < LPW; ++i) {
    const int r = grp[i] * 8 + (lane >> 3);
    const int chunk = (lane & 7) ^ ((r >> 1) & 7);
    if (r < BM) {
      src[i] = p.a + (long)tok_in[i] * p.lda + chunk * 8;
    } else {
      int col = n0 + (r - BM);
      col = col < p.n ? col : p.n - 1;
      src[i] = p.wt + (long)col * p.k + chunk * 8;
    }
  }
  int row_out[TM], tok_out[TM];
  bool live_out[TM];
#pragma unroll
  for (int i = 0; i < TM; ++i) {
    const int row = m0 + wave_m * WM + i * 16 + l16;
    live_out[i] = row < m;
    row_out[i] = row < m ? row : m - 1;
  }
  row_tokens(p.idx, lidx, row_out, tok_out);
  // TRIM: nothing is loaded past the last k-step (steps of 1 x 1024 x 4096, half of the tokens refreshed: 155.5 ->
  // 154.2 us).  Otherwise the loads of k-steps past the end repeat the last one, into a stage that nobody reads any
  // more, so that one loop with one wait serves all k-steps: the last ones of a small tile take less than
  // fetching code of their own does (2 x 201 x 512 28.4 us as it is and 29.6 with TRIM, 4 of 1024 rows 61.0 and 62.5).
  constexpr bool TRIM = TM * TN >= 6;
  auto issue_load = [&](int i, int kt) __attribute__((always_inline)) {
    const int k = TRIM || kt < KT ? kt : KT - 1;
    __builtin_amdgcn_global_load_lds((gptr_t)(src[i] + k * BK),
                                     (lptr_t)(smem + (kt % STAGES) * STAGE_BYTES + grp[i] * 8 * ROW_BYTES), 16, 0, 0);
  };

  typename Op::Acc acc[TM][TN];
#pragma unroll
  for (int i = 0; i < TM; ++i)
#pragma unroll
    for (int j = 0; j < TN; ++j) acc[i][j] = typename Op::Acc{0, 0, 0, 0};

  // fragment offsets: row (base + 16 i + l16), chunk 4 ks + kq at slot chunk ^ ((row >> 1) & 7); the
  // bases are multiples of 16, so the XOR term depends on l16 only
  const int sw = (l16 >> 1) & 7;
  int koff[KS];
#pragma unroll
  for (int ks = 0; ks < KS; ++ks) koff[ks] = ((ks * 4 + kq) ^ sw) * 16;
  const int a_row_off = (wave_m * WM + l16) * ROW_BYTES;
  const int b_row_off = (BM + wave_n * WN + l16) * ROW_BYTES;

  typedef typename Op::Frag Frag;
  Frag fa[2][KS][TM], fb[2][KS][TN];
  auto load_frags = [&](int kt, int set) __attribute__((always_inline)) {
    const unsigned char* st = smem + (kt % STAGES) * STAGE_BYTES;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
#pragma unroll
      for (int i = 0; i < TM; ++i)
        fa[set][ks][i] = *reinterpret_cast<const Frag*>(st + a_row_off + i * 16 * ROW_BYTES + koff[ks]);
#pragma unroll
      for (int j = 0; j < TN; ++j)
        fb[set][ks][j] = *reinterpret_cast<const Frag*>(st + b_row_off + j * 16 * ROW_BYTES + koff[ks]);
    }
  };
  constexpr int NMMA = KS * TM * TN, PRE = NMMA / 4 > 0 ? NMMA / 4 : 1;
  auto mma = [&](int set, int first, int last) __attribute__((always_inline)) {
#pragma unroll
    for (int t = 0; t < NMMA; ++t) {
      if (t < first || t >= last) continue;
      const int ks = t / (TM * TN), i = (t / TN) % TM, j = t % TN;
      acc[i][j] = Op::mfma(fb[set][ks][j], fa[set][ks][i], acc[i][j]);
    }
  };

#pragma unroll
  for (int s = 0; s < STAGES; ++s)
    if (!TRIM || s < KT) {
#pragma unroll
      for (int i = 0; i < LPW; ++i) issue_load(i, s);
    }
  wait_stages_and_barrier<LPW, STAGES - 1>(TRIM ? KT - 1 : STAGES - 1);
  load_frags(0, 0);
  // k-step kt: the barrier publishes stage kt + 1 and, as every wave's fragments of kt have arrived, frees
  // the stage of kt.  (Two k-steps per trip so that the fragment set index is a compile-time constant.)
  // END: one of the last k-steps, which has nothing left to load and waits for as many loads as are under way.
  auto kstep = [&](int kt, auto set_c, auto end_c) __attribute__((always_inline)) {
    constexpr int SET = decltype(set_c)::value;
    constexpr bool END = decltype(end_c)::value;
    mma(SET, 0, PRE);
    __builtin_amdgcn_sched_barrier(0);
    if (!END || kt + 1 < KT) {
      if constexpr (END)
        wait_stages_and_barrier<LPW, STAGES - 2>(KT - 2 - kt);
      else
        wait_vmcnt_and_barrier<LPW*(STAGES - 2)>();
      __builtin_amdgcn_sched_barrier(0);
      load_frags(kt + 1, SET ^ 1);
    }
    __builtin_amdgcn_sched_barrier(0);
    if constexpr (END) {
      mma(SET, PRE, NMMA);
    } else {
#pragma unroll
      for (int i = 0; i < LPW; ++i) {
        mma(SET, PRE + (NMMA - PRE) * i / LPW, PRE + (NMMA - PRE) * (i + 1) / LPW);
        __builtin_amdgcn_sched_barrier(0);
        issue_load(i, kt + STAGES);
        __builtin_amdgcn_sched_barrier(0);
      }
    }
  };
  using Yes = std::true_type;
  using No = std::false_type;
  using Set0 = std::integral_constant<int, 0>;
  using Set1 = std::integral_constant<int, 1>;
  int kt = 0;
  const int loading = TRIM ? KT - STAGES : KT;
  for (; kt + 1 < loading; kt += 2) {
    kstep(kt, Set0{}, No{});
    kstep(kt + 1, Set1{}, No{});
  }
  if constexpr (!TRIM) {
    if (kt < KT) kstep(kt, Set0{}, No{});
    kt = KT;
  } else if (kt < loading) {  // an odd number of k-steps load: the last ones begin with set 1
    kstep(kt, Set0{}, No{});
    kstep(++kt, Set1{}, Yes{});
    ++kt;
  }
  for (; kt < KT; kt += 2) {
    kstep(kt, Set0{}, Yes{});
    if (kt + 1 < KT) kstep(kt + 1, Set1{}, Yes{});
  }
  wait_vmcnt<0>();

  // acc[i][j][e] = C[row, col]: row = m0 + wave_m*WM + 16 i + l16, col = n0 + wave_n*WN + 16 j + 4 kq + e
  int col[TN];
#pragma unroll
  for (int j = 0; j < TN; ++j) col[j] = n0 + wave_n * WN + j * 16 + kq * 4;
  auto value = [&](int i, int j, int e) __attribute__((always_inline)) { return (float)acc[i][j][e]; };
  if constexpr (Op::kScaled)
    Op::template store<4>(p, tok_out, live_out, col, value);
  else if constexpr (LINEAR)
    store_linear<4>(p, tok_out, live_out, col, value);
  else
    store_tile<4>(p, p.c32, tok_out, live_out, col, value);
  return true;
}

// chunk XOR of row r of a 32-row weight block
__device__ __forceinline__ int pp_bkey(int r) { return ((r >> 1) & 1) | (((r >> 3) & 3) << 1); }

// ---- several rounds of large tiles of all rows: 256 x (64 TN), four waves, one per SIMD ----
// A wave owns 128 rows x 32 TN columns, its sums in the accumulator registers, which leaves the others to two sets of
// fragments: a slice of 32 k is multiplied while the next one's fragments are read.  Against gemm_tile_pp, whose eight waves take 64
// rows each: a third fewer bytes read from LDS per k-step (131 KB for 196), one barrier for eight, and what these kernels are bound
// by, power, goes with both (a 256 x 256 tile with 192 k-steps, random operands: 278 us, without the loads into LDS 224, without the
// fragment reads 250, with neither 201).
//   * One instruction stream.  A read every three MFMAs, a load every eight (TN = 4), the address of a load one MFMA later, nothing
//     between two MFMAs that takes longer than one.  The MFMAs are inline assembly: the compiler, which may put the sums into either kind of
//     registers, moved 400 of them per k-step.  It does not know these as MFMAs, so their results wait by hand (s_nop).
//   * LDS: half-stages A(0), B(0), A(1), B(1), .. of a k-step each through a ring of five slots, 160 KB.  The barrier of a
//     k-step lies between its two slices: every wave has read A(kt) and B(kt), and A(kt + 1) and B(kt + 1) have landed.  In front of
//     it A(kt + 2) is loaded (into the slot of B(kt - 1)), behind it B(kt + 2) (into that of A(kt)): a load has one to three
//     slices of 1024 cycles to arrive; never waiting for any is no faster.
//   * The pipeline runs on from tile to tile: a workgroup per CU walks its tiles, the last two k-steps load the next tile's
//     first two and the last slice reads its first fragments, so a tile ends without an empty ring.  Behind the last tile they
//     load their own k-steps again, into slots that nobody reads: the same code, where code of its own for the end and the start, fetched
//     once per launch, cost a launch of one round 3 us.
//   * Stores of whole 128-byte lines: rows 0 .. 7 of a block of 16 in one store and 8 .. 15 in the next, two column blocks side
//     by side (lanes L and L ^ 8 swap halves).  Stores count in vmcnt with the loads, in order, and the loads of the next tile
//     wait for them: with 64-byte runs they took 9 us per round of the CUs.
// The sum over k is formed as in gemm_tile_pp and gemm_tile16, so results are the same bits.
// us, gemm_tile_pp (256 x 192 and 256) and now, one card: 16384 x 12288 x 4096 1148 and 1076 (1.53 PFLOP/s), 16384 x 4096 x 4096 384 and 362,
// 4096 x 24576 x 4096 608 and 541, 4096 x 4096 x 12288 272 and 262, 2331 x 12288 x 4096 184 and 177, with operands in the caches.
// In steps, where they come from other kernels and from memory: 4096 x 24576 with
// the gate 570 and 547, 8192 x 24576 1123 and 1079, 4096 x 4096 x 12288 277 and 270, Q, K and V of 4096 rows, rotated, 314 and 297;
// one round is better off with eight waves (four_waves, gemm_route.h).
// The gate of 128 x 128 sums takes a wave 2.8 us (with the compiler's division 5.5), the rotation 2.
// gemm_tile_pp stays for 256 x 128 (gemm_bf16_pp_kernel), for one round, where k is cut over two workgroups (1024 x 4096 x 12288 92.6 us, in this form 103.6: half as many waves store and add
// the sums) and for listed rows, whose kernel has the eight waves that the small shapes want.
constexpr int kQuadSlot = kPpRows * ROW_BYTES, kQuadSmem = 5 * kQuadSlot;

// Value of a lane from the lane 8 further on in its row of 16, in the lanes of BANKS (four lanes each); `own` in the others
template <int BANKS>
__device__ __forceinline__ unsigned from_half_row(unsigned own, unsigned other) {
  return __builtin_amdgcn_update_dpp(own, other, 0x128, 0xf, BANKS, false);
}
// STREAM: past the L2
template <bool STREAM>
__device__ __forceinline__ void store16(bf16_t* to, const u32x4 v) {
  if constexpr (STREAM)
    __builtin_nontemporal_store(v, reinterpret_cast<u32x4*>(to));
  else
    *reinterpret_cast<u32x4*>(to) = v;
}

// The tiles blockIdx.x, blockIdx.x + gridDim.x, ..; called by all 256 threads.  k of kQuadMinSteps k-steps or more (loads two ahead, and
// the first one's zero sums).
// PART: the columns from part_n on for all rows, those in front of it for the part_m rows of the second list.
// LINEAR: act(sums + bias) + residual.
template <int TN, bool STREAM, bool PART = false, bool LINEAR = false, class Op = Bf16Op>
__device__ __forceinline__ void gemm_tiles_quad(const typename Op::Dev& p, const int m, unsigned char* smem, const int part_m = 0) {
  static_assert(TN == 3 || TN == 4, "column blocks of 32 per wave");
  constexpr int BM = kPpRows, BN = 64 * TN;
  constexpr int SLOT = kQuadSlot;
  constexpr int AL = BM / 8 / 4, BL = BN / 8 / 4;  // loads of a wave per half-stage
  constexpr int NA = 8, NB = 2 * TN;               // fragments of a slice
  constexpr int NM = NA * NB, NR = NA + NB;        // its MFMAs and reads

  const int first_n = PART ? p.part_n : 0;
  const int tiles_m = (m + BM - 1) / BM, tiles_n = (p.n - first_n + BN - 1) / BN, all = tiles_m * tiles_n;
  const int part_tiles_m = (part_m + BM - 1) / BM, part_tiles_n = (first_n + BN - 1) / BN;
  const int total = all + part_tiles_m * part_tiles_n;
  const int per_xcd = (total + 7) >> 3;
  int vb = blockIdx.x, m0, n0;
  int rows_end = m, cols_end = p.n;     // of the tile's list and columns
  const int32_t* list = p.idx;
  auto place = [&]() __attribute__((always_inline)) {
    const int slot = vb >> 3, unit = (vb & 7) * per_xcd + slot;
    if (slot >= per_xcd || unit >= total) return false;
    int tile_m, tile_n;
    if (!PART || unit < all) {
      tile_of_unit(unit, tiles_m, tiles_n, tile_m, tile_n);
      n0 = first_n + tile_n * BN;
    } else {
      tile_of_unit(unit - all, part_tiles_m, part_tiles_n, tile_m, tile_n);
      n0 = tile_n * BN;
      rows_end = part_m;
      cols_end = first_n;
      list = p.part_idx;
    }
    m0 = tile_m * BM;
    return true;
  };
  if (!place()) return;

  const int tid = threadIdx.x;
  const int lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm = wave & 1, wn = wave >> 1;
  const int l16 = lane & 15, kq = lane >> 4;
  const int KT = p.k / BK;

  // the rows of this lane's loads
  int tok_in[AL];
  auto rows = [&]() __attribute__((always_inline)) {
    int row_in[AL];
#pragma unroll
    for (int i = 0; i < AL; ++i) {
      const int row = m0 + (wave * AL + i) * 8 + (lane >> 3);
      row_in[i] = row < rows_end ? row : rows_end - 1;
    }
    row_tokens(Op::kScaled ? nullptr : list, nullptr, row_in, tok_in);
  };
  const bf16_t* src_a[AL];
  const bf16_t* src_b[BL];
  auto addresses = [&]() __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < AL; ++i) {
      const int r = (wave * AL + i) * 8 + (lane >> 3);
      src_a[i] = p.a + (long)tok_in[i] * p.lda + ((lane & 7) ^ ((r >> 1) & 7)) * 8;
    }
#pragma unroll
    for (int j = 0; j < BL; ++j) {
      const int r = (wave * BL + j) * 8 + (lane >> 3);
      const int col = n0 + r < cols_end ? n0 + r : cols_end - 1;
      src_b[j] = p.wt + (long)col * p.k + ((lane & 7) ^ pp_bkey(r & 31)) * 8;
    }
  };
  const unsigned lds0 = (unsigned)(size_t)(lptr_t)smem;
  // (the address is an operand in M0, set by the compiler, which then knows what M0 holds; a wait state, or an MFMA,
  // between the move to M0 and the load)
  auto load = [&](const bf16_t*& src, unsigned lds) __attribute__((always_inline)) {
    asm volatile("s_nop 0\n\tglobal_load_lds_dwordx4 %0, off" ::"v"(src), "{m0}"(lds) : "memory");
    src += BK;
  };

  typedef typename Op::Frag Frag;
  typename Op::Acc acc[NA][NB];
  int a_off[2], b_off[2];
  const int brow = (l16 >> 2) * 8 + (l16 & 3);
#pragma unroll
  for (int ks = 0; ks < 2; ++ks) {
    a_off[ks] = (wm * 128 + l16) * ROW_BYTES + ((ks * 4 + kq) ^ ((l16 >> 1) & 7)) * 16;
    b_off[ks] = (wn * 32 * TN + brow) * ROW_BYTES + ((ks * 4 + kq) ^ pp_bkey(brow)) * 16;
  }
  Frag fa[2][NA], fb[2][NB];
  typedef const __attribute__((address_space(3))) Frag* lds_frag_t;
  // read n of a slice: the first column's fragment, the rows', the other columns'
  auto read = [&](auto ks_c, int n, unsigned at_a, unsigned at_b) __attribute__((always_inline)) {
    constexpr int ks = decltype(ks_c)::value;
    if (n >= 1 && n <= NA)
      fa[ks][n - 1] = *(lds_frag_t)(at_a + (n - 1) * 16 * ROW_BYTES);
    else {
      const int j = n == 0 ? 0 : n - NA;
      fb[ks][j] = *(lds_frag_t)(at_b + (j >> 1) * 32 * ROW_BYTES + (j & 1) * 4 * ROW_BYTES);
    }
  };
  // the MFMAs of a slice with the next slice's reads and the loads of a half-stage between them
  auto slice = [&](auto ks_c, auto zero_c, auto n_loads, const bf16_t** src, unsigned to, int at_a, int at_b) __attribute__((always_inline)) {
    constexpr int ks = decltype(ks_c)::value, NL = decltype(n_loads)::value;
    const unsigned ra = lds0 + at_a + a_off[ks ^ 1], rb = lds0 + at_b + b_off[ks ^ 1];
    constexpr int RS = NM / NR < 3 ? NM / NR : 3, LS = NM / NL;  // MFMAs per read, per load
    static_assert(RS * NR <= NM && LS > 3, "every fragment must have its read, every load its place");
#pragma unroll
    for (int t = 0; t < NM; ++t) {
      const int j = t / NA, i = t % NA;
      const int l = t / LS;
      const bool loads = t % LS == 2 && l < NL;
#define DARE_MFMA(out, name, sum, tail, ...) asm volatile(name " %0, %1, %2, " sum tail : out(acc[i][j]) : "v"(fb[ks][j]), "v"(fa[ks][i])__VA_ARGS__)
#define DARE_STEP(name)                                                                                                             \
  if constexpr (decltype(zero_c)::value) {                                                                                          \
    if (loads)                                                                                                                      \
      DARE_MFMA("=a", name, "0", "\n\tglobal_load_lds_dwordx4 %3, off", , "v"(src[l]), "{m0}"(to + l * 1024) : "memory");           \
    else                                                                                                                            \
      DARE_MFMA("=a", name, "0", "");                                                                                               \
  } else {                                                                                                                          \
    if (loads)                                                                                                                      \
      DARE_MFMA("+a", name, "%0", "\n\tglobal_load_lds_dwordx4 %3, off", , "v"(src[l]), "{m0}"(to + l * 1024) : "memory");          \
    else                                                                                                                            \
      DARE_MFMA("+a", name, "%0", "");                                                                                              \
  }
      if constexpr (Op::kScaled) {
        DARE_STEP("v_mfma_i32_16x16x64_i8")
      } else {
        DARE_STEP("v_mfma_f32_16x16x32_bf16")
      }
#undef DARE_STEP
#undef DARE_MFMA
      __builtin_amdgcn_sched_barrier(0);
      if (t % RS == 0 && t / RS < NR) {
        read(std::integral_constant<int, ks ^ 1>{}, t / RS, ra, rb);
        __builtin_amdgcn_sched_barrier(0);
      }
      if (t % LS == 3 && l < NL) {  // (next to an MFMA of its own)
        src[l] += BK;
        __builtin_amdgcn_sched_barrier(0);
      }
    }
  };
#define DARE_N(n) std::integral_constant<int, n>{}
  using Yes = std::true_type;
  using No = std::false_type;
  auto wrap = [](int at) __attribute__((always_inline)) { return at >= 5 * SLOT ? at - 5 * SLOT : at; };
  int at = 0;  // slot of A(kt)
  auto kstep = [&](auto zero_c) __attribute__((always_inline)) {
    const int b0 = wrap(at + SLOT), a1 = wrap(at + 2 * SLOT), b1 = wrap(at + 3 * SLOT), a2 = wrap(at + 4 * SLOT);
    slice(DARE_N(0), zero_c, DARE_N(AL), src_a, lds0 + a2 + wave * AL * 1024, at, b0);
    wait_vmcnt_and_barrier<AL>();
    __builtin_amdgcn_sched_barrier(0);
    slice(DARE_N(1), No{}, DARE_N(BL), src_b, lds0 + at + wave * BL * 1024, a1, b1);
    at = a1;
  };

  rows();
  addresses();
#pragma unroll
  for (int k = 0; k < 2; ++k) {
#pragma unroll
    for (int i = 0; i < AL; ++i) load(src_a[i], lds0 + 2 * k * SLOT + (wave * AL + i) * 1024);
#pragma unroll
    for (int j = 0; j < BL; ++j) load(src_b[j], lds0 + (2 * k + 1) * SLOT + (wave * BL + j) * 1024);
  }
#pragma unroll
  for (int i = 0; i < NA; ++i)
#pragma unroll
    for (int j = 0; j < NB; ++j) {
      acc[i][j] = typename Op::Acc{0, 0, 0, 0};
      asm volatile("" : "+a"(acc[i][j]));
    }
  wait_vmcnt_and_barrier<AL + BL>();
#pragma unroll
  for (int n = 0; n < NR; ++n) read(DARE_N(0), n, lds0 + a_off[0], lds0 + SLOT + b_off[0]);
  __builtin_amdgcn_sched_barrier(0);
  for (int kt = 0;;) {
    int row_out[NA], tok[NA];
    bool live[NA];
#pragma unroll
    for (int i = 0; i < NA; ++i) {
      const int row = m0 + wm * 128 + i * 16 + l16;
      live[i] = row < rows_end;
      row_out[i] = row < rows_end ? row : rows_end - 1;
    }
    row_tokens(Op::kScaled ? nullptr : list, nullptr, row_out, tok);
    const int col0 = n0 + wn * (32 * TN), n_end = cols_end;
    vb += gridDim.x;
    const bool more = place();
    if (more) rows();
    for (; kt < KT; ++kt) {
      if (kt == KT - 2) {
        if (more) {
          addresses();
        } else {  // the last two k-steps again, into slots that nobody reads
#pragma unroll
          for (int i = 0; i < AL; ++i) src_a[i] -= 2 * BK;
#pragma unroll
          for (int j = 0; j < BL; ++j) src_b[j] -= 2 * BK;
        }
      }
      kstep(No{});
    }
    // (what the compiler would know of MFMAs of its own: their results are there 18 cycles later)
    asm volatile("s_nop 15\n\ts_nop 15" ::: "memory");
    auto value = [&](int i, int j, int e) __attribute__((always_inline)) {
      std::conditional_t<Op::kScaled, int, float> v;
      asm volatile("v_accvgpr_read_b32 %0, %1" : "=v"(v) : "a"(acc[i][j * 2 + (e >> 2)][e & 3]));
      return (float)v;
    };
    // acc[i][2 j + h][e] = C[row, col], row = m0 + 128 wm + 16 i + l16, col = col0 + 32 j + 8 kq + 4 h + e
    const bool low = l16 < 8;
    if constexpr (Op::kScaled) {
      float row_scale[NA];
#pragma unroll
      for (int i = 0; i < NA; ++i) row_scale[i] = p.row_scale[tok[i]];
      // Two column blocks after the other, each with all rows: what belongs to a column (scale, bias) is held for two blocks and not
      // for all, which would be 74 registers more than there are.  The rows' scales and residuals a row of the tile ahead.
      const long ldc = p.ldc;
#pragma unroll
      for (int j = 0; j < TN; j += 2) {
        constexpr int H = 2;
        f32x4 col_scale[H][2];
        bf16x8 bias[H], res[2][H];
        int at_col[H];
#pragma unroll
        for (int h = 0; h < H; ++h)
          if (j + h < TN) {
            const int c = col0 + (j + h) * 32 + kq * 8;
            at_col[h] = c < n_end ? c : n_end - 8;  // (columns behind the last one read the last ones, nobody stores them)
            const f32x4* scale = reinterpret_cast<const f32x4*>(p.col_scale + at_col[h]);
            col_scale[h][0] = scale[0];
            col_scale[h][1] = scale[1];
            bias[h] = p.bias ? *reinterpret_cast<const bf16x8*>(p.bias + at_col[h]) : bf16x8{};
          }
        auto ahead = [&](int i) __attribute__((always_inline)) {
          const bf16_t* row = p.residual + tok[i] * p.ldr;
#pragma unroll
          for (int h = 0; h < H; ++h)
            if (j + h < TN) res[i & 1][h] = *reinterpret_cast<const bf16x8*>(row + at_col[h]);
        };
        if (p.residual) ahead(0);
        const bool pair = j + 1 < TN;
        const int c = col0 + j * 32 + (pair && !low ? 32 : 0);
        bf16_t* to = c >= n_end ? nullptr : p.c0 + c + kq * 8;
#pragma unroll
        for (int i = 0; i < NA; ++i) {
          const int other = from_half_row<0xf>(0, tok[i]);
          const bool live_other = from_half_row<0xf>(0, live[i]) != 0;
          const long own = tok[i] * ldc, far = other * ldc;
          if (p.residual && i + 1 < NA) ahead(i + 1);
          __builtin_amdgcn_sched_barrier(0);
          u32x4 o[H];
#pragma unroll
          for (int h = 0; h < H; ++h)
            if (j + h < TN) {
              float v[8];
              bf16x8 r;
#pragma unroll
              for (int e = 0; e < 8; ++e)
                v[e] = fmaf(value(i, j + h, e) * row_scale[i], col_scale[h][e >> 2][e & 3], (float)bias[h][e]);
              activate<true>(p.act, v);
              if (p.residual) {
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] += (float)res[i & 1][h][e];
              }
#pragma unroll
              for (int e = 0; e < 8; ++e) r[e] = (bf16_t)v[e];
              o[h] = __builtin_bit_cast(u32x4, r);
            }
          if (pair) {
            u32x4 x, y;
#pragma unroll
            for (int q = 0; q < 4; ++q) {
              x[q] = from_half_row<0xc>(o[0][q], o[1][q]);
              y[q] = from_half_row<0x3>(o[1][q], o[0][q]);
            }
            if (to && (low ? live[i] : live_other)) store16<STREAM>(to + (low ? own : far), x);
            if (to && (low ? live_other : live[i])) store16<STREAM>(to + (low ? far : own), y);
          } else if (to && live[i]) {
            store16<STREAM>(to + own, o[0]);
          }
        }
      }
    } else if (!PART && !LINEAR && p.swiglu_pairs) {
      const long ldc = p.ldc;
#pragma unroll
      for (int i = 0; i < NA; ++i) {
        u32x2 o[TN];
        float q[TN][4];
        unsigned lowest = 0;  // as bits: of two negative floats the lower one has the larger bits
#pragma unroll
        for (int j = 0; j < TN; ++j)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float g = value(i, j, 2 * e);
            lowest = max(lowest, __float_as_uint(g));
            q[j][e] = silu<false>(g);
          }
        // (scaled where some lane needs it: scaling every gate made model steps of 1430, 3609 and 3940 us 12, 16 and 19 us longer;
        // traced, 1024 x 24576 x 4096 with the gate takes 149.8 us without this and 149.5 with it)
        if (__builtin_expect(__any(lowest > __float_as_uint(kGateLow)), 0)) {
#pragma unroll
          for (int j = 0; j < TN; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) q[j][e] = silu(value(i, j, 2 * e));
        }
#pragma unroll
        for (int j = 0; j < TN; ++j) {
          bf16x4 r;
#pragma unroll
          for (int e = 0; e < 4; ++e) r[e] = (bf16_t)(q[j][e] * value(i, j, 2 * e + 1));
          o[j] = __builtin_bit_cast(u32x2, r);
        }
        // lanes kq and kq ^ 1 share two column blocks: 16 bytes of one of them each
        u32x4 w[TN / 2];
#pragma unroll
        for (int j = 0; j + 1 < TN; j += 2)
#pragma unroll
          for (int q = 0; q < 2; ++q) {
            const auto sw = __builtin_amdgcn_permlane16_swap(o[j][q], o[j + 1][q], false, false);
            w[j / 2][q] = sw[0];
            w[j / 2][q + 2] = sw[1];
          }
        bf16_t* own = p.c0 + tok[i] * ldc + (col0 >> 1);
        const int at_col = (kq & 1) * 16 + (kq >> 1) * 8;
        if constexpr (TN == 4) {
          const int other = from_half_row<0xf>(0, tok[i]);
          const bool live_other = from_half_row<0xf>(0, live[i]) != 0;
          u32x4 x, y;
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            x[q] = from_half_row<0xc>(w[0][q], w[1][q]);
            y[q] = from_half_row<0x3>(w[1][q], w[0][q]);
          }
          bf16_t* far = p.c0 + other * ldc + (col0 >> 1);
          const int c = at_col + (low ? 0 : 32);
          const bool in = col0 + (low ? 0 : 64) < n_end;
          if (in && (low ? live[i] : live_other)) store16<STREAM>((low ? own : far) + c, x);
          if (in && (low ? live_other : live[i])) store16<STREAM>((low ? far : own) + c, y);
        } else {
          if (live[i] && col0 + (kq & 1) * 32 < n_end) store16<STREAM>(own + at_col, w[0]);
          if (live[i] && col0 + 64 < n_end) *reinterpret_cast<u32x2*>(own + 32 + kq * 4) = o[TN - 1];
        }
      }
    } else {
      // (LINEAR: the residual's rows a row of the tile ahead; columns behind the last one read the last ones, nobody stores them)
      bf16x8 bias[LINEAR ? TN : 1], res[2][LINEAR ? TN : 1];
      int at_col[LINEAR ? TN : 1];
      auto residual = [&](int i) __attribute__((always_inline)) {
        const bf16_t* row = p.residual + tok[i] * p.ldr;
#pragma unroll
        for (int j = 0; j < TN; ++j) res[i & 1][j] = *reinterpret_cast<const bf16x8*>(row + at_col[j]);
      };
      if constexpr (LINEAR) {
#pragma unroll
        for (int j = 0; j < TN; ++j) {
          const int c = col0 + j * 32 + kq * 8;
          at_col[j] = c < n_end ? c : n_end - 8;
          if (p.bias) bias[j] = *reinterpret_cast<const bf16x8*>(p.bias + at_col[j]);
        }
        if (p.residual) residual(0);
      }
      if (!PART && !LINEAR && p.c32 && col0 < p.c32_cols) {
#pragma unroll
        for (int i = 0; i < NA; ++i)
#pragma unroll
          for (int j = 0; j < NB; ++j) {
            const int c = col0 + (j >> 1) * 32 + kq * 8 + (j & 1) * 4;
            f32x4 v;
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = value(i, j >> 1, (j & 1) * 4 + e);
            if (live[i] && c < p.c32_cols) *reinterpret_cast<f32x4*>(p.c32 + (long)tok[i] * p.c32_cols + c) = v;
          }
      }
      if (!LINEAR && p.rope && col0 < p.rope_cols) {
        // (the table's rows a row of the tile ahead of their use; columns that are not rotated read one that is)
        f32x4 cs[2][NB];
        auto table = [&](int i) __attribute__((always_inline)) {
          const float* row = p.rope + (long)((unsigned)tok[i] % (unsigned)p.rope_seq) * p.rope_dh;
#pragma unroll
          for (int j = 0; j < NB; ++j) {
            const int c = col0 + (j >> 1) * 32 + kq * 8 + (j & 1) * 4;
            cs[i & 1][j] = *reinterpret_cast<const f32x4*>(row + ((unsigned)(c < p.rope_cols ? c : col0) % (unsigned)p.rope_dh >> 1) * 2);
          }
        };
        table(0);
#pragma unroll
        for (int i = 0; i < NA; ++i) {
          if (i + 1 < NA) table(i + 1);
          __builtin_amdgcn_sched_barrier(0);
#pragma unroll
          for (int j = 0; j < NB; ++j) {
            const bool turns = col0 + (j >> 1) * 32 + kq * 8 + (j & 1) * 4 < p.rope_cols;
            float v[4], w[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = w[e] = value(i, j >> 1, (j & 1) * 4 + e);
            rope_rotate4(cs[i & 1][j], w[0], w[1], w[2], w[3]);
            acc[i][j] = f32x4{turns ? w[0] : v[0], turns ? w[1] : v[1], turns ? w[2] : v[2], turns ? w[3] : v[3]};
            asm volatile("" : "+a"(acc[i][j]));
          }
          __builtin_amdgcn_sched_barrier(0);
        }
      }
      // the column blocks' places: a pair's first block in the lanes of rows 0 .. 7, its second one in the others
      bf16_t* base[(TN + 1) / 2];
#pragma unroll
      for (int j = 0; j < TN; j += 2) {
        const int c = col0 + j * 32 + (j + 1 < TN && !low ? 32 : 0);
        const int seg = (c >= p.seg_n) + (c >= 2 * p.seg_n);
        bf16_t* to = c >= n_end ? nullptr : seg == 0 ? p.c0 : seg == 1 ? p.c1 : p.c2;
        base[j / 2] = to ? to + (c - seg * p.seg_n) + kq * 8 : nullptr;
      }
      const long ldc = p.ldc;
#pragma unroll
      for (int i = 0; i < NA; ++i) {
        const int other = from_half_row<0xf>(0, tok[i]);
        const bool live_other = from_half_row<0xf>(0, live[i]) != 0;
        const long own = tok[i] * ldc, far = other * ldc;
        if constexpr (LINEAR) {
          if (p.residual && i + 1 < NA) residual(i + 1);
          __builtin_amdgcn_sched_barrier(0);
        }
#pragma unroll
        for (int j = 0; j < TN; j += 2) {
          u32x4 o[2];
#pragma unroll
          for (int h = 0; h < 2; ++h)
            if (j + h < TN) {
              bf16x8 r;
              float v[8];
#pragma unroll
              for (int e = 0; e < 8; ++e) v[e] = value(i, j + h, e);
              if constexpr (LINEAR) {
                if (p.bias) {
#pragma unroll
                  for (int e = 0; e < 8; ++e) v[e] += (float)bias[j + h][e];
                }
                activate(p.act, v);
                if (p.residual) {
#pragma unroll
                  for (int e = 0; e < 8; ++e) v[e] += (float)res[i & 1][j + h][e];
                }
              }
#pragma unroll
              for (int e = 0; e < 8; ++e) r[e] = (bf16_t)v[e];
              o[h] = __builtin_bit_cast(u32x4, r);
            }
          bf16_t* to = base[j / 2];
          if (j + 1 < TN) {
            u32x4 x, y;
#pragma unroll
            for (int q = 0; q < 4; ++q) {
              x[q] = from_half_row<0xc>(o[0][q], o[1][q]);
              y[q] = from_half_row<0x3>(o[1][q], o[0][q]);
            }
            if (to && (low ? live[i] : live_other)) store16<STREAM>(to + (low ? own : far), x);
            if (to && (low ? live_other : live[i])) store16<STREAM>(to + (low ? far : own), y);
          } else if (to && live[i]) {
            store16<STREAM>(to + own, o[0]);
          }
        }
      }
    }
    if (!more) break;
    kstep(Yes{});
    kt = 1;
  }
#undef DARE_N
  wait_vmcnt<0>();
}

// ---- very few rows (at most 16 TMS): a stream over the weight matrix ------------------
// With a handful of refreshed rows (one or two tokens unmasked per denoising step) the
// projection is a matrix-vector product in disguise: what matters is that every CU pulls on
// the weight stream at once and that each weight byte is read once.  A workgroup owns 16
// output columns for the whole of k; its NW waves take contiguous ranges of k, load their
// weight and row fragments straight into registers (no LDS: a fragment is used by one wave
// only), 16 k-steps of 32 in flight per wave (8 with two row blocks), multiply with v_mfma_f32_16x16x32_bf16
// (weight fragment first, so a lane again owns one row and four neighbouring columns), and
// the partial sums of the waves are added in wave order through LDS.
template <int NW, int TMS, bool LINEAR = false, class Op = Bf16Op>
__device__ __forceinline__ void skinny_tile(const typename Op::Dev& p, const int m, unsigned char* smem, const int tid,
                                            lds_idx_t lidx = nullptr) {
  constexpr int UNR = TMS == 1 ? 16 : 8;
  // (the wave number as a scalar: LDS addresses of the global -> LDS loads go through M0, and a
  // wave number held in a vector register would send every one of them through v_readfirstlane)
  const int lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int l16 = lane & 15, kq = lane >> 4;
  const int groups = p.n >> 4;
  const int steps = p.k >> 5;
  const int spw = (steps + NW - 1) / NW;
  const int s0 = wave * spw;
  const int s1 = s0 + spw < steps ? s0 + spw : steps;
  const bf16_t* xrow[TMS];
  int row[TMS], tok[TMS];
  bool live[TMS];
#pragma unroll
  for (int t = 0; t < TMS; ++t) {
    live[t] = t * 16 + l16 < m;
    row[t] = live[t] ? t * 16 + l16 : m - 1;
  }
  row_tokens(p.idx, lidx, row, tok);
#pragma unroll
  for (int t = 0; t < TMS; ++t) xrow[t] = p.a + (long)tok[t] * p.lda + kq * 8;
  typedef typename Op::Frag Frag;
  typedef typename Op::Acc Acc;
  Acc* red = reinterpret_cast<Acc*>(smem);  // [NW][TMS][64]
  for (int grp = blockIdx.x; grp < groups; grp += gridDim.x) {
    const int n0 = grp << 4;
    const bf16_t* wrow = p.wt + (long)(n0 + l16) * p.k + kq * 8;
    Acc acc[TMS];
#pragma unroll
    for (int t = 0; t < TMS; ++t) acc[t] = Acc{0, 0, 0, 0};
    for (int s = s0; s < s1; s += UNR) {
      Frag wf[UNR], xf[TMS][UNR];
#pragma unroll
      for (int u = 0; u < UNR; ++u) {
        const bool live = s + u < s1;
        if (LINEAR && !live) {  // (nothing is loaded, and no infinity meets a zero)
          wf[u] = Frag{};
#pragma unroll
          for (int t = 0; t < TMS; ++t) xf[t][u] = Frag{};
          continue;
        }
        const int ks = (live ? s + u : s0) << 5;
        wf[u] = *reinterpret_cast<const Frag*>(wrow + ks);
#pragma unroll
        for (int t = 0; t < TMS; ++t) xf[t][u] = *reinterpret_cast<const Frag*>(xrow[t] + ks);
        if (!live) wf[u] = Frag{};
      }
#pragma unroll
      for (int u = 0; u < UNR; ++u)
#pragma unroll
        for (int t = 0; t < TMS; ++t)
          acc[t] = Op::mfma(wf[u], xf[t][u], acc[t]);
    }
    // (the wait for the MFMAs by hand: the compiler, which has to put it in front of the stores, left it out
    // here, behind a loop that a second path goes round, and three of four columns were stored too early)
#pragma unroll
    for (int t = 0; t < TMS; ++t) asm volatile("s_nop 7\n\ts_nop 1" : "+v"(acc[t]));
#pragma unroll
    for (int t = 0; t < TMS; ++t) red[(wave * TMS + t) * 64 + lane] = acc[t];
    __syncthreads();
    if (wave == 0) {
#pragma unroll
      for (int t = 0; t < TMS; ++t) {
        acc[t] = red[t * 64 + lane];
        for (int w = 1; w < NW; ++w) acc[t] += red[(w * TMS + t) * 64 + lane];
      }
      const int col[1] = {n0 + kq * 4};
      auto value = [&](int t, int, int e) __attribute__((always_inline)) { return (float)acc[t][e]; };
      if constexpr (Op::kScaled)
        Op::template store<4>(p, tok, live, col, value);
      else if constexpr (LINEAR)
        store_linear<4>(p, tok, live, col, value);
      else
        store_tile<4>(p, p.c32, tok, live, col, value);
    }
    __syncthreads();
  }
}
constexpr int kSkinnyRows = 32;

constexpr int kWideGrid = 256;  // workgroups of a launch that walks over its tiles: one per CU
int grid_for(int tiles) { return ((tiles + 7) / 8) * 8; }

}  // namespace
}  // namespace dare
