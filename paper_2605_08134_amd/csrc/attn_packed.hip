// Attention over packed sequences with shared key heads on the gfx950 matrix cores:
//     out[t, h] = sum_j w_j v_j / sum_j w_j,   w_j = exp(scale q[t, h] . k_j),   j < L(t)
// over the keys of the token's own sequence, head h / G of K and V (G = query heads per key head).  L(t) is the number of
// keys that the token sees: all of them, or those up to the end of its block of positions (attn_packed.h).
//
// Rows.  The G heads of a token read the same keys, so what a workgroup takes is rows (token, head of the group), head
// fastest, of one key head: a key that is in LDS serves G times the tokens, and single tokens fill G rows of a matrix
// instruction instead of one.  A row's keys are a prefix of its sequence, longer from token to token: a mask is needed
// only where a row's last keys lie.
//
// Blocks.  How many rows a sequence has is known on the device only.  Where keys are cut (and for few rows) with up to 256 sequences, every
// wave reads all lengths and lays the blocks and their parts out (Layout).  Else sequence b gets the block numbers from
// floor(rows in front of it / BM) + b on, which is never less than the blocks that it needs: a workgroup finds its sequence by a search over
// q_off, no sum over the sequences in front of it, and the grid is at most a block per sequence larger than a perfect
// one.  Of a sequence the last blocks start first, under a causal mask its longest ones; the sequences start by their number, the last one
// first, whatever their lengths.
//
// What bounds it.  Few rows: the bytes of K and V (one token over 131072 keys of 8 heads 98 to 104 us, 5.2 to 5.5 TB/s, and 6 for joining),
// with short caches the latencies of two launches (10 us).  Many rows: issue (matrix cores busy 47 % of the CU cycles of twelve prompts of 33 to
// 4096 tokens, and 3.6 vector instructions to each of theirs); 4 x 4096 tokens, 32 and 8 heads, bidirectional 955 to 1040 us by the
// card, 1.06 to 1.15 PFLOP/s; 16384 causal 1890 to 1935.  With short sequences starts and masked ends.
//
// Logits are formed transposed, S^T = K Q^T, with v_mfma_f32_16x16x32_bf16: a lane holds logits of one row, and the
// probabilities are in the layout of the second operand of O^T = V^T P^T, whose first operand is read from the row-major
// V tile by the LDS transpose read.  Running maximum (its reference, in base 2) and sum per row in fp32.  The matrix cores take
// probabilities in bf16.  With few rows, where they have little to do, a probability goes in as two of them, 2^-15 of it off at most
// (Rows::softmax; us, rounded and in two parts: one token over 131072 keys 108.8 and 108.6, over each of 64 caches up to 8000 205.5 and 205.3, 8 over
// each of 16 up to 2000 25.3 and 25.7).  With many rows, where a second product is half of the first two again, it is rounded to bf16 (2^-8 of it
// at most), and the sum is taken over what is multiplied (4 x 4096 tokens 950 and 1252, 16384 causal 1868 and 2466, blocks of 32 over 16 caches up to
// 2048 32.5 and 36.6).
//
// Values in masked places do not count, whatever they are: a tile in which some row does not see some key multiplies with
// those elements of V that are not finite replaced by 0, and adds what is not finite to the rows that see it.
#include <type_traits>

#include "attn_packed_rows.h"

namespace dare {
namespace {

constexpr float kLog2e = 1.4426950408889634f;

struct PackedDev {
  const bf16_t* q;
  const bf16_t* k;
  const bf16_t* v;
  bf16_t* out;
  long ldq, ldk, ldv, ldo;
  PackedRows rows;
  int n_kv;
  int max_parts;    // parts launched per block; with one part there is no workspace
  int part_tiles;   // tiles of a part, at least (more than 256 sequences)
  int slots;        // workgroups that parts are made for (up to 256 sequences)
  float* parts;     // [block][key head][part] partial results
  float scale_log2;
};

typedef __attribute__((address_space(3))) void* lptr_t;
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
typedef __attribute__((address_space(3))) s16x4* lds_s16x4_ptr;
typedef const __attribute__((address_space(3))) bf16x8* lds_frag_t;
typedef const __attribute__((address_space(3))) bf16_t* lds_elem_t;

// ---- tiles in LDS ------------------------------------------------------------------------
// Rows of K and V lie in LDS as in memory, 16-byte chunk c of key j at place c ^ swizzle(j): a K fragment (16 keys at one
// chunk) and the transpose read of V (8 keys at 32 bytes at a time) meet no bank twice.  The swizzle of a key depends
// on its place in a run of 16 only.
template <int DH>
__device__ __forceinline__ constexpr int k_swizzle(int key) {
  return DH == 128 ? key & 15 : key >> 1 & 7;
}
template <int DH>
__device__ __forceinline__ constexpr int v_swizzle(int key) {
  return DH == 128 ? (key & 3) << 2 | (key >> 2 & 1) << 1 : (key >> 1 & 3) << 1;
}

template <int N>
__device__ __forceinline__ void wait_vmcnt() {
  static_assert(N >= 0 && N < 64, "vmcnt range");
  asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}
__device__ __forceinline__ void wait_lds() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); }

// KEYS rows of K or V, from key `first` of the sequence on, to LDS address `to`, by one wave; rows from `len` on repeat
// the last one.  Waited for by hand (a compiler that sees the load puts a wait for all of them in front of every transpose read).
template <int DH, int KEYS, bool V>
__device__ __forceinline__ void load_rows(const bf16_t* base, long ld, int first, int len, unsigned to) {
  constexpr int CPR = DH / 8, RPL = 64 / CPR, N = KEYS / RPL;  // chunks per row, rows per load, loads
  const int lane = threadIdx.x & 63;
  const bf16_t* from = base + (long)first * ld;
  const unsigned row_bytes = (unsigned)ld * 2;
  const int end = len - 1 - first;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const int key = i * RPL + lane / CPR;
    const int chunk = (lane % CPR) ^ (V ? v_swizzle<DH>(key) : k_swizzle<DH>(key));
    const unsigned at = (unsigned)(key < end ? key : end) * row_bytes + chunk * 16;
    // (the LDS address is an operand in M0, set by the compiler; a wait state between the move to M0 and the load)
    asm volatile("s_nop 0\n\tglobal_load_lds_dwordx4 %0, %1" ::"v"(at), "s"(from), "{m0}"(to + i * 1024) : "memory");
  }
}

// 32 keys against R blocks of 16 rows.  kt, vt: LDS addresses of the keys' rows; key0: number of the first one.
// MASKED: row r of a lane sees keys below lim[r] only.  REST: probabilities in two parts.
template <int DH, int R, bool REST>
struct Rows {
  static constexpr int CB = DH / 16;  // 16-channel blocks
  static constexpr int PARTS = REST ? 2 : 1;
  static constexpr float kLift = 1.f / 65536;
  bf16x8 qf[R][DH / 32];
  f32x4 acc[CB][R];                   // channels 16 c + 4 kq .. + 3 of row l16
  float m[R], l[R];                   // reference in base 2, this lane's part of the sum
  int lim[R];

  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int r = 0; r < R; ++r) {
      m[r] = -__FLT_MAX__;
      l[r] = 0.f;
#pragma unroll
      for (int c = 0; c < CB; ++c) acc[c][r] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
  }

  // x[r][kb][e]: logit of key key0 + 16 kb + 4 kq + e
  __device__ __forceinline__ void logits(unsigned kt, f32x4 (&x)[R][2]) const {
    constexpr int ROWB = DH * 2;
    const int lane = threadIdx.x & 63, l16 = lane & 15, kq = lane >> 4;
#pragma unroll
    for (int kb = 0; kb < 2; ++kb) {
#pragma unroll
      for (int r = 0; r < R; ++r) x[r][kb] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int ks = 0; ks < DH / 32; ++ks) {
        const bf16x8 kf = *(lds_frag_t)(kt + (kb * 16 + l16) * ROWB + ((ks * 4 + kq) ^ k_swizzle<DH>(l16)) * 16);
#pragma unroll
        for (int r = 0; r < R; ++r) x[r][kb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, qf[r][ks], x[r][kb], 0, 0, 0);
      }
    }
  }

  __device__ __forceinline__ void mask(f32x4 (&x)[R][2], int key0) const {
    const int kq = (threadIdx.x & 63) >> 4;
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
      for (int n = 0; n < 8; ++n)
        if (key0 + (n >> 2) * 16 + kq * 4 + (n & 3) >= lim[r]) x[r][n >> 2][n & 3] = -INFINITY;
  }

  // The reference moves only when a maximum is 2^8 above it (any reference gives the same result up to rounding);
  // it stays finite, so a row that sees nothing has probabilities 0.
  // REST: the first part of p is p cut to 8 bits, c; the second one is p - c + c / 2^16, rounded to 8 bits (it is 2^-7 p at most, its rounding
  // 2^-15 p).  The lift is there because neither part may be 0 next to an infinite value (0 times infinity); what
  // it adds is 2^-16 of every p to 2^-24, so the sum gets it too and the quotient none.
  __device__ __forceinline__ void softmax(const f32x4 (&x)[R][2], bf16x8 (&pf)[PARTS][R], float scale_log2) {
    const bf16x2 ones = {(bf16_t)1.0f, (bf16_t)1.0f};
#pragma unroll
    for (int r = 0; r < R; ++r) {
      float top = x[r][0][0];
#pragma unroll
      for (int n = 1; n < 8; ++n) top = fmaxf(top, x[r][n >> 2][n & 3]);
      top = row_max(top) * scale_log2;  // scale > 0
      const bool grow = top > m[r] + 8.f;
      if (__any(grow)) {
        const float m_new = grow ? top : m[r], alpha = __builtin_amdgcn_exp2f(m[r] - m_new);
        m[r] = m_new;
        l[r] *= alpha;
#pragma unroll
        for (int c = 0; c < CB; ++c) acc[c][r] *= alpha;
      }
      float sum = 0.f;
#pragma unroll
      for (int n = 0; n < 8; n += 2) {
        f32x2 v;
        v[0] = __builtin_amdgcn_exp2f(fmaf(x[r][n >> 2][n & 3], scale_log2, -m[r]));
        v[1] = __builtin_amdgcn_exp2f(fmaf(x[r][n >> 2][(n & 3) + 1], scale_log2, -m[r]));
        bf16x2 pb;
        if constexpr (REST) {
          const float p0 = v[0], p1 = v[1];  // (copied before their bits are taken, as in row_join)
          sum += p0 + p1;
          const unsigned bits[2] = {__builtin_bit_cast(unsigned, p0), __builtin_bit_cast(unsigned, p1)};
          pb = __builtin_bit_cast(bf16x2, __builtin_amdgcn_perm(bits[1], bits[0], 0x07060302u));
#pragma unroll
          for (int i = 0; i < 2; ++i) v[i] = fmaf(__builtin_bit_cast(float, bits[i] & 0xffff0000u), kLift - 1.f, v[i]);
          const bf16x2 rest = __builtin_convertvector(v, bf16x2);
          pf[PARTS - 1][r][n] = rest[0];
          pf[PARTS - 1][r][n + 1] = rest[1];
        } else {
          pb = __builtin_convertvector(v, bf16x2);
          sum = __builtin_amdgcn_fdot2_f32_bf16(pb, ones, sum, false);
        }
        pf[0][r][n] = pb[0];
        pf[0][r][n + 1] = pb[1];
      }
      l[r] += REST ? sum * (1.f + kLift) : sum;
    }
  }

  // O^T += V^T P^T: slot s of a fragment is key 16 (s / 4) + 4 kq + s % 4
  template <bool MASKED>
  __device__ __forceinline__ void values(unsigned vt, const bf16x8 (&pf)[PARTS][R], int key0, int len_k) {
    constexpr int ROWB = DH * 2;
    const int lane = threadIdx.x & 63, l16 = lane & 15, kq = lane >> 4;
    const int key = kq * 4 + (l16 >> 2);
    const unsigned at = key * ROWB + ((l16 >> 1 & 1) ^ v_swizzle<DH>(key)) * 16 + (l16 & 1) * 8;
    u32x4 vf[CB];
#pragma unroll
    for (int c = 0; c < CB; ++c) {
      const unsigned va = vt + (at ^ (c * 32));
      const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_ptr)(va));
      const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_ptr)(va + 16 * ROWB));
      vf[c] = __builtin_bit_cast(u32x4, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
    }
    if constexpr (MASKED) {
      u16x2 top = {0, 0};  // the largest elements without their signs
#pragma unroll
      for (int c = 0; c < CB; ++c)
#pragma unroll
        for (int i = 0; i < 4; ++i) top = __builtin_elementwise_max(top, __builtin_bit_cast(u16x2, vf[c][i] & 0x7fff7fffu));
      if (__builtin_expect(__any(top[0] >= 0x7f80 || top[1] >= 0x7f80), 0)) {
        add_not_finite(vt, key0, len_k);
#pragma unroll
        for (int c = 0; c < CB; ++c)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const unsigned ones = ((vf[c][i] & 0x7f807f80u) + 0x00800080u) & 0x80008000u;  // exponents of all ones
            vf[c][i] &= ~((ones << 1) - (ones >> 15));
          }
      }
    }
#pragma unroll
    for (int c = 0; c < CB; ++c)
#pragma unroll
      for (int r = 0; r < R; ++r)
        acc[c][r] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, vf[c]), pf[0][r], acc[c][r], 0, 0, 0);
    if constexpr (REST) {
#pragma unroll
      for (int c = 0; c < CB; ++c)
#pragma unroll
        for (int r = 0; r < R; ++r)
          acc[c][r] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, vf[c]), pf[PARTS - 1][r], acc[c][r], 0, 0, 0);
    }
  }

  // What is not finite among the values, to the rows that see it (their probability is above 0)
  __device__ __forceinline__ void add_not_finite(unsigned vt, int key0, int len_k) {
    constexpr int ROWB = DH * 2;
    const int kq = (threadIdx.x & 63) >> 4;
    for (int j = 0; j < 32 && key0 + j < len_k; ++j) {
#pragma unroll
      for (int c = 0; c < CB; ++c) {
        const unsigned va = vt + j * ROWB + ((c * 2 + (kq >> 1)) ^ v_swizzle<DH>(j)) * 16 + (kq & 1) * 8;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float v = (float)((lds_elem_t)(va))[e];
          if (fabsf(v) < INFINITY) continue;
#pragma unroll
          for (int r = 0; r < R; ++r)
            if (key0 + j < lim[r]) acc[c][r][e] += v;
        }
      }
    }
  }
};

// This lane's rows: row j of the sequence is token j / G, head j % G of the group; those past the last one repeat it.
template <int DH, int R, bool REST>
__device__ __forceinline__ void take_rows(const PackedDev& p, const Place& at, int kvh, int row0, Rows<DH, R, REST>& w, long (&out_at)[R]) {
  const int lane = threadIdx.x & 63, l16 = lane & 15, kq = lane >> 4;
#pragma unroll
  for (int r = 0; r < R; ++r) {
    int j = row0 + r * 16 + l16;
    j = at.row0 + (j < at.rows ? j : at.rows - 1);
    const int i = divide(j, p.rows.by_group), head = kvh * p.rows.group + (j - i * p.rows.group);
    const bf16_t* row = p.q + (long)(at.q0 + i) * p.ldq + head * DH + kq * 8;
#pragma unroll
    for (int ks = 0; ks < DH / 32; ++ks) w.qf[r][ks] = *reinterpret_cast<const bf16x8*>(row + ks * 32);
    out_at[r] = (long)(at.q0 + i) * p.ldo + head * DH;
    w.lim[r] = packed_limit(i, at.shift, at.len_k, p.rows.causal_block, p.rows.by_causal_block);
  }
}
__device__ __forceinline__ int parts_of(const PackedDev& p, int tiles) {
  int n = (tiles + p.part_tiles - 1) / p.part_tiles;
  n = n < p.max_parts ? n : p.max_parts;
  return n > 1 ? n : 1;
}
template <int DH, int BM>
__device__ __forceinline__ float* part_slot(const PackedDev& p, int g, int kvh, int part) {
  return p.parts + ((long)(g * p.n_kv + kvh) * p.max_parts + part) * packed_slot_floats(DH, BM);
}

// ---- few rows: 16 R of them, the keys shared by the waves -----------------------------------------
// Every wave takes every second (heads of 64 channels: fourth) tile of 32 keys through two stages of its own, so that the waves meet at
// the end only.  64 KB of stages per workgroup, two workgroups on a CU: one reads while the other starts or ends.
constexpr int kFewKeys = 32;
template <int DH>
constexpr int kFewWaves = DH == 128 ? 2 : 4;

template <int DH, int R>
struct FewShared {
  unsigned char stages[kFewWaves<DH> * 4 * kFewKeys * DH * 2];
  float m[kFewWaves<DH>][R][16], l[kFewWaves<DH>][R][16];
};

// Tiles [first, last) of the keys of a block; slot: where a part's results go, nullptr if the block has one part
template <int DH, int R>
__device__ __forceinline__ void few_rows(const PackedDev& p, const Place& at, int kvh, int first, int last, float* slot,
                                         FewShared<DH, R>& shared) {
  constexpr int BM = 16 * R, CB = DH / 16, TILE = kFewKeys * DH * 2, STAGE = 2 * TILE, L = TILE / 1024, NW = kFewWaves<DH>;
  unsigned char* const smem = shared.stages;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int l16 = lane & 15, kq = lane >> 4;
  const int least = row_limit(p.rows, at, at.row0);  // keys that all rows see
  const bf16_t* kbase = p.k + (long)at.k0 * p.ldk + kvh * DH;
  const bf16_t* vbase = p.v + (long)at.k0 * p.ldv + kvh * DH;
  const unsigned lds0 = (unsigned)(size_t)(lptr_t)smem + wave * 2 * STAGE;
  auto load_k = [&](int t, int s) __attribute__((always_inline)) { load_rows<DH, kFewKeys, false>(kbase, p.ldk, t * kFewKeys, at.len_k, lds0 + s * STAGE); };
  auto load_v = [&](int t, int s) __attribute__((always_inline)) { load_rows<DH, kFewKeys, true>(vbase, p.ldv, t * kFewKeys, at.len_k, lds0 + s * STAGE + TILE); };
  int t = first + wave, s = 0;
  if (t < last) {
    load_k(t, 0);
    load_v(t, 0);
  }
  if (t + NW < last) {
    load_k(t + NW, 1);
    load_v(t + NW, 1);
  }
  Rows<DH, R, true> w;
  long out_at[R];
  take_rows(p, at, kvh, 0, w, out_at);
  w.clear();
#pragma unroll
  for (int r = 0; r < R; ++r)
#pragma unroll
    for (int ks = 0; ks < DH / 32; ++ks) asm volatile("" : "+v"(w.qf[r][ks]));  // (the queries in registers, or the loop waits for them in every step)
  for (; t < last; t += NW, s ^= 1) {
    const bool one = t + NW < last, two = t + 2 * NW < last;
    const unsigned kt = lds0 + s * STAGE, vt = kt + TILE;
    const int key0 = t * kFewKeys;
    const bool masked = key0 + kFewKeys > least;
    f32x4 x[R][2];
    bf16x8 pf[2][R];
    if (one) wait_vmcnt<3 * L>(); else wait_vmcnt<L>();
    w.logits(kt, x);
    wait_lds();
    if (two) load_k(t + 2 * NW, s);
    if (masked) w.mask(x, key0);
    w.softmax(x, pf, p.scale_log2);
    if (two) wait_vmcnt<3 * L>(); else if (one) wait_vmcnt<2 * L>(); else wait_vmcnt<0>();
    if (masked) w.template values<true>(vt, pf, key0, at.len_k); else w.template values<false>(vt, pf, key0, at.len_k);
    wait_lds();
    if (two) load_v(t + 2 * NW, s);
  }

  // ---- the waves' results are joined in their order, a share of the channel blocks by each ----
  float* mine = reinterpret_cast<float*>(smem + wave * 2 * STAGE);
#pragma unroll
  for (int r = 0; r < R; ++r) {
    const float l = row_sum(w.l[r]);
    if (kq == 0) {
      shared.m[wave][r][l16] = w.m[r];
      shared.l[wave][r][l16] = l;
    }
#pragma unroll
    for (int c = 0; c < CB; ++c) reinterpret_cast<f32x4*>(mine)[(c * R + r) * 64 + lane] = w.acc[c][r];
  }
  __syncthreads();
  constexpr int OWN = CB / NW;
#pragma unroll
  for (int r = 0; r < R; ++r) {
    float m = shared.m[0][r][l16], l = 0.f, f[NW];
#pragma unroll
    for (int o = 1; o < NW; ++o) m = fmaxf(m, shared.m[o][r][l16]);
#pragma unroll
    for (int o = 0; o < NW; ++o) {
      f[o] = __builtin_amdgcn_exp2f(shared.m[o][r][l16] - m);
      l += shared.l[o][r][l16] * f[o];
    }
    const int row = r * 16 + l16;
    if (row >= at.rows) continue;
    f32x4 sum[OWN];
#pragma unroll
    for (int i = 0; i < OWN; ++i) {
      const int c = wave * OWN + i;
      sum[i] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int o = 0; o < NW; ++o)
        sum[i] += reinterpret_cast<const f32x4*>(smem + o * 2 * STAGE)[(c * R + r) * 64 + lane] * f[o];
    }
    if (slot) {
#pragma unroll
      for (int i = 0; i < OWN; ++i) *reinterpret_cast<f32x4*>(slot + row * DH + (wave * OWN + i) * 16 + kq * 4) = sum[i];
      if (wave == 0 && kq == 0) {
        slot[BM * DH + row] = m;
        slot[BM * DH + BM + row] = l;
      }
    } else {
      const float inv = l == 0.f ? 0.f : 1.f / l;
#pragma unroll
      for (int i = 0; i < OWN; ++i) {
        bf16x4 o;
#pragma unroll
        for (int e = 0; e < 4; ++e) o[e] = (bf16_t)(sum[i][e] * inv);
        *reinterpret_cast<bf16x4*>(p.out + out_at[r] + (wave * OWN + i) * 16 + kq * 4) = o;
      }
    }
  }
}

// Up to 64 S sequences: as many workgroups as run at once walk over what there is to do.  (A workgroup for every part that
// there might be, as with more sequences: those without one take 64 KB of LDS and 1.5 us each before they are gone; one token over
// each of 32 caches of 40 to 4000 keys 33.7 us and in this form 30.1, of 4 of 32000 111 and 100, of 64 of 500 to 8000 158 and 149.)
template <int DH, int R, int S>
__global__ void __launch_bounds__(kFewWaves<DH> * 64) attn_packed_few_kernel(PackedDev p) {
  __shared__ __attribute__((aligned(1024))) FewShared<DH, R> shared;
  Layout<16 * R, kFewKeys, S, false> all;
  all.read(p.rows, p.n_kv, p.slots, p.max_parts);
  for (int u = blockIdx.x; u < all.n_units * p.n_kv; u += gridDim.x) {
    const int kvh = u % p.n_kv;
    Place at;
    int block, part, n_parts;
    all.unit(p.rows, u / p.n_kv, at, block, part, n_parts);
    // (offsets that do not ascend can lead anywhere)
    if (at.row0 < 0 || at.rows <= 0 || (unsigned)block >= (unsigned)p.rows.n_blocks || (unsigned)part >= (unsigned)n_parts) continue;
    const int tiles = (row_limit(p.rows, at, at.row0 + at.rows - 1) + kFewKeys - 1) / kFewKeys;
    if (u != (int)blockIdx.x) __syncthreads();  // the stages are used again
    few_rows<DH, R>(p, at, kvh, (int)((long)tiles * part / n_parts), (int)((long)tiles * (part + 1) / n_parts),
                    n_parts > 1 ? part_slot<DH, 16 * R>(p, block, kvh, part) : nullptr, shared);
  }
}

template <int DH, int R>
__global__ void __launch_bounds__(kFewWaves<DH> * 64) attn_packed_few_searched_kernel(PackedDev p) {
  __shared__ __attribute__((aligned(1024))) FewShared<DH, R> shared;
  const int kvh = blockIdx.x % p.n_kv, unit = blockIdx.x / p.n_kv;
  const int part = unit % p.max_parts, g = p.rows.n_blocks - 1 - unit / p.max_parts;
  Place at;
  if (!find_block<16 * R>(p.rows, g, at)) return;
  const int tiles = (row_limit(p.rows, at, at.row0 + at.rows - 1) + kFewKeys - 1) / kFewKeys, n_parts = parts_of(p, tiles);
  if (part >= n_parts) return;
  few_rows<DH, R>(p, at, kvh, (int)((long)tiles * part / n_parts), (int)((long)tiles * (part + 1) / n_parts),
                  n_parts > 1 ? part_slot<DH, 16 * R>(p, g, kvh, part) : nullptr, shared);
}

// ---- many rows: 128 of them, four waves of 32 rows on the same keys --------------------------------
// Tiles of 64 keys through two stages of K and two of V, shared by the waves.  A wave's keys are two stretches: the tiles that all of its
// rows see whole, and the one to three behind them in which some row's keys end.
// The first stretch runs as one stream of instructions over subtiles of 32 keys: while the logits of one are multiplied, the softmax of
// the one before and the value product of the one before that run, an MFMA or two, an exponential, fragment reads, and so
// on; fragments are read three MFMA groups ahead, and the barrier of a step lies behind its last fragment.  No mask in it,
// and no maximum of every tile: the reference of a row moves when a lane's sum of probabilities says so.  (As attention over many rows
// of one head does it, attn_bf16.hip, where this order was measured.)  The second stretch is plain: logits, mask, softmax, values.
constexpr int kManyWaves = 4, kManyRows = 32 * kManyWaves, kManyKeys = 64;

template <int N>
__device__ __forceinline__ void wait_vmcnt_and_barrier() {
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(N) : "memory");
}

template <int DH>
struct ManyShared {
  unsigned char stages[4 * kManyKeys * DH * 2];
  long out_rows[kManyRows];  // where the rows' outputs lie
};

// Steps (tiles of the keys) [first, first + n_steps) of a block; slot: where a part's results go, nullptr if the block has one part
template <int DH>
__device__ __forceinline__ void many_rows(const PackedDev& p, const Place& at, int kvh, const int first, const int n_steps, float* slot,
                                          ManyShared<DH>& shared) {
  constexpr int BM = kManyRows, CB = DH / 16, ROWB = DH * 2, TILE = kManyKeys * ROWB;
  constexpr int CPR = DH / 8, RPL = 64 / CPR;      // 16-byte chunks per row, rows of a wave's load
  constexpr int KL = TILE / 1024 / kManyWaves;     // a wave's loads of K (or V) per step
  constexpr int NP = CB;                           // fragments of K, and of V, that a subtile takes
  constexpr int AHEAD = 3, RING = AHEAD + 1;       // fragments read ahead of their MFMAs
  static_assert(NP % RING == 0, "fragments must divide");
  using Yes = std::true_type;
  using No = std::false_type;
  using S0 = std::integral_constant<int, 0>;
  using S1 = std::integral_constant<int, 1>;
  unsigned char* const smem = shared.stages;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int l16 = lane & 15, kq = lane >> 4;
  // of the steps the wave's: those that all of its rows see whole, those that one of them sees
  const bool any_row = wave * 32 < at.rows;  // (a wave without rows only loads)
  int whole = 0, mine = 0, ends = 0;  // ends: keys that the wave's last row sees
  if (any_row) {
    const int last = wave * 32 + 31 < at.rows ? wave * 32 + 31 : at.rows - 1;
    whole = row_limit(p.rows, at, at.row0 + wave * 32) / kManyKeys - first;
    ends = row_limit(p.rows, at, at.row0 + last);
    mine = (ends + kManyKeys - 1) / kManyKeys - first;
    mine = mine < 0 ? 0 : mine < n_steps ? mine : n_steps;
    whole = whole < 0 ? 0 : whole < mine ? whole : mine;
  }
  whole = __builtin_amdgcn_readfirstlane(whole);
  mine = __builtin_amdgcn_readfirstlane(mine);
  ends = __builtin_amdgcn_readfirstlane(ends);

  // ---- global -> LDS ----
  const bf16_t* kbase = p.k + (long)at.k0 * p.ldk + kvh * DH;
  const bf16_t* vbase = p.v + (long)at.k0 * p.ldv + kvh * DH;
  const unsigned key0 = (unsigned)wave * KL * RPL + (unsigned)lane / CPR;  // key of this lane's first load of a step
  // (the chunk XOR of a key is that of the lane's first key and that of the distance)
  const unsigned k_chunk = ((unsigned)lane % CPR ^ k_swizzle<DH>(key0)) * 16, v_chunk = ((unsigned)lane % CPR ^ v_swizzle<DH>(key0)) * 16;
  const unsigned lds0 = (unsigned)(size_t)(lptr_t)smem;
  auto load_tiles = [&](auto is_v, int step) __attribute__((always_inline)) {
    constexpr bool V = decltype(is_v)::value;
    const int k0 = (first + step) * kManyKeys;
    const unsigned row_bytes = (unsigned)(V ? p.ldv : p.ldk) * 2;
    const bf16_t* from = V ? vbase + (long)k0 * p.ldv : kbase + (long)k0 * p.ldk;
    const unsigned to = lds0 + (V ? 2 * TILE : 0) + (step & 1) * TILE + wave * KL * 1024;
    const unsigned chunk = V ? v_chunk : k_chunk;
    auto load = [&](unsigned a, const bf16_t* base, int i) __attribute__((always_inline)) {
      asm volatile("s_nop 0\n\tglobal_load_lds_dwordx4 %0, %1" ::"v"(a), "s"(base), "{m0}"(to + i * 1024) : "memory");
    };
#define DARE_SWZ(i) ((V ? v_swizzle<DH>((i) * RPL) : k_swizzle<DH>((i) * RPL)) * 16)
    if (k0 + kManyKeys > at.len_k) {  // keys past the end re-read the last one
#pragma unroll
      for (int i = 0; i < KL; ++i) {
        const unsigned key = key0 + i * RPL, end = at.len_k - 1 - k0;
        load((key < end ? key : end) * row_bytes + (chunk ^ DARE_SWZ(i)), from, i);
      }
    } else {
#pragma unroll
      for (int i = 0; i < KL; ++i) load((chunk ^ DARE_SWZ(i)) + key0 * row_bytes, from + (long)(i * RPL) * (V ? p.ldv : p.ldk), i);
    }
#undef DARE_SWZ
  };
  // Publishes K of step + 1 and V of step; every wave has read K of step and V of step - 1, whose stages are filled again
  auto next_tiles = [&](int step) __attribute__((always_inline)) {
    wait_vmcnt_and_barrier<0>();
    if (step + 2 < n_steps) load_tiles(No{}, step + 2);
    if (step + 1 < n_steps) load_tiles(Yes{}, step + 1);
  };

  // The first tiles and the queries, all on their way at once: what a short sequence takes is latencies
  if (n_steps > 0) {
    load_tiles(No{}, 0);
    load_tiles(Yes{}, 0);
  }
  if (n_steps > 1) load_tiles(No{}, 1);
  Rows<DH, 2, false> w;
  long out_at[2];
  take_rows(p, at, kvh, wave * 32, w, out_at);
  w.clear();
  if (kq == 0) {
#pragma unroll
    for (int r = 0; r < 2; ++r) shared.out_rows[wave * 32 + r * 16 + l16] = out_at[r];
  }

  // ---- fragments ----
  // K fragment j: keys 16 (j & 1) + l16, channels 32 (j / 2) + 8 kq ..
  // V fragment j, by transpose read: channel 16 j + l16, keys 4 kq .. +3 and 16 + 4 kq .. +3
  unsigned k_at[NP / 2], v_at;
#pragma unroll
  for (int ks = 0; ks < NP / 2; ++ks) k_at[ks] = lds0 + l16 * ROWB + ((ks * 4 + kq) ^ k_swizzle<DH>(l16)) * 16;
  {
    const int key = kq * 4 + (l16 >> 2);
    v_at = lds0 + 2 * TILE + key * ROWB + ((l16 >> 1 & 1) ^ v_swizzle<DH>(key)) * 16 + (l16 & 1) * 8;
  }
  bf16x8 kf[RING], vf[RING];
  auto read_k = [&](int j, int sub) __attribute__((always_inline)) {
    kf[j % RING] = *(lds_frag_t)(k_at[j / 2] + (sub * 32 + (j & 1) * 16) * ROWB);
  };
  auto read_v = [&](int j, int sub) __attribute__((always_inline)) {
    const unsigned a = lds0 + ((v_at - lds0) ^ j * 32) + sub * 32 * ROWB;
    const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_ptr)(a));
    const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_ptr)(a + 16 * ROWB));
    vf[j % RING] = __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
  };
  f32x4 sc[2][2][2];        // logits of two subtiles, [set][row block][16 keys]: keys 4 kq ..
  bf16x8 pf[2][2];          // probabilities of two subtiles, [set][row block]

  // ---- softmax of a subtile: logit n = 8 row block + key slot ----
  const bf16x2 ones = {(bf16_t)1.0f, (bf16_t)1.0f};
  float e0 = 0.f, e1 = 0.f;
  auto exp_one = [&](const f32x4 (&x)[2][2], int n) __attribute__((always_inline)) {
    const float v = __builtin_amdgcn_exp2f(fmaf(x[n >> 3][n >> 2 & 1][n & 3], p.scale_log2, -w.m[n >> 3]));
    if (n & 1) e1 = v; else e0 = v;
  };
  auto round_pair = [&](bf16x8 (&pr)[2], int n, float (&sum)[2]) __attribute__((always_inline)) {
    const f32x2 v = {e0, e1};
    const bf16x2 pb = __builtin_convertvector(v, bf16x2);
    sum[n >> 3] = __builtin_amdgcn_fdot2_f32_bf16(pb, ones, sum[n >> 3], false);
    pr[n >> 3][n & 7] = pb[0];
    pr[n >> 3][(n & 7) + 1] = pb[1];
  };
  // The reference of the rows of a block of 16 moves to the maximum of this subtile, which is scored again, and of the next one, where
  // that is 2^8 above it.  A probability below 256 is looked at by nobody: any reference gives the same result up to rounding.
  // FIRST: there is none yet.
  auto move_reference = [&](auto r_c, const f32x4 (&x)[2][2], const f32x4 (&next)[2][2], bf16x8 (&pr)[2], float (&sum)[2], auto first_c) __attribute__((always_inline)) {
    constexpr int r = decltype(r_c)::value;
    float top = x[r][0][0];
#pragma unroll
    for (int n = 1; n < 8; ++n) top = fmaxf(top, x[r][n >> 2][n & 3]);
#pragma unroll
    for (int n = 0; n < 8; ++n) top = fmaxf(top, next[r][n >> 2][n & 3]);
    top = row_max(top) * p.scale_log2;  // scale > 0
    const float moved = top > w.m[r] + 8.f ? top : w.m[r];
    const float m_new = fmaxf(moved, -__FLT_MAX__);  // (finite: logits of -infinity have probability 0)
    if constexpr (!decltype(first_c)::value) {
      const float alpha = __builtin_amdgcn_exp2f(w.m[r] - m_new);
      w.l[r] *= alpha;
#pragma unroll
      for (int c = 0; c < CB; ++c) w.acc[c][r] *= alpha;
    }
    w.m[r] = m_new;
    sum[r] = 0.f;
#pragma unroll
    for (int n = 8 * r; n < 8 * r + 8; n += 2) {
      exp_one(x, n);
      exp_one(x, n + 1);
      round_pair(pr, n, sum);
    }
  };

  // One subtile period.  QK: logits of subtile u (into sc[S ^ 1]); SM: softmax of u - 1 (sc[S], into pf[S]); PV: values of
  // u - 2 (pf[S ^ 1]).  MORE: a period follows.
  auto period = [&](auto s_c, auto qk_c, auto sm_c, auto pv_c, auto more_c, int step) __attribute__((always_inline)) {
    constexpr int S = decltype(s_c)::value, SUB = S ^ 1;  // SUB: subtile of its tile, of K and V alike
    constexpr bool QK = decltype(qk_c)::value, SM = decltype(sm_c)::value, PV = decltype(pv_c)::value;
    constexpr bool MORE = decltype(more_c)::value, EDGE = SUB == 1;  // EDGE: the step's tiles end here
    constexpr int LPP = 16 / NP;        // logits per fragment
    constexpr int SPLIT = NP - AHEAD;   // fragment behind whose MFMAs the step's last ones are in registers
    float sum[2] = {0.f, 0.f};
    auto softmax = [&](int from, int to) __attribute__((always_inline)) {
      if constexpr (SM) {
#pragma unroll
        for (int n = from; n < to; ++n) {
          if (n % 2 == 0 && n > 0) round_pair(pf[S], n - 2, sum);
          exp_one(sc[S], n);
        }
      }
      __builtin_amdgcn_sched_barrier(0);
    };
#pragma unroll
    for (int j = 0; j < NP; ++j) {
      __builtin_amdgcn_sched_barrier(0);
      const f32x4 zero = {0.f, 0.f, 0.f, 0.f};
      f32x4 (&x)[2][2] = sc[S ^ 1];
      if constexpr (QK) x[0][j & 1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf[j % RING], w.qf[0][j / 2], j < 2 ? zero : x[0][j & 1], 0, 0, 0);
      softmax(j * LPP, j * LPP + LPP / 2);
      if constexpr (QK) x[1][j & 1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf[j % RING], w.qf[1][j / 2], j < 2 ? zero : x[1][j & 1], 0, 0, 0);
      __builtin_amdgcn_sched_barrier(0);
      if constexpr (PV) w.acc[j][0] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf[j % RING], pf[S ^ 1][0], w.acc[j][0], 0, 0, 0);
      softmax(j * LPP + LPP / 2, (j + 1) * LPP);
      if constexpr (PV) w.acc[j][1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf[j % RING], pf[S ^ 1][1], w.acc[j][1], 0, 0, 0);
      __builtin_amdgcn_sched_barrier(0);
      if (j + AHEAD < NP) {
        if constexpr (QK) read_k(j + AHEAD, SUB);
        if constexpr (PV) read_v(j + AHEAD, SUB);
      } else if constexpr (MORE && !EDGE) {
        if constexpr (QK) read_k(j + AHEAD - NP, 1);
        if constexpr (PV) read_v(j + AHEAD - NP, 1);
      }
      if constexpr (EDGE && MORE) {
        if (j == SPLIT) {  // all of the step's fragments are in registers: its stages may be filled again
          if constexpr (SM) asm volatile("" : "+v"(sum[0]), "+v"(sum[1]), "+v"(e0), "+v"(e1));  // (what is done so far stays in front of the branches)
          next_tiles(step);
#pragma unroll
          for (int i = 0; i < NP / 2; ++i) k_at[i] = lds0 + ((k_at[i] - lds0) ^ TILE);
          if constexpr (PV) v_at = lds0 + ((v_at - lds0) ^ TILE);
        }
        if (j > SPLIT) {
          const int from = AHEAD * (j - SPLIT - 1) / (AHEAD - 1), to = AHEAD * (j - SPLIT) / (AHEAD - 1);
#pragma unroll
          for (int i = from; i < to; ++i) {
            read_k(i, 0);
            read_v(i, 0);
          }
        }
      }
    }
    __builtin_amdgcn_sched_barrier(0);
    if constexpr (SM) {
      round_pair(pf[S], 14, sum);
      constexpr float kLimit = 256.f;
      if (__any(fmaxf(sum[0], sum[1]) > kLimit)) {
        if (__any(sum[0] > kLimit)) move_reference(S0{}, sc[S], sc[S ^ 1], pf[S], sum, No{});
        if (__any(sum[1] > kLimit)) move_reference(S1{}, sc[S], sc[S ^ 1], pf[S], sum, No{});
      }
      w.l[0] += sum[0];
      w.l[1] += sum[1];
    }
  };

#pragma unroll
  for (int r = 0; r < 2; ++r)
#pragma unroll
    for (int ks = 0; ks < DH / 32; ++ks) asm volatile("" : "+v"(w.qf[r][ks]));  // (the queries in registers)
  wait_vmcnt_and_barrier<0>();
  if (whole > 0) {
#pragma unroll
    for (int j = 0; j < AHEAD; ++j) read_k(j, 0);
    period(S1{}, Yes{}, No{}, No{}, Yes{}, 0);
    period(S0{}, Yes{}, No{}, No{}, Yes{}, 0);
    move_reference(S0{}, sc[0], sc[1], pf[0], w.l, Yes{});
    move_reference(S1{}, sc[0], sc[1], pf[0], w.l, Yes{});
    for (int step = 1; step < whole; ++step) {
      period(S1{}, Yes{}, Yes{}, Yes{}, Yes{}, step);
      period(S0{}, Yes{}, Yes{}, Yes{}, Yes{}, step);
    }
    period(S1{}, No{}, Yes{}, Yes{}, Yes{}, whole);
    period(S0{}, No{}, No{}, Yes{}, No{}, whole);
  }
  // (all waves load, and join the barrier of every step)
  for (int step = whole; step < n_steps; ++step) {
    const unsigned kt = lds0 + (step & 1) * TILE, vt = kt + 2 * TILE;
    const int key = (first + step) * kManyKeys;
    f32x4 x[2][2][2];
    if (step < mine) {
#pragma unroll
      for (int u = 0; u < 2; ++u)
        if (key + u * 32 < ends) w.logits(kt + u * 32 * ROWB, x[u]);
    }
    next_tiles(step);
    if (step < mine) {
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        if (key + u * 32 >= ends) break;
        bf16x8 pr[1][2];
        w.mask(x[u], key + u * 32);
        w.softmax(x[u], pr, p.scale_log2);
        w.template values<true>(vt + u * 32 * ROWB, pr, key + u * 32, at.len_k);
      }
    }
  }

  float l[2];
#pragma unroll
  for (int r = 0; r < 2; ++r) l[r] = row_sum(w.l[r]);
  if (slot) {  // (as the sums lie in the lanes: whole kilobytes)
#pragma unroll
    for (int r = 0; r < 2; ++r) {
      if (wave * 32 + r * 16 >= at.rows) break;
#pragma unroll
      for (int c = 0; c < CB; ++c) reinterpret_cast<f32x4*>(slot)[((wave * CB + c) * 2 + r) * 64 + lane] = w.acc[c][r];
      if (kq == 0) {
        slot[BM * DH + wave * 32 + r * 16 + l16] = w.m[r];
        slot[BM * DH + BM + wave * 32 + r * 16 + l16] = l[r];
      }
    }
    return;
  }
  // Outputs go through the wave's share of the K stages, which nobody reads behind the last barrier, so that a store has whole rows:
  // as the sums lie, 32 bytes of 16 rows each, the stores of a workgroup took 3900 cycles.
  const unsigned own = wave * 32 * ROWB;
#pragma unroll
  for (int r = 0; r < 2; ++r) {
    const float inv = l[r] == 0.f ? 0.f : 1.f / l[r];
#pragma unroll
    for (int c = 0; c < CB; ++c) {
      bf16x4 o;
#pragma unroll
      for (int e = 0; e < 4; ++e) o[e] = (bf16_t)(w.acc[c][r][e] * inv);
      *reinterpret_cast<bf16x4*>(smem + own + (r * 16 + l16) * ROWB + ((c * 2 + (kq >> 1)) ^ (l16 % CPR)) * 16 + (kq & 1) * 8) = o;
    }
  }
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
#pragma unroll
  for (int i = 0; i < 32 / RPL; ++i) {
    const int row = i * RPL + lane / CPR, chunk = lane % CPR;
    const u32x4 o = *reinterpret_cast<const u32x4*>(smem + own + row * ROWB + (chunk ^ (row % CPR)) * 16);
    if (wave * 32 + row < at.rows) *reinterpret_cast<u32x4*>(p.out + shared.out_rows[wave * 32 + row] + chunk * 8) = o;
  }
}

// A workgroup per block (and part: more than 256 sequences), the last one first
template <int DH>
__global__ void __launch_bounds__(kManyWaves * 64, 2) attn_packed_many_kernel(PackedDev p) {
  __shared__ __attribute__((aligned(1024))) ManyShared<DH> shared;
  const int kvh = blockIdx.x % p.n_kv, unit = blockIdx.x / p.n_kv;
  const int part = unit % p.max_parts, g = p.rows.n_blocks - 1 - unit / p.max_parts;
  Place at;
  if (!find_block<kManyRows>(p.rows, g, at)) return;
  const int tiles = (row_limit(p.rows, at, at.row0 + at.rows - 1) + kManyKeys - 1) / kManyKeys, n_parts = parts_of(p, tiles);
  if (part >= n_parts) return;
  const int first = (int)((long)tiles * part / n_parts);
  many_rows<DH>(p, at, kvh, first, (int)((long)tiles * (part + 1) / n_parts) - first,
                n_parts > 1 ? part_slot<DH, kManyRows>(p, g, kvh, part) : nullptr, shared);
}
// Blocks whose keys are cut, by the lengths on the device, into no more parts than there are workgroups
template <int DH, int S>
__global__ void __launch_bounds__(kManyWaves * 64, 2) attn_packed_many_parts_kernel(PackedDev p) {
  __shared__ __attribute__((aligned(1024))) ManyShared<DH> shared;
  const int kvh = blockIdx.x % p.n_kv, u = blockIdx.x / p.n_kv;
  Layout<kManyRows, kManyKeys, S, true> all;
  all.read(p.rows, p.n_kv, p.slots, p.max_parts);
  if (u >= all.n_units) return;
  Place at;
  int block, part, n_parts;
  all.unit(p.rows, u, at, block, part, n_parts);
  // (offsets that do not ascend can lead anywhere)
  if (at.row0 < 0 || at.rows <= 0 || (unsigned)block >= (unsigned)p.rows.n_blocks || (unsigned)part >= (unsigned)n_parts) return;
  const int tiles = (row_limit(p.rows, at, at.row0 + at.rows - 1) + kManyKeys - 1) / kManyKeys;
  n_parts = all.needed(tiles, n_parts);
  if (part >= n_parts) return;
  const int first = (int)((long)tiles * part / n_parts);
  many_rows<DH>(p, at, kvh, first, (int)((long)tiles * (part + 1) / n_parts) - first,
                n_parts > 1 ? part_slot<DH, kManyRows>(p, block, kvh, part) : nullptr, shared);
}

// ---- parts of a row's keys, joined ---------------------------------------------------------------
// What bounds both forms is the latency of what other XCDs have written; so all that a row needs is asked for at once.
// channels c .. c + 3 of the row
__device__ __forceinline__ void join_store(const PackedDev& p, const Place& at, int row, int c, int dh, f32x4 sum, float l) {
  const float inv = l == 0.f ? 0.f : 1.f / l;
  const int j = at.row0 + row, i = divide(j, p.rows.by_group);
  const int head = (int)(blockIdx.x % p.n_kv) * p.rows.group + (j - i * p.rows.group);
  bf16x4 o;
#pragma unroll
  for (int e = 0; e < 4; ++e) o[e] = (bf16_t)(sum[e] * inv);
  *reinterpret_cast<bf16x4*>(p.out + (long)(at.q0 + i) * p.ldo + head * dh + c) = o;
}

// Few rows, up to 64 parts: a wave per row.  Lane q holds the reference and the sum of part q; DH / 4 lanes hold a part's channels, so
// 2 (4) parts are read side by side, eight times that many at once.
// S: sequences per lane of the layout, 0 where the blocks were searched.
template <int DH, int BM, int S>
__global__ void __launch_bounds__(256) attn_packed_join_few_kernel(PackedDev p) {
  constexpr int LANES = DH / 4, SIDE = 64 / LANES, AT_ONCE = 8;
  constexpr long SLOT = packed_slot_floats(DH, BM);
  const int lane = threadIdx.x & 63, row = blockIdx.y * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  Place at;
  int n_parts;
  const int kvh = blockIdx.x % p.n_kv, g = blockIdx.x / p.n_kv;
  if constexpr (S > 0) {
    Layout<BM, kFewKeys, S, false> all;
    all.read(p.rows, p.n_kv, p.slots, p.max_parts);
    if (g >= all.n_blocks) return;
    all.block(p.rows, g, at, n_parts);
    if (at.row0 < 0) return;
  } else {
    if (!find_block<BM>(p.rows, g, at)) return;
    n_parts = parts_of(p, (row_limit(p.rows, at, at.row0 + at.rows - 1) + kFewKeys - 1) / kFewKeys);
  }
  if (row >= at.rows || n_parts < 2) return;
  const float* slot = part_slot<DH, BM>(p, g, kvh, 0);
  const int own = lane < n_parts ? lane : n_parts - 1, c = lane % LANES * 4, side = lane / LANES;
  const float m_own = slot[own * SLOT + BM * DH + row], l_own = slot[own * SLOT + BM * DH + BM + row];
  f32x4 sum = {0.f, 0.f, 0.f, 0.f};
  float m, l, f_own;
  for (int q0 = 0; q0 < n_parts; q0 += SIDE * AT_ONCE) {
    f32x4 v[AT_ONCE];
#pragma unroll
    for (int i = 0; i < AT_ONCE; ++i) {
      const int q = q0 + i * SIDE + side;
      v[i] = *reinterpret_cast<const f32x4*>(slot + (q < n_parts ? q : n_parts - 1) * SLOT + row * DH + c);
    }
    __builtin_amdgcn_sched_barrier(0);
    if (q0 == 0) {
      m = m_own;
#pragma unroll
      for (int o = 32; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor(m, o, 64));
      f_own = lane < n_parts ? __builtin_amdgcn_exp2f(m_own - m) : 0.f;
      l = wave_sum(l_own * f_own);
    }
#pragma unroll
    for (int i = 0; i < AT_ONCE; ++i) {
      const int q = q0 + i * SIDE + side;
      const float f = __shfl(f_own, q & 63, 64);
      if (q < n_parts) sum += v[i] * f;
    }
  }
#pragma unroll
  for (int o = LANES; o < 64; o <<= 1)
#pragma unroll
    for (int e = 0; e < 4; ++e) sum[e] += __shfl_xor(sum[e], o, 64);
  if (side == 0) join_store(p, at, row, c, DH, sum, l);
}

// Many rows, few parts: a thread per row and four channels, as a lane of the parts held them, four parts at once.
template <int DH, int S>
__global__ void __launch_bounds__(256) attn_packed_join_many_kernel(PackedDev p) {
  constexpr int CB = DH / 16, AT_ONCE = 4, BM = kManyRows;
  constexpr long SLOT = packed_slot_floats(DH, BM);
  const int lane = threadIdx.x & 63, f = blockIdx.y * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int row = f / (2 * CB) * 32 + (f & 1) * 16 + (lane & 15), c = (f >> 1) % CB * 16 + (lane >> 4) * 4;
  const int kvh = blockIdx.x % p.n_kv, g = blockIdx.x / p.n_kv;
  Place at;
  int n_parts;
  if constexpr (S > 0) {
    Layout<BM, kManyKeys, S, true> all;
    all.read(p.rows, p.n_kv, p.slots, p.max_parts);
    if (g >= all.n_blocks) return;
    all.block(p.rows, g, at, n_parts);
    if (at.row0 < 0) return;
    n_parts = all.needed((row_limit(p.rows, at, at.row0 + at.rows - 1) + kManyKeys - 1) / kManyKeys, n_parts);
  } else {
    if (!find_block<BM>(p.rows, g, at)) return;
    n_parts = parts_of(p, (row_limit(p.rows, at, at.row0 + at.rows - 1) + kManyKeys - 1) / kManyKeys);
  }
  if (row >= at.rows || n_parts < 2) return;
  const float* slot = part_slot<DH, BM>(p, g, kvh, 0);
  f32x4 sum = {0.f, 0.f, 0.f, 0.f};
  float m = -__FLT_MAX__, l = 0.f;
  for (int q0 = 0; q0 < n_parts; q0 += AT_ONCE) {
    f32x4 v[AT_ONCE];
    float mq[AT_ONCE], lq[AT_ONCE];
#pragma unroll
    for (int i = 0; i < AT_ONCE; ++i) {  // (parts past the end: the last one again, for nothing)
      const float* from = slot + (q0 + i < n_parts ? q0 + i : n_parts - 1) * SLOT;
      mq[i] = from[BM * DH + row];
      lq[i] = from[BM * DH + BM + row];
      v[i] = reinterpret_cast<const f32x4*>(from)[f * 64 + lane];
    }
    __builtin_amdgcn_sched_barrier(0);
    float m_new = m;
#pragma unroll
    for (int i = 0; i < AT_ONCE; ++i) m_new = fmaxf(m_new, mq[i]);
    const float alpha = __builtin_amdgcn_exp2f(m - m_new);
    m = m_new;
    sum *= alpha;
    l *= alpha;
#pragma unroll
    for (int i = 0; i < AT_ONCE; ++i) {
      const float f = q0 + i < n_parts ? __builtin_amdgcn_exp2f(mq[i] - m) : 0.f;
      if (q0 + i < n_parts) sum += v[i] * f;
      l = fmaf(lq[i], f, l);
    }
  }
  join_store(p, at, row, c, DH, sum, l);
}

template <int DH, int R, int S>
hipError_t launch_few_laid(const PackedDev& p, const PackedPlan& plan, hipStream_t s) {
  const long most = (long)plan.blocks * plan.parts * p.n_kv;
  hipLaunchKernelGGL((attn_packed_few_kernel<DH, R, S>), dim3((unsigned)(most < p.slots ? most : p.slots)), dim3(kFewWaves<DH> * 64), 0, s, p);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || plan.parts == 1) return e;
  hipLaunchKernelGGL((attn_packed_join_few_kernel<DH, 16 * R, S>), dim3((unsigned)(plan.blocks * p.n_kv), 4 * R), dim3(256), 0, s, p);
  return hipGetLastError();
}
template <int DH, int R>
hipError_t launch_few(const PackedDev& p, const PackedPlan& plan, hipStream_t s) {
  if (p.rows.batch <= 64) return launch_few_laid<DH, R, 1>(p, plan, s);
  if (p.rows.batch <= 256) return launch_few_laid<DH, R, 4>(p, plan, s);
  const dim3 grid((unsigned)((long)plan.blocks * plan.parts * p.n_kv));
  hipLaunchKernelGGL((attn_packed_few_searched_kernel<DH, R>), grid, dim3(kFewWaves<DH> * 64), 0, s, p);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || plan.parts == 1) return e;
  hipLaunchKernelGGL((attn_packed_join_few_kernel<DH, 16 * R, 0>), dim3((unsigned)(plan.blocks * p.n_kv), 4 * R), dim3(256), 0, s, p);
  return hipGetLastError();
}

template <int DH, int S>
hipError_t launch_many_cut(const PackedDev& p, const PackedPlan& plan, hipStream_t s) {
  if (S > 0)
    hipLaunchKernelGGL((attn_packed_many_parts_kernel<DH, S == 0 ? 1 : S>), dim3((unsigned)p.slots), dim3(kManyWaves * 64), 0, s, p);
  else
    hipLaunchKernelGGL(attn_packed_many_kernel<DH>, dim3((unsigned)((long)plan.blocks * plan.parts * p.n_kv)), dim3(kManyWaves * 64), 0, s, p);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || plan.parts == 1) return e;
  hipLaunchKernelGGL((attn_packed_join_many_kernel<DH, S>), dim3((unsigned)(plan.blocks * p.n_kv), kManyRows * DH / 1024), dim3(256), 0, s, p);
  return hipGetLastError();
}
template <int DH>
hipError_t launch_many(const PackedDev& p, const PackedPlan& plan, hipStream_t s) {
  if (plan.parts == 1 || p.rows.batch > 256) return launch_many_cut<DH, 0>(p, plan, s);
  return p.rows.batch <= 64 ? launch_many_cut<DH, 1>(p, plan, s) : launch_many_cut<DH, 4>(p, plan, s);
}

template <int DH>
hipError_t launch_dh(const PackedDev& p, const PackedPlan& plan, hipStream_t s) {
  if (plan.rows == 16) return launch_few<DH, 1>(p, plan, s);
  if (plan.rows == 32) return launch_few<DH, 2>(p, plan, s);
  return launch_many<DH>(p, plan, s);
}

PackedPlan plan_of(const PackedArgs& a) {
  return packed_plan(a.batch, a.total_q, a.max_q, a.max_k, a.n_heads / a.n_kv_heads, a.n_kv_heads);
}

}  // namespace

size_t packed_workspace_floats(int dtype, const PackedArgs& a) {
  if (dtype != DARE_BF16) return 0;
  const PackedPlan plan = plan_of(a);
  return plan.parts == 1 ? 0 : (size_t)plan.blocks * a.n_kv_heads * plan.parts * packed_slot_floats(a.head_dim, plan.rows);
}

hipError_t launch_attn_packed_bf16(const PackedArgs& a, hipStream_t s) {
  const PackedPlan plan = plan_of(a);
  PackedDev p;
  p.q = static_cast<const bf16_t*>(a.q);
  p.k = static_cast<const bf16_t*>(a.k);
  p.v = static_cast<const bf16_t*>(a.v);
  p.out = static_cast<bf16_t*>(a.out);
  p.ldq = a.ldq;
  p.ldk = a.ldk;
  p.ldv = a.ldv;
  p.ldo = a.ldo;
  p.rows = packed_rows(a, plan.blocks);
  p.n_kv = a.n_kv_heads;
  p.max_parts = plan.parts;
  p.part_tiles = plan.part_keys / (plan.rows == kManyRows ? kManyKeys : kFewKeys);
  // (two on every CU; with many rows, n_kv times a number, and at least two per block that there can be, four where masked rows
  // see half of the keys on average)
  p.slots = 512;
  if (plan.rows == kManyRows) {
    const long least = (a.causal_block > 0 && 2l * a.max_q > a.max_k ? 4l : 2l) * plan.blocks;
    p.slots = (int)((512 / a.n_kv_heads > least ? 512 / a.n_kv_heads : least) * a.n_kv_heads);
  }
  p.parts = a.workspace;
  p.scale_log2 = a.scale * kLog2e;
  return a.head_dim == 128 ? launch_dh<128>(p, plan, s) : launch_dh<64>(p, plan, s);
}

}  // namespace dare
