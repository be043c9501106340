// Rotary embedding by positions: the channel pair (a, b) number i of a head of a token at position p becomes
//     (a cos - b sin, b cos + a sin),   angle p f_i,   cos and sin times a common magnitude,
// for the first rot channels of every head; the others go through as they are.  Queries, keys and values of a token in
// one launch: Q is rotated, K is rotated and stored at the token's cache row, V is stored there as it is.
//
// No table of angles: it would have to reach the largest position, and its rows are bytes that the
// launch has to read.  A wave owns a token (or some of its heads); lane i takes cos and sin of pair i, the angle
// formed and reduced to an eighth of a turn in 64 bits, where a position of 10^9 costs nothing of the last bits in fp32, and
// leaves them to the other lanes in LDS.
//
// What bounds it: bytes where there are many tokens, latencies where there are few.  So a lane asks for its first kAtOnce items
// before it turns to the angles, and few tokens are spread over as many waves as they have items for (rope_split).  us, 32 and 8 heads of
// 128 channels, bf16, part by part with the angles first and now: 1 token 4.4 and 2.9, 8 4.8 and 3.0, 300 7.5 and 3.8,
// 16384 81.2 and 82.8 (4.9 TB/s; a large copy reaches 5.0); 2, 4 and 8 items at once 82.8, 84.2, 83.1.  Halves that no
// 16 bytes divide: 9161 tokens of 16 and 4 heads, 34 of 128 channels rotated, element by element 87 us, in chunks and what they leave 53 (chunks of
// 16 bytes each, 48 channels, 34).
#include "dare_common.h"
#include "attn_packed.h"

namespace dare {
namespace {

struct RopeDev {
  const void* x[3];    // q, k, v
  void* out[3];
  long ldx[3], ldo[3]; // elements between tokens
  // items of a token: chunks of its heads, 64 of a part in a turn of a wave; q's turns, then k's, then v's
  int items[3], turns[3];  // turns: up to and including the part's
  int per_head[3];
  Divider by_per_head[3];
  int n, dim, rot;
  const int32_t* pos;
  const double* freqs;
  const int32_t* rows; // rows of k and v outputs, or nullptr
  int out_rows;
  float magnitude;
};

constexpr int kRopeWaves = 4, kAtOnce = 2;

// 16 bytes, V elements of type E, that are read and written at once, also where they do not lie on 16 bytes (ALIGNED)
template <class E, bool ALIGNED>
struct alignas(ALIGNED ? 16 : sizeof(E)) Chunk {
  static constexpr int V = 16 / sizeof(E);
  E v[V];
};

// PAIRS: channels (2 i, 2 i + 1) are a pair, an item is a chunk of V neighbouring channels.  Else i and i + rot / 2: an item is a chunk
// of V channels i with the one of their partners, or a chunk of channels that are not rotated; !WHOLE: or one channel, with its partner
// or without, of those that are left over where rot / 2 is not a multiple of V.
template <class E, bool PAIRS, bool ALIGNED, bool WHOLE>
__global__ void __launch_bounds__(kRopeWaves * 64) rope_kernel(RopeDev p) {
  typedef Chunk<E, ALIGNED> chunk_t;
  constexpr int V = chunk_t::V;
  __shared__ float cs_all[kRopeWaves][kRopeMaxDim];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const long t = (long)blockIdx.x * kRopeWaves + wave;
  if (t >= p.n) return;  // (no barrier below: a wave reads what its own lanes wrote)
  float* cs = cs_all[wave];
  const int half = p.rot >> 1, step = gridDim.y;
  const int position = p.pos[t], row = p.rows ? p.rows[t] : t;
  const bool stored = !p.rows || (row >= 0 && row < p.out_rows);  // k and v of this token

  for (int w0 = blockIdx.y; w0 < p.turns[2]; w0 += kAtOnce * step) {
    chunk_t a[kAtOnce], b[kAtOnce];
    E* base[kAtOnce];   // the part's output row (the same in all lanes)
    int at[kAtOnce];    // the item's first channel in it, -1: no item
    int pair[kAtOnce];  // number of the item's first pair, -1 if none of its channels is rotated
    bool one[kAtOnce];  // the item is one channel (and its partner)
#pragma unroll
    for (int i = 0; i < kAtOnce; ++i) {
      const int w = w0 + i * step;
      at[i] = pair[i] = -1;
      const int part = w < p.turns[0] ? 0 : w < p.turns[1] ? 1 : 2;
      if (w >= p.turns[2] || (part > 0 && !stored)) continue;
      const E* src = static_cast<const E*>(p.x[part]) + t * p.ldx[part];
      base[i] = static_cast<E*>(p.out[part]) + (part == 0 ? t : row) * p.ldo[part];
      const int item = (w - (part == 0 ? 0 : p.turns[part - 1])) * 64 + lane;
      if (item >= p.items[part]) continue;
      const int head = divide(item, p.by_per_head[part]), u = item - head * p.per_head[part];
      int c = u * V;      // first channel
      bool turns = part < 2 && c < p.rot;
      one[i] = false;
      if (!PAIRS && part < 2) {
        if (WHOLE) {
          turns = c < half;
          c += turns ? 0 : half;
        } else {
          const int chunks = half / V, turning = chunks + half % V, rest = p.dim - p.rot;
          turns = u < turning;
          const int k = turns ? u : u - turning;
          one[i] = turns ? k >= chunks : rest < V;
          c = one[i] ? (turns ? chunks * V + k - chunks : p.rot + k) : (turns ? 0 : p.rot) + k * V;
          c = turns || one[i] || c + V <= p.dim ? c : p.dim - V;  // (the last chunk that is not rotated may overlap the one before)
        }
      }
      at[i] = head * p.dim + c;
      if (turns) pair[i] = PAIRS ? c >> 1 : c;
      if (!WHOLE && one[i]) {
        a[i].v[0] = src[at[i]];
        if (turns) b[i].v[0] = src[at[i] + half];
        continue;
      }
      a[i] = *reinterpret_cast<const chunk_t*>(src + at[i]);
      if (turns && !PAIRS) b[i] = *reinterpret_cast<const chunk_t*>(src + at[i] + half);
    }
    if (w0 == (int)blockIdx.y) {
      __builtin_amdgcn_sched_barrier(0);
      for (int i = lane; i < half; i += 64) {
        const double x = (double)position * p.freqs[i] * 0.318309886183790671538;  // half turns
        const double quarter = rint(2.0 * x);
        float s, c;
        sincospif((float)(x - 0.5 * quarter), &s, &c);
        const int q = (int)(quarter - 4.0 * floor(0.25 * quarter));
        const float co = q & 1 ? s : c, si = q & 1 ? c : s;
        cs[2 * i] = (q == 1 || q == 2 ? -co : co) * p.magnitude;
        cs[2 * i + 1] = (q >= 2 ? -si : si) * p.magnitude;
      }
      __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
      __builtin_amdgcn_wave_barrier();
      __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
    }
#pragma unroll
    for (int i = 0; i < kAtOnce; ++i) {
      if (at[i] < 0) continue;
      E* const to = base[i] + at[i];
      if (PAIRS) {
        if (pair[i] >= 0) {
#pragma unroll
          for (int e = 0; e < V; e += 2) {
            const int j = pair[i] + (e >> 1);
            if (j < half) {
              const float x = (float)a[i].v[e], y = (float)a[i].v[e + 1], co = cs[2 * j], si = cs[2 * j + 1];
              a[i].v[e] = (E)(x * co - y * si);
              a[i].v[e + 1] = (E)(y * co + x * si);
            }
          }
        }
      } else if (pair[i] >= 0) {
#pragma unroll
        for (int e = 0; e < V; ++e) {
          if (!WHOLE && one[i] && e > 0) break;
          const float co = cs[2 * (pair[i] + e)], si = cs[2 * (pair[i] + e) + 1];
          const float x = (float)a[i].v[e], y = (float)b[i].v[e];
          a[i].v[e] = (E)(x * co - y * si);
          b[i].v[e] = (E)(y * co + x * si);
        }
        if (!WHOLE && one[i])
          to[half] = b[i].v[0];
        else
          *reinterpret_cast<chunk_t*>(to + half) = b[i];
      }
      if (!WHOLE && one[i])
        to[0] = a[i].v[0];
      else
        *reinterpret_cast<chunk_t*>(to) = a[i];
    }
  }
}

// Workgroups that share a token's turns: 4096 waves in all where there are turns for them
int rope_split(int n, int turns) {
  const int want = n < 4096 ? 4096 / n : 1;
  return want < turns ? want : turns;
}

template <class E>
hipError_t launch_layout(RopeDev p, const int (&heads)[3], bool pairs, bool aligned, hipStream_t s) {
  constexpr int V = 16 / sizeof(E);
  const int half = p.rot / 2, rest = p.dim - p.rot;
  for (int i = 0, end = 0; i < 3; ++i) {
    p.per_head[i] = pairs || i == 2 ? p.dim / V : half / V + half % V + (rest < V ? rest : (rest + V - 1) / V);
    p.by_per_head[i] = divider(p.per_head[i]);
    p.items[i] = heads[i] * p.per_head[i];
    p.turns[i] = end += (p.items[i] + 63) / 64;
  }
  const dim3 grid((p.n + kRopeWaves - 1) / kRopeWaves, rope_split(p.n, p.turns[2])), block(kRopeWaves * 64);
  if (pairs) {
    if (aligned) hipLaunchKernelGGL((rope_kernel<E, true, true, true>), grid, block, 0, s, p);
    else hipLaunchKernelGGL((rope_kernel<E, true, false, true>), grid, block, 0, s, p);
  } else {
    if (aligned && half % V == 0) hipLaunchKernelGGL((rope_kernel<E, false, true, true>), grid, block, 0, s, p);
    else hipLaunchKernelGGL((rope_kernel<E, false, false, false>), grid, block, 0, s, p);
  }
  return hipGetLastError();
}

}  // namespace

hipError_t launch_rope(int dtype, const RopeArgs& a, hipStream_t s) {
  if (a.n == 0 || (!a.x[0] && !a.x[1] && !a.x[2])) return hipSuccess;
  RopeDev p{};
  const size_t esize = dtype == DARE_BF16 ? 2 : 4;
  uintptr_t bits = 0;  // of all that lies on 16 bytes or does not
  int heads[3];
  for (int i = 0; i < 3; ++i) {
    p.x[i] = a.x[i];
    p.out[i] = a.out[i];
    p.ldx[i] = a.ldx[i];
    p.ldo[i] = a.ldo[i];
    heads[i] = a.x[i] ? a.heads[i] : 0;
    if (heads[i]) bits |= (uintptr_t)a.x[i] | (uintptr_t)a.out[i] | a.ldx[i] * esize | a.ldo[i] * esize;
  }
  p.n = a.n;
  p.dim = a.dim;
  p.rot = a.rot;
  p.pos = a.pos;
  p.freqs = a.freqs;
  p.rows = a.rows;
  p.out_rows = a.out_rows;
  p.magnitude = a.magnitude;
  return dtype == DARE_BF16 ? launch_layout<bf16_t>(p, heads, a.pairs, bits % 16 == 0, s)
                            : launch_layout<float>(p, heads, a.pairs, bits % 16 == 0, s);
}

}  // namespace dare
