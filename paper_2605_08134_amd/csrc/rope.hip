// Rotary embedding by positions: the channel pair (a, b) number i of a head of a token at position p becomes
//     (a cos - b sin, b cos + a sin),   angle p f_i,   cos and sin times a common magnitude,
// for the first rot channels of every head; the others go through as they are.  Queries, keys and values of a token in
// one launch: Q is rotated, K is rotated and stored at the token's cache row, V is stored there as it is.
//
// No table of angles: it would have to reach the largest position, and its rows are bytes that the
// launch has to read.  A wave owns a token (or some of its heads); lane i takes cos and sin of pair i in 64
// bits, where a position of 10^6 costs nothing of the angle's last bits in fp32, and leaves them to the other
// lanes in LDS.
#include "dare_common.h"

namespace dare {
namespace {

struct RopeDev {
  const void* x[3];    // q, k, v
  void* out[3];
  long ldx[3], ldo[3]; // elements between tokens
  int heads[3];        // 0: not there
  int n, dim, rot;
  const int32_t* pos;
  const double* freqs;
  const int32_t* rows; // rows of k and v outputs, or nullptr
  int out_rows;
  float magnitude;
};

constexpr int kRopeWaves = 4;

// V elements (of type E) that are read and written at once
template <class E, int V>
struct alignas(V * sizeof(E) == 16 ? 16 : sizeof(E)) Chunk {
  E v[V];
};

// One token's part x (0 q, 1 k, 2 v) by the lanes of a wave: items `first`, first + step, ...  PAIRS: channels (2 i, 2 i + 1)
// are a pair; else i and i + rot / 2.
template <class E, int V, bool PAIRS>
__device__ __forceinline__ void rope_part(const E* x, E* out, int heads, int dim, int rot, const float* cs, bool turns,
                                          int first, int step) {
  typedef Chunk<E, V> chunk_t;
  const int half = rot >> 1;
  if (!turns || PAIRS) {
    // whole chunks of neighbouring channels
    const int per_head = dim / V, items = heads * per_head;
    for (int it = first; it < items; it += step) {
      const int u = it % per_head;
      chunk_t c = reinterpret_cast<const chunk_t*>(x)[it];
      if constexpr (PAIRS && V > 1) {
        if (turns) {
#pragma unroll
          for (int e = 0; e < V; e += 2) {
            const int i = (u * V + e) >> 1;
            if (i < half) {
              const float a = (float)c.v[e], b = (float)c.v[e + 1], co = cs[2 * i], si = cs[2 * i + 1];
              c.v[e] = (E)(a * co - b * si);
              c.v[e + 1] = (E)(b * co + a * si);
            }
          }
        }
      }
      reinterpret_cast<chunk_t*>(out)[it] = c;
    }
    return;
  }
  // chunk u < half / V with its partner half channels on; behind them the channels that are not rotated
  const int turning = half / V, per_head = turning + (dim - rot) / V, items = heads * per_head;
  for (int it = first; it < items; it += step) {
    const int h = it / per_head, u = it - h * per_head;
    const E* src = x + (long)h * dim;
    E* dst = out + (long)h * dim;
    if (u < turning) {
      chunk_t a = *reinterpret_cast<const chunk_t*>(src + u * V), b = *reinterpret_cast<const chunk_t*>(src + half + u * V);
#pragma unroll
      for (int e = 0; e < V; ++e) {
        const float co = cs[2 * (u * V + e)], si = cs[2 * (u * V + e) + 1];
        const float p = (float)a.v[e], q = (float)b.v[e];
        a.v[e] = (E)(p * co - q * si);
        b.v[e] = (E)(q * co + p * si);
      }
      *reinterpret_cast<chunk_t*>(dst + u * V) = a;
      *reinterpret_cast<chunk_t*>(dst + half + u * V) = b;
    } else {
      const int c = rot + (u - turning) * V;
      *reinterpret_cast<chunk_t*>(dst + c) = *reinterpret_cast<const chunk_t*>(src + c);
    }
  }
}

// gridDim.y workgroups share the heads of a token between them
template <class E, int V, bool PAIRS>
__global__ void __launch_bounds__(kRopeWaves * 64) rope_kernel(RopeDev p) {
  __shared__ float cs_all[kRopeWaves][kRopeMaxDim];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int t = blockIdx.x * kRopeWaves + wave;
  if (t >= p.n) return;  // (no barrier below: a wave reads what its own lanes wrote)
  float* cs = cs_all[wave];
  const double position = (double)p.pos[t];
  for (int i = lane; i < p.rot >> 1; i += 64) {
    double s, c;
    sincospi(position * p.freqs[i] * 0.318309886183790671538, &s, &c);
    cs[2 * i] = (float)(c * p.magnitude);
    cs[2 * i + 1] = (float)(s * p.magnitude);
  }
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
  const int first = blockIdx.y * 64 + lane, step = gridDim.y * 64;
  const long row = p.rows ? (long)p.rows[t] : t;
#pragma unroll
  for (int part = 0; part < 3; ++part) {
    if (p.heads[part] == 0) continue;
    long to = t;
    if (part > 0 && p.rows) {
      if (row < 0 || row >= p.out_rows) continue;
      to = row;
    }
    rope_part<E, V, PAIRS>(static_cast<const E*>(p.x[part]) + t * p.ldx[part], static_cast<E*>(p.out[part]) + to * p.ldo[part],
                           p.heads[part], p.dim, p.rot, cs, part < 2, first, step);
  }
}

// V: elements at once where that is possible; NARROW: channel by channel, or pair by pair where they are neighbours
template <class E, int V, bool NARROW>
hipError_t launch_layout(const RopeDev& p, bool pairs, hipStream_t s) {
  const dim3 grid((p.n + kRopeWaves - 1) / kRopeWaves, 1), block(kRopeWaves * 64);
  if (pairs)
    hipLaunchKernelGGL((rope_kernel<E, NARROW ? 2 : V, true>), grid, block, 0, s, p);
  else
    hipLaunchKernelGGL((rope_kernel<E, NARROW ? 1 : V, false>), grid, block, 0, s, p);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_rope(int dtype, const RopeArgs& a, hipStream_t s) {
  if (a.n == 0) return hipSuccess;
  RopeDev p{};
  const size_t esize = dtype == DARE_BF16 ? 2 : 4;
  uintptr_t bits = 0;  // of everything that has to be a multiple of 16 bytes
  for (int i = 0; i < 3; ++i) {
    p.x[i] = a.x[i];
    p.out[i] = a.out[i];
    p.ldx[i] = a.ldx[i];
    p.ldo[i] = a.ldo[i];
    p.heads[i] = a.x[i] ? a.heads[i] : 0;
    if (p.heads[i]) bits |= (uintptr_t)a.x[i] | (uintptr_t)a.out[i] | a.ldx[i] * esize | a.ldo[i] * esize;
  }
  p.n = a.n;
  p.dim = a.dim;
  p.rot = a.rot;
  p.pos = a.pos;
  p.freqs = a.freqs;
  p.rows = a.rows;
  p.out_rows = a.out_rows;
  p.magnitude = a.magnitude;
  // 16 bytes at a time where everything lies on such a boundary and, by halves, a chunk has its partner in one chunk
  const int v = (int)(16 / esize);
  const bool wide = bits % 16 == 0 && a.dim % v == 0 && (a.pairs || (a.rot / 2) % v == 0);
  if (dtype == DARE_BF16)
    return wide ? launch_layout<bf16_t, 8, false>(p, a.pairs, s) : launch_layout<bf16_t, 8, true>(p, a.pairs, s);
  return wide ? launch_layout<float, 4, false>(p, a.pairs, s) : launch_layout<float, 4, true>(p, a.pairs, s);
}

}  // namespace dare
