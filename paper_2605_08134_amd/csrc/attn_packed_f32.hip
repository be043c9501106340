// fp32 path of attention over packed sequences (attn_packed.hip, same rows and keys) on v_mfma_f32_16x16x4_f32.
//
// A workgroup serves 16 rows of one key head; its four waves take every fourth tile of 16 keys.  Transposed logits
// S^T = K Q^T: lane L holds row L & 15 and four neighbouring keys, which is the operand layout of the probabilities in
// O^T = V^T P^T, so they never leave the lane.  K, V and Q go from global memory straight into registers, all loads of a tile in
// flight at once.  The waves are joined in their order through LDS.
#include "attn_packed_rows.h"

namespace dare {
namespace {

constexpr int kWaves = 4, kRows = 16;

struct PackedF32Dev {
  const float* q;
  const float* k;
  const float* v;
  float* out;
  long ldq, ldk, ldv, ldo;
  PackedRows rows;
  int n_kv;
  float scale;
};

template <int DH>
__global__ void __launch_bounds__(kWaves * 64) attn_packed_f32_kernel(PackedF32Dev p) {
  constexpr int C = DH / 16;  // 16-channel blocks
  __shared__ f32x4 o_part[kWaves][C][64];
  __shared__ float m_part[kWaves][16], l_part[kWaves][16];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int l16 = lane & 15, kq = lane >> 4;
  const int kvh = blockIdx.x % p.n_kv, g = p.rows.n_blocks - 1 - (int)(blockIdx.x / p.n_kv);
  Place at;
  if (!find_block<kRows>(p.rows, g, at)) return;
  const int least = row_limit(p.rows, at, at.row0), most = row_limit(p.rows, at, at.row0 + at.rows - 1);

  const bool valid = l16 < at.rows;
  const int j = at.row0 + (valid ? l16 : at.rows - 1), i = divide(j, p.rows.by_group);
  const int head = kvh * p.rows.group + (j - i * p.rows.group);
  const int lim = packed_limit(i, at.shift, at.len_k, p.rows.causal_block, p.rows.by_causal_block);
  const float* qrow = p.q + (long)(at.q0 + i) * p.ldq + head * DH + kq * 4;
  f32x4 qf[C], acc[C];
#pragma unroll
  for (int c = 0; c < C; ++c) {
    qf[c] = *reinterpret_cast<const f32x4*>(qrow + c * 16);
    acc[c] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  const float* kbase = p.k + (long)at.k0 * p.ldk + kvh * DH;
  const float* vbase = p.v + (long)at.k0 * p.ldv + kvh * DH;
  float m_run = -__FLT_MAX__, l_run = 0.f;
  for (int key0 = wave * 16; key0 < most; key0 += kWaves * 16) {
    f32x4 kf[C];
    float vf[4][C];
    {
      const int key = key0 + l16 < at.len_k ? key0 + l16 : at.len_k - 1;
#pragma unroll
      for (int c = 0; c < C; ++c) kf[c] = *reinterpret_cast<const f32x4*>(kbase + (long)key * p.ldk + c * 16 + kq * 4);
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int key = key0 + kq * 4 + e < at.len_k ? key0 + kq * 4 + e : at.len_k - 1;
      const float* vr = vbase + (long)key * p.ldv + l16;
#pragma unroll
      for (int c = 0; c < C; ++c) vf[e][c] = vr[c * 16];
    }
    __builtin_amdgcn_sched_barrier(0);
    // z[e]: logit of key key0 + 4 kq + e
    f32x4 z = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
      for (int e = 0; e < 4; ++e) z = __builtin_amdgcn_mfma_f32_16x16x4f32(kf[c][e], qf[c][e], z, 0, 0, 0);
    float top = -INFINITY;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      z[e] = key0 + kq * 4 + e < lim ? z[e] * p.scale : -INFINITY;
      top = fmaxf(top, z[e]);
    }
    top = row_max(top);
    const float m_new = fmaxf(m_run, top);  // (finite from below: a row that sees nothing has probabilities 0)
    const float alpha = expf(m_run - m_new);
    m_run = m_new;
    l_run *= alpha;
#pragma unroll
    for (int c = 0; c < C; ++c) acc[c] *= alpha;
    bool bad = false;
    if (key0 + 16 > least) {  // some row does not see some key: values that are not finite one by one, below
#pragma unroll
      for (int e = 0; e < 4; ++e)
#pragma unroll
        for (int c = 0; c < C; ++c)
          if (!(fabsf(vf[e][c]) < INFINITY)) {
            bad = true;
            vf[e][c] = 0.f;
          }
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float pr = expf(z[e] - m_run);
      l_run += pr;
#pragma unroll
      for (int c = 0; c < C; ++c) acc[c] = __builtin_amdgcn_mfma_f32_16x16x4f32(vf[e][c], pr, acc[c], 0, 0, 0);
    }
    if (__builtin_expect(__any(bad), 0)) {
      for (int k = key0; k < key0 + 16 && k < at.len_k; ++k)
#pragma unroll
        for (int c = 0; c < C; ++c) {
          const f32x4 v = *reinterpret_cast<const f32x4*>(vbase + (long)k * p.ldv + c * 16 + kq * 4);
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (k < lim && !(fabsf(v[e]) < INFINITY)) acc[c][e] += v[e];
        }
    }
  }
  l_run = row_sum(l_run);
  if (kq == 0) {
    m_part[wave][l16] = m_run;
    l_part[wave][l16] = l_run;
  }
#pragma unroll
  for (int c = 0; c < C; ++c) o_part[wave][c][lane] = acc[c];
  __syncthreads();
  float m_all = m_part[0][l16], l_all = 0.f, f[kWaves];
#pragma unroll
  for (int w = 1; w < kWaves; ++w) m_all = fmaxf(m_all, m_part[w][l16]);
#pragma unroll
  for (int w = 0; w < kWaves; ++w) {
    f[w] = expf(m_part[w][l16] - m_all);
    l_all += l_part[w][l16] * f[w];
  }
  if (!valid) return;
  const float inv = l_all == 0.f ? 0.f : 1.0f / l_all;
  float* orow = p.out + (long)(at.q0 + i) * p.ldo + head * DH + kq * 4;
  for (int c = wave; c < C; c += kWaves) {
    f32x4 o = o_part[0][c][lane] * f[0];
#pragma unroll
    for (int w = 1; w < kWaves; ++w) o += o_part[w][c][lane] * f[w];
    *reinterpret_cast<f32x4*>(orow + c * 16) = o * inv;
  }
}

}  // namespace

hipError_t launch_attn_packed_f32(const PackedArgs& a, hipStream_t s) {
  PackedF32Dev p;
  p.q = static_cast<const float*>(a.q);
  p.k = static_cast<const float*>(a.k);
  p.v = static_cast<const float*>(a.v);
  p.out = static_cast<float*>(a.out);
  p.ldq = a.ldq;
  p.ldk = a.ldk;
  p.ldv = a.ldv;
  p.ldo = a.ldo;
  p.rows = packed_rows(a, (int)((long)a.total_q * (a.n_heads / a.n_kv_heads) / kRows) + a.batch);
  p.n_kv = a.n_kv_heads;
  p.scale = a.scale;
  const dim3 grid((unsigned)((long)p.rows.n_blocks * p.n_kv));
  if (a.head_dim == 128)
    hipLaunchKernelGGL(attn_packed_f32_kernel<128>, grid, dim3(kWaves * 64), 0, s, p);
  else
    hipLaunchKernelGGL(attn_packed_f32_kernel<64>, grid, dim3(kWaves * 64), 0, s, p);
  return hipGetLastError();
}

}  // namespace dare
