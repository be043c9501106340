// Projection of 8-bit codes on the gfx950 matrix cores:
//     out[t, c] = act(row_scale[t] col_scale[c] sum_k A[t, k] W[c, k] + bias[c]) + residual[t, c]
//
// The sum is formed in 32-bit integers, so it is exact (k below 2^17: 128 * 128 * k < 2^31) whatever its order: a row's
// result does not depend on the shape of the tile it is computed in.  It is rounded to fp32 once and scaled there, by
// the row first; bias, activation and residual sum in fp32, one rounding to the output's type.
//
// Tiles, LDS layout and loops are those of the bf16 projection (gemm_tiles.h): v_mfma_i32_16x16x64_i8 takes the bytes
// and the time of v_mfma_f32_16x16x32_bf16 and twice the k, so k codes cost what k / 2 bf16 do.
#include "gemm_tiles.h"

namespace dare {
namespace {

typedef int i32x4 __attribute__((ext_vector_type(4)));

struct LinearQ8Dev : GemmDev {
  const float* row_scale;
  const float* col_scale;
};

// Codes of 8 bits, outputs of type T
template <typename T>
struct I8Op {
  typedef LinearQ8Dev Dev;
  typedef i32x4 Frag;
  typedef i32x4 Acc;
  static constexpr bool kScaled = true;
  static __device__ __forceinline__ Acc mfma(Frag w, Frag x, Acc sum) { return __builtin_amdgcn_mfma_i32_16x16x64_i8(w, x, sum, 0, 0, 0); }

  // W neighbouring columns col[j] .. of tokens tok[i], as in store_linear
  template <int W, int TM, int TN, class Value>
  static __device__ __forceinline__ void store(const Dev& p, const int (&tok)[TM], const bool (&live)[TM], const int (&col)[TN],
                                               Value value) {
    typedef T out_t __attribute__((ext_vector_type(W)));
    typedef float scale_t __attribute__((ext_vector_type(W)));
    const T* residual = reinterpret_cast<const T*>(p.residual);
    const T* bias = reinterpret_cast<const T*>(p.bias);
    T* out = reinterpret_cast<T*>(p.c0);
    const long ldc = p.ldc, ldr = p.ldr;
    float row_scale[TM];
#pragma unroll
    for (int i = 0; i < TM; ++i) row_scale[i] = p.row_scale[tok[i]];
#pragma unroll
    for (int j = 0; j < TN; ++j) {
      const int c = col[j];
      if (c >= p.n) continue;
      const scale_t col_scale = *reinterpret_cast<const scale_t*>(p.col_scale + c);
      out_t res[TM], b;
      if (residual) {
#pragma unroll
        for (int i = 0; i < TM; ++i) res[i] = *reinterpret_cast<const out_t*>(residual + tok[i] * ldr + c);
      }
      if (bias) b = *reinterpret_cast<const out_t*>(bias + c);
#pragma unroll
      for (int i = 0; i < TM; ++i) {
        float v[W];
#pragma unroll
        for (int e = 0; e < W; ++e) v[e] = fmaf(value(i, j, e) * row_scale[i], col_scale[e], bias ? (float)b[e] : 0.f);
        if constexpr (std::is_same_v<T, float>) {
#pragma unroll
          for (int e = 0; e < W; ++e) v[e] = activate_f32(p.act, v[e]);
        } else {
          activate<true>(p.act, v);
        }
        out_t o;  // (a sum with -0 has all bits of the other term: an activation's -0 stays, as in the wide tiles, which add nothing)
#pragma unroll
        for (int e = 0; e < W; ++e) o[e] = (T)(v[e] + (residual ? (float)res[i][e] : -0.f));
        if (live[i]) *reinterpret_cast<out_t*>(out + tok[i] * ldc + c) = o;
      }
    }
  }
};

template <typename T, int BM, int BN, int WAVES_M, int WAVES_N, int STAGES>
__global__ void __launch_bounds__(WAVES_M* WAVES_N * 64) linear_i8_tile16_kernel(LinearQ8Dev p) {
  __shared__ __attribute__((aligned(1024))) unsigned char smem[smem_bytes<BM, BN, STAGES>()];
  gemm_tile16<BM, BN, WAVES_M, WAVES_N, STAGES, true, I8Op<T>>(p, p.m_max, smem, threadIdx.x, blockIdx.x);
}
template <int TN, bool STREAM>
__global__ void __launch_bounds__(256, 1) linear_i8_quad_kernel(LinearQ8Dev p) {
  __shared__ __attribute__((aligned(1024))) unsigned char smem[kQuadSmem];
  gemm_tiles_quad<TN, STREAM, false, true, I8Op<bf16_t>>(p, p.m_max, smem);
}
template <typename T>
__global__ void __launch_bounds__(512) linear_i8_skinny_kernel(LinearQ8Dev p) {
  __shared__ __attribute__((aligned(1024))) unsigned char smem[8 * 64 * 16];
  skinny_tile<8, 1, true, I8Op<T>>(p, p.m_max, smem, threadIdx.x);
}

template <typename T, int BM, int BN, int WAVES_M, int WAVES_N, int STAGES>
hipError_t launch_tile16(const LinearQ8Dev& p, hipStream_t s) {
  hipLaunchKernelGGL((linear_i8_tile16_kernel<T, BM, BN, WAVES_M, WAVES_N, STAGES>),
                     dim3(grid_for(tiles_of(p.m_max, p.n, BM, BN))), dim3(WAVES_M * WAVES_N * 64), 0, s, p);
  return hipGetLastError();
}
template <int TN, bool STREAM>
hipError_t launch_quad(const LinearQ8Dev& p, hipStream_t s) {
  const int tiles = grid_for(tiles_of(p.m_max, p.n, kPpRows, 64 * TN));
  hipLaunchKernelGGL((linear_i8_quad_kernel<TN, STREAM>), dim3(tiles < kWideGrid ? tiles : kWideGrid), dim3(256), 0, s, p);
  return hipGetLastError();
}
template <typename T>
hipError_t launch(const LinearQ8Dev& p, hipStream_t s) {
  constexpr bool bf16 = std::is_same_v<T, bf16_t>;
  switch (linear_q8_route(p.m_max, p.n, p.k, bf16)) {
    case GemmRoute::kSkinny:
      hipLaunchKernelGGL(linear_i8_skinny_kernel<T>, dim3(p.n / 16), dim3(512), 0, s, p);
      return hipGetLastError();
    case GemmRoute::k32x32: return launch_tile16<T, 32, 32, 2, 2, 8>(p, s);
    case GemmRoute::k64x32: return launch_tile16<T, 64, 32, 4, 2, 6>(p, s);
    case GemmRoute::k32x64: return launch_tile16<T, 32, 64, 1, 4, 6>(p, s);
    case GemmRoute::k64x64: return launch_tile16<T, 64, 64, 2, 4, 4>(p, s);
    case GemmRoute::k64x96: return launch_tile16<T, 64, 96, 4, 2, 6>(p, s);
    case GemmRoute::k64x128: return launch_tile16<T, 64, 128, 2, 4, 5>(p, s);
    case GemmRoute::k128x96: return launch_tile16<T, 128, 96, 4, 2, 4>(p, s);
    case GemmRoute::k128x128: return launch_tile16<T, 128, 128, 2, 4, 4>(p, s);
    case GemmRoute::k128x192: return launch_tile16<T, 128, 192, 2, 4, 3>(p, s);
    case GemmRoute::kQuad192:
      if constexpr (bf16) return launch_quad<3, false>(p, s);
      break;
    case GemmRoute::kQuad256:
      // (outputs larger than half of the last-level cache are stored past the L2, as in the bf16 projection)
      if constexpr (bf16) return (long)p.m_max * p.n * 2 > 128l << 20 ? launch_quad<4, true>(p, s) : launch_quad<4, false>(p, s);
      break;
    default: break;
  }
  return hipErrorInvalidValue;
}

}  // namespace

hipError_t launch_linear_q8(int dtype, const LinearQ8Args& a, hipStream_t s) {
  if (a.m == 0) return hipSuccess;
  LinearQ8Dev p{};
  p.a = reinterpret_cast<const bf16_t*>(a.a);
  p.wt = reinterpret_cast<const bf16_t*>(a.wt);
  p.lda = (int)(a.lda / 2);  // (units of two codes)
  p.k = a.k / 2;
  p.n = p.seg_n = a.n;
  p.m_max = a.m;
  p.k_parts = 1;
  p.c0 = static_cast<bf16_t*>(a.out);
  p.ldc = (int)a.ldo;
  p.bias = static_cast<const bf16_t*>(a.bias);
  p.residual = static_cast<const bf16_t*>(a.residual);
  p.ldr = a.ldr;
  p.act = a.act;
  p.row_scale = a.row_scale;
  p.col_scale = a.col_scale;
  return dtype == DARE_BF16 ? launch<bf16_t>(p, s) : launch<float>(p, s);
}

}  // namespace dare
