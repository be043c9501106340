// Normalisation of token rows into 8-bit codes with a scale per row, with the residual sum in front of it:
//     s = x + o, rounded to the type and stored;   y = s | LayerNorm(s) | s / sqrt(mean(s^2) + eps) * gain
//     scale = max |y| / 127 rounded to fp32;       code = y / scale to the nearest whole number, ties to even
//
// Everything behind s is formed in 64 bits: a code is the one that the formula has.  In fp32 y / scale is off by up to
// 127 * 4 * 2^-24 = 3e-5, and a row's codes would hang on the order in which its sum of squares was formed: one code in
// 10^5 goes to a neighbour, and no other program could say which.
//
// Memory-bound: one read of x and o, one write of s and of a byte per channel.  A row is held in registers from its
// load to its codes, by 8 to 64 lanes (rows of up to 1024 channels) or a workgroup of four waves (up to 16384); longer
// rows are read once per pass.
#include <type_traits>

#include "dare_common.h"
#include "lanes.h"

namespace dare {
namespace {

template <typename T>
struct NormQ8Dev {
  const T* x;
  const T* o;       // or nullptr
  T* x_out;         // or nullptr
  const T* gain;    // nullptr: none
  const T* bias;    // LayerNorm
  int8_t* codes;
  float* scales;
  long ldx, ldo, ldxo, ldc;
  double eps;
  int rows, d;
};

// 8 neighbouring channels
struct Raw8 {
  u32x4 w[2];
};
__device__ __forceinline__ void load8(const bf16_t* p, Raw8& r) { r.w[0] = *reinterpret_cast<const u32x4*>(p); }
__device__ __forceinline__ void load8(const float* p, Raw8& r) {
  r.w[0] = reinterpret_cast<const u32x4*>(p)[0];
  r.w[1] = reinterpret_cast<const u32x4*>(p)[1];
}
__device__ __forceinline__ void values8(const bf16_t*, const Raw8& r, float (&v)[8]) {
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] = __uint_as_float(e & 1 ? r.w[0][e >> 1] & 0xffff0000u : r.w[0][e >> 1] << 16);
}
__device__ __forceinline__ void values8(const float*, const Raw8& r, float (&v)[8]) {
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] = __uint_as_float(r.w[e >> 2][e & 3]);
}
__device__ __forceinline__ void store8(bf16_t* p, const float (&v)[8]) {
  bf16x8 t;
#pragma unroll
  for (int e = 0; e < 8; ++e) t[e] = (bf16_t)v[e];
  *reinterpret_cast<bf16x8*>(p) = t;
}
__device__ __forceinline__ void store8(float* p, const float (&v)[8]) {
#pragma unroll
  for (int h = 0; h < 2; ++h) reinterpret_cast<f32x4*>(p)[h] = f32x4{v[4 * h], v[4 * h + 1], v[4 * h + 2], v[4 * h + 3]};
}

__device__ __forceinline__ double add2(double a, double b) { return a + b; }
__device__ __forceinline__ double max2(double a, double b) { return fmax(a, b); }
// Over the lanes of a row: 8 to 64 neighbouring ones, or the workgroup's 256 through LDS (`sh`: 4 values that nothing else uses)
template <int LANES, class F>
__device__ __forceinline__ double reduce(double v, F f, double* sh) {
  constexpr int STEPS = LANES == 8 ? 3 : LANES == 16 ? 4 : LANES == 32 ? 5 : 6;
  v = over_lanes<0, STEPS>(v, f);
  if constexpr (LANES > 64) {
    static_assert(LANES == 256, "four waves");
    if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = v;
    __syncthreads();
    v = f(f(sh[0], sh[1]), f(sh[2], sh[3]));
  }
  return v;
}

// The code of y: its quotient by the scale (y / scale rounded once, by a product and a correction), to the nearest whole number by
// adding 1.5 * 2^52, which leaves it in the low bits.
__device__ __forceinline__ int code_of(double y, double scale, double inverse) {
  double q = y * inverse;
  q = fma(fma(-q, scale, y), inverse, q);
  const int c = __double2loint(q + 6755399441055744.0);
  return min(max(c, -127), 127);  // (a scale that is no normal number may be off by half)
}
__device__ __forceinline__ u32x2 pack8(const int (&c)[8]) {
  u32x2 r;
#pragma unroll
  for (int h = 0; h < 2; ++h)
    r[h] = (unsigned)(c[4 * h] & 255) | (unsigned)(c[4 * h + 1] & 255) << 8 | (unsigned)(c[4 * h + 2] & 255) << 16 | (unsigned)c[4 * h + 3] << 24;
  return r;
}

struct RowScale {
  double scale, inverse;
  bool finite;
};
// largest: max |y|; rest: 0, or NaN where some y is not finite.  (A scale beyond fp32 is none either.)
__device__ __forceinline__ RowScale row_scale(double largest, double rest, float* to, bool writes) {
  RowScale r;
  float scale = (float)(largest / 127.0);
  r.finite = rest == 0.0 && scale < INFINITY;
  if (!r.finite) scale = __builtin_nanf("");
  r.scale = scale;
  r.inverse = scale > 0.f ? 1.0 / r.scale : 0.0;
  if (writes) *to = scale;
  return r;
}

// Rows of up to 8 LANES HOLD channels, LANES to a row.  y is held from the statistic to the codes where that takes few
// registers; of longer rows s is held, which fp32 does, and y formed twice: fewer registers are more rows on a CU (2000
// x 12288 bf16, rms with a sum 47.3 -> 45.0 us).
template <typename T, int KIND, int LANES, int HOLD>
__global__ void __launch_bounds__(256) norm_q8_kernel(NormQ8Dev<T> p) {
  constexpr int ROWS = 256 / LANES;
  constexpr bool NORM = KIND != DARE_NORM_NONE, LAYER = KIND == DARE_NORM_LAYER, TWICE = NORM && HOLD > 2;
  __shared__ double sh[4][4];
  const int lane = threadIdx.x % LANES;
  const long row = (long)blockIdx.x * ROWS + threadIdx.x / LANES;
  if (row >= p.rows) return;  // (all lanes of a row; no workgroup that shares one)
  const T* x = p.x + row * p.ldx;
  const T* o = p.o + row * p.ldo;
  const int groups = p.d >> 3;
  float s[HOLD][8];
  Raw8 gain[HOLD], bias[HOLD];
  {
    Raw8 a[HOLD], b[HOLD];
#pragma unroll
    for (int h = 0; h < HOLD; ++h) {
      const int g = lane + h * LANES;
      a[h] = b[h] = gain[h] = bias[h] = Raw8{};
      if (g < groups) {
        load8(x + g * 8, a[h]);
        if (p.o) load8(o + g * 8, b[h]);
      }
    }
    if constexpr (NORM) {
#pragma unroll
      for (int h = 0; h < HOLD; ++h) {
        const int g = lane + h * LANES;
        if (g < groups) {
          load8(p.gain + g * 8, gain[h]);
          if (LAYER && p.bias) load8(p.bias + g * 8, bias[h]);
        }
      }
    }
#pragma unroll
    for (int h = 0; h < HOLD; ++h) {
      const int g = lane + h * LANES;
      float w[8];
      values8(x, a[h], s[h]);
      if (p.o) {
        values8(o, b[h], w);
#pragma unroll
        for (int e = 0; e < 8; ++e) s[h][e] = (float)(T)(s[h][e] + w[e]);
      }
      if (p.x_out && g < groups) store8(p.x_out + row * p.ldxo + g * 8, s[h]);
    }
  }
  double mean = 0.0, r = 1.0;
  if constexpr (NORM) {
    double sum = 0.0;
    if constexpr (LAYER) {
#pragma unroll
      for (int h = 0; h < HOLD; ++h)
#pragma unroll
        for (int e = 0; e < 8; ++e) sum += s[h][e];
      mean = reduce<LANES>(sum, add2, sh[0]) / p.d;
      sum = 0.0;
    }
#pragma unroll
    for (int h = 0; h < HOLD; ++h)
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const double v = LAYER ? lane + h * LANES < groups ? s[h][e] - mean : 0.0 : s[h][e];
        sum = fma(v, v, sum);
      }
    r = 1.0 / sqrt(reduce<LANES>(sum, add2, sh[1]) / p.d + p.eps);
  }
  // y of 8 channels (behind the row's end 0: their gain and bias are)
  auto normed = [&](int h, double (&y)[8]) __attribute__((always_inline)) {
    float g[8], b[8];
    values8(x, gain[h], g);
    values8(x, bias[h], b);
#pragma unroll
    for (int e = 0; e < 8; ++e) y[e] = LAYER ? fma(s[h][e] - mean, r * g[e], (double)b[e]) : s[h][e] * (r * g[e]);
  };
  // rest: a NaN that stays if some value is not finite
  double largest = 0.0, rest = 0.0, held[NORM && !TWICE ? HOLD : 1][8];
  if constexpr (NORM) {
#pragma unroll
    for (int h = 0; h < HOLD; ++h) {
      double y[8];
      normed(h, y);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        largest = fmax(largest, fabs(y[e]));
        rest = fma(y[e], 0.0, rest);
        if constexpr (!TWICE) held[h][e] = y[e];
      }
    }
  } else {
    float largest32 = 0.f, rest32 = 0.f;
#pragma unroll
    for (int h = 0; h < HOLD; ++h)
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        largest32 = fmaxf(largest32, fabsf(s[h][e]));
        rest32 = fmaf(s[h][e], 0.f, rest32);
      }
    largest = largest32;
    rest = rest32;
  }
  largest = reduce<LANES>(largest, max2, sh[2]);
  rest = reduce<LANES>(rest, add2, sh[3]);
  const RowScale q = row_scale(largest, rest, p.scales + row, lane == 0);
#pragma unroll
  for (int h = 0; h < HOLD; ++h) {
    const int g = lane + h * LANES;
    int c[8];
    double y[8];
    if constexpr (TWICE) normed(h, y);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      if constexpr (!NORM) y[e] = s[h][e];
      if constexpr (NORM && !TWICE) y[e] = held[h][e];
      c[e] = q.finite ? code_of(y[e], q.scale, q.inverse) : 0;
    }
    if (g < groups) *reinterpret_cast<u32x2*>(p.codes + row * p.ldc + g * 8) = pack8(c);
  }
}

// Rows of any length, a workgroup each, read once for every sum, for the largest value and for the codes
template <typename T, int KIND>
__global__ void __launch_bounds__(256) norm_q8_long_kernel(NormQ8Dev<T> p) {
  __shared__ double sh[4][4];
  const long row = blockIdx.x;
  const T* x = p.x + row * p.ldx;
  const T* o = p.o ? p.o + row * p.ldo : nullptr;
  T* x_out = p.x_out ? p.x_out + row * p.ldxo : nullptr;
  const int groups = p.d >> 3;
  bool summed = false;  // x_out holds the sum (and may be x)
  auto sum_of = [&](int g, double (&y)[8]) {
    Raw8 t;
    float v[8], w[8];
    if (summed) {
      load8(x_out + g * 8, t);
      values8(x, t, v);
    } else {
      load8(x + g * 8, t);
      values8(x, t, v);
      if (o) {
        load8(o + g * 8, t);
        values8(x, t, w);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = (float)(T)(v[e] + w[e]);
      }
      if (x_out) store8(x_out + g * 8, v);
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) y[e] = v[e];
  };
  double mean = 0.0, r = 1.0, y[8];
  if constexpr (KIND == DARE_NORM_LAYER) {
    double sum = 0.0;
    for (int g = threadIdx.x; g < groups; g += 256) {
      sum_of(g, y);
#pragma unroll
      for (int e = 0; e < 8; ++e) sum += y[e];
    }
    summed = x_out != nullptr;
    mean = reduce<256>(sum, add2, sh[0]) / p.d;
  }
  if constexpr (KIND != DARE_NORM_NONE) {
    double sum = 0.0;
    for (int g = threadIdx.x; g < groups; g += 256) {
      sum_of(g, y);
#pragma unroll
      for (int e = 0; e < 8; ++e) sum = fma(y[e] - mean, y[e] - mean, sum);
    }
    summed = x_out != nullptr;
    r = 1.0 / sqrt(reduce<256>(sum, add2, sh[1]) / p.d + p.eps);
  }
  auto value = [&](int g, double (&y)[8]) {
    sum_of(g, y);
    if constexpr (KIND != DARE_NORM_NONE) {
      Raw8 t;
      float v[8];
      load8(p.gain + g * 8, t);
      values8(x, t, v);
#pragma unroll
      for (int e = 0; e < 8; ++e) y[e] = (y[e] - mean) * (r * v[e]);
      if (p.bias) {
        load8(p.bias + g * 8, t);
        values8(x, t, v);
#pragma unroll
        for (int e = 0; e < 8; ++e) y[e] += v[e];
      }
    }
  };
  double largest = 0.0, rest = 0.0;
  for (int g = threadIdx.x; g < groups; g += 256) {
    value(g, y);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      largest = fmax(largest, fabs(y[e]));
      rest = fma(y[e], 0.0, rest);
    }
  }
  summed = x_out != nullptr;
  largest = reduce<256>(largest, max2, sh[2]);
  rest = reduce<256>(rest, add2, sh[3]);
  const RowScale s = row_scale(largest, rest, p.scales + row, threadIdx.x == 0);
  for (int g = threadIdx.x; g < groups; g += 256) {
    value(g, y);
    int c[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) c[e] = s.finite ? code_of(y[e], s.scale, s.inverse) : 0;
    *reinterpret_cast<u32x2*>(p.codes + row * p.ldc + g * 8) = pack8(c);
  }
}

template <typename T, int KIND, int LANES, int HOLD>
hipError_t launch_held(const NormQ8Dev<T>& p, hipStream_t s) {
  constexpr int ROWS = 256 / LANES;
  hipLaunchKernelGGL((norm_q8_kernel<T, KIND, LANES, HOLD>), dim3((p.rows + ROWS - 1) / ROWS), dim3(256), 0, s, p);
  return hipGetLastError();
}
template <typename T, int KIND>
hipError_t launch(const NormQ8Dev<T>& p, hipStream_t s) {
  if (p.d <= 64) return launch_held<T, KIND, 8, 1>(p, s);
  if (p.d <= 128) return launch_held<T, KIND, 16, 1>(p, s);
  if (p.d <= 256) return launch_held<T, KIND, 32, 1>(p, s);
  if (p.d <= 512) return launch_held<T, KIND, 64, 1>(p, s);
  if (p.d <= 1024) return launch_held<T, KIND, 64, 2>(p, s);
  if (p.d <= 2048) return launch_held<T, KIND, 256, 1>(p, s);
  if (p.d <= 4096) return launch_held<T, KIND, 256, 2>(p, s);
  if (p.d <= 6144) return launch_held<T, KIND, 256, 3>(p, s);
  if (p.d <= 8192) return launch_held<T, KIND, 256, 4>(p, s);
  if (p.d <= 12288) return launch_held<T, KIND, 256, 6>(p, s);
  if (p.d <= 16384) return launch_held<T, KIND, 256, 8>(p, s);
  hipLaunchKernelGGL((norm_q8_long_kernel<T, KIND>), dim3(p.rows), dim3(256), 0, s, p);
  return hipGetLastError();
}

template <typename T>
hipError_t launch_type(const NormQ8Args& a, hipStream_t s) {
  NormQ8Dev<T> p;
  p.x = static_cast<const T*>(a.x);
  p.o = static_cast<const T*>(a.o);
  p.x_out = static_cast<T*>(a.x_out);
  p.gain = static_cast<const T*>(a.gain);
  p.bias = static_cast<const T*>(a.bias);
  p.codes = a.codes;
  p.scales = a.scales;
  p.ldx = a.ldx;
  p.ldo = a.ldo;
  p.ldxo = a.ldxo;
  p.ldc = a.ldc;
  p.eps = a.eps;
  p.rows = a.rows;
  p.d = a.d;
  switch (a.kind) {
    case DARE_NORM_NONE: return launch<T, DARE_NORM_NONE>(p, s);
    case DARE_NORM_LAYER: return launch<T, DARE_NORM_LAYER>(p, s);
    case DARE_NORM_RMS: return launch<T, DARE_NORM_RMS>(p, s);
  }
  return hipErrorInvalidValue;
}

}  // namespace

hipError_t launch_norm_q8(int dtype, const NormQ8Args& a, hipStream_t s) {
  if (a.rows == 0) return hipSuccess;
  return dtype == DARE_BF16 ? launch_type<bf16_t>(a, s) : launch_type<float>(a, s);
}

}  // namespace dare
