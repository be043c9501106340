// Log-probabilities of given tokens, entropy and top alternatives of rows of logits x, z = scale x:
//     S = sum exp(z - r),  logprob(v) = z_v - r - log S,  entropy = log S - sum exp(z - r) (z - r) / S,   r about max z
//
// One workgroup per row and one pass over it, bound by memory (exponentials: 64 elements take a SIMD 45 cycles, which
// is 7 TB/s for bf16).  Every lane keeps the sums over its elements relative to its own largest one; they are joined at
// the end.
//
// Alternatives.  Order: the larger logit first, of equal ones the lower id; as whole numbers, `order_key`, in which no
// two elements are equal.  In the pass a lane keeps only its largest chunk (16 bytes) and where that lies.  Take T, the
// k-th largest of the lanes' keys, or a lower one: an element below T has k better ones, so the alternatives lie in the
// lanes whose key is T or more, about k of them; those lanes' elements are read again (k / 1024 of the row), the ones
// from T on are listed, and a listed element's rank is how many others are above it.  Few rows: parts of a row by a
// workgroup each, and a second launch that joins what they found.
// The list may overflow where many of the largest logits fall into the same few lanes; then the alternatives are found
// one after the other.
#include <type_traits>

#include "dare_common.h"
#include "lanes.h"

namespace dare {
namespace {

typedef unsigned long long u64;

template <typename T>
struct LogprobsDev {
  const T* x;
  long ld;
  int vocab, top;
  float scale;
  const int32_t* tokens;
  float* logprobs;
  float* entropy;
  int32_t* top_ids;
  float* top_logprobs;
  // rows cut into parts of part_len elements: of every part its sums, and the keys of its `top` largest elements, 0
  // where it has fewer
  int parts, part_len;
  f32x4* part_sums;  // (r, s, t), and 1 where they do not stand for the part, 2 where they do only beside a part whose r is above kLowest
  unsigned long long* part_keys;
};

// What a workgroup does: a row, a part of one, or the joining of a row's parts (the row itself, where some part's sums say nothing)
enum class Does { kRow, kPart, kJoin };

constexpr int kMostParts = 16;
constexpr int kAhead = 4;       // chunks of a lane in flight
constexpr float kLog2e = 1.44269504f, kLn2 = 0.693147181f;

// Elements of 16 bytes
__device__ __forceinline__ void unpack(const bf16_t*, const u32x4 r, float (&v)[8]) {
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] = __uint_as_float(e & 1 ? r[e >> 1] & 0xffff0000u : r[e >> 1] << 16);
}
__device__ __forceinline__ void unpack(const float*, const u32x4 r, float (&v)[4]) {
#pragma unroll
  for (int e = 0; e < 4; ++e) v[e] = __uint_as_float(r[e]);
}

// (value, place): larger values first, then lower places; 0 is below all.  Both zeros are one value.
__device__ __forceinline__ u64 order_key(float v, unsigned place) {
  const unsigned b = __float_as_uint(v + 0.f);
  return (u64)(b ^ ((int)b < 0 ? 0xffffffffu : 0x80000000u)) << 32 | (unsigned)~place;
}
__device__ __forceinline__ float key_value(u64 key) {
  const unsigned b = (unsigned)(key >> 32);
  return __uint_as_float(b ^ ((int)b < 0 ? 0x80000000u : 0xffffffffu));
}
__device__ __forceinline__ u64 wave_max(u64 v) {
  return over_lanes(v, [](u64 a, u64 b) { return a > b ? a : b; });
}

// Sums of a set of elements in units of 2^r, exponents d = c x - r, c = scale log2(e), by one product and sum each,
// rounded once.  r is c x of the largest element, rounded.  It cancels in every result, so any r near it is right; but
// the largest element's own exponent is that rounding, up to half a step of r: at most 1/4 where |r| is below 2^23, but
// 128 and more, beyond fp32 as a power, from 2^31 on.  So
//   * r is not below kLowest = -2^23.  Elements that far down have exponents below 1/4, or 0 beside any r that is above it.
//   * A row whose r comes out as -2^23 or 2^23 or beyond (scaled logits beyond 5.8e6: temperatures near 0, or all of
//     the row on a low mask) takes a second pass.
// WIDE, the second pass: r stands for an x and exponents are c (x - r), which takes an instruction more and has no such
// limits.  From scales of kWideScale on, where logits of 90 are as much, it is the first and only one (2048 x 126464 at
// a scale of 1e8: 94 us, 161 with both passes, 92 with the first alone).
constexpr float kLowest = -8388608.f, kWideScale = 65536.f;
struct Sums {
  float r;  // kLowest or -FLT_MAX (WIDE: -FLT_MAX) without an element
  float s;  // sum of 2^d
  float t;  // sum of 2^d d
};
template <bool WIDE>
__device__ __forceinline__ float exponent(float x, float r, float c) {
  return WIDE ? (x - r) * c : fmaf(x, c, -r);
}
// The same sums in units of 2^r for a larger r
template <bool WIDE>
__device__ __forceinline__ void raise(Sums& a, float r, float c) {
  const float d = WIDE ? (a.r - r) * c : a.r - r, f = __builtin_amdgcn_exp2f(d);
  a.t = f * fmaf(fmaxf(d, -200.f), a.s, a.t);  // (0 times infinity is none; a NaN stays in the sum)
  a.s *= f;
  a.r = r;
}
// Of 2^TO lanes together
template <bool WIDE, int TO = 6>
__device__ __forceinline__ Sums join(Sums a, float c) {
  raise<WIDE>(a, over_lanes<0, TO>(a.r, [](float x, float y) { return fmaxf(x, y); }), c);
  const auto add = [](float x, float y) { return x + y; };
  return {a.r, over_lanes<0, TO>(a.s, add), over_lanes<0, TO>(a.t, add)};
}

template <typename T, int THREADS, Does DOES>
__global__ void __launch_bounds__(THREADS, DOES == Does::kJoin ? 4 : 8) logprobs_kernel(LogprobsDev<T> p) {
  constexpr int WAVES = THREADS / 64, E = 16 / sizeof(T);
  constexpr int kListed = THREADS == 64 ? 512 : 2048;  // elements that the list holds
  // a wave's largest keys: enough for the k-th largest, and so many that it is near it (of a single wave all)
  constexpr int MOST = WAVES == 1 ? 64 : 32 / WAVES > 4 ? 32 / WAVES : 4;
  __shared__ Sums wave_sums[WAVES];
  __shared__ u64 wave_keys[WAVES * MOST], listed[kListed], limit;
  __shared__ int lanes[THREADS], n_lanes, n_listed;

  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const long row = DOES == Does::kPart ? blockIdx.x / p.parts : blockIdx.x;
  const int offset = DOES == Does::kPart ? (int)(blockIdx.x % p.parts) * p.part_len : 0;
  const int vocab = DOES == Does::kPart && p.vocab - offset > p.part_len ? p.part_len : p.vocab - offset;
  const int top = p.top;
  const T* x = p.x + row * p.ld + offset;
  const float c = p.scale * kLog2e;
  // elements in front of the first 16-byte boundary, whole chunks, elements behind the last one
  const int to_boundary = (int)((16 - ((uintptr_t)x & 15)) & 15) / (int)sizeof(T);
  const int head = to_boundary < vocab ? to_boundary : vocab;
  const int chunks = (vocab - head) / E, singles = vocab - chunks * E;
  const T* body = x + head;
  auto single_place = [&](int i) { return i < head ? i : i + chunks * E; };
  auto chunk = [&](int i) { return reinterpret_cast<const u32x4*>(body)[i]; };
  if (tid == 0) n_lanes = n_listed = 0;

  Sums all;
  const bool wide_first = p.scale >= kWideScale;
  bool wide = wide_first;
  // (a NaN, or the difference of two infinities, is in the sum)
  auto undefined = [&]() { return !(all.s >= 0.f); };
  auto logprob = [&](float v) {
    if (undefined()) return __builtin_nanf("");
    if (v == -INFINITY) return -INFINITY;
    const float log2_sum = __log2f(all.s);
    if (wide) return 2.f * ((0.5f * v - 0.5f * all.r) * p.scale) - kLn2 * log2_sum;  // (the difference may be beyond fp32, times scale it need not)
    const float d = fmaf(v, c, -all.r) - log2_sum;
    return d > -INFINITY ? kLn2 * d : fmaf(v, p.scale, -kLn2 * all.r);  // (c v beyond fp32, scale v perhaps not)
  };
  float token_logit = -INFINITY;  // (read ahead of all else: two reads in a row)
  if (DOES != Does::kPart && p.tokens && tid == 0) {
    const int token = p.tokens[row];
    if (token >= 0 && token < p.vocab) token_logit = (float)x[token];
  }
  auto put_sums = [&]() {
    if (tid != 0) return;
    if (p.tokens) p.logprobs[row] = logprob(token_logit);
    if (p.entropy)
      p.entropy[row] = undefined() ? __builtin_nanf("") : all.s == 0.f ? 0.f : fmaxf(kLn2 * (__log2f(all.s) - all.t / all.s), 0.f);
  };
  // the alternative of rank i, 0: there is none
  auto put = [&](int i, u64 key) {
    if constexpr (DOES == Does::kPart) {
      p.part_keys[(long)blockIdx.x * top + i] = key;
    } else {
      p.top_ids[row * top + i] = key && !undefined() ? (int32_t)~(unsigned)key : -1;
      p.top_logprobs[row * top + i] = logprob(key ? key_value(key) : -INFINITY);
    }
  };
  auto put_listed = [&](int n) {
    for (int i = tid; i < n; i += THREADS) {
      const u64 own = listed[i];
      int above = 0;
#pragma unroll 8
      for (int j = 0; j < n; ++j) above += listed[j] > own;
      if (above < top) put(above, own);
    }
  };
  if constexpr (DOES == Does::kJoin) {
    static_assert(kMostParts * kTopMost <= 2 * THREADS && kMostParts <= 64, "two keys per thread, a part per lane");
    const int n = p.parts * top;  // at most 2 THREADS
    const f32x4 part = lane < p.parts ? p.part_sums[row * p.parts + lane] : f32x4{-__FLT_MAX__, 0.f, 0.f, 0.f};
    u64 keys[2], from = ~0ull;
#pragma unroll
    for (int k = 0; k < 2; ++k) keys[k] = tid + k * THREADS < n ? p.part_keys[row * n + tid + k * THREADS] : 0;
    // every part has this many keys from its own limit on, so the lowest limit has `top` keys from it on
    if (top > 0 && lane < p.parts) from = p.part_keys[(row * p.parts + lane) * top + (top - 1) / p.parts];
    const Sums sums = {part[0], part[1], part[2]};
    all = wide_first ? join<true>(sums, c) : join<false>(sums, c);
    if (!__any(part[3] == 1.f || (part[3] == 2.f && all.r == kLowest))) {
      put_sums();
      if (top == 0) return;
      from = over_lanes(from, [](u64 a, u64 b) { return a < b ? a : b; });
      __syncthreads();
#pragma unroll
      for (int k = 0; k < 2; ++k)
        if (keys[k] != 0 && keys[k] >= from) listed[atomicAdd(&n_listed, 1)] = keys[k];
      __syncthreads();
      const int found = n_listed;
      put_listed(found);
      if (tid >= found && tid < top) put(tid, 0);
      return;
    }
  }

  float best = -INFINITY;  // largest element, and the first place of its chunk
  unsigned place = 0;
  // the row's sums, in wave_sums by waves
  auto pass = [&](auto wide) {
    constexpr bool WIDE = decltype(wide)::value;
    Sums sum = {WIDE ? -__FLT_MAX__ : kLowest, 0.f, 0.f};
    auto take = [&](const float (&v)[E]) {
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const float d = exponent<WIDE>(v[e], sum.r, c), f = __builtin_amdgcn_exp2f(d);
        sum.s += f;
        sum.t = fmaf(f, fmaxf(d, -200.f), sum.t);
      }
    };
    auto rise = [&]() { raise<WIDE>(sum, fmaxf(sum.r, WIDE ? best : best * c), c); };
    for (int i = tid; i < chunks; i += kAhead * THREADS) {
      // Chunks that no lane of the wave has are left out of the arithmetic: bf16, 4096 x 4096 20.1 -> 18.8 us, 1000 x
      // 151936 62.6 -> 60.9; in fp32, with half as much of it per byte, 300 x 32003 16.5 and 16.6, 1024 x 126464 93.8
      // and 95.0.
      constexpr bool kLeaveOut = sizeof(T) == 2;
      const int first = __builtin_amdgcn_readfirstlane(i);
      u32x4 r[kAhead];
#pragma unroll
      for (int a = 0; a < kAhead; ++a) {
        constexpr unsigned none = sizeof(T) == 2 ? 0xff80ff80u : 0xff800000u;  // -infinity
        r[a] = u32x4{none, none, none, none};
        if (i + a * THREADS < chunks) r[a] = chunk(i + a * THREADS);
      }
      float v[kAhead][E];
#pragma unroll
      for (int a = 0; a < kAhead; ++a) {
        if (kLeaveOut && first + a * THREADS >= chunks) continue;
        unpack(x, r[a], v[a]);
        float most = v[a][0];
#pragma unroll
        for (int e = 1; e < E; ++e) most = fmaxf(most, v[a][e]);
        if (most > best) {
          best = most;
          place = head + (i + a * THREADS) * E;
        }
      }
      rise();
#pragma unroll
      for (int a = 0; a < kAhead; ++a)
        if (!kLeaveOut || first + a * THREADS < chunks) take(v[a]);
    }
    if (tid < singles) {
      const unsigned at = single_place(tid);
      float v[E];
#pragma unroll
      for (int e = 0; e < E; ++e) v[e] = -INFINITY;
      v[0] = (float)x[at];
      if (v[0] > best || (v[0] == best && v[0] > -INFINITY && at < place)) {
        best = v[0];
        place = at;
      }
      rise();
      take(v);
    }
    sum = join<WIDE>(sum, c);
    if (lane == 0) wave_sums[wave] = sum;
  };
  auto joined = [&](auto wide) {
    return join<decltype(wide)::value, WAVES == 16 ? 4 : WAVES == 4 ? 2 : 0>(wave_sums[lane % WAVES], c);
  };
  if (wide_first)
    pass(std::true_type{});
  else
    pass(std::false_type{});
  u64 key = best > -INFINITY ? order_key(best, place) : 0;
  if (top > 0) {
    const int most = WAVES == 1 ? 64 : (top + WAVES - 1) / WAVES > 4 ? (top + WAVES - 1) / WAVES : top < 4 ? top : 4;
    float left = best;  // of the lanes that are not taken yet
    if constexpr (WAVES == 1) wave_keys[lane] = key;
    for (int j = 0; WAVES > 1 && j < most; ++j) {
      const float v = over_lanes(left, [](float a, float b) { return fmaxf(a, b); });
      u64 w = 0;
      if (v > -INFINITY) {
        const u64 equal = __ballot(left == v);
        unsigned first;
        if (equal & (equal - 1))  // the lowest place of equal ones
          first = over_lanes(left == v ? place : ~0u, [](unsigned a, unsigned b) { return a < b ? a : b; });
        else
          first = __builtin_amdgcn_readlane(place, __ffsll((long long)equal) - 1);
        w = order_key(v, first);
        if (left == v && place == first) left = -INFINITY;
      }
      if (lane == 0) wave_keys[wave * most + j] = w;
    }
    __syncthreads();
    if (wave == 0) {  // the one with top - 1 keys above it; without so many keys: 1, which is below all
      const int n = WAVES * most;
      const u64 own = lane < n ? wave_keys[lane] : 0;
      int above = 0;
#pragma unroll 8
      for (int j = 0; j < n; ++j) above += wave_keys[j] > own;
      if (lane == 0) limit = 1;
      if (own > 0 && above == top - 1) limit = own;
    }
  }
  __syncthreads();
  all = wide_first ? joined(std::true_type{}) : joined(std::false_type{});
  // r too large (or infinite) for the sums; or too low, which it also is without an element; or an element that is NaN
  const bool again = !wide_first && (!(fabsf(all.r) < -kLowest) || undefined());
  if constexpr (DOES == Does::kPart) {
    // (too low, as where a number masks all places: right beside a part that is not; without an element: right)
    float says = 0.f;
    if (again && (undefined() || all.r > 0.f)) {
      says = 1.f;
    } else if (again) {
      says = __syncthreads_or(best > -INFINITY) ? 2.f : 0.f;
    }
    if (tid == 0) p.part_sums[blockIdx.x] = f32x4{all.r, all.s, all.t, says};
  } else {
    if (again) {
      wide = true;
      __syncthreads();
      pass(std::true_type{});
      __syncthreads();
      all = joined(std::true_type{});
    }
    put_sums();
  }
  if (top == 0) return;
  const u64 from = limit;
  if (key >= from) lanes[atomicAdd(&n_lanes, 1)] = tid;
  __syncthreads();
  // the elements of the listed lanes: chunks l, l + THREADS, .. of each lane, then its single one
  const int per_lane = (chunks + THREADS - 1) / THREADS + 1, n = n_lanes * per_lane;
  auto elements = [&](auto use) {
    for (int i = tid; i < n; i += THREADS) {
      const int l = lanes[i / per_lane], j = i % per_lane;
      if (j < per_lane - 1) {
        const int at = l + j * THREADS;
        if (at >= chunks) continue;
        float v[E];
        unpack(x, chunk(at), v);
#pragma unroll
        for (int e = 0; e < E; ++e) use(v[e], head + at * E, e);
      } else if (l < singles) {
        use((float)x[single_place(l)], single_place(l), 0);
      }
    }
  };
  // (the limit is a lane's key: its value with the first place of its chunk)
  elements([&](float v, int first, int e) {
    if (v > -INFINITY && order_key(v, first) >= from) {
      const int at = atomicAdd(&n_listed, 1);
      if (at < kListed) listed[at] = order_key(v, offset + first + e);
    }
  });
  __syncthreads();
  const int found = n_listed;
  if (found <= kListed) {
    put_listed(found);
    if (tid >= found && tid < top) put(tid, 0);
    return;
  }
  // more than the list holds: one after the other (there are more than `top`)
  u64 last = ~0ull;
  for (int k = 0; k < top; ++k) {
    u64 next = 0;
    elements([&](float v, int first, int e) {
      const u64 own = v > -INFINITY ? order_key(v, offset + first + e) : 0;
      if (own < last && own > next) next = own;
    });
    next = wave_max(next);
    __syncthreads();
    if (lane == 0) wave_keys[wave] = next;
    __syncthreads();
    next = wave_max(wave_keys[lane % WAVES]);
    last = next;
    if (tid == 0) put(k, last);
  }
}

// Few rows are cut so that their parts give every CU a workgroup, into pieces that a workgroup loads at once.  One
// workgroup takes 126464 logits at 16 a ns, a part of 8192 costs it 2 us, and the second launch 3 to 5 (us, bf16, uncut
// and cut: 1 x 126464 with 2 alternatives 12.5 8.2, with 32 14.4 12.9, 32 x 126464 with 8 14.8 11.3, 64 x 126464 in
// four parts 14.9 13.7, in three 85 x 126464 16.0 16.7; 1 x 32768 6.5 7.4).
int logprobs_parts(int rows, int vocab) {
  if (vocab < 65536) return 1;
  int n = 256 / rows < vocab / 8192 ? 256 / rows : vocab / 8192;
  if (n > kMostParts) n = kMostParts;
  return n < 4 ? 1 : n;
}

template <typename T>
hipError_t launch(const LogprobsArgs& a, hipStream_t s) {
  LogprobsDev<T> p;
  p.x = static_cast<const T*>(a.logits);
  p.ld = a.ld;
  p.vocab = a.vocab;
  p.top = a.top;
  p.scale = a.scale;
  p.tokens = a.tokens;
  p.logprobs = a.logprobs;
  p.entropy = a.entropy;
  p.top_ids = a.top_ids;
  p.top_logprobs = a.top_logprobs;
  p.parts = logprobs_parts(a.rows, a.vocab);
  if (p.parts > 1) {
    // (parts begin on 16-byte boundaries if the row does)
    p.part_len = ((a.vocab + p.parts - 1) / p.parts + 63) / 64 * 64;
    p.part_sums = reinterpret_cast<f32x4*>(a.workspace);
    p.part_keys = reinterpret_cast<unsigned long long*>(p.part_sums + (long)a.rows * p.parts);
    if (p.part_len < 16384)
      hipLaunchKernelGGL((logprobs_kernel<T, 256, Does::kPart>), dim3(a.rows * p.parts), dim3(256), 0, s, p);
    else
      hipLaunchKernelGGL((logprobs_kernel<T, 1024, Does::kPart>), dim3(a.rows * p.parts), dim3(1024), 0, s, p);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL((logprobs_kernel<T, 256, Does::kJoin>), dim3(a.rows), dim3(256), 0, s, p);
  } else if (a.vocab < 1024 || (a.vocab < 4096 && a.rows >= 1024)) {
    // a wave: what a row costs beside its elements is four times less than with four waves, its elements take longer
    // (us, it and four waves: 4096 x 300 8.1 13.4, 4096 x 1000 8.3 13.8, 4096 x 4000 15.3 19.9, 70000 x 33 61 167; 1 x
    // 1000 4.7 4.6, 1 x 4000 6.7 5.5, 300 x 4000 8.0 6.8)
    hipLaunchKernelGGL((logprobs_kernel<T, 64, Does::kRow>), dim3(a.rows), dim3(64), 0, s, p);
  } else if (a.vocab < 16384) {
    hipLaunchKernelGGL((logprobs_kernel<T, 256, Does::kRow>), dim3(a.rows), dim3(256), 0, s, p);
  } else {
    hipLaunchKernelGGL((logprobs_kernel<T, 1024, Does::kRow>), dim3(a.rows), dim3(1024), 0, s, p);
  }
  return hipGetLastError();
}

}  // namespace

size_t logprobs_workspace(int rows, int vocab, int top) {
  const int parts = rows > 0 ? logprobs_parts(rows, vocab) : 1;
  return parts > 1 ? (size_t)rows * parts * (sizeof(f32x4) + top * sizeof(u64)) : 0;
}

hipError_t launch_logprobs(int dtype, const LogprobsArgs& a, hipStream_t s) {
  if (a.rows == 0) return hipSuccess;
  return dtype == DARE_BF16 ? launch<bf16_t>(a, s) : launch<float>(a, s);
}

}  // namespace dare
