// A head's norm and rotation, as the lanes that hold it compute them. Shared by
// the kernels that rotate rows (rope.hip) and write them into the cache of 8-bit
// codes (kvq.hip).
//
//   norm      x <- x w / sqrt(mean(x^2) + eps)
//   rotation  of each pair (x, y) of channels: (x, y) <- m (x cos t - y sin t, y cos t + x sin t),
//             t = position * inv_freq[pair]
//
// D / 16 lanes hold a head, 16 channels each: two runs of 8 (kRun), so that a lane
// has both channels of each of its 8 pairs and nothing is exchanged. Lane c of a
// head has the pairs 8c .. 8c + 7 where these turn: half layout, channels 8c .. and
// rotary_dim / 2 + 8c ..; interleaved, channels 16c .. 16c + 15. Lanes past the
// pairs hold channels 16c .. 16c + 15, which only the norm changes.
#pragma once
#include "device_common.h"
#include "rows_kernels.h"

namespace spork {
namespace {

constexpr int kRun = 8;

// Where a lane's two runs begin in a head, and whether they turn.
struct Runs {
  int a, b;
  bool turns;
  __device__ __forceinline__ Runs(const TurnArgs& t, int c) {
    turns = 16 * c < t.rotary_dim;
    const bool half = turns && t.interleaved == 0;
    a = half ? 8 * c : 16 * c;
    b = half ? t.rotary_dim / 2 + 8 * c : 16 * c + 8;
  }
};

// Eight channels as they lie in memory.
template <typename T>
struct Raw;
template <>
struct Raw<__bf16> {
  uint4 w;
  __device__ __forceinline__ void load(const __bf16* p) { w = *reinterpret_cast<const uint4*>(p); }
  __device__ __forceinline__ float get(int i) const { return vec_f<__bf16>(w, i); }
  // Values that the compiler takes for new ones.
  __device__ __forceinline__ void anew() { asm volatile("" : "+v"(w.x), "+v"(w.y), "+v"(w.z), "+v"(w.w)); }
};
template <>
struct Raw<float> {
  uint4 w[2];
  __device__ __forceinline__ void load(const float* p) {
    w[0] = reinterpret_cast<const uint4*>(p)[0];
    w[1] = reinterpret_cast<const uint4*>(p)[1];
  }
  __device__ __forceinline__ float get(int i) const { return vec_f<float>(w[i >> 2], i & 3); }
  __device__ __forceinline__ void anew() {
#pragma unroll
    for (int i = 0; i < 2; ++i) asm volatile("" : "+v"(w[i].x), "+v"(w[i].y), "+v"(w[i].z), "+v"(w[i].w));
  }
};

__device__ __forceinline__ uint32_t bf16_pair(float a, float b) {
  typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
  return __builtin_bit_cast(uint32_t, bf16x2{static_cast<__bf16>(a), static_cast<__bf16>(b)});
}
// Eight channels, rounded to the output type once (to nearest: by at most half of its last place).
template <typename F>
__device__ __forceinline__ void store_run(__bf16* p, const F* x) {
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) w[i] = bf16_pair(static_cast<float>(x[2 * i]), static_cast<float>(x[2 * i + 1]));
  *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
}
template <typename F>
__device__ __forceinline__ void store_run(float* p, const F* x) {
#pragma unroll
  for (int i = 0; i < 2; ++i)
    reinterpret_cast<float4*>(p)[i] = make_float4(static_cast<float>(x[4 * i]), static_cast<float>(x[4 * i + 1]),
                                                  static_cast<float>(x[4 * i + 2]), static_cast<float>(x[4 * i + 3]));
}

// The value of the lane that differs in bit BY (1, 2 or 4) of its number: DPP moves.
template <int BY>
__device__ __forceinline__ float lane_xor(float x) {
  if constexpr (BY == 1) return dpp_mov<0xB1>(x);
  if constexpr (BY == 2) return dpp_mov<0x4E>(x);
  // (within four lanes all are equal by then: the mirror of eight does for a difference of 4)
  return dpp_mov<0x141>(x);
}
template <int BY>
__device__ __forceinline__ double lane_xor(double x) {
  const uint64_t u = __builtin_bit_cast(uint64_t, x);
  const float lo = lane_xor<BY>(__uint_as_float(static_cast<uint32_t>(u)));
  const float hi = lane_xor<BY>(__uint_as_float(static_cast<uint32_t>(u >> 32)));
  return __builtin_bit_cast(double, static_cast<uint64_t>(__float_as_uint(hi)) << 32 | __float_as_uint(lo));
}

// The sum over a head's lanes.
template <int D, typename F>
__device__ __forceinline__ F head_sum(F s) {
  s += lane_xor<1>(s);
  s += lane_xor<2>(s);
  if constexpr (D == 128) s += lane_xor<4>(s);
  return s;
}

// 1 / sqrt(mean(x^2) + eps) of a head, from the lane's sum of squares.
template <int D>
__device__ __forceinline__ double norm_factor(double s, double eps) {
  return 1.0 / sqrt(head_sum<D>(s) * (1.0 / D) + eps);
}

// The head's norm, in 32 bits: w holds the lane's weights. Where some of the squares may be
// lost (their sum is past 2^120, or so small that they and eps, which is at most 2^100,
// count), the head is scaled by a power of two first. A channel times the factor is at most
// sqrt(D), and then comes its weight: factor times weight may lie outside of 2^-126 .. 2^128
// where the result does not. (8,192 tokens take 31.1 us so, 35.4 in 64 bits for all heads,
// 34.5 with 64 bits there.)
template <int D>
__device__ __forceinline__ void norm_head(float (&x)[16], const float (&w)[16], double eps) {
  float s = 0;
#pragma unroll
  for (int i = 0; i < 16; ++i) s += x[i] * x[i];
  s = head_sum<D>(s);
  const float mean = s * (1.0f / D) + static_cast<float>(eps);
  float r = 1.0f / sqrtf(mean);
  const bool safe = mean >= 0x1p-87f && s <= 0x1p120f;
  if (__builtin_expect(__ballot(!safe) != 0, 0)) {
    float top = 0.0f;
#pragma unroll
    for (int i = 0; i < 16; ++i) top = fmaxf(top, fabsf(x[i]));
    top = fmaxf(top, lane_xor<1>(top));
    top = fmaxf(top, lane_xor<2>(top));
    if constexpr (D == 128) top = fmaxf(top, lane_xor<4>(top));
    const int e = safe || top == 0.0f ? 0 : static_cast<int>(__float_as_uint(top) >> 23) - 126;
    float t = 0;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      x[i] = ldexpf(x[i], -e);
      t += x[i] * x[i];
    }
    const double scaled = head_sum<D>(t) * (1.0 / D) + ldexp(eps, -2 * e);
    // (a head of zeros stays one under any eps but 0, however small)
    if (!safe) r = top == 0.0f && eps > 0.0 ? 1.0f : static_cast<float>(1.0 / sqrt(scaled));
  }
#pragma unroll
  for (int i = 0; i < 16; ++i) x[i] = x[i] * r * w[i];
}

// The lane's eight pairs, by their cosines and sines (the magnitude is in them).
template <typename F, typename F2>
__device__ __forceinline__ void turn_pairs(F (&x)[16], const F2 (&cs)[8], bool interleaved) {
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const F a = interleaved ? x[2 * j] : x[j], b = interleaved ? x[2 * j + 1] : x[8 + j];
    const F y = a * cs[j].x - b * cs[j].y, z = b * cs[j].x + a * cs[j].y;
    if (interleaved) {
      x[2 * j] = y;
      x[2 * j + 1] = z;
    } else {
      x[j] = y;
      x[8 + j] = z;
    }
  }
}

// A number of the series, in scalar registers: the compiler would keep all of them in
// vector registers over a loop.
__device__ __forceinline__ double scalar(double x) {
  asm volatile("" : "+s"(x));
  return x;
}

// Cosine and sine of a pair at a position, in 64 bits: at position 131,071 a
// rounded 32-bit angle is off by up to 0.004. Whole and quarter turns are taken off;
// what is left, at most pi / 4, goes into the series of both functions, whose next
// terms are below 2^-58.
__device__ __forceinline__ double2 pair_turn(const TurnArgs& t, int pair, int position) {
  constexpr double kTurns = 0.15915494309189533577;    // 1 / (2 pi)
  constexpr double kQuarter = 1.57079632679489661923;  // pi / 2
  double u = position * t.inv_freq[pair] * kTurns;
  u = 4.0 * (u - rint(u));
  const double whole = rint(u), r = (u - whole) * kQuarter, z = r * r;
  double s = scalar(1.0 / 355687428096000), c = scalar(1.0 / 20922789888000);  // 1 / 17!, 1 / 16!
  constexpr double kSin[] = {-1.0 / 1307674368000, 1.0 / 6227020800, -1.0 / 39916800, 1.0 / 362880, -1.0 / 5040, 1.0 / 120, -1.0 / 6};
  constexpr double kCos[] = {-1.0 / 87178291200, 1.0 / 479001600, -1.0 / 3628800, 1.0 / 40320, -1.0 / 720, 1.0 / 24, -1.0 / 2};
#pragma unroll
  for (int i = 0; i < 7; ++i) {
    s = __builtin_fma(s, z, scalar(kSin[i]));
    c = __builtin_fma(c, z, scalar(kCos[i]));
  }
  s = __builtin_fma(r * z, s, r);
  c = __builtin_fma(c, z, 1.0);
  const int q = static_cast<int>(whole) & 3;
  const double m = t.magnitude, x = (q & 1 ? s : c) * m, y = (q & 1 ? c : s) * m;
  return make_double2((q + 1) & 2 ? -x : x, q & 2 ? -y : y);
}

// The turns of a lane's eight pairs at a position, in 32 bits: each lane of the wave
// computes one pair, and they are exchanged through the wave's table in LDS (64
// entries). Lanes whose channels don't turn get anything.
__device__ __forceinline__ void lane_turns(const TurnArgs& t, int position, float2* table, int lane, int c, float2 (&cs)[8]) {
  if (2 * lane < t.rotary_dim) {
    const double2 x = pair_turn(t, lane, position);
    table[lane] = make_float2(static_cast<float>(x.x), static_cast<float>(x.y));
  }
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
#pragma unroll
  for (int j = 0; j < 8; ++j) cs[j] = table[8 * c + j];
}

}  // namespace
}  // namespace spork
