// What is done to scores, shared by the attention kernels that cap them.
#pragma once
#include <hip/hip_runtime.h>

namespace rdkv {

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr float kRoot = 0.08838834764831845f;      // 1 / sqrt(128)
constexpr float kRootLog2e = 0.12751743f;          // both: 0.0883883476 x 1.4426950409 = 0.12751743 (to 2^-25)

// cap * tanh(s / cap).  Below 0.8 the fifth convergent of Lambert's continued fraction y / (1 + y^2 / (3 + y^2 / (5 + ..))), off by
// less than 1e-8 of its value there; above, 1 - 2 / (e^2y + 1), which would lose the digits of small values.
__device__ __forceinline__ float capped(float s, float cap, float inv_cap) {
  const float y = s * inv_cap, y2 = y * y;
  const float num = __builtin_fmaf(y2, y2 + 105.f, 945.f), den = __builtin_fmaf(y2, __builtin_fmaf(y2, 15.f, 420.f), 945.f);
  const float small = y * num * __builtin_amdgcn_rcpf(den);
  const float large = 1.f - 2.f * __builtin_amdgcn_rcpf(__builtin_amdgcn_exp2f(fabsf(y) * (2.f * kLog2e)) + 1.f);
  return cap * (fabsf(y) < 0.8f ? small : __builtin_copysignf(large, y));
}

// tanh(x scale) for |x scale| < 0.5: x times a polynomial of degree 4 in its square, fitted at Chebyshev's points (off by 3e-8 of the value, 1.4e-7
// with fp32's roundings); the powers of the scale are in its coefficients.
struct TanhSmall {
  float c[5], below;                      // below: what |x| may be
  __device__ __forceinline__ explicit TanhSmall(float scale) {
    const float s2 = scale * scale, s4 = s2 * s2, s5 = s4 * scale;
    c[0] = scale;
    c[1] = -0.3333306909f * s2 * scale;
    c[2] = 0.1332475096f * s5;
    c[3] = -0.0529842377f * s2 * s5;
    c[4] = 0.0171313453f * s4 * s5;
    below = scale > 0x1p-12f && scale < 0x1p12f ? 0.5f / scale : 0.f;         // (so that no power leaves fp32's normal numbers)
  }
  __device__ __forceinline__ float operator()(float x) const {
    const float z = x * x;
    return x * __builtin_fmaf(__builtin_fmaf(__builtin_fmaf(__builtin_fmaf(c[4], z, c[3]), z, c[2]), z, c[1]), z, c[0]);
  }
};
// x: products, scale: what makes them scores over the cap -> tanh of those.  A wavefront whose scores are all below half of the cap, which most are,
// has the polynomial alone: 7 instructions a score instead of 20, three of them of a quarter of the rate.  (Products of 4-bit trees come over their query's
// unit: the scale is below what the coefficients keep, and the long form is taken.  8 tokens on 4 x 8 x 32768 slots 74 us, without a cap 56.)
template <int N>
__device__ __forceinline__ void tanh_all(float (&x)[N], float scale, const TanhSmall& small) {
  float most = 0.f;
#pragma unroll
  for (int i = 0; i < N; ++i) most = fmaxf(most, fabsf(x[i]));
  if (__all(most < small.below)) {
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = small(x[i]);
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      x[i] = capped(x[i] * scale, 1.f, 1.f);
      if (i % 4 == 3) __builtin_amdgcn_sched_barrier(0);       // (all of them side by side do not fit the registers)
    }
  }
}

}  // namespace rdkv
