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

// tanh y for |y| < 0.8: y times a polynomial of degree 6 in its square, fitted at Chebyshev's points (off by 4e-9 of the value, 1e-7 as fp32 rounds it).
__device__ __forceinline__ float tanh_small(float y) {
  const float z = y * y;
  float p = 0.0015656708f;
  p = __builtin_fmaf(p, z, -0.0073702540f);
  p = __builtin_fmaf(p, z, 0.0212719534f);
  p = __builtin_fmaf(p, z, -0.0538406223f);
  p = __builtin_fmaf(p, z, 0.1333200783f);
  p = __builtin_fmaf(p, z, -0.3333328068f);
  p = __builtin_fmaf(p, z, 1.0f);
  return p * y;
}
// x: products, scale: what makes them scores over the cap -> tanh of those.  A wavefront whose scores are all below 0.8 of the cap, which most are,
// has the polynomial alone: 11 instructions a score instead of 20, three of them of a quarter of the rate.
template <int N>
__device__ __forceinline__ void tanh_all(float (&x)[N], float scale) {
  float most = 0.f;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    x[i] *= scale;
    most = fmaxf(most, fabsf(x[i]));
  }
  if (__all(most < 0.8f)) {
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = tanh_small(x[i]);
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      x[i] = capped(x[i], 1.f, 1.f);
      if (i % 4 == 3) __builtin_amdgcn_sched_barrier(0);       // (all of them side by side do not fit the registers)
    }
  }
}

}  // namespace rdkv
