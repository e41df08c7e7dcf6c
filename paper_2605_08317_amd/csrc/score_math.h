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

}  // namespace rdkv
