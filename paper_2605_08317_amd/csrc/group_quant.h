// The group quantizer and the words of quantized rows in 64-row tiles, for the kernels that store rows in 8, 4 or 2 bits.
// Needs a translation unit compiled with floating-point contraction off.
#pragma once
#include "wave_ops.h"

namespace rdkv {

namespace {

__device__ __forceinline__ float bf16_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t w) { return __uint_as_float(w & 0xFFFF0000u); }

// The quantizer of one group: scale, offset and codes.  The correctly rounded quotient d / s without the division
// sequence, by Markstein's scheme (IBM J. Res. Dev. 34, 1990): q0 = d * y with y the hardware reciprocal of s, remainder
// r = d - q0 s exact in one fused multiply-add, q = q0 + r y.  The reciprocal is within one unit in the last place, not
// correctly rounded as the theorem asks; tests/test_quotient.py finds the IEEE quotient all the same for every fp16 s and
// all three y, at 128 million numerators around the half-integers and of differences of bf16 numbers.  A group with a scale
// or offset that is not finite takes the division.
// The scale's division by the largest code Q goes the same way with the correctly rounded 1 / Q, which is the theorem's case.
struct Quant {
  float m, s, y;
  _Float16 sh, mh;
  bool finite;
  // Q: the largest code, inv_q: 1 / Q; EXACT: by division
  template <bool EXACT = false>
  __device__ __forceinline__ void set(float mn, float mx, float Q, float inv_q) {
    mn = mn + 0.0f;            // canonical +0
    const float range = mx - mn;
    float q;
    if constexpr (EXACT) {
      q = range / Q;
    } else {
      const float q0 = range * inv_q;
      q = __builtin_fmaf(__builtin_fmaf(-q0, Q, range), inv_q, q0);
      q = __builtin_copysignf(q, range);         // (-0 of a group of -0)
      asm("" : "+v"(q));       // rounded to fp32 before it is rounded to fp16 (else one instruction does both)
    }
    sh = static_cast<_Float16>(q);               // round to nearest even
    mh = static_cast<_Float16>(mn);
    s = static_cast<float>(sh);
    m = static_cast<float>(mh);
    finite = fabsf(s) < INFINITY && fabsf(m) < INFINITY;     // (false for NaN)
    y = s == 0.0f ? 0.0f : __builtin_amdgcn_rcpf(s);
  }
  // The code: the low 16 bits of what comes back (rounded to an integer by the addition of 1.5 x 2^23, whose low half is
  // zero; clamped before, which is the same as after).  EXACT: by division
  template <bool EXACT>
  __device__ __forceinline__ uint32_t code(float x, float Q) const {
    const float d = x - m;
    float q;
    if constexpr (EXACT) {
      q = d / s;
    } else {                   // (with a finite s = 0: y = 0, q = 0)
      const float q0 = d * y;
      q = __builtin_fmaf(__builtin_fmaf(-q0, s, d), y, q0);
    }
    const float t = fminf(fmaxf(q, 0.0f), Q);
    return __float_as_uint((EXACT && s == 0.0f ? 0.0f : t) + 12582912.0f);
  }
};
// two codes as the halves of a word; four as its bytes, one after the other
__device__ __forceinline__ uint32_t code_halves(uint32_t lo, uint32_t hi) { return __builtin_amdgcn_perm(hi, lo, 0x05040100u); }
template <int I>
__device__ __forceinline__ uint32_t code_byte(uint32_t word, uint32_t code) {      // code in byte I, zeros above it
  return __builtin_amdgcn_perm(code, word, I == 1 ? 0x0C0C0400u : I == 2 ? 0x0C040100u : 0x04020100u);
}

constexpr int kQuadXor1 = 0xB1, kQuadXor2 = 0x4E;

__device__ __forceinline__ void unpack8(const uint4& v, float (&x)[8]) {
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    x[2 * j] = bf16_lo(w[j]);
    x[2 * j + 1] = bf16_hi(w[j]);
  }
}

// Minimum and maximum over a quad of lanes, over rows of 16.  (A minimum that reads another lane is one instruction; out of
// fminf the compiler makes three, because it cannot tell that what comes from another lane is no signalling NaN.  Two wait
// states stand between a write to a register and its use by another lane.)
__device__ __forceinline__ void quad_range(float& mn, float& mx) {
  asm("s_nop 1\n\t"
      "v_min_f32_dpp %0, %0, %0 quad_perm:[1,0,3,2] row_mask:0xf bank_mask:0xf\n\t"
      "v_max_f32_dpp %1, %1, %1 quad_perm:[1,0,3,2] row_mask:0xf bank_mask:0xf\n\t"
      "s_nop 0\n\t"
      "v_min_f32_dpp %0, %0, %0 quad_perm:[2,3,0,1] row_mask:0xf bank_mask:0xf\n\t"
      "v_max_f32_dpp %1, %1, %1 quad_perm:[2,3,0,1] row_mask:0xf bank_mask:0xf"
      : "+v"(mn), "+v"(mx));
}
__device__ __forceinline__ void row_range(float& mn, float& mx) {      // after quad_range
  asm("s_nop 1\n\t"
      "v_min_f32_dpp %0, %0, %0 row_half_mirror row_mask:0xf bank_mask:0xf\n\t"
      "v_max_f32_dpp %1, %1, %1 row_half_mirror row_mask:0xf bank_mask:0xf\n\t"
      "s_nop 0\n\t"
      "v_min_f32_dpp %0, %0, %0 row_mirror row_mask:0xf bank_mask:0xf\n\t"
      "v_max_f32_dpp %1, %1, %1 row_mirror row_mask:0xf bank_mask:0xf"
      : "+v"(mn), "+v"(mx));
}

// Quantizes the 8 channels this lane holds of a token row (the 16 lanes of a row hold it in order, four lanes a group of
// 32 channels); codes as Quant::code gives them.
template <int BITS, bool EXACT>
__device__ __forceinline__ void quantize_row(const uint4& raw, int row_wide, Quant& g, uint32_t (&c)[8]) {
  constexpr float kMost = static_cast<float>((1 << BITS) - 1), kInvMost = 1.0f / kMost;
  float x[8];
  unpack8(raw, x);
  float mn = fminf(fminf(fminf(x[0], x[1]), fminf(x[2], x[3])), fminf(fminf(x[4], x[5]), fminf(x[6], x[7])));
  float mx = fmaxf(fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3])), fmaxf(fmaxf(x[4], x[5]), fmaxf(x[6], x[7])));
  quad_range(mn, mx);
  if (row_wide) row_range(mn, mx);
  g.set<EXACT>(mn, mx, kMost, kInvMost);
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    if constexpr (EXACT) __builtin_amdgcn_sched_barrier(0);      // (eight divisions side by side take 40 registers)
    c[j] = g.code<EXACT>(x[j], kMost);
  }
}

// Tiers 8/4/2: the layout the decode kernels' 4x4x4 MFMA steps want.  A wavefront lane owns a run of 4*BITS 32-bit words,
// word W of lane L stored at byte 1024*(W/4) + 16*L + 4*(W%4).  The run holds four groups of BITS words; a group is
// read in eight steps of four codes: with F = 16/BITS fields per 16-bit half, step s reads field s % F of both
// halves of the word pair s / F, i.e. code k of step s sits at word 2*(s/F) + k/2, bit 16*(k%2) + BITS*(s%F).
//   K: lane = token r; group = c / 32; c % 32 = 4*step + k        (a lane holds one token's row)
//   V: lane = 32*(r/32) + c % 32; group = c / 32; r % 32 = 4*step + k   (a lane holds one channel for 32 tokens)
// Metadata tile = 1024 bytes: K row-major per token [4 scales][4 offsets]; V per block of 4 tokens 4 groups x 16
// bytes: the group's scales of the 4 tokens, then its offsets.
// K words: this lane's two steps of its group; the lanes of a group OR their fields together.  dst: k_words_at of the row's
// tile, plus 16 bytes per row.
template <int BITS>
__device__ __forceinline__ int k_words_at(int grp, int p) {
  const int W = BITS * grp + (BITS == 8 ? 2 * p : BITS == 4 ? (p & 2) : 0);
  return 1024 * (W >> 2) + 4 * (W & 3);
}
template <int BITS>
__device__ __forceinline__ void store_k_words(const uint32_t (&c)[8], uint8_t* dst, int p) {
  const auto word = [&](int k) __attribute__((always_inline)) {     // codes k, k + 1 of steps 2 p and 2 p + 1
    return code_halves(c[k], c[k + 1]) | (code_halves(c[4 + k], c[5 + k]) << BITS);
  };
  uint2 w = make_uint2(word(0), word(2));
  if constexpr (BITS == 4) {               // fields 2 (p % 2), 2 (p % 2) + 1 of word pair p / 2
    const int sh = 8 * (p & 1);
    w.x <<= sh;
    w.y <<= sh;
    w.x |= dpp_u32<kQuadXor1>(w.x);
    w.y |= dpp_u32<kQuadXor1>(w.y);
  } else if constexpr (BITS == 2) {        // fields 2 p, 2 p + 1 of the group's only word pair
    const int sh = 4 * p;
    w.x <<= sh;
    w.y <<= sh;
    w.x |= dpp_u32<kQuadXor1>(w.x);
    w.y |= dpp_u32<kQuadXor1>(w.y);
    w.x |= dpp_u32<kQuadXor2>(w.x);
    w.y |= dpp_u32<kQuadXor2>(w.y);
  }
  if (BITS == 8 || (BITS == 4 && (p & 1) == 0) || (BITS == 2 && p == 0)) *reinterpret_cast<uint2*>(dst) = w;
}

// V codes go through LDS: s_vc[channel][token] bytes, 68 bytes per channel (four tokens of a channel are one word of a
// lane, and both the writes and the reads spread over the banks).
constexpr int kVcStride = 68;
template <int BITS>
__device__ __forceinline__ void store_v_words(const uint8_t* s_vc, uint8_t* tile) {
  constexpr int F = 16 / BITS;
  const int L = threadIdx.x & 63, G = threadIdx.x >> 6;    // lane of the layout, channel group
  const uint32_t* src = reinterpret_cast<const uint32_t*>(s_vc + (32 * G + (L & 31)) * kVcStride + 32 * (L >> 5));
  uint32_t w[BITS];
#pragma unroll
  for (int i = 0; i < BITS; ++i) w[i] = 0;
#pragma unroll
  for (int st = 0; st < 8; ++st) {         // the four tokens of a step: bytes 0, 1 -> halves of one word, 2, 3 -> the other
    const uint32_t d = src[st];
    w[2 * (st / F)] |= __builtin_amdgcn_perm(0u, d, 0x0C010C00u) << (BITS * (st % F));
    w[2 * (st / F) + 1] |= __builtin_amdgcn_perm(0u, d, 0x0C030C02u) << (BITS * (st % F));
  }
  if constexpr (BITS == 2) {
    *reinterpret_cast<uint2*>(tile + 1024 * (G >> 1) + 16 * L + 8 * (G & 1)) = make_uint2(w[0], w[1]);
  } else {
#pragma unroll
    for (int q = 0; q < BITS / 4; ++q)
      *reinterpret_cast<uint4*>(tile + 1024 * (G * (BITS / 4) + q) + 16 * L) =
          make_uint4(w[4 * q], w[4 * q + 1], w[4 * q + 2], w[4 * q + 3]);
  }
}

}  // namespace

}  // namespace rdkv
