// Slot caches, many query rows at once: what the attention of drafted trees and the taking of accepted tokens share.  Scores of 64 slots (a
// tile) and 32 query rows on the matrix cores, in the transposed form of attn_tiles.h.
//
// 4-bit rows need no LDS image: a tile's layout is an operand's already.  K codes: a product takes 16 channels of 32 slots, a lane 8
// of one slot, which are 2 fields of 2 words; the words of a slot's other 16 channels go to the other half of the wavefront (permlane32).  The
// slots of a product are chosen so that a lane's scores are of 16 slots in a row: result register i of lane (half, .) of product x is slot
// 32 half + 16 x + i.  V codes: a lane's word quadruple is one channel's 32 slots of its half, so step f of P V (fields f of the four words)
// takes slots 4 f + 0..3 and 16 + 4 f + 0..3 of the half, which are registers 4 f .. 4 f + 3 of the lane's two products.
//   scores  codes less 8 are fp16 numbers and meet the query's values in fp16 (their 8 bits, over a power of two of the row's: values down to
//           2^-23 of the row's largest keep them all), so that products are exact; a group's sums of products are added with the slots' scales
//           in fp32.  What is left of a value, its offset plus 8 scales, in two fp16 terms, is a product of its own with sums of the query's
//           values over a group, also two.  (With the codes themselves that product and the other sums are large and nearly cancel: 131072
//           slots, largest scores and sums 2.6e-6 of their norm off from fp32 sums over the values)
//   P V     V codes less 8 are scaled to fp16 values by one fused multiply-add (rounded once, 2^-12 of the value; a group's offset plus 8
//           scales, which it starts from, too), probabilities are fp16
#pragma once
#include "attn_tiles.h"
#include "slots.h"

namespace rdkv {
namespace slots {

using namespace attn;

typedef __attribute__((ext_vector_type(8))) _Float16 halfx8;
typedef __attribute__((ext_vector_type(4))) _Float16 halfx4;
typedef __attribute__((ext_vector_type(2))) _Float16 halfx2;

constexpr float kNoScore = -2e38f;       // a finite maximum of nothing, also times log2(e): no score is below it

__device__ __forceinline__ floatx16 product(halfx8 a, halfx8 b, floatx16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0); }
using attn::product;

// Query rows of a wavefront as operands.
struct Query16 {
  bf16x8 op[8];
  static constexpr float kUnits = 1.f;
  float unit;                            // scores come over it
  // q: the lane's row
  __device__ __forceinline__ void load(const uint16_t* q) {
    const int half = (threadIdx.x & 63) >> 5;
#pragma unroll
    for (int kb = 0; kb < 8; ++kb) op[kb] = *reinterpret_cast<const bf16x8*>(q + 16 * kb + 8 * half);
#pragma unroll
    for (int kb = 0; kb < 8; ++kb) arrived(op[kb]);
    unit = 1.f;
  }
};
struct Query4 {
  halfx8 op[8];                          // product 2 group + s: channels 32 group + 16 half + 8 s ..
  halfx8 sums;                           // of the groups' values, twice four: high terms in the lower half's lanes, low ones in the upper's
  float unit;
  __device__ __forceinline__ void load(const uint16_t* q) {
    const int half = (threadIdx.x & 63) >> 5;
    bf16x8 in[8];
    float most = 0.f;
#pragma unroll
    for (int kb = 0; kb < 8; ++kb) {
      in[kb] = *reinterpret_cast<const bf16x8*>(q + 32 * (kb >> 1) + 16 * half + 8 * (kb & 1));
#pragma unroll
      for (int i = 0; i < 8; ++i) most = fmaxf(most, fabsf(static_cast<float>(in[kb][i])));
    }
    most = halves_max(most);
    // The largest value over the unit is in [2^9, 2^10), a group's sum below 2^15; below 2^-111 less, where the unit and one over it, of which the drafted
    // tokens' products take the second, would leave fp32's normal numbers (values down to 2^-126 are 2^-6 there and keep their bits).
    const uint32_t e = min(max(__float_as_uint(most) >> 23, 16u), 254u);
    const float inv = __uint_as_float((263u - e) << 23);              // 2^(136 - e)
    unit = __uint_as_float((e - 9u) << 23);
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      float sum = 0.f;
#pragma unroll
      for (int s = 0; s < 2; ++s)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float x = static_cast<float>(in[2 * g + s][i]) * inv;
          op[2 * g + s][i] = static_cast<_Float16>(x);
          sum += x;
        }
      sum = halves_add(sum);
      const _Float16 hi = static_cast<_Float16>(sum);
      sums[g] = sums[4 + g] = half == 0 ? hi : static_cast<_Float16>(sum - static_cast<float>(hi));
    }
  }
};

// bf16 rows in LDS: products of 32 slots, register i of lane (half, .): slot 8 (i / 4) + 4 half + i % 4 of the step.
// at: LDS address of the image, plus k_lane()
__device__ __forceinline__ floatx16 scores16(uint32_t at, int step, const Query16& q) {
  floatx16 s = {};
#pragma unroll
  for (int kb = 0; kb < 8; ++kb) s = product(read_k(at, kb, step), q.op[kb], s);
  return s;
}

// slot of a 4-bit tile that row r of product x is
__device__ __forceinline__ int slot_of_row(int x, int r) { return 32 * ((r >> 2) & 1) + 16 * x + 4 * (r >> 3) + (r & 3); }

// A 4-bit tile's codes and metadata of one side on their way to a wavefront.  K: the lane's 16 codes of each group are of slot slot_of_row(half, l32);
// metadata of slot `lane`.  V: the codes of channel 32 group + l32 of the half's slots; metadata of slots 4 (lane / 4) .. + 3, group lane % 4.
struct Side4 {
  uint4 codes[4];
  uint4 meta;
  __device__ __forceinline__ void load(const uint8_t* tile, bool is_k) {
    const int lane = threadIdx.x & 63;
    const int at = is_k ? slot_of_row(lane >> 5, lane & 31) : lane;
#pragma unroll
    for (int g = 0; g < 4; ++g) codes[g] = *reinterpret_cast<const uint4*>(tile + 1024 * g + 16 * at);
    meta = *reinterpret_cast<const uint4*>(tile + kTileCodes + 16 * lane);
  }
};

// Of a slot's four scales and offsets: the offsets plus 8 scales, in two terms.
__device__ __forceinline__ halfx8 centres(uint4 meta) {
  union { uint4 u; _Float16 h[8]; } m;
  m.u = meta;
  halfx8 c;
#pragma unroll
  for (int g = 0; g < 4; ++g) {
    const float o = __builtin_fmaf(8.f, static_cast<float>(m.h[g]), static_cast<float>(m.h[4 + g]));
    c[g] = static_cast<_Float16>(o);
    c[4 + g] = static_cast<_Float16>(o - static_cast<float>(c[g]));
  }
  return c;
}
// K metadata into LDS (kKMeta bytes of the wavefront's), of slots from `rows` on zeros: a slot's centres, then the scales, [group][slot].
constexpr int kKMeta = 1024 + 512;
__device__ __forceinline__ void put_k_meta(uint8_t* lds, const uint4& meta, int rows) {
  const int lane = threadIdx.x & 63;
  const bool there = lane < rows;
  const uint4 m = make_uint4(there ? meta.x : 0u, there ? meta.y : 0u, there ? meta.z : 0u, there ? meta.w : 0u);
  *reinterpret_cast<halfx8*>(lds + 16 * lane) = centres(m);
  uint16_t* scales = reinterpret_cast<uint16_t*>(lds + 1024) + lane;
  scales[0] = static_cast<uint16_t>(m.x);
  scales[64] = static_cast<uint16_t>(m.x >> 16);
  scales[128] = static_cast<uint16_t>(m.y);
  scales[192] = static_cast<uint16_t>(m.y >> 16);
}
// V metadata: scales, and offsets plus 8 scales; of slots from `rows` on zeros.  FINITE: of those that are not finite as well; the lanes that had such.
template <bool FINITE>
__device__ __forceinline__ uint64_t put_v_meta(uint8_t* lds, const uint4& meta, int rows) {
  const int lane = threadIdx.x & 63, first = 4 * (lane >> 2);
  union { uint4 u; _Float16 h[8]; } m;
  m.u = meta;
  bool odd = false;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const bool there = first + i < rows;
    const float s = there ? static_cast<float>(m.h[i]) : 0.f, o = there ? static_cast<float>(m.h[4 + i]) : 0.f;
    const _Float16 centre = static_cast<_Float16>(__builtin_fmaf(8.f, s, o));
    const bool fine = !FINITE || (fabsf(s) < INFINITY && fabsf(static_cast<float>(centre)) < INFINITY);
    odd = odd || !fine;
    m.h[i] = static_cast<_Float16>(fine ? s : 0.f);
    m.h[4 + i] = fine ? centre : static_cast<_Float16>(0.f);
  }
  *reinterpret_cast<uint4*>(lds + 16 * lane) = m.u;
  return FINITE ? __ballot(odd) : 0;
}

// What codes become numbers with.  Masks in scalar registers and what is or-ed to them in vector registers, of which an instruction takes one and one: the
// two operations are one instruction then (of constants, which it knows, the compiler makes two).
struct Codes4 {
  uint32_t low, high, v1024, v64;
  __device__ __forceinline__ Codes4() {
    asm("s_mov_b32 %0, 0x000F000F" : "=s"(low));
    asm("s_mov_b32 %0, 0x00F000F0" : "=s"(high));
    asm("v_mov_b32 %0, 0x64006400" : "=v"(v1024));
    asm("v_mov_b32 %0, 0x54005400" : "=v"(v64));
  }
  // Fields f (0 .. 3) of a word's halves, codes, less 8 as fp16: 1024 + code, or 64 + code where the field is four bits up, less 1032 or 72.
  __device__ __forceinline__ halfx2 less_8(uint32_t word, int f) const {
    const uint32_t v = f < 2 ? word : word >> 8;
    return f & 1 ? __builtin_bit_cast(halfx2, (v & high) | v64) - halfx2{72, 72} : __builtin_bit_cast(halfx2, (v & low) | v1024) - halfx2{1032, 1032};
  }
};

// A lane's words of product x, and of them what a product's operand of a group's half is: fields 2 s and 2 s + 1 of two words.
struct Group4 {
  uint32_t w[2][2];
  Group4() = default;
  // word pair (2 half, 2 half + 1) of the slots of product 0, and of product 1
  __device__ __forceinline__ explicit Group4(const uint4& k) {
    uint32_t a = k.x, b = k.y, c = k.z, d = k.w;
    asm("s_nop 1\n\tv_permlane32_swap_b32 %0, %1" : "+v"(a), "+v"(c));
    asm("s_nop 1\n\tv_permlane32_swap_b32 %0, %1" : "+v"(b), "+v"(d));
    w[0][0] = a;
    w[0][1] = b;
    w[1][0] = c;
    w[1][1] = d;
  }
  __device__ __forceinline__ halfx8 operand(const Codes4& codes, int x, int s) const {
    union { halfx2 p[4]; halfx8 h; } op;
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      op.p[j] = codes.less_8(w[x][j], 2 * s);
      op.p[2 + j] = codes.less_8(w[x][j], 2 * s + 1);
    }
    return op.h;
  }
};
struct Words4 {
  Group4 group[4];
  __device__ __forceinline__ explicit Words4(const Side4& k) {
#pragma unroll
    for (int g = 0; g < 4; ++g) group[g] = Group4(k.codes[g]);
  }
  __device__ __forceinline__ halfx8 operand(const Codes4& codes, int x, int g, int s) const { return group[g].operand(codes, x, s); }
};

// Products of the 64 slots, register i of s[x] of lane (half, .): slot 32 half + 16 x + i; over the query's unit.  operand(x, group, half of the group)
template <class Operand>
__device__ __forceinline__ void scores4(const uint8_t* k_meta, const Query4& q, floatx16 (&s)[2], Operand operand) {
  const int lane = threadIdx.x & 63, l32 = lane & 31, half = lane >> 5;
  // (a group's products before the one before's sums are scaled; the scheduler left alone would have all operands first, and spill them)
  floatx16 sums[2];
  const auto multiply = [&](int n) __attribute__((always_inline)) {
    floatx16 p = product(operand(n >> 2, n & 3, 0), q.op[2 * (n & 3)], floatx16{});
    sums[n & 1] = product(operand(n >> 2, n & 3, 1), q.op[2 * (n & 3) + 1], p);
  };
  multiply(0);
#pragma unroll
  for (int x = 0; x < 2; ++x) {
    s[x] = product(*reinterpret_cast<const halfx8*>(k_meta + 16 * slot_of_row(x, l32)), q.sums, floatx16{});
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      if (4 * x + g < 7) multiply(4 * x + g + 1);
      const halfx8* sc = reinterpret_cast<const halfx8*>(k_meta + 1024 + 128 * g + 2 * (32 * half + 16 * x));
      const halfx8 sc0 = sc[0], sc1 = sc[1];
#pragma unroll
      for (int i = 0; i < 16; ++i)
        s[x][i] = __builtin_fmaf(static_cast<float>(i < 8 ? sc0[i & 7] : sc1[i & 7]), sums[g & 1][i], s[x][i]);
      __builtin_amdgcn_sched_barrier(0);
    }
  }
}

// fp16 values of channel 32 group + l32 of slots 32 half + 4 f + 0..3 and + 16..19
template <int F>
__device__ __forceinline__ halfx8 values4(const Codes4& codes, const uint4& words, const uint8_t* v_meta, int group) {
  const int half = (threadIdx.x & 63) >> 5;
  const uint32_t w[4] = {words.x, words.y, words.z, words.w};
  union { halfx2 h[4]; halfx8 v; } x;
#pragma unroll
  for (int p = 0; p < 2; ++p) {
    union { uint4 u; halfx2 h[4]; } m;
    m.u = *reinterpret_cast<const uint4*>(v_meta + 64 * (8 * half + 4 * p + F) + 16 * group);
#pragma unroll
    for (int j = 0; j < 2; ++j) x.h[2 * p + j] = __builtin_elementwise_fma(codes.less_8(w[2 * p + j], F), m.h[j], m.h[2 + j]);
  }
  return x.v;
}

__device__ __forceinline__ halfx8 to_half(const float* p) {
  halfx8 v;
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = static_cast<_Float16>(p[i]);
  return v;
}

}  // namespace slots
}  // namespace rdkv
