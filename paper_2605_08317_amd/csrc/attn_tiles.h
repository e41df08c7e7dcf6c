// Attention of many query rows on the matrix cores: tiles of bf16 rows in LDS and their operands, shared by the attention of prompts
// (prompt_attn.hip) and that of drafted trees (slots_tree.hip).
//
// Products are v_mfma_f32_32x32x16, transposed: keys are its A side, query rows its B side.  Result register i of lane (half, l32) then
// holds key 8 (i / 4) + 4 half + i % 4 of the step for query row l32, so that a lane has one query row and, with the lane of the other
// half, all of its scores: a maximum over the keys is 16 lane-local ones and one exchange.  Probabilities are packed where they are: 8
// consecutive result registers are the keys of one step of P V as its B side has them (8 a half), and the A side takes V's rows in the
// same order, two groups of four keys a lane, by LDS reads that transpose (ds_read_b64_tr_b16: sixteen lanes read 4 rows of 16 channels, and
// each gets one channel of the 4).  Outputs come transposed too, a lane has its query row's channels 32 t + 8 (i / 4) + 4 half + i % 4, and a
// change of the row's reference scales them all by one number.
//
// LDS images are row-major, 256 bytes a row, 16-byte pieces exchanged so that what is read together lies in different banks: K rows at one
// column (piece ^ row % 16), V four rows by 32 bytes (piece ^ 4 (row % 4) ^ 2 (row / 4 % 2)).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "rdkv_internal.h"
#include "score_math.h"

namespace rdkv {
namespace attn {

typedef __attribute__((__vector_size__(8 * sizeof(__bf16)))) __bf16 bf16x8;
typedef __attribute__((__vector_size__(16 * sizeof(float)))) float floatx16;
typedef __attribute__((ext_vector_type(4))) short shortx4;

constexpr int kRowBytes = kHeadDim * 2;
constexpr int kStepKeys = 32;                        // keys of a step: the A side of a product

__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }
__device__ __forceinline__ uint32_t lds_address(const void* p) { return static_cast<uint32_t>(reinterpret_cast<uintptr_t>(p)); }

// 16 bytes per lane from global memory straight into LDS: lane i's bytes, base + offset, land at lds_base + 16 i (base and lds_base are
// uniform).  The compiler does not see the copy, so the reader waits for it by hand (tile_barrier).
__device__ __forceinline__ void copy_to_lds(const void* base, uint32_t offset, uint32_t lds_base) {
  asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1" ::"v"(offset), "s"(base), "s"(lds_base) : "memory", "m0");
}
// The same with 4 bytes per lane.
__device__ __forceinline__ void copy_word_to_lds(const void* base, uint32_t offset, uint32_t lds_base) {
  asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dword %0, %1" ::"v"(offset), "s"(base), "s"(lds_base) : "memory", "m0");
}
// What this wavefront has written to LDS is there for its other lanes, and stays until they have read it: the hardware keeps a wavefront's
// order, this the compiler's.
__device__ __forceinline__ void wave_lds_order() { asm volatile("" ::: "memory"); }
// Barrier of the workgroup after this wavefront's vector memory operations but the last PENDING have completed.
template <int PENDING>
__device__ __forceinline__ void tile_barrier() {
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(PENDING) : "memory");
}

// The number is computed here, not where it is needed (the compiler moves what has time to a later block).
__device__ __forceinline__ void here(float& v) { asm volatile("" : "+v"(v)); }
// Loads that the compiler knows of are waited for here and not at their first use, in a loop whose copies to LDS it does not know of: there it would
// wait for those too.
__device__ __forceinline__ void arrived(bf16x8& v) { asm volatile("" : "+v"(v)); }

__device__ __forceinline__ int k_piece(int row, int piece) { return piece ^ (row & 15); }
__device__ __forceinline__ int v_piece(int row, int piece) { return piece ^ (4 * (row & 3)) ^ (2 * ((row >> 2) & 1)); }

// Where a lane reads in an image at LDS address 0, whose pieces differ between products by exchanged bits alone: images begin at multiples of 256
// bytes, so that a product's address is the lane's, a few bits flipped, and a constant.
__device__ __forceinline__ uint32_t k_lane() {
  const int lane = threadIdx.x & 63, l32 = lane & 31, half = lane >> 5;
  return l32 * kRowBytes + 16 * k_piece(l32, half);
}
__device__ __forceinline__ uint32_t v_lane() {
  const int lane = threadIdx.x & 63, row = 4 * (lane >> 5) + ((lane & 15) >> 2);
  return row * kRowBytes + 16 * v_piece(row, 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1)) + 8 * (lane & 1);
}
template <class T>
__device__ __forceinline__ T from_lds(uint32_t at) {
  typedef const __attribute__((address_space(3))) T* Lds;
  return *(Lds)(uintptr_t)at;
}
// keys l32 of a step as the A side of product kb (channels 16 kb ..); at: the image's first row of the step, plus k_lane()
__device__ __forceinline__ bf16x8 read_k(uint32_t at, int kb, int step = 0) { return from_lds<bf16x8>((at ^ (32 * kb)) + step * (kStepKeys * kRowBytes)); }
// channel 32 t + l32 of the eight keys 16 s + 4 half + 0..3 and + 8..11 of a step, as the A side of P V; at: plus v_lane()
__device__ __forceinline__ bf16x8 read_v(uint32_t at, int t, int s, int step = 0) {
  typedef __attribute__((address_space(3))) shortx4* Lds;
  const uint32_t first = (at ^ (64 * t)) + (16 * s + kStepKeys * step) * kRowBytes;
  union { shortx4 s[2]; bf16x8 b; } v;
  v.s[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds)(uintptr_t)first);
  v.s[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds)(uintptr_t)(first + 8 * kRowBytes));
  return v.b;
}
// two numbers as bf16, nearest
__device__ __forceinline__ uint32_t pair_bf16(float a, float b) {
  typedef __attribute__((ext_vector_type(2))) __bf16 Pair;
  Pair v;
  v[0] = static_cast<__bf16>(a);
  v[1] = static_cast<__bf16>(b);
  return __builtin_bit_cast(uint32_t, v);
}
// eight numbers as bf16, nearest
__device__ __forceinline__ bf16x8 to_bf16(const float* p) {
  bf16x8 v;
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = static_cast<__bf16>(p[i]);
  return v;
}
__device__ __forceinline__ floatx16 product(bf16x8 a, bf16x8 b, floatx16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }

// of the lane's query row: both halves
__device__ __forceinline__ float halves_max(float v) {
  float o = v;
  asm("s_nop 1\n\tv_permlane32_swap_b32 %0, %1" : "+v"(v), "+v"(o));
  return fmaxf(v, o);
}
__device__ __forceinline__ float halves_add(float v) {
  float o = v;
  asm("s_nop 1\n\tv_permlane32_swap_b32 %0, %1" : "+v"(v), "+v"(o));
  return v + o;
}

// Of eight bf16 numbers: those that are finite, 0 for the others, and where +inf or NaN, and -inf or NaN, stand: 1 there.  (Rows that are
// hidden from some query rows of a product and not from others: their probability is 0 where they are hidden, and 0 x inf would be NaN.)
struct Parted {
  bf16x8 finite, up, down;
  bool any;
};
__device__ __forceinline__ Parted part(bf16x8 x) {
  union { bf16x8 b; uint32_t u[4]; } v, f, up, down;
  v.b = x;
  uint32_t any = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t t = ((v.u[i] & 0x7F807F80u) + 0x00800080u) & 0x80008000u;        // top bits of halves with all exponent bits
    const uint32_t odd = (t >> 15) * 0xFFFFu;
    const uint32_t nan = ((((v.u[i] & 0x007F007Fu) + 0x007F007Fu) & 0x00800080u) >> 7) * 0xFFFFu;
    const uint32_t neg = ((v.u[i] >> 15) & 0x00010001u) * 0xFFFFu;
    f.u[i] = v.u[i] & ~odd;
    up.u[i] = odd & (nan | ~neg) & 0x3F803F80u;
    down.u[i] = odd & (nan | neg) & 0x3F803F80u;
    any |= odd;
  }
  return {f.b, up.b, down.b, any != 0};
}

}  // namespace attn
}  // namespace rdkv
