// Slot caches (rdkv_slots_*): what the host side and the kernels share.
#pragma once
#include "rdkv_internal.h"

namespace rdkv {
namespace slots {

constexpr int kTileRows = kTile64;                                     // 4-bit rows: slots of a tile
constexpr int kTileCodes = kTileRows * kHeadDim / 2;                   // its bytes of codes,
constexpr int kTileBytes = kTileCodes + kTileRows * kGroupsPerRow * 4; // and with the scales and offsets behind them

// the struct of the C ABI with typed pointers
struct Args {
  uint8_t* k;
  uint8_t* v;
  int32_t* pos;
  float* weight;
  int32_t* len;
  int32_t* next;
  const float* slopes;
  int32_t hkv, g, capacity, tiles;      // tiles: of an item, 4 bits
  int32_t sinks, recent, window;
  float cap, decay;
  __device__ __forceinline__ int length(int64_t item) const { return min(max(len[item], 0), capacity); }
};

// An order of weights as unsigned numbers, NaN lowest and -0 as +0.
__device__ __forceinline__ uint32_t weight_key(float w) {
  const uint32_t u = __float_as_uint(w + 0.0f);
  return w != w ? 0u : (u & 0x80000000u) ? ~u : u | 0x80000000u;
}

// Sequences of a fill: as many as go with a launch.
constexpr int kFillSeqs = 64;
struct FillArgs {
  Args s;
  const uint16_t* K;
  const uint16_t* V;
  const float* w_tok;
  int32_t seq0;                         // sequence of the cache that the first entry fills
  int32_t T[kFillSeqs];
  int64_t row0[kFillSeqs];              // first row of the sequence's block
  // selection from long prompts, by several workgroups an item (plan_select); tables of the launch's items
  uint16_t* counts;                     // [item][parts][2048]: weights of a part by their first digit
  uint32_t* open;                       // [rows of the launch's sequences]: weights at the border digit, in the order of tokens
  int2* part;                           // [item][parts]: weights above the border digit, and at it in the parts before
  int4* found;                          // [item]: border digit, how many stay at it, how many there are
  int32_t parts, part_rows;             // parts of an item, tokens of a part; 0: a workgroup an item
};
constexpr int kSelectDigits = 2048;

// The parts of prompts of up to `longest` tokens: at least 4096 tokens each, 64 parts where that is not more than a count of 16 bits holds.
// Shorter prompts are one workgroup's.
struct SelectPlan { int32_t parts, part_rows; };
inline SelectPlan plan_select(int64_t longest) {
  constexpr int64_t kOne = 8 * 1024, kLeast = 4096, kMost = 32768;
  if (longest <= kOne) return {0, 0};
  int64_t rows = ((longest + 63) / 64 + kLeast - 1) / kLeast * kLeast;
  rows = rows < kMost ? rows : kMost;
  return {static_cast<int32_t>((longest + rows - 1) / rows), static_cast<int32_t>(rows)};
}

// longest: of the launch's prompts
hipError_t launch_fill(const FillArgs& a, int n_seqs, int longest, int bits, hipStream_t st);
hipError_t launch_append(const Args& a, int bits, int items, const uint16_t* k_new, const uint16_t* v_new, int32_t* slot, hipStream_t st);
hipError_t launch_read(const Args& a, int bits, int items, const int32_t* index, int n, uint16_t* K, uint16_t* V, hipStream_t st);
size_t decode_workspace_floats(int64_t items, int g, int capacity, int bits, bool weights);
hipError_t launch_decode(const Args& a, int bits, int items, const uint16_t* q, float* out, float* lse, float* workspace, hipStream_t st);

}  // namespace slots
}  // namespace rdkv
