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
};

hipError_t launch_fill(const FillArgs& a, int n_seqs, int bits, hipStream_t st);
hipError_t launch_append(const Args& a, int bits, int items, const uint16_t* k_new, const uint16_t* v_new, int32_t* slot, hipStream_t st);
hipError_t launch_read(const Args& a, int bits, int items, const int32_t* index, int n, uint16_t* K, uint16_t* V, hipStream_t st);
size_t decode_workspace_floats(int64_t items, int g, int capacity, int bits, bool weights);
hipError_t launch_decode(const Args& a, int bits, int items, const uint16_t* q, float* out, float* lse, float* workspace, hipStream_t st);

}  // namespace slots
}  // namespace rdkv
