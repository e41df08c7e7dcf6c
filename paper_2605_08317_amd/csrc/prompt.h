// Attention of whole prompts (rdkv_prompt_attn_bf16): what the host side and the kernel share.
#pragma once
#include "rdkv_internal.h"

namespace rdkv {
namespace prompt {

constexpr int kKeys = 64;               // of a tile
constexpr int kSeqs = 64;               // of a launch: they go with its arguments

// where the rows of heads are: element (sequence s, head h, token t, c) at tokens ? (token0[s] + t) row + 128 h : 128 (token0[s] heads + h T[s] + t), + c
struct Side {
  int32_t row;                          // elements from a token's row to the next's: 128 in ragged blocks
  int32_t tokens;
};

struct Args {
  const uint16_t* Q;
  const uint16_t* K;
  const uint16_t* V;
  uint16_t* out;
  float* lse;                           // ragged [hq][T_s], or null
  const float* slopes;                  // [hq], or null
  Side q, k, v, o;
  int32_t hq, hkv, n_seqs;
  int32_t window, sinks;
  float cap;
  int32_t T[kSeqs];
  int32_t first[kSeqs];                 // its first workgroup
  int64_t token0[kSeqs];                // tokens of the batch before the sequence's first
};

constexpr int kRows = 128;              // of a workgroup, or half as many, whose keys two wavefronts share out
// a sequence's workgroups: of an XCD as many as of another, so that the same heads of all sequences are on the same one
inline int64_t workgroups(int T, int hq, int rows = kRows) { return ((static_cast<int64_t>(T) + rows - 1) / rows * hq + 7) / 8 * 8; }
hipError_t launch(const Args& a, int grid, bool shared, hipStream_t st);

}  // namespace prompt
}  // namespace rdkv
