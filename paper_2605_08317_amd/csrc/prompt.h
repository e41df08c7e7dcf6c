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
  int64_t token0[kSeqs];                // tokens of the batch before the sequence's first
};

// rows of a workgroup's, and its workgroups at most, of a launch
inline int64_t workgroups(int longest, int n_seqs, int hq) { return (static_cast<int64_t>(longest) + 127) / 128 * n_seqs * hq; }
hipError_t launch(const Args& a, int longest, hipStream_t st);

}  // namespace prompt
}  // namespace rdkv
