// Trees of drafted tokens over slot caches (rdkv_slots_tree_attn, rdkv_slots_accept): what the host side and the kernels share.
#pragma once
#include <algorithm>
#include <cmath>

#include "slots.h"

namespace rdkv {
namespace slots {

constexpr int kMostDrafted = 64;        // tokens of a tree: a bit each

struct TreeArgs {
  Args s;
  const uint16_t* q;                    // [batch][n][hq][128]
  const uint16_t* k_draft;              // [batch][n][hkv][128]
  const uint16_t* v_draft;
  const int32_t* parent;                // [batch][n]
  const int32_t* counts;                // [batch], or null
  uint16_t* out;                        // [batch][n][hq][128]
  float* stats;                         // [batch][n][hq][2], or null
  float* part_acc;                      // [item][row group][piece][rows of a group][128]
  float* part_ml;                       // the same rows: [4]
  int32_t items, n;
  int32_t wide, row_groups, slot_pieces, pieces;        // plan_tree, as the workspace's size has it
};

// wide: wavefronts of a workgroup that share out rows, 32 each; the others share out slots.  Pieces of an item's slots, and all of them: with one
// for the drafted tokens where the card has room for it, else these go with the last.
struct TreePlan {
  int32_t wide, row_groups, slot_pieces, pieces;
  size_t part_rows(int64_t items) const { return pieces == 1 ? 0 : static_cast<size_t>(items) * row_groups * pieces * 32 * wide; }
  size_t floats(int64_t items) const { return part_rows(items) * (kHeadDim + 4); }
};
inline TreePlan plan_tree(int64_t items, int rows, int capacity, int bits) {
  TreePlan p;
  p.wide = rows <= 32 ? 1 : rows <= 64 ? 2 : rows <= 128 || bits == 4 ? 4 : 8;
  p.row_groups = (rows + 32 * p.wide - 1) / (32 * p.wide);
  const int64_t groups = items * p.row_groups;
  const int64_t tiles = (static_cast<int64_t>(capacity) + kTileRows - 1) / kTileRows;
  const int64_t stage = bits == 16 ? (p.wide == 8 ? 1 : 2) : 4 / p.wide;            // tiles that a workgroup has at once: no piece is smaller
  // As many workgroups as run at once: one a compute unit in bf16, two in 4 bits.  (Twice as many in 4 bits, for items of different lengths: 32 tokens of 4 heads on
  // 32 x 8 x 5/8 C .. C slots 5 % slower at C = 4096 to 7168, the same at 8192 and 12288, 3 % faster at 16384, 4 % at 32768; of equal lengths 1 to 11 %
  // slower at all of them, 8 tokens at 8192 11 %.)
  const int64_t card = bits == 16 ? 256 : 512;
  // Nor more than 4 roots of the stages: a piece costs the join what a sixteenth of a stage costs (one item of 131072 slots, 256 pieces -> 128 or 90: bf16
  // 29.0 -> 24.2 us, 4 bits 32.2 -> 27.1; with 2.4 roots 27.1 and 34.3).
  const int64_t most = std::min(tiles / stage, static_cast<int64_t>(4.0 * std::sqrt(static_cast<double>(tiles / stage))));
  p.slot_pieces = static_cast<int32_t>(std::max<int64_t>(1, std::min(most, card / std::max<int64_t>(groups, 1))));
  p.pieces = p.slot_pieces > 1 && groups * (p.slot_pieces + 1) <= card ? p.slot_pieces + 1 : p.slot_pieces;
  return p;
}

// (largest score, sum of exponentials of what is left) of a row: m, l its reference and sum over it times 2^shift, top the largest product; factor
// makes products exponents of 2, natural scores.  The sum is over the score as it is rounded.
__device__ __forceinline__ void store_stats(float* to, float m, float l, float top, float factor, float natural, float shift) {
  constexpr float kLog2e_ = 1.4426950408889634f;
  const float score = top * natural;
  const float sum = l * __builtin_amdgcn_exp2f(__builtin_fmaf(m - top, factor, __builtin_fmaf(top, natural, -score) * kLog2e_) - shift);
  const bool none = l == 0.f;
  *reinterpret_cast<float2*>(to) = make_float2(none ? -INFINITY : l != l ? l : score, none ? 0.f : sum);
}

struct AcceptArgs {
  Args s;
  const uint16_t* q;                    // as of the tree: [batch][n]..
  const uint16_t* k_draft;
  const uint16_t* v_draft;
  const int32_t* path;                  // [batch][m]
  const float* stats;                   // [batch][n][hq][2]
  int32_t* slot;                        // [batch][hkv][m], or null
  void* leasts;                         // [items][segments of kLeastSlots slots]: kLeastBytes each
  float* begins;                        // [items][kMostDrafted]: what a token's weight begins with
  int32_t items, n, m, pieces;
};
constexpr int kLeastSlots = 32, kLeastBytes = 16;
inline size_t accept_workspace_bytes(int64_t items, int capacity) {
  return static_cast<size_t>(items) * ((static_cast<size_t>(capacity) + kLeastSlots - 1) / kLeastSlots * kLeastBytes + kMostDrafted * sizeof(float));
}

hipError_t launch_accept(const AcceptArgs& a, int bits, hipStream_t st);
hipError_t launch_tree(const TreeArgs& a, int bits, hipStream_t st);

}  // namespace slots
}  // namespace rdkv
