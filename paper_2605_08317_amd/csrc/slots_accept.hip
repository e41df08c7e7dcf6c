// Slot caches: accepted tokens of a drafted tree become part of the cache.
//
// Two launches.  The first gives every slot the attention weight that the tokens' heads gave it: scores as in slots_tree.hip (the same
// products in the same order), probabilities by the largest score and the sum that the tree's step left, summed over heads and tokens, a wavefront
// a tile of 64 slots; V is not read.  The second, a workgroup an item, takes the tokens in one after the other as that many appends would, but
// looks at all slots only once: a thread keeps the least of its own slots, and looks again when one of them was given away or a token has
// become old enough to go.
#include <algorithm>

#include "group_quant.h"
#include "slots_tiles.h"
#include "slots_tree.h"

namespace rdkv {
namespace slots {

namespace {

constexpr int kWaves = 4;

// tokens of a path: up to the first index that is none
__device__ __forceinline__ int path_length(const int32_t* path, int m, int n) {
  const int lane = threadIdx.x & 63;
  const int i = lane < m ? path[lane] : -1;
  const uint64_t bad = __ballot(i < 0 || i >= n);
  return bad == 0 ? 64 : __builtin_ctzll(bad);
}

// decay to the k-th
__device__ __forceinline__ float power(float x, int k) {
  float p = 1.f;
  for (float f = x; k > 0; k >>= 1, f *= f) p = k & 1 ? p * f : p;
  return p;
}

template <int BITS, bool GENERAL>
__global__ __launch_bounds__(64 * kWaves, BITS == 16 ? 1 : 2) void accept_weights_kernel(AcceptArgs a) {
  extern __shared__ __align__(16) uint8_t smem[];
  const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6), l32 = lane & 31, half = lane >> 5;
  const int item = blockIdx.x / a.pieces, piece = blockIdx.x % a.pieces, seq = item / a.s.hkv, kvh = item % a.s.hkv, g = a.s.g;
  const int32_t* path = a.path + static_cast<int64_t>(seq) * a.m;
  const int count = path_length(path, a.m, a.n), rows = count * g;
  if (count == 0) return;
  const int len = a.s.length(item), next = a.s.next[item], tiles = (len + kTileRows - 1) / kTileRows;
  const bool scored = GENERAL && (a.s.cap > 0.f || a.s.slopes);
  const float inv_cap = a.s.cap > 0.f ? 1.f / a.s.cap : 0.f, old = power(a.s.decay, count);
  const int32_t* pos = a.s.pos + static_cast<int64_t>(item) * a.s.capacity;
  float* weight = a.s.weight + static_cast<int64_t>(item) * a.s.capacity;
  const uint32_t lds0 = lds_address(smem);
  using Query = std::conditional_t<BITS == 16, Query16, Query4>;

  // of the tile's slots, scores' register i of product x is slot at(x, i)
  const auto slot_at = [&](int x, int i) __attribute__((always_inline)) {
    return BITS == 16 ? 32 * x + 8 * (i >> 2) + 4 * half + (i & 3) : 32 * half + 16 * x + i;
  };
  // what every query row gives a tile's slots, into sum
  const auto gather = [&](auto scores, int tile, float (&sum)[32]) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < 32; ++i) sum[i] = 0.f;
    for (int r0 = 0; r0 < rows; r0 += 32) {
      const int r = min(r0 + l32, rows - 1), j = r / g, token = path[j];
      const int64_t q_row = (static_cast<int64_t>(seq) * a.n + token) * a.s.hkv * g + kvh * g + r % g;
      Query q;
      q.load(a.q + q_row * kHeadDim);
      const float2 st = *reinterpret_cast<const float2*>(a.stats + 2 * q_row);
      const bool there = r0 + l32 < rows && st.y != 0.f;
      const float share = power(a.s.decay, count - 1 - j) / st.y, natural = q.unit * kRoot;
      floatx16 s[2];
      scores(q, s);
#pragma unroll
      for (int x = 0; x < 2; ++x)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          float e;
          if constexpr (GENERAL) {
            float v = s[x][i] * natural;
            const int p = pos[min(tile * kTileRows + slot_at(x, i), len - 1)], away = next + j - p;
            if (a.s.cap > 0.f) v = capped(v, a.s.cap, inv_cap);
            if (a.s.slopes) v = __builtin_fmaf(-a.s.slopes[kvh * g + r % g], static_cast<float>(away), v);
            e = scored ? v - st.x : __builtin_fmaf(s[x][i], natural, -st.x);
            if (a.s.window > 0 && away >= a.s.window && p >= a.s.sinks) e = -INFINITY;
          } else {
            e = __builtin_fmaf(s[x][i], natural, -st.x);
          }
          const float p = __builtin_amdgcn_exp2f(e * kLog2e) * share;
          sum[16 * x + i] += there ? p : 0.f;
        }
    }
  };
  const auto add = [&](int tile, float (&sum)[32]) __attribute__((always_inline)) {
    const float w = rows_sum(sum);
    const int slot = tile * kTileRows + slot_at(l32 >> 4, l32 & 15);
    if (slot < len) weight[slot] = __builtin_fmaf(old, weight[slot], w);
  };

  const int t0 = static_cast<int>(static_cast<int64_t>(tiles) * piece / a.pieces), t1 = static_cast<int>(static_cast<int64_t>(tiles) * (piece + 1) / a.pieces);
  if constexpr (BITS == 16) {
    // each wavefront has tiles of its own in LDS, two buffers
    constexpr int kTileLds = kTileRows * kRowBytes;
    const uint8_t* K = a.s.k + static_cast<int64_t>(item) * a.s.capacity * kRowBytes;
    const uint32_t k_at = 16 * (lane & 15);
    const auto fetch = [&](int tile, int buffer) __attribute__((always_inline)) {
      const int first = min(tile, t1 - 1) * kTileRows, last = len - 1 - first;
      const uint8_t* k = K + static_cast<int64_t>(first) * kRowBytes;
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const int row = 4 * i + (lane >> 4);
        copy_to_lds(k, min(row, last) * kRowBytes + (k_at ^ (16 * (row & 15))), lds0 + (2 * wave + buffer) * kTileLds + 1024 * i);
      }
    };
    int t = t0 + wave, buffer = 0;
    if (t >= t1) return;
    fetch(t, 0);
    for (; t < t1; t += kWaves, buffer ^= 1) {
      asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
      fetch(t + kWaves, buffer ^ 1);
      const uint8_t* kt = smem + (2 * wave + buffer) * kTileLds;
      float sum[32];
      gather([&](const Query& q, floatx16 (&s)[2]) __attribute__((always_inline)) {
        s[0] = scores16(kt, q);
        s[1] = scores16(kt + kStepKeys * kRowBytes, q);
      }, t, sum);
      add(t, sum);
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  } else {
    uint8_t* meta = smem + wave * kKMeta;
    const uint8_t* K = a.s.k + static_cast<int64_t>(item) * a.s.tiles * kTileBytes;
    for (int t = t0 + wave; t < t1; t += kWaves) {
      Side4 k;
      k.load(K + static_cast<int64_t>(t) * kTileBytes, true);
      put_k_meta(meta, k, len - t * kTileRows);
      wave_lds_order();
      float sum[32];
      gather([&](const Query& q, floatx16 (&s)[2]) __attribute__((always_inline)) { scores4(k, meta, q, s); }, t, sum);
      add(t, sum);
      wave_lds_order();
    }
  }
}

constexpr int kThreads = 1024;

template <int BITS>
__global__ __launch_bounds__(kThreads) void accept_append_kernel(AcceptArgs a) {
  __shared__ float s_weight[kMostDrafted];         // what a token begins with
  __shared__ int s_slot[kMostDrafted], s_path[kMostDrafted];
  __shared__ uint64_t s_key[2][kThreads / 64];
  __shared__ int s_at[2][kThreads / 64];
  const int item = blockIdx.x, seq = item / a.s.hkv, kvh = item % a.s.hkv, g = a.s.g, cap = a.s.capacity;
  const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6);
  const int count = path_length(a.path + static_cast<int64_t>(seq) * a.m, a.m, a.n);
  int32_t* out = a.slot ? a.slot + static_cast<int64_t>(item) * a.m : nullptr;
  if (out && tid < a.m && tid >= count) out[tid] = -1;
  if (count == 0) return;
  if (tid < count) {
    s_path[tid] = a.path[static_cast<int64_t>(seq) * a.m + tid];
    s_weight[tid] = 0.f;
  }
  const int len = a.s.length(item), next = a.s.next[item];
  __syncthreads();
  if (a.s.weight) {
    // token i has from each head of the tokens j >= i: sixteen lanes a product
    const int piece = tid & 15;
    for (int i = tid >> 4; i < count; i += kThreads / 16) {
      const uint16_t* k = a.k_draft + ((static_cast<int64_t>(seq) * a.n + s_path[i]) * a.s.hkv + kvh) * kHeadDim + 8 * piece;
      const bf16x8 kv = *reinterpret_cast<const bf16x8*>(k);
      float sum = 0.f;
      for (int j = i; j < count; ++j)
        for (int h = 0; h < g; ++h) {
          const int64_t q_row = (static_cast<int64_t>(seq) * a.n + s_path[j]) * a.s.hkv * g + kvh * g + h;
          const bf16x8 qv = *reinterpret_cast<const bf16x8*>(a.q + q_row * kHeadDim + 8 * piece);
          float x = 0.f;
#pragma unroll
          for (int c = 0; c < 8; ++c) x = __builtin_fmaf(static_cast<float>(kv[c]), static_cast<float>(qv[c]), x);
          x = row_sum(x);
          const float2 st = *reinterpret_cast<const float2*>(a.stats + 2 * q_row);
          const int away = j - i;
          float e = __builtin_fmaf(x, kRoot, -st.x);
          if (a.s.cap > 0.f || a.s.slopes) {
            x *= kRoot;
            if (a.s.cap > 0.f) x = capped(x, a.s.cap, 1.f / a.s.cap);
            if (a.s.slopes) x = __builtin_fmaf(-a.s.slopes[kvh * g + h], static_cast<float>(away), x);
            e = x - st.x;
          }
          const bool hidden = a.s.window > 0 && away >= a.s.window && next + i >= a.s.sinks;
          if (!hidden && st.y != 0.f) sum += __builtin_amdgcn_exp2f(e * kLog2e) * (power(a.s.decay, count - 1 - j) / st.y);
        }
      if (piece == 0) s_weight[i] = sum;
    }
    __syncthreads();
  }

  int32_t* pos = a.s.pos + static_cast<int64_t>(item) * cap;
  float* weight = a.s.weight ? a.s.weight + static_cast<int64_t>(item) * cap : nullptr;
  // this thread's slots: tid, tid + kThreads, ..
  uint64_t best = ~0ull;                           // least weight, then lowest position, of those that may go
  int at = 0, enters = INT32_MAX;                  // of the others the lowest position
  const auto look = [&](int newest) {
    constexpr int kEach = 8;
    best = ~0ull;
    at = 0;
    enters = INT32_MAX;
    for (int i0 = tid; i0 < cap; i0 += kEach * kThreads) {
      int p[kEach];
      float w[kEach];
#pragma unroll
      for (int k = 0; k < kEach; ++k) {
        const int i = min(i0 + k * kThreads, cap - 1);
        p[k] = pos[i];
        w[k] = weight ? weight[i] : 0.f;
      }
#pragma unroll
      for (int k = 0; k < kEach; ++k) {
        const int i = i0 + k * kThreads;
        if (i >= cap || p[k] < a.s.sinks) continue;
        const uint64_t key = static_cast<uint64_t>(weight_key(w[k])) << 32 | static_cast<uint32_t>(p[k]);
        if (p[k] > newest) enters = min(enters, p[k]);
        else if (key < best) best = key, at = i;
      }
    }
  };
  bool looked = false;
  for (int j = 0; j < count; ++j) {
    int slot = len + j;
    if (slot >= cap) {
      const int newest = next + j - a.s.recent;
      if (!looked || enters <= newest) look(newest);
      looked = true;
      uint64_t key = best;
      int where = at;
      const auto least = [&](uint64_t other, int other_at) __attribute__((always_inline)) {
        if (other < key || (other == key && other_at < where)) {
          key = other;
          where = other_at;
        }
      };
      for (int d = 1; d < 64; d <<= 1) {
        const uint64_t other = __shfl_xor(key, d);
        least(other, __shfl_xor(where, d));
      }
      if (lane == 0) {
        s_key[j & 1][wave] = key;
        s_at[j & 1][wave] = where;
      }
      __syncthreads();
      key = s_key[j & 1][lane & (kThreads / 64 - 1)];
      where = s_at[j & 1][lane & (kThreads / 64 - 1)];
      for (int d = 1; d < kThreads / 64; d <<= 1) {
        const uint64_t other = __shfl_xor(key, d);
        least(other, __shfl_xor(where, d));
      }
      slot = where;
    }
    if (slot % kThreads == tid) {                  // the thread that has the slot
      pos[slot] = next + j;
      if (weight) weight[slot] = s_weight[j];
      s_slot[j] = slot;
      if (out) out[j] = slot;
      if (looked) look(next + j - a.s.recent);
    }
  }
  __syncthreads();
  if (tid == 0) {
    a.s.len[item] = min(len + count, cap);
    a.s.next[item] = next + count;
  }
  // rows: half a wavefront a token, lanes 0..15 its K row, 16..31 its V row.  Of tokens in one slot the last stays
  for (int j = wave; j < count; j += kThreads / 64) {
    const int slot = s_slot[j];
    bool last = true;
    for (int k = j + 1; k < count; ++k) last = last && s_slot[k] != slot;
    if (lane >= 32 || !last) continue;
    const int c16 = lane & 15, grp = c16 >> 2, p = c16 & 3;
    const bool is_v = lane >= 16;
    const uint4 row = reinterpret_cast<const uint4*>(is_v ? a.v_draft : a.k_draft)[((static_cast<int64_t>(seq) * a.n + s_path[j]) * a.s.hkv + kvh) * 16 + c16];
    uint8_t* side = is_v ? a.s.v : a.s.k;
    if constexpr (BITS == 16) {
      reinterpret_cast<uint4*>(side)[(static_cast<int64_t>(item) * cap + slot) * 16 + c16] = row;
    } else {
      Quant q;
      uint32_t c[8];
      quantize_row<4, true>(row, 0, q, c);
      uint8_t* tile = side + (static_cast<int64_t>(item) * a.s.tiles + slot / kTileRows) * kTileBytes;
      const int r = slot % kTileRows;
      uint16_t* meta = reinterpret_cast<uint16_t*>(tile + kTileCodes);
      if (!is_v) store_k_words<4>(c, tile + k_words_at<4>(grp, p) + 16 * r, p);
      if (is_v) {
        // a word holds codes of eight rows, of which others may come as well: bits that are cleared and set, in any order
        const int k = r & 31, shift = 16 * (k & 1) + 4 * ((k >> 2) & 3);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const int ch = c16 * 8 + i, word = 4 * (ch >> 5) + 2 * (k >> 4) + ((k >> 1) & 1);
          uint32_t* to = reinterpret_cast<uint32_t*>(tile + 1024 * (word >> 2) + 16 * (32 * (r >> 5) + (ch & 31)) + 4 * (word & 3));
          atomicAnd(to, ~(15u << shift));
          atomicOr(to, (c[i] & 15u) << shift);
        }
      }
      if (p == 0) {
        const int m = is_v ? 32 * (r >> 2) + 8 * grp + (r & 3) : 8 * r + grp;
        meta[m] = __builtin_bit_cast(unsigned short, q.sh);
        meta[m + 4] = __builtin_bit_cast(unsigned short, q.mh);
      }
    }
  }
}

template <int BITS, bool GENERAL>
hipError_t start(const AcceptArgs& a, hipStream_t st) {
  constexpr int lds = BITS == 16 ? kWaves * 2 * kTileRows * kRowBytes : kWaves * kKMeta;
  const hipError_t e = RDKV_ALLOW_LDS((accept_weights_kernel<BITS, GENERAL>), lds);
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL((accept_weights_kernel<BITS, GENERAL>), dim3(a.items * a.pieces), dim3(64 * kWaves), lds, st, a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_accept(const AcceptArgs& args, int bits, hipStream_t st) {
  AcceptArgs a = args;
  if (a.s.weight) {
    const bool general = a.s.cap > 0.f || a.s.slopes || a.s.window > 0;
    const int tiles = (a.s.capacity + kTileRows - 1) / kTileRows;
    a.pieces = std::max(1, std::min((tiles + kWaves - 1) / kWaves, 1024 / a.items));
    const hipError_t e = bits == 16 ? (general ? start<16, true>(a, st) : start<16, false>(a, st)) : (general ? start<4, true>(a, st) : start<4, false>(a, st));
    if (e != hipSuccess) return e;
  }
  if (bits == 16) hipLaunchKernelGGL(accept_append_kernel<16>, dim3(a.items), dim3(kThreads), 0, st, a);
  else hipLaunchKernelGGL(accept_append_kernel<4>, dim3(a.items), dim3(kThreads), 0, st, a);
  return hipGetLastError();
}

}  // namespace slots
}  // namespace rdkv
