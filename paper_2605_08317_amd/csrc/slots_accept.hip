// Slot caches: accepted tokens of a drafted tree become part of the cache.
//
// Two launches.  The first gives every slot the attention weight that the tokens' heads gave it, and the tokens themselves what they begin with:
// products as in slots_tree.hip, but with the query rows on their A side, so that a lane has one slot and sums over the rows are its own;
// probabilities by the largest score and the sum that the tree's step left.  V is not read.  Where a cache will be full it leaves the least of
// every 32 slots as well.  The second, a workgroup an item, takes the tokens in one after the other as that many appends would, from those
// leasts.
//   bound   the K side, once for every 64 rows (token, head) of a path: HBM.  The second launch: a chain of steps, a few for each token that takes another's slot
#include <algorithm>

#include "group_quant.h"
#include "slots_tiles.h"
#include "slots_tree.h"

namespace rdkv {
namespace slots {

namespace {

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

constexpr int kSegment = kLeastSlots;              // slots of a product

// The least of a segment's slots that may go by (weight, position), and the lowest position of those that may not yet.
struct __align__(16) Least {
  uint64_t key;
  int32_t at, enters;
};
static_assert(sizeof(Least) == kLeastBytes, "as the workspace's size has it");
__device__ __forceinline__ Least nothing() { return {~0ull, 0, INT32_MAX}; }
__device__ __forceinline__ void take(Least& l, uint64_t key, int at) {
  if (key < l.key || (key == l.key && at < l.at)) {
    l.key = key;
    l.at = at;
  }
}
// a slot: newest is the last position that may go
__device__ __forceinline__ void look_at(Least& l, int slot, int pos, float weight, int sinks, int newest) {
  if (pos < sinks) return;
  if (pos > newest) l.enters = min(l.enters, pos);
  else take(l, static_cast<uint64_t>(weight_key(weight)) << 32 | static_cast<uint32_t>(pos), slot);
}

// Rows of a pass over the slots: up to 64, in LDS as operands, with what probabilities are made with.
constexpr int kRows = 64;
struct __align__(16) RowTable {
  float less[kRows], share[kRows];                   // minus the largest score, and the bias at the cache's next position; decay over the sum
  float natural[kRows], slope[kRows];                // what makes products scores; the bias of a step further
  int at[kRows];                                     // position
};
constexpr int kQueryLds = kRows / 32 * 9 * 1024;     // [32 rows][operand][lane], the last operand 4-bit rows' sums
constexpr int kSlotLds = kSegment * kRowBytes + 512; // bf16: a segment's keys, weights, positions

template <int BITS, bool GENERAL, int WAVES>
__global__ __launch_bounds__(64 * WAVES, 2) void accept_weights_kernel(AcceptArgs a) {
  extern __shared__ __align__(256) uint8_t smem[];
  __shared__ RowTable s_row;
  const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6), l32 = lane & 31, half = lane >> 5;
  // the first workgroups have an item's own tokens, the others a piece of its slots
  const bool tokens = static_cast<int>(blockIdx.x) < a.items;
  const int unit = static_cast<int>(blockIdx.x) - a.items, item = tokens ? blockIdx.x : unit / a.pieces, piece = tokens ? 0 : unit % a.pieces;
  const int seq = item / a.s.hkv, kvh = item % a.s.hkv, g = a.s.g;
  const int32_t* path = a.path + static_cast<int64_t>(seq) * a.m;
  const int count = path_length(path, a.m, a.n), rows = count * g;
  if (count == 0) return;
  const int len = a.s.length(item), next = a.s.next[item], cap = a.s.capacity;
  const bool full = len + count > cap;
  const float inv_cap = a.s.cap > 0.f ? 1.f / a.s.cap : 0.f, old = power(a.s.decay, count);
  const int32_t* pos = a.s.pos + static_cast<int64_t>(item) * cap;
  float* weight = a.s.weight + static_cast<int64_t>(item) * cap;
  Least* leasts = reinterpret_cast<Least*>(a.leasts) + static_cast<int64_t>(item) * ((cap + kSegment - 1) / kSegment);
  uint8_t* mine = smem + kQueryLds + wave * (BITS == 16 ? 2 * kSlotLds : 0);
  using Query = std::conditional_t<BITS == 16, Query16, Query4>;

  // this wavefront's segments (4 bits: tiles of two): of its piece every WAVES-th
  constexpr int kUnit = BITS == 16 ? kSegment : kTileRows;
  const int units = (len + kUnit - 1) / kUnit;
  const int u0 = static_cast<int>(static_cast<int64_t>(units) * piece / a.pieces), u1 = static_cast<int>(static_cast<int64_t>(units) * (piece + 1) / a.pieces);

  // rows r0 .. of the path into LDS
  const auto rows_in = [&](auto kind, int r0) __attribute__((always_inline)) {
    using Q = decltype(kind);
    if (r0 > 0) __syncthreads();
    if (wave < kRows / 32) {
      const int r = min(r0 + 32 * wave + l32, rows - 1), j = r / g;
      const int64_t q_row = (static_cast<int64_t>(seq) * a.n + path[j]) * a.s.hkv * g + kvh * g + r % g;
      Q q;
      q.load(a.q + q_row * kHeadDim);
#pragma unroll
      for (int kb = 0; kb < 8; ++kb) *reinterpret_cast<decltype(&q.op[0])>(smem + ((wave * 9 + kb) * 64 + lane) * 16) = q.op[kb];
      if constexpr (std::is_same_v<Q, Query4>) *reinterpret_cast<halfx8*>(smem + ((wave * 9 + 8) * 64 + lane) * 16) = q.sums;
      const float2 st = *reinterpret_cast<const float2*>(a.stats + 2 * q_row);
      if (half == 0) {
        const int to = 32 * wave + l32;
        const bool there = r0 + to < rows && st.y != 0.f;
        const float slope = a.s.slopes ? a.s.slopes[kvh * g + r % g] : 0.f;
        s_row.less[to] = there ? -slope * static_cast<float>(j) - st.x : -INFINITY;        // (no row: probabilities of 0)
        s_row.share[to] = there ? power(a.s.decay, count - 1 - j) / st.y : 0.f;
        s_row.slope[to] = slope;
        s_row.at[to] = next + j;
        s_row.natural[to] = q.unit * kRoot;
      }
    }
    __syncthreads();
  };
  // What the rows in LDS give a lane's slot (TOKENS: one of the path's) at `place`; scores(block): their products.
  const auto given = [&](auto own, int r0, int place, auto scores) __attribute__((always_inline)) {
    const float back = GENERAL ? static_cast<float>(next - place) : 0.f;
    float sum = 0.f;
    for (int b = 0; b < kRows / 32 && r0 + 32 * b < rows; ++b) {
      const floatx16 s = scores(b);
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const int r = 32 * b + 8 * k + 4 * half;
        const float4 less = *reinterpret_cast<const float4*>(s_row.less + r), share = *reinterpret_cast<const float4*>(s_row.share + r);
        const float4 natural = *reinterpret_cast<const float4*>(s_row.natural + r);
        const float sh[4] = {share.x, share.y, share.z, share.w}, na[4] = {natural.x, natural.y, natural.z, natural.w};
        float e[4], le[4] = {less.x, less.y, less.z, less.w};
        if (GENERAL && a.s.slopes) {
          const float4 slope = *reinterpret_cast<const float4*>(s_row.slope + r);
          const float sl[4] = {slope.x, slope.y, slope.z, slope.w};
#pragma unroll
          for (int j = 0; j < 4; ++j) le[j] = __builtin_fmaf(-sl[j], back, le[j]);
        }
        if (GENERAL && a.s.cap > 0.f) {
#pragma unroll
          for (int j = 0; j < 4; ++j) e[j] = s[4 * k + j] * na[j];
          tanh_all(e, inv_cap, TanhSmall(inv_cap));
#pragma unroll
          for (int j = 0; j < 4; ++j) e[j] = __builtin_fmaf(e[j], a.s.cap, le[j]);
        } else {
#pragma unroll
          for (int j = 0; j < 4; ++j) e[j] = __builtin_fmaf(s[4 * k + j], na[j], le[j]);
        }
        if ((GENERAL && a.s.window > 0) || decltype(own)::value) {
          const int4 ats = *reinterpret_cast<const int4*>(s_row.at + r);
          const int away[4] = {ats.x - place, ats.y - place, ats.z - place, ats.w - place};
          if (GENERAL && a.s.window > 0) {
#pragma unroll
            for (int j = 0; j < 4; ++j)
              if (away[j] >= a.s.window && place >= a.s.sinks) e[j] = -INFINITY;
          }
          if constexpr (decltype(own)::value) {
#pragma unroll
            for (int j = 0; j < 4; ++j)
              if (away[j] < 0) e[j] = -INFINITY;
          }
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) sum = __builtin_fmaf(__builtin_amdgcn_exp2f(e[j] * kLog2e), sh[j], sum);
        if constexpr (GENERAL) __builtin_amdgcn_sched_barrier(0);        // (sixteen side by side do not fit the registers)
      }
    }
    return halves_add(sum);
  };
  const auto operand16 = [&](int b, int k) __attribute__((always_inline)) { return *reinterpret_cast<const bf16x8*>(smem + ((b * 9 + k) * 64 + lane) * 16); };
  const auto operand4 = [&](int b, int k) __attribute__((always_inline)) { return *reinterpret_cast<const halfx8*>(smem + ((b * 9 + k) * 64 + lane) * 16); };
  const auto products16 = [&](uint32_t keys, int b) __attribute__((always_inline)) {
    floatx16 s = {};
#pragma unroll
    for (int kb = 0; kb < 8; ++kb) s = product(operand16(b, kb), read_k(keys + k_lane(), kb), s);
    return s;
  };

  if (tokens) {
    // the path's keys behind the rows: wavefronts 0 and 1 have 32 tokens each
    const int token = 32 * wave + l32;
    uint8_t* keys = smem + kQueryLds + wave * (kSegment * kRowBytes);
    if (wave < 2) {
      const uint32_t to = lds_address(keys);
      const uint8_t* k = reinterpret_cast<const uint8_t*>(a.k_draft) + (static_cast<int64_t>(seq) * a.n * a.s.hkv + kvh) * kRowBytes;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int row = 4 * i + (lane >> 4);
        copy_to_lds(k, path[min(32 * wave + row, count - 1)] * a.s.hkv * kRowBytes + 16 * k_piece(row, lane & 15), to + 1024 * i);
      }
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    }
    float sum = 0.f;
    for (int r0 = 0; r0 < rows; r0 += kRows) {
      rows_in(Query16{}, r0);
      if (wave < 2) sum += given(std::true_type{}, r0, next + token, [&](int b) __attribute__((always_inline)) { return products16(lds_address(keys), b); });
    }
    if (wave < 2 && half == 0 && token < count) a.begins[static_cast<int64_t>(item) * kMostDrafted + token] = sum;
    return;
  }

  // a lane's slot gets its weight; the least of the lanes' slots whose numbers differ in the bits of `lanes`
  const auto put = [&](int slot, float before, int place, float sum, float keep, bool last_pass, auto lanes) __attribute__((always_inline)) {
    const float w = __builtin_fmaf(keep, before, sum);
    if (slot < len && half == 0) weight[slot] = w;
    Least l = nothing();
    if (full && last_pass) {
      if (slot < len) look_at(l, slot, place, w, a.s.sinks, next - a.s.recent);
#pragma unroll
      for (int d = 1; d < 32; d <<= 1) {
        if (!(decltype(lanes)::value & d)) continue;
        const uint64_t key = __shfl_xor(l.key, d);
        const int at = __shfl_xor(l.at, d);
        take(l, key, at);
        l.enters = min(l.enters, __shfl_xor(l.enters, d));
      }
    }
    return l;
  };

  for (int r0 = 0; r0 < rows; r0 += kRows) {
    const bool last_pass = r0 + kRows >= rows;
    const float keep = r0 == 0 ? old : 1.f;
    int u = u0 + wave;                               // (the first segment is on its way with the rows)
    if constexpr (BITS == 16) {
      const uint8_t* K = a.s.k + static_cast<int64_t>(item) * cap * kRowBytes;
      const uint32_t lds0 = lds_address(mine);
      const auto fetch = [&](int unit, int buffer) __attribute__((always_inline)) {
        const int first = min(unit, u1 - 1) * kSegment, last = len - 1 - first;
        const uint8_t* k = K + static_cast<int64_t>(first) * kRowBytes;
        const uint32_t to = lds0 + buffer * kSlotLds;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const int row = 4 * i + (lane >> 4);
          copy_to_lds(k, min(row, last) * kRowBytes + 16 * k_piece(row, lane & 15), to + 1024 * i);
        }
        copy_word_to_lds(weight + first, 4 * min(l32, last), to + kSegment * kRowBytes);
        copy_word_to_lds(pos + first, 4 * min(l32, last), to + kSegment * kRowBytes + 256);
      };
      int buffer = 0;
      if (u < u1) fetch(u, 0);
      rows_in(Query{}, r0);
      if (u < u1) {
        for (; u < u1; u += WAVES, buffer ^= 1) {
          fetch(u + WAVES, buffer ^ 1);
          asm volatile("s_waitcnt vmcnt(10)" ::: "memory");
          const uint8_t* keys = mine + buffer * kSlotLds;
          const float before = reinterpret_cast<const float*>(keys + kSegment * kRowBytes)[l32];
          const int place = reinterpret_cast<const int*>(keys + kSegment * kRowBytes + 256)[l32], slot = u * kSegment + l32;
          const float sum = given(std::false_type{}, r0, place, [&](int b) __attribute__((always_inline)) { return products16(lds0 + buffer * kSlotLds, b); });
          const Least l = put(slot, before, place, sum, keep, last_pass, std::integral_constant<int, 31>{});
          if (full && last_pass && lane == 0) leasts[u] = l;
          asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        }
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
      }
    } else {
      const uint8_t* K = a.s.k + static_cast<int64_t>(item) * a.s.tiles * kTileBytes;
      Side4 k;
      const Codes4 codes;
      uint4 meta[2];                               // of the lane's slots
      float before[2];
      int place[2];
      const auto load = [&](int tile) __attribute__((always_inline)) {
        const uint8_t* t = K + static_cast<int64_t>(tile) * kTileBytes;
        k.load(t, true);
#pragma unroll
        for (int x = 0; x < 2; ++x) {
          const int slot = min(tile * kTileRows + slot_of_row(x, l32), len - 1);
          meta[x] = *reinterpret_cast<const uint4*>(t + kTileCodes + 16 * (slot & (kTileRows - 1)));
          before[x] = weight[slot];
          place[x] = pos[slot];
        }
      };
      if (u < u1) load(u);
      rows_in(Query{}, r0);
      for (; u < u1; u += WAVES) {
        const Words4 words(k);
        union { uint4 u; halfx4 h[2]; } m[2];
        float w[2];
        int at[2];
#pragma unroll
        for (int x = 0; x < 2; ++x) {
          m[x].u = meta[x];
          w[x] = before[x];
          at[x] = place[x];
        }
        if (u + WAVES < u1) load(u + WAVES);
        Least l = nothing();
#pragma unroll
        for (int x = 0; x < 2; ++x) {
          const float sum = given(std::false_type{}, r0, at[x], [&](int b) __attribute__((always_inline)) {
            floatx16 s = product(operand4(b, 8), centres(m[x].u), floatx16{});
#pragma unroll
            for (int c = 0; c < 4; ++c) {
              floatx16 sums = product(operand4(b, 2 * c), words.operand(codes, x, c, 0), floatx16{});
              sums = product(operand4(b, 2 * c + 1), words.operand(codes, x, c, 1), sums);
#pragma unroll
              for (int i = 0; i < 16; ++i) s[i] = __builtin_fmaf(static_cast<float>(m[x].h[0][c]), sums[i], s[i]);
            }
            return s;
          });
          // (bit 2 of a product's row is which segment its slot is in)
          const Least some = put(u * kTileRows + slot_of_row(x, l32), w[x], at[x], sum, keep, last_pass, std::integral_constant<int, 27>{});
          take(l, some.key, some.at);
          l.enters = min(l.enters, some.enters);
        }
        const int segment = 2 * u + (lane >> 2);
        if (full && last_pass && (lane == 0 || lane == 4) && segment * kSegment < len) leasts[segment] = l;
      }
    }
  }
}

// The least of the wavefront's by (key, at), and a lane that has it.
struct First {
  uint64_t key;
  int at, lane;
};
template <int CTRL, int ROWS>
__device__ __forceinline__ uint32_t lower(uint32_t v) {
  return min(v, static_cast<uint32_t>(__builtin_amdgcn_update_dpp(-1, static_cast<int>(v), CTRL, ROWS, 0xf, false)));
}
__device__ __forceinline__ uint32_t wave_min(uint32_t v) {
  v = lower<0x118, 0xf>(lower<0x114, 0xf>(lower<0x112, 0xf>(lower<0x111, 0xf>(v))));           // rows of 16
  return __builtin_amdgcn_readlane(lower<0x143, 0xc>(lower<0x142, 0xa>(v)), 63);
}
__device__ __forceinline__ First first_of_wave(uint64_t key, int at) {
  const uint32_t high = wave_min(static_cast<uint32_t>(key >> 32)), low = wave_min(static_cast<uint32_t>(key >> 32) == high ? static_cast<uint32_t>(key) : ~0u);
  First f;
  f.key = static_cast<uint64_t>(high) << 32 | low;
  uint64_t have = __ballot(key == f.key);
  if (have & (have - 1)) {
    const uint32_t lowest = wave_min(key == f.key ? static_cast<uint32_t>(at) : ~0u);
    have = __ballot(key == f.key && static_cast<uint32_t>(at) == lowest);
  }
  f.lane = __builtin_ctzll(have);
  f.at = __builtin_amdgcn_readlane(at, f.lane);
  return f;
}

constexpr int kThreads = 1024, kWaves = kThreads / 64;

// Lists of the wavefronts, each in order, and the walk over all of them: wavefront w's list is lane w's.
struct Lists {
  uint64_t key[kWaves][kMostDrafted];
  int at[kWaves][kMostDrafted];
};
struct Walk {
  const Lists& lists;
  uint64_t key = ~0ull;
  int at = 0, next = 0;
  __device__ __forceinline__ explicit Walk(const Lists& l) : lists(l) { step(); }
  __device__ __forceinline__ void step() {
    const int lane = threadIdx.x & 63;
    key = lane < kWaves && next < kMostDrafted ? lists.key[lane][next] : ~0ull;
    if (key != ~0ull) at = lists.at[lane][next];
    ++next;
  }
};

// The second launch.  Which slots go follows from three kinds of tokens: slots that could go at once, cached tokens that become old enough on the
// way, and accepted ones that do; of the first kind only the least `want` matter, one for each token that takes another's slot.  They are in the
// `want` segments whose leasts are least, so those are found first, then the slots in them; both times each wavefront makes a list of its own least
// ones and a walk over the sixteen lists gives the order.  The tokens' turns then are a walk in which a lane adds the token of the other two kinds
// that it has, and nothing is read from memory.
//   measured   4 tokens in 1000 slots 9.6 us, 8 in each of 256 items' 8192 slots of 4 bits 23 us; a turn that looked at the slots and leasts again in
//              memory took 2 us more (18 and 39)
template <int BITS>
__global__ __launch_bounds__(kThreads) void accept_append_kernel(AcceptArgs a) {
  __shared__ int s_slot[kMostDrafted], s_late[kMostDrafted], s_enters[kMostDrafted], s_n;
  __shared__ Lists s_segments, s_slots;
  const int item = blockIdx.x, seq = item / a.s.hkv, kvh = item % a.s.hkv, cap = a.s.capacity;
  const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6);
  const int32_t* path = a.path + static_cast<int64_t>(seq) * a.m;
  const int len = a.s.length(item), next = a.s.next[item];
  const int count = path_length(path, a.m, a.n);
  int32_t* out = a.slot ? a.slot + static_cast<int64_t>(item) * a.m : nullptr;
  if (out && tid < a.m && tid >= count) out[tid] = -1;
  if (count == 0) return;
  const int first = max(cap - len, 0), want = count - first;           // the first token that takes another's slot, and how many do

  // rows: half a wavefront a token, lanes 0..15 its K row, 16..31 its V row
  const int c16 = lane & 15;
  const bool is_v = lane >= 16;
  const auto row_of = [&](int j) {
    return reinterpret_cast<const uint4*>(is_v ? a.v_draft : a.k_draft)[((static_cast<int64_t>(seq) * a.n + path[min(j, count - 1)]) * a.s.hkv + kvh) * 16 + c16];
  };
  const uint4 first_row = row_of(wave);

  int32_t* pos = a.s.pos + static_cast<int64_t>(item) * cap;
  float* weight = a.s.weight ? a.s.weight + static_cast<int64_t>(item) * cap : nullptr;
  const float* begins = weight ? a.begins + static_cast<int64_t>(item) * kMostDrafted : nullptr;
  const int segments = (cap + kSegment - 1) / kSegment, used = (len + kSegment - 1) / kSegment;
  Least* leasts = reinterpret_cast<Least*>(a.leasts) + static_cast<int64_t>(item) * segments;
  const int newest = next - a.s.recent;            // the last position that may go for the first token
  const auto key_of = [](float w, int p) { return static_cast<uint64_t>(weight_key(w)) << 32 | static_cast<uint32_t>(p); };
  if (want > 0) {
    if (tid < kMostDrafted) s_late[tid] = INT32_MAX;
    if (tid == 0) s_n = 0;
    s_segments.key[wave][lane] = s_slots.key[wave][lane] = ~0ull;
    __syncthreads();
    // the leasts of the lane's segments, and which segments have somebody who becomes old enough
    Least l = nothing();
    for (int e = tid; e < used; e += kThreads) {
      Least of;
      if (weight) {
        of = leasts[e];
      } else {                                     // (no launch has looked: the oldest go)
        int p[kSegment];
#pragma unroll
        for (int i = 0; i < kSegment; ++i) p[i] = pos[min(e * kSegment + i, len - 1)];
        of = nothing();
#pragma unroll
        for (int i = 0; i < kSegment; ++i)
          if (e * kSegment + i < len) look_at(of, e * kSegment + i, p[i], 0.f, a.s.sinks, newest);
        leasts[e] = of;
      }
      take(l, of.key, of.at);
      if (of.enters < newest + count) {
        const int n = atomicAdd(&s_n, 1);
        if (n < kMostDrafted) s_enters[n] = e;     // (as many positions, and so no more segments)
      }
    }
    for (int i = 0; i < want; ++i) {
      const First f = first_of_wave(l.key, l.at);
      if (f.key == ~0ull) break;
      if (lane == 0) {
        s_segments.key[wave][i] = f.key;
        s_segments.at[wave][i] = f.at;
      }
      if (lane == f.lane) {
        l = nothing();
        for (int e = tid; e < used && used > kThreads; e += kThreads) {
          const Least of = leasts[e];
          if (of.key > f.key || (of.key == f.key && of.at > f.at)) take(l, of.key, of.at);
        }
      }
    }
    __syncthreads();
    int segment = -1;                              // lane i: the i-th
    Walk order(s_segments);
    for (int i = 0; i < want; ++i) {
      const First f = first_of_wave(order.key, order.at);
      if (f.key == ~0ull) break;
      if (lane == i) segment = f.at / kSegment;
      if (lane == f.lane) order.step();
    }
    // half of the wavefront a segment, twice; segments that become old enough likewise
    uint64_t key[2];
    int at[2];
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const int which = 2 * wave + (lane >> 5) + 2 * kWaves * k, e = __shfl(segment, which), slot = e * kSegment + (lane & 31);
      key[k] = ~0ull;
      at[k] = slot;
      if (e >= 0 && slot < len) {
        const int p = pos[slot];
        const float w = weight ? weight[slot] : 0.f;
        if (p >= a.s.sinks && p <= newest) key[k] = key_of(w, p);
      }
      if (which < s_n) {
        const int i = s_enters[which] * kSegment + (lane & 31), p = i < len ? pos[i] : -1, after = p - newest - 1;
        if (p >= a.s.sinks && after >= 0 && after < count) atomicMin(&s_late[after], i);
      }
    }
    for (int i = 0; i < want; ++i) {
      const bool second = key[1] < key[0] || (key[1] == key[0] && at[1] < at[0]);
      const First f = first_of_wave(second ? key[1] : key[0], second ? at[1] : at[0]);
      if (f.key == ~0ull) break;
      if (lane == 0) {
        s_slots.key[wave][i] = f.key;
        s_slots.at[wave][i] = f.at;
      }
      if (lane == f.lane) (second ? key[1] : key[0]) = ~0ull;
    }
  }
  __syncthreads();
  if (wave == 0) {
    int slot = len + lane;                         // of accepted token `lane`
    if (want > 0) {
      const int late_at = s_late[lane];
      const uint64_t begin = key_of(lane < count && weight ? begins[lane] : 0.f, next + lane);
      uint64_t late = ~0ull, mine = ~0ull;         // of the lane's token that becomes old enough, and of its accepted one
      if (late_at != INT32_MAX) late = key_of(weight ? weight[late_at] : 0.f, newest + 1 + lane);
      const int age = max(a.s.recent, 1);
      Walk order(s_slots);
      for (int j = first; j < count; ++j) {
        if (lane <= j - age && (j == first || lane == j - age) && next + lane >= a.s.sinks) mine = begin;
        uint64_t key = order.key;
        int at = key == ~0ull ? 0 : order.at, kind = 0;
        const auto look = [&](uint64_t k, int t, int kd) {
          if (k < key || (k == key && k != ~0ull && t < at)) key = k, at = t, kind = kd;
        };
        if (lane < j) look(late, late_at, 1);
        look(mine, slot, 2);
        const First f = first_of_wave(key, at);
        if (lane == j) slot = f.at;                // (nobody may go: slot 0)
        if (lane == f.lane) {
          if (kind == 0) order.step();
          if (kind == 1) late = ~0ull;
          if (kind == 2) mine = ~0ull;
        }
      }
    }
    if (lane < count) {
      s_slot[lane] = slot;
      if (out) out[lane] = slot;
    }
    // positions and weights: of tokens in one slot the last one's
    bool last = lane < count;
    for (int t = 1; t < count; ++t) last = last && !(t > lane && __builtin_amdgcn_readlane(slot, t) == slot);
    if (last) {
      pos[slot] = next + lane;
      if (weight) weight[slot] = begins[lane];
    }
    if (lane == 0) {
      a.s.len[item] = min(len + count, cap);
      a.s.next[item] = next + count;
    }
  }
  __syncthreads();
  // of tokens in one slot the last stays
  for (int j = wave; j < count; j += kWaves) {
    const int slot = s_slot[j];
    bool last = true;
    for (int k = j + 1; k < count; ++k) last = last && s_slot[k] != slot;
    if (lane >= 32 || !last) continue;
    const int grp = c16 >> 2, p = c16 & 3;
    const uint4 row = j == wave ? first_row : row_of(j);
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
hipError_t start(AcceptArgs& a, hipStream_t st) {
  // in bf16 eight wavefronts fill a compute unit's LDS
  constexpr int kWaves = BITS == 16 ? 8 : 4, kUnit = BITS == 16 ? kSegment : kTileRows;
  constexpr int lds = kQueryLds + (BITS == 16 ? kWaves * 2 * kSlotLds : 2 * kSegment * kRowBytes);
  const auto kernel = accept_weights_kernel<BITS, GENERAL, kWaves>;
  const hipError_t e = RDKV_ALLOW_LDS(kernel, lds);
  if (e != hipSuccess) return e;
  const int units = (a.s.capacity + kUnit - 1) / kUnit;
  a.pieces = std::max(1, std::min((units + kWaves - 1) / kWaves, (BITS == 16 ? 512 : 1024) / a.items));
  hipLaunchKernelGGL(kernel, dim3(a.items * (a.pieces + 1)), dim3(64 * kWaves), lds, st, a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_accept(const AcceptArgs& args, int bits, hipStream_t st) {
  AcceptArgs a = args;
  if (a.s.weight) {
    const bool general = a.s.cap > 0.f || a.s.slopes || a.s.window > 0;
    const hipError_t e = bits == 16 ? (general ? start<16, true>(a, st) : start<16, false>(a, st)) : (general ? start<4, true>(a, st) : start<4, false>(a, st));
    if (e != hipSuccess) return e;
  }
  if (bits == 16) hipLaunchKernelGGL(accept_append_kernel<16>, dim3(a.items), dim3(kThreads), 0, st, a);
  else hipLaunchKernelGGL(accept_append_kernel<4>, dim3(a.items), dim3(kThreads), 0, st, a);
  return hipGetLastError();
}

}  // namespace slots
}  // namespace rdkv
