// Slot caches: attention of a tree of drafted tokens.
//
// A token sees the slots, its ancestors and itself: what the steps of a chain would compute, with what the slots cost once for all tokens.  A workgroup
// of four or eight wavefronts has up to 128 (bf16: 256) query rows (token, head) of an item and a piece of its slots.  Its wavefronts share out
// the rows, 32 each, and where these are fewer than the wavefronts the slots as well; results of slots are joined in LDS, those of pieces
// by a second launch.  The last piece of an item has the drafted tokens' own keys and values, bf16 rows whatever the cache holds, behind its slots or
// to itself.  Products and probabilities as of prompts (a lane has one query row); of 4-bit tiles a wavefront's own, codes less 8 as fp16 with
// group sums in fp32, so that scores keep fp32's digits.
//   bound   bf16: HBM up to 64 rows (8 tokens of 4 heads on 4 x 8 x 131072 slots 390 us, 5.5 TB/s), from 128 on the matrix cores, 54 % busy, at the clock that
//           the power leaves them, and waits, 29 % (64 tokens 600 us in a long row of calls, 920 TFLOP/s; the first few 540, those behind them up to 900).
//           4 bits: vector instructions, 63 % of the cycles issue one, about 640 a tile and 32 rows (8 tokens on 4 x 8 x 90001..131072 slots 147 us); above
//           64 rows four wavefronts share what takes the codes apart, 47 %, and wait for each other, 35 % (32 tokens on 32 x 8 x 5000..8192 slots with
//           biases 250 us)
//   tried   query operands in LDS and tiles loaded a tile ahead twice over in 4 bits: slower, they cost the registers of a second wavefront a SIMD
#include <algorithm>

#include "slots_tiles.h"
#include "slots_tree.h"

namespace rdkv {
namespace slots {

namespace {

constexpr float kSlack = 4.f;             // what exponents may exceed a row's reference by before it moves
constexpr float kTopHalf = 11.f;          // fp16 probabilities are over 2^-11: with the slack below fp16's largest, and bits down to 2^-35
constexpr int kTokens = 64;

// What a lane knows of its query row.
struct Row {
  int index;                              // of the item's rows, those of its drafted tokens; past them: of none, as the last
  bool there;
  int token, at;                          // its position
  uint64_t sees;                          // drafted tokens
  float slope, bias;                      // bias: of a key at the cache's next position
};

struct Out {                              // of a lane's row, over 32 or 64 lanes' channels
  floatx16 o[4];
  float m, l, top;                        // reference, sum of exponentials (of the lane's slots) over it, largest score
  __device__ __forceinline__ void init() {
#pragma unroll
    for (int t = 0; t < 4; ++t) o[t] = floatx16{};
    m = top = kNoScore;
    l = 0.f;
  }
};

// Scores of n products to probabilities; factor makes scores exponents of 2.  Of differences from the reference: a large number that scores have
// in common costs nothing.
template <int N>
__device__ __forceinline__ void refer(const float (&x)[N], float factor, Out& r) {
  float top = x[0];
#pragma unroll
  for (int i = 1; i < N; ++i) top = fmaxf(top, x[i]);
  top = halves_max(top);
  r.top = fmaxf(r.top, top);
  if (__any((top - r.m) * factor > kSlack)) {
    const float now = fmaxf(r.m, top), alpha = __builtin_amdgcn_exp2f((r.m - now) * factor);
    r.m = now;
    r.l *= alpha;
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
      for (int i = 0; i < 16; ++i) r.o[t][i] *= alpha;
  }
}
template <int N>
__device__ __forceinline__ void softmax(const float (&x)[N], float factor, float shift, Out& r, float (&p)[N]) {
  refer(x, factor, r);
  float sums[2] = {};                                // (as elsewhere: the same sum of the same scores)
#pragma unroll
  for (int i = 0; i < N; ++i) {
    p[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(x[i] - r.m, factor, shift));
    sums[i & 1] += p[i];
  }
  r.l += sums[0] + sums[1];
}

// o += P V for the channels of register group t; V's operands by value(step).  PARTED: some slots are hidden from some rows, and what is not finite
// in V must not meet their zeros.
template <bool PARTED, int STEPS, class Op, class Value>
__device__ __forceinline__ void add_values(const Op (&p)[STEPS], const float* probabilities, Value value, floatx16& o) {
#pragma unroll
  for (int k = 0; k < STEPS; ++k) {
    const Op v = value(k);
    if constexpr (!PARTED) {
      o = product(v, p[k], o);
    } else {
      const auto parted = part(v);
      o = product(parted.finite, p[k], o);
      if (__any(parted.any)) {
        Op one;
#pragma unroll
        for (int i = 0; i < 8; ++i) one[i] = probabilities[8 * k + i] == 0.f ? 0.f : 1.f;
        const floatx16 up = product(parted.up, one, floatx16{}), down = product(parted.down, one, floatx16{});
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          if (up[i] > 0.f) o[i] += INFINITY;
          if (down[i] > 0.f) o[i] -= INFINITY;
        }
      }
    }
  }
}

// bf16 rows in LDS, STEPS x 32 of them, into a row's result.  x: their scores (registers 16 step + i), -inf where hidden
template <int STEPS, bool PARTED>
__device__ __forceinline__ void add_rows16(const float (&x)[16 * STEPS], float factor, uint32_t vt, float shift, Out& r) {
  float p[16 * STEPS];
  softmax(x, factor, shift, r, p);
  bf16x8 op[2 * STEPS];
#pragma unroll
  for (int k = 0; k < 2 * STEPS; ++k) op[k] = to_bf16(p + 8 * k);
#pragma unroll
  for (int t = 0; t < 4; ++t)
    add_values<PARTED>(op, p, [&](int k) __attribute__((always_inline)) { return read_v(vt, t, k & 1, k >> 1); }, r.o[t]);
}

// What scores are made of products with.
struct Scoring {
  float natural;                          // products to scores, with a cap or biases
  float factor;                           // scores, or products, to exponents of 2
  float cap, inv_cap;
  bool scored, biased;                    // scores are made of products at once; of differences later
  int window, sinks;
};
// Products to scores, -inf where hidden, a step at a time over all of them.  Of products 4 k .. + 3: away(k, d), how far their positions are from the
// cache's next one; four(k, at), their positions.  hide(i): there is no slot, asked if `some` are none
template <bool GENERAL, int N, class Away, class Four, class Hide>
__device__ __forceinline__ void to_scores(const Scoring& sc, const Row& row, float (&x)[N], bool some, Away away, Four four, Hide hide) {
  if constexpr (GENERAL) {
    const float unit = sc.cap > 0.f ? sc.cap : sc.natural;
    if (sc.cap > 0.f) tanh_all(x, sc.natural * sc.inv_cap, TanhSmall(sc.natural * sc.inv_cap));
    if (sc.biased) {
#pragma unroll
      for (int k = 0; k < N / 4; ++k) {
        float d[4];
        away(k, d);
#pragma unroll
        for (int j = 0; j < 4; ++j) x[4 * k + j] = __builtin_fmaf(x[4 * k + j], unit, __builtin_fmaf(-row.slope, d[j], row.bias));
        __builtin_amdgcn_sched_barrier(0);
      }
    } else if (sc.cap > 0.f) {
#pragma unroll
      for (int i = 0; i < N; ++i) x[i] *= unit;
    }
    if (sc.window > 0) {
#pragma unroll
      for (int k = 0; k < N / 4; ++k) {
        int at[4];
        four(k, at);
#pragma unroll
        for (int j = 0; j < 4; ++j)
          if (row.at - at[j] >= sc.window && at[j] >= sc.sinks) x[4 * k + j] = -INFINITY;
        __builtin_amdgcn_sched_barrier(0);
      }
    }
  }
  if (some) {
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = hide(i) ? -INFINITY : x[i];
  }
}

// Wavefronts of a workgroup.  bf16 rows take a compute unit's LDS, eight wavefronts share them: two a SIMD, one's products beside the other's
// exponentials.  With 32 query rows or fewer eight shares of slots would be a tile more than half of the LDS holds.
template <int BITS, int WR>
constexpr int kWaves = BITS == 4 || WR == 1 ? 4 : 8;
template <int WR>
constexpr int kSteps16 = WR <= 2 ? 1 : 2;                       // 32-slot steps of a wavefront's tile
template <int WR>
constexpr int kStage = 32 * kSteps16<WR> * (kWaves<16, WR> / WR);    // slots of a stage
template <int WR>
constexpr int kStages = 256 / kStage<WR>;                       // buffers
constexpr int kStageLds = 256 * 2 * kRowBytes;                  // of all of them: 128 KiB
constexpr int kPosLds = 8 * 4 * 64 * 4;                         // positions of the wavefronts' tiles, up to four buffers
constexpr int kDraftLds = kTokens * 2 * kRowBytes;
constexpr int kJoinLds = 4 * 4 * 16 * 64 * 4;                   // four wavefronts' results
constexpr int kMetaLds = kKMeta + 1024 + 512 + 256;             // of a wavefront: K's, V's, positions and distances, add_odd's flags
constexpr int kImageLds = 32 * 1024;                            // a 4-bit tile's operands, K's, then V's, where wavefronts share them

// Values of a 4-bit tile that are not finite, to the rows that give their slots something.  odd: lanes 4 (slot / 4) + group whose metadata are not; lds:
// 256 bytes of the wavefront's; p: probabilities, register i of slot 32 half + i.
__device__ __forceinline__ void add_odd(uint64_t odd, const uint8_t* tile, int rows, uint8_t* lds, const float (&p)[32], Out& r) {
  const int lane = threadIdx.x & 63, l32 = lane & 31, half = lane >> 5;
  uint32_t* rows_of = reinterpret_cast<uint32_t*>(lds);          // [slot]: a bit a row
#pragma unroll
  for (int i = 0; i < 32; ++i) {
    const uint64_t some = __ballot(p[i] != 0.f);
    rows_of[i] = static_cast<uint32_t>(some);
    rows_of[32 + i] = static_cast<uint32_t>(some >> 32);
  }
  wave_lds_order();
  for (; odd != 0; odd &= odd - 1) {
    const int which = __builtin_ctzll(odd), group = which & 3;
    for (int slot = which & ~3; slot < min((which & ~3) + 4, rows); ++slot) {
      const _Float16* meta = reinterpret_cast<const _Float16*>(tile + kTileCodes + 16 * which);
      const float scale = static_cast<float>(meta[slot & 3]), centre = __builtin_fmaf(8.f, scale, static_cast<float>(meta[4 + (slot & 3)]));
      if (fabsf(scale) < INFINITY && fabsf(static_cast<float>(static_cast<_Float16>(centre))) < INFINITY) continue;
      const bool some = (rows_of[slot] >> l32 & 1) != 0;
      const int k = slot & 31;
      float v[16];
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const int channel = 8 * (i >> 2) + 4 * half + (i & 3);
        const uint32_t word = *reinterpret_cast<const uint32_t*>(tile + 1024 * group + 16 * (32 * (slot >> 5) + channel) + 4 * (2 * (k >> 4) + ((k >> 1) & 1)));
        const int code = (word >> (16 * (k & 1) + 4 * ((k >> 2) & 3))) & 15;
        v[i] = some ? __builtin_fmaf(static_cast<float>(code - 8), scale, centre) : 0.f;
      }
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        if (g != group) continue;
#pragma unroll
        for (int i = 0; i < 16; ++i) r.o[g][i] += v[i];
      }
    }
  }
  wave_lds_order();
}

template <int BITS, int WR, bool GENERAL>
__global__ __launch_bounds__(64 * (kWaves<BITS, WR>), BITS == 4 || WR > 1 ? 2 : 1) void tree_kernel(TreeArgs a) {
  constexpr int NW = kWaves<BITS, WR>;
  extern __shared__ __align__(256) uint8_t smem[];
  __shared__ int s_depth[kTokens];
  __shared__ float s_ml[NW][32][4];
  constexpr int WS = NW / WR;
  const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6), l32 = lane & 31, half = lane >> 5;
  const int wr = wave % WR, ws = wave / WR;
  // row groups of a piece are eight workgroups apart, on one XCD
  const int in = static_cast<int>(blockIdx.x) % (8 * a.row_groups), unit = static_cast<int>(blockIdx.x) / (8 * a.row_groups) * 8 + in % 8, rg = in / 8;
  if (unit >= a.items * a.pieces) return;
  const int item = unit / a.pieces, piece = unit % a.pieces, seq = item / a.s.hkv, kvh = item % a.s.hkv, g = a.s.g, n = a.n;
  const int count = a.counts ? min(max(a.counts[seq], 0), n) : n;
  if (rg * WR * 32 >= count * g) return;

  const int len = a.s.length(item), next = a.s.next[item];
  int parent = lane < n ? a.parent[static_cast<int64_t>(seq) * n + lane] : -1;
  Row row;
  {
    const int r = (rg * WR + wr) * 32 + l32;
    row.there = r < count * g;
    row.index = min(r, count * g - 1);                                    // (rows of tokens from `count` on may hold anything)
    row.token = row.index / g;
    row.slope = GENERAL && a.s.slopes ? a.s.slopes[kvh * g + row.index % g] : 0.f;
  }
  const int64_t q_row = (static_cast<int64_t>(seq) * n + row.token) * a.s.hkv * g + kvh * g + row.index % g;
  using Query = std::conditional_t<BITS == 16, Query16, Query4>;
  Query query;
  query.load(a.q + q_row * kHeadDim);
  // ancestors: a bit of each, and the token's own; lane t token t's, twice as far up in each turn
  {
    uint64_t sees = 1ull << lane;
    if (parent >= lane) parent = -1;
#pragma unroll
    for (int k = 1; k < kTokens; k *= 2) {
      const uint64_t theirs = __shfl(sees, max(parent, 0));
      const int further = __shfl(parent, max(parent, 0));
      if (parent >= 0) {
        sees |= theirs;
        parent = further;
      }
    }
    row.sees = __shfl(sees, row.token);
    row.at = next + __popcll(row.sees) - 1;
    row.bias = -row.slope * static_cast<float>(row.at - next);
    if (wave == 0) s_depth[lane] = __popcll(sees) - 1;                   // (read behind the barriers of the drafted tokens)
  }
  Scoring sc;
  sc.cap = a.s.cap;
  sc.inv_cap = a.s.cap > 0.f ? 1.f / a.s.cap : 0.f;
  sc.biased = a.s.slopes != nullptr;
  sc.window = a.s.window;
  sc.sinks = a.s.sinks;
  sc.scored = GENERAL && (sc.cap > 0.f || sc.biased);
  sc.natural = sc.scored ? query.unit * kRoot : 1.f;
  sc.factor = sc.scored ? kLog2e : query.unit * kRootLog2e;

  Out r;
  // this piece's slots: whole tiles of 64
  const int tiles = (len + kTileRows - 1) / kTileRows;
  const int from = min(piece, a.slot_pieces), to = min(piece + 1, a.slot_pieces);                // (of the drafted tokens' own piece: none)
  const int begin = static_cast<int>(static_cast<int64_t>(tiles) * from / a.slot_pieces) * kTileRows;
  const int end = min(len, static_cast<int>(static_cast<int64_t>(tiles) * to / a.slot_pieces) * kTileRows);
  const int32_t* pos = a.s.pos + static_cast<int64_t>(item) * a.s.capacity;
  const uint32_t lds0 = lds_address(smem);
  const int prow = tid >> 4;
  const uint32_t k_at = 16 * k_piece(prow, tid & 15), v_at = 16 * v_piece(prow, tid & 15);
  // `most` bf16 rows, `stride` bytes apart, into LDS; rows past the last are it again
  const auto fetch_rows = [&](const uint8_t* from, uint32_t at, uint32_t stride, int last, int most, uint32_t to) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < most; i += 4 * NW) copy_to_lds(from, static_cast<uint32_t>(min(prow + i, last)) * stride + at, to + i * kRowBytes + wave * 1024);
  };

  // Careful (bf16): rows of V that a window hides from some query rows, and those behind the last that are the last again, are kept from meeting their
  // zeros, which make NaN of what is not finite.  Done again so where results are not finite.
  const auto walk = [&](auto careful) __attribute__((always_inline)) {
    constexpr bool kCareful = decltype(careful)::value;
    r.init();
    if constexpr (BITS == 16) {
      constexpr int kStepsN = kSteps16<WR>, kSlots = kStage<WR>, kBuffers = kStages<WR>, kMine = 32 * kStepsN;
      constexpr int kCopies = kSlots / (2 * NW) + (GENERAL ? 1 : 0);      // of a wavefront and stage
      const uint8_t* K = a.s.k + static_cast<int64_t>(item) * a.s.capacity * kRowBytes;
      const uint8_t* V = a.s.v + static_cast<int64_t>(item) * a.s.capacity * kRowBytes;
      constexpr uint32_t kSide = kSlots * kRowBytes;
      const int n_it = (end - begin + kSlots - 1) / kSlots, mine = ws * kMine;
      uint8_t* s_pos = smem + kStageLds;
      const auto k_of = [&](int it) { return lds0 + it % kBuffers * kSide; };
      const auto v_of = [&](int it) { return lds0 + (kBuffers + it % kBuffers) * kSide; };
      const auto fetch_k = [&](int it) __attribute__((always_inline)) {
        const int first = begin + min(it, n_it - 1) * kSlots;
        fetch_rows(K + static_cast<int64_t>(first) * kRowBytes, k_at, kRowBytes, end - 1 - first, kSlots, k_of(it));
        if constexpr (GENERAL) copy_word_to_lds(pos + first, 4 * (min(first + mine + lane, end - 1) - first),
                                                lds0 + kStageLds + (wave * kBuffers + it % kBuffers) * 256);
      };
      const auto fetch_v = [&](int it) __attribute__((always_inline)) {
        const int first = begin + min(it, n_it - 1) * kSlots;
        fetch_rows(V + static_cast<int64_t>(first) * kRowBytes, v_at, kRowBytes, end - 1 - first, kSlots, v_of(it));
      };
      const auto left_of = [&](int it) { return end - begin - it * kSlots - mine - 4 * half; };
      const auto finish = [&](int it, float (&x)[16 * kStepsN]) __attribute__((always_inline)) {
        const int left = left_of(it);
        const int4* where = reinterpret_cast<const int4*>(s_pos + (wave * kBuffers + it % kBuffers) * 256);
        to_scores<GENERAL>(sc, row, x, left < kMine, [&](int k, float* d) __attribute__((always_inline)) {
          const int4 at = where[2 * k + half];
          d[0] = static_cast<float>(next - at.x);
          d[1] = static_cast<float>(next - at.y);
          d[2] = static_cast<float>(next - at.z);
          d[3] = static_cast<float>(next - at.w);
        }, [&](int k, int* at) __attribute__((always_inline)) { *reinterpret_cast<int4*>(at) = where[2 * k + half]; },
                           [&](int i) __attribute__((always_inline)) { return 32 * (i >> 4) + 8 * ((i & 15) >> 2) + (i & 3) >= left; });
      };
      const auto multiply = [&](int it, float (&x)[16 * kStepsN]) __attribute__((always_inline)) {
#pragma unroll
        for (int k = 0; k < kStepsN; ++k) {
          const floatx16 s = scores16(k_of(it) + mine * kRowBytes + k_lane(), k, query);
#pragma unroll
          for (int i = 0; i < 16; ++i) x[16 * k + i] = s[i];
        }
      };
      if constexpr (!kCareful && !GENERAL) {
        constexpr int N = 16 * kStepsN, kHalf = N / 2;   // scores of a stage; products of each kind
        // a stage's softmax and P V, and between their instructions the products of the next (MORE): a line is one product and what the plain ALUs do
        // meanwhile
        const auto position = [&](auto more, int it, float (&x)[N], float (&next)[N]) __attribute__((always_inline)) {
          constexpr bool kMore = decltype(more)::value;
          refer(x, sc.factor, r);
          float sums[2] = {}, e[3], y = (x[0] - r.m) * sc.factor;
          union { uint32_t u[N / 2]; bf16x8 op[N / 8]; } p;
          // exponential i, in order; what hangs on another one's result stands behind it
          const auto make = [&](int i) __attribute__((always_inline)) {
            const float now = y;
            if (i < N - 1) y = (x[i + 1] - r.m) * sc.factor;
            if (i < N) e[i % 3] = __builtin_amdgcn_exp2f(now);
            if (i > 0) {
              sums[i & 1] += e[(i - 1) % 3];
              here(sums[i & 1]);
            }
            if (i > 0 && (i & 1) == 0) p.u[(i >> 1) - 1] = pair_bf16(e[(i - 2) % 3], e[(i - 1) % 3]);
          };
          const uint32_t kt = k_of(it + 1) + mine * kRowBytes + k_lane(), vt = v_of(it) + mine * kRowBytes + v_lane();
          constexpr int kAhead = 3;
          bf16x8 op[kAhead];
          const auto ask = [&](int i) __attribute__((always_inline)) {
            if (i < kHalf) op[i % kAhead] = read_k(kt, i & 7, i >> 3);
            else if (i < N) op[i % kAhead] = read_v(vt, i & 3, (i >> 2) & 1, (i - kHalf) >> 3);
          };
          if constexpr (kMore) {
            floatx16 s[kStepsN];
#pragma unroll
            for (int i = 0; i < kAhead; ++i) ask(i);
#pragma unroll
            for (int i = 0; i < kHalf; ++i) {
              s[i >> 3] = product(op[i % kAhead], query.op[i & 7], (i & 7) == 0 ? floatx16{} : s[i >> 3]);
              ask(i + kAhead);
              make(i);
              if (i == kHalf - 1) make(kHalf);
              __builtin_amdgcn_sched_barrier(0);
            }
#pragma unroll
            for (int i = 0; i < N; ++i) next[i] = s[i >> 4][i & 15];
          } else {
#pragma unroll
            for (int i = kHalf; i < kHalf + kAhead; ++i) ask(i);
#pragma unroll
            for (int i = 0; i <= kHalf; ++i) make(i);
          }
#pragma unroll
          for (int i = 0; i < kHalf; ++i) {
            r.o[i & 3] = product(op[(i + kHalf) % kAhead], p.op[i >> 2], r.o[i & 3]);
            ask(i + kHalf + kAhead);
            if (i < kHalf / 2) {
              make(kHalf + 1 + 2 * i);
              make(kHalf + 2 + 2 * i);
            }
            __builtin_amdgcn_sched_barrier(0);
          }
          r.l += sums[0] + sums[1];
          if constexpr (kMore) finish(it + 1, next);
        };
        // K of stage it + 1 and V of stage it are there, K of stage it and V of the one before are done with
        const auto open = [&](int it) __attribute__((always_inline)) {
          tile_barrier<kCopies * (kBuffers - 2)>();
          fetch_k(it + kBuffers);
          fetch_v(it + kBuffers - 1);
        };
        if (n_it > 0) {
          fetch_k(0);
#pragma unroll
          for (int it = 0; it < kBuffers - 1; ++it) {
            fetch_k(it + 1);
            fetch_v(it);
          }
          tile_barrier<kCopies * (kBuffers - 1)>();
          const int n_mine = max(0, (end - begin - mine + kSlots - 1) / kSlots);         // stages in which this wavefront has slots
          float even[N], odd[N];
          int it = 0;
          if (n_mine > 0) {
            multiply(0, even);
            finish(0, even);
          }
          for (; it + 2 < n_mine; it += 2) {
            open(it);
            position(std::true_type{}, it, even, odd);
            open(it + 1);
            position(std::true_type{}, it + 1, odd, even);
          }
          if (it < n_mine) {
            open(it);
            if (it + 1 < n_mine) {
              position(std::true_type{}, it, even, odd);
              open(++it);
              position(std::false_type{}, it, odd, even);
            } else {
              position(std::false_type{}, it, even, odd);
            }
            ++it;
          }
          for (; it < n_it; ++it) open(it);
          tile_barrier<0>();
        }
      } else if (n_it > 0) {
#pragma unroll
        for (int it = 0; it < kBuffers - 1; ++it) {
          fetch_k(it);
          fetch_v(it);
        }
        for (int it = 0; it < n_it; ++it) {
          tile_barrier<kCopies * (kBuffers - 2)>();
          fetch_k(it + kBuffers - 1);
          fetch_v(it + kBuffers - 1);
          if (left_of(it) + 4 * half <= 0) continue;
          float x[16 * kStepsN];
          multiply(it, x);
          finish(it, x);
          add_rows16<kStepsN, kCareful>(x, sc.factor, v_of(it) + mine * kRowBytes + v_lane(), 0.f, r);
        }
        tile_barrier<0>();
      }
    } else {
      constexpr bool kShared = WR == 4;                  // every wavefront has the same tiles
      uint8_t* meta = smem + (kShared ? 2 * kImageLds : kDraftLds) + wave * kMetaLds;
      const uint8_t* K = a.s.k + static_cast<int64_t>(item) * a.s.tiles * kTileBytes;
      const uint8_t* V = a.s.v + static_cast<int64_t>(item) * a.s.tiles * kTileBytes;
      const int t1 = (end + kTileRows - 1) / kTileRows;
      const Codes4 codes;
      // a tile's scores, softmax and P V
      const auto put_positions = [&](int at) __attribute__((always_inline)) {
        if constexpr (GENERAL) {
          reinterpret_cast<int*>(meta + kKMeta + 1024)[lane] = at;
          reinterpret_cast<float*>(meta + kKMeta + 1024 + 256)[lane] = static_cast<float>(next - at);
        }
      };
      const auto finish = [&](int left, const floatx16 (&s)[2], float (&x)[32]) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < 32; ++i) x[i] = s[i >> 4][i & 15];
        const int4* where = reinterpret_cast<const int4*>(meta + kKMeta + 1024) + 8 * half;
        to_scores<GENERAL>(sc, row, x, left < kTileRows,
                           [&](int k, float* d) __attribute__((always_inline)) { *reinterpret_cast<int4*>(d) = where[16 + k]; },
                           [&](int k, int* at) __attribute__((always_inline)) { *reinterpret_cast<int4*>(at) = where[k]; },
                           [&](int i) __attribute__((always_inline)) { return 32 * half + i >= left; });
      };
      // value(channel group, step)
      const auto add = [&](const float (&x)[32], int tile, int left, uint64_t odd, auto value) __attribute__((always_inline)) {
        float p[32], pf[32];
        softmax(x, sc.factor, kTopHalf, r, p);
        halfx8 op[4];
#pragma unroll
        for (int f = 0; f < 4; ++f) {
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            pf[8 * f + j] = p[4 * f + j];
            pf[8 * f + 4 + j] = p[16 + 4 * f + j];
          }
          op[f] = to_half(pf + 8 * f);
        }
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          __builtin_amdgcn_sched_barrier(0);
          add_values<false>(op, pf, [&](int f) __attribute__((always_inline)) { return value(c, f); }, r.o[c]);
        }
        if (GENERAL && odd != 0) add_odd(odd, V + static_cast<int64_t>(tile) * kTileBytes, left, meta + kMetaLds - 256, p, r);
      };
      const auto values = [&](const uint4& words, int c, int f) __attribute__((always_inline)) {
        return f == 0 ? values4<0>(codes, words, meta + kKMeta, c) : f == 1 ? values4<1>(codes, words, meta + kKMeta, c)
             : f == 2 ? values4<2>(codes, words, meta + kKMeta, c) : values4<3>(codes, words, meta + kKMeta, c);
      };
      int t = begin / kTileRows + ws;
      if constexpr (!kShared) {
        Side4 k, v;
        int at = 0;
        // the next tile's K comes while this one's values are added up, its V while its scores are made
        const auto load_k = [&](int tile) __attribute__((always_inline)) {
          k.load(K + static_cast<int64_t>(tile) * kTileBytes, true);
          if constexpr (GENERAL) at = pos[min(tile * kTileRows + lane, len - 1)];
        };
        const auto load_v = [&](int tile) __attribute__((always_inline)) { v.load(V + static_cast<int64_t>(tile) * kTileBytes, false); };
        if (t < t1) {
          load_k(t);
          load_v(t);
        }
        for (; t < t1; t += WS) {
          const int left = end - t * kTileRows;
          put_k_meta(meta, k.meta, left);
          put_positions(at);
          wave_lds_order();
          floatx16 s[2];
          {
            const Words4 words(k);
            scores4(meta, query, s, [&](int x, int g, int h) __attribute__((always_inline)) { return words.operand(codes, x, g, h); });
          }
          load_k(min(t + WS, t1 - 1));
          float x[32];
          finish(left, s, x);
          // with a window, values that are not finite are kept out, and go to those rows that see them afterwards
          const uint64_t odd = put_v_meta<GENERAL>(meta + kKMeta, v.meta, left);
          wave_lds_order();
          add(x, t, left, odd, [&](int c, int f) __attribute__((always_inline)) { return values(v.codes[c], c, f); });
          load_v(min(t + WS, t1 - 1));
          wave_lds_order();
        }
      } else if (t < t1) {
        // Each wavefront makes operands of a group's codes for all four, a tile ahead, into one of two images in LDS.
        uint4 k_codes, k_meta, v_codes, v_meta;
        int at = 0;
        const auto load = [&](int tile) __attribute__((always_inline)) {
          const uint8_t *kt = K + static_cast<int64_t>(tile) * kTileBytes, *vt = V + static_cast<int64_t>(tile) * kTileBytes;
          k_codes = *reinterpret_cast<const uint4*>(kt + 1024 * wave + 16 * slot_of_row(half, l32));
          k_meta = *reinterpret_cast<const uint4*>(kt + kTileCodes + 16 * lane);
          v_codes = *reinterpret_cast<const uint4*>(vt + 1024 * wave + 16 * lane);
          v_meta = *reinterpret_cast<const uint4*>(vt + kTileCodes + 16 * lane);
          if constexpr (GENERAL) at = pos[min(tile * kTileRows + lane, len - 1)];
        };
        const auto image = [&](int tile) { return smem + (tile & 1) * kImageLds + 16 * lane; };
        const auto make = [&](int tile) __attribute__((always_inline)) {
          const uint64_t odd = put_v_meta<GENERAL>(meta + kKMeta, v_meta, end - tile * kTileRows);
          wave_lds_order();
          uint8_t* to = image(tile);
          const Group4 group(k_codes);
#pragma unroll
          for (int x = 0; x < 2; ++x)
#pragma unroll
            for (int h = 0; h < 2; ++h) *reinterpret_cast<halfx8*>(to + ((4 * x + wave) * 2 + h) * 1024) = group.operand(codes, x, h);
#pragma unroll
          for (int f = 0; f < 4; ++f) *reinterpret_cast<halfx8*>(to + kImageLds / 2 + (4 * wave + f) * 1024) = values(v_codes, wave, f);
          return odd;
        };
        load(t);
        uint64_t odd = make(t);
        uint4 meta_now = k_meta;
        int at_now = at;
        load(min(t + 1, t1 - 1));
        tile_barrier<63>();
        for (; t < t1; ++t) {
          const int left = end - t * kTileRows;
          put_k_meta(meta, meta_now, left);
          put_positions(at_now);
          uint64_t odd_next = 0;
          if (t + 1 < t1) odd_next = make(t + 1);
          meta_now = k_meta;
          at_now = at;
          load(min(t + 2, t1 - 1));
          wave_lds_order();
          const uint8_t* from = image(t);
          floatx16 s[2];
          scores4(meta, query, s, [&](int x, int g, int h) __attribute__((always_inline)) {
            return *reinterpret_cast<const halfx8*>(from + ((4 * x + g) * 2 + h) * 1024);
          });
          float x[32];
          finish(left, s, x);
          add(x, t, left, odd, [&](int c, int f) __attribute__((always_inline)) {
            return *reinterpret_cast<const halfx8*>(from + kImageLds / 2 + (4 * c + f) * 1024);
          });
          odd = odd_next;
          tile_barrier<63>();
        }
      }
    }
  };
  walk(std::false_type{});
  if constexpr (BITS == 16) {
    float zero = r.l * 0.f;
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
      for (int i = 0; i < 16; ++i) zero = __builtin_fmaf(r.o[t][i], 0.f, zero);
    if (__syncthreads_or(zero != 0.f)) walk(std::true_type{});
  }

  // the drafted tokens themselves
  if (piece == a.pieces - 1) {
    const int64_t first = (static_cast<int64_t>(seq) * n * a.s.hkv + kvh) * kRowBytes;
    fetch_rows(reinterpret_cast<const uint8_t*>(a.k_draft) + first, k_at, a.s.hkv * kRowBytes, count - 1, kTokens, lds0);
    fetch_rows(reinterpret_cast<const uint8_t*>(a.v_draft) + first, v_at, a.s.hkv * kRowBytes, count - 1, kTokens, lds0 + kTokens * kRowBytes);
    tile_barrier<0>();
    if (ws == 0) {
      Query16 q16;
      q16.load(a.q + q_row * kHeadDim);
      Scoring own = sc;
      own.natural = sc.scored ? kRoot : 1.f / query.unit;        // as of the slots: the unit is a power of two
      float x[32];
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const floatx16 s = scores16(lds0 + k_lane(), k, q16);
#pragma unroll
        for (int i = 0; i < 16; ++i) x[16 * k + i] = s[i];
      }
      const auto token = [&](int i) __attribute__((always_inline)) { return 32 * (i >> 4) + 8 * ((i & 15) >> 2) + 4 * half + (i & 3); };
      if (!sc.scored) {
#pragma unroll
        for (int i = 0; i < 32; ++i) x[i] *= own.natural;
      }
      to_scores<GENERAL>(own, row, x, true, [&](int k, float* d) __attribute__((always_inline)) {
#pragma unroll
        for (int j = 0; j < 4; ++j) d[j] = -static_cast<float>(s_depth[min(token(4 * k + j), n - 1)]);
      }, [&](int k, int* at) __attribute__((always_inline)) {
#pragma unroll
        for (int j = 0; j < 4; ++j) at[j] = next + s_depth[min(token(4 * k + j), n - 1)];
      }, [&](int i) __attribute__((always_inline)) { return (row.sees >> token(i) & 1) == 0; });
      add_rows16<2, true>(x, sc.factor, lds0 + kTokens * kRowBytes + v_lane(), BITS == 4 ? kTopHalf : 0.f, r);
    }
  }

  // one result of the wavefronts that have the same rows
  r.l = halves_add(r.l);
  int t0 = 0, t1 = 4;                     // register groups that this wavefront has of it
  if constexpr (WS > 1) {
    __syncthreads();
    if (half == 0) {
      s_ml[wave][l32][0] = r.m;
      s_ml[wave][l32][1] = r.l;
      s_ml[wave][l32][2] = r.top;
    }
    __syncthreads();
    float m = r.m;
#pragma unroll
    for (int k = 0; k < WS; ++k) m = fmaxf(m, s_ml[k * WR + wr][l32][0]);
    float l = 0.f;
#pragma unroll
    for (int k = 0; k < WS; ++k) {
      const float* ml = s_ml[k * WR + wr][l32];
      l = __builtin_fmaf(ml[1], __builtin_amdgcn_exp2f((ml[0] - m) * sc.factor), l);
      r.top = fmaxf(r.top, ml[2]);
    }
    const float alpha = __builtin_amdgcn_exp2f((r.m - m) * sc.factor);
    r.m = m;
    r.l = l;
    float4* mine = reinterpret_cast<float4*>(smem) + wave * 16 * 64;
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
      for (int b = 0; b < 4; ++b)
        mine[(4 * t + b) * 64 + lane] = make_float4(r.o[t][4 * b] * alpha, r.o[t][4 * b + 1] * alpha, r.o[t][4 * b + 2] * alpha, r.o[t][4 * b + 3] * alpha);
    __syncthreads();
    t0 = ws * 4 / WS;
    t1 = t0 + 4 / WS;
  }
  const int64_t slot = (static_cast<int64_t>(item) * a.row_groups + rg) * a.pieces + piece;
  const int64_t part_row = slot * (32 * WR) + 32 * wr + l32;
  const bool direct = a.pieces == 1;
  const float inv = direct ? (r.l == 0.f ? 0.f : 1.f / r.l) : 1.f;
#pragma unroll
  for (int t = 0; t < 4; ++t) {
    if (t < t0 || t >= t1) continue;
    floatx16 o = r.o[t];
    if constexpr (WS > 1) {
#pragma unroll
      for (int b = 0; b < 4; ++b) {
        float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int k = 0; k < WS; ++k) {
          const float4 w = reinterpret_cast<const float4*>(smem)[(k * WR + wr) * 16 * 64 + (4 * t + b) * 64 + lane];
          v = make_float4(v.x + w.x, v.y + w.y, v.z + w.z, v.w + w.w);
        }
        o[4 * b] = v.x;
        o[4 * b + 1] = v.y;
        o[4 * b + 2] = v.z;
        o[4 * b + 3] = v.w;
      }
    }
    if (!row.there) continue;
    if (direct) {
#pragma unroll
      for (int b = 0; b < 4; ++b) {
        union { __bf16 h[4]; uint2 u; } w;
#pragma unroll
        for (int j = 0; j < 4; ++j) w.h[j] = static_cast<__bf16>(o[4 * b + j] * inv);
        *reinterpret_cast<uint2*>(a.out + q_row * kHeadDim + 32 * t + 8 * b + 4 * half) = w.u;
      }
    } else {
#pragma unroll
      for (int b = 0; b < 4; ++b)
        *reinterpret_cast<float4*>(a.part_acc + part_row * kHeadDim + 32 * t + 8 * b + 4 * half) = make_float4(o[4 * b], o[4 * b + 1], o[4 * b + 2], o[4 * b + 3]);
    }
  }
  if (row.there && half == 0 && ws == 0) {
    if (direct) {
      if (a.stats) store_stats(a.stats + 2 * q_row, r.m, r.l, r.top, sc.factor, sc.scored ? 1.f : query.unit * kRoot, BITS == 4 ? kTopHalf : 0.f);
    } else {
      *reinterpret_cast<float4*>(a.part_ml + part_row * 4) = make_float4(r.m, r.l, r.top, query.unit);
    }
  }
}

// The pieces' results of 8 / PARTS rows, whose pieces PARTS groups of 32 lanes share out: a chain of loads, so that many pieces need several groups
// (a call with 256 of them 97 us by one, 32 by eight).
template <int BITS, int PARTS>
__global__ __launch_bounds__(256) void tree_join_kernel(TreeArgs a, int group_rows) {
  constexpr int kRowsN = 8 / PARTS;
  __shared__ float4 s_v[8][32], s_ml[8];
  const int g = a.s.g, n = a.n, rows = n * g, blocks = (rows + kRowsN - 1) / kRowsN;
  const int group = threadIdx.x >> 5, part = group % PARTS, c = threadIdx.x & 31;
  const int item = blockIdx.x / blocks, row = blockIdx.x % blocks * kRowsN + group / PARTS;
  const int seq = item / a.s.hkv, kvh = item % a.s.hkv;
  const int count = a.counts ? min(max(a.counts[seq], 0), n) : n;
  const bool there = row < count * g;
  const int64_t slot = (static_cast<int64_t>(item) * a.row_groups + row / group_rows) * a.pieces;
  const int64_t first = slot * group_rows + row % group_rows;
  const bool scored = a.s.cap > 0.f || a.s.slopes;
  const int pieces = there ? a.pieces : 0;
  float m = kNoScore, top = kNoScore, unit = 1.f;
#pragma unroll 4
  for (int p = part; p < pieces; p += PARTS) {
    const float4 ml = *reinterpret_cast<const float4*>(a.part_ml + (first + static_cast<int64_t>(p) * group_rows) * 4);
    m = fmaxf(m, ml.x);
    top = fmaxf(top, ml.z);
    unit = ml.w;
  }
  const float factor = scored ? kLog2e : unit * kRootLog2e;
  float l = 0.f;
  float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
  const auto add = [&](const float4& ml, const float4& w, float over, float scale) {
    const float f = __builtin_amdgcn_exp2f((ml.x - over) * scale);
    l = __builtin_fmaf(ml.y, f, l);
    v = make_float4(__builtin_fmaf(w.x, f, v.x), __builtin_fmaf(w.y, f, v.y), __builtin_fmaf(w.z, f, v.z), __builtin_fmaf(w.w, f, v.w));
  };
#pragma unroll 4
  for (int p = part; p < pieces; p += PARTS) {
    const int64_t at = first + static_cast<int64_t>(p) * group_rows;
    add(*reinterpret_cast<const float4*>(a.part_ml + at * 4), *reinterpret_cast<const float4*>(a.part_acc + at * kHeadDim + 4 * c), m, factor);
  }
  if constexpr (PARTS > 1) {
    s_v[group][c] = v;
    if (c == 0) s_ml[group] = make_float4(m, l, top, unit);
    __syncthreads();
    if (part != 0) return;
    const float mine = m;
#pragma unroll
    for (int k = 1; k < PARTS; ++k) {
      m = fmaxf(m, s_ml[group + k].x);
      top = fmaxf(top, s_ml[group + k].z);
    }
    const float4 own = v;
    const float own_l = l;
    l = 0.f;
    v = make_float4(0.f, 0.f, 0.f, 0.f);
    add(make_float4(mine, own_l, 0.f, 0.f), own, m, factor);
#pragma unroll
    for (int k = 1; k < PARTS; ++k) add(s_ml[group + k], s_v[group + k][c], m, factor);
  }
  if (!there) return;
  const float inv = l == 0.f ? 0.f : 1.f / l;
  const int64_t q_row = (static_cast<int64_t>(seq) * n + row / g) * a.s.hkv * g + kvh * g + row % g;
  union { __bf16 h[4]; uint2 u; } out;
  out.h[0] = static_cast<__bf16>(v.x * inv);
  out.h[1] = static_cast<__bf16>(v.y * inv);
  out.h[2] = static_cast<__bf16>(v.z * inv);
  out.h[3] = static_cast<__bf16>(v.w * inv);
  *reinterpret_cast<uint2*>(a.out + q_row * kHeadDim + 4 * c) = out.u;
  if (c == 0 && a.stats) store_stats(a.stats + 2 * q_row, m, l, top, factor, scored ? 1.f : unit * kRoot, BITS == 4 ? kTopHalf : 0.f);
}
template <int BITS>
hipError_t join(const TreeArgs& a, hipStream_t st) {
  // where eight rows a workgroup fill the card, or pieces are few, one group has a row (8 pieces of 32 x 256 rows 10 us, by eight groups 19)
  const int rows = a.n * a.s.g, eights = (rows + 7) / 8;
  if (a.pieces <= 4 || static_cast<int64_t>(a.items) * eights >= 512)
    hipLaunchKernelGGL((tree_join_kernel<BITS, 1>), dim3(a.items * eights), dim3(256), 0, st, a, 32 * a.wide);
  else hipLaunchKernelGGL((tree_join_kernel<BITS, 8>), dim3(a.items * rows), dim3(256), 0, st, a, 32 * a.wide);
  return hipGetLastError();
}

template <int BITS, int WR, bool GENERAL>
hipError_t start(const TreeArgs& a, hipStream_t st) {
  constexpr int NW = kWaves<BITS, WR>;
  constexpr int lds = BITS == 16 ? kStageLds + kPosLds : WR == 4 ? 2 * kImageLds + NW * kMetaLds : std::max(kDraftLds + NW * kMetaLds, kJoinLds);
  const hipError_t e = RDKV_ALLOW_LDS((tree_kernel<BITS, WR, GENERAL>), lds);
  if (e != hipSuccess) return e;
  const int units = (a.items * a.pieces + 7) / 8 * 8;
  hipLaunchKernelGGL((tree_kernel<BITS, WR, GENERAL>), dim3(units * a.row_groups), dim3(64 * NW), lds, st, a);
  return hipGetLastError();
}

template <int BITS, bool GENERAL>
hipError_t start(const TreeArgs& a, int wide, hipStream_t st) {
  if constexpr (BITS == 16) {
    if (wide == 8) return start<BITS, 8, GENERAL>(a, st);
  }
  return wide == 1 ? start<BITS, 1, GENERAL>(a, st) : wide == 2 ? start<BITS, 2, GENERAL>(a, st) : start<BITS, 4, GENERAL>(a, st);
}

}  // namespace

hipError_t launch_tree(const TreeArgs& a, int bits, hipStream_t st) {
  const bool general = a.s.cap > 0.f || a.s.slopes || a.s.window > 0;
  hipError_t e = bits == 16 ? (general ? start<16, true>(a, a.wide, st) : start<16, false>(a, a.wide, st))
                            : (general ? start<4, true>(a, a.wide, st) : start<4, false>(a, a.wide, st));
  if (e != hipSuccess || a.pieces == 1) return e;
  return bits == 16 ? join<16>(a, st) : join<4>(a, st);
}

}  // namespace slots
}  // namespace rdkv
