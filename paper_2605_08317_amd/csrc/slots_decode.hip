// Slot caches: the decode step.
//
// One pass over the rows, as in the other decode kernels (decode_rows.h, decode_mfma_kernels.hip): a wavefront takes tiles of 64 slots,
// makes their scores with four query heads on one side of v_mfma_f32_4x4x4, keeps a running maximum and sum of its softmax, and
// adds P V to accumulators in registers.  What is its own here:
//
//   scores     lane = slot, four heads in a lane's registers: capped, biased and hidden there, and stored for the weights, which need
//              every probability once the whole sum is known: 4 bytes per slot and query head, which stay in the caches
//   precision  bf16 rows meet a probability in three bf16 terms, all of its 24 bits, codes in two fp16 terms (22 bits), scaled so that
//              the largest V scale seen stands just below fp16's largest and a head's largest query value near 2^8.  (What fp16 terms lose
//              of the small beside the large: a query value 2^-33 of its head's largest; of a probability times a V scale 2^-40 of the
//              largest scale seen, so that a probability near 1 keeps 20 bits where its row's scale is 2^20 smaller than that)
//   bound      HBM: 512 bytes a slot in bf16, 160 in 4 bits, and the scores.  4 x 8 items of 128K slots 6.8 and 6.1 TB/s without weights, 5.5
//              and 4.5 with them; items one each to a workgroup 6.3 TB/s (256 of 4000 slots in bf16) and 4.8.  Small caches: latency
//   work       lengths are on the device.  A workgroup takes an item, where there are enough for the card; otherwise it finds its piece
//              of one by itself, nearly equal ones, which leave partial results for the launch that follows
#include <algorithm>

#include "decode_rows.h"
#include "slots.h"

namespace rdkv {
namespace slots {

namespace {

using namespace tile;

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr float kRoot = 0.08838834764831845f;      // 1 / sqrt(128)
constexpr float kRootLog2e = 0.12751743f;          // both: 0.0883883476 x 1.4426950409 = 0.12751743 (to 2^-25)
constexpr float kLowest = -3.402823466e38f;        // a finite maximum of nothing: no score is below it

struct DecodeArgs {
  Args s;
  const uint16_t* q;
  float* out;
  float* lse;
  float* scores;       // [items][score_rows][g], before the last factor; null: no weights are kept
  float* part_acc;     // [slot][g][128]: partials; slot = workgroup + item
  float* part_ml;      // [slot][g][2]: maximum, before the last factor, and sum
  int2* parts;         // [items]: an item's first partial and their number, 0 where it has none
  int32_t held_bytes;  // of scores that a wavefront keeps
  float factor;        // what makes products or, with a cap or biases, scores exponents of 2,
  float natural;       // and what makes them scores
  int32_t items, score_rows;
  int32_t least, start;                 // of a workgroup's share, tiles; 0: a workgroup takes an item.  What a start on one is worth
};

// How the tiles of all items are shared out among the workgroups.  An item is cut into pieces, one for each of its workgroups: the largest
// piece is the smallest of an equal share of all tiles and up to 8 tiles more that leaves no more pieces than workgroups.  If none of these
// does, the items are a line, on which each has `start` places and then its tiles, workgroup w has the places from w * share on, and some
// have the end of one item and the begin of the next, or several: each is a start and a merge, as long as `start` tiles take to pass (4 in
// bf16, 8 in 4 bits).
//   pieces and the line (a start counting nothing), us: 4 bits, 8 heads, 128 items of 4000 slots 35.0 and 41.0, 64 of them 26.9 and 31.5, 8
//   19.1 and 22.5; 8 of 2000 17.8 and 17.1 (finding the pieces costs half a microsecond)
//   starts of 0, 4, 8 and 14 places: bf16, 8 heads, 320 items of 1 to 4000 slots 100, 77, 78, 82, all of 4000 143, 142, 143, 145, 240 of 20
//   to 20000, more short ones than long, 194, 133, 134, 136; 4 bits 68, 56, 49, 51; 71, 69, 68, 74; 123, 70, 65, 66
constexpr int kHeldLengths = 8192;
struct Lengths {                         // of the items: in LDS, where there is room
  const DecodeArgs& a;
  const int* s_len;
  __device__ __forceinline__ int operator()(int i) const { return a.items <= kHeldLengths ? s_len[i] : a.s.length(i); }
  __device__ __forceinline__ int tiles(int i) const { return ((*this)(i) + kTile - 1) / kTile; }
};
__device__ __forceinline__ int lanes_sum(int v) { return __builtin_amdgcn_readlane(static_cast<int>(wave_scan(static_cast<uint32_t>(v))), 63); }
// The item that holds unit `at` (of sum over units(i)), and its first unit.
template <class Units>
__device__ __forceinline__ int item_at(int items, const Units& units, int at, int* first) {
  const int lane = threadIdx.x & 63;
  int base = 0;
  for (int i0 = 0;; i0 += 64) {
    const int n = i0 + lane < items ? units(i0 + lane) : 0;
    const int up_to = base + static_cast<int>(wave_scan(static_cast<uint32_t>(n)));
    const uint64_t past = __ballot(up_to > at);
    if (past != 0 || i0 + 64 >= items) {
      const int k = past != 0 ? __builtin_ctzll(past) : 63;
      *first = __builtin_amdgcn_readlane(up_to - n, k);
      return i0 + k;
    }
    base = __builtin_amdgcn_readlane(up_to, 63);
  }
}
// Of a workgroup: its first item; on the line, or within the item where that is cut into `pieces`, the item's first tile and the tiles from
// `at` to `end`.  Nothing to do: at == end.
struct Place {
  int item, first, at, end, share, pieces;
};
constexpr int kTries = 2;                // of a wavefront
__device__ __forceinline__ Place find_place(const DecodeArgs& a, const Lengths& len, uint64_t* s_tries) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int groups = gridDim.x, group = blockIdx.x;
  int sum = 0, some = 0;
  for (int i = lane; i < a.items; i += 64) {
    const int t = len.tiles(i);
    sum += t;
    some += t > 0;
  }
  const int tiles = lanes_sum(sum), total = tiles + a.start * lanes_sum(some);
  Place p{};
  p.share = max(a.least, (tiles + groups - 1) / groups);
  if (a.items <= groups) {
    // shares + 0, 1, 2, 3, 4, 5, 6, 8: two a wavefront
    const auto more = [](int k) { return k + (k == 7); };
    uint32_t size[kTries], pieces[kTries];
#pragma unroll
    for (int k = 0; k < kTries; ++k) {
      size[k] = p.share + more(kTries * wave + k);
      pieces[k] = 0;
    }
    for (int i = lane; i < a.items; i += 64) {
      const uint32_t t = len.tiles(i);
#pragma unroll
      for (int k = 0; k < kTries; ++k) pieces[k] += (t + size[k] - 1) / size[k];
    }
#pragma unroll
    for (int k = 0; k < kTries; ++k) {
      const uint32_t n = lanes_sum(pieces[k]);
      if (lane == 0) s_tries[kTries * wave + k] = n;
    }
    __syncthreads();
    const uint64_t ok = __ballot(lane < 4 * kTries && s_tries[lane & (4 * kTries - 1)] <= static_cast<uint64_t>(groups));
    if (ok != 0) {
      const int k = __builtin_ctzll(ok);
      if (group >= static_cast<int>(s_tries[k])) return p;
      const uint32_t most = p.share + more(k);
      int before;
      p.item = item_at(a.items, [&](int i) { return static_cast<int>((len.tiles(i) + most - 1) / most); }, group, &before);
      const int t = len.tiles(p.item);
      p.pieces = (t + most - 1) / most;
      const int each = t / p.pieces, rest = t % p.pieces, j = group - before;
      p.at = j * each + min(j, rest);
      p.end = p.at + each + (j < rest);
      return p;
    }
  }
  p.share = max(a.least, (total + groups - 1) / groups);
  p.at = group * p.share;
  p.end = max(p.at, min(p.at + p.share, total));
  if (p.at < p.end) {
    p.item = item_at(a.items, [&](int i) { const int t = len.tiles(i); return t > 0 ? t + a.start : 0; }, p.at, &p.first);
    p.first += a.start;                  // where its tiles begin
    p.at = min(max(p.at, p.first), p.end);
  }
  return p;
}

// cap * tanh(s / cap).  Below 0.8 the fifth convergent of Lambert's continued fraction y / (1 + y^2 / (3 + y^2 / (5 + ..))), off by
// less than 1e-8 of its value there; above, 1 - 2 / (e^2y + 1), which would lose the digits of small values.
__device__ __forceinline__ float capped(float s, float cap, float inv_cap) {
  const float y = s * inv_cap, y2 = y * y;
  const float num = __builtin_fmaf(y2, y2 + 105.f, 945.f), den = __builtin_fmaf(y2, __builtin_fmaf(y2, 15.f, 420.f), 945.f);
  const float small = y * num * __builtin_amdgcn_rcpf(den);
  const float large = 1.f - 2.f * __builtin_amdgcn_rcpf(fast_exp2(fabsf(y) * (2.f * kLog2e)) + 1.f);
  return cap * (fabsf(y) < 0.8f ? small : __builtin_copysignf(large, y));
}

// What a segment's wavefronts need to make scores of products.
struct Scoring {
  int n, at;                     // slots in use; the query's position
  int sure;                      // slots whose memory there is: a workgroup that has an item alone begins before it knows n
  int g, sinks, window;
  float cap, inv_cap;
  bool where;                    // positions matter
  const int32_t* pos;            // of the item
  bool biased;
  float slope[8];                // of the item's heads, where biased
  bool tracked;
  float* scores;                 // of the item: [slot][g]
};

// rows of a tile of an item with n
__device__ __forceinline__ int rows_known(const Scoring& sc, int tile, int n) { return __builtin_amdgcn_readfirstlane(max(0, min(n - tile * kTile, kTile))); }
// the position of this lane's slot of a tile that has `rows`; 0 where there is none or positions do not matter
__device__ __forceinline__ int position(const Scoring& sc, int tile, int rows) {
  const auto of = __builtin_amdgcn_make_buffer_rsrc(const_cast<int32_t*>(sc.pos + static_cast<int64_t>(tile) * kTile), 0, sc.where ? rows * 4 : 0, 0x00027000);
  return static_cast<int>(__builtin_amdgcn_raw_buffer_load_b32(of, 4 * (threadIdx.x & 63), 0, 0));
}

// Products q k come over a power of two of the head's, its unit.  With a cap or biases they become scores at once; otherwise that is left until
// probabilities are made of them, or they are kept.
struct NoUnits {                         // all 1
  __device__ __forceinline__ float score(int, int) const { return kRoot; }
  __device__ __forceinline__ float left(int, int) const { return 1.f; }
};
template <int HS>
struct HeadUnits {
  float of[HS][4];                       // of head 4 hs + i, in scalar registers: unit / sqrt(128), or unit if that is left
  bool scored;
  // unit: of the head 4 hs + lane % 4; comes back as what is left
  __device__ __forceinline__ HeadUnits(const Scoring& sc, float (&unit)[HS]) : scored(sc.cap > 0.f || sc.biased) {
#pragma unroll
    for (int hs = 0; hs < HS; ++hs) {
      const int u = __builtin_bit_cast(int, scored ? unit[hs] * kRoot : unit[hs]);
#pragma unroll
      for (int i = 0; i < 4; ++i) of[hs][i] = __builtin_bit_cast(float, __builtin_amdgcn_readlane(u, i));
      if (scored) unit[hs] = 1.f;
    }
  }
  __device__ __forceinline__ float score(int hs, int i) const { return of[hs][i]; }
  __device__ __forceinline__ float left(int hs, int i) const { return scored ? 1.f : of[hs][i]; }
};
// xt: products over the heads' units; comes back as they are, or as scores, -inf where the slot is not seen.  The slots that are.
//   The last factor, DecodeArgs::factor, is for differences from a maximum alone, here and in the merges, so that what is rounded is small where
// the probability is not (8 items of 3700 slots in bf16: outputs 6.4e-7 -> 5.8e-7 off).
template <int HS, class Units>
__device__ __forceinline__ uint64_t score_tile(const Scoring& sc, int tile, int pos, const Units& units, float (&xt)[HS][4]) {
  const int lane = threadIdx.x & 63, row = tile * kTile + lane;
  bool seen = row < sc.n;
  const int away = sc.at - pos;
  if (sc.window > 0) seen = seen && (away < sc.window || pos < sc.sinks);
  if (sc.cap > 0.f || sc.biased) {
#pragma unroll
    for (int hs = 0; hs < HS; ++hs)
#pragma unroll
      for (int i = 0; i < 4; ++i) xt[hs][i] *= units.score(hs, i);
  }
  if (sc.cap > 0.f) {
#pragma unroll
    for (int hs = 0; hs < HS; ++hs)
#pragma unroll
      for (int i = 0; i < 4; ++i) xt[hs][i] = capped(xt[hs][i], sc.cap, sc.inv_cap);
  }
  if (sc.biased) {
#pragma unroll
    for (int hs = 0; hs < HS; ++hs)
#pragma unroll
      for (int i = 0; i < 4; ++i) xt[hs][i] = __builtin_fmaf(-sc.slope[4 * hs + i], static_cast<float>(away), xt[hs][i]);
  }
#pragma unroll
  for (int hs = 0; hs < HS; ++hs)
#pragma unroll
    for (int i = 0; i < 4; ++i) xt[hs][i] = seen ? xt[hs][i] : -INFINITY;
  return __builtin_amdgcn_ballot_w64(seen);
}

// Online softmax of scores x times factor in the lanes (block, head), maxima as the x are; acc: whatever is scaled with the sums
template <int HS>
__device__ __forceinline__ void softmax_step(const float (&x)[HS][4], const float (&factor)[HS], Run<HS>& run, float (&p)[HS][4]) {
#pragma unroll
  for (int hs = 0; hs < HS; ++hs) {
    const float most = max_of_four(x[hs][0], x[hs][1], x[hs][2], x[hs][3]);
    if (__any(most > run.m[hs])) {
      const float m_new = fmaxf(run.m[hs], head_max(most));
      const float alpha = fast_exp2((run.m[hs] - m_new) * factor[hs]);
      run.l[hs] *= alpha;
      const uint32_t au = __builtin_bit_cast(uint32_t, alpha);
      const float ah[4] = {__builtin_bit_cast(float, quad_bcast<0>(au)), __builtin_bit_cast(float, quad_bcast<1>(au)),
                           __builtin_bit_cast(float, quad_bcast<2>(au)), __builtin_bit_cast(float, quad_bcast<3>(au))};
#pragma unroll
      for (int i = 0; i < 4; ++i) {
#pragma unroll
        for (int grp = 0; grp < 4; ++grp) run.acc[hs][grp][i] *= ah[i];
        run.offv[hs][i] *= ah[i];
      }
      run.m[hs] = m_new;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      p[hs][i] = fast_exp2((x[hs][i] - run.m[hs]) * factor[hs]);
      run.l[hs] += p[hs][i];
    }
  }
}

// The end of a wavefront's tiles: maxima without the unit.  A sum is nothing where its maximum is below what an exponent of 2 can be (0 x NaN
// stays NaN).
template <int HS>
__device__ __forceinline__ void end_maxima(const float (&unit)[HS], float factor, Run<HS>& run) {
#pragma unroll
  for (int hs = 0; hs < HS; ++hs) {
    run.m[hs] *= unit[hs];
    run.l[hs] *= run.m[hs] * factor < kLowest ? 0.f : 1.f;
  }
}

// Scores on their way to the weights, which need them once the item's sums are known.  They wait in LDS: where a workgroup has all of an
// item until then, otherwise until a wavefront's part is full, which then goes to the workspace at once.  Writes among the reads of rows
// cost more than their bytes.  4 x 8 items of 128K slots, 4 heads, us, with the launch that joins them: bf16 318 without weights, 401 with a
// store a tile, 391 so; 4 bits 110, 158, 148.  (334 and 126 of them if nothing is written; with waits that count these stores, or with
// non-temporal ones, no less.)
struct Held {
  uint8_t* at;         // of this wavefront: [tiles][64][g]
  int n, most;         // tiles there, and room; most 0: all of the item's stay
  template <int HS, int NWV, class Units>
  __device__ __forceinline__ void put(const Scoring& sc, int tile, bool last, const float (&xt)[HS][4], const Units& units) {
    if (!sc.tracked) return;
    const int lane = threadIdx.x & 63;
    const auto x = [&](int hs, int i) __attribute__((always_inline)) { return units.left(hs, i) * xt[hs][i]; };
    float* dst = reinterpret_cast<float*>(at) + (n * kTile + lane) * sc.g;
    if constexpr (HS == 2) {
      *reinterpret_cast<float4*>(dst) = make_float4(x(0, 0), x(0, 1), x(0, 2), x(0, 3));
      *reinterpret_cast<float4*>(dst + 4) = make_float4(x(1, 0), x(1, 1), x(1, 2), x(1, 3));
    } else {
      if (sc.g == 4) *reinterpret_cast<float4*>(dst) = make_float4(x(0, 0), x(0, 1), x(0, 2), x(0, 3));
      else if (sc.g == 2) *reinterpret_cast<float2*>(dst) = make_float2(x(0, 0), x(0, 1));
      else *dst = x(0, 0);
    }
    ++n;
    if (n == most || (last && most > 0)) {
      const int bytes = kTile * 4 * sc.g;
      wave_lds_sync();
      for (int k = 0; k < n; ++k) {
        uint8_t* to = reinterpret_cast<uint8_t*>(sc.scores + static_cast<int64_t>(tile - (n - 1 - k) * NWV) * kTile * sc.g);
        for (int i = 16 * lane; i < bytes; i += 1024) *reinterpret_cast<uint4*>(to + i) = *reinterpret_cast<const uint4*>(at + k * bytes + i);
      }
      wave_lds_sync();
      n = 0;
    }
  }
};
// of a wavefront in a workgroup of four, two of which share a compute unit's LDS
__host__ __device__ constexpr int held_bytes_of_four(int bits) { return bits == 16 ? 10240 : 16384; }
// behind everything else: the query's rows of two head sets
constexpr int kQueryBytes = 8 * kRowStride;

template <int HS>
__device__ __forceinline__ void init(Run<HS>& run) {
  run.init();
#pragma unroll
  for (int hs = 0; hs < HS; ++hs) run.m[hs] = kLowest;
}

// Sixteen bytes of a tile.  STREAM: non-temporal, so that rows, which a step reads once, do not push scores out of the caches: 4 x 8 items of
// 128K slots in bf16 430 -> 391 us, without weights 361 -> 318 (6.8 TB/s).  Small caches may still be there from the step before: 32 of 2
// items of 1000 slots 16.0 us each with it, 13.3 without, 4 of 32 items of 8K in 4 bits (40 MB) 22.3, 20.8.  The line is at 64 MiB of rows.
// (here(): a value that the compiler sees the loop make, so that constants added to it become the loads' offsets and not registers each.)
__device__ __forceinline__ int here(int x) {
  asm volatile("" : "+v"(x));
  return x;
}
template <bool STREAM, class Buffer>
__device__ __forceinline__ uint4 stream_load(Buffer tile, int at) {
  const auto v = __builtin_amdgcn_raw_buffer_load_b128(tile, at, 0, STREAM ? 2 : 0);
  return make_uint4(v[0], v[1], v[2], v[3]);
}

// ---- bf16 rows ---------------------------------------------------------------------------------------------------------------------

// a probability as three truncated bf16 terms: all of its 24 bits
__device__ __forceinline__ void split_bf16_3(const float (&p)[4], short4v (&t)[3]) {
  float r[4] = {p[0], p[1], p[2], p[3]};
#pragma unroll
  for (int k = 0; k < 3; ++k) {
    uint32_t b[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      b[i] = __float_as_uint(r[i]) & 0xFFFF0000u;
      r[i] -= __uint_as_float(b[i]);
    }
    t[k] = bf4((b[0] >> 16) | b[1], (b[2] >> 16) | b[3]);
  }
}

constexpr int kStageRows = 32, kHalfBytes = kStageRows * kRowStride;      // V rows that a wavefront has in LDS at a time

template <int A, int HS>
__device__ __forceinline__ void pv_rows_step(const uint8_t* s_stage, int lane, const short4v (&t)[HS][3], Run<HS>& run) {
  uint32_t w[4];
#pragma unroll
  for (int k = 0; k < 4; ++k) w[k] = *reinterpret_cast<const uint32_t*>(s_stage + ((4 * A) % kStageRows + k) * kRowStride + 4 * lane);
  const short4v be = bf4(__builtin_amdgcn_perm(w[1], w[0], 0x05040100u), __builtin_amdgcn_perm(w[3], w[2], 0x05040100u));
  const short4v bo = bf4(__builtin_amdgcn_perm(w[1], w[0], 0x07060302u), __builtin_amdgcn_perm(w[3], w[2], 0x07060302u));
#pragma unroll
  for (int hs = 0; hs < HS; ++hs)
#pragma unroll
    for (int k = 0; k < 3; ++k) {
      run.acc[hs][0] = __builtin_amdgcn_mfma_f32_4x4x4bf16_1k(t[hs][k], be, run.acc[hs][0], 4, A, 0);
      run.acc[hs][1] = __builtin_amdgcn_mfma_f32_4x4x4bf16_1k(t[hs][k], bo, run.acc[hs][1], 4, A, 0);
    }
}
template <int A0, int HS, int... A>
__device__ __forceinline__ void pv_rows(const uint8_t* s_stage, int lane, const short4v (&t)[HS][3], Run<HS>& run, std::integer_sequence<int, A...>) {
  (pv_rows_step<A0 + A, HS>(s_stage, lane, t, run), ...);
}

// Tiles t0 .. t1 - 1 of an item, the workgroup's wavefronts in turn.  kd, vd: the item's rows.
// Rows pass through LDS, half a tile at a time, which leaves room there for scores: loads want whole rows, the matrix unit columns of them.
// Scores: v_mfma_f32_16x16x32 has sixteen slots on one side, a lane eight channels of one; four heads on the other, four times over, so
// that every row of lanes has them, and lane 16 b + c takes those of its slot, c of block b.
// P V: lanes want a channel of four slots (decode_rows.h).
template <int HS, int NWV, bool STREAM>
__device__ __forceinline__ void rows_segment(const uint8_t* __restrict__ kd, const uint8_t* __restrict__ vd, const uint16_t* __restrict__ q,
                                             const Scoring& sc, float factor, int t0, int t1, uint8_t* s_stage, uint8_t* s_query, Held& held,
                                             Run<HS>& run) {
  using Bf8 = __attribute__((ext_vector_type(8))) __bf16;
  const int lane = threadIdx.x & 63, j = lane & 3;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int lr = lane >> 4, lc = lane & 15;
  // K and V of a tile in registers of their own, each loaded again right after its last use: two tiles' sides are always on their way.
  // A tile is a buffer that ends with the item's last row, and what is behind it reads as zeros; behind the last tile it is empty.  (With
  // loads under a condition the compiler cannot count on them, and waits for all there are.)
  uint4 kq[16], vq[16];
  const auto tile_at = [&](const uint8_t* base, int t, int rows) __attribute__((always_inline)) {
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(base + static_cast<int64_t>(t) * (kTile * kHeadDim * 2)), 0, rows * (kHeadDim * 2),
                                             0x00027000);
  };
  const auto load_tile = [&](uint4 (&st)[16], const uint8_t* base, int t, int rows) __attribute__((always_inline)) {
    const auto tile = tile_at(base, t, rows);
    const int at = here(lane * 16);
#pragma unroll
    for (int i = 0; i < 16; ++i) st[i] = stream_load<STREAM>(tile, at + i * 1024);
  };
  const auto store_half = [&](const uint4 (&st)[16], int half) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < 8; ++i) *reinterpret_cast<uint4*>(s_stage + (4 * i + lr) * kRowStride + 16 * lc) = st[8 * half + i];
  };
  // The query: head 4 hs + lane % 4, channels 32 i + 8 (lane / 16) ..  Two head sets' would take the registers of a wavefront with two
  // tiles' sides, and are in LDS.
  constexpr bool kQueryInLds = HS == 2;
  uint4 qa[HS][4];
  const auto query = [&](int hs, int i) __attribute__((always_inline)) {
    return 4 * hs + j < sc.g ? *reinterpret_cast<const uint4*>(q + (4 * hs + j) * kHeadDim + 32 * i + 8 * lr) : make_uint4(0, 0, 0, 0);
  };
  uint4 q_row;
  if constexpr (kQueryInLds) {
    if (threadIdx.x < 128) q_row = *reinterpret_cast<const uint4*>(q + 8 * threadIdx.x);
  } else {
#pragma unroll
    for (int hs = 0; hs < HS; ++hs)
#pragma unroll
      for (int i = 0; i < 4; ++i) qa[hs][i] = query(hs, i);
  }
  const int first_rows = rows_known(sc, t0 + wave, sc.sure);
  int pos = position(sc, t0 + wave, first_rows);
  load_tile(kq, kd, t0 + wave, first_rows);
  load_tile(vq, vd, t0 + wave, first_rows);
  __builtin_amdgcn_sched_barrier(0);
  // the query is here before the loop: waited for inside, it would have every pass wait for all loads under way
  if constexpr (kQueryInLds) {
    if (threadIdx.x < 128) *reinterpret_cast<uint4*>(s_query + (threadIdx.x >> 4) * kRowStride + 16 * (threadIdx.x & 15)) = q_row;
    __syncthreads();
  } else {
#pragma unroll
    for (int hs = 0; hs < HS; ++hs)
#pragma unroll
      for (int i = 0; i < 4; ++i) asm volatile("" : "+v"(qa[hs][i].x), "+v"(qa[hs][i].y), "+v"(qa[hs][i].z), "+v"(qa[hs][i].w));
  }
  const floatx4 zero4 = {0.f, 0.f, 0.f, 0.f};
  float all[HS], ones[HS];
#pragma unroll
  for (int hs = 0; hs < HS; ++hs) {
    all[hs] = factor;
    ones[hs] = 1.f;
  }
  for (int tile = t0 + wave; tile < t1; tile += NWV) {
    const int next = tile + NWV, next_rows = next < t1 ? rows_known(sc, next, sc.n) : 0;
    float xt[HS][4], x[HS][4];
    const int pos_now = pos;
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      store_half(kq, half);
      if (half == 1) {
        __builtin_amdgcn_sched_barrier(0);     // (the next rows into the same registers)
        pos = position(sc, next, next_rows);
        load_tile(kq, kd, next, next_rows);
      }
      wave_lds_sync();
      floatx4 d[2][HS];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        uint4 k[2];
#pragma unroll
        for (int b = 0; b < 2; ++b) k[b] = *reinterpret_cast<const uint4*>(s_stage + (16 * b + lc) * kRowStride + 64 * i + 16 * lr);
#pragma unroll
        for (int hs = 0; hs < HS; ++hs) {
          if constexpr (kQueryInLds) qa[hs][i] = *reinterpret_cast<const uint4*>(s_query + (4 * hs + j) * kRowStride + 64 * i + 16 * lr);
#pragma unroll
          for (int b = 0; b < 2; ++b)
            d[b][hs] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(Bf8, qa[hs][i]), __builtin_bit_cast(Bf8, k[b]), i == 0 ? zero4 : d[b][hs], 0, 0, 0);
        }
      }
      wave_lds_sync();
#pragma unroll
      for (int hs = 0; hs < HS; ++hs)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float v = (lr & 1) ? d[1][hs][i] : d[0][hs][i];
          xt[hs][i] = half == 0 || !(lr & 2) ? (half == 0 ? v : xt[hs][i]) : v;
        }
    }
    const uint64_t seen = score_tile<HS>(sc, tile, pos_now, NoUnits(), xt);
    held.put<HS, NWV>(sc, tile, next >= t1, xt, NoUnits());
    to_head_lanes<HS, HS == 2>(xt, j, x);
    float p[HS][4];
    softmax_step<HS>(x, all, run, p);
    short4v t[HS][3];
#pragma unroll
    for (int hs = 0; hs < HS; ++hs) split_bf16_3(p[hs], t[hs]);
    if (seen != ~0ull) {                // rows that are not seen may hold anything: 0 x NaN
#pragma unroll
      for (int i = 0; i < 16; ++i)
        if (!((seen >> (4 * i + lr)) & 1)) vq[i] = make_uint4(0, 0, 0, 0);
    }
    store_half(vq, 0);
    wave_lds_sync();
    pv_rows<0, HS>(s_stage, lane, t, run, std::make_integer_sequence<int, 8>{});
    wave_lds_sync();
    store_half(vq, 1);
    __builtin_amdgcn_sched_barrier(0);
    load_tile(vq, vd, next, next_rows);
    wave_lds_sync();
    pv_rows<8, HS>(s_stage, lane, t, run, std::make_integer_sequence<int, 8>{});
    wave_lds_sync();                    // before the next rows overwrite the region
  }
  end_maxima<HS>(ones, factor, run);
}

// ---- 4-bit rows --------------------------------------------------------------------------------------------------------------------
// (operand layouts and the codes as fp16 subnormals: decode_mfma_kernels.hip)

// The four codes of step S of a group's words as fp16 numbers code 2^-18: subnormals with the code's highest bit in the mantissa's.
// (As code 2^-24, one AND less in two, they cost precision: the matrix unit lines up a product by its operands' exponents, a
// subnormal's being the lowest whatever zeros it starts with, and cuts the sum off 24 bits below; the products of codes 2^-24 left
// the accumulators 18 bits.)
__device__ __forceinline__ half4 code_operand(const uint4& gw, int s) {
  constexpr uint32_t kMask = 0x03C003C0u;
  const uint32_t w0 = s < 4 ? gw.x : gw.z, w1 = s < 4 ? gw.y : gw.w;
  Pack4 r;
  switch (s & 3) {
    case 0: r.u[0] = (w0 << 6) & kMask; r.u[1] = (w1 << 6) & kMask; break;
    case 1: r.u[0] = (w0 << 2) & kMask; r.u[1] = (w1 << 2) & kMask; break;
    case 2: r.u[0] = (w0 >> 2) & kMask; r.u[1] = (w1 >> 2) & kMask; break;
    default: r.u[0] = (w0 >> 6) & kMask; r.u[1] = (w1 >> 6) & kMask; break;
  }
  return r.h;
}
constexpr float kCode = 262144.0f;       // 2^18

// V codes less 8: in the mantissa of 1024 or 64, from which 1032 or 72 is taken.  A value is then scale x (code - 8) + (offset + 8 scale), whose
// terms are about as large as the value.  (With scale x code + offset the sums of P V are differences of two sums many times as large:
// 4 x 8 items of 90K to 128K slots 3.0e-6 of the outputs' norm off, 1.0e-6 so, for 1 to 3 % more time.  Scores, differences of single products' sums, gain
// nothing by it.)
struct Ones {                            // 1024 and 64 twice, in registers: an instruction takes one constant, the mask
  uint32_t thousand = 0x64006400u, sixty = 0x54005400u;
  __device__ __forceinline__ Ones() { asm volatile("" : "+v"(thousand), "+v"(sixty)); }
};
__device__ __forceinline__ half4 centred_operand(const uint4& gw, int s, const Ones& ones) {
  uint32_t w0 = s < 4 ? gw.x : gw.z, w1 = s < 4 ? gw.y : gw.w;
  if (s & 2) {
    w0 >>= 8;
    w1 >>= 8;
  }
  const uint32_t mask = s & 1 ? 0x00F000F0u : 0x000F000Fu, one = s & 1 ? ones.sixty : ones.thousand;
  const half2v down = s & 1 ? half2v{-72, -72} : half2v{-1032, -1032};
  Pack4 r;
  r.p[0] = __builtin_bit_cast(half2v, (w0 & mask) | one) + down;
  r.p[1] = __builtin_bit_cast(half2v, (w1 & mask) | one) + down;
  return r.h;
}

// two numbers as fp16 pairs whose sums they are, to 22 bits, rounded to nearest (cut off they were low by 2^-21 on average, which the
// codes' sum and the offsets' do not share)
typedef float float2v __attribute__((ext_vector_type(2)));
__device__ __forceinline__ void split_halves(float a, float b, half2v& hi, half2v& lo) {
  hi = __builtin_convertvector((float2v{a, b}), half2v);
  lo = __builtin_convertvector((float2v{a - static_cast<float>(hi[0]), b - static_cast<float>(hi[1])}), half2v);
}

// offset + 8 scale of four pairs
__device__ __forceinline__ void centres(uint32_t s01, uint32_t s23, uint32_t m01, uint32_t m23, Pack4& hi, Pack4& lo) {
  const uint32_t sc[2] = {s01, s23}, of[2] = {m01, m23};
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const half2v a = __builtin_bit_cast(half2v, sc[i]), b = __builtin_bit_cast(half2v, of[i]);
    split_halves(__builtin_fmaf(8.f, static_cast<float>(a[0]), static_cast<float>(b[0])), __builtin_fmaf(8.f, static_cast<float>(a[1]), static_cast<float>(b[1])),
                 hi.p[i], lo.p[i]);
  }
}

constexpr int kQUp = 8;                  // a head's largest query value is near 2^kQUp
constexpr int kPUp = 15;                 // probabilities go into fp16 terms times 2^kPUp.  (Not through the exponentials: x - m + 15 has four bits
                                         // less behind the point than x - m near 0, 5e-7 of a probability)

constexpr float kPScale = 1 << kPUp;
__device__ __forceinline__ int exponent_of(float x) {      // of a number > 0; bounds for the others
  return static_cast<int>((__float_as_uint(x) >> 23) & 255u) - 127;
}

template <int HS, int NWV, bool STREAM>
__device__ __forceinline__ float tiles_segment(const uint8_t* __restrict__ kd, const uint8_t* __restrict__ vd, const uint16_t* __restrict__ q,
                                               const Scoring& sc, float factor, int t0, int t1, Held& held, Run<HS>& run) {
  const int lane = threadIdx.x & 63, blk = lane >> 2, j = lane & 3;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  uint4 qraw[HS];
#pragma unroll
  for (int hs = 0; hs < HS; ++hs) qraw[hs] = load_query(q, 4 * hs + j, sc.g, blk);
  uint4 kr[4], vr[4], kmeta, vmeta;
  int pos;
  // (as in rows_segment: a tile that is there, or an empty one)
  auto load_k = [&](int t, int rows) __attribute__((always_inline)) {
    const auto tile = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(kd + static_cast<int64_t>(t) * kTileBytes), 0, rows > 0 ? kTileBytes : 0, 0x00027000);
    const int at = here(lane * 16);
#pragma unroll
    for (int i = 0; i < 4; ++i) kr[i] = stream_load<STREAM>(tile, at + 1024 * i);
    kmeta = stream_load<STREAM>(tile, at + 4096);
    pos = position(sc, t, rows);
  };
  auto load_v = [&](int t, int rows) __attribute__((always_inline)) {
    const auto tile = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(vd + static_cast<int64_t>(t) * kTileBytes), 0, rows > 0 ? kTileBytes : 0, 0x00027000);
    const int at = here(lane * 16);
    vmeta = stream_load<STREAM>(tile, at + 4096);
#pragma unroll
    for (int i = 0; i < 4; ++i) vr[i] = stream_load<STREAM>(tile, at + 1024 * i);
  };
  load_k(t0 + wave, rows_known(sc, t0 + wave, sc.sure));
  load_v(t0 + wave, rows_known(sc, t0 + wave, sc.sure));

  // ---- query operands: times the power of two that puts a head's largest value near 2^kQUp ------------------------------
  // (What is 2^22 smaller has fewer digits there, what is 2^33 smaller none: 2^-33 of the largest value, as far as its own products in fp32
  // go.)
  half4 qop[HS][2], qhi[HS], qlo[HS];
  float unit[HS];
#pragma unroll
  for (int hs = 0; hs < HS; ++hs) {
    float most = 0.f;
    const uint32_t w[4] = {qraw[hs].x, qraw[hs].y, qraw[hs].z, qraw[hs].w};
#pragma unroll
    for (int k = 0; k < 4; ++k)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const uint32_t u = (e == 0 ? w[k] << 16 : w[k] & 0xFFFF0000u) & 0x7FFFFFFFu;
        most = fmaxf(most, u < 0x7F800000u ? __uint_as_float(u) : 0.f);
      }
    const int up = max(-120, min(120, kQUp - exponent_of(head_max(most))));
    unit[hs] = ldexpf(1.0f, -up);
    float v[8];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      v[2 * k] = __uint_as_float(w[k] << 16);
      v[2 * k + 1] = __uint_as_float(w[k] & 0xFFFF0000u);
    }
    float psum = 0.f;
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      v[k] = ldexpf(v[k], up);
      psum += v[k];
    }
#pragma unroll
    for (int e = 0; e < 2; ++e)
      qop[hs][e] = half4{static_cast<_Float16>(v[4 * e]), static_cast<_Float16>(v[4 * e + 1]), static_cast<_Float16>(v[4 * e + 2]),
                         static_cast<_Float16>(v[4 * e + 3])};
    psum += dpp_f32<0x124>(psum);
    psum += dpp_f32<0x128>(psum);
    float s0 = psum, s1 = psum;          // rows 0 .. 3 of 16 lanes = groups 0 .. 3: every lane gets all four
    swap_rows(s0, s1);
    float s2 = s0, s3 = s1;
    swap_halves(s0, s2);
    swap_halves(s1, s3);
    const float sg[4] = {s0, s1, s2, s3};
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      qhi[hs][k] = static_cast<_Float16>(sg[k]);
      qlo[hs][k] = static_cast<_Float16>(sg[k] - static_cast<float>(qhi[hs][k]));
    }
  }
  const Ones ones;
  int ve = -126;                         // exponent of the largest V scale so far
  float vf = 0.f;                        // what p is multiplied by for it
  const floatx4 zero4 = {0.f, 0.f, 0.f, 0.f};
  const HeadUnits<HS> units(sc, unit);
  float all[HS];
#pragma unroll
  for (int hs = 0; hs < HS; ++hs) all[hs] = unit[hs] * factor;

  for (int tile = t0 + wave; tile < t1; tile += NWV) {
    const int next = tile + NWV, next_rows = next < t1 ? rows_known(sc, next, sc.n) : 0;
    float xt[HS][4], x[HS][4];
    const int pos_now = pos;
    {
      Pack4 boff;
      boff.u[0] = kmeta.z;
      boff.u[1] = kmeta.w;
#pragma unroll
      for (int hs = 0; hs < HS; ++hs) {
        floatx4 d = __builtin_amdgcn_mfma_f32_4x4x4f16(qhi[hs], boff.h, zero4, 0, 0, 0);
        d = __builtin_amdgcn_mfma_f32_4x4x4f16(qlo[hs], boff.h, d, 0, 0, 0);
#pragma unroll
        for (int i = 0; i < 4; ++i) xt[hs][i] = d[i];
      }
#define RDKV_K_STEP(G_, S_)                                                                                        \
  {                                                                                                               \
    const half4 b = code_operand(gw, S_);                                                                      \
    _Pragma("unroll") for (int hs = 0; hs < HS; ++hs)                                                             \
        dg[hs] = __builtin_amdgcn_mfma_f32_4x4x4f16(qop[hs][(S_) & 1], b, dg[hs], 4, (G_) * 4 + (S_) / 2, 0);     \
  }
#define RDKV_K_GROUP(G_)                                                                                           \
  {                                                                                                               \
    \
    const uint4 gw = kr[G_];                                                                                      \
    floatx4 dg[HS];                                                                                               \
    _Pragma("unroll") for (int hs = 0; hs < HS; ++hs) dg[hs] = zero4;                                             \
    RDKV_K_STEP(G_, 0) RDKV_K_STEP(G_, 1) RDKV_K_STEP(G_, 2) RDKV_K_STEP(G_, 3)                                   \
    RDKV_K_STEP(G_, 4) RDKV_K_STEP(G_, 5) RDKV_K_STEP(G_, 6) RDKV_K_STEP(G_, 7)                                   \
    const float sf = kCode * static_cast<float>(__builtin_bit_cast(half2v, (G_) < 2 ? kmeta.x : kmeta.y)[(G_) & 1]); \
    _Pragma("unroll") for (int hs = 0; hs < HS; ++hs)                                                             \
      _Pragma("unroll") for (int i = 0; i < 4; ++i) xt[hs][i] = __builtin_fmaf(sf, dg[hs][i], xt[hs][i]);         \
  }
      RDKV_K_GROUP(0) RDKV_K_GROUP(1) RDKV_K_GROUP(2) RDKV_K_GROUP(3)
#undef RDKV_K_GROUP
#undef RDKV_K_STEP
    }
    load_k(next, next_rows);
    const uint64_t seen = score_tile<HS>(sc, tile, pos_now, units, xt);
    held.put<HS, NWV>(sc, tile, next >= t1, xt, units);
    to_head_lanes<HS, HS == 2>(xt, j, x);
    float p[HS][4];
    softmax_step<HS>(x, all, run, p);

    // ---- P V ---------------------------------------------------------------------------------------------------------
    uint4 vm = vmeta;
    if (seen != ~0ull) {                 // scales and offsets of rows that are not seen may be anything
      const uint32_t four = static_cast<uint32_t>(seen >> (4 * blk)) & 15u;
      const uint32_t lo = ((four & 1u) ? 0xFFFFu : 0u) | ((four & 2u) ? 0xFFFF0000u : 0u);
      const uint32_t hi = ((four & 4u) ? 0xFFFFu : 0u) | ((four & 8u) ? 0xFFFF0000u : 0u);
      vm = make_uint4(vm.x & lo, vm.y & hi, vm.z & lo, vm.w & hi);
    }
    {
      // a scale above all before: everything gathered so far goes down by as much
      const half2v a = __builtin_bit_cast(half2v, vm.x), c = __builtin_bit_cast(half2v, vm.y);
      const float most = fmaxf(fmaxf(static_cast<float>(a[0]), static_cast<float>(a[1])), fmaxf(static_cast<float>(c[0]), static_cast<float>(c[1])));
      if (__any(most >= ldexpf(1.0f, ve + 1))) {
        const int e = __builtin_amdgcn_readfirstlane(max(ve, min(16, exponent_of(wave_max(most)))));
        const float down = ldexpf(1.0f, ve - e);
#pragma unroll
        for (int hs = 0; hs < HS; ++hs)
#pragma unroll
          for (int grp = 0; grp < 4; ++grp)
#pragma unroll
            for (int i = 0; i < 4; ++i) run.acc[hs][grp][i] *= down;
        ve = e;
        vf = ldexpf(1.0f, kPUp - 1 - ve);
      }
    }
    Pack4 ch, cl;
    centres(vm.x, vm.y, vm.z, vm.w, ch, cl);
#pragma unroll
    for (int hs = 0; hs < HS; ++hs) {
      Pack4 hi, lo;
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        split_halves(p[hs][2 * i] * kPScale, p[hs][2 * i + 1] * kPScale, hi.p[i], lo.p[i]);
      }
      run.offv[hs] = __builtin_amdgcn_mfma_f32_4x4x4f16(hi.h, ch.h, run.offv[hs], 0, 0, 0);
      run.offv[hs] = __builtin_amdgcn_mfma_f32_4x4x4f16(lo.h, ch.h, run.offv[hs], 0, 0, 0);
      run.offv[hs] = __builtin_amdgcn_mfma_f32_4x4x4f16(hi.h, cl.h, run.offv[hs], 0, 0, 0);
#pragma unroll
      for (int i = 0; i < 4; ++i) p[hs][i] *= vf;
    }
// (two channel groups side by side: a product waits for the one before it on the same accumulator)
#define RDKV_PV_STEP(G_, A_)                                                                                              \
  {                                                                                                                       \
    const half4 b0 = centred_operand(vr[G_], A_, ones), b1 = centred_operand(vr[G_ + 1], A_, ones);                       \
    _Pragma("unroll") for (int hs = 0; hs < HS; ++hs) {                                                                   \
      run.acc[hs][G_] = __builtin_amdgcn_mfma_f32_4x4x4f16(hi[hs][0].h, b0, run.acc[hs][G_], 3, A_, 0);                   \
      run.acc[hs][G_ + 1] = __builtin_amdgcn_mfma_f32_4x4x4f16(hi[hs][1].h, b1, run.acc[hs][G_ + 1], 3, A_, 0);           \
      run.acc[hs][G_] = __builtin_amdgcn_mfma_f32_4x4x4f16(lo[hs][0].h, b0, run.acc[hs][G_], 3, A_, 0);                   \
      run.acc[hs][G_ + 1] = __builtin_amdgcn_mfma_f32_4x4x4f16(lo[hs][1].h, b1, run.acc[hs][G_ + 1], 3, A_, 0);           \
    }                                                                                                                     \
  }
#define RDKV_PV_GROUPS(G_)                                                                                                \
  {                                                                                                                       \
    Pack4 sv[2], hi[HS][2], lo[HS][2];                                                                                    \
    sv[0].u[0] = quad_bcast<G_>(vm.x); sv[0].u[1] = quad_bcast<G_>(vm.y);                                                 \
    sv[1].u[0] = quad_bcast<G_ + 1>(vm.x); sv[1].u[1] = quad_bcast<G_ + 1>(vm.y);                                         \
    _Pragma("unroll") for (int hs = 0; hs < HS; ++hs)                                                                     \
      _Pragma("unroll") for (int k = 0; k < 2; ++k)                                                                       \
        _Pragma("unroll") for (int i = 0; i < 2; ++i)                                                                     \
          split_halves(p[hs][2 * i] * static_cast<float>(sv[k].p[i][0]), p[hs][2 * i + 1] * static_cast<float>(sv[k].p[i][1]), \
                       hi[hs][k].p[i], lo[hs][k].p[i]);                                                                   \
    RDKV_PV_STEP(G_, 0) RDKV_PV_STEP(G_, 1) RDKV_PV_STEP(G_, 2) RDKV_PV_STEP(G_, 3)                                       \
    RDKV_PV_STEP(G_, 4) RDKV_PV_STEP(G_, 5) RDKV_PV_STEP(G_, 6) RDKV_PV_STEP(G_, 7)                                       \
  }
    RDKV_PV_GROUPS(0) RDKV_PV_GROUPS(2)
#undef RDKV_PV_GROUPS
#undef RDKV_PV_STEP
    load_v(next, next_rows);
  }
  end_maxima<HS>(unit, factor, run);
  return ldexpf(1.0f, 1 + ve - kPUp);    // what brings the accumulators to the sums' scale, vf's inverse
}

// ---- the end of a piece --------------------------------------------------------------------------------------------------------------

// LDS of the wavefronts' merge, floats: per wavefront, head and channel group (maximum, sum, offset sum, -), then the sums [wave][g][128];
// then the heads' maxima and sums' inverses for the weights.
template <int NWV, int HS>
constexpr int ml_floats() { return ml_lds_floats(NWV, HS); }
constexpr int kHeadFloats = 16;          // of up to eight heads
// What a head's probabilities are made of.  (By the difference from a log-sum-exp they would be off by its rounding, the same way in all slots:
// 4e-5 at scores of 1e3.)  Where nothing is seen the inverse is 0, and every probability.
struct HeadSum {
  float top, inv;
  __device__ __forceinline__ static HeadSum of(float m, float l) { return {m, l == 0.f ? 0.f : 1.0f / l}; }
  __device__ __forceinline__ float add(float p, float x, float factor) const { return __builtin_fmaf(fast_exp2((x - top) * factor), inv, p); }
};
static_assert(sizeof(HeadSum) * 8 == kHeadFloats * sizeof(float), "two a head");

// What a thread adds to the weights of its slots: their scores and weights are loaded before the heads' sums are known.
// EACH slots, `step` apart.
template <int G, int EACH>
struct WeightPart {
  static constexpr int kWide = G < 4 ? G : 4;
  using Wide = __attribute__((ext_vector_type(kWide))) float;
  Wide x[EACH][G / kWide];
  float w[EACH];
  // slots i0, i0 + step, ..; the loads stay below `end`, a slot at least there is
  __device__ __forceinline__ void load(const float* __restrict__ scores, const float* __restrict__ weight, int i0, int step, int end) {
#pragma unroll
    for (int k = 0; k < EACH; ++k) {
      const int i = min(i0 + k * step, end - 1);
#pragma unroll
      for (int h = 0; h < G / kWide; ++h) x[k][h] = *reinterpret_cast<const Wide*>(scores + static_cast<int64_t>(i) * G + h * kWide);
      w[k] = weight[i];
    }
  }
  __device__ __forceinline__ void store(float* __restrict__ weight, float decay, float factor, const HeadSum* sums, int i0, int step, int end) const {
    HeadSum of[G];
#pragma unroll
    for (int h = 0; h < G; ++h) of[h] = sums[h];
#pragma unroll
    for (int k = 0; k < EACH; ++k) {
      float p = 0.f;
#pragma unroll
      for (int h = 0; h < G; ++h) p = of[h].add(p, x[k][h / kWide][h % kWide], factor);
      if (i0 + k * step < end) weight[i0 + k * step] = __builtin_fmaf(decay, w[k], p);
    }
  }
};
template <int G>
__device__ __forceinline__ void add_weights(const DecodeArgs& a, int64_t item, const float* scores, const HeadSum* sums, int n, int thread, int threads) {
  constexpr int kEach = G == 8 ? 2 : 4;
  float* weight = a.s.weight + item * a.s.capacity;
  for (int i = thread; i < n; i += kEach * threads) {
    WeightPart<G, kEach> part;
    part.load(scores, weight, i, threads, n);
    part.store(weight, a.s.decay, a.factor, sums, i, threads, n);
  }
}

// The same from scores that a wavefront has kept: tiles wave, wave + NWV, .. of an item.
template <int NWV>
__device__ __forceinline__ void held_weights(const Args& a, int64_t item, int n, int t0, float (&w)[4]) {      // of tiles t0, t0 + NWV, .. of n > 0 slots
#pragma unroll
  for (int j = 0; j < 4; ++j) w[j] = a.weight[item * a.capacity + min((t0 + j * NWV) * kTile + static_cast<int>(threadIdx.x & 63), n - 1)];
}
// w: held_weights of the first tiles
template <int HS, int NWV>
__device__ __forceinline__ void add_held(const DecodeArgs& a, int64_t item, const float* s_held, const HeadSum* sums, int n, int wave, int tiles, float (&w)[4]) {
  const int lane = threadIdx.x & 63, g = a.s.g;
  float* __restrict__ weight = a.s.weight + item * a.s.capacity;
  HeadSum of[4 * HS];
#pragma unroll
  for (int h = 0; h < 4 * HS; ++h) of[h] = sums[h < g ? h : 0];
  for (int t0 = wave, k = 0; t0 < tiles; t0 += 4 * NWV, k += 4) {
    if (k > 0) held_weights<NWV>(a.s, item, n, t0, w);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int i = (t0 + j * NWV) * kTile + lane;
      if (i >= n) break;
      const float* x = s_held + ((k + j) * kTile + lane) * g;
      float p = 0.f;
#pragma unroll
      for (int h = 0; h < 4 * HS; ++h)
        if (HS == 2 || h < g) p = of[h].add(p, x[h], a.factor);
      weight[i] = __builtin_fmaf(a.s.decay, w[j], p);
    }
  }
}

// natural log-sum-exp of a head
__device__ __forceinline__ float log_sum(const DecodeArgs& a, float m, float l) {
  return l == 0.f ? -INFINITY : __builtin_fmaf(m, a.natural, __log2f(l) * kLn2);
}

template <int BITS, int HS, int NWV, bool STREAM>
__global__ __launch_bounds__(NWV * 64, BITS == 16 || HS == 2 ? 2 : 3) void decode_kernel(DecodeArgs a) {
  extern __shared__ __align__(16) uint8_t smem[];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int g = a.s.g;
  // what this workgroup has; one of eight wavefronts has its item
  Place p{};
  p.item = blockIdx.x;
  if constexpr (NWV == 4) {
    int* s_len = reinterpret_cast<int*>(smem);
    if (a.items <= kHeldLengths) {
#pragma unroll 8
      for (int i = tid; i < a.items; i += NWV * 64) s_len[i] = a.s.length(i);
      __syncthreads();
    }
    const Lengths len{a, s_len};
    // items without a token have no tile: their outputs are the first workgroups' to write
    for (int i = blockIdx.x; i < a.items; i += gridDim.x)
      if (len(i) == 0) {
        for (int k = tid; k < g * kHeadDim; k += NWV * 64) a.out[static_cast<int64_t>(i) * g * kHeadDim + k] = 0.f;
        if (a.lse != nullptr && tid < g) a.lse[static_cast<int64_t>(i) * g + tid] = -INFINITY;
        if (tid == 0) a.parts[i] = make_int2(0, 0);
      }
    p = find_place(a, len, reinterpret_cast<uint64_t*>(s_len + kHeldLengths));
    if (p.at == p.end) return;
    __syncthreads();
  }
  int item = p.item, first = p.first, at = p.at;
  // LDS: the wavefronts' staging regions; their scores; the accumulators' area [NWV][g][128], which is the staging regions' memory, or the
  // scores' unless they are kept; the wavefronts' maxima and sums, and the heads'
  constexpr bool kKeep = NWV == 8, kOwnAcc = BITS == 4 && kKeep;
  const int held_bytes = kKeep ? a.held_bytes : held_bytes_of_four(BITS);
  uint8_t* s_stage = smem + wave * kHalfBytes;
  uint8_t* s_held = smem + (BITS == 16 ? NWV * kHalfBytes : 0);
  uint8_t* s_end = s_held + NWV * held_bytes;
  float* s_acc = reinterpret_cast<float*>(kOwnAcc ? s_end : smem);
  float* s_ml = reinterpret_cast<float*>(s_end) + (kOwnAcc ? NWV * g * kHeadDim : 0);
  HeadSum* s_sums = reinterpret_cast<HeadSum*>(s_ml + ml_floats<NWV, HS>());
  do {
    // (all the same for every lane, which buffers need to be known of)
    item = __builtin_amdgcn_readfirstlane(item);
    const int n = __builtin_amdgcn_readfirstlane(a.s.length(item)), tiles = (n + kTile - 1) / kTile;
    const int t0 = __builtin_amdgcn_readfirstlane(at - first), t1 = NWV == 8 ? tiles : __builtin_amdgcn_readfirstlane(min(tiles, p.end - first));
    if (NWV == 4 && t1 <= t0) {          // an item without tiles
      ++item;
      continue;
    }
    const bool whole = NWV == 8 || (t0 == 0 && t1 == tiles);
    if (NWV == 4 && t0 == 0 && tid == 0)
      a.parts[item] = whole ? make_int2(0, 0)
                            : make_int2(static_cast<int>(blockIdx.x) + item, p.pieces > 0 ? p.pieces : (first + tiles - 1) / p.share - static_cast<int>(blockIdx.x) + 1);
    Scoring sc;
    sc.n = n;
    sc.sure = NWV == 8 ? a.s.capacity : n;
    sc.g = g;
    sc.sinks = a.s.sinks;
    sc.window = a.s.window;
    sc.cap = a.s.cap;
    sc.inv_cap = a.s.cap > 0.f ? 1.0f / a.s.cap : 0.f;
    sc.where = a.s.window > 0 || a.s.slopes != nullptr;
    sc.pos = a.s.pos + static_cast<int64_t>(item) * a.s.capacity;
    sc.biased = a.s.slopes != nullptr;
    typedef const __attribute__((address_space(4))) int32_t* ConstInts;      // (scalar loads, which no wait for rows waits for)
    sc.at = ((ConstInts)(a.s.next))[item] - 1;
    if (sc.biased) {
      typedef const __attribute__((address_space(4))) float* ConstFloats;
      const ConstFloats slopes = (ConstFloats)(a.s.slopes) + (item % a.s.hkv) * g;
#pragma unroll
      for (int h = 0; h < 4 * HS; ++h) sc.slope[h] = slopes[min(h, g - 1)];
    }
    sc.tracked = a.s.weight != nullptr;
    sc.scores = a.scores + static_cast<int64_t>(item) * g * a.score_rows;
    const uint16_t* q = a.q + static_cast<int64_t>(item) * g * kHeadDim;
    Run<HS> run;
    init(run);
    float scale = 1.f;
    Held held{s_held + wave * held_bytes, 0, kKeep ? 0 : held_bytes / (kTile * 4 * g)};
    if constexpr (BITS == 16) {
      const int64_t base = static_cast<int64_t>(item) * a.s.capacity * (kHeadDim * 2);
      rows_segment<HS, NWV, STREAM>(a.s.k + base, a.s.v + base, q, sc, a.factor, t0, t1, s_stage, reinterpret_cast<uint8_t*>(s_sums + 8), held, run);
    } else {
      const int64_t base = static_cast<int64_t>(item) * a.s.tiles * kTileBytes;
      scale = tiles_segment<HS, NWV, STREAM>(a.s.k + base, a.s.v + base, q, sc, a.factor, t0, t1, held, run);
    }
    float w_first[4];
    if (kKeep && n > 0 && a.s.weight != nullptr) held_weights<NWV>(a.s, item, n, wave, w_first);
    if constexpr (!kOwnAcc) __syncthreads();      // staging regions or scores become the accumulators' area
    // ---- the wavefronts' results into LDS ------------------------------------------------------------------------------
#pragma unroll
    for (int hs = 0; hs < HS; ++hs) {
      run.l[hs] = head_sum(run.l[hs]);
      float off = 0.f;
      if constexpr (BITS == 4) {         // lanes (block, j): head i's sum of p m of group j over the block's tokens
        float o[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) o[i] = run.offv[hs][i];
        swap_rows(o[0], o[1]);
        swap_rows(o[2], o[3]);
        float lo = o[0] + o[1], hi = o[2] + o[3];
        swap_halves(lo, hi);
        off = lo + hi;
        off += dpp_f32<0x124>(off);
        off += dpp_f32<0x128>(off);
        if ((lane & 12) == 0) s_ml[ml_at<HS>(wave, 4 * hs + (lane >> 4), lane & 3) + 2] = off * (1.0f / kPScale);
      }
      if (lane < 16) {                   // (block, j) -> group block of head j
        float* ml = s_ml + ml_at<HS>(wave, 4 * hs + (lane & 3), lane >> 2);
        *reinterpret_cast<float2*>(ml) = make_float2(run.m[hs], run.l[hs]);
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int head = 4 * hs + i;
        float* dst = s_acc + (wave * g + head) * kHeadDim;
        if constexpr (BITS == 16) {
          if (head < g) *reinterpret_cast<float2*>(dst + 2 * lane) = make_float2(run.acc[hs][0][i], run.acc[hs][1][i]);
        } else {
          const float v0 = halves_sum(run.acc[hs][0][i], run.acc[hs][1][i]), v1 = halves_sum(run.acc[hs][2][i], run.acc[hs][3][i]);
          if (head < g) {
            dst[lane] = v0 * scale;
            dst[64 + lane] = v1 * scale;
          }
        }
      }
    }
    __syncthreads();
    // ---- a wavefront per head adds them up -----------------------------------------------------------------------------
    const int64_t qh0 = static_cast<int64_t>(item) * g, slot = static_cast<int64_t>(blockIdx.x) + item;
    for (int head = wave; head < g; head += NWV) {
      const int ch = 2 * lane;
      float mm = kLowest;
#pragma unroll
      for (int w = 0; w < NWV; ++w) mm = fmaxf(mm, s_ml[ml_at<HS>(w, head, 0)]);
      float l = 0.f, v0 = 0.f, v1 = 0.f;
#pragma unroll
      for (int w = 0; w < NWV; ++w) {
        const float2 ml = *reinterpret_cast<const float2*>(s_ml + ml_at<HS>(w, head, 0));
        const float2 acc = *reinterpret_cast<const float2*>(s_acc + (w * g + head) * kHeadDim + ch);
        const float off = BITS == 4 ? s_ml[ml_at<HS>(w, head, lane >> 4) + 2] : 0.f;
        const float f = fast_exp2((ml.x - mm) * a.factor);
        l = __builtin_fmaf(ml.y, f, l);
        v0 = __builtin_fmaf(acc.x + off, f, v0);
        v1 = __builtin_fmaf(acc.y + off, f, v1);
      }
      if (whole) {
        const HeadSum sum = HeadSum::of(mm, l);
        *reinterpret_cast<float2*>(a.out + (qh0 + head) * kHeadDim + ch) = l == 0.f ? make_float2(0.f, 0.f) : make_float2(v0 * sum.inv, v1 * sum.inv);
        if (lane == 0) {
          if (a.lse != nullptr) a.lse[qh0 + head] = log_sum(a, mm, l);
          s_sums[head] = sum;
        }
      } else {
        *reinterpret_cast<float2*>(a.part_acc + (slot * g + head) * kHeadDim + ch) = make_float2(v0, v1);
        if (lane == 0) *reinterpret_cast<float2*>(a.part_ml + (slot * g + head) * 2) = make_float2(mm, l);
      }
    }
    __syncthreads();
    if (kKeep && a.s.weight != nullptr) {
      add_held<HS, NWV>(a, item, reinterpret_cast<const float*>(held.at), s_sums, n, wave, tiles, w_first);
    } else if (!kKeep && whole && a.s.weight != nullptr) {
      if (HS == 2) add_weights<8>(a, item, sc.scores, s_sums, n, tid, NWV * 64);
      else if (g == 4) add_weights<4>(a, item, sc.scores, s_sums, n, tid, NWV * 64);
      else if (g == 2) add_weights<2>(a, item, sc.scores, s_sums, n, tid, NWV * 64);
      else add_weights<1>(a, item, sc.scores, s_sums, n, tid, NWV * 64);
      __syncthreads();
    }
    at = first + t1;
    if (t1 == tiles) {
      first += tiles + a.start;
      at += a.start;
      ++item;
    }
  } while (NWV == 4 && at < p.end);
}

__device__ __forceinline__ float wave_sum(float v) {
  float o = v = sum_xor16(row_sum(v));
  swap_halves(v, o);
  return v + o;
}

// The items whose tiles several workgroups shared: their partials into the outputs, and their weights.  `rows` workgroups an item, each
// with kJoinSlots slots of it; its loads of them are under way while the heads' sums are made.
constexpr int kJoinThreads = 256, kJoinEach = 4, kJoinSlots = kJoinThreads * kJoinEach;
template <int G>
__global__ __launch_bounds__(kJoinThreads) void join_kernel(DecodeArgs a, int rows) {
  __shared__ HeadSum s_sums[G];
  __shared__ float s_lse[G], s_half[kHeadDim];
  const int item = blockIdx.x / rows, row = blockIdx.x % rows, tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int2 of = a.parts[item];
  const int n = a.s.length(item), parts = of.y, i0 = row * kJoinSlots + tid;
  const int64_t slot0 = of.x, qh0 = static_cast<int64_t>(item) * G;
  const bool tracked = a.s.weight != nullptr && row * kJoinSlots < a.s.capacity;
  float* weight = a.s.weight + static_cast<int64_t>(item) * a.s.capacity;
  WeightPart<G, kJoinEach> part;
  if (tracked) part.load(a.scores + qh0 * a.score_rows, weight, i0, kJoinThreads, a.s.capacity);
  if (parts == 0) return;
  for (int head = wave; head < G; head += kJoinThreads / 64) {
    float m = kLowest, l = 0.f;
    for (int k = lane; k < parts; k += 64) {
      const float2 ml = *reinterpret_cast<const float2*>(a.part_ml + ((slot0 + k) * G + head) * 2);
      const float mm = fmaxf(m, ml.x);
      l = l * fast_exp2((m - mm) * a.factor) + ml.y * fast_exp2((ml.x - mm) * a.factor);
      m = mm;
    }
    float top = row_max(m), o = top;
    swap_rows(top, o);
    top = o = fmaxf(top, o);
    swap_halves(top, o);
    top = fmaxf(top, o);
    l = wave_sum(l * fast_exp2((m - top) * a.factor));
    if (lane == 0) {
      s_sums[head] = HeadSum::of(top, l);
      s_lse[head] = log_sum(a, top, l);
    }
  }
  __syncthreads();
  // heads among the item's workgroups: two halves of the partials, a channel a thread
  for (int head = row; head < G; head += rows) {
    const int c = tid & (kHeadDim - 1), half = tid >> 7;
    const HeadSum sum = s_sums[head];
    float v = 0.f;
    for (int k = half; k < parts; k += 2) {
      const float2 ml = *reinterpret_cast<const float2*>(a.part_ml + ((slot0 + k) * G + head) * 2);
      v = __builtin_fmaf(a.part_acc[((slot0 + k) * G + head) * kHeadDim + c], fast_exp2((ml.x - sum.top) * a.factor), v);
    }
    if (half == 1) s_half[c] = v;
    __syncthreads();
    if (half == 0) {
      v += s_half[c];
      a.out[(qh0 + head) * kHeadDim + c] = sum.inv == 0.f ? 0.f : v * sum.inv;
      if (c == 0 && a.lse != nullptr) a.lse[qh0 + head] = s_lse[head];
    }
    __syncthreads();
  }
  if (tracked) part.store(weight, a.s.decay, a.factor, s_sums, i0, kJoinThreads, n);
}

constexpr size_t kMostLds = 160 << 10;
// Whether a workgroup takes an item alone (if its scores fit).  Then a compute unit's reading bounds a step: 6 us and `own` us a tile, more
// where rows come from memory (`stream`), or all units' reading, `rate`; 256 items at a time.  Shared out, a step is two launches, `base`
// us, and bound by `rate`.  Alone and shared, us, rows of several caches in turn:
//   bf16, 4 heads     8 items of 500 slots  9.3, 13.5   of 1000  13.1, 15.0   of 2000  20.0, 14.9   32 of 1500  17.4, 16.2
//                     64 of 1500  22.5, 22.6   of 4000  47.0, 32.6   128 of 2500  38.4, 39.2   of 4000  51.9, 52.4 (lengths of 1300 to
//                     4000 46.8, 37.1)   256 of 4000  82.5, 98.6   512 of 2000  87.6, 100.9
//   bf16, 8 heads     8 of 2000  24.2, 19.1   32 of 1500  20.4, 19.9   64 of 1500  24.7, 26.6   128 of 2500  39.1, 43.5   512 of 2000  90.5, 111.8
//   4 bits, 4 heads   8 of 1000  9.0, 13.4   of 2000  14.3, 12.9   32 of 3000  20.5, 17.8   64 of 4000  26.6, 20.8   128 of 4000  27.1, 27.7
//                     256 of 4000  33.7, 44.8
//   4 bits, 8 heads   8 of 1000  12.4, 18.7   of 2000  20.0, 17.8   32 of 3000  28.3, 23.3   128 of 2500  27.0, 32.1   512 of 2000  49.8, 58.6
bool one_each(int64_t items, int g, int64_t tiles, int bits, bool stream) {
  const bool wide = g > 4;
  const double own = bits == 4 ? (wide ? 0.5 : 0.31) : stream ? (wide ? 0.85 : 0.77) : (wide ? 0.53 : 0.42);
  const double rate = bits == 4 ? (wide ? 0.0024 : 0.0020) : stream ? 0.0050 : 0.0035;
  const double base = bits == 4 ? (wide ? 18.0 : 13.5) : (wide ? 16.0 : 13.0);
  const int64_t turns = items / 256, rest = items % 256;
  const double alone = static_cast<double>(turns) * std::max(own, 256 * rate) + (rest > 0 ? std::max(own, static_cast<double>(rest) * rate) : 0.0);
  return 6.0 + alone * static_cast<double>(tiles) <= base + rate * static_cast<double>(items) * static_cast<double>(tiles);
}
// LDS of a workgroup of eight wavefronts that keep `held` bytes of scores each
size_t lds_of_eight(int bits, int g, size_t held) {
  return 8 * (held + (bits == 16 ? kHalfBytes : g * kHeadDim * sizeof(float))) + (ml_lds_floats(8, g > 4 ? 2 : 1) + kHeadFloats) * sizeof(float) +
         (bits == 16 && g > 4 ? kQueryBytes : 0);
}
struct Plan {
  bool stream;         // rows past the caches' order
  int waves, groups, least, start, score_rows, join_rows, held_bytes;
  size_t scores, part_acc, part_ml, parts;      // floats
};
Plan make_plan(int64_t items, int g, int capacity, int bits, bool weights) {
  Plan p;
  const int64_t tiles = (capacity + kTile - 1) / kTile;
  p.score_rows = static_cast<int>(tiles) * kTile;
  p.scores = static_cast<size_t>(items) * g * p.score_rows;
  p.stream = items * capacity * (bits == 16 ? 512 : 160) >= (static_cast<int64_t>(64) << 20);
  p.waves = 8;
  // scores that a wavefront keeps, where a workgroup has an item's tiles
  const size_t held = weights ? (tiles + p.waves - 1) / p.waves * kTile * g * sizeof(float) : 0;
  const bool fits = lds_of_eight(bits, g, held) <= kMostLds;
  p.held_bytes = fits ? static_cast<int>(held) : 0;
  if (fits && one_each(items, g, tiles, bits, p.stream)) {
    p.least = p.start = p.join_rows = 0;
    p.groups = static_cast<int>(items);
    p.part_acc = p.part_ml = p.parts = 0;
    return p;
  }
  p.waves = 4;
  p.least = p.waves;
  p.start = bits == 16 ? 4 : 8;
  const int64_t most = (items * tiles + p.waves - 1) / p.waves;
  const int64_t resident = 512;
  p.groups = static_cast<int>(std::min(most, resident));
  p.join_rows = weights ? (capacity + kJoinSlots - 1) / kJoinSlots : g;
  const size_t slots = static_cast<size_t>(p.groups) + items;
  p.part_acc = slots * g * kHeadDim;
  p.part_ml = slots * g * 2;
  p.parts = 2 * static_cast<size_t>(items);
  return p;
}

template <int BITS, int HS, int NWV, bool STREAM>
hipError_t launch_one(const DecodeArgs& a, const Plan& p, hipStream_t st) {
  const size_t lds = NWV == 8 ? lds_of_eight(BITS, a.s.g, a.held_bytes)
                              : NWV * ((BITS == 16 ? kHalfBytes : 0) + held_bytes_of_four(BITS)) + (ml_floats<NWV, HS>() + kHeadFloats) * sizeof(float) +
                                    (BITS == 16 && HS == 2 ? kQueryBytes : 0);
  static_assert(NWV * held_bytes_of_four(BITS) >= kHeldLengths * 4 + 4 * kTries * 8, "the lengths fit");
  static_assert(held_bytes_of_four(4) >= 4 * HS * kHeadDim * 4 && kHalfBytes >= 4 * HS * kHeadDim * 4, "the accumulators fit");
  const hipError_t e = RDKV_ALLOW_LDS((decode_kernel<BITS, HS, NWV, STREAM>), NWV == 8 ? kMostLds : lds);
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL((decode_kernel<BITS, HS, NWV, STREAM>), dim3(p.groups), dim3(NWV * 64), lds, st, a);
  return hipGetLastError();
}

template <int BITS, int HS>
hipError_t launch(const DecodeArgs& a, const Plan& p, hipStream_t st) {
  if (p.waves == 8) return p.stream ? launch_one<BITS, HS, 8, true>(a, p, st) : launch_one<BITS, HS, 8, false>(a, p, st);
  return p.stream ? launch_one<BITS, HS, 4, true>(a, p, st) : launch_one<BITS, HS, 4, false>(a, p, st);
}

}  // namespace

size_t decode_workspace_floats(int64_t items, int g, int capacity, int bits, bool weights) {
  const Plan p = make_plan(items, g, capacity, bits, weights);
  return std::max<size_t>((weights ? p.scores : 0) + p.part_acc + p.part_ml + p.parts, 4);
}

hipError_t launch_decode(const Args& s, int bits, int items, const uint16_t* q, float* out, float* lse, float* workspace, hipStream_t st) {
  const Plan p = make_plan(items, s.g, s.capacity, bits, s.weight != nullptr);
  DecodeArgs a;
  a.s = s;
  a.q = q;
  a.out = out;
  a.lse = lse;
  a.scores = workspace;                  // (of a cache without weights: nothing)
  if (s.weight) workspace += p.scores;
  a.part_acc = workspace;
  a.part_ml = a.part_acc + p.part_acc;
  a.parts = reinterpret_cast<int2*>(a.part_ml + p.part_ml);
  a.items = items;
  a.score_rows = p.score_rows;
  a.least = p.least;
  a.start = p.start;
  a.held_bytes = p.held_bytes;
  const bool scores = s.cap > 0.f || s.slopes != nullptr;
  a.factor = scores ? kLog2e : kRootLog2e;
  a.natural = scores ? 1.f : kRoot;
  const hipError_t e = bits == 16 ? s.g > 4 ? launch<16, 2>(a, p, st) : launch<16, 1>(a, p, st)
                                  : s.g > 4 ? launch<4, 2>(a, p, st) : launch<4, 1>(a, p, st);
  if (e != hipSuccess || p.join_rows == 0) return e;
  const dim3 grid(items * p.join_rows), threads(kJoinThreads);
  switch (s.g) {
    case 8: hipLaunchKernelGGL(join_kernel<8>, grid, threads, 0, st, a, p.join_rows); break;
    case 4: hipLaunchKernelGGL(join_kernel<4>, grid, threads, 0, st, a, p.join_rows); break;
    case 2: hipLaunchKernelGGL(join_kernel<2>, grid, threads, 0, st, a, p.join_rows); break;
    default: hipLaunchKernelGGL(join_kernel<1>, grid, threads, 0, st, a, p.join_rows); break;
  }
  return hipGetLastError();
}

}  // namespace slots
}  // namespace rdkv
