// Causal attention of whole prompts: out_i = sum_j p_ij v_j, p_ij = exp(x_ij - m_i) / sum_j exp(x_ij - m_i), one pass over the keys with a reference m_i
// that follows a row's largest score.
//
// A workgroup has 128 rows of a head, 32 a wavefront, and walks their keys in tiles of 64.  Products have keys on their A side, so that a lane
// has one row: maxima and sums are its own but for one exchange between the halves, and its probabilities, packed where they are, are P V's
// other operand.  K and V go straight into LDS, two tiles of each; a wavefront issues the next tile's 16 products between a tile's first 16
// exponentials, and the other 16 between P V's products.
//   bound   the matrix cores, at the clock that the card's power leaves them: 32768 tokens of 32 heads take 7.8 to 8.5 ms from card to card, 1.13 PFLOP/s at
//           1.70 GHz (a library's product of two matrices of 16384 rows reaches 1.59); matrix cores 63 % busy, vector 66 %.  With a cap vector instructions
//           are, at 80 %.
//   tried   256 rows in eight wavefronts with four tiles on their way: as fast for one long prompt, 10 % slower for many (one barrier for all of a
//           compute unit).  64 rows a wavefront, half the reads from LDS: does not fit the registers, 15 ms.  A tile's exponentials without the
//           next one's products between them: 8.4 ms
#include <algorithm>

#include "attn_tiles.h"
#include "prompt.h"

namespace rdkv {
namespace prompt {

namespace {

using namespace attn;

constexpr int kTileBytes = kKeys * kRowBytes;        // of K, or of V
constexpr int kRing = 2;
constexpr float kLowest = -2e38f;                    // a finite maximum of nothing, also times log2(e): no score is below it
constexpr float kMostOver = 1e38f;                   // the largest cap that scores are kept over: times log2(e) it is finite
constexpr float kSlack = 8.f;                        // what exponents may exceed the reference by before it moves

// element (head, token 0, channel 0) of a sequence
__device__ __forceinline__ int64_t first_of(const Side& s, int64_t token0, int heads, int head, int T) {
  return s.tokens ? token0 * s.row + head * kHeadDim : (token0 * heads + static_cast<int64_t>(head) * T) * kHeadDim;
}

// WS: wavefronts that share the tiles of 32 rows.  A stage is as many tiles, one each.
template <bool GENERAL, int WS>
__global__ __launch_bounds__(2 * kRows, 3 - WS) void prompt_kernel(Args a) {
  extern __shared__ __align__(256) uint8_t smem[];
  constexpr int NW = prompt::kRows / 32, kRows = prompt::kRows / WS, kCopies = WS * 16 / NW;       // kCopies: of a wavefront, for a stage of K or V
  constexpr uint32_t kStage = WS * kTileBytes;
  const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6), l32 = lane & 31, half = lane >> 5;
  // The sequence, the longest is first; of that all heads' last rows first.  Heads of a KV head are beside each other on an XCD where that can be.
  const int mine = static_cast<int>(blockIdx.x), seq = __popcll(__ballot(lane < a.n_seqs && a.first[lane] <= mine)) - 1;
  const int T = a.T[seq], unit = mine - a.first[seq], levels = (T + kRows - 1) / kRows;
  const int level = unit / a.hq, kvh = unit % a.hq % a.hkv, head = kvh * (a.hq / a.hkv) + unit % a.hq / a.hkv;
  if (level >= levels) return;
  const int q0 = (levels - 1 - level) * kRows;
  const int64_t token0 = a.token0[seq];
  const uint16_t* Kh = a.K + first_of(a.k, token0, a.hkv, kvh, T);
  const uint16_t* Vh = a.V + first_of(a.v, token0, a.hkv, kvh, T);

  // the tiles that some row of the workgroup sees: the sinks', and those from the first row's window on
  const int first = a.window > 0 ? max(0, q0 - a.window + 1) / kKeys : 0, n_sink = a.window > 0 ? min((min(a.sinks, T) + kKeys - 1) / kKeys, first) : 0;
  const int n_tiles = (min(T, q0 + kRows) + kKeys - 1) / kKeys - first + n_sink, n_it = (n_tiles + WS - 1) / WS;
  const auto tile_of = [&](int t) { return t < n_sink ? t : t - n_sink + first; };

  const uint32_t lds0 = lds_address(smem);
  const int prow = tid >> 4;                         // this thread's rows prow + 4 NW k
  const uint32_t k_at = 16 * k_piece(prow, tid & 15), v_at = 16 * v_piece(prow, tid & 15);
  const auto slot = [](int it) { return static_cast<uint32_t>(it % kRing) * kStage; };
  const auto fetch = [&](const uint16_t* from, const Side& side, uint32_t at, int it, uint32_t to) __attribute__((always_inline)) {
    to += slot(it) + wave * 1024;
#pragma unroll
    for (int x = 0; x < WS; ++x) {
      const int key0 = tile_of(min(it * WS + x, n_tiles - 1)) * kKeys, last = T - 1 - key0;
      const uint16_t* first_key = from + static_cast<int64_t>(key0) * side.row;
#pragma unroll
      for (int k = 0; k < 16 / NW; ++k)
        copy_to_lds(first_key, static_cast<uint32_t>(min(prow + 4 * NW * k, last) * side.row) * 2 + at, to + x * kTileBytes + 1024 * NW * k);
    }
  };
  const auto fetch_k = [&](int it) __attribute__((always_inline)) { fetch(Kh, a.k, k_at, it, lds0); };
  const auto fetch_v = [&](int it) __attribute__((always_inline)) { fetch(Vh, a.v, v_at, it, lds0 + kRing * kStage); };

  const int ws = wave % WS, r0 = q0 + 32 * (wave / WS), row = r0 + l32;              // this wavefront's first row, and the lane's
  bf16x8 q_op[8];
  const uint16_t* q = a.Q + first_of(a.q, token0, a.hq, head, T) + static_cast<int64_t>(min(row, T - 1)) * a.q.row + 8 * half;
#pragma unroll
  for (int kb = 0; kb < 8; ++kb) q_op[kb] = *reinterpret_cast<const bf16x8*>(q + 16 * kb);
  fetch_k(0);                                        // (on their way together with the queries)
  fetch_v(0);
  fetch_k(1);
#pragma unroll
  for (int kb = 0; kb < 8; ++kb) arrived(q_op[kb]);
  const float slope = GENERAL && a.slopes ? a.slopes[head] : 0.f, inv_cap = GENERAL && a.cap > 0.f ? 1.f / a.cap : 0.f;
  const TanhSmall small(kRoot * inv_cap);
  // What makes the numbers that are kept (products, scores over the cap, or with biases and caps past kMostOver scores) scores, and those exponents of 2;
  // a maximum of nothing among them, in their units: with the factor it stays finite as well.
  const bool scored = GENERAL && (a.slopes || a.cap > kMostOver);
  const float units = GENERAL && a.cap > 0.f ? a.cap : kRoot;
  const float factor = !GENERAL ? kRootLog2e : scored ? kLog2e : units * kLog2e;
  const float lowest = GENERAL && !scored ? kLowest / fmaxf(units, 1.f) : kLowest;

  floatx16 o[4];
  float m, l;
  const auto key_of = [&](int it) { return tile_of(it * WS + ws) * kKeys; };
  const uint32_t k_first = lds0 + ws * kTileBytes + k_lane(), v_first = lds0 + kRing * kStage + ws * kTileBytes + v_lane();
  // The tiles that this wavefront's rows have to do with: until its last row, and from its first row's window on (where there are sinks, from those
  // on).  Of those its own stages.
  const int t_end = min(n_tiles, (r0 + 31) / kKeys - first + n_sink + 1);
  const int t_begin = a.window > 0 && a.sinks == 0 ? min(t_end - 1, max(0, r0 - a.window + 1) / kKeys - first) : 0;
  const int it_end = (t_end - ws + WS - 1) / WS, it_begin = (t_begin - ws + WS - 1) / WS;
  const auto begin = [&]() __attribute__((always_inline)) {
#pragma unroll
    for (int t = 0; t < 4; ++t) o[t] = floatx16{};
    m = lowest;
    l = 0.f;
  };
  const auto key = [](int x, int i) { return 32 * x + 8 * (i >> 2) + (i & 3); };
  // Products of a tile to scores, -inf where hidden; whether it did something.
  const auto finish = [&](int it, floatx16 (&s)[2]) __attribute__((always_inline)) {
    const int key0 = key_of(it), back = row - key0 - 4 * half;           // positions from key 4 half of the tile to the row
    if constexpr (GENERAL) {
      float v[32];
#pragma unroll
      for (int i = 0; i < 32; ++i) v[i] = s[i >> 4][i & 15];
      if (a.cap > 0.f) tanh_all(v, kRoot * inv_cap, small);
      if (scored) {
#pragma unroll
        for (int i = 0; i < 32; ++i) v[i] = __builtin_fmaf(v[i], units, -slope * static_cast<float>(back - key(i >> 4, i & 15)));
      }
#pragma unroll
      for (int i = 0; i < 32; ++i) s[i >> 4][i & 15] = v[i];
    }
    const bool edge = key0 + kKeys - 1 > r0, far = a.window > 0 && r0 + 31 - key0 >= a.window;
    if (edge) {
#pragma unroll
      for (int x = 0; x < 2; ++x)
#pragma unroll
        for (int i = 0; i < 16; ++i) s[x][i] = key(x, i) > back ? -INFINITY : s[x][i];
    }
    if (far) {
      const int sink = a.sinks - key0 - 4 * half;
#pragma unroll
      for (int x = 0; x < 2; ++x)
#pragma unroll
        for (int i = 0; i < 16; ++i) s[x][i] = back - key(x, i) >= a.window && key(x, i) >= sink ? -INFINITY : s[x][i];
    }
    return GENERAL || edge || far;
  };
  const auto multiply = [&](int it, floatx16 (&s)[2]) __attribute__((always_inline)) {
    const uint32_t kt = k_first + slot(it);
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const bf16x8 k = read_k(kt, i & 7, i >> 3);
      s[i >> 3] = product(k, q_op[i & 7], (i & 7) == 0 ? floatx16{} : s[i >> 3]);
    }
  };
  // The exponent of 2 that a change of the reference takes: with care of a difference, as exponents are there; else the difference of what exponents are
  // made with, the references times the factor as they are rounded, so that tiles of different references weigh the same.
  const auto between = [&](float from, float to, bool care) { return care ? (from - to) * factor : from * factor - to * factor; };
  // the row's reference, if its largest score is past it
  const auto refer = [&](float top, bool care) __attribute__((always_inline)) {
    if (__any(care ? top > m : (top - m) * factor > kSlack)) {
      const float now = fmaxf(m, top), alpha = __builtin_amdgcn_exp2f(between(m, now, care));
      m = now;
      l *= alpha;
#pragma unroll
      for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[t][i] *= alpha;
    }
  };
  const auto largest = [&](const floatx16 (&s)[2]) __attribute__((always_inline)) {
    float top = s[0][0];
#pragma unroll
    for (int i = 0; i < 32; ++i) top = fmaxf(top, s[i >> 4][i & 15]);
    return top;
  };

  // A tile's softmax and P V, and between their instructions the next tile's products (MORE), so that the matrix cores have work while
  // exponentials are made: 16 of those stand between the 16 products, 16 between the first 8 of P V.  Each line is one product and what the plain ALUs
  // do meanwhile.
  // top: the lane's largest score of the tile; the next one's comes back.
  const auto position = [&](auto more, int it, floatx16 (&s)[2], floatx16 (&next)[2], float& top) __attribute__((always_inline)) {
    constexpr bool kMore = decltype(more)::value;
    float sums[2] = {}, tops;
    union { uint32_t u[16]; bf16x8 op[4]; } p;
    refer(halves_max(top), false);
    const float ref = -m * factor;
    const uint32_t kt = k_first + slot(it + 1), vt = v_first + slot(it);
    // Exponential i, in order; what hangs on another one's result stands behind it, so that nothing waits for it.
    float x = __builtin_fmaf(s[0][0], factor, ref), e[3];
    const auto make = [&](int i) __attribute__((always_inline)) {
      const float now = x;
      if (i < 31) x = __builtin_fmaf(s[(i + 1) >> 4][(i + 1) & 15], factor, ref);
      if (i < 32) e[i % 3] = __builtin_amdgcn_exp2f(now);
      if (i > 0) {
        sums[i & 1] += e[(i - 1) % 3];
        here(sums[i & 1]);
      }
      if (i > 0 && (i & 1) == 0) p.u[(i >> 1) - 1] = pair_bf16(e[(i - 2) % 3], e[(i - 1) % 3]);
    };
    // operands on their way from LDS, of products 0 .. 15 (K) and 16 .. 31 (V: keys 16 (i / 4) .., channels 32 (i % 4) ..)
    constexpr int kAhead = 3;
    bf16x8 op[kAhead];
    const auto ask = [&](int i) __attribute__((always_inline)) {
      if (i < 16) op[i % kAhead] = read_k(kt, i & 7, i >> 3);
      else if (i < 32) op[i % kAhead] = read_v(vt, i & 3, (i >> 2) & 1, (i - 16) >> 3);
    };
    if constexpr (kMore) {
#pragma unroll
      for (int i = 0; i < kAhead; ++i) ask(i);
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        next[i >> 3] = product(op[i % kAhead], q_op[i & 7], (i & 7) == 0 ? floatx16{} : next[i >> 3]);
        ask(i + kAhead);
        make(i);
        __builtin_amdgcn_sched_barrier(0);
      }
    } else {
#pragma unroll
      for (int i = 16; i < 16 + kAhead; ++i) ask(i);
#pragma unroll
      for (int i = 0; i < 16; ++i) make(i);
    }
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      o[i & 3] = product(op[(i + 16) % kAhead], p.op[i >> 2], o[i & 3]);
      ask(i + 16 + kAhead);
      if (i < 8) {
        make(16 + 2 * i);
        make(17 + 2 * i);
      } else {
        if (i == 8) make(32);
        if (!kMore) continue;
        const int j = 4 * (i - 8);
        const floatx16& n = next[j >> 4];
        const float a = n[j & 15], b = n[(j & 15) + 1], c = n[(j & 15) + 2], d = n[(j & 15) + 3];
        tops = fmaxf(fmaxf(i == 8 ? a : fmaxf(tops, a), b), fmaxf(c, d));
        if (!GENERAL) here(tops);
      }
      __builtin_amdgcn_sched_barrier(0);
    }
    l += sums[0] + sums[1];
    __builtin_amdgcn_s_setprio(0);
    if constexpr (kMore) top = finish(it + 1, next) ? largest(next) : tops;
  };
  const auto walk = [&]() __attribute__((always_inline)) {
    begin();
    tile_barrier<2 * kCopies>();
    floatx16 even[2], odd[2];
    const auto open = [&](int it) __attribute__((always_inline)) {       // K of tile it + 1 and V of tile it are there, K of tile it and V of tile it - 1 done with
      tile_barrier<0>();
      fetch_k(it + 2);
      fetch_v(it + 1);
      __builtin_amdgcn_s_setprio(1);                 // (the other workgroup of the compute unit is elsewhere in its tile)
    };
    int it = 0;
    for (; it < it_begin; ++it) open(it);
    if (WS == 1 || it < it_end) {
      multiply(it, even);
      finish(it, even);
      float top = largest(even);
      for (; it + 2 < it_end; it += 2) {
        open(it);
        position(std::true_type{}, it, even, odd, top);
        open(it + 1);
        position(std::true_type{}, it + 1, odd, even, top);
      }
      open(it);
      if (it + 1 < it_end) {
        position(std::true_type{}, it, even, odd, top);
        open(++it);
        position(std::false_type{}, it, odd, even, top);
      } else {
        position(std::false_type{}, it, even, odd, top);
      }
      ++it;
    }
    for (; it < n_it; ++it) open(it);
    tile_barrier<0>();                               // (copies of tiles past the last have landed as well)
  };
  // Again, with care, where a result is not finite or a row that saw something has next to none of it: rows of V that some rows of a tile do not see are kept
  // from meeting their zeros, which make NaN of what is not finite, and exponents are of differences, so that scores may be of any size (a reference of 2^30
  // times the factor is off by up to 8 when rounded, and from 2^34 on all that a row sees could be below fp32's least, or past its largest).
  const auto walk_with_care = [&]() __attribute__((always_inline)) {
    begin();
    for (int it = 0; it < n_it; ++it) {
      tile_barrier<0>();
      fetch_k(it);
      fetch_v(it);
      tile_barrier<0>();
      if (it < it_begin || it >= it_end) continue;
      floatx16 s[2];
      multiply(it, s);
      const uint32_t vt = v_first + slot(it);
      finish(it, s);
      refer(halves_max(largest(s)), true);
      float p[32];
#pragma unroll
      for (int i = 0; i < 32; ++i) {
        p[i] = __builtin_amdgcn_exp2f((s[i >> 4][i & 15] - m) * factor);
        l += p[i];
      }
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        floatx16 up = {}, down = {};
        bool odd = false;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const Parted v = part(read_v(vt, t, k & 1, k >> 1));
          o[t] = product(v.finite, to_bf16(p + 8 * k), o[t]);
          if (__any(v.any)) {
            float there[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) there[i] = p[8 * k + i] == 0.f ? 0.f : 1.f;
            up = product(v.up, to_bf16(there), up);
            down = product(v.down, to_bf16(there), down);
            odd = true;
          }
        }
        if (odd) {
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            if (up[i] > 0.f) o[t][i] += INFINITY;
            if (down[i] > 0.f) o[t][i] -= INFINITY;
          }
        }
      }
    }
  };
  walk();
  float sum = 0.f;
#pragma unroll
  for (int t = 0; t < 4; ++t)
#pragma unroll
    for (int i = 0; i < 16; ++i) sum = __builtin_fmaf(o[t][i], 0.f, sum);
  sum = __builtin_fmaf(l, 0.f, sum);
  const bool lost = m != lowest && halves_add(l) < 0x1p-20f;
  const bool care = __syncthreads_or(sum != 0.f || lost);
  if (care) walk_with_care();

  l = halves_add(l);
  if constexpr (WS == 2) {
    // the other's result, over the larger reference, to the first one's
    __syncthreads();
    float* theirs = reinterpret_cast<float*>(smem) + wave / WS * (66 * 64) + lane;
    if (ws == 1) {
      theirs[64 * 64] = m;
      theirs[65 * 64] = l;
#pragma unroll
      for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int i = 0; i < 16; ++i) theirs[(16 * t + i) * 64] = o[t][i];
    }
    __syncthreads();
    if (ws == 1) return;
    const float other = theirs[64 * 64], now = fmaxf(m, other);
    const float mine = __builtin_amdgcn_exp2f(between(m, now, care)), its = __builtin_amdgcn_exp2f(between(other, now, care));
    m = now;
    l = __builtin_fmaf(theirs[65 * 64], its, l * mine);
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
      for (int i = 0; i < 16; ++i) o[t][i] = __builtin_fmaf(theirs[(16 * t + i) * 64], its, o[t][i] * mine);
  }
  const float total = l, inv = total == 0.f ? 0.f : 1.f / total;
  if (row >= T) return;
  uint16_t* out = a.out + first_of(a.o, token0, a.hq, head, T) + static_cast<int64_t>(row) * a.o.row + 8 * half;
#pragma unroll
  for (int t = 0; t < 4; ++t)
#pragma unroll
    for (int c = 0; c < 2; ++c) {
    float v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = o[t][8 * c + i] * inv;
    union { bf16x8 b; uint32_t u[4]; } w;
    w.b = to_bf16(v);
    // channels 16 c + 0..7 to the lower half, 8..15 to the upper
    asm("s_nop 1\n\tv_permlane32_swap_b32 %0, %1" : "+v"(w.u[0]), "+v"(w.u[2]));
    asm("s_nop 1\n\tv_permlane32_swap_b32 %0, %1" : "+v"(w.u[1]), "+v"(w.u[3]));
    *reinterpret_cast<uint4*>(out + 32 * t + 16 * c) = make_uint4(w.u[0], w.u[1], w.u[2], w.u[3]);
  }
  if (a.lse && half == 0)
    a.lse[token0 * a.hq + static_cast<int64_t>(head) * T + row] = total == 0.f ? -INFINITY : __builtin_fmaf(m * factor, kLn2, __logf(total));
}

template <bool GENERAL, int WS>
hipError_t start(const Args& a, int grid, hipStream_t st) {
  constexpr int lds = 2 * kRing * WS * kTileBytes;
  const hipError_t e = RDKV_ALLOW_LDS((prompt_kernel<GENERAL, WS>), lds);
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL((prompt_kernel<GENERAL, WS>), dim3(grid), dim3(2 * kRows), lds, st, a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch(const Args& a, int grid, bool shared, hipStream_t st) {
  const bool general = a.cap > 0.f || a.slopes;      // (a window takes no scores of its own)
  if (shared) return general ? start<true, 2>(a, grid, st) : start<false, 2>(a, grid, st);
  return general ? start<true, 1>(a, grid, st) : start<false, 1>(a, grid, st);
}

}  // namespace prompt
}  // namespace rdkv
