// Causal attention of whole prompts.
#include <algorithm>

#include "attn_tiles.h"
#include "prompt.h"

namespace rdkv {
namespace prompt {

namespace {

using namespace attn;

constexpr int kTileBytes = kKeys * kRowBytes;        // of K, or of V
constexpr int kBuffers = 4;
constexpr float kLowest = -2e38f;                    // a finite maximum of nothing, also times log2(e): no score is below it
constexpr float kSlack = 8.f;                        // what exponents may exceed the reference by before it moves

// element (head, token 0, channel 0) of a sequence
__device__ __forceinline__ int64_t first_of(const Side& s, int64_t token0, int heads, int head, int T) {
  return s.tokens ? token0 * s.row + head * kHeadDim : (token0 * heads + static_cast<int64_t>(head) * T) * kHeadDim;
}

template <int NW, bool GENERAL>
__global__ __launch_bounds__(64 * NW, NW == 8 ? 2 : 2) void prompt_kernel(Args a) {
  extern __shared__ __align__(256) uint8_t smem[];
  constexpr int kRows = 32 * NW, kCopies = 32 / NW;       // kCopies: of a wavefront and tile
  const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6), l32 = lane & 31, half = lane >> 5;
  const int items = a.n_seqs * a.hkv, pairs = a.n_seqs * a.hq;
  const int level = static_cast<int>(blockIdx.x) / pairs, pair = static_cast<int>(blockIdx.x) % pairs;
  const int item = pair % items, seq = item / a.hkv, kvh = item % a.hkv, head = kvh * (a.hq / a.hkv) + pair / items;
  const int T = a.T[seq];
  const int q0 = (static_cast<int>(gridDim.x) / pairs - 1 - level) * kRows;
  if (q0 >= T) return;
  const int64_t token0 = a.token0[seq];
  const uint16_t* Kh = a.K + first_of(a.k, token0, a.hkv, kvh, T);
  const uint16_t* Vh = a.V + first_of(a.v, token0, a.hkv, kvh, T);

  // the tiles that some row of the workgroup sees: the sinks', and those from the first row's window on
  const int first = a.window > 0 ? max(0, q0 - a.window + 1) / kKeys : 0, n_sink = a.window > 0 ? min((min(a.sinks, T) + kKeys - 1) / kKeys, first) : 0;
  const int n_it = (min(T, q0 + kRows) + kKeys - 1) / kKeys - first + n_sink;
  const auto tile_of = [&](int it) { return it < n_sink ? it : it - n_sink + first; };

  const uint32_t lds0 = lds_address(smem);
  const int prow = tid >> 4;                         // this thread's rows prow + 4 NW k
  const uint32_t k_at = 16 * k_piece(prow, tid & 15), v_at = 16 * v_piece(prow, tid & 15);
  const auto fetch = [&](int it) __attribute__((always_inline)) {
    const int key0 = tile_of(min(it, n_it - 1)) * kKeys, last = T - 1 - key0;
    const uint16_t* ks = Kh + static_cast<int64_t>(key0) * a.k.row;
    const uint16_t* vs = Vh + static_cast<int64_t>(key0) * a.v.row;
    const uint32_t to = lds0 + (it % kBuffers) * (2 * kTileBytes) + wave * 1024;
#pragma unroll
    for (int k = 0; k < 16 / NW; ++k) {
      const int row = min(prow + 4 * NW * k, last);
      copy_to_lds(ks, static_cast<uint32_t>(row * a.k.row) * 2 + k_at, to + 1024 * NW * k);
      copy_to_lds(vs, static_cast<uint32_t>(row * a.v.row) * 2 + v_at, to + kTileBytes + 1024 * NW * k);
    }
  };

  const int r0 = q0 + 32 * wave, row = r0 + l32;     // this wavefront's first row, and the lane's
  bf16x8 q_op[8];
  {
    const uint16_t* q = a.Q + first_of(a.q, token0, a.hq, head, T) + static_cast<int64_t>(min(row, T - 1)) * a.q.row + 8 * half;
#pragma unroll
    for (int kb = 0; kb < 8; ++kb) q_op[kb] = *reinterpret_cast<const bf16x8*>(q + 16 * kb);
#pragma unroll
    for (int kb = 0; kb < 8; ++kb) arrived(q_op[kb]);
  }
  const float slope = GENERAL && a.slopes ? a.slopes[head] : 0.f, inv_cap = GENERAL && a.cap > 0.f ? 1.f / a.cap : 0.f;
  // What makes the numbers that are kept (products, scores over the cap, or with biases scores) scores, and those exponents of 2.
  const float units = GENERAL && a.cap > 0.f ? a.cap : kRoot;
  const float factor = !GENERAL ? kRootLog2e : a.slopes ? kLog2e : a.cap > 0.f ? a.cap * kLog2e : kRootLog2e;

  floatx16 o[4];
  float m, l;
  const auto key_of = [&](int it) { return tile_of(it) * kKeys; };
  const uint32_t k_first = lds0 + k_lane(), v_first = lds0 + kTileBytes + v_lane();
  const auto buffer_of = [&](int it) { return static_cast<uint32_t>(it % kBuffers) * (2 * kTileBytes); };
  // The tiles that this wavefront has to do with: until its last row, and from its first row's window on (where there are sinks, from those on).
  const int it_end = min(n_it, (r0 + 31) / kKeys - first + n_sink + 1);
  const int it_begin = a.window > 0 && a.sinks == 0 ? min(it_end - 1, max(0, r0 - a.window + 1) / kKeys - first) : 0;
  const auto begin = [&]() __attribute__((always_inline)) {
#pragma unroll
    for (int t = 0; t < 4; ++t) o[t] = floatx16{};
    m = kLowest;
    l = 0.f;
#pragma unroll
    for (int it = 0; it < kBuffers - 1; ++it) fetch(it);
  };
  const auto key = [](int x, int i) { return 32 * x + 8 * (i >> 2) + (i & 3); };
  // Products of a tile to scores, -inf where hidden.
  const auto finish = [&](int it, floatx16 (&s)[2]) __attribute__((always_inline)) {
    const int key0 = key_of(it), back = row - key0 - 4 * half;           // positions from key 4 half of the tile to the row
    if constexpr (GENERAL) {
      float v[32];
#pragma unroll
      for (int i = 0; i < 32; ++i) v[i] = s[i >> 4][i & 15];
      if (a.cap > 0.f) tanh_all(v, kRoot * inv_cap);
      if (a.slopes) {
#pragma unroll
        for (int i = 0; i < 32; ++i) v[i] = __builtin_fmaf(v[i], units, -slope * static_cast<float>(back - key(i >> 4, i & 15)));
      }
#pragma unroll
      for (int i = 0; i < 32; ++i) s[i >> 4][i & 15] = v[i];
    }
    if (key0 + kKeys - 1 > r0) {
#pragma unroll
      for (int x = 0; x < 2; ++x)
#pragma unroll
        for (int i = 0; i < 16; ++i) s[x][i] = key(x, i) > back ? -INFINITY : s[x][i];
    }
    if (a.window > 0 && r0 + 31 - key0 >= a.window) {
      const int sink = a.sinks - key0 - 4 * half;
#pragma unroll
      for (int x = 0; x < 2; ++x)
#pragma unroll
        for (int i = 0; i < 16; ++i) s[x][i] = back - key(x, i) >= a.window && key(x, i) >= sink ? -INFINITY : s[x][i];
    }
  };
  const auto multiply = [&](int it, floatx16 (&s)[2]) __attribute__((always_inline)) {
    const uint32_t kt = k_first + buffer_of(it);
#pragma unroll
    for (int x = 0; x < 2; ++x)
#pragma unroll
      for (int kb = 0; kb < 8; ++kb) s[x] = product(read_k(kt, kb, x), q_op[kb], kb == 0 ? floatx16{} : s[x]);
  };
  // the row's reference, if its largest score is past it
  const auto refer = [&](float top, bool any) __attribute__((always_inline)) {
    if (__any(any ? top > m : (top - m) * factor > kSlack)) {
      const float now = fmaxf(m, top), alpha = __builtin_amdgcn_exp2f((m - now) * factor);
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
    return halves_max(top);
  };

  // A tile's softmax and P V, and between their instructions the next tile's products (MORE), so that the matrix cores have work while
  // exponentials are made: 16 of those stand between the 16 products, 16 between the first 8 of P V.  Each line is one product and what the plain ALUs
  // do meanwhile.
  const auto position = [&](auto more, int it, floatx16 (&s)[2], floatx16 (&next)[2]) __attribute__((always_inline)) {
    constexpr bool kMore = decltype(more)::value;
    refer(largest(s), false);
    const float ref = -m * factor;
    const uint32_t kt = k_first + buffer_of(it + 1), vt = v_first + buffer_of(it);
    union { uint32_t u[16]; bf16x8 op[4]; } p;
    float sums[2] = {0.f, 0.f}, before = 0.f;
    const auto make = [&](int i) __attribute__((always_inline)) {        // in order
      const float e = __builtin_amdgcn_exp2f(__builtin_fmaf(s[i >> 4][i & 15], factor, ref));
      sums[i & 1] += e;
      if (i & 1) p.u[i >> 1] = pair_bf16(before, e);
      before = e;
    };
    constexpr int kAhead = 3;
    bf16x8 k_op[kAhead], v_op[kAhead];
    const auto k_at = [&](int i) __attribute__((always_inline)) { return read_k(kt, i & 7, i >> 3); };
    const auto v_at = [&](int i) __attribute__((always_inline)) { return read_v(vt, i & 3, (i >> 2) & 1, i >> 3); };    // keys 16 (i / 4) .., channels 32 (i % 4) ..
    if constexpr (kMore) {
#pragma unroll
      for (int i = 0; i < kAhead; ++i) k_op[i] = k_at(i);
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        next[i >> 3] = product(k_op[i % kAhead], q_op[i & 7], (i & 7) == 0 ? floatx16{} : next[i >> 3]);
        if (i + kAhead < 16) k_op[i % kAhead] = k_at(i + kAhead);
        else v_op[(i + kAhead) % 16] = v_at((i + kAhead) % 16);
        make(i);
        __builtin_amdgcn_sched_barrier(0);
      }
    } else {
#pragma unroll
      for (int i = 0; i < kAhead; ++i) v_op[i] = v_at(i);
#pragma unroll
      for (int i = 0; i < 16; ++i) make(i);
    }
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      o[i & 3] = product(v_op[i % kAhead], p.op[i >> 2], o[i & 3]);
      if (i + kAhead < 16) v_op[i % kAhead] = v_at(i + kAhead);
      if (i < 8) {
        make(16 + 2 * i);
        make(17 + 2 * i);
      }
      __builtin_amdgcn_sched_barrier(0);
    }
    l += sums[0] + sums[1];
    if constexpr (kMore) finish(it + 1, next);
  };
  const auto walk = [&]() __attribute__((always_inline)) {
    begin();
    tile_barrier<kCopies * (kBuffers - 2)>();
    floatx16 even[2], odd[2];
    const auto open = [&](int it) __attribute__((always_inline)) {       // tile it + 1 is there, and the buffer of tile it - 1 free
      tile_barrier<kCopies * (kBuffers - 3)>();
      fetch(it + kBuffers - 1);
    };
    int it = 0;
    for (; it < it_begin; ++it) open(it);
    multiply(it, even);
    finish(it, even);
    for (; it + 2 < it_end; it += 2) {
      open(it);
      position(std::true_type{}, it, even, odd);
      open(it + 1);
      position(std::true_type{}, it + 1, odd, even);
    }
    open(it);
    if (it + 1 < it_end) {
      position(std::true_type{}, it, even, odd);
      open(++it);
      position(std::false_type{}, it, odd, even);
    } else {
      position(std::false_type{}, it, even, odd);
    }
    for (++it; it < n_it; ++it) open(it);
    tile_barrier<0>();                               // (copies of tiles past the last have landed as well)
  };
  // Again, with care, where a result is not finite: rows of V that some rows of a tile do not see are kept from meeting their zeros, which make NaN of
  // what is not finite, and exponents are differences, so that scores may be of any size.
  const auto walk_with_care = [&]() __attribute__((always_inline)) {
    begin();
    for (int it = 0; it < n_it; ++it) {
      tile_barrier<kCopies * (kBuffers - 2)>();
      fetch(it + kBuffers - 1);
      if (it < it_begin || it >= it_end) continue;
      floatx16 s[2];
      multiply(it, s);
      finish(it, s);
      refer(largest(s), true);
      float p[32];
#pragma unroll
      for (int i = 0; i < 32; ++i) {
        p[i] = __builtin_amdgcn_exp2f((s[i >> 4][i & 15] - m) * factor);
        l += p[i];
      }
      const uint32_t vt = v_first + buffer_of(it);
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
    tile_barrier<0>();
  };
  walk();
  float sum = 0.f;
#pragma unroll
  for (int t = 0; t < 4; ++t)
#pragma unroll
    for (int i = 0; i < 16; ++i) sum = __builtin_fmaf(o[t][i], 0.f, sum);
  sum = __builtin_fmaf(l, 0.f, sum);
  if (__syncthreads_or(sum != 0.f)) walk_with_care();

  const float total = halves_add(l), inv = total == 0.f ? 0.f : 1.f / total;
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
  if (a.lse && half == 0) a.lse[token0 * a.hq + static_cast<int64_t>(head) * T + row] = total == 0.f ? -INFINITY : __builtin_fmaf(m * factor, kLn2, __logf(total));
}

template <int NW, bool GENERAL>
hipError_t start(const Args& a, int longest, hipStream_t st) {
  constexpr int lds = 2 * kBuffers * kTileBytes;
  const hipError_t e = RDKV_ALLOW_LDS((prompt_kernel<NW, GENERAL>), lds);
  if (e != hipSuccess) return e;
  const int tiles = (longest + 32 * NW - 1) / (32 * NW);
  hipLaunchKernelGGL((prompt_kernel<NW, GENERAL>), dim3(tiles * a.n_seqs * a.hq), dim3(64 * NW), lds, st, a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch(const Args& a, int longest, hipStream_t st) {
  const bool general = a.cap > 0.f || a.slopes;      // (a window takes no scores of its own)
  const int64_t large = static_cast<int64_t>(longest + 255) / 256 * a.n_seqs * a.hq;
  if (large >= 512) return general ? start<8, true>(a, longest, st) : start<8, false>(a, longest, st);
  return general ? start<4, true>(a, longest, st) : start<4, false>(a, longest, st);
}

}  // namespace prompt
}  // namespace rdkv
