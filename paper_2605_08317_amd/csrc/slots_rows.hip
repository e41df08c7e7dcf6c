// Slot caches: filling from prompts, appending, reading rows back.
#include "group_quant.h"
#include "slots.h"

namespace rdkv {
namespace slots {

namespace {

constexpr int kSelectThreads = 1024;

// sum over the workgroup's wavefronts below this one, and over all of them; v: this wavefront's
template <int WAVES>
__device__ __forceinline__ uint32_t waves_below(uint32_t v, uint32_t* s_waves, uint32_t* all) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  __syncthreads();
  if (lane == 0) s_waves[wave] = v;
  __syncthreads();
  uint32_t below = 0, sum = 0;
  for (int w = 0; w < WAVES; ++w) {
    if (w < wave) below += s_waves[w];
    sum += s_waves[w];
  }
  *all = sum;
  return below;
}

// Which tokens of an item stay: their positions and weights into the slots.  The weight that the last of the kept ones has is found
// digit by digit, from the highest (radix selection); a token stays if it is a sink, recent, above that weight, or one of the
// first of those at it.
__global__ __launch_bounds__(kSelectThreads) void fill_select_kernel(FillArgs a) {
  __shared__ uint32_t s_hist[256], s_waves[kSelectThreads / 64], s_digit[2];
  const int head = blockIdx.x, sl = blockIdx.y, tid = threadIdx.x, lane = tid & 63;
  const int T = a.T[sl], cap = a.s.capacity;
  const int64_t item = static_cast<int64_t>(a.seq0 + sl) * a.s.hkv + head;
  const float* w = a.w_tok ? a.w_tok + a.row0[sl] + static_cast<int64_t>(head) * T : nullptr;
  int32_t* pos = a.s.pos + item * cap;
  float* weight = a.s.weight ? a.s.weight + item * cap : nullptr;
  if (tid == 0) {
    a.s.len[item] = min(T, cap);
    a.s.next[item] = T;
  }
  if (T <= cap) {
    for (int t = tid; t < T; t += kSelectThreads) {
      pos[t] = t;
      if (weight) weight[t] = w ? w[t] : 0.f;
    }
    return;
  }
  const int lo = a.s.sinks, hi = T - a.s.recent;          // the tokens that may go
  uint32_t left = cap - a.s.sinks - a.s.recent;           // of them, so many stay
  uint32_t prefix = 0;
  if (left > 0)
    for (int shift = 24; shift >= 0; shift -= 8) {
      for (int i = tid; i < 256; i += kSelectThreads) s_hist[i] = 0;
      __syncthreads();
      for (int t = lo + tid; t < hi; t += kSelectThreads) {
        const uint32_t key = weight_key(w[t]);
        if (shift == 24 || (key >> (shift + 8)) == (prefix >> (shift + 8))) atomicAdd(&s_hist[(key >> shift) & 255u], 1u);
      }
      __syncthreads();
      if (tid == 0) {
        uint32_t n = left;
        int d = 255;
        for (; d > 0 && s_hist[d] < n; --d) n -= s_hist[d];
        s_digit[0] = d;
        s_digit[1] = n;
      }
      __syncthreads();
      prefix |= s_digit[0] << shift;
      left = s_digit[1];
    }
  // prefix: the weight at the border; left: how many at it stay
  uint32_t above = 0, ties = 0;                           // so far: tokens that stay for more than a tie, tokens at the border
  const bool none = cap == a.s.sinks + a.s.recent;
  for (int t0 = 0; t0 < T; t0 += kSelectThreads) {
    const int t = t0 + tid;
    bool stay = false, tie = false;
    if (t < T) {
      stay = t < lo || t >= hi;
      if (!stay && !none) {
        const uint32_t key = weight_key(w[t]);
        stay = key > prefix;
        tie = key == prefix;
      }
    }
    const uint64_t bs = __ballot(stay), bt = __ballot(tie), under = (1ull << lane) - 1;
    uint32_t all;
    const uint32_t mine = static_cast<uint32_t>(__popcll(bs)) | static_cast<uint32_t>(__popcll(bt)) << 16;
    const uint32_t below = waves_below<kSelectThreads / 64>(mine, s_waves, &all);
    const uint32_t my_ties = ties + (below >> 16) + __popcll(bt & under);
    const uint32_t at = above + (below & 0xFFFFu) + __popcll(bs & under) + min(my_ties, left);
    if (stay || (tie && my_ties < left)) {
      pos[at] = t;
      if (weight) weight[at] = w[t];
    }
    above += all & 0xFFFFu;
    ties += all >> 16;
  }
}

// bf16 rows: 16 lanes a row
__global__ __launch_bounds__(256) void fill_rows_kernel(FillArgs a) {
  const int head = blockIdx.y, sl = blockIdx.z, T = a.T[sl];
  const int64_t item = static_cast<int64_t>(a.seq0 + sl) * a.s.hkv + head, src = a.row0[sl] + static_cast<int64_t>(head) * T;
  const int i = blockIdx.x * 16 + (threadIdx.x >> 4), c = threadIdx.x & 15;
  if (i >= min(T, a.s.capacity)) return;
  const int64_t from = (src + a.s.pos[item * a.s.capacity + i]) * 16 + c, to = (item * a.s.capacity + i) * 16 + c;
  reinterpret_cast<uint4*>(a.s.k)[to] = reinterpret_cast<const uint4*>(a.K)[from];
  reinterpret_cast<uint4*>(a.s.v)[to] = reinterpret_cast<const uint4*>(a.V)[from];
}

// One tile of 64 slots in 4 bits, as the packing kernels quantize and lay out theirs: 16 lanes a row, four rows a lane.
template <bool EXACT>
__device__ __forceinline__ bool fill_tile(const uint4 (&kq)[4], const uint4 (&vq)[4], uint8_t* kt, uint8_t* vt, uint8_t* s_vc,
                                          uint16_t (*s_km)[8], int row0, int c16) {
  const int grp = c16 >> 2, p = c16 & 3;
  uint64_t odd = 0;
  uint32_t sc[4], of[4], packed[8];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    Quant q;
    uint32_t c[8];
    quantize_row<4, EXACT>(kq[i], 0, q, c);
    odd |= __builtin_amdgcn_ballot_w64(!q.finite);
    store_k_words<4>(c, kt + k_words_at<4>(grp, p) + 16 * (row0 + i), p);
    if (p == 0) {
      s_km[row0 + i][grp] = __builtin_bit_cast(unsigned short, q.sh);
      s_km[row0 + i][4 + grp] = __builtin_bit_cast(unsigned short, q.mh);
    }
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    Quant q;
    uint32_t c[8];
    quantize_row<4, EXACT>(vq[i], 0, q, c);
    odd |= __builtin_amdgcn_ballot_w64(!q.finite);
    sc[i] = __builtin_bit_cast(unsigned short, q.sh);
    of[i] = __builtin_bit_cast(unsigned short, q.mh);
#pragma unroll
    for (int j = 0; j < 8; ++j) packed[j] = i == 0 ? c[j] & 255u : packed[j] | (c[j] & 255u) << (8 * i);
  }
#pragma unroll
  for (int j = 0; j < 8; ++j) *reinterpret_cast<uint32_t*>(s_vc + (c16 * 8 + j) * kVcStride + row0) = packed[j];
  if (p == 0)
    *reinterpret_cast<uint4*>(vt + kTileCodes + 16 * row0 + 16 * grp) =
        make_uint4(sc[0] | (sc[1] << 16), sc[2] | (sc[3] << 16), of[0] | (of[1] << 16), of[2] | (of[3] << 16));
  return odd == 0;
}

__global__ __launch_bounds__(256) void fill_tiles_kernel(FillArgs a) {
  __shared__ __align__(16) uint8_t s_vc[kHeadDim * kVcStride];
  __shared__ __align__(16) uint16_t s_km[kTileRows][8];
  const int tile = blockIdx.x, head = blockIdx.y, sl = blockIdx.z, T = a.T[sl], n = min(T, a.s.capacity);
  if (tile * kTileRows >= n) return;
  const int64_t item = static_cast<int64_t>(a.seq0 + sl) * a.s.hkv + head, src = a.row0[sl] + static_cast<int64_t>(head) * T;
  const int tid = threadIdx.x, lane = tid & 63, c16 = lane & 15, row0 = 16 * (tid >> 6) + 4 * (lane >> 4);
  const int32_t* pos = a.s.pos + item * a.s.capacity;
  uint4 kq[4], vq[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int at = tile * kTileRows + row0 + i;
    const int64_t from = (src + pos[min(at, n - 1)]) * 16 + c16;
    kq[i] = reinterpret_cast<const uint4*>(a.K)[from];
    vq[i] = reinterpret_cast<const uint4*>(a.V)[from];
    if (at >= n) kq[i] = vq[i] = make_uint4(0, 0, 0, 0);
  }
  uint8_t* kt = a.s.k + (item * a.s.tiles + tile) * kTileBytes;
  uint8_t* vt = a.s.v + (item * a.s.tiles + tile) * kTileBytes;
  if (!fill_tile<false>(kq, vq, kt, vt, s_vc, s_km, row0, c16)) fill_tile<true>(kq, vq, kt, vt, s_vc, s_km, row0, c16);
  __syncthreads();
  store_v_words<4>(s_vc, vt);
  if (tid < kTileRows) *reinterpret_cast<uint4*>(kt + kTileCodes + 16 * tid) = *reinterpret_cast<const uint4*>(&s_km[tid][0]);
}

constexpr int kAppendThreads = 256;

template <int BITS>
__global__ __launch_bounds__(kAppendThreads) void append_kernel(Args a, const uint16_t* __restrict__ k_new,
                                                                const uint16_t* __restrict__ v_new, int32_t* __restrict__ slot_out) {
  __shared__ uint64_t s_key[kAppendThreads / 64];
  __shared__ int s_at[kAppendThreads / 64];
  const int64_t item = blockIdx.x;
  const int tid = threadIdx.x, lane = tid & 63, cap = a.capacity, n = a.length(item), next = a.next[item];
  int32_t* pos = a.pos + item * cap;
  int slot = n;
  if (n == cap) {
    // least weight, then lowest position; what may not go is behind everything else
    uint64_t best = ~0ull;
    int at = 0;
    for (int i = tid; i < cap; i += kAppendThreads) {
      const int p = pos[i];
      if (p < a.sinks || p > next - a.recent) continue;
      const uint64_t key = static_cast<uint64_t>(a.weight ? weight_key(a.weight[item * cap + i]) : 0u) << 32 | static_cast<uint32_t>(p);
      if (key < best) {
        best = key;
        at = i;
      }
    }
    for (int d = 1; d < 64; d <<= 1) {
      const uint64_t other = __shfl_xor(best, d);
      const int other_at = __shfl_xor(at, d);
      if (other < best || (other == best && other_at < at)) {
        best = other;
        at = other_at;
      }
    }
    if (lane == 0) {
      s_key[tid >> 6] = best;
      s_at[tid >> 6] = at;
    }
    __syncthreads();
    best = s_key[0];
    at = s_at[0];
    for (int w = 1; w < kAppendThreads / 64; ++w)
      if (s_key[w] < best || (s_key[w] == best && s_at[w] < at)) {
        best = s_key[w];
        at = s_at[w];
      }
    slot = at;
  }
  __syncthreads();                 // len, next and the arrays have been read
  if (tid == 0) {
    pos[slot] = next;
    if (a.weight) a.weight[item * cap + slot] = 0.f;
    a.len[item] = min(n + 1, cap);
    a.next[item] = next + 1;
    if (slot_out) slot_out[item] = slot;
  }
  if (tid >= 32) return;
  // lanes 0..15 K, 16..31 V
  const int c16 = tid & 15, grp = c16 >> 2, p = c16 & 3;
  const bool is_v = tid >= 16;
  const uint4 row = reinterpret_cast<const uint4*>(is_v ? v_new : k_new)[item * 16 + c16];
  uint8_t* side = is_v ? a.v : a.k;
  if constexpr (BITS == 16) {
    reinterpret_cast<uint4*>(side)[(item * cap + slot) * 16 + c16] = row;
  } else {
    Quant q;
    uint32_t c[8];
    quantize_row<4, true>(row, 0, q, c);
    uint8_t* tile = side + (item * a.tiles + slot / kTileRows) * kTileBytes;
    const int r = slot % kTileRows;
    uint16_t* meta = reinterpret_cast<uint16_t*>(tile + kTileCodes);
    if (!is_v) store_k_words<4>(c, tile + k_words_at<4>(grp, p) + 16 * r, p);
    if (is_v) {
      const int k = r & 31, shift = 16 * (k & 1) + 4 * ((k >> 2) & 3);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const int ch = c16 * 8 + j, word = 4 * (ch >> 5) + 2 * (k >> 4) + ((k >> 1) & 1);
        uint32_t* at = reinterpret_cast<uint32_t*>(tile + 1024 * (word >> 2) + 16 * (32 * (r >> 5) + (ch & 31)) + 4 * (word & 3));
        *at = (*at & ~(15u << shift)) | (c[j] & 15u) << shift;
      }
    }
    if (p == 0) {
      const int m = is_v ? 32 * (r >> 2) + 8 * grp + (r & 3) : 8 * r + grp;
      meta[m] = __builtin_bit_cast(unsigned short, q.sh);
      meta[m + 4] = __builtin_bit_cast(unsigned short, q.mh);
    }
  }
}

// nearest bf16, ties to even (NaN stays one)
__device__ __forceinline__ uint32_t to_bf16(float x) {
  const uint32_t u = __float_as_uint(x);
  if ((u & 0x7FFFFFFFu) > 0x7F800000u) return (u >> 16) | 0x40u;
  return (u + 0x7FFFu + ((u >> 16) & 1u)) >> 16;
}

template <int BITS>
__global__ __launch_bounds__(256) void read_kernel(Args a, const int32_t* __restrict__ index, int n, int groups, uint16_t* __restrict__ K,
                                                   uint16_t* __restrict__ V) {
  const int64_t item = blockIdx.x / groups;
  const int i = static_cast<int>(blockIdx.x % groups) * 16 + (threadIdx.x >> 4), c16 = threadIdx.x & 15;
  if (i >= n) return;
  const int slot = index ? index[item * n + i] : i;
  const int64_t to = (item * n + i) * 16 + c16;
  uint4 kq = make_uint4(0, 0, 0, 0), vq = kq;
  if (slot >= 0 && slot < a.length(item)) {
    if constexpr (BITS == 16) {
      kq = reinterpret_cast<const uint4*>(a.k)[(item * a.capacity + slot) * 16 + c16];
      vq = reinterpret_cast<const uint4*>(a.v)[(item * a.capacity + slot) * 16 + c16];
    } else {
      const int r = slot % kTileRows;
      const uint8_t* kt = a.k + (item * a.tiles + slot / kTileRows) * kTileBytes;
      const uint8_t* vt = a.v + (item * a.tiles + slot / kTileRows) * kTileBytes;
      const _Float16* km = reinterpret_cast<const _Float16*>(kt + kTileCodes);
      const _Float16* vm = reinterpret_cast<const _Float16*>(vt + kTileCodes);
      uint32_t ko[8], vo[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const int c = c16 * 8 + j, grp = c >> 5;
        const auto code = [&](const uint8_t* tile, int lane, int k) {
          const int word = 4 * grp + 2 * (k >> 4) + ((k >> 1) & 1);
          return *reinterpret_cast<const uint32_t*>(tile + 1024 * (word >> 2) + 16 * lane + 4 * (word & 3)) >>
                     (16 * (k & 1) + 4 * ((k >> 2) & 3)) & 15u;
        };
        const float ks = km[8 * r + grp], kz = km[8 * r + 4 + grp];
        const int m = 32 * (r >> 2) + 8 * grp + (r & 3);
        const float vs = vm[m], vz = vm[m + 4];
        ko[j] = to_bf16(ks * static_cast<float>(code(kt, r, c & 31)) + kz);
        vo[j] = to_bf16(vs * static_cast<float>(code(vt, 32 * (r >> 5) + (c & 31), r & 31)) + vz);
      }
      kq = make_uint4(ko[0] | ko[1] << 16, ko[2] | ko[3] << 16, ko[4] | ko[5] << 16, ko[6] | ko[7] << 16);
      vq = make_uint4(vo[0] | vo[1] << 16, vo[2] | vo[3] << 16, vo[4] | vo[5] << 16, vo[6] | vo[7] << 16);
    }
  }
  reinterpret_cast<uint4*>(K)[to] = kq;
  reinterpret_cast<uint4*>(V)[to] = vq;
}

}  // namespace

hipError_t launch_fill(const FillArgs& a, int n_seqs, int bits, hipStream_t st) {
  int most = 0;
  for (int i = 0; i < n_seqs; ++i) most = a.T[i] > most ? a.T[i] : most;
  const int n = most < a.s.capacity ? most : a.s.capacity;
  hipLaunchKernelGGL(fill_select_kernel, dim3(a.s.hkv, n_seqs), dim3(kSelectThreads), 0, st, a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || n == 0) return e;
  if (bits == 16)
    hipLaunchKernelGGL(fill_rows_kernel, dim3((n + 15) / 16, a.s.hkv, n_seqs), dim3(256), 0, st, a);
  else
    hipLaunchKernelGGL(fill_tiles_kernel, dim3((n + kTileRows - 1) / kTileRows, a.s.hkv, n_seqs), dim3(256), 0, st, a);
  return hipGetLastError();
}

hipError_t launch_append(const Args& a, int bits, int items, const uint16_t* k_new, const uint16_t* v_new, int32_t* slot, hipStream_t st) {
  if (bits == 16)
    hipLaunchKernelGGL(append_kernel<16>, dim3(items), dim3(kAppendThreads), 0, st, a, k_new, v_new, slot);
  else
    hipLaunchKernelGGL(append_kernel<4>, dim3(items), dim3(kAppendThreads), 0, st, a, k_new, v_new, slot);
  return hipGetLastError();
}

hipError_t launch_read(const Args& a, int bits, int items, const int32_t* index, int n, uint16_t* K, uint16_t* V, hipStream_t st) {
  const int groups = (n + 15) / 16;        // (of 16 rows; less than 2^27 in all)
  if (bits == 16)
    hipLaunchKernelGGL(read_kernel<16>, dim3(groups * items), dim3(256), 0, st, a, index, n, groups, K, V);
  else
    hipLaunchKernelGGL(read_kernel<4>, dim3(groups * items), dim3(256), 0, st, a, index, n, groups, K, V);
  return hipGetLastError();
}

}  // namespace slots
}  // namespace rdkv
