// Slot caches: filling from prompts, appending, reading rows back.
#include "group_quant.h"
#include "slots.h"

namespace rdkv {
namespace slots {

namespace {

constexpr int kSelectThreads = 1024, kSelectWaves = kSelectThreads / 64;

// Sums over the threads below this one; x0, x1: this thread's own.
template <int WAVES>
struct Scan {
  uint32_t s_wave[2][WAVES];
  __device__ __forceinline__ void run(uint32_t x0, uint32_t x1, uint32_t& below0, uint32_t& below1) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const uint32_t up0 = wave_scan(x0), up1 = wave_scan(x1);
    __syncthreads();
    if (lane == 63) {
      s_wave[0][wave] = up0;
      s_wave[1][wave] = up1;
    }
    __syncthreads();
    below0 = up0 - x0;
    below1 = up1 - x1;
#pragma unroll
    for (int w = 0; w < WAVES; ++w)
      if (w < wave) {
        below0 += s_wave[0][w];
        below1 += s_wave[1][w];
      }
  }
};

// An item of a fill: its prompt's weights as numbers to select by.
struct Prompt {
  int T, cap, lo, hi;
  const float* w;
  int32_t* pos;
  float* weight;
  __device__ __forceinline__ Prompt(const FillArgs& a, int head, int sl) {
    T = a.T[sl];
    cap = a.s.capacity;
    const int64_t item = static_cast<int64_t>(a.seq0 + sl) * a.s.hkv + head;
    w = a.w_tok ? a.w_tok + a.row0[sl] + static_cast<int64_t>(head) * T : nullptr;
    pos = a.s.pos + item * cap;
    weight = a.s.weight ? a.s.weight + item * cap : nullptr;
    lo = a.s.sinks;
    hi = T - a.s.recent;
  }
  // sinks and recent tokens above every weight
  __device__ __forceinline__ uint32_t key(int t, float x) const { return t < lo || t >= hi ? 0xFFFFFFFFu : weight_key(x); }
  __device__ __forceinline__ void lengths(const FillArgs& a, int head, int sl) const {
    const int64_t item = static_cast<int64_t>(a.seq0 + sl) * a.s.hkv + head;
    a.s.len[item] = min(T, cap);
    a.s.next[item] = T;
  }
  // tokens first, first + step, .. below `end` of a prompt that stays whole
  __device__ __forceinline__ void keep_all(int first, int end, int step) const {
    for (int t = first; t < end; t += step) {
      pos[t] = t;
      if (weight) weight[t] = w ? w[t] : 0.f;
    }
  }
  __device__ __forceinline__ void keep(int at, int t, float x) const {      // x: w[t]
    pos[at] = t;
    if (weight) weight[at] = x;
  }
};

// Which tokens of an item stay: their positions and weights into the slots.  Weights become unsigned numbers of the same order; the
// capacity's largest stay, found digit by digit from the highest (radix selection: 11, 11 and 10 bits), the first of equal ones before the
// later.
//
// Short prompts: one workgroup an item, its weights in the threads' registers.  A pass counts digits in LDS, with four counters a digit
// that lanes take in turn: weights share their few exponents, and lanes on one counter wait for each other.  Bound: latency.
constexpr int kCopies = 4, kDigits = kSelectDigits;
template <int REGS>      // prompts of up to REGS kSelectThreads tokens, and those that stay whole
__global__ __launch_bounds__(kSelectThreads) void fill_select_kernel(FillArgs a) {
  constexpr int kEntries = REGS * kSelectWaves;
  static_assert(kEntries <= kSelectThreads && 3 * kEntries <= kDigits * kCopies, "an entry a thread");
  __shared__ uint32_t s_hist[kDigits * kCopies];          // later what stays of (register, wavefront), and sums before it
  __shared__ Scan<kSelectWaves> s_scan;
  __shared__ uint32_t s_found[2];
  const int head = blockIdx.x, sl = blockIdx.y, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const Prompt it(a, head, sl);
  const int T = it.T;
  if (tid == 0) it.lengths(a, head, sl);
  if (T <= it.cap) {
    it.keep_all(tid, T, kSelectThreads);
    return;
  }
  uint32_t keys[REGS];                                    // token i kSelectThreads + tid
  float x[REGS];
#pragma unroll
  for (int i = 0; i < REGS; ++i) x[i] = it.w[min(i * kSelectThreads + tid, T - 1)];
#pragma unroll
  for (int i = 0; i < REGS; ++i) keys[i] = it.key(i * kSelectThreads + tid, x[i]);
  uint32_t left = it.cap, border = 0;                     // how many stay of what is in question: keys that begin as border does
  const auto pass = [&](int shift, int bits, int above) __attribute__((always_inline)) {
    __syncthreads();
    for (int i = tid; i < kDigits * kCopies; i += kSelectThreads) s_hist[i] = 0;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < REGS; ++i)
      if (i * kSelectThreads + tid < T && (above == 32 || (keys[i] >> above) == (border >> above)))
        atomicAdd(&s_hist[((keys[i] >> shift) & ((1u << bits) - 1)) * kCopies + (lane & (kCopies - 1))], 1u);
    __syncthreads();
    uint32_t n[2] = {0, 0};                               // of digits 2047 - 2 tid and the one below
#pragma unroll
    for (int e = 0; e < 2; ++e)
#pragma unroll
      for (int c = 0; c < kCopies; ++c) n[e] += s_hist[(kDigits - 1 - 2 * tid - e) * kCopies + c];
    uint32_t higher, unused;
    s_scan.run(n[0] + n[1], 0, higher, unused);
    if (higher < left && left <= higher + n[0] + n[1]) {
      const int e = left > higher + n[0];
      s_found[0] = kDigits - 1 - 2 * tid - e;
      s_found[1] = left - higher - (e ? n[0] : 0);
    }
    __syncthreads();
    border |= s_found[0] << shift;
    left = s_found[1];
  };
  pass(21, 11, 32);
  pass(10, 11, 21);
  pass(0, 10, 10);
  // Their slots.  For every (register, wavefront), in the order of tokens: how many are above the border, how many at it
  uint64_t sure, tie;
  const auto vote = [&](int i) __attribute__((always_inline)) {
    uint32_t k = keys[i];
    asm volatile("" : "+v"(k));                           // (or both loops' votes are kept for the other)
    const bool in = i * kSelectThreads + tid < T;
    sure = __ballot(in && k > border);
    tie = __ballot(in && k == border);
  };
  __syncthreads();
#pragma unroll
  for (int i = 0; i < REGS; ++i) {
    vote(i);
    if (lane == 0) s_hist[i * kSelectWaves + wave] = static_cast<uint32_t>(__popcll(sure)) | static_cast<uint32_t>(__popcll(tie)) << 16;
  }
  __syncthreads();
  const uint32_t mine = tid < kEntries ? s_hist[tid] : 0u;
  uint32_t sure_before, ties_before;
  s_scan.run(mine & 0xFFFFu, mine >> 16, sure_before, ties_before);
  if (tid < kEntries) {
    s_hist[kEntries + tid] = sure_before;
    s_hist[2 * kEntries + tid] = ties_before;
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < REGS; ++i) {
    if (i * kSelectThreads >= T) break;
    vote(i);
    const uint64_t under = (1ull << lane) - 1, me = 1ull << lane;
    const uint32_t ties = s_hist[2 * kEntries + i * kSelectWaves + wave] + __popcll(tie & under);
    const uint32_t at = s_hist[kEntries + i * kSelectWaves + wave] + __popcll(sure & under) + min(ties, left);
    if ((sure & me) || ((tie & me) && ties < left)) it.keep(at, i * kSelectThreads + tid, x[i]);
  }
}

// Long prompts: an item in parts, a workgroup each, in three launches.  count: a part's weights by their first digit.  open: every part
// adds up the counts of all, finds the digit at the border, and puts its weights at that digit into a list of the item's, in the order of
// tokens.  place: every part goes through the list, some hundredths of the weights, for the other two digits, and knows from it what the
// parts before it keep.  Bound: latency of three launches; 4 bytes a token twice.
// 8 items of 32K tokens, 4K kept: 4.5, 6.4 and 9.8 us; of 128K with many ties, 32K kept: 4.8, 9.4 and 10.7 (one workgroup an item took 32 us
// for 32K and 128 for 128K).  Workgroups of 256 threads 5.8, 7.8, 12.6 and of 1024 3.8, 5.8, 8.9, but 128 items of up to 32K then 49 us in
// all, and 36 with 512.
constexpr int kPartBlock = 4096, kPartThreads = 512, kPartWaves = kPartThreads / 64, kPartEach = kPartBlock / kPartThreads;

struct PartOf {
  int g, head, sl, tid, t0, t1;       // part of the item; its tokens
  int64_t local;                      // item of the launch
  __device__ __forceinline__ PartOf(const FillArgs& a) {
    g = blockIdx.x;
    head = blockIdx.y;
    sl = blockIdx.z;
    tid = threadIdx.x;
    local = static_cast<int64_t>(sl) * a.s.hkv + head;
    t0 = g * a.part_rows;
    t1 = t0 + min(a.part_rows, a.T[sl] - t0);      // (t0, if there are none)
  }
};
// weights of tokens t + i kPartThreads + tid (t < t1), and their keys
__device__ __forceinline__ void load_weights(const Prompt& it, int t, int t1, int tid, float (&x)[kPartEach]) {
#pragma unroll
  for (int i = 0; i < kPartEach; ++i) x[i] = it.w[min(t + i * kPartThreads + tid, t1 - 1)];
}
__device__ __forceinline__ void make_keys(const Prompt& it, int t, int tid, const float (&x)[kPartEach], uint32_t (&keys)[kPartEach]) {
#pragma unroll
  for (int i = 0; i < kPartEach; ++i) keys[i] = it.key(t + i * kPartThreads + tid, x[i]);
}
// sums over (i, wavefront) entries before each, of packed pairs of 16 bits (a block has 4096 tokens); s_entries: kPartEach x kPartWaves
__device__ __forceinline__ void scan_entries(uint2* s_entries, uint2* all) {
  static_assert(kPartEach * kPartWaves == 64, "an entry a lane");
  __syncthreads();
  if (threadIdx.x < 64) {
    const uint2 x = s_entries[threadIdx.x];
    const uint2 up = make_uint2(wave_scan(x.x), wave_scan(x.y));
    s_entries[threadIdx.x] = make_uint2(up.x - x.x, up.y - x.y);
    if (threadIdx.x == 63) *all = up;
  }
  __syncthreads();
}

__global__ __launch_bounds__(kPartThreads) void select_count_kernel(FillArgs a) {
  __shared__ uint32_t s_hist[kDigits * kCopies];
  const PartOf p(a);
  const Prompt it(a, p.head, p.sl);
  if (p.g == 0 && p.tid == 0) it.lengths(a, p.head, p.sl);
  if (p.t0 >= it.T) return;
  if (it.T <= it.cap) {
    it.keep_all(p.t0 + p.tid, p.t1, kPartThreads);
    return;
  }
  for (int i = p.tid; i < kDigits * kCopies; i += kPartThreads) s_hist[i] = 0;
  __syncthreads();
  for (int t = p.t0; t < p.t1; t += kPartBlock) {
    float x[kPartEach];
    uint32_t keys[kPartEach];
    load_weights(it, t, p.t1, p.tid, x);
    make_keys(it, t, p.tid, x, keys);
#pragma unroll
    for (int i = 0; i < kPartEach; ++i)
      if (t + i * kPartThreads + p.tid < p.t1) atomicAdd(&s_hist[(keys[i] >> 21) * kCopies + (p.tid & (kCopies - 1))], 1u);
  }
  __syncthreads();
  uint32_t* out = reinterpret_cast<uint32_t*>(a.counts + (p.local * a.parts + p.g) * kDigits);
  for (int i = p.tid; i < kDigits / 2; i += kPartThreads) {
    uint32_t n[2] = {0, 0};
#pragma unroll
    for (int e = 0; e < 2; ++e)
#pragma unroll
      for (int c = 0; c < kCopies; ++c) n[e] += s_hist[(2 * i + e) * kCopies + c];
    out[i] = n[0] | n[1] << 16;
  }
}

// The digit (a thread has PER of them, the highest first: digits first - k) in which the `left` largest end; n: their counts.
template <int PER>
__device__ __forceinline__ uint2 find_digit(Scan<kPartWaves>& scan, uint2* s_found, uint32_t left, int first, const uint32_t (&n)[PER]) {
  uint32_t sum = 0, higher, unused;
#pragma unroll
  for (int k = 0; k < PER; ++k) sum += n[k];
  scan.run(sum, 0, higher, unused);
  if (higher < left && left <= higher + sum) {
#pragma unroll
    for (int k = 0; k < PER; ++k) {
      if (higher < left && left <= higher + n[k]) *s_found = make_uint2(first - k, left - higher);
      higher += n[k];
    }
  }
  __syncthreads();
  return *s_found;
}

__global__ __launch_bounds__(kPartThreads) void select_open_kernel(FillArgs a) {
  __shared__ Scan<kPartWaves> s_scan;
  __shared__ uint2 s_found, s_all, s_entries[kPartEach * kPartWaves];
  __shared__ uint32_t s_sum[3];
  const PartOf p(a);
  const Prompt it(a, p.head, p.sl);
  if (p.t0 >= it.T || it.T <= it.cap) return;
  const int parts = (it.T + a.part_rows - 1) / a.part_rows, lane = p.tid & 63, wave = p.tid >> 6;
  float x[kPartEach];                  // of the block; the first is under way during what comes before it
  load_weights(it, p.t0, p.t1, p.tid, x);
  const uint16_t* counts = a.counts + p.local * a.parts * kDigits;
  // a few digits a thread, thread 0 the highest
  constexpr int kPer = kDigits / kPartThreads;
  using Counts = __attribute__((ext_vector_type(kPer / 2))) uint32_t;
  const int at = kDigits - kPer * (p.tid + 1);
  uint32_t n[kPer], own[kPer];
#pragma unroll
  for (int k = 0; k < kPer; ++k) n[k] = own[k] = 0;
#pragma unroll 8
  for (int g = 0; g < parts; ++g) {
    const Counts c = *reinterpret_cast<const Counts*>(counts + static_cast<int64_t>(g) * kDigits + at);
#pragma unroll
    for (int k = 0; k < kPer; ++k) {
      const uint32_t x = (c[kPer / 2 - 1 - k / 2] >> (k % 2 ? 0 : 16)) & 0xFFFFu;
      n[k] += x;
      own[k] = g == p.g ? x : own[k];
    }
  }
  if (p.tid < 3) s_sum[p.tid] = 0;
  const uint2 f = find_digit<kPer>(s_scan, &s_found, it.cap, kDigits - 1 - kPer * p.tid, n);
  const uint32_t digit = f.x;
  uint32_t sure = 0;
#pragma unroll
  for (int k = 0; k < kPer; ++k)
    if (static_cast<uint32_t>(kDigits - 1 - kPer * p.tid - k) > digit) sure += own[k];
  uint32_t before = 0, all = 0;
  for (int g = p.tid; g < parts; g += kPartThreads) {
    const uint32_t x = counts[static_cast<int64_t>(g) * kDigits + digit];
    all += x;
    if (g < p.g) before += x;
  }
  if (sure) atomicAdd(&s_sum[0], sure);
  if (before) atomicAdd(&s_sum[1], before);
  if (all) atomicAdd(&s_sum[2], all);
  __syncthreads();
  before = s_sum[1];
  if (p.tid == 0) {
    a.part[p.local * a.parts + p.g] = make_int2(static_cast<int>(s_sum[0]), static_cast<int>(before));
    if (p.g == 0) a.found[p.local] = make_int4(static_cast<int>(digit), static_cast<int>(f.y), static_cast<int>(s_sum[2]), 0);
  }
  uint32_t* list = a.open + (a.row0[p.sl] - a.row0[0]) + static_cast<int64_t>(p.head) * it.T;
  for (int t = p.t0; t < p.t1; t += kPartBlock) {
    uint32_t keys[kPartEach];
    make_keys(it, t, p.tid, x, keys);
    if (t + kPartBlock < p.t1) load_weights(it, t + kPartBlock, p.t1, p.tid, x);
    uint64_t in[kPartEach];
#pragma unroll
    for (int i = 0; i < kPartEach; ++i) {
      in[i] = __ballot(t + i * kPartThreads + p.tid < p.t1 && (keys[i] >> 21) == digit);
      if (lane == 0) s_entries[i * kPartWaves + wave] = make_uint2(__popcll(in[i]), 0);
    }
    scan_entries(s_entries, &s_all);
#pragma unroll
    for (int i = 0; i < kPartEach; ++i)
      if ((in[i] >> lane) & 1) list[before + s_entries[i * kPartWaves + wave].x + __popcll(in[i] & ((1ull << lane) - 1))] = keys[i];
    before += s_all.x;
    __syncthreads();
  }
}

__global__ __launch_bounds__(kPartThreads) void select_place_kernel(FillArgs a) {
  __shared__ uint32_t s_hist[kDigits];
  __shared__ Scan<kPartWaves> s_scan;
  __shared__ uint2 s_found, s_all, s_entries[kPartEach * kPartWaves];
  __shared__ uint32_t s_sum[2];
  const PartOf p(a);
  const Prompt it(a, p.head, p.sl);
  if (p.t0 >= it.T || it.T <= it.cap) return;
  const int lane = p.tid & 63, wave = p.tid >> 6;
  const int4 found = a.found[p.local];
  const int2 own = a.part[p.local * a.parts + p.g];
  const int open = found.z;
  float x[kPartEach];                  // of the block; the first is under way during what comes before it
  load_weights(it, p.t0, p.t1, p.tid, x);
  uint32_t left = found.y, border = static_cast<uint32_t>(found.x) << 21;
  const uint32_t* list = a.open + (a.row0[p.sl] - a.row0[0]) + static_cast<int64_t>(p.head) * it.T;
  // the first of the list's weights stay with their threads
  constexpr int kHold = 4096 / kPartThreads;
  uint32_t held[kHold];
#pragma unroll
  for (int i = 0; i < kHold; ++i) held[i] = list[min(i * kPartThreads + p.tid, open - 1)];
  const auto each = [&](auto&& f) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < kHold; ++i)
      if (i * kPartThreads + p.tid < open) f(held[i], i * kPartThreads + p.tid);
    for (int i = kHold * kPartThreads + p.tid; i < open; i += kPartThreads) f(list[i], i);
  };
  constexpr int kPer = kDigits / kPartThreads;
#pragma unroll
  for (int pass = 0; pass < 2; ++pass) {
    const int shift = pass == 0 ? 10 : 0, above = pass == 0 ? 21 : 10;
    __syncthreads();
    for (int i = p.tid; i < kDigits; i += kPartThreads) s_hist[i] = 0;
    __syncthreads();
    each([&](uint32_t k, int) {
      if ((k >> above) == (border >> above)) atomicAdd(&s_hist[(k >> shift) & (pass == 0 ? 2047u : 1023u)], 1u);
    });
    __syncthreads();
    uint32_t n[kPer];
#pragma unroll
    for (int k = 0; k < kPer; ++k) n[k] = s_hist[kDigits - 1 - kPer * p.tid - k];
    const uint2 f = find_digit<kPer>(s_scan, &s_found, left, kDigits - 1 - kPer * p.tid, n);
    border |= f.x << shift;
    left = f.y;
  }
  // what the parts before keep: all above the border digit, and of the list's
  if (p.tid < 2) s_sum[p.tid] = 0;
  __syncthreads();
  uint32_t sure = 0, ties = 0;
  for (int g = p.tid; g < p.g; g += kPartThreads) sure += static_cast<uint32_t>(a.part[p.local * a.parts + g].x);
  each([&](uint32_t k, int i) {
    if (i < own.y) {
      sure += k > border;
      ties += k == border;
    }
  });
  if (sure) atomicAdd(&s_sum[0], sure);
  if (ties) atomicAdd(&s_sum[1], ties);
  __syncthreads();
  sure = s_sum[0];
  ties = s_sum[1];
  for (int t = p.t0; t < p.t1; t += kPartBlock) {
    uint32_t keys[kPartEach];
    if (t > p.t0) load_weights(it, t, p.t1, p.tid, x);
    make_keys(it, t, p.tid, x, keys);
    uint64_t more[kPartEach], same[kPartEach];
#pragma unroll
    for (int i = 0; i < kPartEach; ++i) {
      const bool in = t + i * kPartThreads + p.tid < p.t1;
      more[i] = __ballot(in && keys[i] > border);
      same[i] = __ballot(in && keys[i] == border);
      if (lane == 0) s_entries[i * kPartWaves + wave] = make_uint2(__popcll(more[i]), __popcll(same[i]));
    }
    scan_entries(s_entries, &s_all);
    const uint64_t under = (1ull << lane) - 1, me = 1ull << lane;
#pragma unroll
    for (int i = 0; i < kPartEach; ++i) {
      const uint2 b = s_entries[i * kPartWaves + wave];
      const uint32_t tie = ties + b.y + __popcll(same[i] & under);
      if ((more[i] & me) || ((same[i] & me) && tie < left)) 
        it.keep(sure + b.x + __popcll(more[i] & under) + min(tie, left), t + i * kPartThreads + p.tid, x[i]);
    }
    sure += s_all.x;
    ties += s_all.y;
    __syncthreads();
  }
}

// sixteen bytes of a prompt's row, which is read once
__device__ __forceinline__ uint4 prompt_row(const uint16_t* rows, int64_t at) {
  using Four = __attribute__((ext_vector_type(4))) uint32_t;
  const Four v = __builtin_nontemporal_load(reinterpret_cast<const Four*>(rows) + at);
  return make_uint4(v[0], v[1], v[2], v[3]);
}

// bf16 rows: 16 lanes a row.  Bound: latency; 8 items of 4K slots, 34 MB moved, 7.5 us.
__global__ __launch_bounds__(256) void fill_rows_kernel(FillArgs a) {
  const int head = blockIdx.y, sl = blockIdx.z, T = a.T[sl];
  const int64_t item = static_cast<int64_t>(a.seq0 + sl) * a.s.hkv + head, src = a.row0[sl] + static_cast<int64_t>(head) * T;
  const int i = blockIdx.x * 16 + (threadIdx.x >> 4), c = threadIdx.x & 15;
  if (i >= min(T, a.s.capacity)) return;
  const int64_t from = (src + a.s.pos[item * a.s.capacity + i]) * 16 + c, to = (item * a.s.capacity + i) * 16 + c;
  const uint4 k = prompt_row(a.K, from), v = prompt_row(a.V, from);
  reinterpret_cast<uint4*>(a.s.k)[to] = k;
  reinterpret_cast<uint4*>(a.s.v)[to] = v;
}

// One tile of 64 slots in 4 bits, as the packing kernels quantize and lay out theirs: 16 lanes a row, four rows a lane, so that a lane has
// the four codes of a channel that a V word begins with.  Bound: HBM, 256 bytes read and 80 written a row and side; 128 items of 4K
// slots 66 us, 5.2 TB/s.
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
  const int at = tile * kTileRows + row0;
  uint4 kq[4], vq[4];
  int p[4];                                // all positions, then all rows
#pragma unroll
  for (int i = 0; i < 4; ++i) p[i] = pos[min(at + i, n - 1)];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int64_t from = (src + p[i]) * 16 + c16;
    kq[i] = prompt_row(a.K, from);
    vq[i] = prompt_row(a.V, from);
  }
  if (tile * kTileRows + kTileRows > n) {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (at + i >= n) kq[i] = vq[i] = make_uint4(0, 0, 0, 0);
  }
  uint8_t* kt = a.s.k + (item * a.s.tiles + tile) * kTileBytes;
  uint8_t* vt = a.s.v + (item * a.s.tiles + tile) * kTileBytes;
  if (!fill_tile<false>(kq, vq, kt, vt, s_vc, s_km, row0, c16)) fill_tile<true>(kq, vq, kt, vt, s_vc, s_km, row0, c16);
  __syncthreads();
  store_v_words<4>(s_vc, vt);
  if (tid < kTileRows) *reinterpret_cast<uint4*>(kt + kTileCodes + 16 * tid) = *reinterpret_cast<const uint4*>(&s_km[tid][0]);
}

// A token into an item.  In a full one the least of (weight, position) among what may go is found by the whole workgroup, kEach slots of a
// thread under way at once; the first lanes have the token's rows by then.  Bound: latency; 8 bytes a slot.  256 items of 8K slots 6.7 us (17 MB), 2 of
// 1000 4.5.
constexpr int kAppendThreads = 1024, kAppendWaves = kAppendThreads / 64;

template <int BITS>
__global__ __launch_bounds__(kAppendThreads) void append_kernel(Args a, const uint16_t* __restrict__ k_new,
                                                                const uint16_t* __restrict__ v_new, int32_t* __restrict__ slot_out) {
  constexpr int kEach = 8;
  __shared__ uint64_t s_key[kAppendWaves];
  __shared__ int s_at[kAppendWaves];
  const int64_t item = blockIdx.x;
  const int tid = threadIdx.x, lane = tid & 63, cap = a.capacity;
  // lanes 0..15 hold the new K row, 16..31 the V row
  const int c16 = tid & 15, grp = c16 >> 2, p = c16 & 3;
  const bool is_v = tid >= 16;
  uint4 row = make_uint4(0, 0, 0, 0);
  if (tid < 32) row = reinterpret_cast<const uint4*>(is_v ? v_new : k_new)[item * 16 + c16];
  const int n = a.length(item), next = a.next[item];
  int32_t* pos = a.pos + item * cap;
  int slot = n;
  if (n == cap) {
    // least weight, then lowest position; what may not go is behind everything else
    uint64_t best = ~0ull;
    int at = 0;
    const float* weight = a.weight ? a.weight + item * cap : nullptr;
    for (int i0 = tid; i0 < cap; i0 += kEach * kAppendThreads) {
      int at_pos[kEach];
      float w[kEach];
#pragma unroll
      for (int k = 0; k < kEach; ++k) {
        const int i = min(i0 + k * kAppendThreads, cap - 1);
        at_pos[k] = pos[i];
        w[k] = weight ? weight[i] : 0.f;
      }
#pragma unroll
      for (int k = 0; k < kEach; ++k) {
        const int i = i0 + k * kAppendThreads;
        const uint64_t key = static_cast<uint64_t>(weight_key(w[k])) << 32 | static_cast<uint32_t>(at_pos[k]);
        if (i < cap && at_pos[k] >= a.sinks && at_pos[k] <= next - a.recent && key < best) {
          best = key;
          at = i;
        }
      }
    }
    const auto least = [&](uint64_t other, int other_at) __attribute__((always_inline)) {
      if (other < best || (other == best && other_at < at)) {
        best = other;
        at = other_at;
      }
    };
    for (int d = 1; d < 64; d <<= 1) {
      const uint64_t other = __shfl_xor(best, d);
      least(other, __shfl_xor(at, d));
    }
    if (lane == 0) {
      s_key[tid >> 6] = best;
      s_at[tid >> 6] = at;
    }
    __syncthreads();
    best = s_key[lane & (kAppendWaves - 1)];
    at = s_at[lane & (kAppendWaves - 1)];
    for (int d = 1; d < kAppendWaves; d <<= 1) {
      const uint64_t other = __shfl_xor(best, d);
      least(other, __shfl_xor(at, d));
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

typedef float float2v __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
// scale x code + offset of two values, as bf16
__device__ __forceinline__ uint32_t two_values(uint32_t c0, uint32_t c1, float s0, float s1, float z0, float z1) {
  return __builtin_bit_cast(uint32_t, __builtin_convertvector((float2v{s0 * static_cast<float>(c0) + z0, s1 * static_cast<float>(c1) + z1}), bf16x2));
}
__device__ __forceinline__ float half_of(uint32_t w, int h) { return static_cast<float>(__builtin_bit_cast(_Float16, static_cast<uint16_t>(h ? w >> 16 : w))); }

// Tiles of 4-bit rows, slot after slot.  A workgroup has a tile, a lane eight channels of four rows, as where tiles are filled.  V words
// hold a channel's four rows together and pass through LDS (a group's words 16 bytes apart from where the next's would fall on the same
// banks).  Bound: HBM, 80 bytes read and 256 written a row and side; 4 x 8 items of 32K slots 123 us, 5.2 TB/s.
constexpr int kGroupStride = 1024 + 64, kBlockPad = 16;       // of 8 lanes' words
__global__ __launch_bounds__(256) void read_tiles_kernel(Args a, int n, int groups, uint16_t* __restrict__ K, uint16_t* __restrict__ V) {
  __shared__ __align__(16) uint8_t s_v[4 * (kGroupStride + 8 * kBlockPad)];
  const int64_t item = blockIdx.x / groups;
  const int tile = static_cast<int>(blockIdx.x % groups), tid = threadIdx.x, lane = tid & 63;
  const int c16 = lane & 15, grp = c16 >> 2, p = c16 & 3, row0 = 16 * (tid >> 6) + 4 * (lane >> 4);
  const int len = min(a.length(item), n);
  uint16_t* k_out = K + (item * n + static_cast<int64_t>(tile) * kTileRows) * kHeadDim;
  uint16_t* v_out = V + (item * n + static_cast<int64_t>(tile) * kTileRows) * kHeadDim;
  const int rows = min(kTileRows, n - tile * kTileRows), held = len - tile * kTileRows;      // to write; of them with a token
  uint4 kq[4], vq[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) kq[i] = vq[i] = make_uint4(0, 0, 0, 0);
  if (held > 0) {
    const uint8_t* kt = a.k + (item * a.tiles + tile) * kTileBytes;
    const uint8_t* vt = a.v + (item * a.tiles + tile) * kTileBytes;
    const uint4 raw = *reinterpret_cast<const uint4*>(vt + 16 * tid);
    uint2 kw[4];
    uint4 km[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      kw[i] = *reinterpret_cast<const uint2*>(kt + 1024 * grp + 16 * (row0 + i) + 8 * (p >> 1));
      km[i] = *reinterpret_cast<const uint4*>(kt + kTileCodes + 16 * (row0 + i));
    }
    const uint4 vm = *reinterpret_cast<const uint4*>(vt + kTileCodes + 16 * row0 + 16 * grp);
    const auto v_at = [](int g, int l) { return g * (kGroupStride + 8 * kBlockPad) + 16 * l + kBlockPad * (l >> 3); };
    *reinterpret_cast<uint4*>(s_v + v_at(tid >> 6, lane)) = raw;
#pragma unroll
    for (int i = 0; i < 4; ++i) {        // codes 8 p .. of the group: fields 2 (p % 2) and the next of word pair p / 2
      const uint32_t w0 = kw[i].x >> (8 * (p & 1)), w1 = kw[i].y >> (8 * (p & 1));
      const float s = half_of(grp < 2 ? km[i].x : km[i].y, grp & 1), z = half_of(grp < 2 ? km[i].z : km[i].w, grp & 1);
      kq[i].x = two_values(w0 & 15u, (w0 >> 16) & 15u, s, s, z, z);
      kq[i].y = two_values(w1 & 15u, (w1 >> 16) & 15u, s, s, z, z);
      kq[i].z = two_values((w0 >> 4) & 15u, (w0 >> 20) & 15u, s, s, z, z);
      kq[i].w = two_values((w1 >> 4) & 15u, (w1 >> 20) & 15u, s, s, z, z);
    }
    __syncthreads();
    const int k = row0 & 31, shift = 4 * ((k >> 2) & 3);      // rows row0 .. row0 + 3: a field of words 2 (k / 16), and the next
    uint2 vw[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      vw[j] = *reinterpret_cast<const uint2*>(s_v + v_at(grp, 32 * (row0 >> 5) + 8 * p + j) + 8 * (k >> 4));
      vw[j].x >>= shift;
      vw[j].y >>= shift;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float s = half_of(i < 2 ? vm.x : vm.y, i & 1), z = half_of(i < 2 ? vm.z : vm.w, i & 1);
      uint32_t o[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const uint32_t w0 = i < 2 ? vw[2 * j].x : vw[2 * j].y, w1 = i < 2 ? vw[2 * j + 1].x : vw[2 * j + 1].y;
        o[j] = two_values((w0 >> (16 * (i & 1))) & 15u, (w1 >> (16 * (i & 1))) & 15u, s, s, z, z);
      }
      vq[i] = make_uint4(o[0], o[1], o[2], o[3]);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (row0 + i >= held) kq[i] = vq[i] = make_uint4(0, 0, 0, 0);
  }
  // No load is on its way here.  (With one that a branch above may have left, every store under a condition would wait for the one before
  // it: 4 x 8 items of 32K slots 437 us.)
  __builtin_amdgcn_s_waitcnt(0x0F70);      // vmcnt(0)
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if (row0 + i < rows) {
      *reinterpret_cast<uint4*>(k_out + (row0 + i) * kHeadDim + c16 * 8) = kq[i];
      *reinterpret_cast<uint4*>(v_out + (row0 + i) * kHeadDim + c16 * 8) = vq[i];
    }
}

// Rows by index, and bf16 rows: 16 lanes a row.  Bound: latency for a few rows (64 items of 65: 3.0 us).
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
      uint32_t kc[8], vc[8];
      const int grp = c16 >> 2;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const int c = c16 * 8 + j;
        const auto code = [&](const uint8_t* tile, int lane, int k) {
          const int word = 4 * grp + 2 * (k >> 4) + ((k >> 1) & 1);
          return *reinterpret_cast<const uint32_t*>(tile + 1024 * (word >> 2) + 16 * lane + 4 * (word & 3)) >>
                     (16 * (k & 1) + 4 * ((k >> 2) & 3)) & 15u;
        };
        kc[j] = code(kt, r, c & 31);
        vc[j] = code(vt, 32 * (r >> 5) + (c & 31), r & 31);
      }
      const int m = 32 * (r >> 2) + 8 * grp + (r & 3);
      const float ks = km[8 * r + grp], kz = km[8 * r + 4 + grp], vs = vm[m], vz = vm[m + 4];
      const auto four = [](const uint32_t (&x)[8], float s, float z) {
        return make_uint4(two_values(x[0], x[1], s, s, z, z), two_values(x[2], x[3], s, s, z, z), two_values(x[4], x[5], s, s, z, z),
                          two_values(x[6], x[7], s, s, z, z));
      };
      kq = four(kc, ks, kz);
      vq = four(vc, vs, vz);
    }
  }
  reinterpret_cast<uint4*>(K)[to] = kq;
  reinterpret_cast<uint4*>(V)[to] = vq;
}

}  // namespace

hipError_t launch_fill(const FillArgs& a, int n_seqs, int longest, int bits, hipStream_t st) {
  const int n = longest < a.s.capacity ? longest : a.s.capacity;
  if (a.parts > 0) {
    const dim3 grid(a.parts, a.s.hkv, n_seqs), threads(kPartThreads);
    hipLaunchKernelGGL(select_count_kernel, grid, threads, 0, st, a);
    if (longest > a.s.capacity) {
      hipLaunchKernelGGL(select_open_kernel, grid, threads, 0, st, a);
      hipLaunchKernelGGL(select_place_kernel, grid, threads, 0, st, a);
    }
  } else {
    hipLaunchKernelGGL(fill_select_kernel<8>, dim3(a.s.hkv, n_seqs), dim3(kSelectThreads), 0, st, a);
  }
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
  const int groups = (n + 15) / 16;        // of 16 rows
  const int tiles = (n + kTileRows - 1) / kTileRows;
  if (bits == 4 && !index)
    hipLaunchKernelGGL(read_tiles_kernel, dim3(tiles * items), dim3(256), 0, st, a, n, tiles, K, V);
  else if (bits == 16)
    hipLaunchKernelGGL(read_kernel<16>, dim3(groups * items), dim3(256), 0, st, a, index, n, groups, K, V);
  else
    hipLaunchKernelGGL(read_kernel<4>, dim3(groups * items), dim3(256), 0, st, a, index, n, groups, K, V);
  return hipGetLastError();
}

}  // namespace slots
}  // namespace rdkv
