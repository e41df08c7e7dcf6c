// Slot caches: the decode step.  One workgroup per (item, query head), scores in the workspace.
#include "slots.h"
#include "wave_ops.h"

namespace rdkv {
namespace slots {

namespace {

constexpr int kThreads = 256;

// value of one channel of a slot's row
template <int BITS, bool V>
__device__ __forceinline__ float value(const Args& a, int64_t item, int slot, int c) {
  const uint8_t* side = V ? a.v : a.k;
  if constexpr (BITS == 16) {
    return __uint_as_float(static_cast<uint32_t>(reinterpret_cast<const uint16_t*>(side)[(item * a.capacity + slot) * kHeadDim + c]) << 16);
  } else {
    const uint8_t* tile = side + (item * a.tiles + slot / kTileRows) * kTileBytes;
    const int r = slot % kTileRows, lane = V ? 32 * (r >> 5) + (c & 31) : r, k = V ? r & 31 : c & 31;
    const int word = 4 * (c >> 5) + 2 * (k >> 4) + ((k >> 1) & 1);
    const uint32_t w = *reinterpret_cast<const uint32_t*>(tile + 1024 * (word >> 2) + 16 * lane + 4 * (word & 3));
    const _Float16* meta = reinterpret_cast<const _Float16*>(tile + kTileCodes);
    const int m = V ? 32 * (r >> 2) + 8 * (c >> 5) + (r & 3) : 8 * r + (c >> 5);
    return static_cast<float>(meta[m]) * static_cast<float>(w >> (16 * (k & 1) + 4 * ((k >> 2) & 3)) & 15u) + static_cast<float>(meta[m + 4]);
  }
}

template <int BITS>
__global__ __launch_bounds__(kThreads) void decode_kernel(Args a, const uint16_t* __restrict__ q, float* __restrict__ out,
                                                          float* __restrict__ lse, float* __restrict__ scores) {
  __shared__ float s_q[kHeadDim], s_red[kThreads / 64], s_out[kHeadDim], s_top[8], s_inv[8];
  const int64_t item = blockIdx.x;
  const int tid = threadIdx.x, n = a.length(item), at = a.next[item] - 1;
  for (int h = 0; h < a.g; ++h) {
    const int64_t qh = item * a.g + h;
    float* x = scores + qh * a.capacity;
    __syncthreads();
    if (tid < kHeadDim) {
      s_q[tid] = __uint_as_float(static_cast<uint32_t>(q[qh * kHeadDim + tid]) << 16);
      s_out[tid] = 0.f;
    }
    __syncthreads();
    float top = -INFINITY;
    bool bad = false;
    for (int i = tid; i < n; i += kThreads) {
      float s = 0.f;
      for (int c = 0; c < kHeadDim; ++c) s = fmaf(s_q[c], value<BITS, false>(a, item, i, c), s);
      s *= 0.08838834764831845f;
      if (a.cap > 0.f) s = a.cap * tanhf(s / a.cap);
      const int pos = a.pos[item * a.capacity + i];
      if (a.slopes) s -= a.slopes[qh % (a.hkv * a.g)] * static_cast<float>(at - pos);
      if (a.window > 0 && at - pos >= a.window && pos >= a.sinks) s = -INFINITY;
      x[i] = s;
      bad |= s != s;
      top = fmaxf(top, s);
    }
    top = bad ? NAN : top;
    const auto all = [&](float v, bool sum) {
      for (int d = 1; d < 64; d <<= 1) {
        const float o = __shfl_xor(v, d);
        v = sum ? v + o : (v != v || o != o) ? NAN : fmaxf(v, o);
      }
      __syncthreads();
      if ((tid & 63) == 0) s_red[tid >> 6] = v;
      __syncthreads();
      v = s_red[0];
      for (int w = 1; w < kThreads / 64; ++w) v = sum ? v + s_red[w] : (v != v || s_red[w] != s_red[w]) ? NAN : fmaxf(v, s_red[w]);
      return v;
    };
    top = all(top, false);
    float l = 0.f;
    for (int i = tid; i < n; i += kThreads) l += x[i] == -INFINITY ? 0.f : expf(x[i] - top);
    l = all(l, true);
    const float inv = 1.0f / l;
    // channel, half of the slots
    const int c = tid & 127, half = tid >> 7;
    float o = 0.f;
    for (int i = half; i < n; i += 2)
      if (x[i] != -INFINITY) o = fmaf(expf(x[i] - top) * inv, value<BITS, true>(a, item, i, c), o);
    if (half == 1) s_out[c] = o;
    __syncthreads();
    if (half == 0) out[qh * kHeadDim + c] = n == 0 || l == 0.f ? 0.f : o + s_out[c];
    if (tid == 0 && lse) lse[qh] = l == 0.f ? -INFINITY : top + logf(l);
    if (tid == 0) {
      s_top[h] = top;
      s_inv[h] = l == 0.f ? 0.f : inv;
    }
  }
  __syncthreads();
  if (a.weight)
    for (int i = tid; i < n; i += kThreads) {
      float p = 0.f;
      for (int h = 0; h < a.g; ++h) {
        const float x = scores[(item * a.g + h) * a.capacity + i];
        p += s_inv[h] == 0.f || (x == -INFINITY && s_inv[h] == s_inv[h]) ? 0.f : expf(x - s_top[h]) * s_inv[h];
      }
      float& w = a.weight[item * a.capacity + i];
      w = a.decay * w + p;
    }
}

}  // namespace

size_t decode_workspace_floats(int64_t items, int g, int capacity) { return static_cast<size_t>(items) * g * capacity; }

hipError_t launch_decode(const Args& a, int bits, int items, const uint16_t* q, float* out, float* lse, float* workspace, hipStream_t st) {
  if (bits == 16) hipLaunchKernelGGL(decode_kernel<16>, dim3(items), dim3(kThreads), 0, st, a, q, out, lse, workspace);
  else hipLaunchKernelGGL(decode_kernel<4>, dim3(items), dim3(kThreads), 0, st, a, q, out, lse, workspace);
  return hipGetLastError();
}

}  // namespace slots
}  // namespace rdkv
