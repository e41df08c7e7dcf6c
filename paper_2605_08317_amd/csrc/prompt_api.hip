// Host side of the attention of whole prompts (rdkv_prompt_*): argument checks and launches.
#include <algorithm>
#include <cmath>
#include <utility>

#include "prompt.h"

using namespace rdkv;

namespace {

rdkv_status side_of(const char* name, int64_t stride, int heads, prompt::Side* s) {
  *s = prompt::Side{kHeadDim, 0};
  if (stride == 0) return RDKV_OK;
  if (stride % 8 != 0 || stride < static_cast<int64_t>(heads) * kHeadDim || stride > (1 << 23))
    return fail(RDKV_ERR_SHAPE, "%s_stride = %lld must be 0, or a multiple of 8 from heads * 128 to 2^23", name, static_cast<long long>(stride));
  *s = prompt::Side{static_cast<int32_t>(stride), 1};
  return RDKV_OK;
}

}  // namespace

extern "C" {

rdkv_status rdkv_prompt_default(rdkv_prompt* p) {
  if (!p) return fail(RDKV_ERR_INVALID_ARG, "prompt is null");
  *p = rdkv_prompt{};
  p->head_dim = kHeadDim;
  return RDKV_OK;
}

rdkv_status rdkv_prompt_attn_bf16(const rdkv_prompt* p, const void* Q, const void* K, const void* V, void* out, float* lse, void* stream) {
  if (!p) return fail(RDKV_ERR_INVALID_ARG, "prompt is null");
  if (p->batch < 0 || p->hq <= 0 || p->hkv <= 0) return fail(RDKV_ERR_INVALID_ARG, "batch/hq/hkv must be positive");
  if (p->head_dim != kHeadDim) return fail(RDKV_ERR_SHAPE, "head_dim %d unsupported (must be 128)", p->head_dim);
  if (p->hq % p->hkv != 0) return fail(RDKV_ERR_SHAPE, "hq %d is not a multiple of hkv %d", p->hq, p->hkv);
  const int g = p->hq / p->hkv;
  if (!(g == 1 || g == 2 || g == 4 || g == 8)) return fail(RDKV_ERR_SHAPE, "hq/hkv = %d unsupported (1,2,4,8)", g);
  if (p->hq > 65535) return fail(RDKV_ERR_SHAPE, "hq %d unsupported (at most 65535)", p->hq);
  if (p->window < 0 || p->sinks < 0) return fail(RDKV_ERR_INVALID_ARG, "window and sinks must not be negative");
  if (p->score_cap != 0.f && !(p->score_cap > 0.f && std::isnormal(p->score_cap)))        // (its inverse is finite)
    return fail(RDKV_ERR_INVALID_ARG, "score_cap must be 0 or a normal number > 0");
  if (p->batch > 0 && !p->seq_lens) return fail(RDKV_ERR_INVALID_ARG, "seq_lens is null");
  prompt::Args a{};
  rdkv_status e;
  if ((e = side_of("q", p->q_stride, p->hq, &a.q)) != RDKV_OK || (e = side_of("k", p->k_stride, p->hkv, &a.k)) != RDKV_OK ||
      (e = side_of("v", p->v_stride, p->hkv, &a.v)) != RDKV_OK || (e = side_of("out", p->out_stride, p->hq, &a.o)) != RDKV_OK)
    return e;
  int64_t rows = 0;
  for (int i = 0; i < p->batch; ++i) {
    if (p->seq_lens[i] < 0) return fail(RDKV_ERR_SHAPE, "seq_lens[%d] = %d is negative", i, p->seq_lens[i]);
    rows += static_cast<int64_t>(p->seq_lens[i]) * p->hq;
  }
  if (rows >= (1ll << 31)) return fail(RDKV_ERR_SHAPE, "sum of hq*T_s exceeds 2^31 rows");
  for (int s0 = 0; s0 < p->batch; s0 += prompt::kSeqs) {
    int64_t grid = 0;
    for (int i = s0; i < std::min(s0 + prompt::kSeqs, p->batch); ++i) grid += prompt::workgroups(p->seq_lens[i], p->hq);
    if (grid >= (1ll << 24)) return fail(RDKV_ERR_SHAPE, "sequences %d .. take %lld workgroups: a launch has less than 2^24", s0, static_cast<long long>(grid));
  }
  if (rows == 0) return RDKV_OK;
  if (!Q || !K || !V || !out) return fail(RDKV_ERR_INVALID_ARG, "Q, K, V and out must not be null");
  if (((reinterpret_cast<uintptr_t>(Q) | reinterpret_cast<uintptr_t>(K) | reinterpret_cast<uintptr_t>(V) | reinterpret_cast<uintptr_t>(out)) & 15) != 0)
    return fail(RDKV_ERR_INVALID_ARG, "Q, K, V and out must be aligned to 16 bytes");
  a.Q = static_cast<const uint16_t*>(Q);
  a.K = static_cast<const uint16_t*>(K);
  a.V = static_cast<const uint16_t*>(V);
  a.out = static_cast<uint16_t*>(out);
  a.lse = lse;
  a.slopes = p->slopes;
  a.hq = p->hq;
  a.hkv = p->hkv;
  a.window = p->window;
  a.sinks = p->sinks;
  a.cap = p->score_cap;
  int64_t token0 = 0;
  for (int s0 = 0; s0 < p->batch; s0 += prompt::kSeqs) {
    a.n_seqs = std::min(prompt::kSeqs, p->batch - s0);
    std::pair<int32_t, int64_t> seqs[prompt::kSeqs];                // (length, first token), the longest of the launch first
    for (int i = 0; i < a.n_seqs; ++i) {
      seqs[i] = {p->seq_lens[s0 + i], token0};
      token0 += seqs[i].first;
    }
    std::stable_sort(seqs, seqs + a.n_seqs, [](const auto& x, const auto& y) { return x.first > y.first; });
    // Fewer workgroups than compute units: twice as many, of half the rows, whose tiles two wavefronts take by turns (2048 tokens of 8 heads 45 -> 32 us,
    // 600 of 4 19 -> 16).
    int64_t all = 0;
    for (int i = 0; i < a.n_seqs; ++i) all += prompt::workgroups(seqs[i].first, p->hq);
    const bool shared = all <= 256 && seqs[0].first > prompt::kRows;
    int grid = 0;
    for (int i = 0; i < a.n_seqs; ++i) {
      a.T[i] = seqs[i].first;
      a.token0[i] = seqs[i].second;
      a.first[i] = grid;
      grid += static_cast<int>(prompt::workgroups(a.T[i], p->hq, shared ? prompt::kRows / 2 : prompt::kRows));
    }
    if (grid > 0) RDKV_HIP(prompt::launch(a, grid, shared, static_cast<hipStream_t>(stream)));
  }
  return RDKV_OK;
}

}  // extern "C"
