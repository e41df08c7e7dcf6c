// Host side of the slot caches (rdkv_slots_*): argument checks and launches.
#include <algorithm>
#include <cmath>

#include "slots.h"

using namespace rdkv;

namespace {

constexpr int64_t kMostThreads = 1ll << 32;      // of a launch

rdkv_status check_slots(const rdkv_slots* s, bool memory) {
  if (!s) return fail(RDKV_ERR_INVALID_ARG, "slots is null");
  if (s->batch < 0 || s->hq <= 0 || s->hkv <= 0) return fail(RDKV_ERR_INVALID_ARG, "batch/hq/hkv must be positive");
  if (s->head_dim != kHeadDim) return fail(RDKV_ERR_SHAPE, "head_dim %d unsupported (must be 128)", s->head_dim);
  if (s->hq % s->hkv != 0) return fail(RDKV_ERR_SHAPE, "hq %d is not a multiple of hkv %d", s->hq, s->hkv);
  const int g = s->hq / s->hkv;
  if (!(g == 1 || g == 2 || g == 4 || g == 8)) return fail(RDKV_ERR_SHAPE, "hq/hkv = %d unsupported (1,2,4,8)", g);
  if (s->hkv > 65535) return fail(RDKV_ERR_SHAPE, "hkv %d unsupported (at most 65535)", s->hkv);
  if (s->capacity < 1) return fail(RDKV_ERR_SHAPE, "capacity %d must be positive", s->capacity);
  if (s->bits != 16 && s->bits != 4) return fail(RDKV_ERR_SHAPE, "bits %d unsupported (16 or 4)", s->bits);
  if (s->sinks < 0 || s->recent < 0 || s->window < 0) return fail(RDKV_ERR_INVALID_ARG, "sinks, recent and window must not be negative");
  if (static_cast<int64_t>(s->sinks) + std::max(s->recent, 1) > s->capacity)
    return fail(RDKV_ERR_SHAPE, "%d sinks and %d recent tokens leave no slot of %d to evict from", s->sinks, s->recent, s->capacity);
  if (s->score_cap != 0.f && !(s->score_cap > 0.f && std::isnormal(s->score_cap)))        // (its inverse is finite)
    return fail(RDKV_ERR_INVALID_ARG, "score_cap must be 0 or a normal number > 0");
  if (!(s->decay >= 0.f) || s->decay > 1.f) return fail(RDKV_ERR_INVALID_ARG, "decay must be in [0, 1]");
  const int64_t items = static_cast<int64_t>(s->batch) * s->hkv;
  if (items * (static_cast<int64_t>(s->capacity) + kTile64) >= (1ll << 31)) return fail(RDKV_ERR_SHAPE, "batch * hkv * capacity exceeds 2^31 slots");
  if (static_cast<int64_t>(s->batch) * s->hq >= kMostThreads / 1024)        // (a workgroup of up to 1024 threads for each item)
    return fail(RDKV_ERR_SHAPE, "batch * hq exceeds 2^22 query heads");
  if (memory && s->batch > 0) {
    if (!s->k || !s->v || !s->pos || !s->len || !s->next) return fail(RDKV_ERR_INVALID_ARG, "k, v, pos, len and next must not be null");
    if (((reinterpret_cast<uintptr_t>(s->k) | reinterpret_cast<uintptr_t>(s->v)) & 15) != 0)
      return fail(RDKV_ERR_INVALID_ARG, "k and v must be aligned to 16 bytes");
  }
  return RDKV_OK;
}

bool aligned16(std::initializer_list<const void*> ps) {
  uintptr_t all = 0;
  for (const void* p : ps) all |= reinterpret_cast<uintptr_t>(p);
  return (all & 15) == 0;
}

slots::Args args_of(const rdkv_slots* s) {
  slots::Args a;
  a.k = static_cast<uint8_t*>(s->k);
  a.v = static_cast<uint8_t*>(s->v);
  a.pos = s->pos;
  a.weight = s->weight;
  a.len = s->len;
  a.next = s->next;
  a.slopes = s->slopes;
  a.hkv = s->hkv;
  a.g = s->hq / s->hkv;
  a.capacity = s->capacity;
  a.tiles = (s->capacity + slots::kTileRows - 1) / slots::kTileRows;
  a.sinks = s->sinks;
  a.recent = s->recent;
  a.window = s->window;
  a.cap = s->score_cap;
  a.decay = s->decay;
  return a;
}

rdkv_status check_prompts(const rdkv_slots* s, int32_t n, const int32_t* seq_lens, int32_t* longest) {
  if (n < 0) return fail(RDKV_ERR_INVALID_ARG, "n = %d is negative", n);
  if (n > 0 && !seq_lens) return fail(RDKV_ERR_INVALID_ARG, "seq_lens is null");
  int64_t rows = 0;
  *longest = 0;
  for (int i = 0; i < n; ++i) {
    if (seq_lens[i] < 0) return fail(RDKV_ERR_SHAPE, "seq_lens[%d] = %d is negative", i, seq_lens[i]);
    rows += static_cast<int64_t>(seq_lens[i]) * s->hkv;
    *longest = std::max(*longest, seq_lens[i]);
  }
  if (rows >= (1ll << 31)) return fail(RDKV_ERR_SHAPE, "sum of hkv*T_s exceeds 2^31 rows");
  return RDKV_OK;
}

// What the launches of a fill's selection have in the workspace, one group of sequences after the other: the largest group's.
struct SelectBytes { size_t counts, open, part, found, total; };
SelectBytes select_bytes(const rdkv_slots* s, int32_t n, const int32_t* seq_lens) {
  SelectBytes b{};
  for (int s0 = 0; s0 < n; s0 += slots::kFillSeqs) {
    const int ns = std::min(slots::kFillSeqs, n - s0);
    int64_t rows = 0, longest = 0;
    for (int i = 0; i < ns; ++i) {
      rows += static_cast<int64_t>(seq_lens[s0 + i]) * s->hkv;
      longest = std::max<int64_t>(longest, seq_lens[s0 + i]);
    }
    const slots::SelectPlan p = slots::plan_select(longest);
    if (p.parts == 0 || longest <= s->capacity) continue;
    const size_t items = static_cast<size_t>(ns) * s->hkv, parts = items * p.parts;
    b.counts = std::max(b.counts, parts * slots::kSelectDigits * sizeof(uint16_t));
    b.open = std::max(b.open, (static_cast<size_t>(rows) * sizeof(uint32_t) + 15) / 16 * 16);
    b.part = std::max(b.part, (parts * sizeof(int2) + 15) / 16 * 16);
    b.found = std::max(b.found, items * sizeof(int4));
  }
  b.total = b.counts + b.open + b.part + b.found;
  return b;
}

}  // namespace

extern "C" {

rdkv_status rdkv_slots_default(rdkv_slots* s) {
  if (!s) return fail(RDKV_ERR_INVALID_ARG, "slots is null");
  *s = rdkv_slots{};
  s->head_dim = kHeadDim;
  s->bits = 16;
  s->decay = 1.0f;
  return RDKV_OK;
}

size_t rdkv_slots_side_bytes(const rdkv_slots* s) {
  if (check_slots(s, false) != RDKV_OK) return 0;
  const size_t items = static_cast<size_t>(s->batch) * s->hkv;
  if (s->bits == 16) return items * s->capacity * kHeadDim * sizeof(uint16_t);
  return items * ((static_cast<size_t>(s->capacity) + slots::kTileRows - 1) / slots::kTileRows) * slots::kTileBytes;
}

size_t rdkv_slots_fill_workspace_bytes(const rdkv_slots* s, int32_t n, const int32_t* seq_lens) {
  int32_t longest;
  if (check_slots(s, false) != RDKV_OK || check_prompts(s, n, seq_lens, &longest) != RDKV_OK) return 0;
  return select_bytes(s, n, seq_lens).total;
}

rdkv_status rdkv_slots_fill(const rdkv_slots* s, int32_t first, int32_t n, const int32_t* seq_lens, const void* K, const void* V,
                            const float* w_tok, void* workspace, size_t workspace_bytes, void* stream) {
  rdkv_status e = check_slots(s, true);
  if (e != RDKV_OK) return e;
  int32_t longest;
  if ((e = check_prompts(s, n, seq_lens, &longest)) != RDKV_OK) return e;
  if (first < 0 || first > s->batch || n > s->batch - first)
    return fail(RDKV_ERR_INVALID_ARG, "sequences %d .. %d of %d", first, first + n - 1, s->batch);
  if (n == 0) return RDKV_OK;
  if (longest > 0 && (!K || !V)) return fail(RDKV_ERR_INVALID_ARG, "K and V must not be null");
  if (longest > s->capacity && !w_tok)
    return fail(RDKV_ERR_INVALID_ARG, "a prompt of %d tokens for %d slots needs w_tok", longest, s->capacity);
  // sixteen rows a workgroup, sixteen threads a row (fewer in tiles): a launch has less than 2^32 threads
  const int64_t rows = std::min(longest, s->capacity);
  if ((rows + 15) / 16 * 256 >= kMostThreads)
    return fail(RDKV_ERR_SHAPE, "%lld rows of an item: at most 2^28 - 16", static_cast<long long>(rows));
  const SelectBytes need = select_bytes(s, n, seq_lens);
  if (need.total > 0 && (!workspace || workspace_bytes < need.total))
    return fail(RDKV_ERR_INVALID_ARG, "workspace of %zu bytes is smaller than the %zu required", workspace ? workspace_bytes : 0, need.total);
  if (!aligned16({K, V, workspace})) return fail(RDKV_ERR_INVALID_ARG, "K, V and workspace must be aligned to 16 bytes");
  int64_t row = 0;
  for (int s0 = 0; s0 < n; s0 += slots::kFillSeqs) {
    const int ns = std::min(slots::kFillSeqs, n - s0);
    slots::FillArgs a;
    a.s = args_of(s);
    a.K = static_cast<const uint16_t*>(K);
    a.V = static_cast<const uint16_t*>(V);
    a.w_tok = w_tok;
    a.seq0 = first + s0;
    int32_t most = 0;
    uint8_t* ws = static_cast<uint8_t*>(workspace);
    a.counts = reinterpret_cast<uint16_t*>(ws);
    a.open = reinterpret_cast<uint32_t*>(ws + need.counts);
    a.part = reinterpret_cast<int2*>(ws + need.counts + need.open);
    a.found = reinterpret_cast<int4*>(ws + need.counts + need.open + need.part);
    for (int i = 0; i < ns; ++i) {
      most = std::max(most, seq_lens[s0 + i]);
      a.T[i] = seq_lens[s0 + i];
      a.row0[i] = row;
      row += static_cast<int64_t>(seq_lens[s0 + i]) * s->hkv;
    }
    const slots::SelectPlan plan = slots::plan_select(most);
    a.parts = plan.parts;
    a.part_rows = plan.part_rows;
    RDKV_HIP(slots::launch_fill(a, ns, most, s->bits, static_cast<hipStream_t>(stream)));
  }
  return RDKV_OK;
}

rdkv_status rdkv_slots_append(const rdkv_slots* s, const void* k_new, const void* v_new, int32_t* slot, void* stream) {
  const rdkv_status e = check_slots(s, true);
  if (e != RDKV_OK) return e;
  if (s->batch == 0) return RDKV_OK;
  if (!k_new || !v_new) return fail(RDKV_ERR_INVALID_ARG, "k_new and v_new must not be null");
  if (!aligned16({k_new, v_new})) return fail(RDKV_ERR_INVALID_ARG, "k_new and v_new must be aligned to 16 bytes");
  RDKV_HIP(slots::launch_append(args_of(s), s->bits, s->batch * s->hkv, static_cast<const uint16_t*>(k_new),
                                static_cast<const uint16_t*>(v_new), slot, static_cast<hipStream_t>(stream)));
  return RDKV_OK;
}

size_t rdkv_slots_decode_workspace_bytes(const rdkv_slots* s) {
  if (check_slots(s, false) != RDKV_OK || s->batch == 0) return 0;
  return slots::decode_workspace_floats(static_cast<int64_t>(s->batch) * s->hkv, s->hq / s->hkv, s->capacity, s->bits, s->weight != nullptr) * sizeof(float);
}

rdkv_status rdkv_slots_decode_attn(const rdkv_slots* s, const void* q, float* out, float* lse, void* workspace,
                                   size_t workspace_bytes, void* stream) {
  const rdkv_status e = check_slots(s, true);
  if (e != RDKV_OK) return e;
  if (s->batch == 0) return RDKV_OK;
  if (!q || !out || !workspace) return fail(RDKV_ERR_INVALID_ARG, "q, out and workspace must not be null");
  if (!aligned16({q, out, workspace})) return fail(RDKV_ERR_INVALID_ARG, "q, out and workspace must be aligned to 16 bytes");
  const size_t need = rdkv_slots_decode_workspace_bytes(s);
  if (workspace_bytes < need)
    return fail(RDKV_ERR_INVALID_ARG, "workspace of %zu bytes is smaller than the %zu required", workspace_bytes, need);
  RDKV_HIP(slots::launch_decode(args_of(s), s->bits, s->batch * s->hkv, static_cast<const uint16_t*>(q), out, lse,
                                static_cast<float*>(workspace), static_cast<hipStream_t>(stream)));
  return RDKV_OK;
}

rdkv_status rdkv_slots_read(const rdkv_slots* s, const int32_t* index, int32_t n, void* K, void* V, void* stream) {
  const rdkv_status e = check_slots(s, true);
  if (e != RDKV_OK) return e;
  if (n < 0) return fail(RDKV_ERR_INVALID_ARG, "n = %d is negative", n);
  if (s->batch == 0 || n == 0) return RDKV_OK;
  if (!K || !V) return fail(RDKV_ERR_INVALID_ARG, "K and V must not be null");
  if (!aligned16({K, V})) return fail(RDKV_ERR_INVALID_ARG, "K and V must be aligned to 16 bytes");
  if (static_cast<int64_t>(s->batch) * s->hkv * (static_cast<int64_t>(n) + kTile64) >= kMostThreads / 16)
    return fail(RDKV_ERR_SHAPE, "batch * hkv * n exceeds 2^28 rows");
  RDKV_HIP(slots::launch_read(args_of(s), s->bits, s->batch * s->hkv, index, n, static_cast<uint16_t*>(K),
                              static_cast<uint16_t*>(V), static_cast<hipStream_t>(stream)));
  return RDKV_OK;
}

}  // extern "C"
