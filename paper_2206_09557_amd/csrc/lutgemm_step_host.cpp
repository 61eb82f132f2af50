// Host side of what surrounds products and attention: how low-rank adapters split their work, where outputs may stand.  Nothing here touches the GPU.
#include "lutgemm_step.h"

#include <algorithm>

namespace lutgemm_step_detail {

bool apart(const Rows& a, const Rows& b) {
  const uintptr_t a_end = a.at + (uintptr_t)((a.rows - 1) * a.pitch + a.bytes), b_end = b.at + (uintptr_t)((b.rows - 1) * b.pitch + b.bytes);
  if (a_end <= b.at || b_end <= a.at) return true;
  if (a.rows > 1 && b.rows > 1 && a.pitch == b.pitch) {        // where a row of b begins, from the beginning of the row of a before it
    const int64_t behind = a.at < b.at ? (int64_t)(b.at - a.at) % a.pitch : (a.pitch - (int64_t)(a.at - b.at) % a.pitch) % a.pitch;
    return behind >= a.bytes && behind + b.bytes <= a.pitch;
  }
  // Both in the order of their addresses, from the first row that may meet the other's first one.  (All rows of both in the worst case:
  // matrices of different strides within one another, which hardly anybody has.)
  auto first = [](const Rows& of, uintptr_t at) { return at > of.at && of.rows > 1 ? std::min((int64_t)(at - of.at) / of.pitch, of.rows - 1) : (int64_t)0; };
  for (int64_t i = first(a, b.at), j = first(b, a.at); i < a.rows && j < b.rows;) {
    const uintptr_t p = a.at + (uintptr_t)(i * a.pitch), q = b.at + (uintptr_t)(j * b.pitch);
    if (p < q + (uintptr_t)b.bytes && q < p + (uintptr_t)a.bytes) return false;
    p < q ? ++i : ++j;
  }
  return true;
}

int check_adapters(const lutgemm_adapters* a, int tokens) {
  if (!a || a->m < 1 || a->n < 8 || a->n % 8 != 0 || a->count < 1 || a->rank < 8 || a->rank % 8 != 0 || tokens < 0) return LUTGEMM_EINVAL;
  if (a->count > kMostAdapters || a->rank > kMostRank || tokens > kMostAdapted || a->m > 1 << 20 || a->n > 1 << 20) return LUTGEMM_EUNSUPPORTED;
  return LUTGEMM_OK;
}

AdaptPlan plan_adapt(const lutgemm_adapters* a, int tokens) {
  AdaptPlan p;
  const int t = std::max(tokens, 1);
  // Tiles as large as the adapters' shares of the tokens are on average.
  const int64_t share = t / std::min(a->count, t);
  p.tile = share >= 48 && a->rank <= 128 ? 64 : (share >= 24 && a->rank <= 128 ? 32 : 16);
  // Groups by adapter, those without one included: each ends in a tile that may be part empty.
  const int64_t groups = std::min(a->count + 1, t);
  p.tiles = (int)(groups + (t - groups) / p.tile);
  const int64_t rank_blocks = (a->rank + kRankBlock - 1) / kRankBlock;
  // Of the first product as many workgroups as leave none waiting (1024 of them fit the device where a tile and a chunk of the ranks are small,
  // else 512, but a third fewer is about as fast, and leaves fewer parts to add up: 4096 tokens, rank 64: 5120 columns 18.7 us in five parts and
  // 18.5 in seven, 12288 columns 37.0 and 34.4 (39.5 in four); 1000 tokens, 5120 columns 9.2 in ten, 11.1 in seven, 8.9 in twenty).
  const int64_t chunk = p.tile == 16 && a->rank <= 32 ? 512 : 256, units = p.tiles * rank_blocks;
  const int64_t parts = std::max<int64_t>(1, std::min<int64_t>({(a->n + chunk - 1) / chunk, (chunk == 512 ? 1024 : 352) / units, 32}));
  p.part = (int)(((a->n + parts - 1) / parts + chunk - 1) / chunk * chunk);
  p.parts = (int)((a->n + p.part - 1) / p.part);
  // Of the second one, which has 768 or 512 at work, about as many as that: a round more for a few would be as long as the first, and
  // each begins with 4 us in which it streams nothing (32 adapters of rank 16, 36864 rows: 12.9 us in 768 workgroups, 17.2 in 1152;
  // 12288 rows of 4096 tokens, rank 64: 50.5 in 469, 52.7 in 804).
  const int64_t step = p.tile == 16 && a->rank <= 16 ? 512 : 256, pieces = std::max<int64_t>(1, (p.tile == 16 && a->rank <= 32 ? 768 : 512) / p.tiles);
  p.rows = (int)(std::max<int64_t>(1, ((a->m + pieces - 1) / pieces + step / 2) / step) * step);
  return p;
}

}  // namespace lutgemm_step_detail

using namespace lutgemm_step_detail;

extern "C" {

size_t lutgemm_adapt_workspace_bytes(const lutgemm_adapters* adapters, int tokens) {
  if (check_adapters(adapters, tokens) != LUTGEMM_OK) return 0;
  const AdaptPlan p = plan_adapt(adapters, tokens);
  return (size_t)(kCounterBytes + 4 * (adapt_table_ints(p, tokens) + p.parts * adapt_part_floats(p, adapters->rank) + adapt_joined_floats(p, tokens, adapters->rank)));
}

int lutgemm_plan_adapt(const lutgemm_adapters* adapters, int tokens, int* out) {
  if (!out) return LUTGEMM_EINVAL;
  const int rc = check_adapters(adapters, tokens);
  if (rc != LUTGEMM_OK) return rc;
  const AdaptPlan p = plan_adapt(adapters, tokens);
  const int v[5] = {p.tile, p.tiles, p.parts, p.part, p.rows};
  std::copy(v, v + 5, out);
  return LUTGEMM_OK;
}

}  // extern "C"
