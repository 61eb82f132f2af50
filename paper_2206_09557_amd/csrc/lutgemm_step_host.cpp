// Host side of what surrounds products and attention: how low-rank adapters split their work.  Nothing here touches the GPU.
#include "lutgemm_step.h"

#include <algorithm>

namespace lutgemm_step_detail {

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
  p.tile = share >= 48 && a->rank <= 128 ? 64 : (share >= 24 ? 32 : 16);
  // Groups by adapter, those without one included: each ends in a tile that may be part empty.
  const int64_t groups = std::min(a->count + 1, t);
  p.tiles = (int)(groups + (t - groups) / p.tile);
  const int64_t rank_blocks = (a->rank + kRankBlock - 1) / kRankBlock;
  const int64_t most = (a->n + 511) / 512, wanted = p.tile == 16 ? 1024 : 256;
  int64_t parts = std::max<int64_t>(1, std::min<int64_t>({most, (wanted + p.tiles * rank_blocks - 1) / (p.tiles * rank_blocks), 32}));
  p.part = (int)(((a->n + parts - 1) / parts + 127) / 128 * 128);
  p.parts = (int)((a->n + p.part - 1) / p.part);
  p.rows = (int)(std::max<int64_t>(1, (a->m * p.tiles / 1536 + 255) / 256) * 256);
  return p;
}

}  // namespace lutgemm_step_detail

using namespace lutgemm_step_detail;

extern "C" {

size_t lutgemm_adapt_workspace_bytes(const lutgemm_adapters* adapters, int tokens) {
  if (check_adapters(adapters, tokens) != LUTGEMM_OK) return 0;
  const AdaptPlan p = plan_adapt(adapters, tokens);
  return (size_t)(kCounterBytes + 4 * (adapt_table_ints(p, tokens) + p.parts * adapt_part_floats(p, adapters->rank)));
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
