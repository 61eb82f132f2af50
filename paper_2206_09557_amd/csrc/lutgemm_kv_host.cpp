// Host side of the attention half: sizes of caches and workspaces, how attention splits its work, rotary frequencies.
// Nothing here touches the GPU.
#include "lutgemm_kv.h"

#include <algorithm>
#include <cmath>

namespace lutgemm_kv_detail {

namespace {
constexpr int64_t kComputeUnits = 256;

// Share of the device that is at work while workgroups come in rounds of `room`.
double filled(int64_t workgroups, int64_t room) { return (double)workgroups / (double)(room * ((workgroups + room - 1) / room)); }
}  // namespace

AttentionPlan plan_attention(int heads, int head_dim, int bits, int group, int q_heads, int seqs, int most_tokens, int64_t most_positions) {
  AttentionPlan p;
  const int64_t rows = (int64_t)std::min(most_tokens, kMostTokens) * (q_heads / heads);
  const int64_t blocks = std::max<int64_t>(1, (most_positions + kBlock - 1) / kBlock);
  // Up to 32 rows (16 of long heads) each wavefront holds all of them; beyond, eight wavefronts share them out (32 each, or 16) and
  // the blocks' operands; of 256 channels 16 each, all eight of a block (two sets of four do not fit their registers).
  // A few blocks are worked on 32 rows at a time also where there are more, if the device has room for that many workgroups (265 rows over 81
  // positions, 30 key heads: 9.5 us, all rows of a head in two workgroups 17.9).
  const int most_tiles = head_dim <= 128 ? 16 : 8;
  const bool small = blocks <= 8 && (int64_t)seqs * heads * ((rows + 31) / 32) <= 4 * kComputeUnits;
  p.row_tiles = rows <= 16 ? 1 : ((rows <= 32 || small) && head_dim <= 128 ? 2 : (head_dim == 256 ? 8 : 4));
  while (p.row_tiles >= 4 && p.row_tiles < most_tiles && 16 * p.row_tiles < rows) p.row_tiles *= 2;
  p.row_blocks = (int)std::max<int64_t>(1, (rows + 16 * p.row_tiles - 1) / (16 * p.row_tiles));
  const int64_t units = (int64_t)seqs * heads * p.row_blocks;
  const int simd = p.row_tiles >= 4 ? 2 : attention_waves_per_simd(head_dim, bits, group, p.row_tiles);
  p.waves = p.row_tiles >= 4 ? 8 : 4;
  // Splits until the device is full, but none so short that its ends cost more than it saves: three blocks a wavefront (one sequence of
  // 3000 positions and 8 key heads of 8 query heads, 8 bits: 10.7 us in 8 splits of four wavefronts, 12.3 in 6 of eight; 600 positions of
  // 32 heads 9.9 unsplit, 11.2 in two of eight), two at up to 32 rows (6000 positions, 20 rows: 12.2 in 24, 15.1 in 15), and where
  // wavefronts share a block two or, in sets that take blocks in turn, four a split (6000 positions, 100 rows: 17.6 in 38, 25.8 in 8;
  // 3000 positions, 64 rows, 2 key heads: 15.6 in 24, 18.4 in 11).
  const int64_t least = p.row_tiles >= 4 ? (p.row_tiles == most_tiles ? 2 : 4) : (p.row_tiles == 2 ? 2 : 3) * p.waves;
  const int64_t room = kComputeUnits * 4 * simd / p.waves;
  int64_t splits = std::max<int64_t>(1, std::min<int64_t>({room / units, blocks / least, kMostSplits}));
  if (p.row_tiles == 1) {
    // What is added at the end grows with the splits, what is read before falls with them: no more than the square root of the blocks (80801
    // positions of 4 key heads: 26 us in 50 to 64 splits, 32 in 127).
    const int64_t root = (int64_t)std::sqrt((double)blocks);
    splits = std::max<int64_t>(1, std::min(splits, root));
    // Sums of all of a compute unit's wavefronts meet in LDS rather than in memory, which pays from 15 blocks each on (131072 positions of
    // 8 key heads at 4 bits: 42 us against 49, 4000 of 16 sequences of 64 heads at 8 bits 117 against 122; 2000 of 40 heads at 16 bits
    // 73 against 70) where that fills the device as well (20 sequences of 8 heads, 6600 positions: 160 workgroups 47, 480 of four
    // wavefronts 41).
    const int64_t of_all = std::max<int64_t>(1, std::min<int64_t>({kComputeUnits / units, root, kMostSplits}));
    if (blocks >= 15 * 4 * simd * of_all && filled(units * of_all, kComputeUnits) >= 0.85 * filled(units * splits, room)) {
      p.waves = 4 * simd;
      splits = of_all;
    }
  }
  const int64_t per = (blocks + splits - 1) / splits;
  p.chunk = (int)std::min<int64_t>(per, 1 << 24) * kBlock;
  p.splits = (int)((blocks + per - 1) / per);
  return p;
}

int64_t attention_partial_floats(const AttentionPlan& p, int heads, int head_dim, int q_heads, int seqs, int most_tokens) {
  if (p.splits == 1) return 0;
  const int64_t rows = std::min<int64_t>(16 * p.row_tiles, (int64_t)std::min(most_tokens, kMostTokens) * (q_heads / heads));
  return (int64_t)seqs * heads * p.row_blocks * p.splits * split_floats((int)rows, head_dim);
}

// What the sizes of a call must be, for the call itself and for what is asked about it before; the plan of one that is offered.
int check_attention(const lutgemm_kv_cache* cache, const lutgemm_kv_step* step, int q_heads, int64_t most_positions, AttentionPlan* plan) {
  if (!cache || !step || step->seqs < 1 || step->table_pages < 1 || step->tokens < 0 || step->most_tokens < 0 || q_heads < 1 || most_positions < 0) return LUTGEMM_EINVAL;
  const int rc = check_shape(cache->pages, cache->page_tokens, cache->heads, cache->head_dim, cache->bits, cache->group);
  if (rc != LUTGEMM_OK) return rc;
  if (q_heads % cache->heads != 0) return LUTGEMM_EINVAL;
  if (step->seqs > kMostSeqs || step->most_tokens > kMostTokens || q_heads > kMostQueryHeads) return LUTGEMM_EUNSUPPORTED;
  const int64_t held = (int64_t)step->table_pages * cache->page_tokens;
  if (held > kMostHeld) return LUTGEMM_EUNSUPPORTED;
  if (most_positions == 0 || most_positions > held) most_positions = held;
  *plan = plan_attention(cache->heads, cache->head_dim, cache->bits, group_of(cache->head_dim, cache->bits, cache->group), q_heads, step->seqs, step->most_tokens, most_positions);
  return LUTGEMM_OK;
}

}  // namespace lutgemm_kv_detail

using namespace lutgemm_kv_detail;

extern "C" {

size_t lutgemm_kv_pool_bytes(int64_t pages, int page_tokens, int heads, int head_dim, int bits, int group) {
  if (check_shape(pages, page_tokens, heads, head_dim, bits, group) != LUTGEMM_OK) return 0;
  return (size_t)pages * heads * (page_tokens / kBlock) * block_bytes(head_dim, bits, group_of(head_dim, bits, group));
}

size_t lutgemm_attention_workspace_bytes(const lutgemm_kv_cache* cache, const lutgemm_kv_step* step, int q_heads, int64_t most_positions) {
  AttentionPlan p;
  if (check_attention(cache, step, q_heads, most_positions, &p) != LUTGEMM_OK) return 0;
  return 32768 + 4 * (size_t)attention_partial_floats(p, cache->heads, cache->head_dim, q_heads, step->seqs, step->most_tokens);
}

int lutgemm_plan_attention(const lutgemm_kv_cache* cache, const lutgemm_kv_step* step, int q_heads, int64_t most_positions, int* out) {
  AttentionPlan p;
  if (!out) return LUTGEMM_EINVAL;
  const int rc = check_attention(cache, step, q_heads, most_positions, &p);
  if (rc != LUTGEMM_OK) return rc;
  const int v[5] = {p.row_tiles, p.row_blocks, p.splits, p.chunk, p.waves};
  std::copy(v, v + 5, out);
  return LUTGEMM_OK;
}

int lutgemm_rope_frequencies(int rot_dim, double base, int scaling, double factor, double low, double high, double trained, uint64_t* turns) {
  if (!turns || rot_dim < 2 || rot_dim % 2 != 0 || rot_dim > 65536 || !(base > 1.0) || !std::isfinite(base)) return LUTGEMM_EINVAL;
  if (scaling < LUTGEMM_ROPE_PLAIN || scaling > LUTGEMM_ROPE_PARTS) return LUTGEMM_EUNSUPPORTED;
  if (scaling != LUTGEMM_ROPE_PLAIN && (!(factor >= 1.0) || !std::isfinite(factor))) return LUTGEMM_EINVAL;
  if (scaling == LUTGEMM_ROPE_PARTS && (!(low < high) || !(trained > 0.0) || !std::isfinite(low) || !std::isfinite(high) || !std::isfinite(trained)))
    return LUTGEMM_EINVAL;
  constexpr double kTwoPi = 6.283185307179586476925286766559;
  if (scaling == LUTGEMM_ROPE_BASE && rot_dim > 2) base *= std::pow(factor, (double)rot_dim / (rot_dim - 2));
  if (!std::isfinite(base)) return LUTGEMM_EINVAL;
  for (int i = 0; i < rot_dim / 2; ++i) {
    double f = std::pow(base, -2.0 * i / rot_dim);
    if (scaling == LUTGEMM_ROPE_LINEAR) f /= factor;
    if (scaling == LUTGEMM_ROPE_PARTS) {
      const double kept = std::min(1.0, std::max(0.0, (f * trained / kTwoPi - low) / (high - low)));
      f = f * kept + f / factor * (1.0 - kept);
    }
    turns[i] = (uint64_t)std::nearbyint(std::ldexp(f / kTwoPi, 64));   // f <= 1: below 2^62
  }
  return LUTGEMM_OK;
}

}  // extern "C"
