// The key/value cache's layout as the kernels and the host helpers number it (the contract is in lutgemm.h), and the
// checks that every entry point on a cache shares.
#ifndef LUTGEMM_KV_H
#define LUTGEMM_KV_H

#include <cstddef>
#include <cstdint>

#include "lutgemm.h"

namespace lutgemm_kv_detail {

constexpr int kBlock = 32;        // positions of a block, channels of a unit
constexpr int kMostSplits = 128;  // of the positions
constexpr int kMostTokens = 64;   // new tokens of a sequence that attention takes: one bit each in a mask word
constexpr int kMostSeqs = 65535;  // a grid's third side
// Of attention: query heads (a grid's second side has heads * row_blocks of AttentionPlan, with 128 rows and more to a block where there are
// several: 12288 at most), positions of a table (so that any two are less than 2^31 apart).
constexpr int kMostQueryHeads = 1 << 14;
constexpr int64_t kMostHeld = (int64_t)1 << 30;

// Bytes of one block's keys (or values): codes, then scales.
inline int code_bytes(int head_dim, int bits) { return kBlock * head_dim * bits / 8; }
inline int scale_bytes(int head_dim, int bits, int group) {
  return bits == 16 ? 0 : head_dim / group * kBlock * (bits == 8 ? 2 : 4);
}
inline int block_bytes(int head_dim, int bits, int group) {
  return 2 * (code_bytes(head_dim, bits) + scale_bytes(head_dim, bits, group));
}

inline int group_of(int head_dim, int bits, int group) { return group == 0 || bits == 16 ? head_dim : group; }

// LUTGEMM_OK if a cache can have this shape.
inline int check_shape(int64_t pages, int page_tokens, int heads, int head_dim, int bits, int group) {
  if (pages < 1 || page_tokens < kBlock || page_tokens % kBlock != 0 || heads < 1 || head_dim < 1 || group < 0) return LUTGEMM_EINVAL;
  if (bits != 4 && bits != 8 && bits != 16) return LUTGEMM_EUNSUPPORTED;
  if (head_dim != 64 && head_dim != 96 && head_dim != 128 && head_dim != 192 && head_dim != 256) return LUTGEMM_EUNSUPPORTED;
  const int g = group_of(head_dim, bits, group);
  if (head_dim % g != 0) return LUTGEMM_EINVAL;
  if (g % kBlock != 0) return LUTGEMM_EUNSUPPORTED;
  if (pages > INT32_MAX || page_tokens > 1 << 20 || heads > 1 << 12) return LUTGEMM_EUNSUPPORTED;
  int64_t bytes;                  // of the pool: an offset in it has to fit (a page alone is 2^42 bytes at most)
  if (__builtin_mul_overflow(pages, (int64_t)heads * (page_tokens / kBlock) * block_bytes(head_dim, bits, g), &bytes)) return LUTGEMM_EUNSUPPORTED;
  return LUTGEMM_OK;
}

inline int check_cache(const lutgemm_kv_cache* c) {
  if (!c || !c->pool || ((uintptr_t)c->pool & 15) != 0) return LUTGEMM_EINVAL;
  return check_shape(c->pages, c->page_tokens, c->heads, c->head_dim, c->bits, c->group);
}

inline int check_step(const lutgemm_kv_step* s) {
  if (!s || !s->first || !s->past || !s->table) return LUTGEMM_EINVAL;
  if ((((uintptr_t)s->first | (uintptr_t)s->past | (uintptr_t)s->table) & 3) != 0) return LUTGEMM_EINVAL;
  if (s->seqs < 1 || s->table_pages < 1 || s->tokens < 0 || s->most_tokens < 0) return LUTGEMM_EINVAL;
  if (s->seqs > kMostSeqs) return LUTGEMM_EUNSUPPORTED;
  return LUTGEMM_OK;
}

// The kernel whose wavefronts hold all rows (`row_tiles` of 16, 1 or 2): registers, as compiled, with `sets` blocks of
// codes and scales in them; and what follows from it: two sets where that leaves two wavefronts a SIMD, else one;
// one wavefront where not even one set does.
constexpr int attention_registers(int head_dim, int bits, int group, int row_tiles, int sets) {
  const int units = head_dim / 32, scales = bits == 8 ? 5 * (head_dim / group) : (bits == 4 ? 10 * (head_dim / group) : 0);
  return 32 + row_tiles * (12 * units + 26) + sets * (units * bits + scales) + (bits == 16 ? 5 * units : 0);
}
constexpr int attention_sets(int head_dim, int bits, int group, int row_tiles) {
  const int two = attention_registers(head_dim, bits, group, row_tiles, 2);
  return two <= 252 || (attention_registers(head_dim, bits, group, row_tiles, 1) > 252 && two <= 400) ? 2 : 1;
}
constexpr int attention_waves_per_simd(int head_dim, int bits, int group, int row_tiles) {
  const int r = attention_registers(head_dim, bits, group, row_tiles, attention_sets(head_dim, bits, group, row_tiles));
  return r <= 122 ? 4 : (r <= 168 ? 3 : (r <= 252 ? 2 : 1));
}

// How lutgemm_attention splits its work; see plan_attention in lutgemm_kv_host.cpp.
struct AttentionPlan {
  int row_tiles;    // tiles of 16 rows (token, query head) of a workgroup: 1 or 2, which every wavefront holds, or 4 and more, shared out
  int row_blocks;   // workgroups along the rows of a key head
  int splits;       // workgroups along the positions, at most
  int chunk;        // positions of a split: a multiple of 32
  int waves;        // wavefronts of a workgroup
};
AttentionPlan plan_attention(int heads, int head_dim, int bits, int group, int q_heads, int seqs, int most_tokens, int64_t most_positions);
int check_attention(const lutgemm_kv_cache* cache, const lutgemm_kv_step* step, int q_heads, int64_t most_positions, AttentionPlan* plan);
// Floats of a split's partial results: sums, a top and a total for each row; the next split's begin on 16 bytes again.
constexpr int64_t split_floats(int rows, int head_dim) { return ((int64_t)rows * (head_dim + 2) + 3) / 4 * 4; }
// Floats of the partial results behind the workspace's counters (0: nothing is split).
int64_t attention_partial_floats(const AttentionPlan& p, int heads, int head_dim, int q_heads, int seqs, int most_tokens);

}  // namespace lutgemm_kv_detail

#endif
