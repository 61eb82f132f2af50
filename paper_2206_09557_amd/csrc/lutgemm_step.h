// What surrounds the products and attention of a step: sizes and plans that the kernels and the host helpers share.
#ifndef LUTGEMM_STEP_H
#define LUTGEMM_STEP_H

#include <cstddef>
#include <cstdint>

#include "lutgemm.h"

namespace lutgemm_step_detail {

constexpr int64_t kCounterBytes = 32768;   // of a workspace, which products keep their arrival counters in
constexpr int64_t kCacheBytes = 32 << 20;   // of the L2 caches

// ---- where outputs may stand ----
// Rows of a matrix in memory, in bytes.  At least one; `pitch` is at least `bytes` and of more rows than one.
struct Rows {
  uintptr_t at;
  int64_t rows, pitch, bytes;
};
inline Rows rows_of(const void* p, int64_t rows, int64_t stride, int64_t n, int64_t size) { return {(uintptr_t)p, rows, stride * size, n * size}; }
// A kernel that reads a row of one before it writes that row of the other may be given both.
inline bool same_rows(const Rows& a, const Rows& b) { return a.at == b.at && a.rows == b.rows && a.bytes == b.bytes && (a.pitch == b.pitch || a.rows == 1); }
// Whether no byte is in both (parts of the same rows next to each other are apart).
bool apart(const Rows& a, const Rows& b);

// ---- low-rank adapters ----
constexpr int kMostAdapters = 1024;
constexpr int kMostRank = 256;
constexpr int kMostAdapted = 1 << 16;      // tokens of a call
constexpr int64_t kMostAdaptStride = (int64_t)1 << 40;     // (so that offsets in bytes stay within 64 bits)
constexpr int kFewTokens = 256;            // as many as a wavefront groups by itself
constexpr int kRankBlock = 64;             // ranks of a workgroup of the first product

struct AdaptPlan {
  int tile;        // tokens of a workgroup of the second product: 16, 32 or 64
  int tiles;       // of one adapter each: as many as there can be
  int parts;       // of the n columns, in the first product
  int part;        // columns of one: a multiple of 256
  int rows;        // of the m rows that a workgroup of the second product has: a multiple of 256
};
AdaptPlan plan_adapt(const lutgemm_adapters* a, int tokens);
int check_adapters(const lutgemm_adapters* a, int tokens);

// The workspace behind the counters: tiles' table and their tokens (where there are more tokens than a wavefront groups), then
// the first product's sums, [part][tile][token of the tile][rank], and where these are joined [tile] high and low numbers [token][rank] and a power for each token.
inline int64_t adapt_table_ints(const AdaptPlan& p, int tokens) { return tokens <= kFewTokens ? 0 : 4 + (4 + (int64_t)p.tile) * p.tiles; }
inline int64_t adapt_part_floats(const AdaptPlan& p, int rank) { return (int64_t)p.tiles * p.tile * rank; }
// Whether the first product's parts are added up once, by a kernel of its own.  Beside 8192 x 8192: 256 tokens of one adapter of rank 64,
// 64 to a tile, 23.7 us against 33.4 when each workgroup adds them up; 65 tokens of eight of rank 16 15.5 against 12.1 (256: 21.3, 16.6).
inline bool adapt_joins(const AdaptPlan& p, int tokens) { return tokens > kFewTokens || (tokens > 64 && p.tile == 64); }
inline int64_t adapt_joined_floats(const AdaptPlan& p, int tokens, int rank) {
  int pad = 32;
  while (pad < rank) pad *= 2;
  return adapt_joins(p, tokens) ? (int64_t)p.tiles * p.tile * (pad + 1) : 0;
}

}  // namespace lutgemm_step_detail

#endif
