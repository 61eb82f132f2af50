// Low-rank adapters of many requests beside a product whose weights they share: y[t] = base[t] + c_a B_a (A_a x[t]), a the adapter of
// token t.  include/lutgemm.h has the layouts.
//
// Tokens with the same adapter are taken together, up to TILE of them, so that its A and B are read once for them: of up to 256 tokens
// every wavefront finds the tiles by itself, from ballots over the bits of their adapters; of more a kernel of one workgroup sorts them
// first.  Then two products on the 16 x 16 x 32 matrix instructions:
//     H^T (ranks x tokens) = A (ranks x n) X^T,      Y (tokens x m) = H B^T (B m x ranks)
// A decode step streams A and B (2 r (n + m) bytes an adapter), a prompt x, base and y; the time is that and two launches, each with a chain of
// loads before it streams: adapters -> A and x -> sums, adapters -> sums of all parts -> H.  n is shared out among workgroups; their
// sums are added up in an order that the sizes decide, by each workgroup of the second product or, of tiles of 64 tokens or many tokens, once.  H stays fp32 until
// then, and meets B as two fp16 numbers (22 bits) of a power of two that the token's largest decides: rounded to one, it would add as much
// error as the result's own rounding to fp16, and more than that of fp32 results.  Measured: 32 adapters of rank 16 beside 36864 x 12288, one
// token each, 56 MB: 6 + 12.8 us; three of up to 64 beside 12288 x 5120, 4096 tokens, 236 MB: sorting 7.6, products 19 and 50, joining 5.5.
#include <hip/hip_fp16.h>
#include <hip/hip_runtime.h>

#include "lutgemm_step.h"

using namespace lutgemm_step_detail;

namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef _Float16 half8v __attribute__((ext_vector_type(8)));
typedef float float4v __attribute__((ext_vector_type(4)));

struct AdaptParams {
  const _Float16* x;
  const void* base;
  void* y;
  const _Float16* down;
  const _Float16* up;
  const int32_t* of;
  const int32_t* owner;
  const int32_t* ranks;
  const float* scales;
  int32_t* table;              // how many tiles, theirs (adapter, tokens), then their tokens [tile][place]
  float* sums;
  float* joined;               // null: the second product adds the first one's parts up by itself
  int64_t x_stride, base_stride, y_stride, m, n, part_floats;
  int tokens, seqs, count, rank, tiles, parts, part, rows;
  bool copies;                 // tokens without an adapter are copied
};

__device__ __forceinline__ float4v mfma(half8v a, half8v b, float4v c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }

// The adapter of a token, `count` if it has none.
__device__ __forceinline__ int adapter_of(const AdaptParams& p, int token) {
  int at = token;
  if (p.owner) {
    at = p.owner[token];
    if (at < 0 || at >= p.seqs) return p.count;
  }
  const int a = p.of[at];
  return a < 0 || a >= p.count ? p.count : a;
}

// A tile of up to `most` tokens: its adapter, how many tokens it has (0: there is no such tile, or nothing to do for it), which ones (of the workgroup, in LDS).
struct Tile {
  int adapter, tokens, rank;   // (the rank as rank_of finds it, which is one more trip to memory)
};
// Among up to 64 RUNS tokens, token 64 u + lane in a lane's u-th place: the tiles are numbered by their first tokens.  Against sorting
// first, beside 8192 x 8192: 65 tokens of eight adapters of rank 16 12.1 us against 15.8, 256 16.7 against 20.3; 64 to a tile, 128 tokens
// 21.5 against 22.3, 256 23.6 against 23.4 (5120 x 5120: 21.3, 20.6), where the ballots of every workgroup are as long as the launch.
template <int RUNS>
__device__ __forceinline__ void find_tile(const AdaptParams& p, int number, int most, int* token, Tile* t) {
  const int lane = threadIdx.x & 63;
  const uint64_t below = ((uint64_t)1 << lane) - 1;
  int mine[RUNS], rank[RUNS];
  uint64_t same[RUNS][RUNS];                     // the tokens of run v that have the adapter of this lane's u-th
#pragma unroll
  for (int u = 0; u < RUNS; ++u) mine[u] = 64 * u + lane < p.tokens ? adapter_of(p, 64 * u + lane) : -1;
#pragma unroll
  for (int v = 0; v < RUNS; ++v) {
    const uint64_t live = __ballot(mine[v] >= 0);
#pragma unroll
    for (int u = 0; u < RUNS; ++u) same[u][v] = live;
  }
  for (int bit = 1; bit <= p.count; bit *= 2) {
#pragma unroll
    for (int v = 0; v < RUNS; ++v) {
      const uint64_t set = __ballot((mine[v] & bit) != 0);
#pragma unroll
      for (int u = 0; u < RUNS; ++u) same[u][v] &= (mine[u] & bit) != 0 ? set : ~set;
    }
  }
  int before = 0;                                // tiles that begin in earlier runs
#pragma unroll
  for (int u = 0; u < RUNS; ++u) {
    rank[u] = __popcll(same[u][u] & below);
#pragma unroll
    for (int v = 0; v < u; ++v) rank[u] += __popcll(same[u][v]);
    const bool head = mine[u] >= 0 && (rank[u] & (most - 1)) == 0;
    const uint64_t heads = __ballot(head), chosen = __ballot(head && before + __popcll(heads & below) == number);
    before += __popcll(heads);
    if (chosen != 0) {
      const int first = __builtin_ctzll(chosen), from = __builtin_amdgcn_readlane(rank[u], first);
      t->adapter = __builtin_amdgcn_readlane(mine[u], first);
      t->rank = from;                            // (of the first token, till the members are known)
      t->tokens = 1;
    }
  }
  if (t->tokens == 0) return;
  const int from = t->rank;
  t->tokens = t->rank = 0;
#pragma unroll
  for (int u = 0; u < RUNS; ++u) {
    const bool member = mine[u] == t->adapter && rank[u] >= from && rank[u] < from + most;
    t->tokens += __popcll(__ballot(member));
    if (threadIdx.x < 64 && member) token[rank[u] - from] = 64 * u + lane;
  }
}
__device__ __forceinline__ Tile tile_of(const AdaptParams& p, int number, int most, bool copies, int* token) {
  Tile t = {p.count, 0, 0};
  if (p.tokens <= 64) {
    find_tile<1>(p, number, most, token, &t);
  } else if (p.tokens <= kFewTokens) {
    find_tile<kFewTokens / 64>(p, number, most, token, &t);
  } else if (number < p.table[0]) {
    const int32_t* entry = p.table + 4 + 4 * number;
    const int mine = p.table[4 + 4 * p.tiles + number * most + min((int)threadIdx.x, most - 1)];       // (of places without a token anything)
    t.adapter = entry[0];
    t.tokens = entry[1];
    if ((int)threadIdx.x < t.tokens) token[threadIdx.x] = mine;
  }
  if (t.adapter >= p.count && !copies) t.tokens = 0;
  __syncthreads();
  return t;
}
__device__ __forceinline__ int rank_of(const AdaptParams& p, const Tile& t) {
  return t.adapter >= p.count ? 0 : (p.ranks ? min(max(p.ranks[t.adapter], 0), p.rank) : p.rank);
}

// Sorts the tokens by adapter, each adapter's in their order, and cuts them into tiles.  One workgroup; a wavefront has a stretch of the
// tokens, 64 at a time, and counts of its own, so that no place depends on an order of arrival.  Up to 8192 tokens their adapters, and their
// places among the stretch's tokens of one adapter, stay in registers between the two turns.
constexpr int kSortThreads = 1024, kSortWaves = kSortThreads / 64, kSortRuns = 8;
__global__ __launch_bounds__(kSortThreads) void lutgemm_adapt_sort_kernel(AdaptParams p, int tile) {
  extern __shared__ int32_t counts[];            // [wavefront][adapter], then the adapters' tokens and first tiles
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, kinds = p.count + 1;
  int32_t* totals = counts + kSortWaves * kinds;
  int32_t* tiles = totals + kinds;
  int32_t* mine = counts + wave * kinds;
  int32_t* order = p.table + 4 + 4 * p.tiles;
  const int each = (p.tokens + kSortThreads - 1) / kSortThreads * 64;      // tokens of a wavefront
  const int from = wave * each, end = min(from + each, p.tokens);
  int adapter[kSortRuns], place[kSortRuns];
  auto look = [&](int first) {                   // (looked up together)
#pragma unroll
    for (int u = 0; u < kSortRuns; ++u) adapter[u] = first + 64 * u + lane < end ? adapter_of(p, first + 64 * u + lane) : -1;
  };
  // The run's tokens are counted: `place` becomes each one's among the stretch's of its adapter.
  auto count = [&](int a, int* place) {
    const bool live = a >= 0;
    uint64_t same = __ballot(live);
    for (int bit = 1; bit <= p.count; bit *= 2) {
      const uint64_t set = __ballot((a & bit) != 0);
      same &= (a & bit) != 0 ? set : ~set;
    }
    const int rank = __popcll(same & (((uint64_t)1 << lane) - 1));
    if (live) {
      const int at = mine[a];
      *place = at + rank;
      if (rank == 0) mine[a] = at + __popcll(same);
    }
    __builtin_amdgcn_fence(__ATOMIC_SEQ_CST, "wavefront");
  };
  look(from);
  for (int i = tid; i < kSortWaves * kinds; i += kSortThreads) counts[i] = 0;
  __syncthreads();
  for (int first = from; first < end; first += 64 * kSortRuns) {
    if (first != from) look(first);
#pragma unroll
    for (int u = 0; u < kSortRuns; ++u)
      if (first + 64 * u < end) count(adapter[u], &place[u]);
  }
  __syncthreads();
  // counts become places: of each adapter over the wavefronts; its tiles stand one after the other (which one wavefront adds up)
  for (int a = tid; a < kinds; a += kSortThreads) {
    int sum = 0;
    for (int w = 0; w < kSortWaves; ++w) {
      const int have = counts[w * kinds + a];
      counts[w * kinds + a] = sum;
      sum += have;
    }
    totals[a] = sum;
  }
  __syncthreads();
  if (wave == 0) {
    int cut = 0;
    for (int base = 0; base < kinds; base += 64) {
      const int a = base + lane;
      const int pieces = a < kinds ? (totals[a] + tile - 1) / tile : 0;
      int c = pieces;
#pragma unroll
      for (int d = 1; d < 64; d *= 2) {
        const int other = __shfl_up(c, d);
        if (lane >= d) c += other;
      }
      if (a < kinds) tiles[a] = cut + c - pieces;
      cut += __shfl(c, 63);
    }
    if (lane == 0) {
      tiles[kinds] = cut;
      p.table[0] = cut;
    }
  }
  __syncthreads();
  for (int i = tid; i < tiles[kinds]; i += kSortThreads) {     // the adapter of a tile: the last whose first tile is not behind it
    int lo = 0, hi = kinds - 1;
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if (tiles[mid] <= i)
        lo = mid;
      else
        hi = mid - 1;
    }
    int32_t* entry = p.table + 4 + 4 * i;
    entry[0] = lo;
    entry[1] = min(totals[lo] - (i - tiles[lo]) * tile, tile);
  }
  if (each <= 64 * kSortRuns) {
#pragma unroll
    for (int u = 0; u < kSortRuns; ++u)
      if (adapter[u] >= 0) order[tiles[adapter[u]] * tile + mine[adapter[u]] + place[u]] = from + 64 * u + lane;
  } else {                                       // counted again, from the stretch's first places on
    for (int first = from; first < end; first += 64 * kSortRuns) {
      look(first);
#pragma unroll
      for (int u = 0; u < kSortRuns; ++u) {
        if (first + 64 * u >= end) continue;
        count(adapter[u], &place[u]);
        if (adapter[u] >= 0) order[tiles[adapter[u]] * tile + place[u]] = first + 64 * u + lane;
      }
    }
  }
}

constexpr int kThreads = 256, kWaves = kThreads / 64;

// A token's A x as two fp16 numbers of a power of two that brings its largest to 2^14 .. 2^15 (so that neither overflows, and what is lost
// is 2^-22 of the largest): `each` lanes of a wavefront have a token's ranks, from `part` on.  `value(r)` is beyond the rank's end 0.
template <typename Value>
__device__ __forceinline__ void split_h(int part, int each, int ranks, Value value, _Float16* high, _Float16* low, int* drop) {
  float top = 0.0f;
  for (int r = part; r < ranks; r += each) top = fmaxf(top, fabsf(value(r)));
  for (int d = 1; d < each; d *= 2) top = fmaxf(top, __shfl_xor(top, d));
  // (no power where the largest is an infinity: the result is no number then; or zero)
  const int lift = top > 0.0f && top < __builtin_inff() ? 15 - __builtin_amdgcn_frexp_expf(top) : 0;
  for (int r = part; r < ranks; r += each) {
    const float v = ldexpf(value(r), lift);
    const _Float16 hi = (_Float16)v;
    high[r] = hi;
    low[r] = fabsf((float)hi) < __builtin_inff() ? (_Float16)(v - (float)hi) : (_Float16)0.0f;
  }
  if (part == 0) *drop = -lift;
}

// H of a tile, for a part of the columns and RANKS of its ranks.  Rows of x and A pass through LDS, CHUNK columns at
// a time, so that a wavefront reads them a kilobyte (or two halves) at a time: as matrix operands, straight from memory, 16 neighbouring lanes
// would touch 16 rows, which takes longer (4096 tokens of 5120 columns, rank 64: 24 to 27 us so, 19 through LDS).  The next columns are on
// their way meanwhile.  Every wavefront has some of a chunk's steps of 32 columns, for all tokens and RANKS; their sums meet in LDS.
template <int NT, int RANKS, int CHUNK>
__global__ __launch_bounds__(kThreads) void lutgemm_adapt_down_kernel(AdaptParams p) {
  constexpr int TILE = 16 * NT, RT = RANKS / 16, PITCH = CHUNK + 8, OF = CHUNK / 8, AT_ONCE = 64 / OF, ROWS = TILE + RANKS;   // lanes of a row, rows an instruction
  constexpr int LOADS = ROWS / (AT_ONCE * kWaves), STEPS = CHUNK / 32 / kWaves;
  constexpr int OPERANDS = 2 * ROWS * PITCH, SUMS = 4 * kWaves * TILE * (RANKS + 4);
  static_assert(ROWS % (AT_ONCE * kWaves) == 0 && CHUNK % (32 * kWaves) == 0, "rows and steps are dealt evenly");
  __shared__ int token[TILE];
  __shared__ __attribute__((aligned(16))) char shared[OPERANDS > SUMS ? OPERANDS : SUMS];
  _Float16* rows = reinterpret_cast<_Float16*>(shared);
  Tile tile = tile_of(p, blockIdx.y, TILE, false, token);
  if (tile.tokens == 0) return;
  tile.rank = rank_of(p, tile);
  const int first_rank = blockIdx.z * RANKS, ranks = min(tile.rank - first_rank, RANKS);
  if (ranks <= 0) return;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, col = lane & 15, four = lane >> 4;
  const int64_t begin = (int64_t)blockIdx.x * p.part, end = min(begin + p.part, p.n);
  // Row i of LDS: token i, or rank i - TILE.  What there is none of is a row of zeros.
  auto row_of = [&](int u) { return (u * kWaves + wave) * AT_ONCE + (AT_ONCE == 1 ? 0 : lane / OF); };
  const _Float16* from[LOADS];
  bool there[LOADS];
#pragma unroll
  for (int u = 0; u < LOADS; ++u) {
    const int row = row_of(u);
    there[u] = row < TILE ? row < tile.tokens : row - TILE < ranks;
    from[u] = row < TILE ? p.x + token[min(row, tile.tokens - 1)] * p.x_stride
                         : p.down + ((int64_t)tile.adapter * p.rank + first_rank + min(row - TILE, ranks - 1)) * p.n;
  }
  u32x4 next[LOADS];
  auto fetch = [&](int64_t k) {
    const int64_t at = k + 8 * (lane % OF);      // (n is a multiple of 8)
#pragma unroll
    for (int u = 0; u < LOADS; ++u) next[u] = *reinterpret_cast<const u32x4*>(from[u] + min(at, end - 8));
#pragma unroll
    for (int u = 0; u < LOADS; ++u) next[u] = there[u] && at < end ? next[u] : (u32x4){0, 0, 0, 0};
  };
  fetch(begin);
  float4v acc[NT][RT];
#pragma unroll
  for (int i = 0; i < NT * RT; ++i) acc[i / RT][i % RT] = (float4v){0, 0, 0, 0};
  for (int64_t k = begin; k < end; k += CHUNK) {
    if (k != begin) __syncthreads();             // (everybody has read the last columns)
#pragma unroll
    for (int u = 0; u < LOADS; ++u) *reinterpret_cast<u32x4*>(&rows[row_of(u) * PITCH + 8 * (lane % OF)]) = next[u];
    __syncthreads();
    if (k + CHUNK < end) fetch(k + CHUNK);
#pragma unroll
    for (int u = 0; u < STEPS; ++u) {
      const int at = 32 * (u * kWaves + wave) + 8 * four;
      half8v xs[NT];
#pragma unroll
      for (int i = 0; i < NT; ++i) xs[i] = *reinterpret_cast<const half8v*>(&rows[(16 * i + col) * PITCH + at]);
#pragma unroll
      for (int j = 0; j < RT; ++j) {
        const half8v as = *reinterpret_cast<const half8v*>(&rows[(TILE + 16 * j + col) * PITCH + at]);
#pragma unroll
        for (int i = 0; i < NT; ++i) acc[i][j] = mfma(as, xs[i], acc[i][j]);
      }
    }
  }
  __syncthreads();
  float* sums = reinterpret_cast<float*>(shared);      // [wavefront][token][rank]
  constexpr int kPitch = RANKS + 4;
#pragma unroll
  for (int i = 0; i < NT; ++i)
#pragma unroll
    for (int j = 0; j < RT; ++j) *reinterpret_cast<float4v*>(&sums[(wave * TILE + 16 * i + col) * kPitch + 16 * j + 4 * four]) = acc[i][j];
  __syncthreads();
  float* to = p.sums + blockIdx.x * p.part_floats + (int64_t)blockIdx.y * TILE * p.rank + first_rank;
  for (int i = threadIdx.x; i < tile.tokens * (RANKS / 4); i += kThreads) {
    const int t = i / (RANKS / 4), r = i % (RANKS / 4) * 4;
    if (r >= ranks) continue;
    float4v v = *reinterpret_cast<const float4v*>(&sums[t * kPitch + r]);
#pragma unroll
    for (int w = 1; w < kWaves; ++w) v += *reinterpret_cast<const float4v*>(&sums[(w * TILE + t) * kPitch + r]);
    *reinterpret_cast<float4v*>(to + (int64_t)t * p.rank + r) = v;
  }
}

// What the first product's parts have of `tokens` of a tile (`from`: the first part's), added up and scaled: h [token][rank] in LDS, zeros
// beyond the adapter's rank.
__device__ __forceinline__ void add_parts(const AdaptParams& p, const Tile& tile, const float* from, int tokens, float* h) {
  __shared__ __attribute__((aligned(16))) float4v meet[kThreads];
  const int tid = threadIdx.x, items = tokens * p.rank / 4;
  const float scale = p.scales ? p.scales[tile.adapter] : 1.0f;
  // Where there are few numbers to a part the parts are shared out, four or more to each of up to eight sharers, `share` threads apart.
  int share = kThreads;
  while (share / 2 >= items && p.parts > 4 * (kThreads / share) && share > kThreads / 8) share /= 2;
  const int sharers = kThreads / share, mine = tid / share;
  for (int base = 0; base < items; base += share) {
    const int i = base + tid % share;
    float4v s = {0, 0, 0, 0};
    if (i < items) {
      for (int k = mine; k < p.parts; k += 4 * sharers) {
        float4v v[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) v[u] = *reinterpret_cast<const float4v*>(from + min(k + u * sharers, p.parts - 1) * p.part_floats + 4 * (int64_t)i);
#pragma unroll
        for (int u = 0; u < 4; ++u)
          if (k + u * sharers < p.parts) s += v[u];
      }
    }
    if (sharers > 1) {                           // (one turn of the loop)
      meet[tid] = s;
      __syncthreads();
      if (mine != 0) continue;
#pragma unroll
      for (int g = 1; g < 8; ++g)
        if (g < sharers) s += meet[g * share + tid];
    }
    if (i < items) {
      const int r = 4 * i % p.rank;
#pragma unroll
      for (int e = 0; e < 4; ++e) h[4 * i + e] = r + e < tile.rank ? s[e] * scale : 0.0f;      // (beyond the rank there may be anything)
    }
  }
  __syncthreads();
}

// Of many tokens, or 64 to a tile, this is done once for all workgroups of the second product (which otherwise spend a third of their time
// on it: 4096 tokens, 5120 -> 12288, rank 64, three parts: 78 us, 54 without): 16 tokens of a tile, high and low numbers and powers to memory.
__global__ __launch_bounds__(kThreads) void lutgemm_adapt_join_kernel(AdaptParams p, int tile_tokens, int pad) {
  __shared__ float h[16 * kMostRank];
  __shared__ int token[64];
  const int first = 16 * blockIdx.x;
  Tile tile = tile_of(p, blockIdx.y, tile_tokens, false, token);
  const int tokens = min(tile.tokens - first, 16);
  if (tokens <= 0) return;
  tile.rank = rank_of(p, tile);
  if (tile.rank == 0) return;
  add_parts(p, tile, p.sums + ((int64_t)blockIdx.y * tile_tokens + first) * p.rank, tokens, h);
  const int t = threadIdx.x / 16;
  auto value = [&](int r) { return t < tokens && r < tile.rank ? h[t * p.rank + r] : 0.0f; };
  float* to = p.joined + (int64_t)blockIdx.y * tile_tokens * (pad + 1);
  _Float16* high = reinterpret_cast<_Float16*>(to) + (first + t) * pad;
  split_h(threadIdx.x % 16, 16, pad, value, high, high + tile_tokens * pad, reinterpret_cast<int*>(to + tile_tokens * pad) + first + t);
}

// The tile's H for the second product, in LDS: PAD ranks, zeros beyond the adapter's.  What was joined is asked for (`ask`) before
// anything is known of the tile, all of its places.
template <int TILE, int PAD>
struct Joined {
  static constexpr int LOADS = TILE * PAD / 8 / kThreads > 0 ? TILE * PAD / 8 / kThreads : 1;
  static_assert(LOADS <= 4, "in registers meanwhile");
  u32x4 high[LOADS], low[LOADS];
  int drop;
  __device__ __forceinline__ static int at(int u) { return min(u * kThreads + (int)threadIdx.x, TILE * PAD / 8 - 1); }
  __device__ __forceinline__ void ask(const AdaptParams& p) {
    if (!p.joined) return;
    const u32x4* from = reinterpret_cast<const u32x4*>(p.joined + (int64_t)blockIdx.y * TILE * (PAD + 1));
#pragma unroll
    for (int u = 0; u < LOADS; ++u) high[u] = from[at(u)], low[u] = from[TILE * PAD / 8 + at(u)];
    drop = reinterpret_cast<const int*>(from + TILE * PAD / 4)[min((int)threadIdx.x, TILE - 1)];
  }
  __device__ __forceinline__ void put(_Float16* to_high, _Float16* to_low, int pitch, int* to_drop) const {
#pragma unroll
    for (int u = 0; u < LOADS; ++u) {
      const int place = at(u) / (PAD / 8) * pitch + at(u) % (PAD / 8) * 8;
      *reinterpret_cast<u32x4*>(to_high + place) = high[u];
      *reinterpret_cast<u32x4*>(to_low + place) = low[u];
    }
    if (threadIdx.x < TILE) to_drop[threadIdx.x] = drop;
  }
};
template <int TILE, int PAD>
__device__ __forceinline__ void load_h(const AdaptParams& p, const Tile& tile, const Joined<TILE, PAD>& joined, float* h, _Float16* high, _Float16* low, int pitch, int* drop) {
  const int tid = threadIdx.x;
  if (p.joined) {
    joined.put(high, low, pitch, drop);
  } else {
    add_parts(p, tile, p.sums + (int64_t)blockIdx.y * TILE * p.rank, tile.tokens, h);
    constexpr int kEach = kThreads / TILE;       // lanes of a token
    const int t = tid / kEach;
    auto value = [&](int r) { return t < tile.tokens && r < tile.rank ? h[t * p.rank + r] : 0.0f; };
    split_h(tid % kEach, kEach, PAD, value, high + t * pitch, low + t * pitch, drop + t);
  }
  __syncthreads();
}

// What the second product wants to know of a token, in LDS.
struct Target {
  int64_t base, y;             // its rows, in elements
  float one, other;            // the power of two that its results are multiplied with, in two factors: one may leave 32 bits
};

// Four values of a row, which begins on as many bytes as they are together (WIDE) or as one of them is: the compiler knows which and
// has an instruction of any alignment for the second.  Whole calls with values one by one, none of them ahead, took up to 2.2 times as
// long: 1954 tokens, rank 16, 512 -> 28350: 172 us against 84; 2023, rank 128, 5808 -> 20791: 295 against 132.
template <bool WIDE, typename Run, typename Y>
__device__ __forceinline__ Run run_at(const Y* from) {
  if (WIDE) return *reinterpret_cast<const Run*>(from);
  Run v;
  __builtin_memcpy(&v, from, sizeof v);
  return v;
}
template <bool WIDE, typename Run, typename Y>
__device__ __forceinline__ void run_to(Y* to, Run v) {
  if (WIDE)
    *reinterpret_cast<Run*>(to) = v;
  else
    __builtin_memcpy(to, &v, sizeof v);
}

// Y of a tile, for p.rows rows of m (tokens are the rows of the matrix instructions' results, m their columns).  A wavefront takes 64 rows
// of B at a time (BLOCKS times that): they are contiguous in memory, and pass through LDS so that they are read that way and
// are operands dealt out four by four: lane c of a result has rows 4 c .. 4 c + 3 of a token, the 16 lanes of a token
// 64 next to each other.  Up to 16 ranks take half of an instruction's 32: the high numbers of H meet them in one half, the low ones in the
// other.  The next rows are on their way, as is all that the next results are added to: with less of it in flight the latency of memory is
// what a long call takes.  Loads have no branches, so that a wait is for the loads that it needs; what there is none of is the nearest that there is.
template <int TILE, typename Y, int RANKS>
struct Up {
  static constexpr int BLOCKS = RANKS == 16 && TILE == 16 ? 2 : 1, STEPS = (RANKS + 31) / 32, ROWS = 64 * BLOCKS, PAD = 32 * STEPS;
  static constexpr bool AHEAD = RANKS <= 64;     // (of more ranks neither the next rows nor all of these rows' operands fit the registers)
  static constexpr int LOADS = AHEAD ? BLOCKS * RANKS / 8 : 8;
  static constexpr int PITCH = PAD + 8;          // of H (a row's padding keeps rows in different banks)
  static constexpr int STAGE = RANKS + 8;        // of B, an odd number of 16 bytes, as RANKS / 8 is even
  typedef Y Run __attribute__((ext_vector_type(4)));

  const AdaptParams& p;
  const Tile& tile;
  const _Float16 *high, *low, *up;
  _Float16* stage;
  const Target* target;
  int eights;                                    // of a row of B
  uint32_t magic;                                // row = (number * magic) >> 32 of the eights: exact below 2^12
  int lane, col, four;
  u32x4 next[LOADS];

  __device__ __forceinline__ int number_of(int j) const { return min(64 * j + lane, 64 * BLOCKS * eights - 1); }
  __device__ __forceinline__ void fetch(int64_t m0, int j0 = 0) {
    const int end = (int)((p.m - m0) * p.rank) - 8;          // (below 2^28)
    const _Float16* rows = up + m0 * p.rank;
#pragma unroll
    for (int j = 0; j < LOADS; ++j) next[j] = *reinterpret_cast<const u32x4*>(rows + (uint32_t)min(8 * number_of(j0 + j), end));
  }
  __device__ __forceinline__ void put(int j0 = 0) const {
#pragma unroll
    for (int j = 0; j < LOADS; ++j) {
      const int q = number_of(j0 + j), at = eights == 1 ? q : (int)__umulhi((uint32_t)q, magic);
      *reinterpret_cast<u32x4*>(stage + ((at & ~63) + 16 * (at & 3) + (at >> 2 & 15)) * STAGE + 8 * (q - at * eights)) = next[j];
    }
  }
  __device__ __forceinline__ half8v operand(int b, int k, int i, int rank0, u32x4 live, bool masked) const {
    const u32x4 v = *reinterpret_cast<const u32x4*>(stage + (64 * b + 16 * i + col) * STAGE + 32 * k + rank0);
    return __builtin_bit_cast(half8v, masked ? v & live : v);
  }

  // NT times 16 tokens, of which a lane has EACH of each (four, or one: up to four tokens in all).
  template <int NT, int EACH, bool WIDE>
  __device__ __forceinline__ void run(int64_t m0, int64_t last) {
    const int rank0 = 8 * (RANKS == 16 ? four & 1 : four);
    const _Float16* half = RANKS == 16 && four >= 2 ? low : high;
    const int row = 4 * (col & 3) + (col >> 2);  // (row 4 g + e of a matrix result is token 4 e + g: few tokens are all in the lanes' first)
    u32x4 live[STEPS];                           // of the operands: ranks that there are
#pragma unroll
    for (int k = 0; k < STEPS; ++k)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int left = tile.rank - (32 * k + rank0 + 2 * e);
        live[k][e] = left >= 2 ? 0xffffffffu : (left == 1 ? 0xffffu : 0u);
      }
    const bool masked = tile.rank < RANKS;
    constexpr int DEPTH = sizeof(Y) == 4 && NT == 4 ? 2 : NT;        // (fp32 takes twice the registers)
    Run held[DEPTH][EACH][BLOCKS];               // of base, for the next results
    const int64_t end = WIDE || p.m >= 4 ? p.m - 4 : 0;
    auto look = [&](int64_t at, int n) {
#pragma unroll
      for (int e = 0; e < EACH; ++e) {
        const Y* base = static_cast<const Y*>(p.base) + target[min(16 * n + 4 * e + four, tile.tokens - 1)].base;
#pragma unroll
        for (int b = 0; b < BLOCKS; ++b) {
          Run& to = held[n % DEPTH][e][b];
          if (WIDE || p.m >= 4)
            to = run_at<WIDE, Run>(base + min(at + 64 * b + 4 * col, end));
          else
            to = (Run){base[0], base[min(1, (int)p.m - 1)], base[p.m - 1], base[p.m - 1]};
        }
      }
    };
#pragma unroll
    for (int n = 0; n < DEPTH; ++n) look(m0, n);

    for (; m0 < last; m0 += ROWS * kWaves) {
      const int64_t after = m0 + ROWS * kWaves < last ? m0 + ROWS * kWaves : m0;
      half8v bs[BLOCKS][AHEAD ? STEPS : 1][4];
      if (AHEAD) {
        put();
        __builtin_amdgcn_fence(__ATOMIC_SEQ_CST, "wavefront");
        fetch(after);
#pragma unroll
        for (int b = 0; b < BLOCKS; ++b)
#pragma unroll
          for (int k = 0; k < STEPS; ++k)
#pragma unroll
            for (int i = 0; i < 4; ++i) bs[b][k][i] = operand(b, k, i, rank0, live[k], masked);
      } else {
        for (int j = 0; j < eights; j += LOADS) {
          fetch(m0, j);
          put(j);
        }
      }
      __builtin_amdgcn_fence(__ATOMIC_SEQ_CST, "wavefront");
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        float4v acc[BLOCKS][4];
#pragma unroll
        for (int i = 0; i < 4 * BLOCKS; ++i) acc[i / 4][i % 4] = (float4v){0, 0, 0, 0};
#pragma unroll
        for (int k = 0; k < STEPS; ++k) {
          const int at = (16 * n + row) * PITCH + 32 * k + rank0;
          const half8v hs = *reinterpret_cast<const half8v*>(half + at);
          half8v ls;
          if (RANKS > 16) ls = *reinterpret_cast<const half8v*>(low + at);
#pragma unroll
          for (int b = 0; b < BLOCKS; ++b)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const half8v w = AHEAD ? bs[b][AHEAD ? k : 0][i] : operand(b, k, i, rank0, live[k], masked);
              if (RANKS > 16) acc[b][i] = mfma(ls, w, acc[b][i]);
              acc[b][i] = mfma(hs, w, acc[b][i]);
            }
        }
        Run result[EACH][BLOCKS];
#pragma unroll
        for (int e = 0; e < EACH; ++e) {
          const float one = target[16 * n + 4 * e + four].one, other = target[16 * n + 4 * e + four].other;
#pragma unroll
          for (int b = 0; b < BLOCKS; ++b) {
            Run from = held[n % DEPTH][e][b];
            if (!WIDE)                           // (a row's last one to three are behind others, which begin at `end`)
              for (int64_t at = m0 + 64 * b + 4 * col; at > end && at < p.m; --at) from = (Run){from[1], from[2], from[3], from[3]};
#pragma unroll
            for (int i = 0; i < 4; ++i) result[e][b][i] = (Y)fmaf(acc[b][i][e] * one, other, (float)from[i]);
          }
        }
        look(n + DEPTH < NT ? m0 : after, (n + DEPTH) % NT);
#pragma unroll
        for (int e = 0; e < EACH; ++e) {
          const int t = 16 * n + 4 * e + four;
          const Target& to = target[t];
#pragma unroll
          for (int b = 0; b < BLOCKS; ++b) {
            const int64_t m = m0 + 64 * b + 4 * col;
            Y* y = static_cast<Y*>(p.y) + to.y + m;
            if (t < tile.tokens && m + 4 <= p.m) {
              run_to<WIDE>(y, result[e][b]);
            } else if (!WIDE && t < tile.tokens && m < p.m) {
#pragma unroll
              for (int i = 0; i < 3; ++i)
                if (m + i < p.m) y[i] = result[e][b][i];
            }
          }
        }
      }
    }
  }
};

template <int TILE, typename Y, bool WIDE, int RANKS>
__global__ __launch_bounds__(kThreads, TILE == 16 && RANKS <= (WIDE ? 32 : 0) && sizeof(Y) == 2 ? 3 : 2) void lutgemm_adapt_up_kernel(AdaptParams p) {
  typedef Up<TILE, Y, RANKS> U;
  extern __shared__ __attribute__((aligned(16))) char shared[];
  __shared__ int token[TILE];
  __shared__ int drop[TILE];
  __shared__ __attribute__((aligned(16))) Target target[TILE];
  Joined<TILE, U::PAD> joined;
  joined.ask(p);
  Tile tile = tile_of(p, blockIdx.y, TILE, p.copies, token);
  if (tile.tokens == 0) return;
  const int64_t first = (int64_t)blockIdx.x * p.rows, last = min(first + p.rows, p.m);
  _Float16* high = reinterpret_cast<_Float16*>(shared);
  _Float16* low = high + TILE * U::PITCH;
  _Float16* stages = low + TILE * U::PITCH;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int eights = p.rank / 8;
  U u{p, tile, high, low, p.up + (int64_t)min(tile.adapter, p.count - 1) * p.m * p.rank, stages + wave * U::ROWS * U::STAGE, target,
      eights, (uint32_t)((((uint64_t)1 << 32) + eights - 1) / eights), lane, lane & 15, lane >> 4, {}};
  const int64_t m0 = first + U::ROWS * wave;
  if (U::AHEAD) u.fetch(min(m0, last - 1));
  tile.rank = rank_of(p, tile);
  if (tile.rank == 0) {                          // nothing is added
    typedef typename U::Run Run;
    constexpr int kTogether = 8;                 // tokens on their way at a time
    const int end = (int)(last - first) & 3;     // values behind the last four
    if (!WIDE)
      for (int i = threadIdx.x; i < tile.tokens * end; i += kThreads) {
        const int64_t t = token[i / end], m = last - end + i % end;
        static_cast<Y*>(p.y)[t * p.y_stride + m] = static_cast<const Y*>(p.base)[t * p.base_stride + m];
      }
    for (int64_t m = first + 4 * threadIdx.x; m + 4 <= last; m += 4 * kThreads) {
      for (int t0 = 0; t0 < tile.tokens; t0 += kTogether) {
        Run v[kTogether];
#pragma unroll
        for (int u = 0; u < kTogether; ++u) {
          const Y* base = static_cast<const Y*>(p.base) + token[min(t0 + u, tile.tokens - 1)] * p.base_stride + m;
          v[u] = run_at<WIDE, Run>(base);
        }
#pragma unroll
        for (int u = 0; u < kTogether; ++u) {
          Y* y = static_cast<Y*>(p.y) + token[min(t0 + u, tile.tokens - 1)] * p.y_stride + m;
          if (t0 + u < tile.tokens) run_to<WIDE>(y, v[u]);
        }
      }
    }
    return;
  }
  if (threadIdx.x < TILE) {
    const int64_t t = token[min((int)threadIdx.x, tile.tokens - 1)];
    target[threadIdx.x].base = t * p.base_stride;
    target[threadIdx.x].y = t * p.y_stride;
  }
  load_h<TILE, U::PAD>(p, tile, joined, reinterpret_cast<float*>(stages), high, low, U::PITCH, drop);
  if (threadIdx.x < TILE) {
    const int power = drop[threadIdx.x];
    target[threadIdx.x].one = ldexpf(1.0f, power / 2);
    target[threadIdx.x].other = ldexpf(1.0f, power - power / 2);
  }
  __syncthreads();
  if (m0 >= last) return;
  if (tile.tokens <= 4)
    u.template run<1, 1, WIDE>(m0, last);
  else if (TILE == 16 || tile.tokens <= 16)
    u.template run<1, 4, WIDE>(m0, last);
  else
    u.template run<TILE / 16, 4, WIDE>(m0, last);
}

// Ranks as the second product's kernels have them.
int ranks_of(int rank) { return rank <= 16 ? 16 : (rank <= 32 ? 32 : (rank <= 64 ? 64 : (rank <= 128 ? 128 : 256))); }

template <int TILE, typename Y, bool WIDE>
const void* pick_up(int ranks) {
  switch (ranks) {
    case 16: return reinterpret_cast<const void*>(lutgemm_adapt_up_kernel<TILE, Y, WIDE, 16>);
    case 32: return reinterpret_cast<const void*>(lutgemm_adapt_up_kernel<TILE, Y, WIDE, 32>);
    case 64: return reinterpret_cast<const void*>(lutgemm_adapt_up_kernel<TILE, Y, WIDE, 64>);
    case 128: return reinterpret_cast<const void*>(lutgemm_adapt_up_kernel<TILE, Y, WIDE, 128>);
    default: return reinterpret_cast<const void*>(lutgemm_adapt_up_kernel<16, Y, WIDE, 256>);    // (larger tiles are of up to 128)
  }
}
template <int TILE>
const void* pick_up(bool f32, bool wide, int ranks) {
  return f32 ? (wide ? pick_up<TILE, float, true>(ranks) : pick_up<TILE, float, false>(ranks))
             : (wide ? pick_up<TILE, _Float16, true>(ranks) : pick_up<TILE, _Float16, false>(ranks));
}
template <int NT>
const void* pick_down(int ranks) {
  return ranks == 16   ? reinterpret_cast<const void*>(lutgemm_adapt_down_kernel<NT, 16, NT == 1 ? 512 : 256>)
         : ranks == 32 ? reinterpret_cast<const void*>(lutgemm_adapt_down_kernel<NT, 32, NT == 1 ? 512 : 256>)
                       : reinterpret_cast<const void*>(lutgemm_adapt_down_kernel<NT, kRankBlock, 256>);
}

int launch(const void* kern, dim3 grid, int threads, void** args, size_t lds, void* stream) {
  return hipLaunchKernel(kern, grid, dim3(threads), args, lds, static_cast<hipStream_t>(stream)) == hipSuccess ? LUTGEMM_OK : LUTGEMM_EHIP;
}

}  // namespace

extern "C" int lutgemm_adapt(const void* x, const void* base, const lutgemm_adapters* adapters, const int32_t* of, const int32_t* owner, void* y,
                             int tokens, int seqs, int64_t x_stride, int64_t base_stride, int64_t y_stride, unsigned flags, void* workspace,
                             size_t workspace_bytes, void* hip_stream) {
  int rc = check_adapters(adapters, tokens);
  if (rc != LUTGEMM_OK) return rc;
  const lutgemm_adapters& a = *adapters;
  if (!x || !base || !y || !of || !workspace || !a.down || !a.up || (owner && seqs < 1)) return LUTGEMM_EINVAL;
  if ((flags & ~(unsigned)LUTGEMM_Y_F32) != 0) return LUTGEMM_EUNSUPPORTED;
  const uintptr_t size = flags & LUTGEMM_Y_F32 ? 4 : 2;
  if ((((uintptr_t)x | (uintptr_t)a.down | (uintptr_t)a.up | (uintptr_t)workspace) & 15) != 0) return LUTGEMM_EINVAL;
  if ((((uintptr_t)of | (uintptr_t)owner | (uintptr_t)a.ranks | (uintptr_t)a.scales) & 3) != 0 || ((uintptr_t)base | (uintptr_t)y) % size != 0) return LUTGEMM_EINVAL;
  if (x_stride < a.n || x_stride % 8 != 0 || base_stride < a.m || y_stride < a.m || (base == y && base_stride != y_stride)) return LUTGEMM_EINVAL;
  if (x_stride > kMostAdaptStride || base_stride > kMostAdaptStride || y_stride > kMostAdaptStride) return LUTGEMM_EUNSUPPORTED;
  const AdaptPlan plan = plan_adapt(adapters, tokens);
  const int64_t ints = adapt_table_ints(plan, tokens), part_floats = adapt_part_floats(plan, a.rank);
  if (workspace_bytes < (size_t)(kCounterBytes + 4 * (ints + plan.parts * part_floats + adapt_joined_floats(plan, tokens, a.rank)))) return LUTGEMM_EWORKSPACE;
  if (tokens == 0) return LUTGEMM_OK;
  const Rows x_rows = rows_of(x, tokens, x_stride, a.n, 2), base_rows = rows_of(base, tokens, base_stride, a.m, (int64_t)size), y_rows = rows_of(y, tokens, y_stride, a.m, (int64_t)size);
  if (!apart(x_rows, y_rows) || (base != y && !apart(base_rows, y_rows))) return LUTGEMM_EINVAL;
  AdaptParams p = {};
  p.x = static_cast<const _Float16*>(x);
  p.base = base;
  p.y = y;
  p.down = static_cast<const _Float16*>(a.down);
  p.up = static_cast<const _Float16*>(a.up);
  p.of = of;
  p.owner = owner;
  p.ranks = a.ranks;
  p.scales = a.scales;
  p.table = reinterpret_cast<int32_t*>(static_cast<char*>(workspace) + kCounterBytes);
  p.sums = reinterpret_cast<float*>(p.table + ints);
  p.joined = adapt_joins(plan, tokens) ? p.sums + plan.parts * part_floats : nullptr;
  p.x_stride = x_stride;
  p.base_stride = base_stride;
  p.y_stride = y_stride;
  p.m = a.m;
  p.n = a.n;
  p.part_floats = part_floats;
  p.tokens = tokens;
  p.seqs = seqs;
  p.count = a.count;
  p.rank = a.rank;
  p.tiles = plan.tiles;
  p.parts = plan.parts;
  p.part = plan.part;
  p.rows = plan.rows;
  p.copies = base != y;
  if (tokens > kFewTokens) {
    int cut = plan.tile;
    void* args[] = {&p, &cut};
    rc = launch(reinterpret_cast<const void*>(lutgemm_adapt_sort_kernel), dim3(1), kSortThreads, args, 4 * (size_t)((kSortWaves + 2) * (a.count + 1) + 1), hip_stream);
    if (rc != LUTGEMM_OK) return rc;
  }
  void* args[] = {&p};
  const int ranks = ranks_of(a.rank);
  const int at_once = ranks < kRankBlock ? ranks : kRankBlock;
  const void* down = plan.tile == 16 ? pick_down<1>(ranks) : (plan.tile == 32 ? pick_down<2>(ranks) : pick_down<4>(ranks));
  rc = launch(down, dim3(plan.parts, plan.tiles, (a.rank + at_once - 1) / at_once), kThreads, args, 0, hip_stream);
  if (rc != LUTGEMM_OK) return rc;
  if (p.joined) {
    int tile = plan.tile, pad = ranks < 32 ? 32 : ranks;
    void* join_args[] = {&p, &tile, &pad};
    rc = launch(reinterpret_cast<const void*>(lutgemm_adapt_join_kernel), dim3(plan.tile / 16, plan.tiles), kThreads, join_args, 0, hip_stream);
    if (rc != LUTGEMM_OK) return rc;
  }
  const bool wide = (((uintptr_t)base | (uintptr_t)y | (uintptr_t)(base_stride * size) | (uintptr_t)(y_stride * size)) & (4 * size - 1)) == 0 && a.m % 4 == 0;
  const int pitch = (ranks < 32 ? 32 : ranks) + 8;
  const size_t lds = 2 * (size_t)(2 * plan.tile * pitch + kWaves * (ranks == 16 && plan.tile == 16 ? 128 : 64) * (ranks + 8));
  const void* up = plan.tile == 16 ? pick_up<16>(size == 4, wide, ranks) : (plan.tile == 32 ? pick_up<32>(size == 4, wide, ranks) : pick_up<64>(size == 4, wide, ranks));
  return launch(up, dim3((a.m + plan.rows - 1) / plan.rows, plan.tiles), kThreads, args, lds, hip_stream);
}
