// Low-rank adapters of many requests beside a product whose weights they share: y[t] = base[t] + c_a B_a (A_a x[t]), a the adapter of
// token t.  include/lutgemm.h has the layouts.
//
// Tokens with the same adapter are taken together, up to TILE of them, so that its A and B are read once for them: of up to 64 tokens
// every wavefront finds the tiles by itself, from a ballot over the bits of their adapters; of more a kernel of one workgroup sorts them
// first.  Then two products on the 16 x 16 x 32 matrix instructions, transposed (a lane owns a token):
//     H^T (ranks x tokens) = A (ranks x n) X^T,      Y^T (m x tokens) = B (m x ranks) H^T
// Both stream A and B, which is what bounds a decode step (2 r (n + m) bytes an adapter).  n is shared out among workgroups; their
// sums meet where the second product reads them, in an order that the sizes decide.  H stays fp32 there, and meets B as two fp16 numbers
// (22 bits) of a power of two that the token's largest decides: rounded to one, it would add as much error as the
// result's own rounding to fp16, and more than that of fp32 results.
#include <hip/hip_fp16.h>
#include <hip/hip_runtime.h>

#include "lutgemm_step.h"

using namespace lutgemm_step_detail;

namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef _Float16 half8v __attribute__((ext_vector_type(8)));
typedef _Float16 half4v __attribute__((ext_vector_type(4)));
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
  int32_t* table;              // tiles by number, then the tokens by adapter
  float* sums;
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

// A tile: its adapter, how many tokens it has (0: there is no such tile, or nothing to do for it), which ones (of the workgroup, in LDS).
struct Tile {
  int adapter, tokens, rank;
};
template <int TILE>
__device__ __forceinline__ Tile tile_of(const AdaptParams& p, int number, bool copies, int* token) {
  Tile t = {p.count, 0, 0};
  if (p.tokens <= kFewTokens) {
    const int lane = threadIdx.x & 63;
    const bool live = lane < p.tokens;
    const int mine = live ? adapter_of(p, lane) : -1;
    uint64_t same = __ballot(live);
    for (int bit = 1; bit <= p.count; bit *= 2) {
      const uint64_t set = __ballot((mine & bit) != 0);
      same &= (mine & bit) != 0 ? set : ~set;
    }
    const uint64_t below = ((uint64_t)1 << lane) - 1;
    const int rank = __popcll(same & below);
    const uint64_t heads = __ballot(live && rank % TILE == 0);
    const uint64_t chosen = __ballot(live && rank % TILE == 0 && __popcll(heads & below) == number);
    if (chosen != 0) {
      const int head = __builtin_ctzll(chosen);
      t.adapter = __builtin_amdgcn_readlane(mine, head);
      const int from = __builtin_amdgcn_readlane(rank, head);
      const bool member = live && mine == t.adapter && rank >= from && rank < from + TILE;
      t.tokens = __popcll(__ballot(member));
      if (threadIdx.x < 64 && member) token[rank - from] = lane;
    }
  } else if (number < p.table[0]) {
    const int32_t* entry = p.table + 4 + 4 * number;
    t.adapter = entry[0];
    t.tokens = entry[2];
    const int32_t* order = p.table + 4 + 4 * p.tiles + entry[1];
    if ((int)threadIdx.x < t.tokens) token[threadIdx.x] = order[threadIdx.x];
  }
  if (t.adapter >= p.count && !copies) t.tokens = 0;
  if (t.adapter < p.count) t.rank = p.ranks ? min(max(p.ranks[t.adapter], 0), p.rank) : p.rank;
  __syncthreads();
  return t;
}

// Sorts the tokens by adapter, each adapter's in their order, and cuts them into tiles.  One workgroup; a wavefront has every 16th
// run of 64 tokens and counts of its own, so that no count depends on an order of arrival.
constexpr int kSortThreads = 1024, kSortWaves = kSortThreads / 64;
__global__ __launch_bounds__(kSortThreads) void lutgemm_adapt_sort_kernel(AdaptParams p, int tile) {
  extern __shared__ int32_t counts[];            // [wavefront][adapter], then the adapters' begins and first tiles
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, kinds = p.count + 1;
  int32_t* begins = counts + kSortWaves * kinds;
  int32_t* tiles = begins + kinds + 1;
  for (int i = tid; i < kSortWaves * kinds; i += kSortThreads) counts[i] = 0;
  __syncthreads();
  int32_t* mine = counts + wave * kinds;
  const int each = (p.tokens + kSortThreads - 1) / kSortThreads * 64;      // tokens of a wavefront, next to each other
  for (int turn = 0; turn < 2; ++turn) {
    constexpr int kAhead = 8;
    int ahead[kAhead];
    for (int i = 0; i < each; i += 64) {
      const int token = wave * each + i + lane, k = i / 64 % kAhead;
      if (k == 0) {                              // (the next runs' are looked up together)
#pragma unroll
        for (int u = 0; u < kAhead; ++u) ahead[u] = token + 64 * u < p.tokens && i + 64 * u < each ? adapter_of(p, token + 64 * u) : -1;
      }
      int a = ahead[0];
#pragma unroll
      for (int u = 1; u < kAhead; ++u) a = k == u ? ahead[u] : a;
      const bool live = a >= 0;
      uint64_t same = __ballot(live);
      for (int bit = 1; bit <= p.count; bit *= 2) {
        const uint64_t set = __ballot((a & bit) != 0);
        same &= (a & bit) != 0 ? set : ~set;
      }
      const int rank = __popcll(same & (((uint64_t)1 << lane) - 1));
      if (live) {
        const int at = mine[a];
        if (turn == 1) p.table[4 + 4 * p.tiles + at + rank] = token;
        __builtin_amdgcn_wave_barrier();
        if (rank == 0) mine[a] = at + __popcll(same);
      }
      __builtin_amdgcn_fence(__ATOMIC_SEQ_CST, "wavefront");
    }
    if (turn == 1) break;
    __syncthreads();
    // counts become places: of each adapter over the wavefronts, then over the adapters (which one wavefront adds up)
    for (int a = tid; a < kinds; a += kSortThreads) {
      int sum = 0;
      for (int w = 0; w < kSortWaves; ++w) sum += counts[w * kinds + a];
      begins[a] = sum;
    }
    __syncthreads();
    if (wave == 0) {
      int tokens = 0, cut = 0;
      for (int base = 0; base < kinds; base += 64) {
        const int a = base + lane;
        const int have = a < kinds ? begins[a] : 0, pieces = (have + tile - 1) / tile;
        int t = have, c = pieces;
#pragma unroll
        for (int d = 1; d < 64; d *= 2) {
          const int ot = __shfl_up(t, d), oc = __shfl_up(c, d);
          if (lane >= d) t += ot, c += oc;
        }
        if (a < kinds) {
          begins[a] = tokens + t - have;
          tiles[a] = cut + c - pieces;
        }
        tokens += __shfl(t, 63);
        cut += __shfl(c, 63);
      }
      if (lane == 0) {
        begins[kinds] = tokens;
        tiles[kinds] = cut;
        p.table[0] = cut;
      }
    }
    __syncthreads();
    for (int a = tid; a < kinds; a += kSortThreads) {
      int at = begins[a];
      for (int w = 0; w < kSortWaves; ++w) {
        const int have = counts[w * kinds + a];
        counts[w * kinds + a] = at;
        at += have;
      }
    }
    for (int i = tid; i < tiles[kinds]; i += kSortThreads) {     // the adapter of a tile: the last whose first tile is not behind it
      int lo = 0, hi = kinds - 1;
      while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (tiles[mid] <= i)
          lo = mid;
        else
          hi = mid - 1;
      }
      const int from = begins[lo] + (i - tiles[lo]) * tile;
      int32_t* entry = p.table + 4 + 4 * i;
      entry[0] = lo;
      entry[1] = from;
      entry[2] = min(begins[lo + 1] - from, tile);
    }
    __syncthreads();
  }
}

// H^T of a tile, for a part of the columns and RANKS of its ranks: four wavefronts take a quarter of the part each, AHEAD steps of 32 columns
// on their way at a time.
constexpr int kThreads = 256, kWaves = kThreads / 64;
template <int TILE, int RANKS>
__global__ __launch_bounds__(kThreads) void lutgemm_adapt_down_kernel(AdaptParams p) {
  constexpr int NT = TILE / 16, RT = RANKS / 16, AHEAD = NT * RT >= 8 ? 2 : 4;
  __shared__ int token[TILE];
  __shared__ __attribute__((aligned(16))) float sums[kWaves][TILE][RANKS + 4];
  const Tile tile = tile_of<TILE>(p, blockIdx.y, false, token);
  const int first_rank = blockIdx.z * RANKS;
  if (tile.tokens == 0 || first_rank >= tile.rank) return;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, col = lane & 15, eight = 8 * (lane >> 4);
  const int64_t begin = (int64_t)blockIdx.x * p.part + wave * (p.part / kWaves), end = min(begin + p.part / kWaves, p.n);
  const _Float16* x[NT];
  const _Float16* a[RT];
#pragma unroll
  for (int i = 0; i < NT; ++i) x[i] = p.x + token[min(16 * i + col, tile.tokens - 1)] * p.x_stride;       // (a dead column's lane reads a live one's row)
#pragma unroll
  for (int j = 0; j < RT; ++j) a[j] = p.down + ((int64_t)tile.adapter * p.rank + min(first_rank + 16 * j + col, p.rank - 1)) * p.n;
  float4v acc[NT][RT];
#pragma unroll
  for (int i = 0; i < NT; ++i)
#pragma unroll
    for (int j = 0; j < RT; ++j) acc[i][j] = (float4v){0, 0, 0, 0};
  for (int64_t k = begin; k < end; k += 32 * AHEAD) {
    half8v xs[AHEAD][NT], as[AHEAD][RT];
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) {
      const int64_t at = min(k + 32 * u + eight, p.n - 8);        // (n is a multiple of 8)
#pragma unroll
      for (int i = 0; i < NT; ++i) xs[u][i] = *reinterpret_cast<const half8v*>(x[i] + at);
#pragma unroll
      for (int j = 0; j < RT; ++j) as[u][j] = *reinterpret_cast<const half8v*>(a[j] + at);
    }
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) {
      if (k + 32 * u + 32 > end) {               // columns that there are not, or that are another wavefront's
        const bool inside = k + 32 * u + eight < end;
        const half8v none = {0, 0, 0, 0, 0, 0, 0, 0};
#pragma unroll
        for (int i = 0; i < NT; ++i) xs[u][i] = inside ? xs[u][i] : none;
#pragma unroll
        for (int j = 0; j < RT; ++j) as[u][j] = inside ? as[u][j] : none;
      }
#pragma unroll
      for (int i = 0; i < NT; ++i)
#pragma unroll
        for (int j = 0; j < RT; ++j) acc[i][j] = mfma(as[u][j], xs[u][i], acc[i][j]);
    }
  }
#pragma unroll
  for (int i = 0; i < NT; ++i)
#pragma unroll
    for (int j = 0; j < RT; ++j) *reinterpret_cast<float4v*>(&sums[wave][16 * i + col][16 * j + 4 * (lane >> 4)]) = acc[i][j];
  __syncthreads();
  float* to = p.sums + blockIdx.x * p.part_floats + (int64_t)blockIdx.y * TILE * p.rank + first_rank;
  for (int i = threadIdx.x; i < tile.tokens * (RANKS / 4); i += kThreads) {
    const int t = i / (RANKS / 4), r = i % (RANKS / 4) * 4;
    if (first_rank + r >= p.rank) continue;
    float4v s = *reinterpret_cast<const float4v*>(&sums[0][t][r]);
#pragma unroll
    for (int w = 1; w < kWaves; ++w) s += *reinterpret_cast<const float4v*>(&sums[w][t][r]);
    *reinterpret_cast<float4v*>(to + (int64_t)t * p.rank + r) = s;
  }
}

// The tile's A x, added up over the parts and scaled, as two fp16 numbers of a power of two that brings a token's largest to 2^14 .. 2^15
// (so that neither overflows, and what is lost is 2^-22 of the largest), [token][rank] in LDS.
template <int TILE>
__device__ __forceinline__ void load_h(const AdaptParams& p, const Tile& tile, int steps, float* h, _Float16* high, _Float16* low, int pitch, int* drop) {
  __shared__ __attribute__((aligned(16))) float4v meet[kThreads];
  const int tid = threadIdx.x, items = tile.tokens * p.rank / 4;
  const float scale = p.scales ? p.scales[tile.adapter] : 1.0f;
  const float* from = p.sums + (int64_t)blockIdx.y * TILE * p.rank;
  // Where there are few numbers to a part the parts are shared out: sharers are 256 / share threads apart.
  int share = kThreads;
  while (share / 2 >= items && share > 1) share /= 2;
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
      for (int g = 1; g < sharers; ++g) s += meet[g * share + tid];
    }
    if (i < items) {
      const int r = 4 * i % p.rank;
#pragma unroll
      for (int e = 0; e < 4; ++e) h[4 * i + e] = r + e < tile.rank ? s[e] * scale : 0.0f;      // (beyond the rank there may be anything)
    }
  }
  __syncthreads();
  constexpr int kOf = kThreads / TILE;           // lanes of a token
  const int t = tid / kOf, part = tid % kOf;
  float top = 0.0f;
  if (t < tile.tokens)
    for (int r = part; r < tile.rank; r += kOf) top = fmaxf(top, fabsf(h[t * p.rank + r]));
#pragma unroll
  for (int d = 1; d < kOf; d *= 2) top = fmaxf(top, __shfl_xor(top, d));
  // (no power where the largest is an infinity: the result is no number then; or zero)
  const int lift = top > 0.0f && top < __builtin_inff() ? 15 - __builtin_amdgcn_frexp_expf(top) : 0;
  for (int r = part; r < 32 * steps; r += kOf) {
    const float v = t < tile.tokens && r < tile.rank ? ldexpf(h[t * p.rank + r], lift) : 0.0f;
    const _Float16 hi = (_Float16)v;
    high[t * pitch + r] = hi;
    low[t * pitch + r] = fabsf((float)hi) < __builtin_inff() ? (_Float16)(v - (float)hi) : (_Float16)0.0f;
  }
  if (part == 0) drop[t] = -lift;
  __syncthreads();
}

// Y^T of a tile, for p.rows rows of m.  A wavefront takes 64 rows at a time as four matrix tiles, dealt so that every 16 bytes of
// a lane's results are next to those of the three lanes that have the same token.  STEPS: of 32 ranks, whose operands are in registers; of up to
// two the next rows' are on their way, as is what the next results are added to.
template <int TILE, typename Y, bool WIDE, int STEPS>
__global__ __launch_bounds__(kThreads) void lutgemm_adapt_up_kernel(AdaptParams p) {
  constexpr int NT = TILE / 16, RUN = 16 / sizeof(Y), RUNS = 16 / RUN;   // a lane's 16 rows: RUNS runs of RUN
  constexpr bool AHEAD = STEPS <= 2;
  extern __shared__ __attribute__((aligned(16))) char shared[];
  __shared__ int token[TILE];
  __shared__ int drop[TILE];                     // the power of two that a token's results are multiplied with
  const Tile tile = tile_of<TILE>(p, blockIdx.y, p.copies, token);
  if (tile.tokens == 0) return;
  constexpr int pitch = 32 * STEPS + 8;          // (a row's padding keeps rows in different banks)
  float* h = reinterpret_cast<float*>(shared);
  _Float16* high = reinterpret_cast<_Float16*>(h + TILE * p.rank);
  _Float16* low = high + TILE * pitch;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, col = lane & 15, four = lane >> 4;
  const int64_t last = min((int64_t)(blockIdx.x + 1) * p.rows, p.m);
  const _Float16* up = p.up + (int64_t)min(tile.adapter, p.count - 1) * p.m * p.rank;
  // The row of m that lane `col` of matrix tile i reads: row 4 g + e of it is row e % RUN of run 4 (i * 4 + e) / RUN of lane g.
  const int own = RUN == 4 ? col : 8 * (col >> 2) + (col & 3);
  u32x4 next[STEPS][4];
  auto fetch = [&](int64_t m0) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const _Float16* row = up + min(m0 + own + (RUN == 4 ? 16 * i : 32 * (i >> 1) + 4 * (i & 1)), p.m - 1) * p.rank;
#pragma unroll
      for (int k = 0; k < STEPS; ++k) next[k][i] = *reinterpret_cast<const u32x4*>(row + min(32 * k + 8 * four, p.rank - 8));
    }
  };
  int64_t m0 = (int64_t)blockIdx.x * p.rows + 64 * wave;
  if (AHEAD) fetch(m0);
  u32x4 held[RUNS];                              // of base, for the next results
  auto look = [&](int64_t at, int n) {
    if (!WIDE || 16 * n + col >= tile.tokens) return;
    const Y* base = static_cast<const Y*>(p.base) + token[16 * n + col] * p.base_stride;
#pragma unroll
    for (int c = 0; c < RUNS; ++c) {
      const int64_t m = at + 4 * RUN * c + RUN * four;
      if (m + RUN <= p.m) held[c] = *reinterpret_cast<const u32x4*>(base + m);
    }
  };
  look(m0, 0);
  if (tile.rank > 0) load_h<TILE>(p, tile, STEPS, h, high, low, pitch, drop);
  u32x4 live[STEPS];                             // of the operands: ranks that there are
#pragma unroll
  for (int k = 0; k < STEPS; ++k)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int left = tile.rank - (32 * k + 8 * four + 2 * e);
      live[k][e] = left >= 2 ? 0xffffffffu : (left == 1 ? 0xffffu : 0u);
    }

  for (; m0 < last; m0 += 64 * kWaves) {
    if (!AHEAD) fetch(m0);
    half8v bs[STEPS][4];
#pragma unroll
    for (int k = 0; k < STEPS; ++k)
#pragma unroll
      for (int i = 0; i < 4; ++i) bs[k][i] = __builtin_bit_cast(half8v, next[k][i] & live[k]);
    const bool more = m0 + 64 * kWaves < last;
    if (AHEAD && more) fetch(m0 + 64 * kWaves);
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      const int t = 16 * n + col;
      u32x4 base[RUNS];
#pragma unroll
      for (int c = 0; c < RUNS; ++c) base[c] = held[c];
      if (n + 1 < NT)
        look(m0, n + 1);
      else if (more)
        look(m0 + 64 * kWaves, 0);
      float4v acc[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) acc[i] = (float4v){0, 0, 0, 0};
      if (tile.rank > 0) {
#pragma unroll
        for (int k = 0; k < STEPS; ++k) {
          const half8v hi = *reinterpret_cast<const half8v*>(high + t * pitch + 32 * k + 8 * four);
          const half8v lo = *reinterpret_cast<const half8v*>(low + t * pitch + 32 * k + 8 * four);
#pragma unroll
          for (int i = 0; i < 4; ++i) acc[i] = mfma(bs[k][i], hi, mfma(bs[k][i], lo, acc[i]));
        }
      }
      if (t >= tile.tokens) continue;
      const int power = tile.rank > 0 ? drop[t] : 0;
      const Y* from = static_cast<const Y*>(p.base) + token[t] * p.base_stride;
      Y* y = static_cast<Y*>(p.y) + token[t] * p.y_stride;
#pragma unroll
      for (int c = 0; c < RUNS; ++c) {
        const int64_t m = m0 + 4 * RUN * c + RUN * four;
        float d[RUN];
#pragma unroll
        for (int e = 0; e < RUN; ++e) d[e] = ldexpf(acc[c * (RUN / 4) + e / 4][e % 4], power);
        if (WIDE && m + RUN <= p.m) {
          Y v[RUN];
          *reinterpret_cast<u32x4*>(v) = base[c];
#pragma unroll
          for (int e = 0; e < RUN; ++e) v[e] = tile.rank > 0 ? (Y)((float)v[e] + d[e]) : v[e];
          *reinterpret_cast<u32x4*>(y + m) = *reinterpret_cast<const u32x4*>(v);
        } else {
#pragma unroll
          for (int e = 0; e < RUN; ++e)
            if (m + e < p.m) y[m + e] = tile.rank > 0 ? (Y)((float)from[m + e] + d[e]) : from[m + e];
        }
      }
    }
  }
}

template <int TILE, typename Y, bool WIDE>
const void* pick_up(int rank) {
  return rank <= 32   ? reinterpret_cast<const void*>(lutgemm_adapt_up_kernel<TILE, Y, WIDE, 1>)
         : rank <= 64 ? reinterpret_cast<const void*>(lutgemm_adapt_up_kernel<TILE, Y, WIDE, 2>)
         : rank <= 128 ? reinterpret_cast<const void*>(lutgemm_adapt_up_kernel<TILE, Y, WIDE, 4>)
                      : reinterpret_cast<const void*>(lutgemm_adapt_up_kernel<(TILE < 64 ? TILE : 32), Y, WIDE, 8>);
}
template <int TILE>
const void* pick_up(bool f32, bool wide, int rank) {
  return f32 ? (wide ? pick_up<TILE, float, true>(rank) : pick_up<TILE, float, false>(rank))
             : (wide ? pick_up<TILE, _Float16, true>(rank) : pick_up<TILE, _Float16, false>(rank));
}
template <int TILE>
const void* pick_down(int rank) {
  return rank <= 16   ? reinterpret_cast<const void*>(lutgemm_adapt_down_kernel<TILE, 16>)
         : rank <= 32 ? reinterpret_cast<const void*>(lutgemm_adapt_down_kernel<TILE, 32>)
                      : reinterpret_cast<const void*>(lutgemm_adapt_down_kernel<TILE, 64>);
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
  const AdaptPlan plan = plan_adapt(adapters, tokens);
  const int64_t ints = adapt_table_ints(plan, tokens), part_floats = adapt_part_floats(plan, a.rank);
  if (workspace_bytes < (size_t)(kCounterBytes + 4 * (ints + plan.parts * part_floats))) return LUTGEMM_EWORKSPACE;
  if (tokens == 0) return LUTGEMM_OK;
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
    int tile = plan.tile;
    void* args[] = {&p, &tile};
    rc = launch(reinterpret_cast<const void*>(lutgemm_adapt_sort_kernel), dim3(1), kSortThreads, args, 4 * (size_t)((kSortWaves + 2) * (a.count + 1) + 2), hip_stream);
    if (rc != LUTGEMM_OK) return rc;
  }
  void* args[] = {&p};
  const int ranks = a.rank <= 16 ? 16 : (a.rank <= 32 ? 32 : kRankBlock);
  const void* down = plan.tile == 16 ? pick_down<16>(a.rank) : (plan.tile == 32 ? pick_down<32>(a.rank) : pick_down<64>(a.rank));
  rc = launch(down, dim3(plan.parts, plan.tiles, (a.rank + ranks - 1) / ranks), kThreads, args, 0, hip_stream);
  if (rc != LUTGEMM_OK) return rc;
  const bool wide = (((uintptr_t)base | (uintptr_t)y | (uintptr_t)(base_stride * size) | (uintptr_t)(y_stride * size)) & 15) == 0;
  const int pitch = 32 * (a.rank <= 32 ? 1 : (a.rank <= 64 ? 2 : (a.rank <= 128 ? 4 : 8))) + 8;
  const size_t lds = (size_t)plan.tile * (4 * a.rank + 4 * pitch);
  const void* up = plan.tile == 16 ? pick_up<16>(size == 4, wide, a.rank) : (plan.tile == 32 ? pick_up<32>(size == 4, wide, a.rank) : pick_up<64>(size == 4, wide, a.rank));
  return launch(up, dim3((a.m + plan.rows - 1) / plan.rows, plan.tiles), kThreads, args, lds, hip_stream);
}
