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
    for (int i = 0; i < each; i += 64) {
      const int token = wave * each + i + lane;
      const bool live = token < p.tokens;
      const int a = live ? adapter_of(p, token) : -1;
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
        p.table[0] = cut;
      }
    }
    __syncthreads();
    for (int a = tid; a < kinds; a += kSortThreads) {
      const int end = begins[a + 1];
      int at = begins[a], number = tiles[a];
      for (int from = at; from < end; from += tile, ++number) {
        int32_t* entry = p.table + 4 + 4 * number;
        entry[0] = a;
        entry[1] = from;
        entry[2] = min(end - from, tile);
      }
      for (int w = 0; w < kSortWaves; ++w) {
        const int have = counts[w * kinds + a];
        counts[w * kinds + a] = at;
        at += have;
      }
    }
    __syncthreads();
  }
}

// H^T of a tile, for a part of the columns and RANKS of its ranks: four wavefronts take a quarter of the part each.
constexpr int kThreads = 256, kWaves = kThreads / 64;
template <int TILE, int RANKS>
__global__ __launch_bounds__(kThreads) void lutgemm_adapt_down_kernel(AdaptParams p) {
  constexpr int NT = TILE / 16, RT = RANKS / 16;
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
  for (int64_t k = begin; k < end; k += 32) {
    const bool inside = k + eight < end;         // (n is a multiple of 8)
    const int64_t at = inside ? k + eight : 0;
    half8v xs[NT], as[RT];
#pragma unroll
    for (int i = 0; i < NT; ++i) xs[i] = *reinterpret_cast<const half8v*>(x[i] + at);
#pragma unroll
    for (int j = 0; j < RT; ++j) as[j] = *reinterpret_cast<const half8v*>(a[j] + at);
    const half8v none = {0, 0, 0, 0, 0, 0, 0, 0};
#pragma unroll
    for (int i = 0; i < NT; ++i) xs[i] = inside ? xs[i] : none;
#pragma unroll
    for (int j = 0; j < RT; ++j) as[j] = inside ? as[j] : none;
#pragma unroll
    for (int i = 0; i < NT; ++i)
#pragma unroll
      for (int j = 0; j < RT; ++j) acc[i][j] = mfma(as[j], xs[i], acc[i][j]);
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

// Y^T of a tile, for p.rows rows of m.  A wavefront takes 64 rows at a time as four matrix tiles, dealt so that a lane's results are 16
// rows of its token next to each other (row 16 g + 4 i + e is row 4 g + e of tile i).
template <int TILE, typename Y, bool WIDE>
__global__ __launch_bounds__(kThreads) void lutgemm_adapt_up_kernel(AdaptParams p) {
  constexpr int NT = TILE / 16;
  extern __shared__ __attribute__((aligned(16))) char shared[];
  __shared__ int token[TILE];
  __shared__ float back[TILE];                   // what a token's results are multiplied with
  const Tile tile = tile_of<TILE>(p, blockIdx.y, p.copies, token);
  if (tile.tokens == 0) return;
  const int steps = (tile.rank + 31) / 32, pitch = 32 * ((p.rank + 31) / 32) + 8;      // (a row's padding keeps rows in different banks)
  float* h = reinterpret_cast<float*>(shared);
  _Float16* high = reinterpret_cast<_Float16*>(h + TILE * p.rank);
  _Float16* low = high + TILE * pitch;
  if (tile.rank > 0) {
    const float scale = p.scales ? p.scales[tile.adapter] : 1.0f;
    const float* from = p.sums + (int64_t)blockIdx.y * TILE * p.rank;
    for (int i = threadIdx.x; i < tile.tokens * p.rank; i += kThreads) {
      float s = 0.0f;
      if (i % p.rank < tile.rank) {
        s = from[i];
        for (int k = 1; k < p.parts; ++k) s += from[k * p.part_floats + i];
        s *= scale;
      }
      h[i] = s;
    }
    __syncthreads();
    constexpr int kOf = kThreads / TILE;         // lanes of a token
    const int t = threadIdx.x / kOf, part = threadIdx.x % kOf;
    float top = 0.0f;
    if (t < tile.tokens)
      for (int r = part; r < tile.rank; r += kOf) top = fmaxf(top, fabsf(h[t * p.rank + r]));
#pragma unroll
    for (int d = 1; d < kOf; d *= 2) top = fmaxf(top, __shfl_xor(top, d));
    // a power of two that brings the largest to 2^14 .. 2^15; none where it is an infinity (the result is no number then), or zero
    int lift = 0;
    if (top > 0.0f && top < __builtin_inff()) lift = 15 - __builtin_amdgcn_frexp_expf(top);
    for (int r = part; r < 32 * steps; r += kOf) {
      const float v = t < tile.tokens && r < tile.rank ? ldexpf(h[t * p.rank + r], lift) : 0.0f;
      const _Float16 hi = (_Float16)v;
      const float rest = v - (float)hi;
      high[t * pitch + r] = hi;
      low[t * pitch + r] = fabsf((float)hi) < __builtin_inff() ? (_Float16)rest : (_Float16)0.0f;
    }
    if (part == 0) back[t] = (float)lift;
    __syncthreads();
  }
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, col = lane & 15, four = lane >> 4;
  const int64_t last = min((int64_t)(blockIdx.x + 1) * p.rows, p.m);
  for (int64_t m0 = (int64_t)blockIdx.x * p.rows + 64 * wave; m0 < last; m0 += 64 * kWaves) {
    const _Float16* b[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) b[i] = p.up + ((int64_t)min(tile.adapter, p.count - 1) * p.m + min(m0 + 16 * (col >> 2) + 4 * i + (col & 3), p.m - 1)) * p.rank;
    float4v acc[NT][4];
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int i = 0; i < 4; ++i) acc[n][i] = (float4v){0, 0, 0, 0};
    for (int k = 0; k < steps; ++k) {
      const int r = 32 * k + 8 * four, live = tile.rank - r;      // ranks of this lane's eight that there are
      half8v bs[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        bs[i] = *reinterpret_cast<const half8v*>(b[i] + min(r, p.rank - 8));
#pragma unroll
        for (int e = 0; e < 8; ++e) bs[i][e] = e < live ? bs[i][e] : (_Float16)0.0f;
      }
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        const half8v hi = *reinterpret_cast<const half8v*>(high + (16 * n + col) * pitch + r);
        const half8v lo = *reinterpret_cast<const half8v*>(low + (16 * n + col) * pitch + r);
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[n][i] = mfma(bs[i], hi, mfma(bs[i], lo, acc[n][i]));
      }
    }
    const int64_t m = m0 + 16 * four;
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      const int t = 16 * n + col;
      if (t >= tile.tokens || m >= p.m) continue;
      const int drop = tile.rank > 0 ? -(int)back[t] : 0;
      const Y* base = static_cast<const Y*>(p.base) + token[t] * p.base_stride + m;
      Y* y = static_cast<Y*>(p.y) + token[t] * p.y_stride + m;
      const int rows = (int)min(p.m - m, (int64_t)16);
      if (WIDE && rows == 16) {
        Y v[16];
#pragma unroll
        for (unsigned i = 0; i < sizeof(v) / 16; ++i) reinterpret_cast<u32x4*>(v)[i] = reinterpret_cast<const u32x4*>(base)[i];
#pragma unroll
        for (int e = 0; e < 16; ++e) v[e] = tile.rank > 0 ? (Y)((float)v[e] + ldexpf(acc[n][e / 4][e % 4], drop)) : v[e];
#pragma unroll
        for (unsigned i = 0; i < sizeof(v) / 16; ++i) reinterpret_cast<u32x4*>(y)[i] = reinterpret_cast<const u32x4*>(v)[i];
      } else {
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          if (e < rows) y[e] = tile.rank > 0 ? (Y)((float)base[e] + ldexpf(acc[n][e / 4][e % 4], drop)) : base[e];
        }
      }
    }
  }
}

template <int TILE>
const void* pick_up(bool f32, bool wide) {
  return f32 ? (wide ? reinterpret_cast<const void*>(lutgemm_adapt_up_kernel<TILE, float, true>) : reinterpret_cast<const void*>(lutgemm_adapt_up_kernel<TILE, float, false>))
             : (wide ? reinterpret_cast<const void*>(lutgemm_adapt_up_kernel<TILE, _Float16, true>) : reinterpret_cast<const void*>(lutgemm_adapt_up_kernel<TILE, _Float16, false>));
}
template <int TILE>
const void* pick_down(int rank, int* ranks) {
  *ranks = rank <= 16 ? 16 : (rank <= 32 ? 32 : 64);
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
    rc = launch(reinterpret_cast<const void*>(lutgemm_adapt_sort_kernel), dim3(1), kSortThreads, args, 4 * (size_t)((kSortWaves + 2) * (a.count + 1) + 1), hip_stream);
    if (rc != LUTGEMM_OK) return rc;
  }
  void* args[] = {&p};
  int ranks;
  const void* down = pick_down<16>(a.rank, &ranks);
  rc = launch(down, dim3(plan.parts, plan.tiles, (a.rank + ranks - 1) / ranks), kThreads, args, 0, hip_stream);
  if (rc != LUTGEMM_OK) return rc;
  const bool wide = (((uintptr_t)base | (uintptr_t)y | (uintptr_t)(base_stride * size) | (uintptr_t)(y_stride * size)) & 15) == 0;
  const int pitch = 32 * ((a.rank + 31) / 32) + 8;
  const size_t lds = (size_t)plan.tile * (4 * a.rank + 4 * pitch);
  const void* up = pick_up<16>(size == 4, wide);
  return launch(up, dim3((a.m + plan.rows - 1) / plan.rows, plan.tiles), kThreads, args, lds, hip_stream);
}
