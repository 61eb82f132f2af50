// Attention of a few new tokens over the key/value cache: include/lutgemm.h has the formula and the cache's layout.
//
// Mapping.  A workgroup owns a key head of a sequence, a row block (a row is a (token, query head) pair that shares the key
// head) and a split of the positions.  Its wavefronts take blocks of 32 positions in turn, each for all rows of the
// block, straight from memory into registers: a key or value that no two wavefronts want need not pass
// through LDS.  The products run transposed on the 16 x 16 x 32 matrix instructions:
//     S^T (positions x rows) = K (positions x channels) Q^T,     O^T (channels x rows) += V^T (channels x positions) P^T
// so that a lane owns one row (its column) and eight positions of it, the softmax needs no exchange
// between lanes but the maximum's, and its weights are the second product's operand as they stand: the cache's layout
// deals the positions to the lanes so that they are (place 8 a + 4 j + b is row 4 a + b of the j-th tile of S^T).
// The maximum that the weights are relative to is only raised where a score passes it by 2^8, which is seldom;
// the sum of the weights is one more product, of a tile of ones, so it adds what the other products add.
//
// At the end the wavefronts' sums meet in LDS, and where the positions are split the last workgroup to
// arrive adds the splits in order (the hand-off is the one of finish_row_range in lutgemm_device.hip: write-through stores,
// a wait for them, a barrier, a relaxed counter).  Results do not depend on who is last.
#include <hip/hip_fp16.h>
#include <hip/hip_runtime.h>

#include "lutgemm_kv.h"

#ifndef LUT_PART
#error "compiled once per part, -DLUT_PART=0 .. 14: bits (16, 8, 4) x head size (64, 96, 128, 192, 256)"
#endif

using namespace lutgemm_kv_detail;

namespace lutgemm_attention_parts {

struct Params {
  const _Float16* q;
  const uint64_t* mask;
  const char* pool;
  const int32_t* first;
  const int32_t* past;
  const int32_t* table;
  _Float16* y;
  float* partial;
  uint32_t* counters;
  int64_t q_stride, y_stride, pages;
  int tokens, most_tokens, table_pages, page_blocks, heads, shared;   // shared: query heads of a key head
  int block_bytes, splits, chunk, row_blocks, partial_rows;
  float scale;                                           // of the scores, times log2 e
};

typedef const void* (*Family)(int group_units, int row_tiles);
#define DECLARE(k) const void* family##k(int group_units, int row_tiles);
DECLARE(0) DECLARE(1) DECLARE(2) DECLARE(3) DECLARE(4) DECLARE(5) DECLARE(6) DECLARE(7)
DECLARE(8) DECLARE(9) DECLARE(10) DECLARE(11) DECLARE(12) DECLARE(13) DECLARE(14)
#undef DECLARE

}  // namespace lutgemm_attention_parts

namespace {

using lutgemm_attention_parts::Params;

typedef _Float16 half2v __attribute__((ext_vector_type(2)));
typedef _Float16 half4v __attribute__((ext_vector_type(4)));
typedef _Float16 half8v __attribute__((ext_vector_type(8)));
typedef float float2v __attribute__((ext_vector_type(2)));
typedef float float4v __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr int kWaves = 4;
constexpr float kSlack = 8.0f;    // how far, in powers of two, a score may pass the kept maximum: weights up to 2^8 in fp16

__device__ __forceinline__ void store_coherent(float* p, float v) { __hip_atomic_store(p, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
__device__ __forceinline__ float load_coherent(const float* p) { return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }

// The larger of a lane's value and those of the lanes 16, 32 and 48 away.
__device__ __forceinline__ float max_of_column(float v) {
  const uint32_t x = __builtin_bit_cast(uint32_t, v);
  const auto a = __builtin_amdgcn_permlane16_swap(x, x, false, false);
  const float m = fmaxf(__builtin_bit_cast(float, (uint32_t)a[0]), __builtin_bit_cast(float, (uint32_t)a[1]));
  const uint32_t y = __builtin_bit_cast(uint32_t, m);
  const auto b = __builtin_amdgcn_permlane32_swap(y, y, false, false);
  return fmaxf(__builtin_bit_cast(float, (uint32_t)b[0]), __builtin_bit_cast(float, (uint32_t)b[1]));
}

// (By value: a bit cast of a vector's element in place takes the vector's first.)
__device__ __forceinline__ uint32_t bits_of(_Float16 v) { return __builtin_bit_cast(uint16_t, v); }

__device__ __forceinline__ half2v both(_Float16 v) { return (half2v){v, v}; }

// Code words to fp16.  8 bits: the byte becomes the low mantissa bits of 1024 (0x6400), less 1152 = 1024 + 128.
__device__ __forceinline__ half2v bytes_to_half(uint32_t w, uint32_t selector) {
  return __builtin_bit_cast(half2v, __builtin_amdgcn_perm(0x64646464u, w, selector)) - both((_Float16)1152.0f);
}
// 4 bits: nibbles 0 and 4 (low), or 1 and 5 of a word, likewise; the latter count 16ths of 1024 + 16 u.
__device__ __forceinline__ half2v low_nibbles(uint32_t w) {
  return __builtin_bit_cast(half2v, (w & 0x000f000fu) | 0x64006400u) - both((_Float16)1024.0f);
}
__device__ __forceinline__ half2v high_nibbles(uint32_t w) {
  return __builtin_elementwise_fma(__builtin_bit_cast(half2v, (w & 0x00f000f0u) | 0x64006400u), both((_Float16)0.0625f), both((_Float16)-64.0f));
}

// The raw words of a unit (32 places x 32 channels) as a lane holds them: two runs of eight values.
template <int BITS>
struct Unit {
  uint32_t w[BITS];            // 16, 8 or 4 words
};
template <int BITS>
__device__ __forceinline__ void load_unit(Unit<BITS>& u, const char* codes, int c, int lane) {
  if constexpr (BITS == 16) {
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const u32x4 v = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(codes + (c * 2 + j) * 1024) + lane);
#pragma unroll
      for (int i = 0; i < 4; ++i) u.w[4 * j + i] = v[i];
    }
  } else if constexpr (BITS == 8) {
    const u32x4 v = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(codes + c * 1024) + lane);
#pragma unroll
    for (int i = 0; i < 4; ++i) u.w[i] = v[i];
  } else {
    const u32x2 v = __builtin_nontemporal_load(reinterpret_cast<const u32x2*>(codes + c * 512) + lane);
    u.w[0] = v[0];
    u.w[1] = v[1];
  }
}

__device__ __forceinline__ half8v join(half2v a, half2v b, half2v c, half2v d) {
  return __builtin_shufflevector(__builtin_shufflevector(a, b, 0, 1, 2, 3), __builtin_shufflevector(c, d, 0, 1, 2, 3), 0, 1, 2, 3, 4, 5, 6, 7);
}

// Key unit, run j: the lane's place of tile j, eight channels.  s, z: that place's scale and offset.
template <int BITS>
__device__ __forceinline__ half8v key_values(const Unit<BITS>& u, int j, _Float16 s, _Float16 z) {
  if constexpr (BITS == 16) {
    const u32x4 w = {u.w[4 * j], u.w[4 * j + 1], u.w[4 * j + 2], u.w[4 * j + 3]};
    return __builtin_bit_cast(half8v, w);
  } else if constexpr (BITS == 8) {
    half2v h[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) h[i] = bytes_to_half(u.w[2 * j + (i >> 1)], i & 1 ? 0x04030402u : 0x04010400u) * both(s);
    return join(h[0], h[1], h[2], h[3]);
  } else {
    const uint32_t w = u.w[j];
    half2v h[4] = {low_nibbles(w), high_nibbles(w), low_nibbles(w >> 8), high_nibbles(w >> 8)};
#pragma unroll
    for (int i = 0; i < 4; ++i) h[i] = __builtin_elementwise_fma(h[i], both(s), both(z));
    return join(h[0], h[1], h[2], h[3]);
  }
}
// Value unit, run j: channel 16 j + lane % 16, eight places.  s, z: those places' scales and offsets.
template <int BITS>
__device__ __forceinline__ half8v value_values(const Unit<BITS>& u, int j, const half8v s, const half8v z) {
  if constexpr (BITS == 16) {
    const u32x4 w = {u.w[4 * j], u.w[4 * j + 1], u.w[4 * j + 2], u.w[4 * j + 3]};
    return __builtin_bit_cast(half8v, w);
  } else if constexpr (BITS == 8) {
    half2v h[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) h[i] = bytes_to_half(u.w[2 * j + (i >> 1)], i & 1 ? 0x04030402u : 0x04010400u);
    return join(h[0], h[1], h[2], h[3]) * s;
  } else {
    half2v h[4];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      h[2 * i] = j ? high_nibbles(u.w[i]) : low_nibbles(u.w[i]);
      h[2 * i + 1] = j ? high_nibbles(u.w[i] >> 8) : low_nibbles(u.w[i] >> 8);
    }
    return __builtin_elementwise_fma(join(h[0], h[1], h[2], h[3]), s, z);
  }
}

// Codes and scales of a block's keys or values on their way: DC units, and DC / GU groups' scales.
template <int BITS, int DC, int GU>
struct KeyWords {
  Unit<BITS> unit[DC];
  uint32_t scale[BITS == 16 ? 1 : (DC / GU) * (BITS == 8 ? 1 : 2)];
};
template <int BITS, int DC, int GU>
struct ValueWords {
  Unit<BITS> unit[DC];
  half8v scale[BITS == 16 ? 1 : DC / GU];
  half8v offset[BITS == 4 ? DC / GU : 1];
};

template <int BITS, int DC, int GU>
__device__ __forceinline__ void load_keys(KeyWords<BITS, DC, GU>& k, const char* block, int lane) {
#pragma unroll
  for (int c = 0; c < DC; ++c) load_unit<BITS>(k.unit[c], block, c, lane);
  if constexpr (BITS != 16) {
    const char* scales = block + kBlock * DC * 32 * BITS / 8;
#pragma unroll
    for (int g = 0; g < DC / GU; ++g) {
      if constexpr (BITS == 8) {
        k.scale[g] = reinterpret_cast<const uint32_t*>(scales + g * 64)[lane & 15];
      } else {
        const u32x2 v = reinterpret_cast<const u32x2*>(scales + g * 128)[lane & 15];
        k.scale[2 * g] = v[0];
        k.scale[2 * g + 1] = v[1];
      }
    }
  }
}
template <int BITS, int DC, int GU>
__device__ __forceinline__ void load_values(ValueWords<BITS, DC, GU>& v, const char* block, int lane) {
#pragma unroll
  for (int c = 0; c < DC; ++c) load_unit<BITS>(v.unit[c], block, c, lane);
  if constexpr (BITS != 16) {
    const char* scales = block + kBlock * DC * 32 * BITS / 8;
#pragma unroll
    for (int g = 0; g < DC / GU; ++g) {
      v.scale[g] = reinterpret_cast<const half8v*>(scales + g * (BITS == 8 ? 64 : 128))[lane >> 4];
      if constexpr (BITS == 4) v.offset[g] = reinterpret_cast<const half8v*>(scales + g * 128 + 64)[lane >> 4];
    }
  }
}
template <int BITS, int DC, int GU>
__device__ __forceinline__ half8v key_operand(const KeyWords<BITS, DC, GU>& k, int c, int j) {
  if constexpr (BITS == 16) return key_values<16>(k.unit[c], j, (_Float16)0, (_Float16)0);
  if constexpr (BITS == 8) return key_values<8>(k.unit[c], j, __builtin_bit_cast(half2v, k.scale[c / GU])[j], (_Float16)0);
  if constexpr (BITS == 4) {
    const half2v sz = __builtin_bit_cast(half2v, k.scale[2 * (c / GU) + j]);
    return key_values<4>(k.unit[c], j, sz[0], sz[1]);
  }
}
template <int BITS, int DC, int GU>
__device__ __forceinline__ half8v value_operand(const ValueWords<BITS, DC, GU>& v, int c, int j) {
  return value_values<BITS>(v.unit[c], j, v.scale[BITS == 16 ? 0 : c / GU], v.offset[BITS == 4 ? c / GU : 0]);
}

__device__ __forceinline__ float4v mfma(half8v a, half8v b, float4v c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }

// A walk over every kWaves-th block of a split: which page a block is in, without a division a block.  The table's entries are
// fetched 64 at a time, one a lane.
struct Walk {
  const int32_t* table;        // of the sequence
  int64_t pages;
  int table_pages, page_blocks;
  int col, in_page;            // page of the sequence, block in it
  int col_step, block_step;
  int base;                    // first table entry held
  int held;                    // this lane's
};
__device__ __forceinline__ void walk_fetch(Walk& w, int lane) {
  w.base = w.col;
  w.held = w.col + lane < w.table_pages ? w.table[w.col + lane] : -1;
}
__device__ __forceinline__ void walk_begin(Walk& w, int block, int lane) {
  w.col = block / w.page_blocks;
  w.in_page = block - w.col * w.page_blocks;
  w.col_step = kWaves / w.page_blocks;
  w.block_step = kWaves - w.col_step * w.page_blocks;
  walk_fetch(w, lane);
}
__device__ __forceinline__ void walk_on(Walk& w, int lane) {
  w.col += w.col_step;
  w.in_page += w.block_step;
  if (w.in_page >= w.page_blocks) {
    w.in_page -= w.page_blocks;
    ++w.col;
  }
  if (w.col - w.base >= 64) walk_fetch(w, lane);
}
// Number of the page (-1: none).
__device__ __forceinline__ int walk_page(const Walk& w) {
  const int page = __builtin_amdgcn_readlane(w.held, w.col - w.base);
  return page >= 0 && page < w.pages ? page : -1;
}

// One workgroup: a split (blockIdx.x), a key head and row block (blockIdx.y), a sequence (blockIdx.z).
// BITS of a code, DC units of 32 channels to a head, GU of them to a scale, RT tiles of 16 rows.
template <int BITS, int DC, int GU, int RT>
__global__ __launch_bounds__(kWaves * 64) void lutgemm_attention_kernel(Params p) {
  constexpr int kTiles = 2 * DC;            // of 16 channels
  constexpr int kRows = 16 * RT;
  // The wavefronts' sums meet kMeet units of channels at a time.
  constexpr int kMeet = RT == 1 ? DC : (RT == 2 ? (DC % 2 == 0 ? 2 : 1) : 1);
  __shared__ float sums[kWaves][kRows][kMeet * 32 + 4];
  __shared__ float tops[kWaves][kRows], totals[kWaves][kRows];
  __shared__ uint32_t last;

  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int column = lane & 15, quarter = lane >> 4;
  const int seq = blockIdx.z, head = blockIdx.y / p.row_blocks, row_block = blockIdx.y - head * p.row_blocks;

  // What the step says of the sequence, within what the host said.
  const int row_first = max(p.first[seq], 0);
  const int count = min(min(p.first[seq + 1], p.tokens) - row_first, p.most_tokens);   // (at most kMostTokens)
  const int rows = count * p.shared;         // of the key head
  const int row0 = row_block * kRows;
  if (count <= 0 || row0 >= rows) return;
  const int past = max(p.past[seq], 0);
  const int64_t capacity = (int64_t)p.table_pages * p.page_blocks * kBlock;
  const int64_t length = min((int64_t)past + count, capacity);
  int64_t chunk = p.chunk;
  if (chunk * p.splits < length) chunk = ((length + p.splits - 1) / p.splits + kBlock - 1) / kBlock * kBlock;
  const int active = max(1, (int)((length + chunk - 1) / chunk));
  if ((int)blockIdx.x >= active) return;
  const int first_block = (int)(blockIdx.x * chunk / kBlock);
  const int end_block = (int)((min((blockIdx.x + 1) * chunk, length) + kBlock - 1) / kBlock);

  // Queries: lane holds row `column` of a tile, channels 32 c + 8 quarter + (0..7).
  half8v query[RT][DC];
  uint32_t mask_low[RT], mask_high[RT];
#pragma unroll
  for (int t = 0; t < RT; ++t) {
    const int row = row0 + 16 * t + column;
    const bool live = row < rows;
    const int token = live ? row / p.shared : 0;
    const _Float16* q = p.q + (int64_t)(row_first + token) * p.q_stride + ((int64_t)head * p.shared + (live ? row - token * p.shared : 0)) * (DC * 32);
#pragma unroll
    for (int c = 0; c < DC; ++c) {
      const half8v none = {0, 0, 0, 0, 0, 0, 0, 0};
      query[t][c] = live ? *reinterpret_cast<const half8v*>(q + 32 * c + 8 * quarter) : none;
    }
    const uint64_t sees = !live ? 0 : (p.mask ? p.mask[row_first + token] : ~0ull >> (63 - token));
    mask_low[t] = (uint32_t)sees;
    mask_high[t] = (uint32_t)(sees >> 32);
  }

  float4v out[RT][kTiles], total[RT];
  float top[RT];
#pragma unroll
  for (int t = 0; t < RT; ++t) {
    top[t] = -__builtin_inff();
    total[t] = (float4v){0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int u = 0; u < kTiles; ++u) out[t][u] = (float4v){0.0f, 0.0f, 0.0f, 0.0f};
  }
  const half2v one = both((_Float16)1.0f);
  const half8v ones = join(one, one, one, one);

  int block = first_block + wave;
  if (block < end_block) {
    Walk walk;
    walk.table = p.table + (int64_t)seq * p.table_pages;
    walk.pages = p.pages;
    walk.table_pages = p.table_pages;
    walk.page_blocks = p.page_blocks;
    walk_begin(walk, block, lane);
    const int64_t page_bytes = (int64_t)p.heads * p.page_blocks * p.block_bytes;
    const char* head_base = p.pool + (int64_t)head * p.page_blocks * p.block_bytes;
    const int value_offset = p.block_bytes / 2;

    int page = walk_page(walk);
    const char* at = head_base + max(page, 0) * page_bytes + (int64_t)walk.in_page * p.block_bytes;
    KeyWords<BITS, DC, GU> keys;
    ValueWords<BITS, DC, GU> values;
    load_keys<BITS, DC, GU>(keys, at, lane);
    load_values<BITS, DC, GU>(values, at + value_offset, lane);

    while (true) {
      // ---- scores
      float4v score[RT][2];
#pragma unroll
      for (int t = 0; t < RT; ++t) score[t][0] = score[t][1] = (float4v){0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int c = 0; c < DC; ++c) {
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const half8v k = key_operand<BITS, DC, GU>(keys, c, j);
#pragma unroll
          for (int t = 0; t < RT; ++t) score[t][j] = mfma(k, query[t][c], score[t][j]);
        }
      }
      const int next = block + kWaves;
      const bool more = next < end_block;
      const bool dead = page < 0;
      const char* following = at;
      if (more) {
        walk_on(walk, lane);
        page = walk_page(walk);
        following = head_base + max(page, 0) * page_bytes + (int64_t)walk.in_page * p.block_bytes;
        load_keys<BITS, DC, GU>(keys, following, lane);
      }

      // ---- weights.  A lane has positions 32 block + 8 quarter + 4 j + i of its rows.
      const bool whole = (int64_t)(block + 1) * kBlock <= past && !dead;       // every row sees all of the block
      half8v weight[RT];
      uint32_t visible[RT];                    // bit 4 j + i
      const int place = block * kBlock + 8 * quarter - past;     // of the lane's first position, counted from the new ones
      const int limit = dead ? -(1 << 30) : (int)(length - past);   // positions from here on do not exist
#pragma unroll
      for (int t = 0; t < RT; ++t) {
        float s[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) s[i] = score[t][i >> 2][i & 3] * p.scale;
        visible[t] = 0xffu;
        if (!whole) {
          visible[t] = 0u;
          const uint64_t sees = (uint64_t)mask_high[t] << 32 | mask_low[t];
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const int n = place + i;
            const bool v = n < limit && (n < 0 || ((sees >> (n & 63)) & 1u) != 0);
            visible[t] |= v ? 1u << i : 0u;
          }
        }
        float most = -__builtin_inff();
#pragma unroll
        for (int i = 0; i < 8; ++i) most = fmaxf(most, whole || (visible[t] >> i & 1u) ? s[i] : -__builtin_inff());
        if (__any(most > top[t] + kSlack)) {
          most = max_of_column(most);
          const float raised = most > top[t] + kSlack ? most : top[t];     // (a row's own need: others do not change its result)
          const float shrink = raised == top[t] ? 1.0f : __builtin_amdgcn_exp2f(top[t] - raised);
          top[t] = raised;
          total[t] *= shrink;
#pragma unroll
          for (int u = 0; u < kTiles; ++u) out[t][u] *= shrink;
        }
        half2v w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          float2v e = {__builtin_amdgcn_exp2f(s[2 * i] - top[t]), __builtin_amdgcn_exp2f(s[2 * i + 1] - top[t])};
          if (!whole) {
            e[0] = visible[t] >> (2 * i) & 1u ? e[0] : 0.0f;
            e[1] = visible[t] >> (2 * i + 1) & 1u ? e[1] : 0.0f;
          }
          w[i] = __builtin_convertvector(e, half2v);
        }
        weight[t] = join(w[0], w[1], w[2], w[3]);
        total[t] = mfma(ones, weight[t], total[t]);
      }

      // ---- weighted values
#pragma unroll
      for (int c = 0; c < DC; ++c) {
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          half8v v = value_operand<BITS, DC, GU>(values, c, j);
          if (!whole) {
            // A weight of zero must not meet an infinity or a NaN: what is not finite is taken out of the operand, and
            // counted for the rows that see it: +inf as 1, -inf as 64, NaN as 4096 (there are at most 32 of each).
            half8v odd = {0, 0, 0, 0, 0, 0, 0, 0};
            bool any = false;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
              const uint32_t bits = bits_of(v[i]);
              const bool exists = place + i < limit, infinite = (bits & 0x7c00u) == 0x7c00u;
              if (infinite && exists) odd[i] = (_Float16)((bits & 0x3ffu) ? 4096.0f : (bits & 0x8000u ? 64.0f : 1.0f));
              any |= infinite && exists;
              if (infinite || !exists) v[i] = (_Float16)0;
            }
            if (__any(any)) {
#pragma unroll
              for (int t = 0; t < RT; ++t) {
                half8v seen;
#pragma unroll
                for (int i = 0; i < 8; ++i) seen[i] = visible[t] >> i & 1u ? (_Float16)1.0f : (_Float16)0;
                const float4v n = mfma(odd, seen, (float4v){0.0f, 0.0f, 0.0f, 0.0f});
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                  const int found = (int)n[i];
                  const bool plus = (found & 63) != 0, minus = (found >> 6 & 63) != 0, nan = found >= 4096 || (plus && minus);
                  out[t][2 * c + j][i] += nan ? __builtin_nanf("") : (plus ? __builtin_inff() : (minus ? -__builtin_inff() : 0.0f));
                }
              }
            }
          }
#pragma unroll
          for (int t = 0; t < RT; ++t) out[t][2 * c + j] = mfma(v, weight[t], out[t][2 * c + j]);
        }
      }
      if (!more) break;
      block = next;
      at = following;
      load_values<BITS, DC, GU>(values, at + value_offset, lane);
    }
  }

  // ---- the wavefronts' sums meet.  out[t][u][i]: row 16 t + column, channel 16 u + 4 quarter + i.
  if (quarter == 0) {
#pragma unroll
    for (int t = 0; t < RT; ++t) {
      tops[wave][16 * t + column] = top[t];
      totals[wave][16 * t + column] = total[t][0];
    }
  }
  __syncthreads();
  const int live_rows = min(rows - row0, kRows);
  float factor[RT];                            // of this wavefront's sums
#pragma unroll
  for (int t = 0; t < RT; ++t) {
    float raised = -__builtin_inff();
#pragma unroll
    for (int w = 0; w < kWaves; ++w) raised = fmaxf(raised, tops[w][16 * t + column]);
    factor[t] = top[t] == -__builtin_inff() ? 0.0f : __builtin_amdgcn_exp2f(top[t] - raised);
    if (factor[t] == 0.0f && !(total[t][0] == total[t][0])) factor[t] = total[t][0];     // a NaN stays one
  }
  const int unit = (seq * p.heads + head) * p.row_blocks + row_block;
  float* partial = p.partial + ((int64_t)unit * p.splits + blockIdx.x) * p.partial_rows * (DC * 32 + 2);
#pragma unroll
  for (int m = 0; m < DC / kMeet; ++m) {
    if (m > 0) __syncthreads();
#pragma unroll
    for (int t = 0; t < RT; ++t)
#pragma unroll
      for (int u = 0; u < 2 * kMeet; ++u) {
        const float4v o = out[t][2 * kMeet * m + u] * factor[t];
        *reinterpret_cast<float4v*>(&sums[wave][16 * t + column][16 * u + 4 * quarter]) = o;
      }
    __syncthreads();
    // a thread takes two channels
    constexpr int kPairs = kMeet * 16;
    for (int i = threadIdx.x; i < live_rows * kPairs; i += kWaves * 64) {
      const int row = i / kPairs, d = i % kPairs * 2;
      float a = 0.0f, b = 0.0f;
#pragma unroll
      for (int w = 0; w < kWaves; ++w) {
        a += sums[w][row][d];
        b += sums[w][row][d + 1];
      }
      if (active > 1) {
        store_coherent(partial + row * (DC * 32) + m * kMeet * 32 + d, a);
        store_coherent(partial + row * (DC * 32) + m * kMeet * 32 + d + 1, b);
      } else {
        float raised = -__builtin_inff(), sum = 0.0f;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) raised = fmaxf(raised, tops[w][row]);
#pragma unroll
        for (int w = 0; w < kWaves; ++w) sum += tops[w][row] == -__builtin_inff() ? totals[w][row] : __builtin_amdgcn_exp2f(tops[w][row] - raised) * totals[w][row];
        const int r = row0 + row, token = r / p.shared;
        const float inverse = sum == 0.0f ? 0.0f : 1.0f / sum;
        const half2v y = __builtin_convertvector((float2v){a * inverse, b * inverse}, half2v);
        *reinterpret_cast<half2v*>(p.y + (int64_t)(row_first + token) * p.y_stride + ((int64_t)head * p.shared + r - token * p.shared) * (DC * 32) +
                                   m * kMeet * 32 + d) = y;
      }
    }
  }
  if (active == 1) return;

  // ---- the splits' sums meet: the last workgroup to arrive adds them in order
  float* ends = partial + p.partial_rows * (DC * 32);
  for (int row = threadIdx.x; row < live_rows; row += kWaves * 64) {
    float raised = -__builtin_inff(), sum = 0.0f;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) raised = fmaxf(raised, tops[w][row]);
#pragma unroll
    for (int w = 0; w < kWaves; ++w) sum += tops[w][row] == -__builtin_inff() ? totals[w][row] : __builtin_amdgcn_exp2f(tops[w][row] - raised) * totals[w][row];
    store_coherent(ends + 2 * row, raised);
    store_coherent(ends + 2 * row + 1, sum);
  }
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  __syncthreads();
  if (threadIdx.x == 0) last = __hip_atomic_fetch_add(p.counters + unit, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == (uint32_t)(active - 1) ? 1u : 0u;
  __syncthreads();
  if (last == 0u) return;
  const float* all = p.partial + (int64_t)unit * p.splits * p.partial_rows * (DC * 32 + 2);
  const int64_t stride = (int64_t)p.partial_rows * (DC * 32 + 2);
  for (int i = threadIdx.x; i < live_rows * DC * 16; i += kWaves * 64) {
    const int row = i / (DC * 16), d = i % (DC * 16) * 2;
    float raised = -__builtin_inff();
    for (int s = 0; s < active; ++s) raised = fmaxf(raised, load_coherent(all + s * stride + p.partial_rows * (DC * 32) + 2 * row));
    float a = 0.0f, b = 0.0f, sum = 0.0f;
    for (int s = 0; s < active; ++s) {
      const float* one_split = all + s * stride;
      const float t = load_coherent(one_split + p.partial_rows * (DC * 32) + 2 * row);
      const float n = load_coherent(one_split + p.partial_rows * (DC * 32) + 2 * row + 1);
      const float f = t == -__builtin_inff() ? (n == n ? 0.0f : n) : __builtin_amdgcn_exp2f(t - raised);
      a += f * load_coherent(one_split + row * (DC * 32) + d);
      b += f * load_coherent(one_split + row * (DC * 32) + d + 1);
      sum += f * n;
    }
    const int r = row0 + row, token = r / p.shared;
    const float inverse = sum == 0.0f ? 0.0f : 1.0f / sum;
    const half2v y = __builtin_convertvector((float2v){a * inverse, b * inverse}, half2v);
    *reinterpret_cast<half2v*>(p.y + (int64_t)(row_first + token) * p.y_stride + ((int64_t)head * p.shared + r - token * p.shared) * (DC * 32) + d) = y;
  }
  if (threadIdx.x == 0) __hip_atomic_store(p.counters + unit, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

template <int BITS, int DC, int GU>
const void* pick_tiles(int row_tiles) {
  if (row_tiles == 1) return reinterpret_cast<const void*>(lutgemm_attention_kernel<BITS, DC, GU, 1>);
  if (row_tiles == 2) return reinterpret_cast<const void*>(lutgemm_attention_kernel<BITS, DC, GU, 2>);
  if constexpr (DC <= 4) {
    if (row_tiles == 4) return reinterpret_cast<const void*>(lutgemm_attention_kernel<BITS, DC, GU, 4>);
  }
  return nullptr;
}
template <int BITS, int DC>
const void* pick_group(int units, int row_tiles) {
  if (BITS == 16 || units == DC) return pick_tiles<BITS, DC, DC>(row_tiles);
  if constexpr (BITS != 16) {
    if (units == 1) return pick_tiles<BITS, DC, 1>(row_tiles);
    if constexpr (DC % 2 == 0 && DC > 2) {
      if (units == 2) return pick_tiles<BITS, DC, 2>(row_tiles);
    }
    if constexpr (DC == 6) {
      if (units == 3) return pick_tiles<BITS, DC, 3>(row_tiles);
    }
    if constexpr (DC == 8) {
      if (units == 4) return pick_tiles<BITS, DC, 4>(row_tiles);
    }
  }
  return nullptr;
}

}  // namespace

namespace lutgemm_attention_parts {
#define NAME2(k) family##k
#define NAME(k) NAME2(k)
const void* NAME(LUT_PART)(int group_units, int row_tiles) {
  constexpr int kBits = LUT_PART / 5 == 0 ? 16 : (LUT_PART / 5 == 1 ? 8 : 4);
  constexpr int kUnits = LUT_PART % 5 == 0 ? 2 : (LUT_PART % 5 == 1 ? 3 : (LUT_PART % 5 == 2 ? 4 : (LUT_PART % 5 == 3 ? 6 : 8)));
  return pick_group<kBits, kUnits>(group_units, row_tiles);
}
}  // namespace lutgemm_attention_parts

#if LUT_PART == 0
extern "C" int lutgemm_attention(const void* q, const uint64_t* mask, const lutgemm_kv_cache* cache, const lutgemm_kv_step* step, void* y,
                                 int q_heads, int64_t q_stride, int64_t y_stride, float scale, int64_t most_positions, void* workspace,
                                 size_t workspace_bytes, void* hip_stream) {
  using namespace lutgemm_attention_parts;
  int rc = check_cache(cache);
  if (rc == LUTGEMM_OK) rc = check_step(step);
  if (rc != LUTGEMM_OK) return rc;
  if (!q || !y || !workspace || q_heads < 1 || q_heads % cache->heads != 0 || most_positions < 0) return LUTGEMM_EINVAL;
  if ((((uintptr_t)q | (uintptr_t)y | (uintptr_t)workspace) & 15) != 0 || ((uintptr_t)mask & 7) != 0) return LUTGEMM_EINVAL;
  const int64_t row = (int64_t)q_heads * cache->head_dim;
  if (q_stride < row || y_stride < row || q_stride % 8 != 0 || y_stride % 8 != 0) return LUTGEMM_EINVAL;
  if (step->most_tokens > kMostTokens || q_heads > 1 << 14) return LUTGEMM_EUNSUPPORTED;
  const int64_t held = (int64_t)step->table_pages * cache->page_tokens;
  if (held > (int64_t)1 << 30) return LUTGEMM_EUNSUPPORTED;
  if (most_positions == 0 || most_positions > held) most_positions = held;
  const int group = group_of(cache->head_dim, cache->bits, cache->group);
  const AttentionPlan plan = plan_attention(cache->heads, cache->head_dim, cache->bits, q_heads, step->seqs, step->most_tokens, most_positions);
  if (workspace_bytes < 32768 + 4 * (size_t)attention_partial_floats(plan, cache->heads, cache->head_dim, q_heads, step->seqs, step->most_tokens))
    return LUTGEMM_EWORKSPACE;
  if (step->tokens == 0 || step->most_tokens == 0) return LUTGEMM_OK;
  if ((int64_t)cache->heads * plan.row_blocks > 65535) return LUTGEMM_EUNSUPPORTED;
  Params p = {};
  p.q = static_cast<const _Float16*>(q);
  p.mask = mask;
  p.pool = static_cast<const char*>(cache->pool);
  p.first = step->first;
  p.past = step->past;
  p.table = step->table;
  p.y = static_cast<_Float16*>(y);
  p.partial = reinterpret_cast<float*>(static_cast<char*>(workspace) + 32768);
  p.counters = static_cast<uint32_t*>(workspace);
  p.q_stride = q_stride;
  p.y_stride = y_stride;
  p.pages = cache->pages;
  p.tokens = step->tokens;
  p.most_tokens = step->most_tokens;
  p.table_pages = step->table_pages;
  p.page_blocks = cache->page_tokens / kBlock;
  p.heads = cache->heads;
  p.shared = q_heads / cache->heads;
  p.block_bytes = block_bytes(cache->head_dim, cache->bits, group);
  p.splits = plan.splits;
  p.chunk = plan.chunk;
  p.row_blocks = plan.row_blocks;
  const int most_rows = step->most_tokens * p.shared;
  p.partial_rows = most_rows < 16 * plan.row_tiles ? most_rows : 16 * plan.row_tiles;
  p.scale = scale * 1.44269504088896340736f;
  static const Family families[15] = {family0, family1, family2, family3, family4, family5, family6, family7,
                                      family8, family9, family10, family11, family12, family13, family14};
  const int bits = cache->bits == 16 ? 0 : (cache->bits == 8 ? 1 : 2), d = cache->head_dim;
  const int size = d == 64 ? 0 : (d == 96 ? 1 : (d == 128 ? 2 : (d == 192 ? 3 : 4)));
  const void* kern = families[bits * 5 + size](group / 32, plan.row_tiles);
  if (!kern) return LUTGEMM_EUNSUPPORTED;
  void* args[] = {&p};
  if (hipLaunchKernel(kern, dim3(plan.splits, cache->heads * plan.row_blocks, step->seqs), dim3(kWaves * 64), args, 0,
                      static_cast<hipStream_t>(hip_stream)) != hipSuccess)
    return LUTGEMM_EHIP;
  return LUTGEMM_OK;
}
#endif
