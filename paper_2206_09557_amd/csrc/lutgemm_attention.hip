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
// What the weights are relative to is only raised where a score passes it by 2^15, which is seldom;
// the sum of the weights is one more product, of a tile of ones, so it adds what the other products add.  Weights are fp16 there, because the
// values are and matrix instructions take operands of one type; twice as many of them (a weight in two parts) would be what more bits cost.
// The rounding is 0.25 to 0.3 x 10^-3 of a result's norm together with the result's own, which alone is 0.21 x 10^-3.
//
// At the end the wavefronts' sums meet in LDS, and where the positions are split the splits' sums meet in memory: of up to 16 rows the
// last workgroup to arrive adds them (the hand-off is the one of finish_row_range in lutgemm_device.hip: write-through
// stores, a wait for them, a barrier, a relaxed counter), of more rows a second small kernel.  Both
// add in an order that the numbers of rows and splits decide (every 2nd, 4th, ... split by itself, then those sums), not the one in which
// workgroups arrive.  131072 positions of one sequence in 32 splits: meeting in LDS, handing off and adding take 8 us of 40.
#include <hip/hip_fp16.h>
#include <hip/hip_runtime.h>

#include <type_traits>

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
  float inverse_shared;
  float scale;                                           // of the scores, times log2 e; not negative ...
  uint32_t flip;                                         // ... the queries' signs are
};

typedef const void* (*Family)(int group_units, int row_tiles, int waves);
#define DECLARE(k) const void* family##k(int group_units, int row_tiles, int waves);
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

constexpr int kJoinThreads = 256, kJoinAhead = 4;      // splits that a thread asks for at once
// Weights are fp16 where they meet the values, from 2^-14 (2^-25, with fewer bits) to 2^15.  What they are relative to is put kLift below a
// score that raises it, and raised again where a score passes it by kSlack, all in powers of two: the row's largest is worth 2^7 to 2^15, and a
// weight is off by 2^-32 of it at most where it is not by 2^-11 of itself.  (Relative to the score itself a weight would vanish at 2^-25 of the
// largest, and some ten thousand of those together are 2^-11 of a result.)
constexpr float kLift = 7.0f, kSlack = 15.0f;
constexpr float kNothing = -3.402823466e38f;      // what weights are relative to before a row has seen a score: finite, so that one of -inf weighs nothing
// Scores that fp32 holds without fractions.  The weights' multiply-add brings back what rounding took off a maximum like that: from 2^28 on more
// than fp16's exponents hold.  So where a row has one the tile's are rounded before the maximum, which is rounded too, is taken off.
constexpr float kFar = 16777216.0f;

// Partial results that cross workgroups inside one kernel: stores that are written through to the device's point of coherence and loads
// that are served from it (what a relaxed atomic of device scope is, but of 16 or 8 bytes).
constexpr int kDeviceScope = 16;     // sc1
typedef __amdgpu_buffer_rsrc_t Buffer;
__device__ __forceinline__ Buffer buffer_of(float* p, int64_t floats) {
  return __builtin_amdgcn_make_buffer_rsrc(p, 0, (int)(floats * 4), 0x00027000);
}
__device__ __forceinline__ void store4(Buffer b, int at, float4v v) {
  __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, v), b, at * 4, 0, kDeviceScope);
}
__device__ __forceinline__ void store2(Buffer b, int at, float2v v) {
  __builtin_amdgcn_raw_buffer_store_b64(__builtin_bit_cast(u32x2, v), b, at * 4, 0, kDeviceScope);
}
__device__ __forceinline__ float4v load4(Buffer b, int at) {
  return __builtin_bit_cast(float4v, __builtin_amdgcn_raw_buffer_load_b128(b, at * 4, 0, kDeviceScope));
}
__device__ __forceinline__ float2v load2(Buffer b, int at) {
  return __builtin_bit_cast(float2v, __builtin_amdgcn_raw_buffer_load_b64(b, at * 4, 0, kDeviceScope));
}

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
// (One and_or each: the instruction takes no literal, so the constants are made to live in registers.)
__device__ __forceinline__ uint32_t nibbles(uint32_t w, uint32_t mask) {
  uint32_t exponent = 0x64006400u;
  asm("" : "+s"(mask));
  asm("" : "+v"(exponent));
  return (w & mask) | exponent;
}
__device__ __forceinline__ half2v low_nibbles(uint32_t w) { return __builtin_bit_cast(half2v, nibbles(w, 0x000f000fu)) - both((_Float16)1024.0f); }
__device__ __forceinline__ half2v high_nibbles(uint32_t w) {
  return __builtin_elementwise_fma(__builtin_bit_cast(half2v, nibbles(w, 0x00f000f0u)), both((_Float16)0.0625f), both((_Float16)-64.0f));
}

// The raw words of a unit (32 places x 32 channels) as a lane holds them: two runs of eight values.
template <int BITS>
struct Unit {
  uint32_t w[BITS];            // 16, 8 or 4 words
};
// The cache's memory, by its address space: the compiler must not take it for memory that may be LDS, whose loads it can only wait for
// all together.
typedef const __attribute__((address_space(1))) char* Memory;
template <typename T>
__device__ __forceinline__ T load_at(Memory p, int i) {
  return reinterpret_cast<const __attribute__((address_space(1))) T*>(p)[i];
}
template <typename T>
__device__ __forceinline__ T load_past(Memory p, int i) {          // codes are read once
  return __builtin_nontemporal_load(reinterpret_cast<const __attribute__((address_space(1))) T*>(p) + i);
}

template <int BITS>
__device__ __forceinline__ void load_unit(Unit<BITS>& u, Memory codes, int c, int lane) {
  if constexpr (BITS == 16) {
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const u32x4 v = load_past<u32x4>(codes + (c * 2 + j) * 1024, lane);
#pragma unroll
      for (int i = 0; i < 4; ++i) u.w[4 * j + i] = v[i];
    }
  } else if constexpr (BITS == 8) {
    const u32x4 v = load_past<u32x4>(codes + c * 1024, lane);
#pragma unroll
    for (int i = 0; i < 4; ++i) u.w[i] = v[i];
  } else {
    const u32x2 v = load_past<u32x2>(codes + c * 512, lane);
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

__device__ __forceinline__ _Float16 half_of(uint32_t word, int which) { return __builtin_bit_cast(_Float16, (uint16_t)(which ? word >> 16 : word)); }

template <int I>
__device__ __forceinline__ uint32_t word_of(u32x4 v) { return v[I]; }
__device__ __forceinline__ uint32_t one_of(uint32_t a, uint32_t b, uint32_t second) { return (a & ~second) | (b & second); }   // second: a mask

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
__device__ __forceinline__ void load_keys(KeyWords<BITS, DC, GU>& k, Memory block, int lane) {
#pragma unroll
  for (int c = 0; c < DC; ++c) load_unit<BITS>(k.unit[c], block, c, lane);
  if constexpr (BITS != 16) {
    const Memory scales = block + kBlock * DC * 32 * BITS / 8;
#pragma unroll
    for (int g = 0; g < DC / GU; ++g) {
      if constexpr (BITS == 8) {
        k.scale[g] = load_at<uint32_t>(scales + g * 64, lane & 15);
      } else {
        const u32x2 v = load_at<u32x2>(scales + g * 128, lane & 15);
        k.scale[2 * g] = v[0];
        k.scale[2 * g + 1] = v[1];
      }
    }
  }
}
template <int BITS, int DC, int GU>
__device__ __forceinline__ void load_values(ValueWords<BITS, DC, GU>& v, Memory block, int lane) {
#pragma unroll
  for (int c = 0; c < DC; ++c) load_unit<BITS>(v.unit[c], block, c, lane);
  if constexpr (BITS != 16) {
    const Memory scales = block + kBlock * DC * 32 * BITS / 8;
#pragma unroll
    for (int g = 0; g < DC / GU; ++g) {
      v.scale[g] = load_at<half8v>(scales + g * (BITS == 8 ? 64 : 128), lane >> 4);
      if constexpr (BITS == 4) v.offset[g] = load_at<half8v>(scales + g * 128 + 64, lane >> 4);
    }
  }
}
template <int BITS, int DC, int GU>
__device__ __forceinline__ half8v key_operand(const KeyWords<BITS, DC, GU>& k, int c, int j) {
  if constexpr (BITS == 16) return key_values<16>(k.unit[c], j, (_Float16)0, (_Float16)0);
  if constexpr (BITS == 8) return key_values<8>(k.unit[c], j, half_of(k.scale[c / GU], j), (_Float16)0);
  if constexpr (BITS == 4) return key_values<4>(k.unit[c], j, half_of(k.scale[2 * (c / GU) + j], 0), half_of(k.scale[2 * (c / GU) + j], 1));
}
template <int BITS, int DC, int GU>
__device__ __forceinline__ half8v value_operand(const ValueWords<BITS, DC, GU>& v, int c, int j) {
  return value_values<BITS>(v.unit[c], j, v.scale[BITS == 16 ? 0 : c / GU], v.offset[BITS == 4 ? c / GU : 0]);
}

__device__ __forceinline__ float4v mfma(half8v a, half8v b, float4v c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }

// A walk over every STEP-th block of a split: which page a block is in, without a division a block.  The next block's entry of the
// page table is on its way while a block is worked on, by a scalar load: a wait for it is no wait for the codes in flight.
typedef const __attribute__((address_space(4))) int32_t* Table;
template <int STEP>
struct Walk {
  Table table;                 // of the sequence
  int last_col, page_blocks;
  int64_t pages;
  int col, in_page;            // page of the sequence, block in it
  int col_step, block_step;
  int entry;                   // of the table
};
template <int STEP>
__device__ __forceinline__ void walk_begin(Walk<STEP>& w, int block) {
  w.col = block / w.page_blocks;
  w.in_page = block - w.col * w.page_blocks;
  w.entry = w.table[min(w.col, w.last_col)];
}
template <int STEP>
__device__ __forceinline__ Walk<STEP> walk_of(const Params& p, int seq, int block) {
  Walk<STEP> w;
  w.table = (Table)(p.table + (int64_t)seq * p.table_pages);
  w.last_col = p.table_pages - 1;
  w.page_blocks = p.page_blocks;
  w.pages = p.pages;
  w.col_step = STEP / p.page_blocks;
  w.block_step = STEP - w.col_step * p.page_blocks;
  walk_begin(w, block);
  return w;
}
template <int STEP>
__device__ __forceinline__ void walk_on(Walk<STEP>& w) {
  w.col += w.col_step;
  w.in_page += w.block_step;
  if (w.in_page >= w.page_blocks) {
    w.in_page -= w.page_blocks;
    ++w.col;
  }
  w.entry = w.table[min(w.col, w.last_col)];
}
// Number of the block's page (-1: none).
template <int STEP>
__device__ __forceinline__ int walk_page(const Walk<STEP>& w) {
  return w.col <= w.last_col && w.entry >= 0 && w.entry < w.pages ? w.entry : -1;
}

// Factor of a part's sums where parts meet: its top is at most `raised`.  (A part that saw nothing has sums of zero; a NaN stays one.)
__device__ __forceinline__ float part_factor(float top, float raised) { return __builtin_amdgcn_exp2f(top - raised); }
// Row / query heads of a key head.  (row + 1/2) / shared is at least 1/2 / shared away from a whole number: 3e-5 at least, where the
// product is off by 64 * 2^-23 at most.
__device__ __forceinline__ int token_of(const Params& p, int row) { return (int)(((float)row + 0.5f) * p.inverse_shared); }
// Four channels of a row's result (a row that saw nothing has a total of zero).
__device__ __forceinline__ void store_row(const Params& p, int row_first, int head, int row, int dim, int d, float4v a, float total) {
  const int token = token_of(p, row);
  const float inverse = total == 0.0f ? 0.0f : 1.0f / total;
  *reinterpret_cast<half4v*>(p.y + (int64_t)(row_first + token) * p.y_stride + ((int64_t)head * p.shared + row - token * p.shared) * dim + d) =
      __builtin_convertvector(a * inverse, half4v);
}

__device__ __forceinline__ half8v masked(half8v v, u32x4 mask) { return __builtin_bit_cast(half8v, __builtin_bit_cast(u32x4, v) & mask); }

// What a wavefront carries from block to block.
template <int DC, int RT>
struct Sums {
  half8v query[RT][DC];                // row `column` of a tile, channels 32 c + 8 quarter + (0..7)
  float4v out[RT][2 * DC], total[RT];  // row `column`, channels 16 u + 4 quarter + (0..3)
  float top[RT];                       // what the weights are relative to, in powers of two
};

// The scores' turn: S^T of a block's 32 positions.
template <int BITS, int DC, int GU, int RT>
__device__ __forceinline__ void block_scores(float4v (&score)[RT][2], const KeyWords<BITS, DC, GU>& keys, const Sums<DC, RT>& s) {
#pragma unroll
  for (int t = 0; t < RT; ++t) score[t][0] = score[t][1] = (float4v){0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
  for (int c = 0; c < DC; ++c) {
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const half8v k = key_operand<BITS, DC, GU>(keys, c, j);
#pragma unroll
      for (int t = 0; t < RT; ++t) score[t][j] = mfma(k, s.query[t][c], score[t][j]);
    }
  }
}

// (Not the first half of a multiply-add.)
__device__ __forceinline__ float rounded_product(float a, float b) {
#pragma clang fp contract(off)
  const float c = a * b;
  return c;
}

// The weights' turn: of one tile's eight positions a lane, as the next product's operand.  Of a block that not every row sees all of,
// `visible` has a bit for each position (4 j + i: position 8 quarter + 4 j + i of the block).
template <int DC, int RT>
__device__ __forceinline__ half8v block_weights(float4v (&score)[2], Sums<DC, RT>& s, int t, float scale, bool whole, uint32_t visible, half8v ones) {
  if (!whole) {
#pragma unroll
    for (int i = 0; i < 8; ++i) score[i >> 2][i & 3] = visible >> i & 1u ? score[i >> 2][i & 3] : -__builtin_inff();
  }
  float most = score[0][0];
#pragma unroll
  for (int i = 1; i < 8; ++i) most = fmaxf(most, score[i >> 2][i & 3]);
  float factor = scale;
  if (__any(__builtin_fmaf(most, scale, -s.top[t]) > kSlack)) {         // (as the weights are worked out: none passes 2^kSlack)
    most = max_of_column(most);
    const bool own = __builtin_fmaf(most, scale, -s.top[t]) > kSlack;   // (a row's own need: others do not change its result)
    const float raised = own ? rounded_product(most, scale) - kLift : s.top[t];
    const float shrink = raised == s.top[t] ? 1.0f : __builtin_amdgcn_exp2f(s.top[t] - raised);
    s.top[t] = raised;
    s.total[t] *= shrink;
#pragma unroll
    for (int u = 0; u < 2 * DC; ++u) s.out[t][u] *= shrink;
    if (__builtin_expect(__any(own && fabsf(raised) >= kFar), 0)) {     // (but for this rounding of the tile's scores, within their own)
#pragma unroll
      for (int i = 0; i < 8; ++i) score[i >> 2][i & 3] = rounded_product(score[i >> 2][i & 3], scale);
      factor = 1.0f;
    }
  }
  half2v w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    float2v e;
#pragma unroll
    for (int k = 0; k < 2; ++k) e[k] = __builtin_amdgcn_exp2f(__builtin_fmaf(score[i >> 1][(2 * i + k) & 3], factor, -s.top[t]));
    w[i] = __builtin_convertvector(e, half2v);
  }
  half8v weight = join(w[0], w[1], w[2], w[3]);
  if (!whole) {                                  // (with a scale of zero those that are not seen are no numbers)
    u32x4 m;
#pragma unroll
    for (int i = 0; i < 4; ++i) m[i] = (visible >> (2 * i) & 1u ? 0x0000ffffu : 0u) | (visible >> (2 * i + 1) & 1u ? 0xffff0000u : 0u);
    weight = masked(weight, m);
  }
  s.total[t] = mfma(ones, weight, s.total[t]);
  return weight;
}

// What a workgroup has to do: a split of the positions, a row block of a key head (blockIdx.y), a sequence (blockIdx.z).
struct Place {
  int seq, head, row_block;
  int row_first;               // the sequence's first row of q and y
  int rows, row0;              // (token, query head) pairs of the key head; the row block's first
  int past;
  int64_t length;              // positions that exist
  int active;                  // splits that have any
  int first_block, end_block;  // of this one
};
// From what the step says, within what the host said.  False: nothing to do.
__device__ __forceinline__ bool find_place(const Params& p, int block_rows, int split, Place* w) {
  w->seq = blockIdx.z;
  w->head = blockIdx.y / p.row_blocks;
  w->row_block = blockIdx.y - w->head * p.row_blocks;
  w->row_first = max(p.first[w->seq], 0);
  const int count = min(min(max(p.first[w->seq + 1], 0), p.tokens) - w->row_first, p.most_tokens);   // (at most kMostTokens)
  w->past = max(p.past[w->seq], 0);
  w->rows = count * p.shared;
  w->row0 = w->row_block * block_rows;
  if (count <= 0 || w->row0 >= w->rows) return false;
  w->length = min((int64_t)w->past + count, (int64_t)p.table_pages * p.page_blocks * kBlock);
  int64_t chunk = p.chunk;
  if (chunk * p.splits < w->length) chunk = ((w->length + p.splits - 1) / p.splits + kBlock - 1) / kBlock * kBlock;
  w->active = max(1, (int)((w->length + chunk - 1) / chunk));
  w->first_block = (int)(split * chunk / kBlock);
  w->end_block = (int)((min((split + 1) * chunk, w->length) + kBlock - 1) / kBlock);
  return split < w->active;
}

template <int DC, int RT>
__device__ __forceinline__ void clear_sums(Sums<DC, RT>& s) {
#pragma unroll
  for (int t = 0; t < RT; ++t) {
    s.top[t] = kNothing;
    s.total[t] = (float4v){0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int u = 0; u < 2 * DC; ++u) s.out[t][u] = (float4v){0.0f, 0.0f, 0.0f, 0.0f};
  }
}
// Queries of the rows from `row` on, and which new positions their tokens see.
template <int DC, int RT>
__device__ __forceinline__ void load_queries(const Params& p, const Place& w, int row, int lane, Sums<DC, RT>& s, uint64_t (&sees)[RT]) {
  const int column = lane & 15, quarter = lane >> 4;
#pragma unroll
  for (int t = 0; t < RT; ++t) {
    const int r = row + 16 * t + column;
    const bool live = r < w.rows;
    const int token = live ? token_of(p, r) : 0;
    const _Float16* q = p.q + (int64_t)(w.row_first + token) * p.q_stride + ((int64_t)w.head * p.shared + (live ? r - token * p.shared : 0)) * (DC * 32);
#pragma unroll
    for (int c = 0; c < DC; ++c) {
      u32x4 v = {0u, 0u, 0u, 0u};
      if (live) v = *reinterpret_cast<const u32x4*>(q + 32 * c + 8 * quarter) ^ p.flip;     // (a negative scale's sign)
      s.query[t][c] = __builtin_bit_cast(half8v, v);
    }
    sees[t] = !live ? 0 : (p.mask ? p.mask[w.row_first + token] : ~0ull >> (63 - token));
  }
}
// Which of a lane's eight positions of a block a tile's row sees: bit 4 j + i for position 8 quarter + 4 j + i.
__device__ __forceinline__ uint32_t visible_places(int place, int limit, uint64_t sees) {
  uint32_t visible = 0u;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int n = place + i;
    visible |= n < limit && (n < 0 || (sees >> (n & 63) & 1u) != 0) ? 1u << i : 0u;
  }
  return visible;
}
// For blocks that not every row sees all of.  Which of a lane's eight positions exist, as a mask of half words.
__device__ __forceinline__ u32x4 existing_places(int place, int limit) {
  u32x4 m;
#pragma unroll
  for (int i = 0; i < 4; ++i) m[i] = (place + 2 * i < limit ? 0x0000ffffu : 0u) | (place + 2 * i + 1 < limit ? 0xffff0000u : 0u);
  return m;
}
// Zero, or a NaN where some of v is not finite.
__device__ __forceinline__ half8v oddness(half8v v, half8v sum) {
  const half8v zero = {0, 0, 0, 0, 0, 0, 0, 0};
  return __builtin_elementwise_fma(v, zero, sum);
}
__device__ __forceinline__ bool any_odd(half8v sum) {
  half8v t = sum;
  bool odd = false;
#pragma unroll
  for (int i = 0; i < 8; ++i) odd |= t[i] != t[i];
  return __any(odd);
}
// A weight of zero must not meet an infinity or a NaN: of a block that not every row sees all of, what is not finite is taken out of
// the values, after this has counted it for the rows that see it: +inf as 1, -inf as 64, NaN as 4096 (there are at most
// 32 of each), which get it added.
template <int DC, int RT>
__device__ __forceinline__ void add_odd(half8v v, const uint32_t (&visible)[RT], Sums<DC, RT>& s, int u) {
  __builtin_amdgcn_sched_barrier(0);             // (seldom run: one tile after the other, for the sake of the registers)
  half8v odd = {0, 0, 0, 0, 0, 0, 0, 0};
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const uint32_t bits = bits_of(v[i]);
    if ((bits & 0x7c00u) == 0x7c00u) odd[i] = (_Float16)((bits & 0x3ffu) ? 4096.0f : (bits & 0x8000u ? 64.0f : 1.0f));
  }
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
      s.out[t][u][i] += nan ? __builtin_nanf("") : (plus ? __builtin_inff() : (minus ? -__builtin_inff() : 0.0f));
    }
  }
}
__device__ __forceinline__ half8v finite_only(half8v v) {
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = (bits_of(v[i]) & 0x7c00u) == 0x7c00u ? (_Float16)0 : v[i];
  return v;
}

// A split's partial results: sums [partial_rows][dim], then a top and a total for each row.
__device__ __forceinline__ float* partial_of(const Params& p, const Place& w, int split, int dim) {
  const int64_t unit = ((int64_t)w.seq * p.heads + w.head) * p.row_blocks + w.row_block;
  return p.partial + (unit * p.splits + split) * split_floats(p.partial_rows, dim);
}

// The kernel's arguments once more, from memory: what only its end needs would else take up scalar registers through its loops.
__device__ __forceinline__ Params arguments_again() {
  typedef const __attribute__((address_space(4))) Params* Kernarg;
  Kernarg args = (Kernarg)__builtin_amdgcn_kernarg_segment_ptr();
  asm("" : "+s"(args));
  return *(const Params*)args;
}

// The end of a workgroup, of GROUPS_R x PARTS wavefronts: PARTS that took different positions for the same RT tiles of rows, GROUPS_R
// that took different rows.  The parts' sums meet in LDS in their order, then the splits' through memory.
template <int DC, int RT, int GROUPS_R, int PARTS>
struct Ending {
  static constexpr int kRows = 16 * RT * GROUPS_R, kThreads = 64 * GROUPS_R * PARTS, kDim = DC * 32, kPitch = kDim + 4;
  static constexpr bool kLastAdds = kRows == 16;
  static constexpr int kMeetFloats = PARTS * kRows * (kPitch + 3) + 2 * kRows;
  static constexpr int kJoinFloats = kLastAdds ? 2 * kRows * kMostSplits + kRows + kThreads * 4 : 0;
  static constexpr int kFloats = kMeetFloats > kJoinFloats ? kMeetFloats : kJoinFloats;
};
template <int DC, int RT, int GROUPS_R, int PARTS>
__device__ __forceinline__ void end_workgroup(const Params& p, const Place& w, float* lds, Sums<DC, RT>& s, int group, int part, int lane) {
  using E = Ending<DC, RT, GROUPS_R, PARTS>;
  constexpr int kRows = E::kRows, kThreads = E::kThreads, kDim = E::kDim, kPitch = E::kPitch, kFours = kDim / 4;
  const int column = lane & 15, quarter = lane >> 4;
  float* sums = lds;                                                              // [PARTS][kRows][kPitch]
  float2v* ends = reinterpret_cast<float2v*>(lds + PARTS * kRows * kPitch);       // [PARTS][kRows]: top, total
  float* factors = reinterpret_cast<float*>(ends + PARTS * kRows);                // [PARTS][kRows]
  float2v* row_ends = reinterpret_cast<float2v*>(factors + PARTS * kRows);        // [kRows]
  const int live_rows = min(w.rows - w.row0, kRows), mine0 = 16 * RT * group + column;   // (the lane's first row)
  if (quarter == 0) {
#pragma unroll
    for (int t = 0; t < RT; ++t) {
      ends[part * kRows + mine0 + 16 * t][0] = s.top[t];
      ends[part * kRows + mine0 + 16 * t][1] = s.total[t][0];
    }
  }
  __syncthreads();
  constexpr int kLanes = PARTS <= 1 ? 1 : (PARTS <= 2 ? 2 : (PARTS <= 4 ? 4 : (PARTS <= 8 ? 8 : 16)));      // a row's parts side by side
  static_assert(kRows * kLanes <= kThreads, "");
  if ((int)threadIdx.x < kRows * kLanes) {
    const int row = threadIdx.x / kLanes, k = threadIdx.x % kLanes;
    float2v end = {kNothing, 0.0f};
    if (k < PARTS) end = ends[k * kRows + row];
    float raised = end[0];
#pragma unroll
    for (int d = kLanes / 2; d >= 1; d >>= 1) raised = fmaxf(raised, __shfl_xor(raised, d, kLanes));
    const float factor = part_factor(end[0], raised);
    float total = factor * end[1];
#pragma unroll
    for (int d = kLanes / 2; d >= 1; d >>= 1) total += __shfl_xor(total, d, kLanes);
    if (k < PARTS) factors[k * kRows + row] = factor;
    if (k == 0) row_ends[row] = (float2v){raised, total};
  }
  __syncthreads();
#pragma unroll
  for (int t = 0; t < RT; ++t) {
    const int row = mine0 + 16 * t;
    if (row < live_rows) {
      const float factor = factors[part * kRows + row];
#pragma unroll
      for (int u = 0; u < 2 * DC; ++u) *reinterpret_cast<float4v*>(&sums[(part * kRows + row) * kPitch + 16 * u + 4 * quarter]) = s.out[t][u] * factor;
    }
  }
  __syncthreads();
  float* mine = partial_of(p, w, blockIdx.x, kDim);
  const int64_t next = split_floats(p.partial_rows, kDim);                       // from a split's to the next one's
  const Buffer through = buffer_of(mine, next);
#pragma unroll 1
  for (int i = threadIdx.x; i < live_rows * kFours; i += kThreads) {              // a thread takes four channels
    const int row = i / kFours, d = i % kFours * 4;
    float4v a = *reinterpret_cast<const float4v*>(&sums[row * kPitch + d]);
#pragma unroll
    for (int k = 1; k < PARTS; ++k) a += *reinterpret_cast<const float4v*>(&sums[(k * kRows + row) * kPitch + d]);
    if (w.active == 1)
      store_row(p, w.row_first, w.head, w.row0 + row, kDim, d, a, row_ends[row][1]);
    else
      store4(through, row * kDim + d, a);
  }
  if (w.active == 1) return;
  if ((int)threadIdx.x < live_rows) store2(through, p.partial_rows * kDim + 2 * threadIdx.x, row_ends[threadIdx.x]);
  if constexpr (E::kLastAdds) {
    uint32_t* last = reinterpret_cast<uint32_t*>(lds);            // (what was there has been added)
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    const int64_t unit = ((int64_t)w.seq * p.heads + w.head) * p.row_blocks + w.row_block;
    if (threadIdx.x == 0)
      *last = __hip_atomic_fetch_add(p.counters + unit, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == (uint32_t)(w.active - 1) ? 1u : 0u;
    __syncthreads();
    const bool adds = *last != 0u;
    __syncthreads();
    if (!adds) return;
    const Buffer all = buffer_of(partial_of(p, w, 0, kDim), p.splits * next);
    float2v* split_ends = reinterpret_cast<float2v*>(lds);        // [live_rows][active]: top and total, then factor and total
    float* row_total = lds + 2 * kRows * kMostSplits;             // [kRows]
    float* shares = row_total + kRows;                            // [kThreads][4]
    // An item is four channels of a row; where there are fewer items than threads, several threads share one's splits.  The first
    // loads of an item do not wait for the splits' factors.
    constexpr int kAhead = 8;
    const int items = live_rows * kFours;
    int sharers = 1;
    while (sharers < 16 && 2 * sharers * items <= kThreads && 2 * sharers <= w.active) sharers *= 2;
    const int side = kThreads / sharers, share = threadIdx.x / side, place = threadIdx.x - share * side;
    float4v ahead[kAhead];
    auto load_ahead = [&](int i, int split) {
      const int at = min(i, items - 1) * 4;                       // row * kDim + d
#pragma unroll
      for (int k = 0; k < kAhead; ++k) ahead[k] = load4(all, min(split + k * sharers, w.active - 1) * (int)next + at);
    };
    load_ahead(place, share);
#pragma unroll 1
    for (int i = threadIdx.x; i < live_rows * w.active; i += kThreads) {
      const int split = i / live_rows, row = i - split * live_rows;
      split_ends[row * w.active + split] = load2(all, split * (int)next + p.partial_rows * kDim + 2 * row);
    }
    __syncthreads();
#pragma unroll 1
    for (int row = threadIdx.x >> 4; row < live_rows; row += kThreads / 16) {      // sixteen lanes a row
      float raised = kNothing, sum = 0.0f;
#pragma unroll 1
      for (int i = column; i < w.active; i += 16) raised = fmaxf(raised, split_ends[row * w.active + i][0]);
#pragma unroll
      for (int d = 8; d >= 1; d >>= 1) raised = fmaxf(raised, __shfl_xor(raised, d, 16));
#pragma unroll 1
      for (int i = column; i < w.active; i += 16) {
        const float2v end = split_ends[row * w.active + i];
        const float factor = part_factor(end[0], raised);
        split_ends[row * w.active + i][0] = factor;
        sum += factor * end[1];
      }
#pragma unroll
      for (int d = 8; d >= 1; d >>= 1) sum += __shfl_xor(sum, d, 16);
      if (column == 0) row_total[row] = sum;
    }
    __syncthreads();
#pragma unroll 1
    for (int base = 0; base < items; base += side) {
      const int i = base + place, row = min(i, items - 1) / kFours;
      float4v a = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll 1
      for (int split = share; split < w.active; split += kAhead * sharers) {
        if (base > 0 || split != share) load_ahead(i, split);
#pragma unroll
        for (int k = 0; k < kAhead; ++k)
          if (split + k * sharers < w.active) a += ahead[k] * split_ends[row * w.active + split + k * sharers][0];
      }
      if (sharers > 1) {
        __syncthreads();
        *reinterpret_cast<float4v*>(&shares[threadIdx.x * 4]) = a;
        __syncthreads();
        if (share == 0)
          for (int k = 1; k < sharers; ++k) a += *reinterpret_cast<const float4v*>(&shares[(threadIdx.x + k * side) * 4]);
      }
      if (i < items && share == 0) store_row(p, w.row_first, w.head, w.row0 + row, kDim, i % kFours * 4, a, row_total[row]);
    }
    if (threadIdx.x == 0) __hip_atomic_store(p.counters + unit, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  }
}

// The splits' sums meet.  DIM / 4 lanes take a row, four channels each; `sharers` such sets share a row's splits, every sharers-th each, where
// there are many.  blockIdx as in the kernels before, .x counting rows.  Nothing here is work: what it takes is
// a trip to memory, so all of it is asked for at once, before the sequence's length says how many splits there are, by as many wavefronts as
// there is room for (16384 rows of 128 channels in 4 splits: 10 us; with eight splits a thread in flight, two wavefronts a SIMD, 19).
template <int DIM>
__global__ __launch_bounds__(kJoinThreads, DIM == 64 ? 7 : 8) void lutgemm_attention_join_kernel(Params p, int block_rows, int sharers) {
  constexpr int kLanes = DIM / 4, kSets = kJoinThreads / kLanes, kAhead = kJoinAhead;       // (48 lanes: some threads idle)
  __shared__ __attribute__((aligned(16))) float shares[kSets][DIM];
  __shared__ float share_total[kSets];
  __shared__ float2v ends[kSets][kMostSplits];                    // of a row: top, total of every split
  const int set = threadIdx.x / kLanes, lane = threadIdx.x - set * kLanes;
  const int share = set % sharers, slot = set / sharers, row = blockIdx.x * (kSets / sharers) + slot;
  Place w;
  w.seq = blockIdx.z;
  w.head = blockIdx.y / p.row_blocks;
  w.row_block = blockIdx.y - w.head * p.row_blocks;
  const float* partial = partial_of(p, w, 0, DIM);
  const int64_t next = split_floats(p.partial_rows, DIM);
  const bool held = set < kSets / sharers * sharers && row < p.partial_rows;       // (sets that make up no row are idle)
  const float* sums = partial + row * DIM + 4 * lane;
  float4v ahead[kAhead];
#pragma unroll
  for (int k = 0; k < kAhead; ++k)
    if (held && share + k * sharers < p.splits) ahead[k] = *reinterpret_cast<const float4v*>(sums + (share + k * sharers) * next);
  if (held)
    for (int i = share * kLanes + lane; i < p.splits; i += sharers * kLanes)
      ends[slot][i] = *reinterpret_cast<const float2v*>(partial + i * next + p.partial_rows * DIM + 2 * row);
  const bool joined = find_place(p, block_rows, 0, &w) && w.active > 1;
  const bool live = held && joined && row < min(w.rows - w.row0, block_rows);
  __syncthreads();
  float4v a = {0.0f, 0.0f, 0.0f, 0.0f};
  float total = 0.0f;
  if (live) {
    float raised = kNothing;
    for (int i = 0; i < w.active; ++i) raised = fmaxf(raised, ends[slot][i][0]);
    auto add = [&](float4v v, int split) {
      const float2v end = ends[slot][split];
      const float factor = part_factor(end[0], raised);
      total += factor * end[1];
      a += v * factor;
    };
#pragma unroll
    for (int k = 0; k < kAhead; ++k)
      if (share + k * sharers < w.active) add(ahead[k], share + k * sharers);
#pragma unroll 2
    for (int i = share + kAhead * sharers; i < w.active; i += sharers) add(*reinterpret_cast<const float4v*>(sums + i * next), i);
    if (share != 0) {
      *reinterpret_cast<float4v*>(&shares[set][4 * lane]) = a;
      if (lane == 0) share_total[set] = total;
    }
  }
  __syncthreads();
  if (!live || share != 0) return;
  for (int k = 1; k < sharers; ++k) {
    a += *reinterpret_cast<const float4v*>(&shares[set + k][4 * lane]);
    total += share_total[set + k];
  }
  store_row(p, w.row_first, w.head, w.row0 + row, DIM, 4 * lane, a, total);
}

// The values of a block that not every row sees all of: those that do not exist become zero, and those that are not finite are
// added to the rows that see them and become zero.  Of quantised ones the scales say which they are.
template <int BITS, int DC, int GU, int RT>
__device__ __forceinline__ void mask_values(ValueWords<BITS, DC, GU>& v, int place, int limit, const uint32_t (&visible)[RT], Sums<DC, RT>& s) {
  const u32x4 exist = existing_places(place, limit);
  half8v odd = {0, 0, 0, 0, 0, 0, 0, 0};
  if constexpr (BITS == 16) {
#pragma unroll
    for (int c = 0; c < DC; ++c)
#pragma unroll
      for (int i = 0; i < 8; ++i) v.unit[c].w[i] &= exist[i & 3];
#pragma unroll
    for (int u = 0; u < 2 * DC; ++u) odd = oddness(value_operand<BITS, DC, GU>(v, u / 2, u % 2), odd);
  } else {
#pragma unroll
    for (int g = 0; g < DC / GU; ++g) {
      v.scale[g] = masked(v.scale[g], exist);
      odd = oddness(v.scale[g], odd);
      if constexpr (BITS == 4) {
        v.offset[g] = masked(v.offset[g], exist);
        odd = oddness(v.offset[g], odd);
      }
    }
  }
  if (__builtin_expect(any_odd(odd), 0)) {
#pragma unroll
    for (int u = 0; u < 2 * DC; ++u) add_odd<DC, RT>(value_operand<BITS, DC, GU>(v, u / 2, u % 2), visible, s, u);
    if constexpr (BITS == 16) {
#pragma unroll
      for (int c = 0; c < DC; ++c)
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const u32x4 w = __builtin_bit_cast(u32x4, finite_only(value_operand<BITS, DC, GU>(v, c, j)));
#pragma unroll
          for (int i = 0; i < 4; ++i) v.unit[c].w[4 * j + i] = w[i];
        }
    } else {
      // a scale or an offset that is not finite makes all it stands for so: both go
#pragma unroll
      for (int g = 0; g < DC / GU; ++g) {
        const half8v both_sum = oddness(v.scale[g], oddness(BITS == 4 ? v.offset[BITS == 4 ? g : 0] : v.scale[g], (half8v){0, 0, 0, 0, 0, 0, 0, 0}));
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const bool gone = both_sum[i] != both_sum[i];
          v.scale[g][i] = gone ? (_Float16)0 : v.scale[g][i];
          if constexpr (BITS == 4) v.offset[g][i] = gone ? (_Float16)0 : v.offset[g][i];
        }
      }
    }
  }
}

// Address of a block's codes: of the page that `page` numbers (0 where there is none: its values are not used).
struct Blocks {
  Memory head;                 // the head's first block of page 0
  int64_t page_bytes;
  int block_bytes;
};
__device__ __forceinline__ Blocks blocks_of(const Params& p, int head) {
  return {(Memory)p.pool + (int64_t)head * p.page_blocks * p.block_bytes, (int64_t)p.heads * p.page_blocks * p.block_bytes, p.block_bytes};
}
__device__ __forceinline__ Memory block_address(const Blocks& b, int page, int in_page) {
  return b.head + max(page, 0) * b.page_bytes + (int64_t)in_page * b.block_bytes;
}

// Few rows: every wavefront takes all of them, and blocks of its own, from memory straight into registers.  Two blocks are on
// their way while one is worked on: a set's keys are asked for when the set's last ones have met the queries, its values
// when those have been added.  Bound by the stream of codes where it is long (16 sequences of 64 heads, up to 4000 positions at 8 bits:
// 654 MB in 112 us, 5.8 TB/s where a read-only kernel has 6.9), else by what begins and ends it: the chain lengths, page, codes,
// and the sums (331 positions of 40 heads at 16 bits 6.2 us, of which an empty kernel takes 2).
// BITS of a code, DC units of 32 channels to a head, GU of them to a scale, RT tiles of 16 rows.
template <int BITS, int DC, int GU, int RT, int WAVES>
__global__ __launch_bounds__(WAVES * 64, attention_waves_per_simd(DC * 32, BITS, GU * 32, RT)) void lutgemm_attention_kernel(Params p) {
  constexpr int kSets = attention_sets(DC * 32, BITS, GU * 32, RT);
  __shared__ __attribute__((aligned(16))) float lds[Ending<DC, RT, 1, WAVES>::kFloats];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), quarter = lane >> 4;
  // The page table does not wait for the sequence's lengths (a split begins elsewhere only if it is longer than planned).
  const int planned = (int)min((int64_t)blockIdx.x * (p.chunk / kBlock), (int64_t)p.table_pages * p.page_blocks) + wave;
  Walk<WAVES> walk = walk_of<WAVES>(p, blockIdx.z, planned);
  Place w;
  if (!find_place(p, 16 * RT, blockIdx.x, &w)) return;
  if (w.first_block + wave != planned) walk_begin(walk, w.first_block + wave);

  Sums<DC, RT> s;
  clear_sums(s);
  const half2v one = both((_Float16)1.0f);
  const half8v ones = join(one, one, one, one);
  const Blocks blocks = blocks_of(p, w.head);
  const int value_offset = p.block_bytes / 2;
  KeyWords<BITS, DC, GU> keys[kSets];
  ValueWords<BITS, DC, GU> values[kSets];
  uint64_t sees[RT];

  // A block's keys are asked for when those kSets blocks before have met the queries, its values when those before have been added.
  // The fetches are free of branches, so that the compiler knows at every wait how many loads are younger than the one it waits
  // for: a wavefront that runs out of blocks fetches its last one again.
  const int whole_end = w.past / kBlock;      // every row sees all of the blocks before it
  int block = w.first_block + wave;
  if (block < w.end_block) {
    bool dead[kSets];
    Memory at = nullptr;
    int ahead = block;                        // the next block to be asked for
    auto find = [&](int set) {
      if (ahead < w.end_block) {
        const int page = walk_page(walk);
        dead[set] = page < 0;
        at = block_address(blocks, page, walk.in_page);
        ahead += WAVES;
        walk_on(walk);
      }
      asm("" : "+s"(at));                     // (the same address again is not the same load again)
    };
#pragma unroll
    for (int set = 0; set < kSets; ++set) {
      find(set);
      load_keys<BITS, DC, GU>(keys[set], at, lane);
      load_values<BITS, DC, GU>(values[set], at + value_offset, lane);
    }
    load_queries<DC, RT>(p, w, w.row0, lane, s, sees);
    bool more = true;
    while (more) {
#pragma unroll
      for (int set = 0; set < kSets; ++set) {
        float4v score[RT][2];
        block_scores<BITS, DC, GU, RT>(score, keys[set], s);
        const bool skip = dead[set], whole = block < whole_end;
        find(set);
        load_keys<BITS, DC, GU>(keys[set], at, lane);
        if (!skip) {
          const int place = block * kBlock + 8 * quarter - w.past;      // of the lane's first position, counted from the new ones
          const int limit = (int)(w.length - w.past);                   // positions from here on do not exist
          half8v weight[RT];
          uint32_t visible[RT];
#pragma unroll
          for (int t = 0; t < RT; ++t) {
            visible[t] = 0u;
            if (!whole) visible[t] = visible_places(place, limit, sees[t]);
            weight[t] = block_weights<DC, RT>(score[t], s, t, p.scale, whole, visible[t], ones);
          }
          if (!whole) mask_values<BITS, DC, GU, RT>(values[set], place, limit, visible, s);
#pragma unroll
          for (int u = 0; u < 2 * DC; ++u) {
            const half8v v = value_operand<BITS, DC, GU>(values[set], u / 2, u % 2);
#pragma unroll
            for (int t = 0; t < RT; ++t) s.out[t][u] = mfma(v, weight[t], s.out[t][u]);
          }
        }
        load_values<BITS, DC, GU>(values[set], at + value_offset, lane);
        block += WAVES;
        more = block < w.end_block;
        if (!more) break;
      }
    }
  }
  end_workgroup<DC, RT, 1, WAVES>(arguments_again(), w, lds, s, 0, wave, lane);
}

// Many rows: GROUPS_R wavefronts share a block, RT tiles of rows each, so that its codes are fetched and made fp16 once for all of them:
// each does its share of the block's 2 DC units (keys, values) and puts the operands into LDS, in the order
// in which the lanes want them back (16 bytes each, no bank conflicts).  Where there are fewer rows than eight wavefronts
// hold, PARTS sets of GROUPS_R take blocks in turn.
// Two wavefronts share a SIMD, and a block is matrix work (scores, weighted values) and vector work (the weights) of about the same
// length: so the first four wavefronts and the last four run half a block apart, held there by two barriers a block, and
// the one's matrix work hides under the other's vector work.  Between its barriers a wavefront
//     works out the weights of block n,  then  adds its weighted values, puts the operands of block n + 2 into LDS where block n's
//                                              were, and forms the scores of block n + 1;
// each operand of 16 bytes a lane is asked for as soon as the product before it has used the register, so a block's values are in
// registers when its keys have been used.  (The last operands of a block are put one barrier before the early four
// read them, and the late four have read a block one barrier before the early four put another in its place.)
// Bound by both kinds of instruction, which hide under each other in part only: with 256 rows of 128 channels a block takes 1.0 us, its
// products alone 0.5, its vector instructions alone 0.8 (64 tokens x 8 query heads a key head over 4 x 8192 positions at 8 bits: 93 us,
// 750 TFLOP/s, of which the sums' way through memory and the second kernel are 20; all eight wavefronts in step, 112).
template <int BITS, int DC, int GU, int RT, int GROUPS_R, int PARTS>
__global__ __launch_bounds__(GROUPS_R * PARTS * 64, 2) void lutgemm_attention_shared_kernel(Params p) {
  constexpr int kEach = (2 * DC + GROUPS_R - 1) / GROUPS_R;        // units of a wavefront
  constexpr int kOperands = 2 * DC * 2 * 1024;                     // bytes of a block's: units x runs
  constexpr int kHeld = 2 * DC;                                    // of a block's keys, or of its values
  static_assert(GROUPS_R * PARTS == 8, "");
  using E = Ending<DC, RT, GROUPS_R, PARTS>;
  constexpr int kBytes = 2 * PARTS * kOperands > E::kFloats * 4 ? 2 * PARTS * kOperands : E::kFloats * 4;
  __shared__ __attribute__((aligned(16))) char lds[kBytes];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), quarter = lane >> 4;
  const int group = wave % GROUPS_R, part = wave / GROUPS_R;
  Place w;
  if (!find_place(p, 16 * RT * GROUPS_R, blockIdx.x, &w)) return;

  Sums<DC, RT> s;
  clear_sums(s);
  const half2v one = both((_Float16)1.0f);
  const half8v ones = join(one, one, one, one);
  Walk<PARTS> walk = walk_of<PARTS>(p, w.seq, w.first_block + part);
  const Blocks blocks = blocks_of(p, w.head);

  constexpr int kCode = kBlock * DC * 32 * BITS / 8;
  Unit<BITS> unit[kEach];
  u32x4 scale[BITS == 16 ? 1 : kEach], offset[BITS == 4 ? kEach : 1];
  const uint32_t odd_lane = lane & 1 ? ~0u : 0u, upper_lane = lane & 2 ? ~0u : 0u;
  constexpr int kAhead = 2;                                        // blocks from the one at hand to the one found last
  uint32_t dead = 0;                                               // which of the last fetched blocks have no page, the last in bit 0
  int ahead = w.first_block + part;                                // the next block to be fetched
  Memory at = blocks.head;                                         // (of page 0: a part without a block fetches that)
  // Finds the block `ahead`, and fetches this wavefront's units of it.  (Apart: the page table's next entry is asked for where no product
  // waits for operands, which could only wait for it too.)
  auto find = [&]() {
    dead <<= 1;
    if (ahead < w.end_block) {                                     // (else the last one again: the loads are free of branches)
      const int page = walk_page(walk);
      dead |= page < 0;
      at = block_address(blocks, page, walk.in_page);
      ahead += PARTS;
      walk_on(walk);
    }
    asm("" : "+s"(at));                                            // (the same address again is not the same load again)
  };
  auto fetch = [&]() {
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      const int u = min(group + i * GROUPS_R, 2 * DC - 1);
      const bool key = u < DC;
      const int c = key ? u : u - DC, g = c / GU;
      const Memory half_block = at + (key ? 0 : p.block_bytes / 2);
      load_unit<BITS>(unit[i], half_block, c, lane);
      // Scales: the sixteen bytes that the lane's are among, of a key's or a value's unit by the same loads.
      if constexpr (BITS != 16) {
        const Memory scales = half_block + kCode + g * (BITS == 8 ? 64 : 128) + (key ? (lane & (BITS == 8 ? 12 : 14)) * (BITS == 8 ? 4 : 8) : (lane >> 4) * 16);
        scale[i] = load_at<u32x4>(scales, 0);
        if constexpr (BITS == 4) offset[i] = load_at<u32x4>(scales + (key ? 0 : 64), 0);
      }
    }
  };
  // The fetched units, as operands in a buffer (beyond the last block ones that nothing reads: a branch would hide from the compiler
  // how many loads are younger than those it waits for).
  auto put = [&](char* buffer) {
    u32x4* to = reinterpret_cast<u32x4*>(buffer) + lane;
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      const int u = group + i * GROUPS_R;
      if (kEach * GROUPS_R > 2 * DC && u >= 2 * DC) continue;
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        half8v v;
        if constexpr (BITS == 16) {
          const half8v none = {0, 0, 0, 0, 0, 0, 0, 0};
          v = value_values<16>(unit[i], j, none, none);
        } else if (u >= DC) {
          v = value_values<BITS>(unit[i], j, __builtin_bit_cast(half8v, scale[i]), __builtin_bit_cast(half8v, offset[BITS == 4 ? i : 0]));
        } else if constexpr (BITS == 8) {
          v = key_values<BITS>(unit[i], j, half_of(one_of(one_of(word_of<0>(scale[i]), word_of<1>(scale[i]), odd_lane),
                                                               one_of(word_of<2>(scale[i]), word_of<3>(scale[i]), odd_lane), upper_lane), j), (_Float16)0);
        } else {
          const uint32_t word = j ? one_of(word_of<1>(scale[i]), word_of<3>(scale[i]), odd_lane)
                                  : one_of(word_of<0>(scale[i]), word_of<2>(scale[i]), odd_lane);
          v = key_values<BITS>(unit[i], j, half_of(word, 0), half_of(word, 1));
        }
        to[(u * 2 + j) * 64] = __builtin_bit_cast(u32x4, v);
      }
    }
  };

  int block = w.first_block + part;                                // this part's
  char* buffer = lds + part * kOperands;                           // of its operands, and the next block's
  char* buffer1 = buffer + PARTS * kOperands;
  find();
  fetch();
  uint64_t sees[RT];
  load_queries<DC, RT>(p, w, w.row0 + 16 * RT * group, lane, s, sees);
  put(buffer);
  find();
  fetch();
  put(buffer1);
  find();
  fetch();
  const int stages = (w.end_block - w.first_block + PARTS - 1) / PARTS;
  const int whole_end = min(w.past / kBlock, w.end_block);         // every row sees all of the blocks before it
  const int whole_stages = max(0, whole_end - w.first_block) / PARTS;
  const bool idle = w.row0 + 16 * RT * group >= w.rows;            // no row of this wavefront's lives: it only helps with the operands
  const int limit_of_rows = (int)(w.length - w.past);
  half8v held[kHeld];
  float4v score[RT][2];
  auto operand = [&](const char* from, int u) { return reinterpret_cast<const half8v*>(from)[u * 64 + lane]; };
  // Scores of a block whose keys are held; leaves its values there.
  auto form_scores = [&](const char* from) {
#pragma unroll
    for (int t = 0; t < RT; ++t) score[t][0] = score[t][1] = (float4v){0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int u = 0; u < kHeld; ++u) {
#pragma unroll
      for (int t = 0; t < RT; ++t) score[t][u % 2] = mfma(held[u], s.query[t][u / 2], score[t][u % 2]);
      held[u] = operand(from, 2 * DC + u);
      __builtin_amdgcn_sched_barrier(0);
    }
  };
  __syncthreads();
  if (!idle) {
#pragma unroll
    for (int u = 0; u < kHeld; ++u) held[u] = operand(buffer, u);
    form_scores(buffer);
  }
  if (wave >= 4) __syncthreads();
  auto stage = [&](auto all_whole) {
    constexpr bool kWhole = decltype(all_whole)::value;
    const bool none = block >= w.end_block || (dead >> kAhead & 1u);
    half8v weight[RT];
    find();
    if (!idle) {
      const int limit = none ? INT32_MIN : limit_of_rows, place = block * kBlock + 8 * quarter - w.past;
      uint32_t visible[RT];
#pragma unroll
      for (int t = 0; t < RT; ++t) {
        visible[t] = kWhole ? 0u : visible_places(place, limit, sees[t]);
        weight[t] = block_weights<DC, RT>(score[t], s, t, p.scale, kWhole, visible[t], ones);
      }
      if constexpr (!kWhole) {
        const u32x4 exist = existing_places(place, limit);
        half8v odd = {0, 0, 0, 0, 0, 0, 0, 0};
#pragma unroll
        for (int u = 0; u < kHeld; ++u) {
          held[u] = masked(held[u], exist);
          odd = oddness(held[u], odd);
        }
        if (__builtin_expect(any_odd(odd), 0)) {
#pragma unroll
          for (int u = 0; u < kHeld; ++u) {
            add_odd<DC, RT>(held[u], visible, s, u);
            held[u] = finite_only(held[u]);
          }
        }
      }
    }
    __syncthreads();
    __builtin_amdgcn_s_setprio(1);                                 // (the products' issue before the other wavefront's vector work: 107 -> 104 us)
    if (!idle) {
#pragma unroll
      for (int u = 0; u < kHeld; ++u) {
#pragma unroll
        for (int t = 0; t < RT; ++t) s.out[t][u] = mfma(held[u], weight[t], s.out[t][u]);
        held[u] = operand(buffer1, u);
        __builtin_amdgcn_sched_barrier(0);
      }
    }
    put(buffer);
    fetch();
    if (!idle) form_scores(buffer1);
    char* other = buffer;
    buffer = buffer1;
    buffer1 = other;
    __builtin_amdgcn_s_setprio(0);
    block += PARTS;
    __syncthreads();
  };
  // (Whole blocks without a page go through the code that can mask them.)
  for (int done = 0; done < stages; ++done) {
    for (; done < whole_stages && !(dead >> kAhead & 1u); ++done) stage(std::true_type());
    if (done >= stages) break;
    stage(std::false_type());
  }
  if (wave < 4) __syncthreads();
  __syncthreads();
  end_workgroup<DC, RT, GROUPS_R, PARTS>(arguments_again(), w, reinterpret_cast<float*>(lds), s, group, part, lane);
}

template <int BITS, int DC, int GU>
const void* pick_tiles(int row_tiles, int waves) {
  constexpr int kAll = 4 * attention_waves_per_simd(DC * 32, BITS, GU * 32, 1);
  if (row_tiles == 1 && waves == 4) return reinterpret_cast<const void*>(lutgemm_attention_kernel<BITS, DC, GU, 1, 4>);
  if (row_tiles == 1 && waves == kAll) return reinterpret_cast<const void*>(lutgemm_attention_kernel<BITS, DC, GU, 1, kAll>);
  if constexpr (DC <= 4) {
    if (row_tiles == 2 && waves == 4) return reinterpret_cast<const void*>(lutgemm_attention_kernel<BITS, DC, GU, 2, 4>);
  }
  if (waves != 8) return nullptr;
  if constexpr (DC <= 4) {
    if (row_tiles == 4) return reinterpret_cast<const void*>(lutgemm_attention_shared_kernel<BITS, DC, GU, 2, 2, 4>);
    if (row_tiles == 8) return reinterpret_cast<const void*>(lutgemm_attention_shared_kernel<BITS, DC, GU, 2, 4, 2>);
    if (row_tiles == 16) return reinterpret_cast<const void*>(lutgemm_attention_shared_kernel<BITS, DC, GU, 2, 8, 1>);
  } else {
    if constexpr (DC == 6) {
      if (row_tiles == 4) return reinterpret_cast<const void*>(lutgemm_attention_shared_kernel<BITS, DC, GU, 1, 4, 2>);
    }
    if (row_tiles == 8) return reinterpret_cast<const void*>(lutgemm_attention_shared_kernel<BITS, DC, GU, 1, 8, 1>);
  }
  return nullptr;
}
template <int BITS, int DC>
const void* pick_group(int units, int row_tiles, int waves) {
  if (BITS == 16 || units == DC) return pick_tiles<BITS, DC, DC>(row_tiles, waves);
  if constexpr (BITS != 16) {
    if (units == 1) return pick_tiles<BITS, DC, 1>(row_tiles, waves);
    if constexpr (DC % 2 == 0 && DC > 2) {
      if (units == 2) return pick_tiles<BITS, DC, 2>(row_tiles, waves);
    }
    if constexpr (DC == 6) {
      if (units == 3) return pick_tiles<BITS, DC, 3>(row_tiles, waves);
    }
    if constexpr (DC == 8) {
      if (units == 4) return pick_tiles<BITS, DC, 4>(row_tiles, waves);
    }
  }
  return nullptr;
}

}  // namespace

namespace lutgemm_attention_parts {
#define NAME2(k) family##k
#define NAME(k) NAME2(k)
const void* NAME(LUT_PART)(int group_units, int row_tiles, int waves) {
  constexpr int kBits = LUT_PART / 5 == 0 ? 16 : (LUT_PART / 5 == 1 ? 8 : 4);
  constexpr int kUnits = LUT_PART % 5 == 0 ? 2 : (LUT_PART % 5 == 1 ? 3 : (LUT_PART % 5 == 2 ? 4 : (LUT_PART % 5 == 3 ? 6 : 8)));
  return pick_group<kBits, kUnits>(group_units, row_tiles, waves);
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
  if (!q || !y || !workspace) return LUTGEMM_EINVAL;
  if ((((uintptr_t)q | (uintptr_t)y | (uintptr_t)workspace) & 15) != 0 || ((uintptr_t)mask & 7) != 0) return LUTGEMM_EINVAL;
  AttentionPlan plan;
  rc = check_attention(cache, step, q_heads, most_positions, &plan);
  if (rc != LUTGEMM_OK) return rc;
  const int64_t row = (int64_t)q_heads * cache->head_dim;
  if (q_stride < row || y_stride < row || q_stride % 8 != 0 || y_stride % 8 != 0) return LUTGEMM_EINVAL;
  const int group = group_of(cache->head_dim, cache->bits, cache->group);
  if (workspace_bytes < 32768 + 4 * (size_t)attention_partial_floats(plan, cache->heads, cache->head_dim, q_heads, step->seqs, step->most_tokens))
    return LUTGEMM_EWORKSPACE;
  if (step->tokens == 0 || step->most_tokens == 0) return LUTGEMM_OK;
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
  p.inverse_shared = 1.0f / (float)p.shared;
  p.block_bytes = block_bytes(cache->head_dim, cache->bits, group);
  p.splits = plan.splits;
  p.chunk = plan.chunk;
  p.row_blocks = plan.row_blocks;
  const int most_rows = step->most_tokens * p.shared;
  p.partial_rows = most_rows < 16 * plan.row_tiles ? most_rows : 16 * plan.row_tiles;
  p.scale = (scale < 0.0f ? -scale : scale) * 1.44269504088896340736f;
  p.flip = scale < 0.0f ? 0x80008000u : 0u;
  static const Family families[15] = {family0, family1, family2, family3, family4, family5, family6, family7,
                                      family8, family9, family10, family11, family12, family13, family14};
  const int bits = cache->bits == 16 ? 0 : (cache->bits == 8 ? 1 : 2), d = cache->head_dim;
  const int size = d == 64 ? 0 : (d == 96 ? 1 : (d == 128 ? 2 : (d == 192 ? 3 : 4)));
  const void* kern = families[bits * 5 + size](group / 32, plan.row_tiles, plan.waves);
  if (!kern) return LUTGEMM_EUNSUPPORTED;
  void* args[] = {&p};
  if (hipLaunchKernel(kern, dim3(plan.splits, cache->heads * plan.row_blocks, step->seqs), dim3(plan.waves * 64), args, 0,
                      static_cast<hipStream_t>(hip_stream)) != hipSuccess)
    return LUTGEMM_EHIP;
  if (plan.splits == 1 || plan.row_tiles == 1) return LUTGEMM_OK;      // (of 16 rows the last workgroup adds the splits)
  // Sets of DIM / 4 lanes in a workgroup; up to four splits a set.
  const int sets = kJoinThreads / (d / 4);
  int sharers = 1, block_rows = 16 * plan.row_tiles;
  while (2 * sharers <= sets && sharers * kJoinAhead < plan.splits) sharers *= 2;
  const int rows = sets / sharers;
  const void* join = d == 64    ? reinterpret_cast<const void*>(lutgemm_attention_join_kernel<64>)
                     : d == 96  ? reinterpret_cast<const void*>(lutgemm_attention_join_kernel<96>)
                     : d == 128 ? reinterpret_cast<const void*>(lutgemm_attention_join_kernel<128>)
                     : d == 192 ? reinterpret_cast<const void*>(lutgemm_attention_join_kernel<192>)
                                : reinterpret_cast<const void*>(lutgemm_attention_join_kernel<256>);
  void* join_args[] = {&p, &block_rows, &sharers};
  if (hipLaunchKernel(join, dim3((p.partial_rows + rows - 1) / rows, cache->heads * plan.row_blocks, step->seqs), dim3(kJoinThreads), join_args, 0,
                      static_cast<hipStream_t>(hip_stream)) != hipSuccess)
    return LUTGEMM_EHIP;
  return LUTGEMM_OK;
}
#endif
