// Rotary positions, and the key/value cache as it is written and read back: include/lutgemm.h has the formulas and the
// layout.  All three move data, so what bounds them is HBM (the write's 14 vector instructions a value come near it), and for a few
// tokens the launch and two trips to memory, one after the other.
#include <hip/hip_fp16.h>
#include <hip/hip_runtime.h>

#include <type_traits>

#include "lutgemm_kv.h"

using namespace lutgemm_kv_detail;

namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint16_t ushort2v __attribute__((ext_vector_type(2)));
typedef _Float16 half2v __attribute__((ext_vector_type(2)));

bool aligned16(const void* p) { return ((uintptr_t)p & 15) == 0; }

constexpr int64_t kCacheBytes = 32 << 20;      // of the L2 caches

// ---- rotary positions ----------------------------------------------------------------------------

struct RopeParams {
  const void* x;
  void* y;
  const int32_t* positions;
  const uint64_t* turns;
  int64_t x_stride, y_stride;
  int tokens, heads, head_dim, rot_dim;
  int pair_runs;       // runs of kRun pairs in rot_dim
  int heads_a_thread;
  float amplitude;
  float sign;          // of the angle
};

// sin and cos of 2 pi p / 2^32.  The quarter turn nearest to the angle comes off in integers, which is exact; the rest
// is at most pi / 4, where Taylor's series to the 9th and 8th power are within 2e-9 and 3e-8.
__device__ __forceinline__ void sin_cos_turn(uint32_t p, float* s, float* c) {
  const uint32_t quarter = (p + 0x20000000u) >> 30;
  const float x = (float)(int32_t)(p - (quarter << 30)) * 1.46291807926715968e-9f;   // 2 pi / 2^32
  const float x2 = x * x;
  float sn = fmaf(x2, 2.75573192e-6f, -1.98412698e-4f);
  sn = fmaf(sn, x2, 8.33333333e-3f);
  sn = fmaf(sn, x2, -1.66666667e-1f);
  sn = fmaf(sn * x2, x, x);
  float cs = fmaf(x2, 2.48015873e-5f, -1.38888889e-3f);
  cs = fmaf(cs, x2, 4.16666667e-2f);
  cs = fmaf(cs, x2, -0.5f);
  cs = fmaf(cs, x2, 1.0f);
  const bool swap = (quarter & 1u) != 0;
  const float a = swap ? cs : sn, b = swap ? sn : cs;
  *s = (quarter & 2u) ? -a : a;
  *c = ((quarter + 1u) & 2u) ? -b : b;
}

template <typename T, int N>
struct Run {
  T v[N];
};

template <typename T, int N>
__device__ __forceinline__ Run<T, N> load_run(const T* p) {
  if constexpr (N * sizeof(T) >= 16) {
    Run<T, N> r;
    const u32x4* s = reinterpret_cast<const u32x4*>(p);
    u32x4* d = reinterpret_cast<u32x4*>(&r);
#pragma unroll
    for (unsigned i = 0; i < N * sizeof(T) / 16; ++i) d[i] = s[i];
    return r;
  } else {
    Run<T, N> r;
#pragma unroll
    for (int i = 0; i < N; ++i) r.v[i] = p[i];
    return r;
  }
}
template <bool PAST, typename T, int N>
__device__ __forceinline__ void store_run(T* p, const Run<T, N>& r) {
  if constexpr (N * sizeof(T) >= 16) {
    const u32x4* s = reinterpret_cast<const u32x4*>(&r);
    u32x4* d = reinterpret_cast<u32x4*>(p);
#pragma unroll
    for (unsigned i = 0; i < N * sizeof(T) / 16; ++i) {
      if constexpr (PAST)
        __builtin_nontemporal_store(s[i], d + i);
      else
        d[i] = s[i];
    }
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i) p[i] = r.v[i];
  }
}

// A thread owns a run of PAIRS pairs (threadIdx.x) of one token for some heads, so that the angles, which no table holds, are worked
// out once for them: 64-bit position * frequency, one sine and cosine.  Runs behind the pairs' copy
// what is not turned, 2 PAIRS channels each.  PAST: more is written than the caches hold till it is read, so it goes past them (75 MB
// read and as many written 24.6 to 26.5 us, 5.7 to 6.1 TB/s, against 31.9; small outputs stay, for the next kernel).
template <typename T, int PAIRS, bool NEIGHBOURS, bool PAST>
__global__ __launch_bounds__(256) void lutgemm_rope_kernel(RopeParams p) {
  const int token = blockIdx.x * blockDim.z + threadIdx.z;
  if (token >= p.tokens) return;
  const int run = threadIdx.x, first_head = blockIdx.y * blockDim.y * p.heads_a_thread + threadIdx.y;
  const T* x = static_cast<const T*>(p.x) + token * p.x_stride;
  T* y = static_cast<T*>(p.y) + token * p.y_stride;
  const bool turned = run < p.pair_runs;
  int a, b;      // first channel of the two halves of the run
  if (!turned) {
    a = p.rot_dim + (run - p.pair_runs) * 2 * PAIRS;
    b = a + PAIRS;
  } else if (NEIGHBOURS) {
    a = run * 2 * PAIRS;
    b = a + PAIRS;
  } else {
    a = run * PAIRS;
    b = a + p.rot_dim / 2;
  }
  float sn[PAIRS], cs[PAIRS];
  if (turned) {
    const uint64_t position = (uint64_t)(int64_t)p.positions[token];
#pragma unroll
    for (int i = 0; i < PAIRS; ++i) {
      sin_cos_turn((uint32_t)(position * p.turns[run * PAIRS + i] >> 32), &sn[i], &cs[i]);
      sn[i] *= p.amplitude * p.sign;
      cs[i] *= p.amplitude;
    }
  }
  for (int k = 0; k < p.heads_a_thread; ++k) {
    const int head = first_head + k * blockDim.y;
    if (head >= p.heads) break;
    const int64_t at = (int64_t)head * p.head_dim;
    Run<T, PAIRS> u = load_run<T, PAIRS>(x + at + a), v = load_run<T, PAIRS>(x + at + b);
    if (turned) {
#pragma unroll
      for (int i = 0; i < PAIRS; ++i) {
        // the i-th pair: across the two runs, or neighbours within them
        T& first = NEIGHBOURS && PAIRS > 1 ? (2 * i < PAIRS ? u.v[(2 * i) % PAIRS] : v.v[(2 * i) % PAIRS]) : u.v[i];
        T& second = NEIGHBOURS && PAIRS > 1 ? (2 * i < PAIRS ? u.v[(2 * i + 1) % PAIRS] : v.v[(2 * i + 1) % PAIRS]) : v.v[i];
        const float f = (float)first, s = (float)second;
        first = (T)fmaf(f, cs[i], -(s * sn[i]));
        second = (T)fmaf(f, sn[i], s * cs[i]);
      }
    }
    store_run<PAST, T, PAIRS>(y + at + a, u);
    store_run<PAST, T, PAIRS>(y + at + b, v);
  }
}

template <typename T, int PAIRS, bool PAST>
const void* pick_rope(bool neighbours) {
  return neighbours ? reinterpret_cast<const void*>(lutgemm_rope_kernel<T, PAIRS, true, PAST>)
                    : reinterpret_cast<const void*>(lutgemm_rope_kernel<T, PAIRS, false, PAST>);
}
template <typename T, int WIDE>
const void* pick_rope(bool vectors, bool neighbours, bool past) {
  return !vectors ? pick_rope<T, 1, false>(neighbours) : (past ? pick_rope<T, WIDE, true>(neighbours) : pick_rope<T, WIDE, false>(neighbours));
}

// ---- the cache, written and read ------------------------------------------------------------------

struct KvParams {
  const void* k;               // written from, or read into
  const void* v;
  const int32_t* rows;
  char* pool;
  const int32_t* first;
  const int32_t* past;
  const int32_t* table;
  int64_t k_stride, v_stride;
  int64_t pages;
  int block_bytes, value_offset;       // of a block; of its value half
  int tokens, table_pages, page_blocks, heads;
};

// Where the tokens of a sequence are, checked against what the host said.
struct Rows {
  int row, count, past;        // first row, rows, position of the first
};
__device__ __forceinline__ Rows rows_of(const KvParams& p, int seq) {
  Rows r;
  const int lo = max(p.first[seq], 0), hi = min(max(p.first[seq + 1], 0), p.tokens);      // (hi - lo fits 32 bits)
  r.row = lo;
  r.count = max(hi - lo, 0);
  r.past = max(p.past[seq], 0);
  return r;
}
// (By value: a bit cast of a vector's element in place takes the vector's first.)
__device__ __forceinline__ uint32_t bits_of(_Float16 v) { return __builtin_bit_cast(uint16_t, v); }
__device__ __forceinline__ _Float16 half_of(uint32_t bits) { return __builtin_bit_cast(_Float16, (uint16_t)bits); }

// Both kernels give a wavefront the keys of 32 positions of a head, or the values.  When writing, a lane has runs of eight channels: run
// `quarter` of every unit of 32 channels, of two places, 4 apart.  In memory that is 64 bytes of a row for each four lanes, which are also
// what a group's statistics need first; and both places' codes of a key lie side by side in the cache, so that keys
// pass through no LDS.
struct Seat {
  int quarter, place[2];       // place of run j in the block
  int lane;                    // of the layout's units: where its keys are
};
__device__ __forceinline__ Seat seat_of(int lane) {
  const int r = lane >> 2 & 3, eight = lane >> 4;
  return {lane & 3, {8 * eight + r, 8 * eight + r + 4}, 16 * (lane & 3) + 4 * eight + r};
}

// The block of this wavefront and its live places.
struct Span {
  int64_t row0;                // row of place 0
  int from, to;                // live places; from >= to: nothing to do
  int page, in_page;           // page number as the table has it (-1: beyond the table), block in the page
  bool whole;
};
__device__ __forceinline__ Span span_of(const KvParams& p) {
  const Rows rows = rows_of(p, blockIdx.z);
  const int64_t end = (int64_t)rows.past + rows.count, block = rows.past / kBlock + (int64_t)blockIdx.x;
  Span s = {rows.row + block * kBlock - rows.past, 0, 0, -1, 0, false};
  if (block * kBlock >= end || rows.count == 0) return s;
  s.from = (int)max(rows.past - block * kBlock, (int64_t)0);
  s.to = (int)min(end - block * kBlock, (int64_t)kBlock);
  s.whole = s.from == 0 && s.to == kBlock && !p.rows;
  const int col = (int)min(block, (int64_t)INT32_MAX) / p.page_blocks;
  s.in_page = (int)(block - (int64_t)col * p.page_blocks);
  const int page = p.table[(int64_t)blockIdx.z * p.table_pages + min(col, p.table_pages - 1)];
  s.page = col < p.table_pages ? page : -1;
  return s;
}
// Its keys or values; null where there is no page.
__device__ __forceinline__ char* base_of(const KvParams& p, const Span& s, int value) {
  if (s.page < 0 || s.page >= p.pages) return nullptr;
  return p.pool + (((int64_t)s.page * p.heads + blockIdx.y) * p.page_blocks + s.in_page) * p.block_bytes + (value ? p.value_offset : 0);
}

// What another of the four lanes that hold a unit's runs has: the next, or the one after.
__device__ __forceinline__ uint32_t other_lane(uint32_t v, bool two) {
  return two ? (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x4e, 0xf, 0xf, true) : (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0xb1, 0xf, 0xf, true);
}
// (By value: a conditional operator between an array's elements is one between their addresses, and keeps the array in memory.)
__device__ __forceinline__ uint32_t either(bool which, uint32_t a, uint32_t b) { return which ? a : b; }
// What lane k of the four holds.
__device__ __forceinline__ uint32_t of_lane(uint32_t v, int k) {
  return k == 0   ? (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x00, 0xf, 0xf, true)
         : k == 1 ? (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x55, 0xf, 0xf, true)
         : k == 2 ? (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0xaa, 0xf, 0xf, true)
                  : (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0xff, 0xf, 0xf, true);
}
__device__ __forceinline__ float of_lane(float v, int k) { return __builtin_bit_cast(float, of_lane(__builtin_bit_cast(uint32_t, v), k)); }
__device__ __forceinline__ uint32_t most_of(uint32_t a, uint32_t b) {        // of both 16-bit halves
  return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(ushort2v, a), __builtin_bit_cast(ushort2v, b)));
}
// (NaN if either is.)
__device__ __forceinline__ half2v most_of(half2v a, half2v b) { return __builtin_elementwise_maximum(a, b); }
__device__ __forceinline__ half2v least_of(half2v a, half2v b) { return __builtin_elementwise_minimum(a, b); }

// Correctly rounded n / d for a d of at most 11 bits, by its correctly rounded reciprocal: the quotient's error, which is exact, times the
// reciprocal is right to far less than the 2^-12 of a last place that such a quotient is away from the middle of two numbers.
__device__ __forceinline__ float divided(float n, float d, float reciprocal) {
  const float q = n * reciprocal;
  return fmaf(fmaf(-q, d, n), reciprocal, q);
}
__device__ __forceinline__ float reciprocal_of(float d) {                    // 0 for 0
  const float r = __builtin_amdgcn_rcpf(d);
  return d > 0.0f ? fmaf(fmaf(-d, r, 1.0f), r, r) : 0.0f;
}

// A group's scale and offset, ready for use.
struct Group {
  float scale, reciprocal, offset;
  _Float16 scale_bits, offset_bits;      // as stored
  bool bad;                              // it holds an infinity or a NaN
};
// With 8 bits the largest |x| as bits (infinities and NaNs come out on top); with 4 the largest -x and x (NaNs come through).
template <int BITS>
__device__ __forceinline__ Group group_of_ends(uint32_t magnitude, half2v ends) {
  Group g;
  g.bad = BITS == 8 ? magnitude >= 0x7c00u : !((float)ends[0] < __builtin_inff() && (float)ends[1] < __builtin_inff());
  const float range = BITS == 8 ? divided((float)half_of(magnitude), 127.0f, 1.0f / 127.0f) : divided((float)ends[1] + (float)ends[0], 15.0f, 1.0f / 15.0f);
  const auto down = __builtin_amdgcn_cvt_pkrtz(range, 0.0f);                 // towards zero
  const _Float16 scale = (_Float16)down[0];
  g.scale = g.bad ? 0.0f : (float)scale;
  g.reciprocal = reciprocal_of(g.scale);
  g.scale_bits = g.bad ? half_of(0x7e00u) : scale;
  g.offset_bits = g.bad ? (_Float16)0.0f : -ends[0];
  g.offset = (float)g.offset_bits;
  return g;
}
// A code in the low bits of a float's: adding 3 * 2^22 rounds to a whole number, to even.
// With 8 bits x / s, both of 11 bits, is either midway between two whole numbers or more than 2^-12.1 from it.  Rounded to
// 2^-13 (by adding 3 * 2^9) x times the reciprocal keeps its side of the middle, or is the middle: that saves the quotient's correction.
// With 4 bits x - z may have more bits than 11, and the quotient is worked out.
constexpr float kWhole = 12582912.0f, kGrid = 1536.0f;
template <int BITS>
__device__ __forceinline__ uint32_t code_of(_Float16 x, const Group& g) {
  const float least = BITS == 8 ? kWhole - 127.0f : kWhole, most = BITS == 8 ? kWhole + 127.0f : kWhole + 15.0f;
  const float u = BITS == 8 ? fmaf((float)x, g.reciprocal, kGrid) + (kWhole - kGrid) : divided((float)x - g.offset, g.scale, g.reciprocal) + kWhole;
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_fmed3f(u, least, most));
}
__device__ __forceinline__ uint32_t bytes_of(uint32_t a, uint32_t b, uint32_t c, uint32_t d) {       // their low bytes, a's lowest
  return __builtin_amdgcn_perm(__builtin_amdgcn_perm(d, c, 0x0c0c0400u), __builtin_amdgcn_perm(b, a, 0x0c0c0400u), 0x05040100u);
}

constexpr int kKvThreads = 128;          // two wavefronts: keys and values

// Writes the block of 32 positions that blockIdx.x counts from the one with the sequence's first new position, for one
// head.  Values are transposed on the way, through LDS; whole units leave together, 16 bytes a lane.  Of a block that holds others'
// positions too only the live places' codes are stored, to the byte.
// 4096 tokens of 64 heads of 128 channels, rows that are parts of a product's: 4 bits in groups of 32, 176 MB, 41 us, 4.3 TB/s
// (a copy of 75 MB that goes past the caches: 6.3), the vector units three quarters busy; one token of each of 16 sequences 6 us.
template <int BITS, int DC, int GU>
__global__ __launch_bounds__(kKvThreads) void lutgemm_kv_write_kernel(KvParams p) {
  constexpr int kCode = kBlock * DC * 4 * BITS;
  constexpr int kPitch = DC * 4 * BITS + 16;        // of a row of codes in LDS
  __shared__ __attribute__((aligned(16))) unsigned char codes[kBlock * kPitch];
  const int lane = threadIdx.x & 63, value = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const _Float16* source = static_cast<const _Float16*>(value ? p.v : p.k);
  const int64_t stride = value ? p.v_stride : p.k_stride;
  if (!source) return;
  const Span span = span_of(p);
  if (span.from >= span.to) return;
  const Seat seat = seat_of(lane);

  u32x4 x[DC][2];                                   // (on their way while the page table is looked up)
  bool live[2];
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    live[j] = seat.place[j] >= span.from && seat.place[j] < span.to;
    int64_t row = span.row0 + min(max(seat.place[j], span.from), span.to - 1);      // (a dead place's lane reads a live one's row)
    if (p.rows) {
      row = p.rows[row];
      live[j] = live[j] && row >= 0;
    }
    const u32x4* from = reinterpret_cast<const u32x4*>(source + row * stride + (int64_t)blockIdx.y * DC * 32 + seat.quarter * 8);
    if (!p.rows || row >= 0) {
#pragma unroll
      for (int c = 0; c < DC; ++c) x[c][j] = __builtin_nontemporal_load(from + c * 4);
    } else {
#pragma unroll
      for (int c = 0; c < DC; ++c) x[c][j] = (u32x4){0u, 0u, 0u, 0u};
    }
  }

  char* base = base_of(p, span, value);
  if (!base) return;
  // The groups' statistics, run j of group k in ends[2 k + j], which the four lanes of a row then share out: each works out the scales of every
  // fourth, stores them, and gives them to the others (all of it by every lane is 15.3 vector instructions a value where this is 13.6, 4 bits in groups of 32).
  constexpr int kGroups = BITS == 16 ? 0 : 2 * (DC / GU), kMine = (kGroups + 3) / 4;
  Group mine[kMine > 0 ? kMine : 1];
  if constexpr (BITS != 16) {
    uint32_t ends[4 * kMine];
#pragma unroll
    for (int k = 0; k < 4 * kMine; ++k) {
      if (k >= kGroups) {
        ends[k] = 0u;
        continue;
      }
      const int first = k / 2 * GU, j = k % 2;
      uint32_t magnitude = 0;
      half2v low = __builtin_bit_cast(half2v, x[first][j][0]), high = low;
#pragma unroll
      for (int c = first; c < first + GU; ++c) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const uint32_t w = x[c][j][i];
          if (BITS == 8) magnitude = most_of(magnitude, w & 0x7fff7fffu);
          if (BITS == 4) {
            low = least_of(low, __builtin_bit_cast(half2v, w));
            high = most_of(high, __builtin_bit_cast(half2v, w));
          }
        }
      }
      if constexpr (BITS == 8) {
        magnitude = max(magnitude & 0xffffu, magnitude >> 16);
        magnitude = max(magnitude, other_lane(magnitude, false));
        ends[k] = max(magnitude, other_lane(magnitude, true));
      } else {
        half2v e = {(_Float16)-__builtin_elementwise_minimum(low[0], low[1]), __builtin_elementwise_maximum(high[0], high[1])};
        e = most_of(e, __builtin_bit_cast(half2v, other_lane(__builtin_bit_cast(uint32_t, e), false)));
        e = most_of(e, __builtin_bit_cast(half2v, other_lane(__builtin_bit_cast(uint32_t, e), true)));
        ends[k] = __builtin_bit_cast(uint32_t, e);
      }
    }
    bool bad = false;
    _Float16* scales = reinterpret_cast<_Float16*>(base + kCode);
#pragma unroll
    for (int m = 0; m < kMine; ++m) {
      const uint32_t e = either(seat.quarter & 2, either(seat.quarter & 1, ends[4 * m + 3], ends[4 * m + 2]), either(seat.quarter & 1, ends[4 * m + 1], ends[4 * m]));
      mine[m] = group_of_ends<BITS>(e, __builtin_bit_cast(half2v, e));
      bad = bad || mine[m].bad;
      const int k = 4 * m + seat.quarter, j = k & 1;
      if (k >= kGroups || !either(j, live[1], live[0])) continue;
      _Float16* to = scales + (k >> 1) * (BITS == 8 ? 32 : 64);
      const int place = (int)either(j, seat.place[1], seat.place[0]);
      if (value) {
        to[place] = mine[m].scale_bits;
        if (BITS == 4) to[place + 32] = mine[m].offset_bits;
      } else if (BITS == 8) {
        to[seat.lane % 16 * 2 + j] = mine[m].scale_bits;
      } else {
        reinterpret_cast<uint32_t*>(to)[seat.lane % 16 * 2 + j] = bits_of(mine[m].scale_bits) | bits_of(mine[m].offset_bits) << 16;
      }
    }
    if (__any(bad)) {                                // codes of a group with an infinity or a NaN are zeros'
#pragma unroll
      for (int k = 0; k < kGroups; ++k) {
        const bool gone = of_lane(mine[k / 4].bad ? 1u : 0u, k % 4) != 0u;
#pragma unroll
        for (int c = k / 2 * GU; c < k / 2 * GU + GU; ++c) {
#pragma unroll
          for (int i = 0; i < 4; ++i) x[c][k % 2][i] = gone ? 0u : x[c][k % 2][i];
        }
      }
    }
  }
#pragma unroll
  for (int first = 0; first < DC; first += GU) {
    Group group[2];
    if constexpr (BITS != 16) {
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const int k = first / GU * 2 + j;
        group[j].scale = of_lane(mine[k / 4].scale, k % 4);
        group[j].reciprocal = of_lane(mine[k / 4].reciprocal, k % 4);
        group[j].offset = BITS == 4 ? of_lane(mine[k / 4].offset, k % 4) : 0.0f;
      }
    }
#pragma unroll
    for (int c = first; c < first + GU; ++c) {
      uint32_t words[2][4];                          // codes of the two runs: 4, 2 or 1 words (of values with 4 bits, two of a byte each)
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        if constexpr (BITS == 16) {
#pragma unroll
          for (int i = 0; i < 4; ++i) words[j][i] = x[c][j][i];
        } else {
          uint32_t u[8];
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const uint32_t w = x[c][j][i / 2];
            u[i] = code_of<BITS>(half_of(i % 2 ? w >> 16 : w & 0xffffu), group[j]);
          }
          if (BITS == 4 && !value) {
            words[j][0] = __builtin_amdgcn_perm(u[1] | u[3] << 4 | u[5] << 8 | u[7] << 12, u[0] | u[2] << 4 | u[4] << 8 | u[6] << 12, 0x05040100u);
          } else {
            words[j][0] = bytes_of(u[0], u[1], u[2], u[3]) ^ (BITS == 8 ? 0x80808080u : 0u);
            words[j][1] = bytes_of(u[4], u[5], u[6], u[7]) ^ (BITS == 8 ? 0x80808080u : 0u);
          }
          if (BITS == 4 && value) {                   // channels d and d + 16 share a byte: the lower ones' lane has both
#pragma unroll
            for (int i = 0; i < 2; ++i) words[j][i] = (words[j][i] & 0x0f0f0f0fu) | (other_lane(words[j][i], true) & 0x0f0f0f0fu) << 4;
          }
        }
      }
      if (value) {
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          unsigned char* to = codes + seat.place[j] * kPitch + c * 4 * BITS;
          if constexpr (BITS == 16) *reinterpret_cast<u32x4*>(to + seat.quarter * 16) = (u32x4){words[j][0], words[j][1], words[j][2], words[j][3]};
          if constexpr (BITS == 8) *reinterpret_cast<u32x2*>(to + seat.quarter * 8) = (u32x2){words[j][0], words[j][1]};
          if constexpr (BITS == 4)
            if (seat.quarter < 2) *reinterpret_cast<u32x2*>(to + seat.quarter * 8) = (u32x2){words[j][0], words[j][1]};
        }
      } else {
        char* to = base + (BITS == 16 ? (c * 128 + seat.lane) * 16 : (c * 64 + seat.lane) * 2 * BITS);
        if constexpr (BITS == 16) {
          if (live[0]) *reinterpret_cast<u32x4*>(to) = (u32x4){words[0][0], words[0][1], words[0][2], words[0][3]};
          if (live[1]) *reinterpret_cast<u32x4*>(to + 1024) = (u32x4){words[1][0], words[1][1], words[1][2], words[1][3]};
        } else if (span.whole) {
          if constexpr (BITS == 8) *reinterpret_cast<u32x4*>(to) = (u32x4){words[0][0], words[0][1], words[1][0], words[1][1]};
          if constexpr (BITS == 4) *reinterpret_cast<u32x2*>(to) = (u32x2){words[0][0], words[1][0]};
        } else {
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            if (!live[j]) continue;
            if constexpr (BITS == 8) *reinterpret_cast<u32x2*>(to + j * 8) = (u32x2){words[j][0], words[j][1]};
            if constexpr (BITS == 4) *reinterpret_cast<uint32_t*>(to + j * 4) = words[j][0];
          }
        }
      }
    }
  }
  if (!value) return;
  // Values: a lane has two channels, 16 apart, of eight places.  (The rows were written by this wavefront itself.)
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
  const int eight = lane >> 4, channel = lane & 15;
  const bool all = span.whole || (!p.rows && 8 * eight >= span.from && 8 * eight + 8 <= span.to);
  if (all) {
    const unsigned char* from = codes + 8 * eight * kPitch;
#pragma unroll
    for (int c = 0; c < DC; ++c) {
      if constexpr (BITS == 16) {
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          u32x4 w;
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const unsigned char* pair = from + 2 * i * kPitch + (c * 32 + j * 16 + channel) * 2;
            w[i] = *reinterpret_cast<const uint16_t*>(pair) | (uint32_t)*reinterpret_cast<const uint16_t*>(pair + kPitch) << 16;
          }
          *reinterpret_cast<u32x4*>(base + ((c * 2 + j) * 64 + lane) * 16) = w;
        }
      } else {
        constexpr int kWords = BITS / 2;
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < kWords; ++i) {
          const int e = 4 * (i & 1), at = c * 4 * BITS + i / 2 * 16 + channel;
          const unsigned char* b = from + e * kPitch + at;
          w[i] = BITS == 8 ? bytes_of(b[0], b[kPitch], b[2 * kPitch], b[3 * kPitch]) : bytes_of(b[0], b[2 * kPitch], b[kPitch], b[3 * kPitch]);
        }
        if constexpr (BITS == 8) *reinterpret_cast<u32x4*>(base + (c * 64 + lane) * 16) = (u32x4){w[0], w[1], w[2], w[3]};
        if constexpr (BITS == 4) *reinterpret_cast<u32x2*>(base + (c * 64 + lane) * 8) = (u32x2){w[0], w[1]};
      }
    }
  }
  if (span.whole) return;
#pragma unroll 1
  for (int e = 0; e < 8; ++e) {
    const int place = 8 * eight + e, byte = BITS == 4 ? (e & 4) + ((e & 1) << 1 | (e >> 1 & 1)) : e;
    if (all || place < span.from || place >= span.to || (p.rows && p.rows[span.row0 + place] < 0)) continue;
    const unsigned char* from = codes + place * kPitch + channel * (BITS == 16 ? 2 : 1);
    char* to = base + lane * (BITS == 4 ? 8 : 16) + byte * (BITS == 16 ? 2 : 1);
#pragma unroll
    for (int c = 0; c < DC; ++c) {
#pragma unroll
      for (int j = 0; j < (BITS == 4 ? 1 : 2); ++j) {
        const unsigned char* code = from + c * 4 * BITS + j * BITS * 2;
        if constexpr (BITS == 16)
          *reinterpret_cast<uint16_t*>(to + (c * 2 + j) * 1024) = *reinterpret_cast<const uint16_t*>(code);
        else
          to[c * 128 * BITS + j * 8] = (char)*code;
      }
    }
  }
}

// Two codes, each in the low byte of 16 bits, as the fp16 values 1024 + code.
__device__ __forceinline__ half2v above_1024(uint32_t codes) { return __builtin_bit_cast(half2v, codes | 0x64006400u); }
// Their values: one rounding each.
template <int BITS>
__device__ __forceinline__ uint32_t values_of(uint32_t codes, _Float16 scale, _Float16 offset) {
  const half2v s = {scale, scale}, o = {offset, offset}, zero = BITS == 8 ? half2v{(_Float16)1152.0f, (_Float16)1152.0f} : half2v{(_Float16)1024.0f, (_Float16)1024.0f};
  const half2v u = above_1024(codes) - zero;
  return __builtin_bit_cast(uint32_t, BITS == 8 ? u * s : __builtin_elementwise_fma(u, s, o));
}

// The reverse, with the same grid.  The half block passes through LDS as it is in the cache, codes and scales; an item is a run of eight
// channels of a live place, and neighbouring lanes have neighbouring runs: stores of whole rows, 256 bytes at 128
// channels (stores of 64 bytes a place, as the write's loads are, took 60 us where these take 39: 4096 rows of 64 heads of 128
// channels, 4 bits).  Rows that no cache keeps till they are read go past it (29.5 us, 5.9 TB/s).
template <int BITS, int DC, int GU, bool PAST>
__global__ __launch_bounds__(kKvThreads) void lutgemm_kv_read_kernel(KvParams p) {
  constexpr int kCode = kBlock * DC * 4 * BITS, kHalves = BITS == 16 ? 0 : (BITS == 8 ? 32 : 64) * (DC / GU);
  constexpr int kBytes = kCode + 2 * kHalves, kRuns = 4 * DC;
  __shared__ __attribute__((aligned(16))) unsigned char lds[2 * kBytes];
  const int lane = threadIdx.x & 63, value = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  _Float16* target = static_cast<_Float16*>(const_cast<void*>(value ? p.v : p.k));
  const int64_t stride = value ? p.v_stride : p.k_stride;
  if (!target) return;
  const Span span = span_of(p);
  if (span.from >= span.to) return;
  const char* base = base_of(p, span, value);
  unsigned char* half = lds + value * kBytes;
  if (base) {
    u32x4 piece[(kBytes / 16 + 63) / 64];
#pragma unroll
    for (int i = 0; i < (int)(sizeof(piece) / 16); ++i) {
      const int at = i * 64 + lane;
      if (at < kBytes / 16) piece[i] = reinterpret_cast<const u32x4*>(base)[at];
    }
#pragma unroll
    for (int i = 0; i < (int)(sizeof(piece) / 16); ++i) {
      const int at = i * 64 + lane;
      if (at < kBytes / 16) reinterpret_cast<u32x4*>(half)[at] = piece[i];
    }
  }
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
  const _Float16* scales = reinterpret_cast<const _Float16*>(half + kCode);
  const int first = (span.from >> 3) * 4 * kRuns, end = ((span.to + 7) >> 3) * 4 * kRuns;
#pragma unroll 4
  for (int item = first + lane; item < end; item += 64) {
    const int pair = item / kRuns, run = item % kRuns, c = run >> 2, quarter = run & 3, eight = pair >> 2, r = pair & 3;
    const int key_lane = 16 * quarter + pair;                                        // of a key's codes
    const int value_lane = 16 * eight + 8 * (quarter & 1), upper = quarter >> 1;     // of the first of eight values' codes
    u32x4 x[2] = {{0u, 0u, 0u, 0u}, {0u, 0u, 0u, 0u}};
    if (base) {
      if constexpr (BITS == 16) {
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          if (!value) {
            x[j] = *reinterpret_cast<const u32x4*>(half + ((c * 2 + j) * 64 + key_lane) * 16);
          } else {
            const unsigned char* from = half + ((c * 2 + upper) * 64 + value_lane) * 16 + j * 8 + r * 2;
#pragma unroll
            for (int i = 0; i < 4; ++i)
              x[j][i] = *reinterpret_cast<const uint16_t*>(from + 32 * i) | (uint32_t)*reinterpret_cast<const uint16_t*>(from + 32 * i + 16) << 16;
          }
        }
      } else {
        uint32_t pairs[2][4];                         // two codes in a word
        const unsigned char* from = half + (c * 64 + (value ? value_lane : key_lane)) * 2 * BITS;
        if (!value) {
          uint32_t w[BITS / 2];
          if constexpr (BITS == 8) *reinterpret_cast<u32x4*>(w) = *reinterpret_cast<const u32x4*>(from);
          if constexpr (BITS == 4) *reinterpret_cast<u32x2*>(w) = *reinterpret_cast<const u32x2*>(from);
#pragma unroll
          for (int j = 0; j < 2; ++j) {
#pragma unroll
            for (int i = 0; i < 4; ++i)
              pairs[j][i] = BITS == 8 ? __builtin_amdgcn_perm(0u, w[BITS == 8 ? 2 * j + i / 2 : 0], i % 2 ? 0x0c030c02u : 0x0c010c00u) : w[j] >> (4 * i) & 0x000f000fu;
          }
        } else {
          if (BITS == 8) from += upper * 8;
          const uint32_t b = BITS == 8 ? r : ((r & 1) << 1 | r >> 1), pick = b | 0x0c00u | (4 + b) << 16 | 0x0c000000u;
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const u32x2 one = *reinterpret_cast<const u32x2*>(from + 4 * BITS * i), two = *reinterpret_cast<const u32x2*>(from + 4 * BITS * i + 2 * BITS);
#pragma unroll
            for (int j = 0; j < 2; ++j) {
              pairs[j][i] = __builtin_amdgcn_perm(two[j], one[j], pick);
              if (BITS == 4) pairs[j][i] = pairs[j][i] >> (4 * upper) & 0x000f000fu;
            }
          }
        }
        const _Float16* of = scales + c / GU * (BITS == 8 ? 32 : 64);
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const int k = value ? 8 * eight + r + 4 * j : (BITS == 8 ? 1 : 2) * (pair * 2 + j);
          const _Float16 scale = of[k], offset = BITS == 4 ? of[k + (value ? 32 : 1)] : (_Float16)0;
#pragma unroll
          for (int i = 0; i < 4; ++i) x[j][i] = values_of<BITS>(pairs[j][i], scale, offset);
        }
      }
    }
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const int place = 8 * eight + r + 4 * j;
      u32x4* to = reinterpret_cast<u32x4*>(target + (span.row0 + place) * stride + (int64_t)blockIdx.y * DC * 32 + run * 8);
      if (place < span.from || place >= span.to) continue;
      if constexpr (PAST)
        __builtin_nontemporal_store(x[j], to);
      else
        *to = x[j];
    }
  }
}

enum Move { kWrite, kRead, kReadPast };          // the last: rows go past the caches

template <int BITS, int DC, int GU>
const void* kernel_of(Move move) {
  return move == kWrite  ? reinterpret_cast<const void*>(lutgemm_kv_write_kernel<BITS, DC, GU>)
         : move == kRead ? reinterpret_cast<const void*>(lutgemm_kv_read_kernel<BITS, DC, GU, false>)
                         : reinterpret_cast<const void*>(lutgemm_kv_read_kernel<BITS, DC, GU, true>);
}
template <int BITS, int DC>
const void* pick_group(Move move, int units) {
  if (BITS == 16 || units == DC) return kernel_of<BITS, DC, DC>(move);
  if constexpr (BITS != 16) {
    if (units == 1) return kernel_of<BITS, DC, 1>(move);
    if constexpr (DC % 2 == 0 && DC > 2) {
      if (units == 2) return kernel_of<BITS, DC, 2>(move);
    }
    if constexpr (DC == 6) {
      if (units == 3) return kernel_of<BITS, DC, 3>(move);
    }
    if constexpr (DC == 8) {
      if (units == 4) return kernel_of<BITS, DC, 4>(move);
    }
  }
  return nullptr;
}
template <int BITS>
const void* pick_kernel(Move move, int dim, int units) {
  switch (dim) {
    case 64: return pick_group<BITS, 2>(move, units);
    case 96: return pick_group<BITS, 3>(move, units);
    case 128: return pick_group<BITS, 4>(move, units);
    case 192: return pick_group<BITS, 6>(move, units);
    case 256: return pick_group<BITS, 8>(move, units);
    default: return nullptr;
  }
}

// Both directions: k and v are the rows' ends of the move.
int move_rows(bool write, const void* k, const void* v, const int32_t* rows, const lutgemm_kv_cache* cache, const lutgemm_kv_step* step,
              int64_t k_stride, int64_t v_stride, void* hip_stream) {
  int rc = check_cache(cache);
  if (rc == LUTGEMM_OK) rc = check_step(step);
  if (rc != LUTGEMM_OK) return rc;
  if ((!k && !v) || !aligned16(k) || !aligned16(v) || ((uintptr_t)rows & 3) != 0) return LUTGEMM_EINVAL;
  const int64_t row = (int64_t)cache->heads * cache->head_dim;
  if ((k && (k_stride < row || k_stride % 8 != 0)) || (v && (v_stride < row || v_stride % 8 != 0))) return LUTGEMM_EINVAL;
  if (step->tokens == 0 || step->most_tokens == 0) return LUTGEMM_OK;
  const int group = group_of(cache->head_dim, cache->bits, cache->group);
  KvParams p = {};
  p.k = k;
  p.v = v;
  p.rows = rows;
  p.pool = static_cast<char*>(cache->pool);
  p.first = step->first;
  p.past = step->past;
  p.table = step->table;
  p.k_stride = k_stride;
  p.v_stride = v_stride;
  p.pages = cache->pages;
  p.block_bytes = block_bytes(cache->head_dim, cache->bits, group);
  p.value_offset = p.block_bytes / 2;
  p.tokens = step->tokens;
  p.table_pages = step->table_pages;
  p.page_blocks = cache->page_tokens / kBlock;
  p.heads = cache->heads;
  const int most = step->most_tokens < step->tokens ? step->most_tokens : step->tokens;
  const int units = group / 32, d = cache->head_dim;
  const Move move = write ? kWrite : ((int64_t)step->tokens * row * 4 > kCacheBytes ? kReadPast : kRead);
  const void* kern = cache->bits == 16 ? pick_kernel<16>(move, d, units) : cache->bits == 8 ? pick_kernel<8>(move, d, units) : pick_kernel<4>(move, d, units);
  if (!kern) return LUTGEMM_EUNSUPPORTED;
  void* args[] = {&p};
  // positions past .. past + most - 1 touch at most this many blocks
  const dim3 grid((most + 2 * kBlock - 2) / kBlock, cache->heads, step->seqs);
  if (hipLaunchKernel(kern, grid, dim3(kKvThreads), args, 0, static_cast<hipStream_t>(hip_stream)) != hipSuccess) return LUTGEMM_EHIP;
  return LUTGEMM_OK;
}

}  // namespace

extern "C" {

int lutgemm_rope(const void* x, void* y, const int32_t* positions, const uint64_t* turns, int tokens, int heads, int head_dim,
                 int rot_dim, int64_t x_stride, int64_t y_stride, float amplitude, unsigned flags, void* hip_stream) {
  if (!x || !y || !positions || !turns || tokens < 0 || heads < 1 || head_dim < 2 || head_dim % 2 != 0 || rot_dim < 2 || rot_dim % 2 != 0 || rot_dim > head_dim)
    return LUTGEMM_EINVAL;
  if (x_stride < (int64_t)heads * head_dim || y_stride < (int64_t)heads * head_dim || (x == y && x_stride != y_stride)) return LUTGEMM_EINVAL;
  const bool f32 = (flags & LUTGEMM_Y_F32) != 0;
  const uintptr_t size = f32 ? 4 : 2;
  if (((uintptr_t)x | (uintptr_t)y) % size != 0 || ((uintptr_t)positions & 3) != 0 || ((uintptr_t)turns & 7) != 0) return LUTGEMM_EINVAL;
  if ((flags & ~(unsigned)(LUTGEMM_Y_F32 | LUTGEMM_ROPE_NEIGHBOURS | LUTGEMM_ROPE_TRANSPOSE)) != 0) return LUTGEMM_EUNSUPPORTED;
  if (head_dim > 512 || heads > 1 << 16) return LUTGEMM_EUNSUPPORTED;
  if (tokens == 0) return LUTGEMM_OK;
  RopeParams p = {};
  p.x = x;
  p.y = y;
  p.positions = positions;
  p.turns = turns;
  p.x_stride = x_stride;
  p.y_stride = y_stride;
  p.tokens = tokens;
  p.heads = heads;
  p.head_dim = head_dim;
  p.rot_dim = rot_dim;
  p.amplitude = amplitude;
  p.sign = (flags & LUTGEMM_ROPE_TRANSPOSE) ? -1.0f : 1.0f;
  // Runs of 16 bytes where rows, heads and the halves of the turned part begin on 16 bytes, else single pairs.
  const int wide = (int)(16 / size);
  const bool vectors = aligned16(x) && aligned16(y) && x_stride % wide == 0 && y_stride % wide == 0 && head_dim % wide == 0 &&
                       rot_dim % (2 * wide) == 0 && (head_dim - rot_dim) % (2 * wide) == 0;
  const int pairs = vectors ? wide : 1;
  p.pair_runs = rot_dim / (2 * pairs);
  const int runs = x == y ? p.pair_runs : head_dim / (2 * pairs);
  const bool neighbours = (flags & LUTGEMM_ROPE_NEIGHBOURS) != 0;
  const bool past = (int64_t)tokens * heads * (x == y ? rot_dim : head_dim) * (int64_t)size > kCacheBytes;
  const void* kern = f32 ? pick_rope<float, 4>(vectors, neighbours, past) : pick_rope<_Float16, 8>(vectors, neighbours, past);
  // Heads a thread: the angles are worked out once for them, but only from half a million threads on, which fill the device.
  p.heads_a_thread = 1;
  while (p.heads_a_thread < 8 && p.heads_a_thread < heads && (int64_t)tokens * heads * runs / (2 * p.heads_a_thread) >= 1 << 19) p.heads_a_thread *= 2;
  int lanes = 256 / runs;                                             // heads side by side
  const int needed = (heads + p.heads_a_thread - 1) / p.heads_a_thread;
  lanes = lanes < 1 ? 1 : (lanes > needed ? needed : lanes);
  int side = 256 / (runs * lanes);                                    // tokens of a workgroup
  side = side < 1 ? 1 : (side > tokens ? tokens : (side > 64 ? 64 : side));
  const dim3 grid((tokens + side - 1) / side, (needed + lanes - 1) / lanes);
  void* args[] = {&p};
  if (hipLaunchKernel(kern, grid, dim3(runs, lanes, side), args, 0, static_cast<hipStream_t>(hip_stream)) != hipSuccess) return LUTGEMM_EHIP;
  return LUTGEMM_OK;
}

int lutgemm_kv_write(const void* k, const void* v, const int32_t* rows, const lutgemm_kv_cache* cache, const lutgemm_kv_step* step,
                     int64_t k_stride, int64_t v_stride, void* hip_stream) {
  return move_rows(true, k, v, rows, cache, step, k_stride, v_stride, hip_stream);
}

int lutgemm_kv_read(const lutgemm_kv_cache* cache, const lutgemm_kv_step* step, void* k, void* v, int64_t k_stride, int64_t v_stride,
                    void* hip_stream) {
  return move_rows(false, k, v, nullptr, cache, step, k_stride, v_stride, hip_stream);
}

}  // extern "C"
