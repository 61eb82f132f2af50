// Rotary positions, and the key/value cache as it is written and read back: include/lutgemm.h has the formulas and the
// layout.  All three move data and compute next to nothing, so what bounds them is HBM, and for a few tokens the
// launch and one trip to memory.
#include <hip/hip_fp16.h>
#include <hip/hip_runtime.h>

#include <type_traits>

#include "lutgemm_kv.h"

using namespace lutgemm_kv_detail;

namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef _Float16 half8 __attribute__((ext_vector_type(8)));

bool aligned16(const void* p) { return ((uintptr_t)p & 15) == 0; }

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
  int whole;           // nothing is left to copy: y is x
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
template <typename T, int N>
__device__ __forceinline__ void store_run(T* p, const Run<T, N>& r) {
  if constexpr (N * sizeof(T) >= 16) {
    const u32x4* s = reinterpret_cast<const u32x4*>(&r);
    u32x4* d = reinterpret_cast<u32x4*>(p);
#pragma unroll
    for (unsigned i = 0; i < N * sizeof(T) / 16; ++i) d[i] = s[i];
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i) p[i] = r.v[i];
  }
}

// A thread owns a run of PAIRS pairs (threadIdx.x) of one token for some heads, so that the angles, which no table holds, are worked
// out once for them: 64-bit position * frequency, one sine and cosine.  Runs behind the pairs' copy
// what is not turned, 2 PAIRS channels each.
template <typename T, int PAIRS, bool NEIGHBOURS>
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
    store_run<T, PAIRS>(y + at + a, u);
    store_run<T, PAIRS>(y + at + b, v);
  }
}

template <typename T, int PAIRS>
const void* pick_rope(bool neighbours) {
  return neighbours ? reinterpret_cast<const void*>(lutgemm_rope_kernel<T, PAIRS, true>)
                    : reinterpret_cast<const void*>(lutgemm_rope_kernel<T, PAIRS, false>);
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
  int tokens, seqs, table_pages, page_blocks, heads, group;
};

struct Codes8 {                // eight values of a run: the bytes of a piece of the layout
  uint32_t w[4];               // 16 bits: all; 8 bits: two; 4 bits: one (keys), or one nibble a byte in two (values)
};

// Where the tokens of a sequence are, checked against what the host said.
struct Rows {
  int row, count, past;        // first row, rows, position of the first
};
__device__ __forceinline__ Rows rows_of(const KvParams& p, int seq) {
  Rows r;
  const int lo = max(p.first[seq], 0), hi = min(p.first[seq + 1], p.tokens);
  r.row = lo;
  r.count = max(hi - lo, 0);
  r.past = max(p.past[seq], 0);
  return r;
}
// The block that holds positions 32 * block .. of a sequence for a head; null where there is none.
__device__ __forceinline__ char* block_at(const KvParams& p, int seq, int block, int head) {
  const int col = block / p.page_blocks;
  if (col >= p.table_pages) return nullptr;
  const int page = p.table[(int64_t)seq * p.table_pages + col];
  if (page < 0 || page >= p.pages) return nullptr;
  return p.pool + (((int64_t)page * p.heads + head) * p.page_blocks + (block - col * p.page_blocks)) * p.block_bytes;
}

// Lane, run and place of a value in the layout's units.
__device__ __forceinline__ int key_lane(int place, int g) { return 16 * g + 4 * (place >> 3) + (place & 3); }
__device__ __forceinline__ int key_run(int place) { return (place >> 2) & 1; }

// Byte of a key piece (eight channels of one place, unit c, quarter g) within the key codes.
template <int BITS>
__device__ __forceinline__ int key_piece(int place, int c, int g) {
  const int lane = key_lane(place, g), j = key_run(place);
  return BITS == 16 ? ((c * 2 + j) * 64 + lane) * 16 : ((c * 64 + lane) * 2 + j) * BITS;
}
// Byte of one value code (channel d of a place; with 4 bits of channels d and d + 16, d % 32 < 16).
template <int BITS>
__device__ __forceinline__ int value_byte(int place, int d) {
  const int c = d >> 5, j = (d >> 4) & 1, lane = 16 * (place >> 3) + (d & 15), e = place & 7;
  if (BITS == 16) return (((c * 2 + j) * 64 + lane) * 8 + e) * 2;
  if (BITS == 8) return ((c * 64 + lane) * 2 + j) * 8 + e;
  return (c * 64 + lane) * 8 + (e & 4) + (((e & 1) << 1) | ((e >> 1) & 1));   // 0 2 1 3
}
// Half word of a scale (the offset's, with 4 bits: 1 behind for keys, 32 for values).
template <int BITS>
__device__ __forceinline__ int key_scale(int group, int place) {
  return (BITS == 8 ? 1 : 2) * (group * 32 + (4 * (place >> 3) + (place & 3)) * 2 + key_run(place));
}
template <int BITS>
__device__ __forceinline__ int value_scale(int group, int place) {
  return (BITS == 8 ? 32 : 64) * group + place;
}

// (By value: a bit cast of a vector's element in place takes the vector's first.)
__device__ __forceinline__ uint32_t bits_of(_Float16 v) { return __builtin_bit_cast(uint16_t, v); }

// What a run of eight values adds to its group's statistics.
struct Stats {
  uint32_t magnitude;          // largest bits of |x|: infinities and NaNs come out on top
  _Float16 low, high;
};
__device__ __forceinline__ Stats stats_of(const half8 x) {
  Stats s = {0u, x[0], x[0]};
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    s.magnitude = max(s.magnitude, bits_of(x[i]) & 0x7fffu);
    s.low = x[i] < s.low ? x[i] : s.low;
    s.high = x[i] > s.high ? x[i] : s.high;
  }
  return s;
}
__device__ __forceinline__ Stats joined(Stats a, Stats b) {
  a.magnitude = max(a.magnitude, b.magnitude);
  a.low = b.low < a.low ? b.low : a.low;
  a.high = b.high > a.high ? b.high : a.high;
  return a;
}
// A group's scale and offset.  fp32 division is IEEE's here, as it is in what checks it.
template <int BITS>
__device__ __forceinline__ void scale_of_group(Stats s, _Float16* scale, _Float16* offset) {
  const float range = BITS == 8 ? (float)__builtin_bit_cast(_Float16, (uint16_t)s.magnitude) / 127.0f : ((float)s.high - (float)s.low) / 15.0f;
  const auto down = __builtin_amdgcn_cvt_pkrtz(range, 0.0f);   // towards zero
  const bool bad = s.magnitude >= 0x7c00u;
  *scale = bad ? __builtin_bit_cast(_Float16, (uint16_t)0x7e00u) : (_Float16)down[0];
  *offset = s.low;
}
template <int BITS>
__device__ __forceinline__ uint32_t code_of(_Float16 x, float scale, float offset) {
  if (BITS == 8) {
    const float u = scale > 0.0f ? rintf((float)x / scale) : 0.0f;
    return (uint32_t)((int)fminf(fmaxf(u, -127.0f), 127.0f) + 128);
  }
  const float u = scale > 0.0f ? rintf(((float)x - offset) / scale) : 0.0f;
  return (uint32_t)(int)fminf(fmaxf(u, 0.0f), 15.0f);
}
template <int BITS>
__device__ __forceinline__ _Float16 value_of(uint32_t code, _Float16 scale, _Float16 offset) {
  if (BITS == 8) return scale * (_Float16)(int)(code - 128);              // one rounding each
  return __builtin_elementwise_fma(scale, (_Float16)(int)code, offset);
}

constexpr int kKvThreads = 256;

// Writes the block of 32 positions that blockIdx.x counts from the one with the sequence's first new position, for one
// head.  An item is a run of eight channels of one place, of the key or of the value; what quantising needs of the
// whole group goes through LDS.  Codes are put together in LDS in the layout's order and copied out 16 or 8 bytes a
// thread: values are transposed on the way, and whole lines leave together.
template <int BITS, int DIM>
__global__ __launch_bounds__(kKvThreads) void lutgemm_kv_write_kernel(KvParams p) {
  constexpr int kRuns = DIM / 8;                    // of a place
  constexpr int kItems = 2 * kBlock * kRuns;
  constexpr int kEach = (kItems + kKvThreads - 1) / kKvThreads;
  constexpr int kCode = kBlock * DIM * BITS / 8;
  __shared__ __attribute__((aligned(16))) unsigned char codes[2 * kCode];
  __shared__ Stats stats[BITS == 16 ? 1 : kItems];
  const int seq = blockIdx.z, head = blockIdx.y;
  const Rows rows = rows_of(p, seq);
  const int64_t end = (int64_t)rows.past + rows.count;
  const int64_t block = rows.past / kBlock + (int64_t)blockIdx.x;
  if (block * kBlock >= end || rows.count == 0 || block > INT32_MAX) return;
  char* base = block_at(p, seq, (int)block, head);
  if (!base) return;
  const int from = (int)max(rows.past - block * kBlock, (int64_t)0), to = (int)min(end - block * kBlock, (int64_t)kBlock);   // live places
  const int64_t row0 = rows.row + block * kBlock - rows.past;   // of place 0

  half8 x[kEach];
  bool live[kEach];
#pragma unroll
  for (int k = 0; k < kEach; ++k) {
    const int item = threadIdx.x + k * kKvThreads;
    const int value = item / (kBlock * kRuns), place = item / kRuns % kBlock, run = item % kRuns;
    live[k] = item < kItems && place >= from && place < to && (value ? p.v : p.k) != nullptr;
    int64_t row = row0 + place;
    if (live[k] && p.rows) {
      row = p.rows[row];
      live[k] = row >= 0;
    }
    const half8 none = {0, 0, 0, 0, 0, 0, 0, 0};
    x[k] = none;
    if (live[k])
      x[k] = *reinterpret_cast<const half8*>(static_cast<const _Float16*>(value ? p.v : p.k) + row * (value ? p.v_stride : p.k_stride) +
                                             (int64_t)head * DIM + run * 8);
    if (BITS != 16 && item < kItems) stats[item] = stats_of(x[k]);
  }
  if (BITS != 16) __syncthreads();
#pragma unroll
  for (int k = 0; k < kEach; ++k) {
    const int item = threadIdx.x + k * kKvThreads;
    const int value = item / (kBlock * kRuns), place = item / kRuns % kBlock, run = item % kRuns;
    if (!live[k]) continue;
    uint32_t u[8];
    if constexpr (BITS != 16) {
      const int runs = p.group / 8, g0 = run / runs * runs;
      Stats s = stats[item - run + g0];
      for (int i = 1; i < runs; ++i) s = joined(s, stats[item - run + g0 + i]);
      _Float16 scale, offset;
      scale_of_group<BITS>(s, &scale, &offset);
      if (run == g0) {
        _Float16* scales = reinterpret_cast<_Float16*>(base + (value ? p.value_offset : 0) + kCode);
        const int at = value ? value_scale<BITS>(run / runs, place) : key_scale<BITS>(run / runs, place);
        scales[at] = scale;
        if (BITS == 4) scales[at + (value ? 32 : 1)] = offset;
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) u[i] = code_of<BITS>(x[k][i], (float)scale, (float)offset);
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) u[i] = bits_of(x[k][i]);
    }
    unsigned char* to_lds = codes + value * kCode;
    if (!value) {
      uint32_t* w = reinterpret_cast<uint32_t*>(to_lds + key_piece<BITS>(place, run >> 2, run & 3));
      if constexpr (BITS == 16) {
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = u[2 * i] | (u[2 * i + 1] << 16);
      } else if constexpr (BITS == 8) {
        w[0] = u[0] | (u[1] << 8) | (u[2] << 16) | (u[3] << 24);
        w[1] = u[4] | (u[5] << 8) | (u[6] << 16) | (u[7] << 24);
      } else {
        w[0] = u[0] | (u[2] << 4) | (u[4] << 8) | (u[6] << 12) | (u[1] << 16) | (u[3] << 20) | (u[5] << 24) | (u[7] << 28);
      }
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int d = run * 8 + i;
        unsigned char* b = to_lds + value_byte<BITS>(place, d);
        if constexpr (BITS == 16) *reinterpret_cast<uint16_t*>(b) = (uint16_t)u[i];
        if constexpr (BITS == 8) *b = (unsigned char)u[i];
        // 4 bits: channels d and d + 16 share a byte: the lower ones' thread writes it, once it has both
        if constexpr (BITS == 4) {
          const uint32_t other = (uint32_t)__shfl_xor((int)u[i], 2, 64);   // run ^ 2: the channel 16 away
          if ((run & 2) == 0) *b = (unsigned char)(u[i] | (other << 4));
        }
      }
    }
  }
  __syncthreads();
  // Pieces of eight values: of one place (keys), of places 8 g .. 8 g + 7 (values).
  constexpr int kPiece = BITS == 16 ? 16 : 8;      // bytes; with 4 bits two key places, or a byte for two channels
  constexpr int kPieces = kCode / kPiece;
  for (int i = threadIdx.x; i < 2 * kPieces; i += kKvThreads) {
    const int value = i / kPieces, piece = i % kPieces;
    if ((value ? p.v : p.k) == nullptr) continue;
    const unsigned char* src = codes + value * kCode + piece * kPiece;
    char* dst = base + (value ? p.value_offset : 0) + piece * kPiece;
    const int lane = BITS == 8 ? (piece >> 1) & 63 : piece & 63;
    if (p.rows == nullptr) {
      bool all, any;
      if (!value && BITS != 4) {
        const int j = BITS == 8 ? piece & 1 : (piece >> 6) & 1, place = 8 * ((lane >> 2) & 3) + 4 * j + (lane & 3);
        all = any = place >= from && place < to;
      } else {
        const int place = 8 * (value ? lane >> 4 : (lane >> 2) & 3);
        all = place >= from && place + 8 <= to;
        any = place + 8 > from && place < to;
      }
      if (!any) continue;
      if (all) {
        if constexpr (kPiece == 16)
          *reinterpret_cast<u32x4*>(dst) = *reinterpret_cast<const u32x4*>(src);
        else
          *reinterpret_cast<uint64_t*>(dst) = *reinterpret_cast<const uint64_t*>(src);
        continue;
      }
    }
    // a piece that others' positions share: only the live places
    if (!value) {
#pragma unroll
      for (int j = 0; j < (BITS == 4 ? 2 : 1); ++j) {
        const int run = BITS == 4 ? j : (BITS == 8 ? piece & 1 : (piece >> 6) & 1), place = 8 * ((lane >> 2) & 3) + 4 * run + (lane & 3);
        if (place < from || place >= to || (p.rows && p.rows[row0 + place] < 0)) continue;
        constexpr int kWords = BITS == 16 ? 4 : (BITS == 8 ? 2 : 1);
#pragma unroll
        for (int w = 0; w < kWords; ++w)
          reinterpret_cast<uint32_t*>(dst)[j + w] = reinterpret_cast<const uint32_t*>(src)[j + w];
      }
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int place = 8 * (lane >> 4) + e;
        if (place < from || place >= to || (p.rows && p.rows[row0 + place] < 0)) continue;
        if constexpr (BITS == 16) {
          reinterpret_cast<uint16_t*>(dst)[e] = reinterpret_cast<const uint16_t*>(src)[e];
        } else {
          const int byte = BITS == 8 ? e : (e & 4) + (((e & 1) << 1) | ((e >> 1) & 1));
          dst[byte] = (char)src[byte];
        }
      }
    }
  }
}

// The reverse, the same grid: codes of the block come whole into LDS, items leave as rows.
template <int BITS, int DIM>
__global__ __launch_bounds__(kKvThreads) void lutgemm_kv_read_kernel(KvParams p) {
  constexpr int kRuns = DIM / 8;
  constexpr int kItems = 2 * kBlock * kRuns;
  constexpr int kCode = kBlock * DIM * BITS / 8;
  __shared__ __attribute__((aligned(16))) unsigned char codes[2 * kCode];
  const int seq = blockIdx.z, head = blockIdx.y;
  const Rows rows = rows_of(p, seq);
  const int64_t end = (int64_t)rows.past + rows.count;
  const int64_t block = rows.past / kBlock + (int64_t)blockIdx.x;
  if (block * kBlock >= end || rows.count == 0) return;
  const char* base = block > INT32_MAX ? nullptr : block_at(p, seq, (int)block, head);
  const int from = (int)max(rows.past - block * kBlock, (int64_t)0), to = (int)min(end - block * kBlock, (int64_t)kBlock);
  const int64_t row0 = rows.row + block * kBlock - rows.past;
  if (base) {
    for (int i = threadIdx.x; i < 2 * kCode / 16; i += kKvThreads) {
      const int value = i / (kCode / 16), piece = i % (kCode / 16);
      reinterpret_cast<u32x4*>(codes)[i] = *reinterpret_cast<const u32x4*>(base + (value ? p.value_offset : 0) + piece * 16);
    }
  }
  __syncthreads();
  for (int item = threadIdx.x; item < kItems; item += kKvThreads) {
    const int value = item / (kBlock * kRuns), place = item / kRuns % kBlock, run = item % kRuns;
    void* out = const_cast<void*>(value ? p.v : p.k);
    if (place < from || place >= to || !out) continue;
    half8 x = {0, 0, 0, 0, 0, 0, 0, 0};
    if (base) {
      _Float16 scale = 0, offset = 0;
      if constexpr (BITS != 16) {
        const _Float16* scales = reinterpret_cast<const _Float16*>(base + (value ? p.value_offset : 0) + kCode);
        const int group = run / (p.group / 8), at = value ? value_scale<BITS>(group, place) : key_scale<BITS>(group, place);
        scale = scales[at];
        if (BITS == 4) offset = scales[at + (value ? 32 : 1)];
      }
      const unsigned char* src = codes + value * kCode;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        if (!value) {
          const unsigned char* b = src + key_piece<BITS>(place, run >> 2, run & 3);
          if constexpr (BITS == 16) x[i] = reinterpret_cast<const _Float16*>(b)[i];
          if constexpr (BITS == 8) x[i] = value_of<BITS>(b[i], scale, offset);
          if constexpr (BITS == 4) x[i] = value_of<BITS>(*reinterpret_cast<const uint32_t*>(b) >> (4 * (i / 2 + 4 * (i % 2))) & 15u, scale, offset);
        } else {
          const unsigned char* b = src + value_byte<BITS>(place, run * 8 + i);
          if constexpr (BITS == 16) x[i] = *reinterpret_cast<const _Float16*>(b);
          if constexpr (BITS == 8) x[i] = value_of<BITS>(*b, scale, offset);
          if constexpr (BITS == 4) x[i] = value_of<BITS>(*b >> (4 * ((run >> 1) & 1)) & 15u, scale, offset);
        }
      }
    }
    *reinterpret_cast<half8*>(static_cast<_Float16*>(out) + (row0 + place) * (value ? p.v_stride : p.k_stride) + (int64_t)head * DIM + run * 8) = x;
  }
}

template <int BITS>
const void* pick_write(int dim) {
  switch (dim) {
    case 64: return reinterpret_cast<const void*>(lutgemm_kv_write_kernel<BITS, 64>);
    case 96: return reinterpret_cast<const void*>(lutgemm_kv_write_kernel<BITS, 96>);
    case 128: return reinterpret_cast<const void*>(lutgemm_kv_write_kernel<BITS, 128>);
    case 192: return reinterpret_cast<const void*>(lutgemm_kv_write_kernel<BITS, 192>);
    default: return reinterpret_cast<const void*>(lutgemm_kv_write_kernel<BITS, 256>);
  }
}
template <int BITS>
const void* pick_read(int dim) {
  switch (dim) {
    case 64: return reinterpret_cast<const void*>(lutgemm_kv_read_kernel<BITS, 64>);
    case 96: return reinterpret_cast<const void*>(lutgemm_kv_read_kernel<BITS, 96>);
    case 128: return reinterpret_cast<const void*>(lutgemm_kv_read_kernel<BITS, 128>);
    case 192: return reinterpret_cast<const void*>(lutgemm_kv_read_kernel<BITS, 192>);
    default: return reinterpret_cast<const void*>(lutgemm_kv_read_kernel<BITS, 256>);
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
  if (cache->heads > 65535) return LUTGEMM_EUNSUPPORTED;
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
  p.seqs = step->seqs;
  p.table_pages = step->table_pages;
  p.page_blocks = cache->page_tokens / kBlock;
  p.heads = cache->heads;
  p.group = group;
  const int most = step->most_tokens < step->tokens ? step->most_tokens : step->tokens;
  const void* kern = write ? (cache->bits == 16 ? pick_write<16>(cache->head_dim) : cache->bits == 8 ? pick_write<8>(cache->head_dim) : pick_write<4>(cache->head_dim))
                           : (cache->bits == 16 ? pick_read<16>(cache->head_dim) : cache->bits == 8 ? pick_read<8>(cache->head_dim) : pick_read<4>(cache->head_dim));
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
  const void* kern = f32 ? (vectors ? pick_rope<float, 4>(neighbours) : pick_rope<float, 1>(neighbours))
                         : (vectors ? pick_rope<_Float16, 8>(neighbours) : pick_rope<_Float16, 1>(neighbours));
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
