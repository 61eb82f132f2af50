// The residual's addition and the root-mean-square norm in front of a product: include/lutgemm.h has the formulas.
//
// A workgroup owns a row and holds it in registers between the two things that are done with it, so that every value
// is read once: s = x + r, the sum of squares (in 64 bits: squares of fp32 values leave 32), then s * inv * w.  What bounds it is
// HBM: 4096 rows of 12288 channels, 403 MB, 68.4 us, 5.9 TB/s (a copy past the caches: 6.3); of few rows the launch and one chain of
// load, sum and store (3.4 us for one).  Rows that begin anywhere: 4096 of 12289 channels 91 us (280 value by value).  The next row on its way during a row's sum (512 workgroups that stay) was no faster: 75 to 79 us.
#include <hip/hip_fp16.h>
#include <hip/hip_runtime.h>

#include "lutgemm_step.h"

#ifndef LUT_PART
#error "compiled once per part, -DLUT_PART=0 .. 3: x in fp16 or fp32 (1), the residual stream in fp16 or fp32 (2)"
#endif

namespace lutgemm_norm_parts {

struct Params {
  const void* x;
  const void* residual;        // null: nothing is added
  const _Float16* weight;      // null: ones
  void* sum;                   // null: not kept
  void* y;
  float* scales;               // null: y is fp16
  int64_t x_stride, stream_stride, y_stride;
  int n, group, groups;
  float eps;
  bool past;                   // outputs go past the caches: there is more of them than they hold
};

typedef const void* (*Family)(int threads, int runs, bool wide, bool bytes);
const void* family0(int threads, int runs, bool wide, bool bytes);
const void* family1(int threads, int runs, bool wide, bool bytes);
const void* family2(int threads, int runs, bool wide, bool bytes);
const void* family3(int threads, int runs, bool wide, bool bytes);

}  // namespace lutgemm_norm_parts

namespace {

using lutgemm_norm_parts::Params;

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

typedef uint32_t Loose __attribute__((ext_vector_type(4), aligned(2)));      // 16 bytes that begin on any value's

constexpr int kRun = 8;      // channels that a thread has next to each other

// Eight values as they are in memory, 16 bytes at a time; those of a row that begins anywhere (not WIDE) too, with the compiler's
// instructions for that; of a row of fewer as many as there are.
template <typename T>
struct Eight {
  u32x4 part[sizeof(T) * kRun / 16];
  template <bool WIDE>
  __device__ __forceinline__ void load(const T* p, int n) {
    if (WIDE) {
#pragma unroll
      for (unsigned i = 0; i < sizeof(part) / 16; ++i) part[i] = reinterpret_cast<const u32x4*>(p)[i];
    } else {
      if (n >= kRun) {
#pragma unroll
        for (unsigned i = 0; i < sizeof(part) / 16; ++i) part[i] = reinterpret_cast<const Loose*>(p)[i];
      } else {
        constexpr int kEach = 16 / sizeof(T);
        typedef T Values __attribute__((ext_vector_type(kEach)));
#pragma unroll
        for (unsigned i = 0; i < sizeof(part) / 16; ++i) {
          Values t;
#pragma unroll
          for (int e = 0; e < kEach; ++e) t[e] = p[min((int)(kEach * i) + e, n - 1)];
          part[i] = __builtin_bit_cast(u32x4, t);
        }
      }
    }
  }
  __device__ __forceinline__ float value(int e) const { return (float)reinterpret_cast<const T*>(part)[e]; }
};
template <typename T>
__device__ __forceinline__ void store_wide(T* p, const float* v, bool past) {
  T t[kRun];
#pragma unroll
  for (int e = 0; e < kRun; ++e) t[e] = (T)v[e];
#pragma unroll
  for (unsigned i = 0; i < sizeof(t) / 16; ++i) {
    if (past)
      __builtin_nontemporal_store(reinterpret_cast<const u32x4*>(t)[i], reinterpret_cast<u32x4*>(p) + i);
    else
      reinterpret_cast<u32x4*>(p)[i] = reinterpret_cast<const u32x4*>(t)[i];
  }
}
template <int COUNT = kRun, typename T>
__device__ __forceinline__ void store_any(T* p, const float* v) {
  T t[COUNT];
#pragma unroll
  for (int e = 0; e < COUNT; ++e) t[e] = (T)v[e];
  __builtin_memcpy(p, t, sizeof t);
}

// A thread's runs are eight channels next to each other.  WIDE: rows begin on 16 bytes and are whole runs; else they begin anywhere and
// have any length: the last run is read from the row's last eight channels, and those that the run before it has are left out.
template <typename X, typename S, bool BYTES, bool WIDE, int THREADS, int RUNS>
__global__ __launch_bounds__(THREADS) void lutgemm_rms_norm_kernel(Params p) {
  constexpr int kWaves = THREADS / 64;
  extern __shared__ uint32_t tops[];               // of every group: the largest |y|, as bits
  __shared__ double squares[kWaves];
  const int tid = threadIdx.x;
  auto channel = [&](int run) { return (run * THREADS + tid) * kRun; };
  // (Loads have no branches: beyond the row's end they repeat its last eight channels.)
  auto place = [&](int run) { return WIDE ? min(channel(run), p.n - kRun) : max(min(channel(run), p.n - kRun), 0); };
  auto has = [&](int run, int e) { return WIDE ? channel(run) < p.n : place(run) + e >= channel(run) && place(run) + e < p.n; };
  auto keep = [&](int run, const float* v, auto* row, bool past) {
    const int c = channel(run);
    if (WIDE) {
      if (c < p.n) store_wide(row + c, v, past);
    } else if (c + kRun <= p.n) {
      store_any(row + c, v);
    } else if (c < p.n) {
#pragma unroll
      for (int e = 0; e < kRun; ++e)
        if (has(run, e)) store_any<1>(row + place(run) + e, v + e);
    }
  };

  Eight<_Float16> w[RUNS];
  if (p.weight) {
#pragma unroll
    for (int k = 0; k < RUNS; ++k) w[k].template load<WIDE>(p.weight + place(k), p.n);
  }
  Eight<X> x[RUNS];
  Eight<S> r[RUNS];
  const int64_t row = blockIdx.x;
#pragma unroll
  for (int k = 0; k < RUNS; ++k) x[k].template load<WIDE>(static_cast<const X*>(p.x) + row * p.x_stride + place(k), p.n);
  if (p.residual) {
#pragma unroll
    for (int k = 0; k < RUNS; ++k) r[k].template load<WIDE>(static_cast<const S*>(p.residual) + row * p.stream_stride + place(k), p.n);
  }
  float v[RUNS][kRun];
#pragma unroll
  for (int k = 0; k < RUNS; ++k)
#pragma unroll
    for (int e = 0; e < kRun; ++e) {
      v[k][e] = x[k].value(e);
      if (p.residual) v[k][e] += r[k].value(e);
      v[k][e] = has(k, e) ? v[k][e] : 0.0f;
    }
  if (BYTES) {
    for (int g = tid; g < p.groups; g += THREADS) tops[g] = 0;
  }
  double square = 0.0;
#pragma unroll
  for (int k = 0; k < RUNS; ++k)
#pragma unroll
    for (int e = 0; e < kRun; ++e) square = fma((double)v[k][e], (double)v[k][e], square);
  if (p.sum) {
    S* sum = static_cast<S*>(p.sum) + row * p.stream_stride;
#pragma unroll
    for (int k = 0; k < RUNS; ++k) keep(k, v[k], sum, p.past);
  }
#pragma unroll
  for (int d = 1; d < 64; d *= 2) square += __shfl_xor(square, d);
  if ((tid & 63) == 0) squares[tid >> 6] = square;
  __syncthreads();
  double total = 0.0;
#pragma unroll
  for (int k = 0; k < kWaves; ++k) total += squares[k];
  const float inv = (float)(1.0 / sqrt(total / (double)p.n + (double)p.eps));
#pragma unroll
  for (int k = 0; k < RUNS; ++k) {
#pragma unroll
    for (int e = 0; e < kRun; ++e) v[k][e] = v[k][e] * inv * (p.weight ? w[k].value(e) : 1.0f);
  }

  if constexpr (!BYTES) {
    _Float16* y = static_cast<_Float16*>(p.y) + row * p.y_stride;
#pragma unroll
    for (int k = 0; k < RUNS; ++k) keep(k, v[k], y, p.past);
  } else {
    int8_t* y = static_cast<int8_t*>(p.y) + row * p.y_stride;
#pragma unroll
    for (int k = 0; k < RUNS; ++k) {
      uint32_t top = 0;                            // (as bits: infinities and NaNs come out on top)
#pragma unroll
      for (int e = 0; e < kRun; ++e) top = has(k, e) ? max(top, __builtin_bit_cast(uint32_t, v[k][e]) & 0x7fffffffu) : top;
      top = max(top, (uint32_t)__shfl_xor((int)top, 1));
      top = max(top, (uint32_t)__shfl_xor((int)top, 2));         // of 32 channels, which are of one group: a group has 32 channels' multiple, or all
      if ((tid & 3) == 0 && channel(k) < p.n) atomicMax(&tops[(uint32_t)channel(k) / (uint32_t)p.group], top);
    }
    __syncthreads();
    for (int g = tid; g < p.groups; g += THREADS) {
      const float top = __builtin_bit_cast(float, tops[g]);
      p.scales[row * p.groups + g] = !(top < __builtin_inff()) ? __builtin_nanf("") : (top < 0x1p-100f ? 0.0f : top / 127.0f);
    }
#pragma unroll
    for (int k = 0; k < RUNS; ++k) {
      // (a group's codes: none where it has an infinity or a NaN, or nothing that is a number's worth)
      auto per = [&](uint32_t bits) {
        const float top = __builtin_bit_cast(float, bits);
        return top < __builtin_inff() && !(top < 0x1p-100f) ? 127.0f / top : 0.0f;
      };
      auto code = [&](float value, float per) { return per == 0.0f ? 0 : (int)rintf(value * per); };
      const int c = channel(k);
      if (c >= p.n) continue;
      const float steps = per(tops[(uint32_t)c / (uint32_t)p.group]);
      if (WIDE || c + kRun <= p.n) {
        uint32_t word[2] = {0, 0};
#pragma unroll
        for (int e = 0; e < kRun; ++e) word[e / 4] |= ((uint32_t)code(v[k][e], steps) & 0xffu) << (8 * (e % 4));
        if (WIDE)
          *reinterpret_cast<u32x2*>(y + c) = (u32x2){word[0], word[1]};
        else
          __builtin_memcpy(y + c, word, sizeof word);
      } else {
#pragma unroll
        for (int e = 0; e < kRun; ++e)
          if (has(k, e)) y[place(k) + e] = (int8_t)code(v[k][e], steps);
      }
    }
  }
}

template <typename X, typename S, bool BYTES, bool WIDE>
const void* pick(int threads, int runs) {
#define CASE(t, r) \
  if (threads == t && runs == r) return reinterpret_cast<const void*>(lutgemm_rms_norm_kernel<X, S, BYTES, WIDE, t, r>);
  CASE(64, 1) CASE(64, 2) CASE(64, 4) CASE(256, 2) CASE(256, 3) CASE(256, 4) CASE(512, 3) CASE(512, 4) CASE(1024, 3) CASE(1024, 4)
  if constexpr (BYTES) {                           // few rows, over more threads
    CASE(256, 1) CASE(1024, 1) CASE(1024, 2)
  }
#undef CASE
  return nullptr;
}
template <typename X, typename S>
const void* pick(int threads, int runs, bool wide, bool bytes) {
  return wide ? (bytes ? pick<X, S, true, true>(threads, runs) : pick<X, S, false, true>(threads, runs))
              : (bytes ? pick<X, S, true, false>(threads, runs) : pick<X, S, false, false>(threads, runs));
}

}  // namespace

namespace lutgemm_norm_parts {
#if LUT_PART == 0
const void* family0(int threads, int runs, bool wide, bool bytes) { return pick<_Float16, _Float16>(threads, runs, wide, bytes); }
#elif LUT_PART == 1
const void* family1(int threads, int runs, bool wide, bool bytes) { return pick<float, _Float16>(threads, runs, wide, bytes); }
#elif LUT_PART == 2
const void* family2(int threads, int runs, bool wide, bool bytes) { return pick<_Float16, float>(threads, runs, wide, bytes); }
#else
const void* family3(int threads, int runs, bool wide, bool bytes) { return pick<float, float>(threads, runs, wide, bytes); }
#endif
}  // namespace lutgemm_norm_parts

#if LUT_PART == 0
extern "C" int lutgemm_rms_norm(const void* x, const void* residual, const void* weight, void* sum, void* y, float* scales, int tokens, int n,
                                int group, int64_t x_stride, int64_t stream_stride, int64_t y_stride, float eps, unsigned flags, void* hip_stream) {
  using namespace lutgemm_norm_parts;
  using namespace lutgemm_step_detail;
  if (!x || !y || tokens < 0 || n < 1 || x_stride < n || y_stride < n || !(eps > 0.0f) || !(eps < __builtin_inff())) return LUTGEMM_EINVAL;
  if (group < 0 || (!scales && group != 0)) return LUTGEMM_EINVAL;
  if ((residual || sum) && stream_stride < n) return LUTGEMM_EINVAL;
  if ((flags & ~(unsigned)(LUTGEMM_Y_F32 | LUTGEMM_NORM_STREAM_F32)) != 0) return LUTGEMM_EUNSUPPORTED;
  const int64_t xs = flags & LUTGEMM_Y_F32 ? 4 : 2, ss = flags & LUTGEMM_NORM_STREAM_F32 ? 4 : 2, ys = scales ? 1 : 2;
  if ((uintptr_t)x % xs != 0 || ((uintptr_t)residual | (uintptr_t)sum) % ss != 0 || (uintptr_t)y % ys != 0 || (uintptr_t)weight % 2 != 0 ||
      (uintptr_t)scales % 4 != 0)
    return LUTGEMM_EINVAL;
  if (scales && group != 0 && n % group != 0) return LUTGEMM_EINVAL;
  if (n > 32768 || tokens > 1 << 21 || (scales && group % 32 != 0)) return LUTGEMM_EUNSUPPORTED;   // (a grid has less than 2^32 threads)
  if (tokens == 0) return LUTGEMM_OK;
  const int64_t most_stride = (int64_t)1 << 28;          // (so that offsets in bytes stay within 64 bits)
  if (x_stride > most_stride || y_stride > most_stride || ((residual || sum) && stream_stride > most_stride)) return LUTGEMM_EUNSUPPORTED;
  const Rows x_rows = rows_of(x, tokens, x_stride, n, xs), y_rows = rows_of(y, tokens, y_stride, n, ys), weight_rows = rows_of(weight, 1, n, n, 2);
  const Rows residual_rows = rows_of(residual, tokens, stream_stride, n, ss), sum_rows = rows_of(sum, tokens, stream_stride, n, ss);
  auto clash = [](const Rows& in, const Rows& out) { return !apart(in, out) && !same_rows(in, out); };
  if (clash(x_rows, y_rows) || (residual && clash(residual_rows, y_rows)) || (weight && !apart(weight_rows, y_rows))) return LUTGEMM_EINVAL;
  if (sum && (clash(x_rows, sum_rows) || (residual && clash(residual_rows, sum_rows)) || (weight && !apart(weight_rows, sum_rows)) || !apart(sum_rows, y_rows)))
    return LUTGEMM_EINVAL;
  if (scales) {
    const int64_t all = (int64_t)tokens * (group == 0 ? 1 : n / group);
    const Rows scale_rows = rows_of(scales, 1, all, all, 4);
    if (!apart(x_rows, scale_rows) || (residual && !apart(residual_rows, scale_rows)) || (weight && !apart(weight_rows, scale_rows)) ||
        (sum && !apart(sum_rows, scale_rows)) || !apart(y_rows, scale_rows))
      return LUTGEMM_EINVAL;
  }
  Params p = {};
  p.x = x;
  p.residual = residual;
  p.weight = static_cast<const _Float16*>(weight);
  p.sum = sum;
  p.y = y;
  p.scales = scales;
  p.x_stride = x_stride;
  p.stream_stride = stream_stride;
  p.y_stride = y_stride;
  p.n = n;
  p.group = group == 0 ? n : group;
  p.groups = n / p.group;
  p.eps = eps;
  auto rows16 = [&](const void* a, int64_t stride, int64_t size) { return ((uintptr_t)a | (uintptr_t)(stride * size)) % 16 == 0; };
  const bool bytes = scales != nullptr;
  const bool wide = n % (bytes ? 32 : 8) == 0 && rows16(x, x_stride, xs) && (!residual || rows16(residual, stream_stride, ss)) &&
                    (!sum || rows16(sum, stream_stride, ss)) && (uintptr_t)weight % 16 == 0 &&
                    (bytes ? ((uintptr_t)y | (uintptr_t)y_stride) % 8 == 0 : rows16(y, y_stride, 2));
  const int units = (n + 7) / 8;
  // Threads enough for four runs each; more where there are few rows to 8 bits.  Groups of 128, an fp32 stream, us with a run a thread
  // and with four: 64 rows of 8192 channels 5.2 and 5.8, 509 10.7 and 12.8, 1024 19.9 and 21.0, 4096 64.2 and 66.4; of 2048 channels 3.6 and 4.9,
  // 5.0 and 6.3, 7.0 and 8.6, 19.0 and 20.6: less and less, but nowhere the other way round.  (To fp16, rows that begin anywhere: 300 of 5003
  // 6.6 with more threads and 5.3 with 256, 1000 12.4 and 9.3.)
  const bool spread = tokens <= 1024 && bytes;
  const int threads = spread ? (units <= 64 ? 64 : (units <= 256 ? 256 : 1024)) : (units <= 256 ? 64 : (units <= 1024 ? 256 : (units <= 2048 ? 512 : 1024)));
  int runs = (units + threads - 1) / threads;
  if (threads == 64 && runs == 3) runs = 4;
  // (4096 rows, fp16: 5120 channels 25.3 us so and 30.8 by way of the caches, 12288 68.7 and 70.9)
  p.past = (int64_t)tokens * n * ((sum ? ss : 0) + ys) > kCacheBytes;
  static const Family families[4] = {family0, family1, family2, family3};
  const void* kern = families[(xs == 4 ? 1 : 0) + (ss == 4 ? 2 : 0)](threads, runs, wide, bytes);
  void* args[] = {&p};
  if (hipLaunchKernel(kern, dim3(tokens), dim3(threads), args, bytes ? 4 * (size_t)p.groups : 0, static_cast<hipStream_t>(hip_stream)) != hipSuccess)
    return LUTGEMM_EHIP;
  return LUTGEMM_OK;
}
#endif
