// Where a step's tokens stand, from lengths that are in device memory: include/lutgemm.h has the rules.  A few words a token are
// written; the time is that of a launch and of the chain lengths -> prefix sums -> rows and pages: 16 sequences of a token 4.8 us, 96 prompts
// with 786432 rows, 16 bytes each, 9.8 and 3.3 for the second launch.
//
// A workgroup takes 4096 sequences at a time: four a thread, prefix sums of their tokens and pages by lane, wavefront and workgroup,
// whose ends stay in LDS.  Rows and pages are then dealt out evenly, and each looks up its sequence there.
#include <hip/hip_runtime.h>

#include "lutgemm_kv.h"
#include "lutgemm_step.h"

using namespace lutgemm_kv_detail;

namespace {

constexpr int kThreads = 1024, kEach = 4, kSeqs = kThreads * kEach;
constexpr int kAtOnce = 2;       // rows, or pages, that a thread works on together
constexpr int64_t kMostSum = 1 << 30;      // of rows, of pages: two such sums fit 32 bits

struct PlaceParams {
  int32_t* free;
  int32_t* count;
  int32_t* owned;
  int32_t* table;
  const int32_t* past;      // of trim: the lengths
  const int32_t* fresh;
  int32_t* first;
  int32_t* positions;
  int32_t* owner;
  int64_t* slots;
  int pages, page_tokens, seqs, table_pages, tokens, most_tokens;
};

// Sums of rows and of pages.  They stop at a bound just above what can be served (`most`), so that 32 bits hold any of them: below it they are
// exact, at it somebody waits, and they do not fall.
struct Pair {
  uint32_t rows, pages;
};
__device__ __forceinline__ Pair plus(Pair a, Pair b, Pair most) { return {min(a.rows + b.rows, most.rows), min(a.pages + b.pages, most.pages)}; }
// What a lane before this one has (in its row of 16, or the last of an earlier row), 0 where there is none.
template <int CTRL, int ROWS>
__device__ __forceinline__ Pair before_it(Pair v) {
  return {(uint32_t)__builtin_amdgcn_update_dpp(0, (int)v.rows, CTRL, ROWS, 0xf, false), (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v.pages, CTRL, ROWS, 0xf, false)};
}
__device__ __forceinline__ Pair row_sums(Pair v, Pair most) {      // over 16 lanes, this one included
  v = plus(v, before_it<0x111, 0xf>(v), most);
  v = plus(v, before_it<0x112, 0xf>(v), most);
  v = plus(v, before_it<0x114, 0xf>(v), most);
  return plus(v, before_it<0x118, 0xf>(v), most);
}
__device__ __forceinline__ Pair of_lane(Pair v, int lane) {
  return {(uint32_t)__builtin_amdgcn_readlane((int)v.rows, lane), (uint32_t)__builtin_amdgcn_readlane((int)v.pages, lane)};
}
// Over the workgroup: of the threads before this one, and of all.
struct Scan {
  Pair before, all;
};
__device__ __forceinline__ Scan scan_of(Pair mine, Pair most, Pair* sums) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  Pair in = row_sums(mine, most);
  in = plus(in, before_it<0x142, 0xa>(in), most);          // lane 15 of the row before, to rows 1 and 3
  in = plus(in, before_it<0x143, 0xc>(in), most);          // lane 31, to rows 2 and 3
  if (lane == 63) sums[wave] = in;
  const Pair earlier = before_it<0x138, 0xf>(in);          // (the lane before, of any row)
  __syncthreads();
  static_assert(kThreads / 64 == 16, "a row of lanes has the wavefronts' sums");
  const Pair waves = row_sums(sums[lane & 15], most);
  const Pair of_waves = of_lane(waves, max(wave - 1, 0));
  Scan s;
  s.before = plus(earlier, wave > 0 ? of_waves : Pair{0, 0}, most);
  s.all = of_lane(waves, 15);
  return s;
}

// The sequences that N items belong to: the first whose end is beyond each (below the last end).  Their searches go along together, as each is
// a chain of reads of LDS.
template <int N>
__device__ __forceinline__ void seqs_of(const uint32_t* ends, int count, const uint32_t* item, int* seq) {
#pragma unroll
  for (int u = 0; u < N; ++u) seq[u] = 0;
  for (int step = 1 << (31 - __builtin_clz(count)); step > 0; step >>= 1) {
#pragma unroll
    for (int u = 0; u < N; ++u) {
      const int next = seq[u] + step;
      if (next < count && ends[next - 1] <= item[u]) seq[u] = next;
    }
  }
}

__device__ __forceinline__ int pages_for(uint32_t positions, int page_tokens) { return (int)((positions + (uint32_t)page_tokens - 1) / (uint32_t)page_tokens); }

// FILL: writes rows and pages (any number of workgroups, which share them out); KEEP: what the calls keep, `owned` and `count` (one
// workgroup).  With one workgroup both at once; else a second launch keeps, as others may not have read yet what the first changes.
template <bool FILL, bool KEEP>
__global__ __launch_bounds__(kThreads) void lutgemm_kv_place_kernel(PlaceParams p) {
  __shared__ uint32_t ends[kSeqs], page_ends[kSeqs];
  __shared__ int32_t had[kSeqs], held[kSeqs];
  __shared__ Pair sums[kThreads / 64];
  __shared__ Pair stop;                // of all that are served
  __shared__ bool waits;
  const int tid = threadIdx.x;
  const uint32_t share = blockIdx.x * kThreads + tid, shares = gridDim.x * kThreads;
  const uint32_t free = (uint32_t)min(max(p.count[0], 0), p.pages);
  const Pair most = {(uint32_t)p.tokens + 1, free + 1};
  Pair before = {0, 0};                // of the sequences of earlier turns, served or not
  Pair served = {0, 0};
  bool over = false;                   // somebody waits: nobody behind is served
  for (int base = 0; base < p.seqs; base += kSeqs) {
    const int seqs = min(p.seqs - base, kSeqs);
    int32_t past[kEach], fresh[kEach], owned[kEach];
    Pair want[kEach], mine = {0, 0};
#pragma unroll
    for (int e = 0; e < kEach; ++e) {
      const int s = base + min(tid * kEach + e, seqs - 1);
      past[e] = p.past[s];
      fresh[e] = p.fresh[s];
      owned[e] = min(max(p.owned[s], 0), p.table_pages);
    }
#pragma unroll
    for (int e = 0; e < kEach; ++e) {
      const uint32_t end = (uint32_t)past[e] + (uint32_t)fresh[e];         // (of two that are not negative)
      const bool fits = tid * kEach + e < seqs && past[e] >= 0 && fresh[e] > 0 && fresh[e] <= p.most_tokens && end <= (uint32_t)(p.table_pages * p.page_tokens);
      want[e] = {fits ? (uint32_t)fresh[e] : 0u, fits ? (uint32_t)max(pages_for(end, p.page_tokens) - owned[e], 0) : 0u};
      mine = plus(mine, {min(want[e].rows, most.rows), want[e].pages}, most);
    }
    if (tid == 0) waits = false;
    const Scan scan = scan_of(mine, most, sums);         // (a barrier stands in it)
    Pair at = plus(before, scan.before, most);
    Pair to[kEach];
    bool ok[kEach];
#pragma unroll
    for (int e = 0; e < kEach; ++e) {
      const Pair from = at;
      const bool was = at.rows <= (uint32_t)p.tokens && at.pages <= free;
      at = plus(at, {min(want[e].rows, most.rows), want[e].pages}, most);
      to[e] = at;
      ok[e] = at.rows <= (uint32_t)p.tokens && at.pages <= free;
      if (was && !ok[e] && !over) {                      // (one thread's, as the sums do not fall)
        stop = from;
        waits = true;
      }
    }
    before = plus(before, scan.all, most);
    __syncthreads();
    const Pair start = served;
    if (!over) {
      over = waits;
      served = over ? stop : before;
    }
#pragma unroll
    for (int e = 0; e < kEach; ++e) {
      const int s = tid * kEach + e;
      if (s >= seqs) break;
      const Pair end = ok[e] ? to[e] : served;
      if (FILL) {
        ends[s] = end.rows;
        page_ends[s] = end.pages;
        had[s] = owned[e];
        held[s] = past[e];
        if (blockIdx.x == 0) p.first[base + s + 1] = (int32_t)end.rows;
      }
      if (KEEP && ok[e] && want[e].pages > 0) p.owned[base + s] = owned[e] + (int32_t)want[e].pages;
    }
    if (FILL) {
      __syncthreads();
      // (the last threads first: they have the fewest rows)
      for (uint32_t i0 = start.pages + (shares - 1 - share); i0 < served.pages; i0 += kAtOnce * shares) {
        uint32_t i[kAtOnce];
        int s[kAtOnce], page[kAtOnce];
#pragma unroll
        for (int u = 0; u < kAtOnce; ++u) i[u] = min(i0 + u * shares, served.pages - 1);
        seqs_of<kAtOnce>(page_ends, seqs, i, s);
#pragma unroll
        for (int u = 0; u < kAtOnce; ++u) page[u] = p.free[free - 1 - i[u]];
#pragma unroll
        for (int u = 0; u < kAtOnce; ++u) {
          const uint32_t first_page = s[u] == 0 ? start.pages : page_ends[s[u] - 1];
          if (i0 + u * shares < served.pages) p.table[(int64_t)(base + s[u]) * p.table_pages + had[s[u]] + (int)(i[u] - first_page)] = page[u];
        }
      }
      for (uint32_t i0 = start.rows + share; i0 < served.rows; i0 += kAtOnce * shares) {
        uint32_t i[kAtOnce], position[kAtOnce], col[kAtOnce];
        int s[kAtOnce], page[kAtOnce];
#pragma unroll
        for (int u = 0; u < kAtOnce; ++u) i[u] = min(i0 + u * shares, served.rows - 1);
        seqs_of<kAtOnce>(ends, seqs, i, s);
#pragma unroll
        for (int u = 0; u < kAtOnce; ++u) {
          position[u] = (uint32_t)held[s[u]] + (i[u] - (s[u] == 0 ? start.rows : ends[s[u] - 1]));
          if (p.slots) {
            col[u] = position[u] / (uint32_t)p.page_tokens;
            // (pages of this step straight from the stack: the table's entries may not be written yet)
            const uint32_t taken = (s[u] == 0 ? start.pages : page_ends[s[u] - 1]) + col[u] - (uint32_t)had[s[u]];
            const int32_t* at = (int)col[u] < had[s[u]] ? p.table + (int64_t)(base + s[u]) * p.table_pages + col[u] : p.free + (free - 1 - taken);
            page[u] = *at;
          }
        }
#pragma unroll
        for (int u = 0; u < kAtOnce; ++u) {
          if (i0 + u * shares >= served.rows) continue;
          if (p.positions) p.positions[i[u]] = (int32_t)position[u];
          if (p.owner) p.owner[i[u]] = base + s[u];
          if (p.slots) p.slots[i[u]] = page[u] < 0 || page[u] >= p.pages ? -1 : (int64_t)page[u] * p.page_tokens + (position[u] - col[u] * (uint32_t)p.page_tokens);
        }
      }
    }
    __syncthreads();
  }
  if (FILL) {
    if (share == 0) p.first[0] = 0;
    for (uint32_t i = served.rows + share; i < (uint32_t)p.tokens; i += shares) {
      if (p.positions) p.positions[i] = 0;
      if (p.owner) p.owner[i] = -1;
      if (p.slots) p.slots[i] = -1;
    }
  }
  if (KEEP && share == 0) p.count[0] = (int32_t)(free - served.pages);
}

// The reverse: pages beyond those that a sequence's positions take go back on the stack, the first of the first sequence on top: what a
// step took comes back in the order in which it would be taken again.
template <bool FILL, bool KEEP>
__global__ __launch_bounds__(kThreads) void lutgemm_kv_trim_kernel(PlaceParams p) {
  __shared__ uint32_t page_ends[kSeqs];
  __shared__ int32_t kept[kSeqs];
  __shared__ Pair sums[kThreads / 64];
  const int tid = threadIdx.x;
  const uint32_t share = blockIdx.x * kThreads + tid, shares = gridDim.x * kThreads;
  const uint32_t free = (uint32_t)min(max(p.count[0], 0), p.pages);
  const Pair most = {0, 1u << 31};     // (a table has 2^30 entries at most)
  // The first page's place on the stack needs the sum of all: a turn over the sequences for it where they do not fit one.
  uint32_t back = 0;
  for (int turn = p.seqs > kSeqs ? 0 : 1; turn < 2; ++turn) {
    uint32_t before = 0;
    for (int base = 0; base < p.seqs; base += kSeqs) {
      const int seqs = min(p.seqs - base, kSeqs);
      int32_t keep[kEach], give[kEach];
      Pair mine = {0, 0};
#pragma unroll
      for (int e = 0; e < kEach; ++e) {
        const int s = base + min(tid * kEach + e, seqs - 1);
        const int length = p.past[s], owned = min(max(p.owned[s], 0), p.table_pages);
        keep[e] = length < 0 ? owned : min(pages_for((uint32_t)length, p.page_tokens), owned);
        give[e] = tid * kEach + e < seqs ? owned - keep[e] : 0;
        mine.pages += (uint32_t)give[e];
      }
      const Scan scan = scan_of(mine, most, sums);
      const uint32_t all = scan.all.pages;
      if (turn == 0 || p.seqs <= kSeqs) back = before + all;
      if (turn == 1) {
        uint32_t at = scan.before.pages;
#pragma unroll
        for (int e = 0; e < kEach; ++e) {
          const int s = tid * kEach + e;
          at += (uint32_t)give[e];
          if (s >= seqs) break;
          if (FILL) {
            page_ends[s] = at;
            kept[s] = keep[e];
          }
          if (KEEP && give[e] > 0) p.owned[base + s] = keep[e];
        }
        if (FILL) {
          __syncthreads();
          for (uint32_t i0 = share; i0 < all; i0 += kAtOnce * shares) {
            uint32_t i[kAtOnce];
            int s[kAtOnce], page[kAtOnce];
            int32_t* entry[kAtOnce];
#pragma unroll
            for (int u = 0; u < kAtOnce; ++u) i[u] = min(i0 + u * shares, all - 1);
            seqs_of<kAtOnce>(page_ends, seqs, i, s);
#pragma unroll
            for (int u = 0; u < kAtOnce; ++u) {
              entry[u] = p.table + (int64_t)(base + s[u]) * p.table_pages + kept[s[u]] + (int)(i[u] - (s[u] == 0 ? 0 : page_ends[s[u] - 1]));
              page[u] = *entry[u];
            }
#pragma unroll
            for (int u = 0; u < kAtOnce; ++u) {
              if (i0 + u * shares >= all) continue;
              const int64_t place = (int64_t)free + back - 1 - ((int64_t)before + i[u]);
              if (place < p.pages) p.free[place] = page[u];
              *entry[u] = -1;
            }
          }
        }
      }
      before += all;
      __syncthreads();
    }
  }
  if (KEEP && share == 0) p.count[0] = (int32_t)min((int64_t)free + back, (int64_t)p.pages);
}

__global__ __launch_bounds__(256) void lutgemm_kv_pages_init_kernel(PlaceParams p) {
  const int64_t share = (int64_t)blockIdx.x * 256 + threadIdx.x, shares = (int64_t)gridDim.x * 256;
  for (int64_t i = share; i < p.pages; i += shares) p.free[i] = (int32_t)(p.pages - 1 - i);
  for (int64_t i = share; i < (int64_t)p.seqs * p.table_pages; i += shares) p.table[i] = -1;
  for (int64_t i = share; i < p.seqs; i += shares) p.owned[i] = 0;
  if (share == 0) p.count[0] = p.pages;
}

int check_pages(const lutgemm_kv_pages* g) {
  if (!g || !g->free || !g->count || !g->owned || !g->table) return LUTGEMM_EINVAL;
  if ((((uintptr_t)g->free | (uintptr_t)g->count | (uintptr_t)g->owned | (uintptr_t)g->table) & 3) != 0) return LUTGEMM_EINVAL;
  if (g->pages < 1 || g->page_tokens < kBlock || g->page_tokens % kBlock != 0 || g->seqs < 1 || g->table_pages < 1) return LUTGEMM_EINVAL;
  if (g->pages > kMostSum || g->page_tokens > 1 << 20 || g->seqs > kMostSeqs) return LUTGEMM_EUNSUPPORTED;
  if ((int64_t)g->table_pages * g->page_tokens > kMostHeld || (int64_t)g->table_pages * g->seqs > kMostSum) return LUTGEMM_EUNSUPPORTED;
  return LUTGEMM_OK;
}
PlaceParams params_of(const lutgemm_kv_pages* g) {
  PlaceParams p = {};
  p.free = g->free;
  p.count = g->count;
  p.owned = g->owned;
  p.table = g->table;
  p.pages = (int)g->pages;
  p.page_tokens = g->page_tokens;
  p.seqs = g->seqs;
  p.table_pages = g->table_pages;
  return p;
}
int launch(const void* kern, int groups, int threads, PlaceParams* p, void* stream) {
  void* args[] = {p};
  return hipLaunchKernel(kern, dim3(groups), dim3(threads), args, 0, static_cast<hipStream_t>(stream)) == hipSuccess ? LUTGEMM_OK : LUTGEMM_EHIP;
}

// One workgroup where it has few rows (or pages, of which most calls move far fewer than the most that there can be), as the second launch costs
// more; else as many as have a row a thread (8000 rows of 1000 sequences: 13.4 us in one, 8.9 in three, 7.2 in seven, and 3.3 for the second launch).
int groups_for(int64_t items, int64_t alone) { return (int)(items <= alone ? 1 : (items / kThreads < 256 ? items / kThreads : 256)); }

}  // namespace

extern "C" {

int lutgemm_kv_pages_init(const lutgemm_kv_pages* pages, void* hip_stream) {
  const int rc = check_pages(pages);
  if (rc != LUTGEMM_OK) return rc;
  PlaceParams p = params_of(pages);
  return launch(reinterpret_cast<const void*>(lutgemm_kv_pages_init_kernel), 256, 256, &p, hip_stream);
}

int lutgemm_kv_place(const lutgemm_kv_pages* pages, const int32_t* past, const int32_t* fresh, int tokens, int most_tokens, int32_t* first,
                     int32_t* positions, int32_t* owner, int64_t* slots, void* hip_stream) {
  const int rc = check_pages(pages);
  if (rc != LUTGEMM_OK) return rc;
  if (!past || !fresh || !first || tokens < 0 || most_tokens < 0) return LUTGEMM_EINVAL;
  if ((((uintptr_t)past | (uintptr_t)fresh | (uintptr_t)first | (uintptr_t)positions | (uintptr_t)owner) & 3) != 0 || ((uintptr_t)slots & 7) != 0)
    return LUTGEMM_EINVAL;
  if (tokens > kMostSum) return LUTGEMM_EUNSUPPORTED;
  PlaceParams p = params_of(pages);
  p.past = past;
  p.fresh = fresh;
  p.first = first;
  p.positions = positions;
  p.owner = owner;
  p.slots = slots;
  p.tokens = tokens;
  p.most_tokens = most_tokens;
  const int groups = groups_for(tokens, 4096);
  if (groups == 1) return launch(reinterpret_cast<const void*>(lutgemm_kv_place_kernel<true, true>), 1, kThreads, &p, hip_stream);
  const int filled = launch(reinterpret_cast<const void*>(lutgemm_kv_place_kernel<true, false>), groups, kThreads, &p, hip_stream);
  return filled != LUTGEMM_OK ? filled : launch(reinterpret_cast<const void*>(lutgemm_kv_place_kernel<false, true>), 1, kThreads, &p, hip_stream);
}

int lutgemm_kv_trim(const lutgemm_kv_pages* pages, const int32_t* lengths, void* hip_stream) {
  const int rc = check_pages(pages);
  if (rc != LUTGEMM_OK) return rc;
  if (!lengths || ((uintptr_t)lengths & 3) != 0) return LUTGEMM_EINVAL;
  PlaceParams p = params_of(pages);
  p.past = lengths;
  const int64_t items = (int64_t)p.seqs * p.table_pages;
  const int groups = groups_for(items < p.pages ? items : p.pages, 32768);
  if (groups == 1) return launch(reinterpret_cast<const void*>(lutgemm_kv_trim_kernel<true, true>), 1, kThreads, &p, hip_stream);
  const int filled = launch(reinterpret_cast<const void*>(lutgemm_kv_trim_kernel<true, false>), groups, kThreads, &p, hip_stream);
  return filled != LUTGEMM_OK ? filled : launch(reinterpret_cast<const void*>(lutgemm_kv_trim_kernel<false, true>), 1, kThreads, &p, hip_stream);
}

}  // extern "C"
