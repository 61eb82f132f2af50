// Where a step's tokens stand, from lengths that are in device memory: include/lutgemm.h has the rules.  A few words a token are
// written; the time is that of a launch and of the chain lengths -> prefix sums -> rows and pages.
//
// A workgroup takes 4096 sequences at a time: four a thread, prefix sums of their tokens and pages by lane, wavefront and workgroup,
// whose ends stay in LDS.  Rows and pages are then dealt out evenly, and each looks up its sequence there.
#include <hip/hip_runtime.h>

#include "lutgemm_kv.h"
#include "lutgemm_step.h"

using namespace lutgemm_kv_detail;

namespace {

constexpr int kThreads = 1024, kEach = 4, kSeqs = kThreads * kEach;

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

// Sums over the workgroup of what each thread has, before it and of all; both fit 63 bits (65535 sequences, 31 bits each).
struct Pair {
  int64_t rows, pages;
};
struct Scan {
  Pair before, all;
};
__device__ __forceinline__ Scan scan_of(Pair mine, Pair* sums) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  Pair in = mine;
#pragma unroll
  for (int d = 1; d < 64; d *= 2) {
    const int64_t r = __shfl_up(in.rows, d), g = __shfl_up(in.pages, d);
    if (lane >= d) in.rows += r, in.pages += g;
  }
  if (lane == 63) sums[wave] = in;
  __syncthreads();
  Scan s = {{in.rows - mine.rows, in.pages - mine.pages}, {0, 0}};
#pragma unroll
  for (int w = 0; w < kThreads / 64; ++w) {
    const Pair t = sums[w];
    if (w < wave) s.before.rows += t.rows, s.before.pages += t.pages;
    s.all.rows += t.rows, s.all.pages += t.pages;
  }
  return s;
}

// The sequence that item i belongs to: the first whose end is beyond it.
__device__ __forceinline__ int seq_of(const int32_t* ends, int count, int i) {
  int lo = 0, hi = count - 1;          // (i is below the last end)
  while (lo < hi) {
    const int mid = (lo + hi) >> 1;
    if (ends[mid] > i)
      hi = mid;
    else
      lo = mid + 1;
  }
  return lo;
}

__device__ __forceinline__ int pages_for(int64_t positions, int page_tokens) { return (int)((positions + page_tokens - 1) / page_tokens); }

// FILL: writes rows and pages (any number of workgroups, which share them out); KEEP: what the calls keep, `owned` and `count` (one
// workgroup).  With one workgroup both at once; else a second launch keeps, as others may not have read yet what the first changes.
template <bool FILL, bool KEEP>
__global__ __launch_bounds__(kThreads) void lutgemm_kv_place_kernel(PlaceParams p) {
  __shared__ int32_t ends[kSeqs], page_ends[kSeqs], had[kSeqs];
  __shared__ Pair sums[kThreads / 64];
  __shared__ Pair stop;                // of all that are served
  const int tid = threadIdx.x, share = blockIdx.x * kThreads + tid, shares = gridDim.x * kThreads;
  const int64_t free = min(max(p.count[0], 0), p.pages);
  Pair before = {0, 0};                // of the sequences of earlier turns, served or not
  Pair served = {0, 0};
  bool over = false;                   // somebody waits: nobody behind is served
  for (int base = 0; base < p.seqs; base += kSeqs) {
    const int seqs = min(p.seqs - base, kSeqs);
    int32_t past[kEach], want[kEach], need[kEach], owned[kEach];
    Pair mine = {0, 0};
#pragma unroll
    for (int e = 0; e < kEach; ++e) {
      const int s = base + min(tid * kEach + e, seqs - 1);
      past[e] = p.past[s];
      want[e] = p.fresh[s];
      owned[e] = min(max(p.owned[s], 0), p.table_pages);
    }
#pragma unroll
    for (int e = 0; e < kEach; ++e) {
      const int64_t end = (int64_t)past[e] + want[e];
      const bool fits = tid * kEach + e < seqs && past[e] >= 0 && want[e] > 0 && want[e] <= p.most_tokens && end <= (int64_t)p.table_pages * p.page_tokens;
      want[e] = fits ? want[e] : 0;
      need[e] = fits ? max(pages_for(end, p.page_tokens) - owned[e], 0) : 0;
      mine.rows += want[e];
      mine.pages += need[e];
    }
    if (tid == 0) stop = {-1, 0};
    const Scan scan = scan_of(mine, sums);               // (a barrier stands in it)
    Pair at = {before.rows + scan.before.rows, before.pages + scan.before.pages};
    bool ok[kEach];
#pragma unroll
    for (int e = 0; e < kEach; ++e) {
      const bool was = at.rows <= p.tokens && at.pages <= free;
      const Pair from = at;
      at.rows += want[e];
      at.pages += need[e];
      ok[e] = at.rows <= p.tokens && at.pages <= free;
      if (was && !ok[e] && !over) stop = from;           // (one thread's, as the sums do not fall)
    }
    before.rows += scan.all.rows;
    before.pages += scan.all.pages;
    __syncthreads();
    const Pair start = served;
    if (!over) {
      over = stop.rows >= 0;
      served = over ? stop : before;
    }
    at = {before.rows - scan.all.rows + scan.before.rows, before.pages - scan.all.pages + scan.before.pages};
#pragma unroll
    for (int e = 0; e < kEach; ++e) {
      const int s = tid * kEach + e;
      at.rows += want[e];
      at.pages += need[e];
      if (s >= seqs) break;
      const int32_t end = (int32_t)(ok[e] ? at.rows : served.rows), page_end = (int32_t)(ok[e] ? at.pages : served.pages);
      if (FILL) {
        ends[s] = end;
        page_ends[s] = page_end;
        had[s] = owned[e];
        if (blockIdx.x == 0) p.first[base + s + 1] = end;
      }
      if (KEEP && ok[e] && need[e] > 0) p.owned[base + s] = owned[e] + need[e];
    }
    if (FILL) {
      __syncthreads();
      for (int64_t i = start.pages + share; i < served.pages; i += shares) {
        const int s = seq_of(page_ends, seqs, (int)i);
        const int first_page = s == 0 ? (int)start.pages : page_ends[s - 1];
        p.table[(int64_t)(base + s) * p.table_pages + had[s] + ((int)i - first_page)] = p.free[free - 1 - i];
      }
      for (int64_t i = start.rows + share; i < served.rows; i += shares) {
        const int s = seq_of(ends, seqs, (int)i);
        const int first_row = s == 0 ? (int)start.rows : ends[s - 1], first_page = s == 0 ? (int)start.pages : page_ends[s - 1];
        const int position = p.past[base + s] + ((int)i - first_row);
        if (p.positions) p.positions[i] = position;
        if (p.owner) p.owner[i] = base + s;
        if (p.slots) {
          const int col = position / p.page_tokens;
          // (pages of this step straight from the stack: the table's entries may not be written yet)
          const int page = col < had[s] ? p.table[(int64_t)(base + s) * p.table_pages + col] : p.free[free - 1 - (first_page + col - had[s])];
          p.slots[i] = page < 0 || page >= p.pages ? -1 : (int64_t)page * p.page_tokens + position % p.page_tokens;
        }
      }
    }
    __syncthreads();
  }
  if (FILL) {
    if (share == 0) p.first[0] = 0;
    for (int64_t i = served.rows + share; i < p.tokens; i += shares) {
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
  __shared__ int32_t page_ends[kSeqs], kept[kSeqs];
  __shared__ Pair sums[kThreads / 64];
  const int tid = threadIdx.x, share = blockIdx.x * kThreads + tid, shares = gridDim.x * kThreads;
  const int64_t free = min(max(p.count[0], 0), p.pages);
  // The first page's place on the stack needs the sum of all: a turn over the sequences for it where they do not fit one.
  int64_t back = 0;
  for (int turn = p.seqs > kSeqs ? 0 : 1; turn < 2; ++turn) {
    int64_t before = 0;
    for (int base = 0; base < p.seqs; base += kSeqs) {
      const int seqs = min(p.seqs - base, kSeqs);
      int32_t keep[kEach], give[kEach];
      Pair mine = {0, 0};
#pragma unroll
      for (int e = 0; e < kEach; ++e) {
        const int s = base + min(tid * kEach + e, seqs - 1);
        const int length = p.past[s], owned = min(max(p.owned[s], 0), p.table_pages);
        keep[e] = length < 0 ? owned : min(pages_for(length, p.page_tokens), owned);
        give[e] = tid * kEach + e < seqs ? owned - keep[e] : 0;
        mine.pages += give[e];
      }
      const Scan scan = scan_of(mine, sums);
      if (turn == 0 || p.seqs <= kSeqs) back = before + scan.all.pages;
      if (turn == 1) {
        int64_t at = before + scan.before.pages;
#pragma unroll
        for (int e = 0; e < kEach; ++e) {
          const int s = tid * kEach + e;
          at += give[e];
          if (s >= seqs) break;
          if (FILL) {
            page_ends[s] = (int32_t)(at - before);
            kept[s] = keep[e];
          }
          if (KEEP && give[e] > 0) p.owned[base + s] = keep[e];
        }
        if (FILL) {
          __syncthreads();
          for (int64_t i = share; i < scan.all.pages; i += shares) {
            const int s = seq_of(page_ends, seqs, (int)i);
            int32_t* entry = p.table + (int64_t)(base + s) * p.table_pages + kept[s] + ((int)i - (s == 0 ? 0 : page_ends[s - 1]));
            const int64_t place = free + back - 1 - (before + i);
            if (place < p.pages) p.free[place] = *entry;
            *entry = -1;
          }
        }
      }
      before += scan.all.pages;
      __syncthreads();
    }
  }
  if (KEEP && share == 0) p.count[0] = (int32_t)min(free + back, (int64_t)p.pages);
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
  if (g->pages > INT32_MAX || g->page_tokens > 1 << 20 || g->seqs > kMostSeqs) return LUTGEMM_EUNSUPPORTED;
  if ((int64_t)g->table_pages * g->page_tokens > kMostHeld) return LUTGEMM_EUNSUPPORTED;
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

// Rows (or pages to be moved) that one workgroup does by itself.
constexpr int64_t kAlone = 16384;
int groups_for(int64_t items) { return (int)(items <= kAlone ? 1 : (items / 4096 < 256 ? items / 4096 : 256)); }

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
  PlaceParams p = params_of(pages);
  p.past = past;
  p.fresh = fresh;
  p.first = first;
  p.positions = positions;
  p.owner = owner;
  p.slots = slots;
  p.tokens = tokens;
  p.most_tokens = most_tokens;
  const int groups = groups_for(tokens);
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
  const int groups = groups_for(items < p.pages ? items : p.pages);
  if (groups == 1) return launch(reinterpret_cast<const void*>(lutgemm_kv_trim_kernel<true, true>), 1, kThreads, &p, hip_stream);
  const int filled = launch(reinterpret_cast<const void*>(lutgemm_kv_trim_kernel<true, false>), groups, kThreads, &p, hip_stream);
  return filled != LUTGEMM_OK ? filled : launch(reinterpret_cast<const void*>(lutgemm_kv_trim_kernel<false, true>), 1, kThreads, &p, hip_stream);
}

}  // extern "C"
