// The pages of a pool on MI355X (gfx950): which sequences hold which pages
// from one step to the next, moving the live ones together, and copying them.
//
// All of it is integers in int32, decided by rules in which every page and row
// has one place (lowest first), so the results do not depend on the order in
// which workgroups run: counts are sums of atomic additions, "the lowest row"
// an atomic minimum, places come from prefix sums.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "pda_pages.h"

namespace pda {
namespace {

typedef unsigned u32x4 __attribute__((ext_vector_type(4)));
typedef int i32x4 __attribute__((ext_vector_type(4)));

constexpr int kThreads = 256;
constexpr int kScanThreads = 1024;

__device__ __forceinline__ int clamp_to(int x, int hi) { return x < 0 ? 0 : (x > hi ? hi : x); }

// A table entry as a page of the pool, or -1.
__device__ __forceinline__ int page_of(int id, int num_pages) {
  return static_cast<unsigned>(id) < static_cast<unsigned>(num_pages) ? id : -1;
}

// What row r of an update does: `kept` tokens of its parent's, `total` in all.
struct Row {
  const int32_t* from;  // the parent's table row (of no kept tokens where there is no parent)
  int kept, total;
  int full;      // pages wholly of kept tokens
  int first;     // first page without any kept token
  int pages;     // pages in all
  bool writes;   // it writes into page `full`, which holds kept tokens too
  int lo;        // first token its queries see under the window
};

__device__ __forceinline__ Row row_of(const PagesUpdateArgs& a, int r) {
  const int most = a.maxp << a.page_shift;
  const int b = a.parents ? a.parents[r] : r;
  const bool has = static_cast<unsigned>(b) < static_cast<unsigned>(a.batch);
  Row w;
  w.from = a.table + static_cast<int64_t>(has ? b : 0) * a.maxp;
  w.total = clamp_to(a.new_lens[r], most);
  const int len = has ? clamp_to(a.lens[b], most) : 0;
  w.kept = len < w.total ? len : w.total;
  const int page = 1 << a.page_shift;
  w.full = w.kept >> a.page_shift;
  w.first = (w.kept + page - 1) >> a.page_shift;
  w.pages = (w.total + page - 1) >> a.page_shift;
  w.writes = w.first > w.full && w.total > w.kept;
  const int64_t lo = static_cast<int64_t>(w.total) - a.nq + 1 - a.window;
  w.lo = a.window > 0 && lo > 0 ? static_cast<int>(lo) : 0;
  return w;
}

// Page j of a row, j < first: the parent's, or -1 where it holds none or no
// query of the row sees any of its tokens (past the sinks and before the
// window; a page with tokens yet to come is kept).
__device__ __forceinline__ int kept_page(const PagesUpdateArgs& a, const Row& w, int j) {
  const int64_t t = static_cast<int64_t>(j) << a.page_shift;
  return j < w.full && t >= a.sinks && t + (1 << a.page_shift) <= w.lo ? -1 : page_of(w.from[j], a.num_pages);
}

constexpr int kNoPage = -2;         // `written` of a row that writes into no page that it shares (-1: into none that it has)
constexpr int kNoRow = 0x7FFFFFFF;  // `writer` of a page that no row writes into

__global__ __launch_bounds__(kThreads) void update_start_kernel(PagesUpdateArgs a) {
  const int p = blockIdx.x * kThreads + threadIdx.x;
  if (p >= a.num_pages) return;
  a.cnt[p] = a.refcount[p];
  a.writer[p] = kNoRow;
}

// References of the old table off, those of the new one on, except of the
// pages that rows write into: there the lowest row is found.  blockIdx.y: the
// old sequences, then the new rows.
__global__ __launch_bounds__(kThreads) void update_count_kernel(PagesUpdateArgs a) {
  const int j = blockIdx.x * kThreads + threadIdx.x;
  if (static_cast<int>(blockIdx.y) < a.batch) {
    const int b = blockIdx.y;
    const int page = 1 << a.page_shift;
    const int pages = (clamp_to(a.lens[b], a.maxp << a.page_shift) + page - 1) >> a.page_shift;
    if (j >= pages) return;
    const int id = page_of(a.table[static_cast<int64_t>(b) * a.maxp + j], a.num_pages);
    if (id >= 0) atomicSub(a.cnt + id, 1);
    return;
  }
  const int r = blockIdx.y - a.batch;
  const Row w = row_of(a, r);
  if (j == 0) a.grows[r] = w.pages - w.first;
  if (j == 0 && !w.writes) a.written[r] = kNoPage;
  if (j >= w.first) return;
  const int id = kept_page(a, w, j);
  const bool writes = j == w.full && w.writes;
  if (writes) a.written[r] = id;
  if (id < 0) return;
  if (writes)
    atomicMin(a.writer + id, r);
  else
    atomicAdd(a.cnt + id, 1);
}

// Inclusive sum over the workgroup's threads of x, and the total.
__device__ __forceinline__ int scan_sum(int x, int* part, int& total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
  int s = x;
#pragma unroll
  for (int off = 1; off < 64; off <<= 1) {
    const int v = __shfl_up(s, off, 64);
    if (lane >= off) s += v;
  }
  __syncthreads();  // (the previous call's reads of part)
  if (lane == 63) part[wave] = s;
  __syncthreads();
  int before = 0;
  total = 0;
  for (int i = 0; i < waves; ++i) {
    before += i < wave ? part[i] : 0;
    total += part[i];
  }
  return s + before;
}

// Which rows copy, each row's place among the fresh pages (start, in row order)
// and the fresh pages themselves.  A page that a row writes into and nothing
// else holds is kept by the lowest such row, so a page is free where its count
// is zero and no row writes into it: nothing here changes a count that is read.
// A workgroup of kScanThreads calls it; returns the pages taken, *lacking the
// others.  counts_too: refcount_out is written here, for every page.
__device__ __forceinline__ int place_rows(const PagesUpdateArgs& a, int32_t* start, int32_t* fresh, int* part, int* lacking,
                                          bool counts_too) {
  const int tid = threadIdx.x;
  constexpr int kPerThread = 4;
  // the first pages' counts are asked for together with the rows
  int cnt[kPerThread], who[kPerThread];
  auto ask = [&](int p0) {
#pragma unroll
    for (int i = 0; i < kPerThread; ++i) {
      const int p = p0 + kPerThread * tid + i;
      cnt[i] = p < a.num_pages ? a.cnt[p] : 1;
      who[i] = p < a.num_pages ? a.writer[p] : 0;
    }
  };
  ask(0);
  int want = 0;
  for (int r0 = 0; r0 < a.rows; r0 += kScanThreads) {
    const int r = r0 + tid;
    int n = 0;
    bool copies = false;
    if (r < a.rows) {
      const int id = a.written[r];
      n = a.grows[r];
      copies = id == -1 || (id >= 0 && !(a.writer[id] == r && a.cnt[id] == 0));
      n += copies ? 1 : 0;
    }
    int total;
    const int incl = scan_sum(n, part, total);
    if (r < a.rows) start[r] = (want + incl - n) | (copies ? static_cast<int>(0x80000000u) : 0);
    want += total;
  }
  int found = 0;
  for (int p0 = 0; p0 < a.num_pages && (found < want || counts_too); p0 += kPerThread * kScanThreads) {
    if (p0 > 0) ask(p0);
    int n = 0;
#pragma unroll
    for (int i = 0; i < kPerThread; ++i) n += cnt[i] == 0 && who[i] == kNoRow;
    int total;
    int at = found + scan_sum(n, part, total) - n;
#pragma unroll
    for (int i = 0; i < kPerThread; ++i)
    {
      const int p = p0 + kPerThread * tid + i;
      const bool is_free = cnt[i] == 0 && who[i] == kNoRow, taken = is_free && at < want;
      if (taken) fresh[at] = p;
      // a page that a row writes into and nothing else holds is that row's
      if (counts_too && p < a.num_pages) a.refcount_out[p] = taken || (cnt[i] == 0 && !is_free) ? 1 : cnt[i];
      at += is_free;
    }
    found += total;
  }
  const int have = found < want ? found : want;
  *lacking = want - have;
  return have;
}

__global__ __launch_bounds__(kScanThreads) void update_place_kernel(PagesUpdateArgs a) {
  __shared__ int part[kScanThreads / 64];
  int lacking;
  const int have = place_rows(a, a.start, a.fresh, part, &lacking, false);
  if (threadIdx.x == 0) {
    a.info[0] = have;
    a.info[1] = lacking;
  }
}

// Entry (r, j) of the new table; kCounts: and the counts of the pages that the
// row takes or keeps.
template <bool kCounts>
__device__ __forceinline__ void write_entry(const PagesUpdateArgs& a, int r, int j, int start_of_row, const int32_t* fresh, int have) {
  const Row w = row_of(a, r);
  const bool copies = start_of_row < 0;
  const int start = start_of_row & 0x7FFFFFFF;
  int id = -1;
  if (j < w.first) {
    id = kept_page(a, w, j);
    if (j == w.full && w.writes) {
      if (copies) {
        const int from = id;
        id = start < have ? fresh[start] : -1;
        a.src[r] = id >= 0 ? from : -1;
        a.dst[r] = from >= 0 ? id : -1;
      }
      if (kCounts && id >= 0) a.refcount_out[id] = 1;  // (a page kept had no other holder)
    }
  } else if (j < w.pages) {
    const int at = start + (copies ? 1 : 0) + j - w.first;
    id = at < have ? fresh[at] : -1;
    if (kCounts && id >= 0) a.refcount_out[id] = 1;
  }
  if (j == 0 && !copies) a.src[r] = a.dst[r] = -1;
  a.table_out[static_cast<int64_t>(r) * a.maxp + j] = id;
}

__global__ __launch_bounds__(kThreads) void update_table_kernel(PagesUpdateArgs a) {
  const int j = blockIdx.x * kThreads + threadIdx.x;
  if (j < a.maxp) write_entry<true>(a, blockIdx.y, j, a.start[blockIdx.y], a.fresh, a.info[0]);
}

// The same where every workgroup finds the places for itself, in LDS, instead of
// a kernel in between: for few rows and pages, whose places take less than a
// launch (32 rows, 2900 pages: 16 us for the update's kernels, 14 so), and no
// more workgroups than run at once, since each repeats the work.
constexpr int kOwnPlaceLds = 60 * 1024;  // places and starts: what any launch may ask for, less `part`
constexpr int kOwnPlaceRows = kScanThreads;
constexpr int kOwnPlaceBlocks = 256;
__global__ __launch_bounds__(kScanThreads) void update_place_table_kernel(PagesUpdateArgs a) {
  extern __shared__ int32_t lds[];  // [num_pages] fresh pages, [rows] starts
  __shared__ int part[kScanThreads / 64];
  int32_t* start = lds + a.num_pages;
  const unsigned e = blockIdx.x * kScanThreads + threadIdx.x;  // (below 2^31)
  const int r = static_cast<int>(e / static_cast<unsigned>(a.maxp));
  int lacking;
  const int have = place_rows(a, start, lds, part, &lacking, blockIdx.x == 0);
  __syncthreads();
  if (blockIdx.x == 0 && threadIdx.x == 0) {
    a.info[0] = have;
    a.info[1] = lacking;
  }
  if (r < a.rows) write_entry<false>(a, r, static_cast<int>(e - static_cast<unsigned>(r) * a.maxp), start[r], lds, have);
}

// ------------------------------------------------------------------ compact
__device__ __forceinline__ int live_of(const int32_t* refcount, int p, int n) { return p < n && refcount[p] > 0; }

constexpr int kPer = kCompactPages / kThreads;  // pages a thread counts

// Sums of x and y over the workgroup, and the sum of x over the threads before this one.
__device__ __forceinline__ int sum_two(int x, int y, int (*part)[2], int& all_x, int& all_y) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int s = x, t = y;
#pragma unroll
  for (int off = 1; off < 64; off <<= 1) {
    const int v = __shfl_up(s, off, 64);
    if (lane >= off) s += v;
    t += __shfl_xor(t, off, 64);
  }
  __syncthreads();  // (the previous call's reads of part)
  if (lane == 63) {
    part[wave][0] = s;
    part[wave][1] = t;
  }
  __syncthreads();
  int before = s - x;
  all_x = all_y = 0;
#pragma unroll
  for (int i = 0; i < kThreads / 64; ++i) {
    before += i < wave ? part[i][0] : 0;
    all_x += part[i][0];
    all_y += part[i][1];
  }
  return before;
}

__global__ __launch_bounds__(kThreads) void compact_count_kernel(PagesCompactArgs a) {
  __shared__ int part[kThreads / 64][2];
  int n = 0;
#pragma unroll
  for (int i = 0; i < kPer; ++i) n += live_of(a.refcount, blockIdx.x * kCompactPages + i * kThreads + threadIdx.x, a.num_pages);
  int total, none;
  sum_two(n, 0, part, total, none);
  if (threadIdx.x == 0) a.counts[blockIdx.x] = total;
}

// Every page's place by its rank among the live ones (`place`): a live page
// below their number n stays; the i-th hole below n, in order, is where the
// i-th live page from n on goes, whose rank is `stay` + i with stay the rank of
// page n.  That page's thread writes the two numbers down.
__global__ __launch_bounds__(kThreads) void compact_place_kernel(PagesCompactArgs a) {
  __shared__ int part[kThreads / 64][2];
  const int tid = threadIdx.x;
  const int p0 = blockIdx.x * kCompactPages + kPer * tid;
  int is_live[kPer], own = 0;
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    is_live[i] = live_of(a.refcount, p0 + i, a.num_pages);
    own += is_live[i];
  }
  int n = 0, m = 0;  // live pages of the blocks before this one, of all
  for (int i = tid; i < static_cast<int>(gridDim.x); i += kThreads) {
    const int c = a.counts[i];
    m += c;
    n += i < static_cast<int>(blockIdx.x) ? c : 0;
  }
  int before, live, total, none;
  sum_two(n, m, part, before, live);
  int rank = before + sum_two(own, 0, part, total, none);  // live pages before p0
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    const int p = p0 + i;
    if (p < a.num_pages) {
      if (p == live || (p == a.num_pages - 1 && live == a.num_pages)) {  // (all of them live: none moves)
        a.info[0] = live;
        a.info[1] = live - rank - (live == a.num_pages ? 1 : 0);
      }
      if (p < live) {
        if (!is_live[i]) a.dst[p - rank] = p;
      } else if (is_live[i]) {
        a.place[p] = rank;
        a.ranked[rank] = p;
      }
      rank += is_live[i];
    }
  }
}

// The lists, the map and the counts (the first blocks), and the table.
__global__ __launch_bounds__(kThreads) void compact_table_kernel(PagesCompactArgs a, int list_blocks) {
  const int live = a.info[0], moves = a.info[1], stay = live - moves;
  if (static_cast<int>(blockIdx.x) < list_blocks) {
    const int at = blockIdx.x * kThreads + threadIdx.x;
    if (at >= a.num_pages) return;
    a.src[at] = at < moves ? a.ranked[stay + at] : -1;
    if (at < moves) {
      const int from = a.ranked[stay + at], to = a.dst[at];
      a.map[from] = to;
      a.refcount_out[to] = a.refcount[from];
    } else {
      a.dst[at] = -1;
    }
    const int c = a.refcount[at];
    if (at < live || c <= 0) a.map[at] = c > 0 ? at : -1;             // (one that moves: above)
    if (at >= live || c > 0) a.refcount_out[at] = at < live ? c : 0;  // (a hole: above)
    return;
  }
  const int64_t e = static_cast<int64_t>(blockIdx.x - list_blocks) * kThreads + threadIdx.x;
  if (e >= static_cast<int64_t>(a.batch) * a.maxp) return;
  const int b = static_cast<int>(static_cast<unsigned>(e) / static_cast<unsigned>(a.maxp));
  const int j = static_cast<int>(e - static_cast<int64_t>(b) * a.maxp);
  const int page = 1 << a.page_shift;
  const int pages = (clamp_to(a.lens[b], a.maxp << a.page_shift) + page - 1) >> a.page_shift;
  int id = j < pages ? page_of(a.table[e], a.num_pages) : -1;
  if (id >= 0) id = a.refcount[id] <= 0 ? -1 : id < live ? id : a.dst[a.place[id] - stay];
  a.table_out[e] = id;
}

// --------------------------------------------------------------------- copy
// A workgroup takes 16 KB of one page of one pool at a time: four 16-byte
// loads in flight per thread, then their stores.
constexpr int kCopyBytes = 16 * 1024;

__global__ __launch_bounds__(kThreads) void copy_kernel(PagesCopyArgs a, int parts) {
  int n = a.most;
  if (a.count) n = clamp_to(*a.count, a.most);
  const unsigned per = a.pools * parts, items = n * per;  // (below 2^31: pda_pages_copy)
  for (unsigned it = blockIdx.x; it < items; it += gridDim.x) {
    const unsigned pair = it / per;
    const int rest = static_cast<int>(it - pair * per);
    const int k = rest / parts;
    const int64_t bytes = a.pool[k].bytes;
    const int64_t off = static_cast<int64_t>(rest - k * parts) * kCopyBytes;
    const int from = page_of(a.src[pair], a.num_pages), to = page_of(a.dst[pair], a.num_pages);
    if (from < 0 || to < 0 || off >= bytes) continue;
    const char* s = a.pool[k].data + from * bytes + off;
    char* d = a.pool[k].data + to * bytes + off;
    const int len = static_cast<int>(bytes - off < kCopyBytes ? bytes - off : kCopyBytes);
    u32x4 v[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int o = 16 * (i * kThreads + threadIdx.x);
      if (o < len) v[i] = *reinterpret_cast<const u32x4*>(s + o);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int o = 16 * (i * kThreads + threadIdx.x);
      if (o < len) *reinterpret_cast<u32x4*>(d + o) = v[i];
    }
  }
}

}  // namespace

hipError_t launch_pages_update(const PagesUpdateArgs& args, hipStream_t st) {
  PagesUpdateArgs a = args;
  const int64_t entries = static_cast<int64_t>(a.rows) * a.maxp;
  const bool own_place = a.rows > 0 && a.rows <= kOwnPlaceRows && entries <= kOwnPlaceBlocks * kScanThreads &&
                         4 * (static_cast<int64_t>(a.num_pages) + a.rows) <= kOwnPlaceLds;
  if (!own_place) a.cnt = a.refcount_out;
  const unsigned over_pages = (a.num_pages + kThreads - 1) / kThreads, over_row = (a.maxp + kThreads - 1) / kThreads;
  hipLaunchKernelGGL(update_start_kernel, dim3(over_pages), dim3(kThreads), 0, st, a);
  if (a.batch + a.rows > 0)
    hipLaunchKernelGGL(update_count_kernel, dim3(over_row, a.batch + a.rows), dim3(kThreads), 0, st, a);
  if (own_place) {
    hipLaunchKernelGGL(update_place_table_kernel, dim3(static_cast<unsigned>((entries + kScanThreads - 1) / kScanThreads)),
                       dim3(kScanThreads), 4 * (a.num_pages + a.rows), st, a);
    return hipGetLastError();
  }
  hipLaunchKernelGGL(update_place_kernel, dim3(1), dim3(kScanThreads), 0, st, a);
  if (a.rows > 0) hipLaunchKernelGGL(update_table_kernel, dim3(over_row, a.rows), dim3(kThreads), 0, st, a);
  return hipGetLastError();
}

hipError_t launch_pages_compact(const PagesCompactArgs& a, hipStream_t st) {
  const unsigned blocks = (a.num_pages + kCompactPages - 1) / kCompactPages;
  const unsigned list = (a.num_pages + kThreads - 1) / kThreads;
  const unsigned table = static_cast<unsigned>((static_cast<int64_t>(a.batch) * a.maxp + kThreads - 1) / kThreads);
  hipLaunchKernelGGL(compact_count_kernel, dim3(blocks), dim3(kThreads), 0, st, a);
  hipLaunchKernelGGL(compact_place_kernel, dim3(blocks), dim3(kThreads), 0, st, a);
  hipLaunchKernelGGL(compact_table_kernel, dim3(list + table), dim3(kThreads), 0, st, a, static_cast<int>(list));
  return hipGetLastError();
}

int64_t pages_copy_parts(int64_t most_bytes) { return (most_bytes + kCopyBytes - 1) / kCopyBytes; }

hipError_t launch_pages_copy(const PagesCopyArgs& a, int64_t most_bytes, int cus, hipStream_t st) {
  const int parts = static_cast<int>(pages_copy_parts(most_bytes));
  const int64_t items = static_cast<int64_t>(a.most) * a.pools * parts;
  const int64_t most = static_cast<int64_t>(cus) * 8;
  hipLaunchKernelGGL(copy_kernel, dim3(static_cast<unsigned>(items < most ? items : most)), dim3(kThreads), 0, st, a, parts);
  return hipGetLastError();
}

}  // namespace pda
