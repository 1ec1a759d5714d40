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

__device__ __forceinline__ Row row_with(const PagesUpdateArgs& a, int parent, int kept, int total) {
  Row w;
  w.from = a.table + static_cast<int64_t>(parent) * a.maxp;
  w.total = total;
  w.kept = kept;
  const int page = 1 << a.page_shift;
  w.full = w.kept >> a.page_shift;
  w.first = (w.kept + page - 1) >> a.page_shift;
  w.pages = (w.total + page - 1) >> a.page_shift;
  w.writes = w.first > w.full && w.total > w.kept;
  const int64_t lo = static_cast<int64_t>(w.total) - a.nq + 1 - a.window;
  w.lo = a.window > 0 && lo > 0 ? static_cast<int>(lo) : 0;
  return w;
}

// The numbers that decide it: the parent (0 where there is none), its tokens
// that are kept, and those of the row.
struct RowInts {
  int parent, kept, total;
};

__device__ __forceinline__ RowInts row_ints(const PagesUpdateArgs& a, int r) {
  const int most = a.maxp << a.page_shift;
  const int b = a.parents ? a.parents[r] : r;
  const bool has = static_cast<unsigned>(b) < static_cast<unsigned>(a.batch);
  const int total = clamp_to(a.new_lens[r], most);
  const int len = has ? clamp_to(a.lens[b], most) : 0;
  return {has ? b : 0, len < total ? len : total, total};
}

__device__ __forceinline__ Row row_of(const PagesUpdateArgs& a, int r) {
  const RowInts n = row_ints(a, r);
  return row_with(a, n.parent, n.kept, n.total);
}

__device__ __forceinline__ int pages_of(const PagesUpdateArgs& a, int b) {
  const int page = 1 << a.page_shift;
  return (clamp_to(a.lens[b], a.maxp << a.page_shift) + page - 1) >> a.page_shift;
}

// Page j of a row, j < first: the parent's, or -1 where it holds none or no
// query of the row sees any of its tokens (past the sinks and before the
// window; a page with tokens yet to come is kept).
__device__ __forceinline__ bool released(const PagesUpdateArgs& a, const Row& w, int j) {
  const int64_t t = static_cast<int64_t>(j) << a.page_shift;
  return j < w.full && t >= a.sinks && t + (1 << a.page_shift) <= w.lo;
}
__device__ __forceinline__ int kept_page(const PagesUpdateArgs& a, const Row& w, int j) {
  return released(a, w, j) ? -1 : page_of(w.from[j], a.num_pages);
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
    if (j >= pages_of(a, b)) return;
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

// One workgroup, which goes through the pool until it has found enough free
// pages: what a step costs in a large pool is how far up they lie.  256 sequences
// by a token, 30 pages taken, us an update: 59 of 131072 pages with the free ones
// right behind 66000 live, 101 with them at the pool's end; at the end of 400000
// 283, of 1000000 683.
__global__ __launch_bounds__(kScanThreads) void update_place_kernel(PagesUpdateArgs a) {
  __shared__ int part[kScanThreads / 64];
  int lacking;
  const int have = place_rows(a, a.start, a.fresh, part, &lacking, false);
  if (threadIdx.x == 0) {
    a.info[0] = have;
    a.info[1] = lacking;
  }
}

// Entry (r, j) of the new table; `from`: the parent's page there, -1 for j >=
// w.first.  kCounts: and the counts of the pages that the row takes or keeps.
template <bool kCounts>
__device__ __forceinline__ void write_entry(const PagesUpdateArgs& a, const Row& w, int r, int j, int from, int start_of_row,
                                            const int32_t* fresh, int have) {
  const bool copies = start_of_row < 0;
  const int start = start_of_row & 0x7FFFFFFF;
  int id = from;
  if (j < w.first) {
    if (j == w.full && w.writes) {
      if (copies) {
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
  if (j >= a.maxp) return;
  const Row w = row_of(a, blockIdx.y);
  write_entry<true>(a, w, blockIdx.y, j, j < w.first ? kept_page(a, w, j) : -1, a.start[blockIdx.y], a.fresh, a.info[0]);
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
  if (r >= a.rows) return;
  const int j = static_cast<int>(e - static_cast<unsigned>(r) * a.maxp);
  const Row w = row_of(a, r);
  write_entry<false>(a, w, r, j, j < w.first ? kept_page(a, w, j) : -1, start[r], lds, have);
}

// The whole update in one launch, for fewer still: every workgroup counts the
// references for itself, too, in LDS, where a thread can ask for all its entries
// of the two tables together (rows as wide as a power of two).  Update and copy,
// 31 sequences of 11 pages as 48 rows 12.4 -> 9.4 us, 6 of 124 as 42 rows 13.5 ->
// 11.3; with three such rounds (32 rows of up to 512) it is 14.2 -> 16.5, so not
// there.
constexpr int kOneLaunchEach = 8;
constexpr int kOneLaunchEntries = kOneLaunchEach * kScanThreads;
inline int log2_up(int x) {  // x up to 2^30
  int s = 0;
  while ((1 << s) < x) ++s;
  return s;
}
inline int64_t one_launch_lds(const PagesUpdateArgs& a) {
  return 4 * (2 * static_cast<int64_t>(a.num_pages) + 9 * static_cast<int64_t>(a.rows) + 3 * static_cast<int64_t>(a.batch));
}
__global__ __launch_bounds__(kScanThreads) void update_one_kernel(PagesUpdateArgs a, int width_log2) {
  extern __shared__ int32_t lds[];
  __shared__ int part[kScanThreads / 64];
  PagesUpdateArgs l = a;
  l.cnt = lds;  // and, once the counts have been read, the fresh pages: a free page's rank is at most its number
  l.writer = l.cnt + a.num_pages;
  l.start = l.writer + a.num_pages;
  l.written = l.start + a.rows;
  l.grows = l.written + a.rows;
  int32_t* parent = l.grows + a.rows;
  int32_t* kept = parent + a.rows;
  int32_t* total = kept + a.rows;
  // the sequences, then the rows: where their entries lie, how many they are,
  // and the one that is written into (-1: none)
  const int jobs = a.batch + a.rows;
  int32_t* at = total + a.rows;
  int32_t* many = at + jobs;
  int32_t* into = many + jobs;
  const int tid = threadIdx.x;
  for (int i = tid; i < jobs; i += kScanThreads) {
    const int r = i - a.batch;
    if (r < 0) {
      at[i] = i * a.maxp;
      many[i] = pages_of(a, i);
      into[i] = -1;
      continue;
    }
    const RowInts n = row_ints(a, r);
    parent[r] = n.parent;
    kept[r] = n.kept;
    total[r] = n.total;
    const Row w = row_with(a, n.parent, n.kept, n.total);
    at[i] = n.parent * a.maxp;
    many[i] = w.first;
    into[i] = w.writes ? w.full : -1;
    l.grows[r] = w.pages - w.first;
    l.written[r] = kNoPage;
  }
  for (int p = tid; p < a.num_pages; p += kScanThreads) {
    l.cnt[p] = a.refcount[p];
    l.writer[p] = kNoRow;
  }
  const unsigned mine = blockIdx.x * kScanThreads + tid;
  const int my_row = static_cast<int>(mine / static_cast<unsigned>(a.maxp));
  const int my_j = static_cast<int>(mine - static_cast<unsigned>(my_row) * a.maxp);
  __syncthreads();
  // this thread's own entry, needed at the end
  Row w = {};
  int from = -1;
  if (my_row < a.rows) {
    w = row_with(a, parent[my_row], kept[my_row], total[my_row]);
    if (my_j < w.first) from = kept_page(a, w, my_j);
  }
  // a thread's entries are asked for together, then counted
  const int all = jobs << width_log2;
  int id[kOneLaunchEach];
#pragma unroll
  for (int i = 0; i < kOneLaunchEach; ++i) {
    const int e = tid + i * kScanThreads, job = e >> width_log2, j = e - (job << width_log2);
    id[i] = -1;
    if (e < all && j < many[job]) id[i] = page_of(a.table[at[job] + j], a.num_pages);
    if (a.window > 0 && id[i] >= 0 && job >= a.batch) {
      const int r = job - a.batch;
      if (released(a, row_with(a, parent[r], kept[r], total[r]), j)) id[i] = -1;
    }
  }
#pragma unroll
  for (int i = 0; i < kOneLaunchEach; ++i) {
    const int e = tid + i * kScanThreads, job = e >> width_log2, j = e - (job << width_log2);
    if (e >= all) break;
    const bool writes = into[job] == j;
    if (writes) l.written[job - a.batch] = id[i];
    if (id[i] < 0) continue;
    if (writes)
      atomicMin(l.writer + id[i], job - a.batch);
    else
      atomicAdd(l.cnt + id[i], job < a.batch ? -1 : 1);
  }
  __syncthreads();
  int lacking;
  const int have = place_rows(l, l.start, l.cnt, part, &lacking, blockIdx.x == 0);
  __syncthreads();
  if (blockIdx.x == 0 && tid == 0) {
    a.info[0] = have;
    a.info[1] = lacking;
  }
  if (my_row < a.rows) write_entry<false>(a, w, my_row, my_j, from, l.start[my_row], l.cnt, have);
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

// The same in one launch, for pools that every workgroup can go through for
// itself: a bit per page says which are live, and with the live pages before
// every 64 of them the rank of a page is one word, the k-th live page or hole a
// search.  Where a wave can ask for all its pages together, and with no more
// workgroups than run at once: compaction and copy, a pool of 71 pages 13.1 ->
// 8.8 us, of 7462 12.6 -> 9.3; with three such rounds (24672 pages) it is 117.5
// -> 123, so not there.
constexpr int kOneLaunchEachWave = 8;
constexpr int kOneLaunchWords = kOneLaunchEachWave * kScanThreads / 64;  // of 64 pages
constexpr int64_t kOneLaunchCompact = 256 * kScanThreads;               // pages and table entries

// The k-th set bit of x.
__device__ __forceinline__ int bit_of(uint64_t x, int k) {
  int at = 0;
#pragma unroll
  for (int half = 32; half > 0; half >>= 1) {
    const int n = __popcll(x & ((uint64_t{1} << half) - 1));
    if (k >= n) {
      k -= n;
      at += half;
      x >>= half;
    }
  }
  return at;
}

__global__ __launch_bounds__(kScanThreads) void compact_one_kernel(PagesCompactArgs a) {
  __shared__ uint64_t word[kOneLaunchWords + 1];
  __shared__ int before[kOneLaunchWords + 1];  // live pages before each word
  __shared__ int part[kScanThreads / 64];
  const int tid = threadIdx.x, lane = tid & 63;
  const int words = (a.num_pages + 63) / 64;
  // what this thread decides at the end: a page's count, or a table entry
  const int64_t e = static_cast<int64_t>(blockIdx.x) * kScanThreads + tid;
  const int64_t entry = e - a.num_pages;
  const bool in_table = entry >= 0 && entry < static_cast<int64_t>(a.batch) * a.maxp;
  const int b = in_table ? static_cast<int>(static_cast<unsigned>(entry) / static_cast<unsigned>(a.maxp)) : 0;
  const int j = static_cast<int>(entry - static_cast<int64_t>(b) * a.maxp);
  int own_count = 0, id = -1, len = 0;
  if (entry < 0) own_count = a.refcount[e];
  if (in_table) {
    id = a.table[entry];
    len = a.lens[b];
  }
  constexpr int kWaves = kScanThreads / 64;
  int c[kOneLaunchEachWave];
#pragma unroll
  for (int i = 0; i < kOneLaunchEachWave; ++i) {
    const int p = 64 * ((tid >> 6) + i * kWaves) + lane;
    c[i] = p < a.num_pages ? a.refcount[p] : 0;
  }
#pragma unroll
  for (int i = 0; i < kOneLaunchEachWave; ++i) {
    const uint64_t bits = __ballot(c[i] > 0);
    if (lane == 0) word[(tid >> 6) + i * kWaves] = bits;
  }
  __syncthreads();
  const int own = tid < words ? __popcll(word[tid]) : 0;
  int live;
  const int upto = scan_sum(own, part, live);
  if (tid < words) before[tid] = upto - own;
  if (tid == 0) {  // (a rank may be asked for just past the last word)
    if (words == kOneLaunchWords) word[words] = 0;
    before[words] = live;
  }
  __syncthreads();
  auto rank = [&](int p) { return before[p >> 6] + __popcll(word[p >> 6] & ((uint64_t{1} << (p & 63)) - 1)); };
  // the k-th live page, the k-th hole: the last word with at most k before it holds it
  auto kth = [&](int k, bool hole) {
    int lo = 0, hi = words - 1;
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if ((hole ? 64 * mid - before[mid] : before[mid]) <= k) lo = mid; else hi = mid - 1;
    }
    return 64 * lo + bit_of(hole ? ~word[lo] : word[lo], k - (hole ? 64 * lo - before[lo] : before[lo]));
  };
  const int stay = rank(live), moves = live - stay;  // live pages that keep their number
  if (blockIdx.x == 0 && tid == 0) {
    a.info[0] = live;
    a.info[1] = moves;
  }
  if (entry < 0) {
    const int at = static_cast<int>(e);
    const bool is_live = own_count > 0;
    const int r = rank(at);
    if (at >= moves) a.src[at] = a.dst[at] = -1;
    if (is_live == (at < live)) {  // it stays, live or free
      a.map[at] = is_live ? at : -1;
      a.refcount_out[at] = is_live ? own_count : 0;
    } else {  // the i-th page that moves and the i-th hole
      const int i = is_live ? r - stay : at - r;
      const int other = kth(is_live ? i : stay + i, is_live);
      (is_live ? a.src : a.dst)[i] = at;
      a.map[at] = is_live ? other : -1;
      a.refcount_out[at] = is_live ? 0 : a.refcount[other];
    }
    return;
  }
  if (!in_table) return;
  const int page = 1 << a.page_shift;
  const int pages = (clamp_to(len, a.maxp << a.page_shift) + page - 1) >> a.page_shift;
  id = j < pages ? page_of(id, a.num_pages) : -1;
  if (id >= 0) id = !(word[id >> 6] >> (id & 63) & 1) ? -1 : id < live ? id : kth(rank(id) - stay, true);
  a.table_out[entry] = id;
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
  const int width_log2 = own_place ? log2_up(a.maxp) : 0;
  if (own_place && (static_cast<int64_t>(a.batch + a.rows) << width_log2) <= kOneLaunchEntries &&
      one_launch_lds(a) <= kOwnPlaceLds) {
    hipLaunchKernelGGL(update_one_kernel, dim3(static_cast<unsigned>((entries + kScanThreads - 1) / kScanThreads)),
                       dim3(kScanThreads), static_cast<size_t>(one_launch_lds(a)), st, a, width_log2);
    return hipGetLastError();
  }
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
  const int64_t threads = a.num_pages + static_cast<int64_t>(a.batch) * a.maxp;
  if (a.num_pages <= 64 * kOneLaunchWords && threads <= kOneLaunchCompact) {
    hipLaunchKernelGGL(compact_one_kernel, dim3(static_cast<unsigned>((threads + kScanThreads - 1) / kScanThreads)),
                       dim3(kScanThreads), 0, st, a);
    return hipGetLastError();
  }
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
