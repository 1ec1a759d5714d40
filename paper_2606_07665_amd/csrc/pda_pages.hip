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
  const int32_t* from;  // the parent's table row (NULL: no parent)
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
  w.from = has ? a.table + static_cast<int64_t>(b) * a.maxp : nullptr;
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
  if (j < w.full && t >= a.sinks && t + (1 << a.page_shift) <= w.lo) return -1;
  return page_of(w.from[j], a.num_pages);
}

__global__ __launch_bounds__(kThreads) void update_start_kernel(PagesUpdateArgs a) {
  const int p = blockIdx.x * kThreads + threadIdx.x;
  if (p >= a.num_pages) return;
  a.refcount_out[p] = a.refcount[p];
  a.writer[p] = 0x7FFFFFFF;
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
    if (id >= 0) atomicSub(a.refcount_out + id, 1);
    return;
  }
  const int r = blockIdx.y - a.batch;
  const Row w = row_of(a, r);
  if (j >= w.first) return;
  const int id = kept_page(a, w, j);
  if (id < 0) return;
  if (j == w.full && w.writes)
    atomicMin(a.writer + id, r);
  else
    atomicAdd(a.refcount_out + id, 1);
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

// One workgroup: which rows copy, each row's place among the fresh pages, and
// the fresh pages themselves: the lowest ones that nothing refers to.
__global__ __launch_bounds__(kScanThreads) void update_place_kernel(PagesUpdateArgs a) {
  __shared__ int part[kScanThreads / 64];
  const int tid = threadIdx.x;
  int want = 0;
  for (int r0 = 0; r0 < a.rows; r0 += kScanThreads) {
    const int r = r0 + tid;
    int n = 0;
    bool copies = false;
    if (r < a.rows) {
      const Row w = row_of(a, r);
      if (w.writes) {
        const int id = kept_page(a, w, w.full);
        // (a row that keeps its page refers to it from here on; other rows
        // that write into it are not its lowest)
        const bool keeps = id >= 0 && a.writer[id] == r && atomicCAS(a.refcount_out + id, 0, 1) == 0;
        copies = !keeps;
      }
      n = (copies ? 1 : 0) + w.pages - w.first;
    }
    int total;
    const int incl = scan_sum(n, part, total);
    if (r < a.rows) a.start[r] = (want + incl - n) | (copies ? static_cast<int>(0x80000000u) : 0);
    want += total;
  }
  __syncthreads();  // every kept page is marked
  int found = 0;
  for (int p0 = 0; p0 < a.num_pages && found < want; p0 += 4 * kScanThreads) {
    const int p = p0 + 4 * tid;
    bool is_free[4];
    int n = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      is_free[i] = p + i < a.num_pages && __hip_atomic_load(a.refcount_out + p + i, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == 0;
      n += is_free[i];
    }
    int total;
    int at = found + scan_sum(n, part, total) - n;
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (is_free[i] && at < want) a.fresh[at++] = p + i;
    found += total;
  }
  if (tid == 0) {
    a.info[0] = found < want ? found : want;
    a.info[1] = found < want ? want - found : 0;
  }
}

__global__ __launch_bounds__(kThreads) void update_table_kernel(PagesUpdateArgs a) {
  const int j = blockIdx.x * kThreads + threadIdx.x;
  const int r = blockIdx.y;
  if (j >= a.maxp) return;
  const Row w = row_of(a, r);
  const int s = a.start[r];
  const bool copies = s < 0;
  const int start = s & 0x7FFFFFFF;
  const int have = a.info[0];
  int id = -1;
  if (j < w.first) {
    id = kept_page(a, w, j);
    if (copies && j == w.full) {
      const int from = id;
      id = start < have ? a.fresh[start] : -1;
      a.src[r] = id >= 0 ? from : -1;
      a.dst[r] = from >= 0 ? id : -1;
      if (id >= 0) a.refcount_out[id] = 1;
    }
  } else if (j < w.pages) {
    const int at = start + (copies ? 1 : 0) + j - w.first;
    id = at < have ? a.fresh[at] : -1;
    if (id >= 0) a.refcount_out[id] = 1;
  }
  if (j == 0 && !copies) a.src[r] = a.dst[r] = -1;
  a.table_out[static_cast<int64_t>(r) * a.maxp + j] = id;
}

// ------------------------------------------------------------------ compact
__device__ __forceinline__ int live_of(const int32_t* refcount, int p, int n) { return p < n && refcount[p] > 0; }

__global__ __launch_bounds__(kScanThreads) void compact_count_kernel(PagesCompactArgs a) {
  __shared__ int part[kScanThreads / 64];
  int n = 0;
#pragma unroll
  for (int i = 0; i < kCompactPages / kScanThreads; ++i)
    n += live_of(a.refcount, blockIdx.x * kCompactPages + i * kScanThreads + threadIdx.x, a.num_pages);
  int total;
  scan_sum(n, part, total);
  if (threadIdx.x == 0) a.counts[blockIdx.x] = total;
}

// Places in the list: of a hole below the number of live pages, the holes
// before it; of a live page past that, the live ones between.
__global__ __launch_bounds__(kScanThreads) void compact_place_kernel(PagesCompactArgs a) {
  __shared__ int part[kScanThreads / 64];
  const int tid = threadIdx.x;
  const int blocks = gridDim.x;
  int n = 0, m = 0;  // live pages of the blocks before this one, of all
  for (int i = tid; i < blocks; i += kScanThreads) {
    const int c = a.counts[i];
    m += c;
    n += i < static_cast<int>(blockIdx.x) ? c : 0;
  }
  int before, live;
  scan_sum(n, part, before);
  scan_sum(m, part, live);
  // live pages below `live`: whole blocks before the one it falls in, and its part of that one
  const int cut = live / kCompactPages;
  n = 0;
  for (int i = tid; i < cut && i < blocks; i += kScanThreads) n += a.counts[i];
  for (int p = cut * kCompactPages + tid; p < live; p += kScanThreads) n += live_of(a.refcount, p, a.num_pages);
  int stay;
  scan_sum(n, part, stay);

  constexpr int kPer = kCompactPages / kScanThreads;
  const int p0 = blockIdx.x * kCompactPages + kPer * tid;
  bool is_live[kPer];
  n = 0;
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    is_live[i] = live_of(a.refcount, p0 + i, a.num_pages);
    n += is_live[i];
  }
  int total;
  int rank = before + scan_sum(n, part, total) - n;  // live pages before p0
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    const int p = p0 + i;
    if (p >= a.num_pages) break;
    if (p < live) {
      a.map[p] = is_live[i] ? p : -1;
      if (is_live[i]) a.refcount_out[p] = a.refcount[p];
      else a.dst[p - rank] = p;
    } else {
      a.refcount_out[p] = 0;
      if (is_live[i]) {
        a.src[rank - stay] = p;
        a.place[p] = rank - stay;
      } else {
        a.map[p] = -1;
      }
    }
    rank += is_live[i];
  }
  if (blockIdx.x == 0 && tid == 0) {
    a.info[0] = live;
    a.info[1] = live - stay;
  }
}

// The list's pairs (blockIdx.y = 0), then the table's rows.
__global__ __launch_bounds__(kThreads) void compact_table_kernel(PagesCompactArgs a) {
  const int live = a.info[0], moves = a.info[1];
  if (blockIdx.y == 0) {
    for (int i = blockIdx.x * kThreads + threadIdx.x; i < a.num_pages; i += gridDim.x * kThreads) {
      if (i < moves) {
        const int from = a.src[i], to = a.dst[i];
        a.map[from] = to;
        a.refcount_out[to] = a.refcount[from];
      } else {
        a.src[i] = a.dst[i] = -1;
      }
    }
    return;
  }
  const int b = blockIdx.y - 1;
  const int page = 1 << a.page_shift;
  const int pages = (clamp_to(a.lens[b], a.maxp << a.page_shift) + page - 1) >> a.page_shift;
  for (int j = blockIdx.x * kThreads + threadIdx.x; j < a.maxp; j += gridDim.x * kThreads) {
    const int64_t e = static_cast<int64_t>(b) * a.maxp + j;
    int id = j < pages ? page_of(a.table[e], a.num_pages) : -1;
    if (id >= 0) id = a.refcount[id] <= 0 ? -1 : id < live ? id : a.dst[a.place[id]];
    a.table_out[e] = id;
  }
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

hipError_t launch_pages_update(const PagesUpdateArgs& a, hipStream_t st) {
  const unsigned over_pages = (a.num_pages + kThreads - 1) / kThreads, over_row = (a.maxp + kThreads - 1) / kThreads;
  hipLaunchKernelGGL(update_start_kernel, dim3(over_pages), dim3(kThreads), 0, st, a);
  hipLaunchKernelGGL(update_count_kernel, dim3(over_row, a.batch + a.rows), dim3(kThreads), 0, st, a);
  hipLaunchKernelGGL(update_place_kernel, dim3(1), dim3(kScanThreads), 0, st, a);
  if (a.rows > 0) hipLaunchKernelGGL(update_table_kernel, dim3(over_row, a.rows), dim3(kThreads), 0, st, a);
  return hipGetLastError();
}

hipError_t launch_pages_compact(const PagesCompactArgs& a, hipStream_t st) {
  const unsigned blocks = (a.num_pages + kCompactPages - 1) / kCompactPages;
  const unsigned over_row = (a.maxp + kThreads - 1) / kThreads;
  hipLaunchKernelGGL(compact_count_kernel, dim3(blocks), dim3(kScanThreads), 0, st, a);
  hipLaunchKernelGGL(compact_place_kernel, dim3(blocks), dim3(kScanThreads), 0, st, a);
  hipLaunchKernelGGL(compact_table_kernel, dim3(over_row < 16 ? over_row : 16, a.batch + 1), dim3(kThreads), 0, st, a);
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
