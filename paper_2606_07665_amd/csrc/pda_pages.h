// Internal interface of the page kernels (not part of the public ABI).
#pragma once
#include <hip/hip_runtime.h>
#include <cstdint>

namespace pda {

constexpr int kMaxPoolPages = 1 << 24;  // pages of a pool that the page calls manage
constexpr int kMaxCopyPools = 128;      // pools a copy launch takes (2 KB of arguments)

struct PagesUpdateArgs {
  const int32_t* table;     // [batch, maxp]
  const int32_t* lens;      // [batch]
  const int32_t* parents;   // [rows], or NULL: row r continues sequence r
  const int32_t* new_lens;  // [rows]
  const int32_t* refcount;  // [num_pages]
  int32_t* table_out;       // [rows, maxp]
  int32_t* refcount_out;    // [num_pages]
  int32_t* src;             // [rows]
  int32_t* dst;             // [rows]
  int32_t* info;            // [2]
  int32_t* cnt;             // workspace [num_pages]: references without those of the rows that write into a page
  int32_t* writer;          // workspace [num_pages]: the lowest row that writes into a page
  int32_t* fresh;           // workspace [num_pages]: the free pages, ascending, as many as are wanted
  int32_t* start;           // workspace [rows]: a row's place among the fresh pages, and bit 31: it copies
  int32_t* written;         // workspace [rows]: the page a row writes into
  int32_t* grows;           // workspace [rows]: fresh pages it takes, a copy apart
  int batch, rows, page_shift, num_pages, maxp, nq, window, sinks;
};

struct PagesCompactArgs {
  const int32_t* table;
  const int32_t* lens;
  const int32_t* refcount;
  int32_t* table_out;     // [batch, maxp]
  int32_t* refcount_out;  // [num_pages]
  int32_t* map;           // [num_pages]
  int32_t* src;           // [num_pages]
  int32_t* dst;           // [num_pages]
  int32_t* info;          // [2]
  int32_t* counts;        // workspace [ceil(num_pages / kCompactPages)]
  int32_t* place;         // workspace [num_pages]: a moving page's rank among the live ones
  int32_t* ranked;        // workspace [num_pages]: the moving page of each rank
  int batch, page_shift, num_pages, maxp;
};
constexpr int kCompactPages = 1024;  // pages per workgroup of the counting passes

struct PagesCopyArgs {
  struct Pool {
    char* data;
    int64_t bytes;  // of a page, a multiple of 16
  } pool[kMaxCopyPools];
  const int32_t* src;
  const int32_t* dst;
  const int32_t* count;  // device, or NULL
  int pools, most, num_pages;
};

hipError_t launch_pages_update(const PagesUpdateArgs& a, hipStream_t st);
hipError_t launch_pages_compact(const PagesCompactArgs& a, hipStream_t st);
int64_t pages_copy_parts(int64_t most_bytes);  // pieces a page of so many bytes is copied in
hipError_t launch_pages_copy(const PagesCopyArgs& a, int64_t most_bytes, int cus, hipStream_t st);

}  // namespace pda
