// ra_cache_pages.h -- arguments of the operators on the pages of the 4-bit
// paged KV cache: fork, trim, compact (library-internal).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace ra {

// The tables as they are and as they are left: each pair is one array, or two
// that do not overlap.
struct PageTables {
  const int* seq_in;     // [R]
  const int* table_in;   // [R][max_blocks]
  const int* refs_in;    // [num_pages], holders beyond the first
  const int* free_in;    // [num_pages], the top of the stack at count - 1
  const int* count_in;
  int* seq;
  int* table;
  int* refs;
  int* free;
  int* count;
  int* status;           // [4]
  uint8_t* cache;
  int* ws;
  int64_t page_bytes;
  int R, max_blocks, num_pages, page, page_log;
};

struct ForkArgs {
  PageTables t;
  const int* parents;    // [n]
  const int* children;
  const int* lens;       // [n] or nullptr
  int n;
};

struct TrimArgs {
  PageTables t;
  const int* keep;       // [R] or nullptr
  int sinks, window;     // pages between the first tokens and the window go too, where sinks >= 0 and window > 0
};

hipError_t launch_cache_fork(const ForkArgs& a, hipStream_t s);
hipError_t launch_cache_trim(const TrimArgs& a, hipStream_t s);
hipError_t launch_cache_compact(const PageTables& t, hipStream_t s);
size_t cache_pages_workspace_bytes(int R, int num_pages);

}  // namespace ra
