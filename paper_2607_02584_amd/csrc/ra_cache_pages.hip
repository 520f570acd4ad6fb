// ra_cache_pages.hip -- operators on the pages of the 4-bit paged KV cache
// (gfx950): requests that begin as others do (fork), tokens and pages given back
// (trim), the pages in use moved together (compact).
//
// Pages are copied as bytes.  Lengths, tables and the stack live on the device,
// so each operator begins with one workgroup that looks at everything, refuses
// the call as a whole or writes down what is to be done, beside others that copy
// tables into buffers of their own; the launches after it do it.  Bound by HBM
// where pages are copied, by launches otherwise.
#include "../../include/rotate_attn.h"
#include "ra_cache_pages.h"

namespace ra {
namespace {

constexpr int kPlan = 1024;           // threads of the workgroup that plans
// Of a page, what one workgroup copies at a time: 16 bytes a thread.  (With four or two times as much 125
// pages of 26 KB took 16 us to move, not 4, and 255 of 1.4 MB 78, not 70.)
constexpr int kCopyBytes = 4096;
constexpr int kCopyGroups = 8192;     // workgroups that go round pieces of pages
constexpr int kChunkLog = 12;         // pages that one workgroup gives back to the stack
constexpr int kMaxRequests = 65536;

__device__ __forceinline__ bool is_page(int id, const PageTables& t) {
  return static_cast<unsigned>(id) < static_cast<unsigned>(t.num_pages);
}
__device__ __forceinline__ int blocks_of(int n, const PageTables& t) { return (n + t.page - 1) >> t.page_log; }
__device__ __forceinline__ int longest_of(const PageTables& t) { return t.max_blocks << t.page_log; }

__device__ __forceinline__ int wave_scan(int v, int lane) {
#pragma unroll
  for (int d = 1; d < 64; d *= 2) {
    const int o = __shfl_up(v, d);
    if (lane >= d) v += o;
  }
  return v;
}

// Exclusive sum over the workgroup of N threads; *total gets the sum.
template <int N>
__device__ __forceinline__ int block_scan(int v, int (&wave)[N / 64], int* total) {
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  const int s = wave_scan(v, lane);
  __syncthreads();
  if (lane == 63) wave[w] = s;
  __syncthreads();
  int before = 0, all = 0;
#pragma unroll
  for (int i = 0; i < N / 64; ++i) {
    if (i < w) before += wave[i];
    all += wave[i];
  }
  *total = all;
  return before + s - v;
}

// The largest value over the workgroup, and whether a flag is set anywhere.
template <int N>
__device__ __forceinline__ int block_max(int v, int (&wave)[N / 64]) {
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
#pragma unroll
  for (int d = 32; d; d >>= 1) {
    const int o = __shfl_xor(v, d);
    v = o > v ? o : v;
  }
  __syncthreads();
  if (lane == 0) wave[w] = v;
  __syncthreads();
  v = wave[0];
#pragma unroll
  for (int i = 1; i < N / 64; ++i) v = wave[i] > v ? wave[i] : v;
  return v;
}
template <int N>
__device__ __forceinline__ int block_or(int v, int* shared) {
  __syncthreads();
  if (threadIdx.x == 0) *shared = 0;
  __syncthreads();
  if (v) atomicOr(shared, v);
  __syncthreads();
  return *shared;
}

// Workgroups 1 .. of a planning launch: what is left in arrays of its own
// begins as a copy.  (Lengths and count are written by the plan.)
__device__ __forceinline__ void copy_tables(const PageTables& t, int group, int groups) {
  const int64_t at = static_cast<int64_t>(group) * kPlan + threadIdx.x, step = static_cast<int64_t>(groups) * kPlan;
  if (t.table != t.table_in)
    for (int64_t i = at; i < static_cast<int64_t>(t.R) * t.max_blocks; i += step) t.table[i] = t.table_in[i];
  if (t.refs != t.refs_in)
    for (int64_t i = at; i < t.num_pages; i += step) t.refs[i] = t.refs_in[i];
  if (t.free != t.free_in)
    for (int64_t i = at; i < t.num_pages; i += step) t.free[i] = t.free_in[i];
}
int copy_groups(const PageTables& t) {
  int64_t n = 0;
  if (t.table != t.table_in) n = static_cast<int64_t>(t.R) * t.max_blocks;
  if ((t.refs != t.refs_in || t.free != t.free_in) && t.num_pages > n) n = t.num_pages;
  n = (n + 4 * kPlan - 1) / (4 * kPlan);
  return static_cast<int>(n > 255 ? 255 : n);
}

// Piece `c` of a page's bytes.
__device__ __forceinline__ void copy_piece(const PageTables& t, int src, int dst, int c) {
  const int64_t at = static_cast<int64_t>(c) * kCopyBytes + threadIdx.x * 16;
  if (at < t.page_bytes)   // whole pieces of 128 bytes
    *reinterpret_cast<uint4*>(t.cache + static_cast<int64_t>(dst) * t.page_bytes + at) =
        *reinterpret_cast<const uint4*>(t.cache + static_cast<int64_t>(src) * t.page_bytes + at);
}
static_assert(kCopyBytes == 256 * 16, "a workgroup's 16 bytes a thread");
__host__ __device__ __forceinline__ int pieces_of(const PageTables& t) {
  return static_cast<int>((t.page_bytes + kCopyBytes - 1) / kCopyBytes);
}

// ------------------------------------------------------------------- fork --
//
// Pair i makes request `child` begin with the first L tokens of `parent`: its
// first L / P entries are the parent's, whose pages have one holder more, and
// where L % P tokens are left a page from the stack gets the bytes of the page
// that holds them, so that the page a request appends to is never shared.  Where
// that entry is no page (a window lost it) there is nothing to copy, and a page of
// leftover bytes would be seen: none is taken, and the child's entry is -1.
//
// Workspace: L [n], {page copied or -1, its copy or -1} [n].

__global__ __launch_bounds__(kPlan) void k_fork_plan(ForkArgs a) {
  const PageTables& t = a.t;
  if (blockIdx.x) return copy_tables(t, blockIdx.x - 1, gridDim.x - 1);
  __shared__ int wave[kPlan / 64], flag;
  __shared__ unsigned seen[kMaxRequests / 32];   // children met so far
  const int tid = threadIdx.x, most = longest_of(t);
  int* len = t.ws;
  int2* copy = reinterpret_cast<int2*>(t.ws + ((a.n + 1) & ~1));
  for (int i = tid; i < (t.R + 31) / 32; i += kPlan) seen[i] = 0;
  __syncthreads();
  int flags = 0, longest = 0, need = 0;
  for (int i = tid; i < a.n; i += kPlan) {
    const int p = a.parents[i], c = a.children[i];
    if (static_cast<unsigned>(p) >= static_cast<unsigned>(t.R) || static_cast<unsigned>(c) >= static_cast<unsigned>(t.R)) {
      flags = 1;
      continue;
    }
    const int has = t.seq_in[p], L = a.lens ? a.lens[i] : has;
    const bool twice = atomicOr(&seen[c >> 5], 1u << (c & 31)) >> (c & 31) & 1;
    if (twice || t.seq_in[c] != 0 || has < 0 || has > most || L < 0 || L > has) flags = 1;
    len[i] = L;
    int from = -1;
    if (L & (t.page - 1) && L > 0 && L <= has && has <= most)
      from = t.table_in[static_cast<int64_t>(p) * t.max_blocks + (L >> t.page_log)];
    from = is_page(from, t) ? from : -1;
    copy[i].x = from;
    need += from >= 0;
  }
  for (int r = tid; r < t.R; r += kPlan) {
    const int n = t.seq_in[r];
    if (n <= most) longest = n > longest ? n : longest;
  }
  longest = block_max<kPlan>(longest, wave);   // (a child is no longer than its parent)
  int total;
  block_scan<kPlan>(need, wave, &total);
  const int count = t.count_in[0];
  if (count < 0 || count > t.num_pages) flags |= 8;
  else if (total > count) flags |= 4;
  flags = block_or<kPlan>(flags, &flag);
  if (t.seq != t.seq_in)
    for (int r = tid; r < t.R; r += kPlan) t.seq[r] = t.seq_in[r];
  if (!flags) {
    int carry = 0;
    for (int i0 = 0; i0 < a.n; i0 += kPlan) {
      const int i = i0 + tid;
      const int from = i < a.n ? copy[i].x : -1;   // (this thread's own)
      int all;
      const int at = carry + block_scan<kPlan>(from >= 0, wave, &all);
      if (i < a.n) copy[i].y = from >= 0 ? t.free_in[count - 1 - at] : -1;
      carry += all;
    }
    __syncthreads();   // lengths of parents were read before, those of children are written now
    for (int i = tid; i < a.n; i += kPlan) t.seq[a.children[i]] = len[i];
  }
  if (tid == 0) {
    t.count[0] = count - (flags ? 0 : total);
    t.status[0] = flags;
    t.status[1] = total;
    t.status[2] = 0;      // entries shared: k_fork adds them up
    t.status[3] = longest;
  }
}

__global__ __launch_bounds__(256) void k_fork(ForkArgs a) {
  const PageTables& t = a.t;
  const int* len = t.ws;
  const int2* copy = reinterpret_cast<const int2*>(t.ws + ((a.n + 1) & ~1));
  const int pieces = pieces_of(t), per = pieces + 1;
  const int64_t units = static_cast<int64_t>(a.n) * per;
  // (loads that do not depend on each other are asked for together: each takes a microsecond here.
  // There are n entries whatever the status, and a workgroup has a unit.)
  int2 x = copy[blockIdx.x / per];
  const int refused = t.status[0];
  if (refused) return;
  for (int64_t u = blockIdx.x; u < units; u += gridDim.x) {
    const int i = static_cast<int>(u / per), c = static_cast<int>(u - static_cast<int64_t>(i) * per);
    if (u != blockIdx.x) x = copy[i];
    if (c < pieces) {
      if (is_page(x.x, t) && is_page(x.y, t)) copy_piece(t, x.x, x.y, c);
      continue;
    }
    const int64_t from = static_cast<int64_t>(a.parents[i]) * t.max_blocks, to = static_cast<int64_t>(a.children[i]) * t.max_blocks;
    const int full = len[i] >> t.page_log;
    int shared = 0;
    for (int j = threadIdx.x; j < full; j += 256) {
      const int id = t.table_in[from + j];
      t.table[to + j] = id;
      if (is_page(id, t)) {
        atomicAdd(&t.refs[id], 1);
        ++shared;
      }
    }
#pragma unroll
    for (int d = 32; d; d >>= 1) shared += __shfl_xor(shared, d);
    if ((threadIdx.x & 63) == 0 && shared) atomicAdd(&t.status[2], shared);
    if (threadIdx.x == 0 && len[i] & (t.page - 1)) t.table[to + full] = is_page(x.y, t) ? x.y : -1;
  }
}

// ------------------------------------------------------------------- trim --
//
// Request r keeps its first k tokens: blocks ceil(k / P) .. ceil(L / P) - 1 are
// let go, and where a window is given those whose tokens all lie behind the
// first `sinks` ones and before every key that a query at k or later sees.
// Where k ends inside a page that others hold too, the request gets a copy of
// it, as it will append there.
//
// A page that is let go has one holder less; one that had no other is marked by
// the count falling to -1, whoever came last, so that the set of marked pages does not
// depend on the order.  k_give_back puts them on the stack by page number.
//
// Workspace: copies {request, page, its copy, 0} [R], blocks held [R], the number of
// copies and the stack's top once they have their pages, marked pages in each
// chunk of 2^12.

struct TrimSpace {
  int4* copy;
  int* held;
  int* copies;   // [2]
  int* chunk;
};
__host__ __device__ __forceinline__ int chunks_of(int num_pages) { return (num_pages + (1 << kChunkLog) - 1) >> kChunkLog; }
__device__ __forceinline__ TrimSpace trim_space(const PageTables& t) {
  TrimSpace s;
  s.copy = reinterpret_cast<int4*>(t.ws);
  s.held = t.ws + 4 * static_cast<int64_t>(t.R);
  s.copies = s.held + t.R;
  s.chunk = s.copies + 2;
  return s;
}

__global__ __launch_bounds__(kPlan) void k_trim_plan(TrimArgs a) {
  const PageTables& t = a.t;
  if (blockIdx.x) return copy_tables(t, blockIdx.x - 1, gridDim.x - 1);
  __shared__ int wave[kPlan / 64], flag;
  const TrimSpace s = trim_space(t);
  const int tid = threadIdx.x, most = longest_of(t);
  for (int i = tid; i < chunks_of(t.num_pages); i += kPlan) s.chunk[i] = 0;
  auto kept = [&](int r, int L) {
    const int k = a.keep ? a.keep[r] : -1;
    return k < 0 ? L : k;
  };
  // the page that the kept tokens end in, if others hold it too
  auto to_copy = [&](int r, int k) {
    if (!(k & (t.page - 1))) return -1;
    const int id = t.table_in[static_cast<int64_t>(r) * t.max_blocks + (k >> t.page_log)];
    return is_page(id, t) && t.refs_in[id] > 0 ? id : -1;
  };
  int flags = 0, longest = 0, need = 0;
  for (int r = tid; r < t.R; r += kPlan) {
    const int L = t.seq_in[r];
    if (L < 0 || L > most) {
      flags = 1;
      continue;
    }
    const int k = kept(r, L);
    if (k > L) {
      flags = 1;
      continue;
    }
    longest = k > longest ? k : longest;
    need += to_copy(r, k) >= 0;
  }
  longest = block_max<kPlan>(longest, wave);
  int total;
  block_scan<kPlan>(need, wave, &total);
  const int count = t.count_in[0];
  if (count < 0 || count > t.num_pages) flags |= 8;
  else if (total > count) flags |= 4;
  flags = block_or<kPlan>(flags, &flag);
  if (flags) {
    for (int r = tid; r < t.R; r += kPlan) t.seq[r] = t.seq_in[r];
  } else {
    int carry = 0;
    for (int r0 = 0; r0 < t.R; r0 += kPlan) {
      const int r = r0 + tid;
      int id = -1;
      if (r < t.R) {
        const int L = t.seq_in[r], k = kept(r, L);
        id = to_copy(r, k);
        s.held[r] = blocks_of(L, t);
        t.seq[r] = k;
      }
      int all;
      const int at = carry + block_scan<kPlan>(id >= 0, wave, &all);
      if (id >= 0) s.copy[at] = make_int4(r, id, t.free_in[count - 1 - at], 0);
      carry += all;
    }
  }
  if (tid == 0) {
    s.copies[0] = total;
    s.copies[1] = count - total;
    t.count[0] = count - (flags ? 0 : total);
    t.status[0] = flags;
    t.status[1] = total;
    t.status[2] = 0;
    t.status[3] = longest;
  }
}

// (A workgroup counts its marked pages in LDS first: one addition in memory for each of them
// met at a few dozen addresses and made 123 us of what takes 10, 1000 requests that let go of 60 000 entries.)
constexpr int kNear = 4096;   // chunks that are counted so
__device__ __forceinline__ void let_go(const PageTables& t, const TrimSpace& s, int* near, int id) {
  if (!is_page(id, t) || atomicSub(&t.refs[id], 1) != 0) return;
  const int c = id >> kChunkLog;
  atomicAdd(c < kNear ? &near[c] : &s.chunk[c], 1);
}

__global__ __launch_bounds__(256) void k_trim(TrimArgs a) {
  const PageTables& t = a.t;
  __shared__ int near[kNear];
  const TrimSpace s = trim_space(t);
  const int refused = t.status[0], copies = s.copies[0];
  if (refused) return;
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  const int pieces = pieces_of(t), chunks = chunks_of(t.num_pages) < kNear ? chunks_of(t.num_pages) : kNear;
  for (int i = threadIdx.x; i < chunks; i += 256) near[i] = 0;
  __syncthreads();
  const int rows = (t.R + 3) / 4;   // units of four requests, a wave each
  const int64_t units = rows + static_cast<int64_t>(copies) * pieces;
  for (int64_t u = blockIdx.x; u < units; u += gridDim.x) {
    if (u < rows) {
      const int r = static_cast<int>(u) * 4 + w;
      if (r >= t.R) continue;
      int* row = t.table + static_cast<int64_t>(r) * t.max_blocks;
      const int k = t.seq[r], held = s.held[r], left = blocks_of(k, t);
      int e0 = left, e1 = left;
      if (a.sinks >= 0 && a.window > 0) {
        e0 = blocks_of(a.sinks < k ? a.sinks : k, t);
        const int before = k - a.window + 1;
        e1 = before > 0 ? before >> t.page_log : 0;
      }
      auto go = [&](int j0, int j1) {
        for (int j = j0 + lane; j < j1; j += 64) {
          let_go(t, s, near, row[j]);
          row[j] = -1;
        }
      };
      go(e0, e1);
      go(left, held);
      continue;
    }
    const int64_t v = u - rows;
    const int i = static_cast<int>(v / pieces), c = static_cast<int>(v - static_cast<int64_t>(i) * pieces);
    const int4 x = s.copy[i];
    if (is_page(x.z, t)) copy_piece(t, x.y, x.z, c);
    if (c == 0 && threadIdx.x == 0) {
      t.table[static_cast<int64_t>(x.x) * t.max_blocks + (t.seq[x.x] >> t.page_log)] = is_page(x.z, t) ? x.z : -1;
      let_go(t, s, near, x.y);
    }
  }
  __syncthreads();
  for (int i = threadIdx.x; i < chunks; i += 256)
    if (near[i]) atomicAdd(&s.chunk[i], near[i]);
}

__global__ __launch_bounds__(kPlan) void k_give_back(TrimArgs a) {
  const PageTables& t = a.t;
  if (t.status[0]) return;
  __shared__ int wave[kPlan / 64];
  const TrimSpace s = trim_space(t);
  const int b = blockIdx.x, tid = threadIdx.x, chunks = chunks_of(t.num_pages);
  if (b && s.chunk[b] == 0) return;
  int before = 0, all = 0;
  for (int i = tid; i < (b ? b : chunks); i += kPlan) {
    all += s.chunk[i];
    if (i < b) before += s.chunk[i];
  }
  int total, total_before;
  block_scan<kPlan>(all, wave, &total);
  block_scan<kPlan>(before, wave, &total_before);
  const int base = s.copies[1];
  if (b == 0 && tid == 0) {
    const int64_t n = static_cast<int64_t>(base) + total;
    t.count[0] = static_cast<int>(n < t.num_pages ? n : t.num_pages);
    t.status[2] = total;
  }
  constexpr int N = (1 << kChunkLog) / kPlan;
  const int p0 = (b << kChunkLog) + tid * N;
  int gone = 0;
#pragma unroll
  for (int e = 0; e < N; ++e) gone |= (p0 + e < t.num_pages && t.refs[p0 + e] < 0) << e;
  int sum;
  int at = base + total_before + block_scan<kPlan>(__popc(gone), wave, &sum);
#pragma unroll
  for (int e = 0; e < N; ++e)
    if (gone >> e & 1) {
      if (at < t.num_pages) t.free[at] = p0 + e;
      t.refs[p0 + e] = 0;
      ++at;
    }
}

// ---------------------------------------------------------------- compact --
//
// With `count` pages free, k = num_pages - count are in use: the i-th of them
// that lies at k or behind moves to the i-th free page before k.  Sources and
// targets are disjoint, so pages are copied in any order.
//
// The plan marks the free pages as bits in LDS, kBits pages at a time (all of
// them, for caches of up to 2^18 pages), and sums the bits of each word: a page's
// place among the free ones, and among those in use, follows from that.  Every
// round goes through the whole stack, in one workgroup: 36 us for 2^17 pages of which half
// are free, 69 for 2^18, 175, 515 and 1850 for 2^19, 2^20 and 2^21.
//
// Workspace: the number of moves, source pages and targets [num_pages / 2 + 1 each],
// for every page from k on its number among the sources or -1.
constexpr int kBits = 1 << 18;

struct CompactSpace {
  int* moves;
  int* src;
  int* dst;
  int* number;   // of page - k
};
__device__ __forceinline__ CompactSpace compact_space(const PageTables& t) {
  CompactSpace s;
  const int half = t.num_pages / 2 + 1;
  s.moves = t.ws;
  s.src = t.ws + 4;
  s.dst = s.src + half;
  s.number = s.dst + half;
  return s;
}

__global__ __launch_bounds__(kPlan) void k_compact_plan(PageTables t) {
  if (blockIdx.x) return copy_tables(t, blockIdx.x - 1, gridDim.x - 1);
  __shared__ unsigned bits[kBits / 32];
  __shared__ int sums[kBits / 32];   // free pages before a word, of the round
  __shared__ int wave[kPlan / 64], flag;
  const CompactSpace s = compact_space(t);
  const int tid = threadIdx.x, most = longest_of(t), half = t.num_pages / 2 + 1;
  const int count = t.count_in[0];
  int flags = count < 0 || count > t.num_pages ? 8 : 0;
  for (int r = tid; r < t.R; r += kPlan) {
    const int L = t.seq_in[r];
    if (L < 0 || L > most) flags |= 1;
    if (t.seq != t.seq_in) t.seq[r] = L;
  }
  flags = block_or<kPlan>(flags, &flag);
  int targets = 0, before = 0;   // free pages before k, and before the round
  if (!(flags & 8)) {
    const int k = t.num_pages - count;
    for (int first = 0; first < t.num_pages; first += kBits) {
      const int n = t.num_pages - first < kBits ? t.num_pages - first : kBits, words = (n + 31) / 32;
      __syncthreads();
      for (int i = tid; i < words; i += kPlan) bits[i] = 0;
      __syncthreads();
      int bad = 0;
      for (int i0 = tid; i0 < count; i0 += 8 * kPlan) {   // eight loads under way
        int id[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) id[e] = i0 + e * kPlan < count ? t.free_in[i0 + e * kPlan] : 0;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          if (i0 + e * kPlan >= count) continue;
          if (!is_page(id[e], t)) bad = 16;
          else if (id[e] >= first && id[e] - first < n)
            bad |= atomicOr(&bits[(id[e] - first) >> 5], 1u << (id[e] & 31)) >> (id[e] & 31) & 1 ? 16 : 0;
        }
      }
      flags |= block_or<kPlan>(bad, &flag);
      const int per = (words + kPlan - 1) / kPlan, w0 = tid * per, w1 = w0 + per < words ? w0 + per : words;
      int own = 0, all;
      for (int w = w0; w < w1; ++w) own += __popc(bits[w]);
      own = block_scan<kPlan>(own, wave, &all);
      for (int w = w0; w < w1; ++w) {
        sums[w] = own;
        own += __popc(bits[w]);
      }
      __syncthreads();
      auto free_before = [&](int p) { return before + sums[p >> 5] + __popc(bits[p >> 5] & ((1u << (p & 31)) - 1)); };   // p: of the round
      if (k >= first + n) targets = before + all;
      else if (k >= first) targets = free_before(k - first);
      for (int p = tid; p < n; p += kPlan) {
        const int page = first + p, f = free_before(p);
        const bool free = bits[p >> 5] >> (p & 31) & 1;
        if (page < k) {
          if (free && f < half) s.dst[f] = page;
        } else {
          const int i = (page - f) - (k - targets);   // pages in use between k and this one
          s.number[page - k] = free ? -1 : i;
          if (!free && i >= 0 && i < half) s.src[i] = page;
        }
      }
      before += all;
    }
  }
  if (tid == 0) {
    // a stack of other pages than the free ones has been seen above: sources == targets otherwise
    t.count[0] = count;
    s.moves[0] = flags ? 0 : targets;
    t.status[0] = flags;
    t.status[1] = flags ? 0 : targets;
    t.status[2] = t.num_pages - count;
    t.status[3] = 0;
  }
}

__global__ __launch_bounds__(256) void k_compact(PageTables t, int copiers) {
  if (t.status[0]) return;
  const CompactSpace s = compact_space(t);
  const int moves = s.moves[0];
  if (static_cast<int>(blockIdx.x) < copiers) {
    const int pieces = pieces_of(t);
    const int64_t units = static_cast<int64_t>(moves) * pieces;
    for (int64_t u = blockIdx.x; u < units; u += copiers) {
      const int i = static_cast<int>(u / pieces);
      copy_piece(t, s.src[i], s.dst[i], static_cast<int>(u - static_cast<int64_t>(i) * pieces));
    }
    return;
  }
  // tables, holders and the stack
  const int groups = gridDim.x - copiers, g = blockIdx.x - copiers, k = t.status[2], count = t.num_pages - k;
  for (int r = g; r < t.R; r += groups) {
    int* row = t.table + static_cast<int64_t>(r) * t.max_blocks;
    const int held = blocks_of(t.seq[r], t);
    for (int j = threadIdx.x; j < held; j += 256) {
      const int id = row[j];
      if (!is_page(id, t) || id < k) continue;
      const int x = s.number[id - k];
      if (x >= 0) row[j] = s.dst[x];
    }
  }
  const int at = g * 256 + threadIdx.x, step = groups * 256;
  for (int i = at; i < moves; i += step) {
    const int from = s.src[i];
    t.refs[s.dst[i]] = t.refs_in[from];
    t.refs[from] = 0;
  }
  for (int i = at; i < count; i += step) t.free[i] = t.num_pages - 1 - i;
}

unsigned groups_for(int64_t units) { return static_cast<unsigned>(units < 1 ? 1 : units > kCopyGroups ? kCopyGroups : units); }

}  // namespace

size_t cache_pages_workspace_bytes(int R, int num_pages) {
  const size_t fork = 4 * static_cast<size_t>(R + 1) + 8 * static_cast<size_t>(R);
  const size_t trim = 20 * static_cast<size_t>(R) + 4 * (static_cast<size_t>(chunks_of(num_pages)) + 2);
  const size_t compact = 4 * (2 * static_cast<size_t>(num_pages) + 8);
  size_t most = fork > trim ? fork : trim;
  most = most > compact ? most : compact;
  return (most + 255) / 256 * 256;
}

hipError_t launch_cache_fork(const ForkArgs& a, hipStream_t s) {
  k_fork_plan<<<dim3(1 + copy_groups(a.t)), dim3(kPlan), 0, s>>>(a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || a.n == 0) return e;
  k_fork<<<dim3(groups_for(static_cast<int64_t>(a.n) * (pieces_of(a.t) + 1))), dim3(256), 0, s>>>(a);
  return hipGetLastError();
}

hipError_t launch_cache_trim(const TrimArgs& a, hipStream_t s) {
  k_trim_plan<<<dim3(1 + copy_groups(a.t)), dim3(kPlan), 0, s>>>(a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  // (how many pages are copied is known on the device: few, as a rule)
  k_trim<<<dim3(groups_for((a.t.R + 3) / 4 + static_cast<int64_t>(a.t.R) * pieces_of(a.t))), dim3(256), 0, s>>>(a);
  e = hipGetLastError();
  if (e != hipSuccess) return e;
  k_give_back<<<dim3(chunks_of(a.t.num_pages)), dim3(kPlan), 0, s>>>(a);
  return hipGetLastError();
}

hipError_t launch_cache_compact(const PageTables& t, hipStream_t s) {
  k_compact_plan<<<dim3(1 + copy_groups(t)), dim3(kPlan), 0, s>>>(t);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const int copiers = static_cast<int>(groups_for(static_cast<int64_t>(t.num_pages / 2 + 1) * pieces_of(t)));
  int others = (t.num_pages + 1023) / 1024 > t.R ? (t.num_pages + 1023) / 1024 : t.R;
  others = others < 1 ? 1 : others > 512 ? 512 : others;
  k_compact<<<dim3(copiers + others), dim3(256), 0, s>>>(t, copiers);
  return hipGetLastError();
}

}  // namespace ra
