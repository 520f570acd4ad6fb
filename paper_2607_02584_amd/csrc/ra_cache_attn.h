// ra_cache_attn.h -- attention over the 4-bit paged KV cache: what its kernels
// are made of (library-internal; each source that includes it has its own copy).
//
// For every request, query token i (position p = len - queries + i) and head:
//   s_j = scale * q . k_j,   o = sum_j softmax(s)_j v_j,   lse = ln sum_j e^{s_j}
// over the keys j that the mask leaves (j <= p where causal, j > p - window),
// K and V being code * scale of their token.  One pass over the keys with a
// running maximum m and sum l (FlashAttention's recurrence), base 2.
//
// The G = Hq / Hkv query heads of a KV head and a request's tokens form one
// list of rows (row = token * G + head in group), so that a tile of rows
// shares the K and V it reads.
#pragma once
#include <type_traits>
#include <utility>

#include "../../include/rotate_attn.h"
#include "ra_cache.h"

namespace ra {
namespace {

typedef float v4f __attribute__((ext_vector_type(4)));
typedef __bf16 v8bf __attribute__((ext_vector_type(8)));
typedef _Float16 v8h __attribute__((ext_vector_type(8)));

constexpr float kNegInf = -__builtin_inff();
constexpr float kLn2 = 0.693147180559945309417232121458f;

// --------------------------------------------------------------- schedule --
//
// Work is cut into pieces of (request, tile of M rows, part of the keys), the
// same for every KV head.  Lengths live on the device (a captured graph runs
// with whatever they are then), so every workgroup cuts alone, in the same
// way: with W the sum over tiles of their blocks of 64 keys, a part has
// C = max(least, W / target) blocks, and a request's tiles have
// n = ceil(blocks / C) parts.  There are then at most (tiles + target) pieces, and at most
// 2 * target of tiles that have several parts, whatever the lengths: the grid
// and the workspace follow from that.
constexpr int kBlock = 64;        // keys

// Which keys a call's rows see:
//   kAll     the request's, cut by causality and a window
//   kSinks   those, and its first `sinks` tokens whatever the window
//   kShared  those of a prefix that a group of requests holds together, and the request's behind it:
//            either is a request of its own here, numbers below `groups` being the groups' prefixes
//            (rows: the queries of all the group's requests).  Its pieces are
//            listed by a launch before (ra_cache_shared.hip).
enum Keys { kAll, kSinks, kShared };

// The two kernels share a call's requests by their number of rows: up to
// kFewRows a request is bound by its keys (k_few), above by the matrix cores
// (k_rows).
constexpr int kFewRows = 32;
// Blocks of the least part: a step of 32 keys for each of the four waves of k_few, twice; for many rows enough
// to pay for a partial output of M rows.
template <int M>
constexpr int least_blocks() { return M <= kFewRows ? 4 : 16; }

struct Request {
  int q0, ql, n;    // first query row, queries to compute (max_q at most), cached tokens
  int first;        // position of the first query
  int tiles, blocks;
  int lo, table;    // kShared: the first key, and the request whose table names the pages
};

template <int M, Keys K>
__device__ __forceinline__ Request request_of(const CacheAttnArgs& a, int r) {
  Request x;
  x.lo = 0;
  x.table = r;
  int q0 = a.q_start[r], q1 = a.q_start[r + 1];
  const int most = a.max_blocks << a.g.page_log;
  int n = a.seq_lens[r];
  // whatever the device holds, nothing outside the tensors is touched
  q0 = q0 < 0 ? 0 : q0 > a.T ? a.T : q0;
  q1 = q1 < q0 ? q0 : q1 > a.T ? a.T : q1;
  x.q0 = q0;
  x.ql = q1 - q0 < a.max_q ? q1 - q0 : a.max_q;
  x.n = n < 0 ? 0 : n > most ? most : n;
  x.first = x.n - (q1 - q0);
  const int rows = x.ql * a.G;
  x.tiles = (rows <= kFewRows) == (M <= kFewRows) ? (rows + M - 1) / M : 0;
  int keys = x.n;
  if (a.window) {
    const int first = x.first - a.window + 1;
    keys = x.n - (first > 0 ? first : 0);
    const int tile = a.window + M / a.G + 1 + kBlock;   // keys that one tile can see, in whole blocks
    keys = keys < tile ? keys : tile;
  }
  x.blocks = (keys + kBlock - 1) / kBlock;
  if constexpr (K == kSinks) {
    // with the blocks of the first tokens (of no more than there are)
    const int all = (x.n + kBlock - 1) / kBlock, more = (a.sinks + kBlock - 1) / kBlock;
    x.blocks = x.blocks + more < all ? x.blocks + more : all;
  }
  return x;
}

// The largest over a wave of values that are not negative.
__device__ __forceinline__ int wave_most(int v) {
  auto take = [&](int o) { v = o > v ? o : v; };
  take(__builtin_amdgcn_update_dpp(0, v, 0x111, 0xF, 0xF, false));
  take(__builtin_amdgcn_update_dpp(0, v, 0x112, 0xF, 0xF, false));
  take(__builtin_amdgcn_update_dpp(0, v, 0x114, 0xF, 0xF, false));
  take(__builtin_amdgcn_update_dpp(0, v, 0x118, 0xF, 0xF, false));
  take(__builtin_amdgcn_update_dpp(0, v, 0x142, 0xA, 0xF, false));
  take(__builtin_amdgcn_update_dpp(0, v, 0x143, 0xC, 0xF, false));
  return __builtin_amdgcn_readlane(v, 63);
}

// Blocks of a part, W blocks in all: at least W / target, the sum's roundings
// (the same in every workgroup) included.
template <int M, Keys K>
__device__ __forceinline__ unsigned part_blocks(float W, int target) {
  const float c = W * (1.0f + 0x1p-10f) / static_cast<float>(target) + 1.0f;
  const unsigned C = c < 0x1p26f ? static_cast<unsigned>(c) : 1u << 26;   // a request has 2^24 at most
  // kSinks: parts of many rows as short as those of few while they fill a quarter of the places at most (one request of 64
  // rows over 600 keys 31 -> 22 us).  Where they would fill all, what waits for a place loses more than they gain
  // (30 requests of one query beside a prompt of 300 tokens 59 -> 69 us).
  if (K == kSinks && M > kFewRows && C < static_cast<unsigned>(least_blocks<M>())) {
    const unsigned quarter = static_cast<unsigned>(4.0f * c);
    return quarter < 4 ? 4 : quarter < static_cast<unsigned>(least_blocks<M>()) ? quarter : least_blocks<M>();
  }
  return C < static_cast<unsigned>(least_blocks<M>()) ? least_blocks<M>() : C;
}

struct Piece {
  Request q;
  int r, tile, part, parts, slot;   // slot: place in the workspace of part 0 of this tile (kShared: of the request, in rows)
  bool two;                         // kSinks, kShared: of no more than kTwoTerms rows
};

// How many bf16 values hold P times V's scale in a piece of many rows: as many as the output shows, so three for binary32
// and two for binary16 outputs.  For bf16 ones one leaves as much error as their own rounding does (2.3e-3 of both, 1.65e-3
// of the latter) and saves a quarter of the time where the matrix cores bind, as they do in requests of many rows (prompts
// under a window 451 us with one value, 560 with two).  cache_attn_sinks and cache_attn_shared take it there only: a
// request's own rows (queries * Hq) decide, whatever else the call holds or has room for, and for a prefix the least of its
// requests'.  (A decode step of 64 requests over a prefix of 32 700 tokens 90 us with one value, 100 with two.)
constexpr int kTwoTerms = 512;   // rows of all heads up to which there are two

struct SchedShared {
  float w[4];
  int s[4][2];
  int hit[10];
};

// Inclusive sum over a wave by register moves (row shifts, then the rows' last
// lanes broadcast on).
__device__ __forceinline__ int wave_sums(int v) {
  v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xF, 0xF, false);   // row_shr:1
  v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xF, 0xF, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xF, 0xF, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xF, 0xF, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xA, 0xF, false);   // row_bcast:15
  v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xC, 0xF, false);   // row_bcast:31
  return v;
}
__device__ __forceinline__ float wave_total(float v) {
#pragma unroll
  for (int i = 0; i < 6; ++i) {
    const int u = __float_as_int(v);
    const int o = i == 0   ? __builtin_amdgcn_update_dpp(0, u, 0x111, 0xF, 0xF, false)
                  : i == 1 ? __builtin_amdgcn_update_dpp(0, u, 0x112, 0xF, 0xF, false)
                  : i == 2 ? __builtin_amdgcn_update_dpp(0, u, 0x114, 0xF, 0xF, false)
                  : i == 3 ? __builtin_amdgcn_update_dpp(0, u, 0x118, 0xF, 0xF, false)
                  : i == 4 ? __builtin_amdgcn_update_dpp(0, u, 0x142, 0xA, 0xF, false)
                           : __builtin_amdgcn_update_dpp(0, u, 0x143, 0xC, 0xF, false);
    v += __int_as_float(o);
  }
  return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), 63));
}

// Piece number x (or, for the merge, tile number x of those with several
// parts); false past the end.  All 256 threads of the workgroup call it.  Up to
// 64 requests every wave finds it alone, from one load of the lengths; above,
// 256 requests at a time through LDS.
template <int M, Keys K>
__device__ __forceinline__ bool find_piece(const CacheAttnArgs& a, SchedShared& sh, int x, bool merge, int target,
                                           Piece* out) {
  const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
  auto parts_of = [&](const Request& q, unsigned C) {
    return q.tiles ? (q.blocks ? static_cast<int>((q.blocks + C - 1) / C) : 1) : 0;
  };
  auto finish = [&](int r, int at, int n, int slot, const Request& q) {
    out->r = r;
    out->q = q;
    out->parts = n;
    out->tile = merge ? at : at / n;
    out->part = merge ? 0 : at - out->tile * n;
    out->slot = slot + out->tile * n;
    out->q.lo = 0;
    out->q.table = r;
    out->two = K == kSinks && q.ql * a.Hq <= kTwoTerms;
  };
  if (a.R <= 64) {
    Request q = {};
    if (lane < a.R) q = request_of<M, K>(a, lane);
    const float W = wave_total(static_cast<float>(q.tiles) * static_cast<float>(q.blocks));
    const int n = parts_of(q, part_blocks<M, K>(W, target));
    const int split = n > 1 ? q.tiles * n : 0, mine = merge ? (n > 1 ? q.tiles : 0) : q.tiles * n;
    const int from = wave_sums(mine) - mine, slot = wave_sums(split) - split;
    const unsigned long long hit = __ballot(x >= from && x < from + mine);
    if (!hit) return false;
    const int r = __builtin_ctzll(hit);
    auto take = [&](int v) { return __builtin_amdgcn_readlane(v, r); };
    finish(r, x - take(from), take(n), take(slot), {take(q.q0), take(q.ql), take(q.n), take(q.first), take(q.tiles), take(q.blocks)});
    return true;
  }
  float W = 0.0f;
  int longest = 0;
  Request q0 = {};
  for (int r = tid; r < a.R; r += 256) {
    const Request q = request_of<M, K>(a, r);
    if (r == tid) q0 = q;
    W += static_cast<float>(q.tiles) * static_cast<float>(q.blocks);
    if (K == kSinks && q.tiles && q.blocks > longest) longest = q.blocks;
  }
  W = wave_total(W);
  if (lane == 0) sh.w[w] = W;
  if constexpr (K == kSinks) {
    longest = wave_most(longest);
    if (lane == 0) sh.s[w][0] = longest;
  }
  if (tid == 0) sh.hit[0] = -1;
  __syncthreads();
  const unsigned C = part_blocks<M, K>((sh.w[0] + sh.w[1]) + (sh.w[2] + sh.w[3]), target);
  // kSinks: pieces of long requests come first.  Windows make most of them equally long, and more of them than run at
  // once: what begins last should be short.  (256 requests of up to 4064 keys: 155 -> 143 us.)
  bool first = false;   // piece x is one of those
  if (K == kSinks && !merge) {
    longest = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) longest = sh.s[i][0] > longest ? sh.s[i][0] : longest;
    int n = 0;
    for (int r = tid; r < a.R; r += 256) {
      const Request q = r == tid ? q0 : request_of<M, K>(a, r);
      if (2 * q.blocks > longest) n += q.tiles * parts_of(q, C);
    }
    n = wave_sums(n);
    __syncthreads();
    if (lane == 63) sh.s[w][0] = n;
    __syncthreads();
    n = (sh.s[0][0] + sh.s[1][0]) + (sh.s[2][0] + sh.s[3][0]);
    first = x < n;
    if (!first) x -= n;
    __syncthreads();
  }
  int base = 0, slot = 0;
  for (int r0 = 0; r0 < a.R; r0 += 256) {
    const int r = r0 + tid;
    Request q = {};
    if (r < a.R) q = r0 == 0 ? q0 : request_of<M, K>(a, r);
    const int n = parts_of(q, C);
    const int split = n > 1 ? q.tiles * n : 0, mine = merge ? (n > 1 ? q.tiles : 0) : K == kSinks && (2 * q.blocks > longest) != first ? 0 : q.tiles * n;
    const int s0 = wave_sums(mine), s1 = wave_sums(split);
    if (lane == 63) {
      sh.s[w][0] = s0;
      sh.s[w][1] = s1;
    }
    __syncthreads();
    int t0 = 0, t1 = 0, p0 = 0, p1 = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (i < w) {
        p0 += sh.s[i][0];
        p1 += sh.s[i][1];
      }
      t0 += sh.s[i][0];
      t1 += sh.s[i][1];
    }
    const int from = base + p0 + s0 - mine;
    if (x >= from && x < from + mine) {
      const int found[10] = {r, x - from, n, slot + p1 + s1 - split, q.q0, q.ql, q.n, q.first, q.tiles, q.blocks};
#pragma unroll
      for (int i = 0; i < 10; ++i) sh.hit[i] = found[i];
    }
    base += t0;
    slot += t1;
    __syncthreads();
    if (x < base) break;   // found
  }
  // the same in every lane, and known to be: loops and addresses stay scalar
  auto take = [&](int i) { return __builtin_amdgcn_readfirstlane(sh.hit[i]); };
  if (take(0) < 0) return false;
  finish(take(0), take(1), take(2), take(3), {take(4), take(5), take(6), take(7), take(8), take(9)});
  return true;
}

// ------------------------------------------------------------------- rows --

// A finished row in a wave, D / 64 neighbouring channels per lane: normalised,
// turned back where V was rotated, rounded once and stored.  l == 0: no key
// was left by the mask, the row is 0 and its lse -infinity.
template <int D>
__device__ __forceinline__ void finish_row(const CacheAttnArgs& a, int row_token, int head, float (&y)[D / 64], float m,
                                           float l, int lane) {
  const float inv = l == 0.0f ? 0.0f : 1.0f / l;
#pragma unroll
  for (int i = 0; i < D / 64; ++i) y[i] *= inv;
  if (a.vhad) {
    butterfly_regs(y);
    butterfly_lanes<1>(y, lane);
    butterfly_lanes<2>(y, lane);
    butterfly_lanes<4>(y, lane);
    butterfly_lanes<8>(y, lane);
    butterfly_lanes<16>(y, lane);
    butterfly_lanes<32>(y, lane);
#pragma unroll
    for (int i = 0; i < D / 64; ++i) y[i] *= D == 128 ? 0.0883883476483184405501055452631f : 0.125f;
  }
  const int64_t at = (static_cast<int64_t>(row_token) * a.Hq + head) * D + lane * (D / 64);
  if (a.out_dtype == RA_FP32) {
    float* o = static_cast<float*>(a.o) + at;
#pragma unroll
    for (int i = 0; i < D / 64; ++i) o[i] = y[i];
  } else {
    const bool h = a.out_dtype == RA_FP16;
    uint16_t* o = static_cast<uint16_t*>(a.o) + at;
    if constexpr (D == 128) *reinterpret_cast<uint32_t*>(o) = pack16(y[0], y[1], h);
    else *o = static_cast<uint16_t>(pack16(y[0], 0.0f, h));
  }
  if (a.lse && lane == 0)
    a.lse[static_cast<int64_t>(row_token) * a.Hq + head] = l == 0.0f ? kNegInf : (m + log2f(l)) * kLn2;
}

// 2^(m - M) for a partial result whose maximum is m, 0 where it saw no key.
__device__ __forceinline__ float rescale(float m, float M) { return m == kNegInf ? 0.0f : exp2f(m - M); }

// The blocks of keys that a tile goes through, numbered without gaps.  kSinks:
// those of the first tokens, then those of the window, `skip` blocks on.
template <Keys K>
struct Span {
  int first, total;   // numbers first .. total - 1 (kSinks: from 0)
  int sinks, skip;    // blocks of the first tokens, and of the gap behind them
  __device__ __forceinline__ Span(const CacheAttnArgs& a, int lo, int hi) {
    first = lo / kBlock;
    total = hi > lo ? (hi + kBlock - 1) / kBlock : first;
    sinks = skip = 0;
    if constexpr (K == kSinks) {
      const int s = a.sinks < hi ? a.sinks : hi;
      sinks = s > 0 ? (s + kBlock - 1) / kBlock : 0;
      skip = first > sinks ? first - sinks : 0;
      total = total - skip > sinks ? total - skip : sinks;
      first = 0;
    }
  }
  // of a number in units of 1 / per block
  __device__ __forceinline__ int real(int x, int per) const {
    if constexpr (K == kSinks) return x < sinks * per ? x : x + skip * per;
    return x;
  }
  // how many numbers lie before block b
  __device__ __forceinline__ int before(int b) const {
    if constexpr (K == kSinks) return b <= sinks ? b : b - skip > sinks ? b - skip : sinks;
    return b;
  }
};

// Place in the workspace of a row's part, kShared: parts of requests of few rows from the
// front, of many from the back; -1 where lengths on the device do not fit the call.
template <bool MANY>
__device__ __forceinline__ int64_t shared_at(const CacheAttnArgs& a, int base, int parts, int part, int rows, int row, int h) {
  const int64_t i = static_cast<int64_t>(base) + static_cast<int64_t>(part) * rows + row;
  if (base < 0 || part < 0 || part >= parts || i < 0 || i >= a.part_rows) return -1;
  return (MANY ? a.part_rows - 1 - i : i) * a.g.Hkv + h;
}
// A piece's rows' positions come with the call where their requests differ.
__device__ __forceinline__ int row_position(const CacheAttnArgs& a, const Piece& p, int row) {
  if (p.r >= a.groups) return p.q.first + row / a.G;
  return row < p.q.ql * a.G ? a.positions[p.q.q0 + row / a.G] : 0x3fffffff;
}
// Piece x of the list for few (0) or many (1) rows: {request, tile, part, parts}; of a request {q0, ql, n, first}, {lo, table, slot, two}.
template <int MANY>
__device__ __forceinline__ bool listed_piece(const CacheAttnArgs& a, int x, Piece* out) {
  if (x >= __builtin_amdgcn_readfirstlane(a.counts[MANY])) return false;
  auto all = [](int v) { return __builtin_amdgcn_readfirstlane(v); };
  const int4 c = a.pieces[MANY][x];
  out->r = all(c.x);
  out->tile = all(c.y);
  out->part = all(c.z);
  out->parts = all(c.w);
  const int4 u = a.requests[2 * out->r], v = a.requests[2 * out->r + 1];
  out->q.q0 = all(u.x);
  out->q.ql = all(u.y);
  out->q.n = all(u.z);
  out->q.first = all(u.w);
  out->q.lo = all(v.x);
  out->q.table = all(v.y);
  out->slot = all(v.z);
  out->two = all(v.w);
  out->q.tiles = out->q.blocks = 0;
  return true;
}
template <int M, Keys K>
__device__ __forceinline__ bool take_piece(const CacheAttnArgs& a, SchedShared& sh, int x, int target, Piece* out) {
  if constexpr (K == kShared) return listed_piece<(M > kFewRows)>(a, x, out);
  else return find_piece<M, K>(a, sh, x, false, target, out);
}
// Q of cache_attn_sinks and cache_attn_shared for many rows where it is rotated: a row, scaled by a power of two so that its largest
// element is in [1, 2), as the sum of kTerms digits to the base 32, multiples of 1/8 up to 2 times 32^-z.  An E2M3 code holds such a
// digit (its value times 8 and its sign are the code), and the matrix cores take 6-bit codes of Q and the 4-bit ones of K, as
// they lie in the page, at four times the rate of 16 bits.  Five digits hold every element to within 2^-24 of the row's largest,
// in 20 products of 32 cycles for a wave's 32 rows and 64 keys; two binary16 values need 32, codes turned into
// binary16 and four times the LDS for K.  (sinks_prompt 545 -> 457 us, shared_documents 780 -> 674, shared_decode 98 -> 89;
// four digits would leave 2e-6 of an lse over few keys.)
//
// Every element of a rotated row is a sum of all channels, which binary32 rounds by 2^-24 of its partial sums: no finer, as a
// rule, than digits hold it.  Without the rotation one channel can be far larger than the rest while keys are
// 0 there: what binary32 then holds to 2^-24 of the rest, digits would hold to 2^-24 of that channel (a channel 1000 times the
// others: 2e-4 of a score, 2e-6 in binary32).  There many rows take two binary16 values, as few rows do, 2^-23 of each element
// (sinks_prompt without rotation 441 us with digits, 523 so; shared_documents 675 and 766).
constexpr int kTerms = 5;
// 1.5 * 2^k with k such that adding it leaves multiples of 32^-z / 8
__host__ __device__ constexpr float digit_of(int z) { return 1.5f * (1 << 20 >> (5 * z)); }
template <int D>
__host__ __device__ constexpr int row_bytes6() { return kTerms * D * 3 / 4; }

// 16 bytes of a row's Q, turned and in two values by the launch before: hi of its D channels, then lo.
template <int D>
__device__ __forceinline__ uint4 turned(const CacheAttnArgs& a, const Piece& p, int h, int row, int z, int channel) {
  if (row >= p.q.ql * a.G) return uint4{};
  const int i = row / a.G;
  const int64_t at = static_cast<int64_t>(p.q.q0 + i) * a.Hq + h * a.G + row - i * a.G;
  return *reinterpret_cast<const uint4*>(a.turned + at * 2 * D + z * D + channel);
}
// The lane's half of a row's Q in terms of 6 bits (many rows), as the launch before left it.
template <int D>
__device__ __forceinline__ void turned6(const CacheAttnArgs& a, const Piece& p, int h, int row, int hh, uint32_t (&q)[D / 64][kTerms][6]) {
  uint32_t w[kTerms][D * 3 / 32] = {};
  if (row < p.q.ql * a.G) {
    const int i = row / a.G;
    const int64_t at = static_cast<int64_t>(p.q.q0 + i) * a.Hq + h * a.G + row - i * a.G;
    typedef typename std::conditional<D == 128, uint4, uint2>::type V;
    const V* src = reinterpret_cast<const V*>(a.turned6 + at * row_bytes6<D>() + hh * (D * 3 / 8));
#pragma unroll
    for (int z = 0; z < kTerms; ++z)
#pragma unroll
      for (int i = 0; i < 3; ++i) {
        const V v = src[z * 6 + i];
        constexpr int N = sizeof(V) / 4;
        w[z][N * i] = v.x;
        w[z][N * i + 1] = v.y;
        if constexpr (D == 128) w[z][N * i + 2] = v.z, w[z][N * i + 3] = v.w;
      }
  }
#pragma unroll
  for (int z = 0; z < kTerms; ++z)
#pragma unroll
    for (int i = 0; i < D * 3 / 32; ++i) q[i / 6][z][i % 6] = w[z][i];
}
__device__ __forceinline__ float turned_back(const CacheAttnArgs& a, const Piece& p, int h, int row) {
  if (row >= p.q.ql * a.G) return 1.0f;
  const int i = row / a.G;
  return a.back[static_cast<int64_t>(p.q.q0 + i) * a.Hq + h * a.G + row - i * a.G];
}

// ------------------------------------------------------ few rows per request --
//
// A wave takes 16 NT rows and its own part of the keys, 32 per step, in
// registers (NT = 2 at D = 128 spills 12 of its 256): per 16 keys one load each
// of K codes, V codes and their scales, S^T = K Q^T (keys as rows, so that a
// lane holds one query's scores), and O^T += V^T P^T, for which the lane's four
// keys of two 16-key tiles are already the eight that the product's second
// operand wants from it.  V's first operand, eight keys of one channel, comes from the four tokens per
// load by exchanging nibbles of neighbouring tokens (two operations for eight
// codes) before the conversion.
//
// Q (scaled) and P * (V's scale) are each the sum of two bf16 values, within
// 2^-17 of each element over the whole range of the scales: the matrix cores
// have time for both.  Outputs are 5e-6 off before their rounding (relative, over
// 130k keys) and lse 4e-5 at most; binary32 products throughout give 6e-7 and
// 3e-6, which 16-bit outputs do not show.  (P in one value saved 2 % of a decode
// step and added half again to a bf16 output's error.)
//
// Bound by HBM, (D + 8) bytes per token and KV head, with the vector units
// close behind: about 235 operations per step, 80 of them conversions of codes.  The
// four waves of a workgroup are joined through LDS, the parts of a split tile
// by k_merge.

template <int D>
struct Tile16 {   // a lane's share of 16 tokens
  typename std::conditional<D == 128, uint4, uint2>::type k, v;
  float4 ks, vs;
};

template <int D>
__device__ __forceinline__ void load_tile(const CacheAttnArgs& a, Tile16<D>& t, int id, int h, int key, int lane) {
  typedef typename std::conditional<D == 128, uint4, uint2>::type V;
  const int page = a.g.page, tok = key & (page - 1);
  const uint8_t* b = a.g.cache + static_cast<uint64_t>(static_cast<unsigned>(id)) * static_cast<uint32_t>(a.g.page_bytes) +
                     static_cast<unsigned>(h * head_bytes<D>(page));
  const int kb = page * D / 2;
  t.k = *reinterpret_cast<const V*>(b + tok * (D / 2) + lane * (D / 8));
  t.v = *reinterpret_cast<const V*>(b + kb + tok * (D / 2) + lane * (D / 8));
  const float* sc = reinterpret_cast<const float*>(b + 2 * kb) + tok + (lane >> 4) * 4;
  t.ks = *reinterpret_cast<const float4*>(sc);
  t.vs = *reinterpret_cast<const float4*>(sc + page);
}

// Lets the matrix products that write x finish: for uses behind control flow.
template <typename V>
__device__ __forceinline__ void settle(V& x) {
#if defined(__HIP_DEVICE_COMPILE__)
  asm volatile("s_nop 15\n\ts_nop 7" : "+v"(x));
#else
  (void)x;
#endif
}

// Keeps what is computed from x behind this place (the compiler otherwise moves
// it up to where x is loaded, and waits there).
template <typename V>
__device__ __forceinline__ void pin(V& x) {
#if defined(__HIP_DEVICE_COMPILE__)
  asm volatile("" : "+v"(x));
#else
  (void)x;
#endif
}

template <int B>
__device__ __forceinline__ v2bf codes2(uint32_t w) { return __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, 1.0f, B); }

__device__ __forceinline__ v8bf join(v2bf a, v2bf b, v2bf c, v2bf d) {
  return v8bf{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

constexpr uint32_t kLow = 0x0f0f0f0fu;
// nibbles of two tokens: channel pairs' even / odd channels, token 0 low
__device__ __forceinline__ uint32_t even_of(uint32_t a, uint32_t b) { return (a & kLow) | ((b << 4) & ~kLow); }
__device__ __forceinline__ uint32_t odd_of(uint32_t a, uint32_t b) { return ((a >> 4) & kLow) | (b & ~kLow); }

// ---- binary32 outputs (FINE) ----
//
// Two bf16 values of Q and P would show in binary32 outputs.  There Q is two
// binary16 values, 2^-23 of each element (and 2^-39 of the row's largest), of
// the row times the power of two that brings its largest to [2^14, 2^15); K's
// codes are exact in either type, and the power goes back with K's scale.  P *
// (V's scale), whose range no row bounds, is three bf16 values.  Outputs are
// then 4e-7 off and lse 4e-6 at most, no more than with binary32 products; 64
// requests of 564k keys take 140 us (135 with two bf16 values of both), prompts
// of 26k tokens 3.0 ms (2.5).
__device__ __forceinline__ float row_power(float largest) {
  const int up = 141 - static_cast<int>((__float_as_uint(largest) >> 23) & 0xff);
  return __uint_as_float(static_cast<uint32_t>(127 + (up > 120 ? 120 : up)) << 23);
}
__device__ __forceinline__ float inverse_power(float power) { return __uint_as_float((254u << 23) - __float_as_uint(power)); }

// x = hi + lo, both of the 16-bit type, for each of eight values.  What is left
// over is taken from hi's bits: another conversion may round a tie the other way.
__device__ __forceinline__ void split8(const float* x, bool fp16, uint4& hi, uint4& lo) {
  uint32_t h[4], l[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    h[e] = pack16(x[2 * e], x[2 * e + 1], fp16);
    pin(h[e]);
    l[e] = pack16(x[2 * e] - cache_h2f(static_cast<uint16_t>(h[e] & 0xffff), fp16),
                  x[2 * e + 1] - cache_h2f(static_cast<uint16_t>(h[e] >> 16), fp16), fp16);
  }
  hi = make_uint4(h[0], h[1], h[2], h[3]);
  lo = make_uint4(l[0], l[1], l[2], l[3]);
}

// codes, two per 32 bits, as either 16-bit type
template <bool F16, int B>
__device__ __forceinline__ uint32_t codes2_bits(uint32_t w) {
  if constexpr (F16) return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, 1.0f, B));
  else return __builtin_bit_cast(uint32_t, codes2<B>(w));
}
template <bool F16>
__device__ __forceinline__ uint4 codes8(uint32_t w) {
  return make_uint4(codes2_bits<F16, 0>(w), codes2_bits<F16, 1>(w), codes2_bits<F16, 2>(w), codes2_bits<F16, 3>(w));
}
template <bool FINE>
__device__ __forceinline__ v4f score16(uint4 k, uint4 q, v4f c) {
  if constexpr (FINE)
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(v8h, k), __builtin_bit_cast(v8h, q), c, 0, 0, 0);
  else
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(v8bf, k), __builtin_bit_cast(v8bf, q), c, 0, 0, 0);
}

// The rows' Q as the second operand of K Q^T: lane = 16 * part + row, its
// D / 4 channels from part * D / 4 on, after RoPE and rotation.  Returns what
// the row's scores are to be multiplied by.
template <int D, bool FINE>
__device__ __forceinline__ float load_q(const CacheAttnArgs& a, const Piece& p, int h, int row, int lane,
                                        uint4 (&hi)[D / 32], uint4 (&lo)[D / 32]) {
  constexpr int N = D / 4;
  const int part = lane >> 4;
  const bool ok = row < p.q.ql * a.G;
  const int i = ok ? row / a.G : 0, head = h * a.G + (ok ? row - i * a.G : 0);
  float y[N];
  const uint16_t* src = a.q + static_cast<int64_t>(p.q.q0 + i) * a.q_ts + head * a.q_hs + part * N;
#pragma unroll
  for (int c = 0; c < N / 8; ++c) {
    uint4 w = {};
    if (ok) w = *reinterpret_cast<const uint4*>(src + 8 * c);
    const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      y[8 * c + 2 * e] = cache_h2f(static_cast<uint16_t>(u[e] & 0xffff), a.is_fp16);
      y[8 * c + 2 * e + 1] = cache_h2f(static_cast<uint16_t>(u[e] >> 16), a.is_fp16);
    }
  }
  if (a.rope) {
    int pos = p.q.first + i;
    pos = pos < 0 ? 0 : pos >= a.rope_rows ? a.rope_rows - 1 : pos;
    const float2* cs = reinterpret_cast<const float2*>(a.rope + static_cast<int64_t>(pos) * D) + part * (N / 2);
#pragma unroll
    for (int e = 0; e < N / 2; ++e) {
      const float2 t = cs[e];
      const float u = y[2 * e], v = y[2 * e + 1];
      y[2 * e] = u * t.x - v * t.y;
      y[2 * e + 1] = u * t.y + v * t.x;
    }
  }
  if (a.had) {
    butterfly_regs(y);
    butterfly_lanes<16>(y, lane);
    butterfly_lanes<32>(y, lane);
  }
#pragma unroll
  for (int e = 0; e < N; ++e) y[e] *= a.c;   // scores come out in base 2
  float power = 1.0f;
  if constexpr (FINE) {
    float m = 0.0f;
#pragma unroll
    for (int e = 0; e < N; ++e) m = fmaxf(m, fabsf(y[e]));
    m = fmaxf(m, lane_xor<16>(m));
    power = row_power(fmaxf(m, lane_xor<32>(m)));
#pragma unroll
    for (int e = 0; e < N; ++e) y[e] *= power;
  }
#pragma unroll
  for (int c = 0; c < D / 32; ++c) split8(y + 8 * c, FINE, hi[c], lo[c]);
  return inverse_power(power);
}

template <int D>
__device__ __forceinline__ uint32_t dword_of(const typename std::conditional<D == 128, uint4, uint2>::type& v, int i) {
  if constexpr (D == 128) return i == 0 ? v.x : i == 1 ? v.y : i == 2 ? v.z : v.w;
  else return i == 0 ? v.x : v.y;
}

// Scores are taken relative to a reference per row that moves only when one
// passes it by kSlack (weights up to 2^8 keep their precision in either type):
// x = s * (K's scale) - ref is one operation, and most tiles rescale nothing.
constexpr float kSlack = 8.0f;

// The rows' state in a wave: O^T, reference and sum.  (Q is in LDS, read again
// in every step: in registers it cost a wave per SIMD.)
template <int D, int NT>
struct Rows {
  v4f o[NT][D / 16];
  float m[NT], l[NT];
  float back[NT];       // fine Q: what scores are multiplied by
  int hi[NT], lo[NT];   // keys that the lane's row sees: [lo, hi)
};

// One step of 16 KT keys for the first 16 N rows.  `there` bit i: the i-th 16 keys are on a page; whole:
// every row sees every key.
//
// Control flow here must not skip over a block between a matrix product and the
// first use of its result: the compiler then leaves out the wait states that
// the use needs on the skipping path (seen as wrong first registers when the
// second 16 rows were skipped inside the step).  N is therefore a constant.
// Q is two binary16 values for binary32 outputs, and for all of cache_attn_sinks and cache_attn_shared: their lse is as
// exact as binary32 arithmetic whatever the outputs' type.  (Two bf16 values left 2e-6 of an lse over few keys.)
// For many rows these hold a rotated Q as digits.
template <bool FINE, Keys K>
constexpr bool fine_q() { return FINE || K != kAll; }

template <int D, int NT, int N, int KT, bool FINE, Keys K>
__device__ __forceinline__ void few_step(Rows<D, NT>& x, const uint4* sq, const Tile16<D> (&t)[KT], unsigned there, bool whole, int key0,
                                          int g, int sinks) {
  constexpr int KC = D / 32;
  constexpr bool QF = fine_q<FINE, K>();
  v4f s[N][KT];
#pragma unroll
  for (int i = 0; i < KT; ++i) {
#pragma unroll
    for (int nt = 0; nt < N; ++nt) s[nt][i] = v4f{0, 0, 0, 0};
#pragma unroll
    for (int c = 0; c < KC; ++c) {
      const uint4 k = codes8<QF>(dword_of<D>(t[i].k, c));
#pragma unroll
      for (int nt = 0; nt < N; ++nt) {
        s[nt][i] = score16<QF>(k, sq[(nt * KC + c) * 128], s[nt][i]);
        s[nt][i] = score16<QF>(k, sq[(nt * KC + c) * 128 + 64], s[nt][i]);
      }
    }
    const float ks[4] = {t[i].ks.x, t[i].ks.y, t[i].ks.z, t[i].ks.w};
#pragma unroll
    for (int nt = 0; nt < N; ++nt) {
      const float base = x.m[nt] == kNegInf ? 0.0f : x.m[nt];
#pragma unroll
      for (int e = 0; e < 4; ++e) s[nt][i][e] = __fmaf_rn(s[nt][i][e], QF ? ks[e] * x.back[nt] : ks[e], -base);
    }
  }
  constexpr int PN = FINE ? 3 : 2;
  v8bf pw[N][KT / 2][PN];
#pragma unroll
  for (int nt = 0; nt < N; ++nt) {
    unsigned seen = 0xffff;   // bit 4 i + e: this lane's row sees key 16 i + 4 g + e of the step
    if (!whole) {
      seen = 0;
#pragma unroll
      for (int i = 0; i < KT; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int key = key0 + 16 * i + 4 * g + e;
          const bool on = ((there >> i) & 1) && key < x.hi[nt] && (key >= x.lo[nt] || (K == kSinks && key < sinks));
          seen |= static_cast<unsigned>(on) << (4 * i + e);
          s[nt][i][e] = on ? s[nt][i][e] : kNegInf;
        }
    }
    float mx = kNegInf;
#pragma unroll
    for (int i = 0; i < KT; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) mx = fmaxf(mx, s[nt][i][e]);
    mx = fmaxf(mx, lane_xor<16>(mx));
    mx = fmaxf(mx, lane_xor<32>(mx));
    const bool move = x.m[nt] == kNegInf ? mx > kNegInf : mx > kSlack;
    if (__any(move)) {
      const float by = move ? mx : 0.0f;
      const float alpha = x.m[nt] == kNegInf ? 0.0f : __builtin_amdgcn_exp2f(-by);
      x.m[nt] = move ? (x.m[nt] == kNegInf ? 0.0f : x.m[nt]) + by : x.m[nt];
      x.l[nt] *= alpha;
#pragma unroll
      for (int e = 0; e < D / 16; ++e) x.o[nt][e] *= alpha;
#pragma unroll
      for (int i = 0; i < KT; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) s[nt][i][e] -= by;
    }
#pragma unroll
    for (int i = 0; i < KT; ++i) {
      const float vs[4] = {t[i].vs.x, t[i].vs.y, t[i].vs.z, t[i].vs.w};
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float pr = __builtin_amdgcn_exp2f(s[nt][i][e]);
        x.l[nt] += pr;
        float w = pr * vs[e];
        // a scale that is not finite must not reach rows that do not see its token
        if (!whole) w = (seen >> (4 * i + e)) & 1 ? w : 0.0f;
#pragma unroll
        for (int z = 0; z < PN; ++z) {   // w = their sum
          const __bf16 y = static_cast<__bf16>(w);
          pw[nt][i / 2][z][4 * (i % 2) + e] = y;
          w -= static_cast<float>(y);
        }
      }
    }
  }
  // V: eight keys of one channel, channel e of the lane's chunk
#pragma unroll
  for (int u = 0; u < KT / 2; ++u) {
    uint32_t ev[D / 32], od[D / 32];
#pragma unroll
    for (int y = 0; y < 2; ++y) {
      if constexpr (D == 128) {
        const uint4 v = t[2 * u + y].v;
        ev[2 * y] = even_of(v.x, v.y);
        od[2 * y] = odd_of(v.x, v.y);
        ev[2 * y + 1] = even_of(v.z, v.w);
        od[2 * y + 1] = odd_of(v.z, v.w);
      } else {
        const uint2 v = t[2 * u + y].v;
        const uint32_t t02 = (v.x & 0xffffu) | (v.y << 16), t13 = (v.x >> 16) | (v.y & 0xffff0000u);
        ev[y] = even_of(t02, t13);
        od[y] = odd_of(t02, t13);
      }
    }
    auto pv = [&](auto bb, const uint32_t (&n)[D / 32], int e) {
      constexpr int B = decltype(bb)::value;
      v8bf v;
      if constexpr (D == 128) v = join(codes2<B>(n[0]), codes2<B>(n[1]), codes2<B>(n[2]), codes2<B>(n[3]));
      else v = join(codes2<B>(n[0]), codes2<B + 2>(n[0]), codes2<B>(n[1]), codes2<B + 2>(n[1]));
#pragma unroll
      for (int nt = 0; nt < N; ++nt)
#pragma unroll
        for (int z = 0; z < PN; ++z)
          x.o[nt][e] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, pw[nt][u][z], x.o[nt][e], 0, 0, 0);
    };
    pv(std::integral_constant<int, 0>{}, ev, 0);
    pv(std::integral_constant<int, 0>{}, od, 1);
    pv(std::integral_constant<int, 1>{}, ev, 2);
    pv(std::integral_constant<int, 1>{}, od, 3);
    if constexpr (D == 128) {
      pv(std::integral_constant<int, 2>{}, ev, 4);
      pv(std::integral_constant<int, 2>{}, od, 5);
      pv(std::integral_constant<int, 3>{}, ev, 6);
      pv(std::integral_constant<int, 3>{}, od, 7);
    }
  }
}

template <int D, int NT, bool QF>
struct FewLds {
  static constexpr int M = 16 * NT, kStride = D + 4;   // floats, against bank conflicts
  __align__(16) float so[4][16][kStride];
  float sm[4][M], sl[4][M];
  SchedShared sched;
  __align__(16) uint4 sq_all[NT * (D / 32) * 128];   // [nt][channel step][hi, lo][lane]
  float sback[QF ? M : 1];
};

// Piece x0 of KV head h.
template <int D, int NT, int KT, bool FINE, Keys K>
__device__ __forceinline__ void few_rows(const CacheAttnArgs& a, FewLds<D, NT, fine_q<FINE, K>()>& lds, int x0, int h) {
  constexpr bool QF = fine_q<FINE, K>();
  constexpr int M = 16 * NT, E = D / 16, kStep = 16 * KT, S = kBlock / kStep;
  auto& so = lds.so;
  auto& sm = lds.sm;
  auto& sl = lds.sl;
  auto& sq_all = lds.sq_all;
  auto& sback = lds.sback;
  const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6), g = lane >> 4;
  Piece p;
  if (!take_piece<M, K>(a, lds.sched, x0, a.target, &p)) return;
  const bool prefix = K == kShared && p.r < a.groups;   // causal only: its rows may be at any position

  const int rows = p.q.ql * a.G - p.tile * M < M ? p.q.ql * a.G - p.tile * M : M;   // of this tile
  const int first = p.q.first;
  const int i0 = p.tile * M / a.G, i1 = (p.tile * M + rows - 1) / a.G;
  // keys that any row of the tile sees, and this part of them
  int hi = p.q.n, lo = p.q.lo;
  if (a.causal && !prefix) hi = first + i1 + 1;
  if (hi < 0) hi = 0;
  if (a.window) lo = first + i0 - a.window + 1 > 0 ? first + i0 - a.window + 1 : 0;
  // bounds that every row of the tile sees
  int all_hi = a.causal ? first + i0 + 1 : p.q.n;
  const int all_lo = a.window ? first + i1 - a.window + 1 : p.q.lo;
  const Span<K> span(a, lo, hi);
  const int bl = span.first, bh = span.total;
  const int per = (bh - bl + p.parts - 1) / p.parts;
  const int b0 = bl + p.part * per, b1 = b0 + per < bh ? b0 + per : bh;
  const int wper = (b1 - b0) > 0 ? ((b1 - b0) * S + 3) / 4 : 0;
  const int w0 = b0 * S + w * wper, w1 = w0 + wper < b1 * S ? w0 + wper : b1 * S;   // this wave's steps

  // Page numbers of 64 tiles of 16 keys at a time, one per lane, and of the 64 after them.
  const int page_shift = a.g.page_log - 4;
  const int* row_table = a.block_table + static_cast<int64_t>(K == kShared ? p.q.table : p.r) * a.max_blocks;
  const int last16 = (p.q.n + 15) / 16;   // tiles that hold cached tokens
  auto ids_from = [&](int t16) {   // (looked at when used, so that nothing waits here)
    const int t = span.real(t16 + lane, kBlock / 16);
    return row_table[(t < last16 ? t : last16 - 1) >> page_shift];
  };
  int ids = -1, ids_next = -1;
  if (w0 < w1) {
    ids = ids_from(w0 * KT);
    if (w0 + 64 / KT < w1) ids_next = ids_from(w0 * KT + 64);
  }
  auto load = [&](int b, Tile16<D> (&t)[KT]) {   // steps in order (the last one again); the bits of pages that are there
    const int at = (b - w0) * KT;
    unsigned there = 0;
#pragma unroll
    for (int i = 0; i < KT; ++i) {
      const int id = __builtin_amdgcn_readlane(ids, (at + i) & 63);
      // an entry that is no page leaves its keys out (those behind the end are masked)
      const bool page = static_cast<unsigned>(id) < static_cast<unsigned>(a.g.num_pages);
      there |= static_cast<unsigned>(page) << i;
      load_tile<D>(a, t[i], page ? id : 0, h, (span.real(b, S) * KT + i) * 16, lane);
    }
    if (((at + KT) & 63) == 0 && b + 1 < w1) {   // the next step begins the next 64
      ids = ids_next;
      if (b + 1 + 64 / KT < w1) ids_next = ids_from((b + 1) * KT + 64);
    }
    return there;
  };

  // One step's loads are in flight while another is computed (two in flight
  // cost a wave per SIMD for registers: 564k tokens, 131 against 133 us).
  Tile16<D> ring[2][KT];
  unsigned there[2];
  if (w0 < w1) there[0] = load(w0, ring[0]);

  Rows<D, NT> x;
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    const int row = p.tile * M + nt * 16 + (lane & 15);
    if constexpr (K == kShared) {
      if (w < D / 32) {   // 8 channels of each part of D / 4 for each of the waves
#pragma unroll
        for (int z = 0; z < 2; ++z) sq_all[(w * 2 + z) * 64 + lane] = turned<D>(a, p, h, row, z, g * (D / 4) + w * 8);
      }
      if (w == 0 && lane < 16) sback[lane] = turned_back(a, p, h, row);
    } else if (w == nt) {   // one wave for all four
      uint4 qh[D / 32], ql[D / 32];
      const float back = load_q<D, QF>(a, p, h, row, lane, qh, ql);
      if (QF && lane < 16) sback[nt * 16 + lane] = back;
#pragma unroll
      for (int c = 0; c < D / 32; ++c) {
        sq_all[(nt * (D / 32) + c) * 128 + lane] = qh[c];
        sq_all[(nt * (D / 32) + c) * 128 + 64 + lane] = ql[c];
      }
    }
    const int pos = K == kShared ? row_position(a, p, row) : first + row / a.G;
    x.hi[nt] = a.causal ? pos + 1 : p.q.n;
    if (x.hi[nt] > p.q.n) x.hi[nt] = p.q.n;
    x.lo[nt] = a.window ? pos - a.window + 1 : p.q.lo;
    x.m[nt] = kNegInf;
    x.l[nt] = 0.0f;
#pragma unroll
    for (int e = 0; e < E; ++e) x.o[nt][e] = v4f{0, 0, 0, 0};
  }
  __syncthreads();
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) x.back[nt] = QF ? sback[nt * 16 + (lane & 15)] : 1.0f;
  if constexpr (K == kShared) {
    static_assert(NT == 1, "one product's rows");
    if (prefix) {
      all_hi = x.hi[0];
      auto least = [&](int o) { all_hi = o < all_hi ? o : all_hi; };
      least(lane_xor<1>(all_hi));
      least(lane_xor<2>(all_hi));
      least(lane_xor<4>(all_hi));
      least(lane_xor<8>(all_hi));
      all_hi = __builtin_amdgcn_readfirstlane(all_hi);
    }
  }
  auto whole = [&](int b, unsigned there) {
    const int key = span.real(b, S) * kStep;
    return (key >= all_lo || (K == kSinks && key + kStep <= a.sinks)) && key + kStep <= all_hi && key + kStep <= p.q.n &&
           there == (1u << KT) - 1;
  };
  // Behind the last step the last one is asked for again, so that every step
  // waits for its own loads alone.
  auto run = [&](auto nn) {
    constexpr int N = decltype(nn)::value;
    for (int b = w0; b < w1; b += 2) {
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        if (b + i >= w1) break;
        there[i ^ 1] = load(b + i + 1 < w1 ? b + i + 1 : w1 - 1, ring[i ^ 1]);
        __builtin_amdgcn_sched_barrier(0);
        few_step<D, NT, N, KT, FINE, K>(x, sq_all + lane, ring[i], there[i], whole(b + i, there[i]), span.real(b + i, S) * kStep, g,
                                        a.sinks);
      }
    }
  };
  if (NT == 1 || rows <= 16) run(std::integral_constant<int, 1>{});
  else run(std::integral_constant<int, NT>{});
#pragma unroll
  for (int nt = 0; nt < NT; ++nt)
#pragma unroll
    for (int e = 0; e < E; ++e) settle(x.o[nt][e]);

  // join the four waves
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    x.l[nt] += lane_xor<16>(x.l[nt]);
    x.l[nt] += lane_xor<32>(x.l[nt]);
    if (lane < 16) {
      sm[w][nt * 16 + lane] = x.m[nt];
      sl[w][nt * 16 + lane] = x.l[nt];
    }
  }
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    __syncthreads();
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      float* dst = &so[w][lane & 15][(g * 4 + r) * E];
#pragma unroll
      for (int e = 0; e < E; e += 4)
        *reinterpret_cast<float4*>(dst + e) = make_float4(x.o[nt][e][r], x.o[nt][e + 1][r], x.o[nt][e + 2][r], x.o[nt][e + 3][r]);
    }
    __syncthreads();
    for (int rr = w; rr < 16; rr += 4) {
      const int row = nt * 16 + rr;
      if (row >= rows) break;
      float mm = sm[0][row];
#pragma unroll
      for (int i = 1; i < 4; ++i) mm = fmaxf(mm, sm[i][row]);
      float ll = 0.0f, y[D / 64] = {};
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float f = rescale(sm[i][row], mm);
        ll += f * sl[i][row];
#pragma unroll
        for (int z = 0; z < D / 64; ++z) y[z] += f * so[i][rr][lane * (D / 64) + z];
      }
      if (K != kShared && p.parts == 1) {
        const int i = (p.tile * M + row) / a.G;
        finish_row<D>(a, p.q.q0 + i, h * a.G + p.tile * M + row - i * a.G, y, mm, ll, lane);
      } else {
        int64_t at = (static_cast<int64_t>(p.slot + p.part) * a.g.Hkv + h) * M + row;
        if constexpr (K == kShared) {
          at = shared_at<false>(a, p.slot, p.parts, p.part, p.q.ql * a.G, row, h);
          if (at < 0) continue;
        }
#pragma unroll
        for (int z = 0; z < D / 64; ++z) a.part_o[at * D + lane * (D / 64) + z] = y[z];
        if (lane == 0) a.part_ml[at] = make_float2(mm, ll);
      }
    }
  }
}

// --------------------------------------------------------- many rows per request --
//
// Bound by the matrix cores and the softmax beside them.  NW waves of 32 rows
// share tiles of 64 keys in LDS, as bf16 values of the codes (exact; K of the operators with digits as it
// lies in the page), scales apart: each wave loads its share of the next tile's codes while the present
// one is computed, and converts them into the other LDS buffer at its end.
// S^T = K Q^T and O^T += V^T P^T on the 32x32x16 product: a lane holds one
// query's scores (key 32 c + 8 (r / 4) + 4 hh + r % 4 in register r of chunk
// c), which rounded to 16 bits are the second operand of the next product, and
// the same query's output, so that rescaling it is a factor per lane.
//
// Q (after RoPE, rotation and scale, in binary32) is for cache_attn the sum of two bf16
// values, within 2^-17 of each element.  P * (V's scale) is one, within 2^-8,
// where the output is bf16, which is then 2.3e-3 off (relative) instead of
// 1.7e-3, and two (LO) where it is binary16: prompts of 26k tokens take 2.0 ms
// with one and 2.5 ms with two.  (Binary32 outputs: FINE, above.)  Both are bf16
// for binary16 inputs as well, whose range holds neither a scaled Q (the softmax
// scale is the caller's) nor a weight up to 2^8 times a scale from 2^-100 to
// 2^127: in units of a tile's largest scale, binary16 loses the rows that do not
// see that token.
//
// LDS: K [chunk of 8 channels][key] (as digits meet it: [chunk of 32 channels][key]), V [octet of keys][channel position], 16
// bytes each, read by 32 neighbouring lanes in a row without bank conflicts.
// Channel d of V sits at position (d % E) * 16 + d / E, E = D / 16 (its page
// order), an octet holds keys 16 s + 4 hh + {0..3, 8..11} of step s.

typedef float v16f __attribute__((ext_vector_type(16)));

__device__ __forceinline__ v16f mfma32(uint4 a, uint4 b, v16f c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(v8bf, a), __builtin_bit_cast(v8bf, b), c, 0, 0, 0);
}
template <bool FINE>
__device__ __forceinline__ v16f score32(uint4 k, uint4 q, v16f c) {
  if constexpr (FINE)
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(v8h, k), __builtin_bit_cast(v8h, q), c, 0, 0, 0);
  else return mfma32(k, q, c);
}

// D / 2 channels of a row after RoPE, rotation and scale.
template <int D, bool F16>
__device__ __forceinline__ void values_q32(const CacheAttnArgs& a, const Piece& p, int h, int row, int lane, float (&y)[D / 2]) {
  constexpr int N = D / 2;
  const int hh = lane >> 5;
  const bool ok = row < p.q.ql * a.G;
  const int i = ok ? row / a.G : 0, head = h * a.G + (ok ? row - i * a.G : 0);
  const uint16_t* src = a.q + static_cast<int64_t>(p.q.q0 + i) * a.q_ts + head * a.q_hs + hh * N;
#pragma unroll
  for (int c = 0; c < N / 8; ++c) {
    uint4 w = {};
    if (ok) w = *reinterpret_cast<const uint4*>(src + 8 * c);
    const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      y[8 * c + 2 * e] = cache_h2f(static_cast<uint16_t>(u[e] & 0xffff), F16);
      y[8 * c + 2 * e + 1] = cache_h2f(static_cast<uint16_t>(u[e] >> 16), F16);
    }
  }
  if (a.rope) {
    int pos = p.q.first + i;
    pos = pos < 0 ? 0 : pos >= a.rope_rows ? a.rope_rows - 1 : pos;
    const float2* cs = reinterpret_cast<const float2*>(a.rope + static_cast<int64_t>(pos) * D) + hh * (N / 2);
#pragma unroll
    for (int e = 0; e < N / 2; ++e) {
      const float2 t = cs[e];
      const float u = y[2 * e], v = y[2 * e + 1];
      y[2 * e] = u * t.x - v * t.y;
      y[2 * e + 1] = u * t.y + v * t.x;
    }
  }
  if (a.had) {
    butterfly_regs(y);
    butterfly_lanes<32>(y, lane);
  }
#pragma unroll
  for (int e = 0; e < N; ++e) y[e] *= a.c;   // scores come out in base 2
}

// As load_q, D / 2 channels per lane.
template <int D, bool F16, bool FINE>
__device__ __forceinline__ float load_q32(const CacheAttnArgs& a, const Piece& p, int h, int row, int lane,
                                          uint4 (&hi)[D / 16], uint4 (&lo)[D / 16]) {
  constexpr int N = D / 2;
  float y[N];
  values_q32<D, F16>(a, p, h, row, lane, y);
  float power = 1.0f;
  if constexpr (FINE) {
    float m = 0.0f;
#pragma unroll
    for (int e = 0; e < N; ++e) m = fmaxf(m, fabsf(y[e]));
    power = row_power(fmaxf(m, lane_xor<32>(m)));
#pragma unroll
    for (int e = 0; e < N; ++e) y[e] *= power;
  }
#pragma unroll
  for (int c = 0; c < N / 8; ++c) split8(y + 8 * c, FINE, hi[c], lo[c]);
  return inverse_power(power);
}

// The lowest n bits (n below 0: none, above 64: all).
__device__ __forceinline__ unsigned long long bits_below(int n) {
  return n <= 0 ? 0ull : n >= 64 ? ~0ull : (1ull << n) - 1;
}

// f(0) .. f(N - 1), each index a compile-time constant
template <typename F, int... I>
__device__ __forceinline__ void each_(F&& f, std::integer_sequence<int, I...>) {
  (f(std::integral_constant<int, I>()), ...);
}
template <int N, typename F>
__device__ __forceinline__ void each(F&& f) {
  each_(f, std::make_integer_sequence<int, N>());
}

// 32 values -> 6-bit codes (E2M3) of value / scale, the two sources interleaved.  The
// instruction writes its result before it has read all of its sources, and reads their first registers a cycle
// early, which the compiler does not know; nor does it see that a product may follow.
__device__ __forceinline__ void pack6(const v16f& even, const v16f& odd, float scale, uint32_t (&to)[6]) {
  typedef uint32_t v6u __attribute__((ext_vector_type(6)));
  v6u r = {};
#if defined(__HIP_DEVICE_COMPILE__)
  asm volatile("s_nop 0\n\tv_cvt_scalef32_2xpk16_fp6_f32 %0, %1, %2, %3\n\ts_nop 1" : "=&v"(r) : "v"(even), "v"(odd), "s"(scale));
#endif
#pragma unroll
  for (int i = 0; i < 6; ++i) to[i] = r[i];
}

// c += K times digit Z of Q: 32 keys, 32 rows, 64 channels.  (The form without scales is a single instruction word.)
template <int Z>
__device__ __forceinline__ v16f score6(uint4 k, const uint32_t (&q)[6], v16f c) {
  typedef int v8i __attribute__((ext_vector_type(8)));
  const v8i A = {static_cast<int>(k.x), static_cast<int>(k.y), static_cast<int>(k.z), static_cast<int>(k.w), 0, 0, 0, 0};
  const v8i B = {static_cast<int>(q[0]), static_cast<int>(q[1]), static_cast<int>(q[2]), static_cast<int>(q[3]),
                 static_cast<int>(q[4]), static_cast<int>(q[5]), 0, 0};
  if constexpr (Z == 0) return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(A, B, c, 4, 2, 0, 0, 0, 0);
  // biased exponents 127 - 5, - 10, - 15, - 20, a byte each
  else return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(A, B, c, 4, 2, 0, 0x7f7f7f7f, Z - 1, 0x6b70757a);
}

// load_q32 as digits.
template <int D, bool F16>
__device__ __forceinline__ float load_q6(const CacheAttnArgs& a, const Piece& p, int h, int row, int lane,
                                         uint32_t (&q)[D / 64][kTerms][6]) {
  constexpr int N = D / 2;
  float y[N];
  values_q32<D, F16>(a, p, h, row, lane, y);
  float m = 0.0f, bad = 0.0f;   // bad: NaN where an element is not finite, which no digit is
#pragma unroll
  for (int e = 0; e < N; ++e) {
    m = fmaxf(m, fabsf(y[e]));
    bad = __fmaf_rn(y[e], 0.0f, bad);
  }
  bad += lane_xor<32>(bad);
  const float power = row_power(fmaxf(m, lane_xor<32>(m))), unit = power * 0x1p-14f;
#pragma unroll
  for (int e = 0; e < N; ++e) y[e] *= unit;
  each<N / 32>([&](auto st) {
    each<kTerms>([&](auto zz) {
      constexpr int z = decltype(zz)::value, n = 32 * decltype(st)::value;
      v16f t[2];
#pragma unroll
      for (int e = 0; e < 32; ++e) {
        float d = y[n + e];
        if constexpr (z + 1 < kTerms) {
          d = (d + digit_of(z)) - digit_of(z);
          y[n + e] -= d;
        }
        t[e & 1][e >> 1] = d;
      }
      pack6(t[0], t[1], 1.0f / (1 << (5 * z)), q[n / 32][z]);
    });
  });
  return inverse_power(power) * 0x1p14f + bad;
}

// Pipeline over tiles: a tile begins with its scores in registers.  Once a
// chunk of 32 keys has its probabilities, its score registers take the next
// tile's scores of that chunk; those products and the chunk's P V run on the
// matrix cores beside the next chunk's probabilities, their LDS operands read
// kAhead products ahead.  So K is staged two tiles ahead and V (with both
// scales) one, and two LDS buffers of each suffice.
// TERMS: bf16 values that hold P * (V's scale); three come with binary16 pairs of Q.
template <int D, bool SIX>
struct TilesLds {
  struct Scales {
    float ks[64], vs[64];
    unsigned long long there, plain;   // keys that are on a page; those of them with a finite V
  };
  __align__(16) uint4 k[2][SIX ? D / 32 : D / 8][64];   // chunks of 8 channels in 16 bits, of 32 in 4
  __align__(16) uint4 v[2][8][D];
  Scales sc[2];
};
template <int D, Keys K>
struct RowsLds {
  union {
    TilesLds<D, false> pairs;
    TilesLds<D, K != kAll> six;
  };
  SchedShared sched;   // (read while the first waves fill tiles)
};

// Piece p of KV head h.  SIX: Q as digits, K as it lies in the page.
template <int D, bool F16, int TERMS, Keys K, bool SIX>
__device__ __forceinline__ void many_rows(const CacheAttnArgs& a, TilesLds<D, SIX>& buf, Piece p, int h) {
  constexpr bool QF = fine_q<TERMS == 3, K>();   // scores are multiplied by `back`
  typedef typename std::conditional<D == 128, uint4, uint2>::type Codes;   // a lane's share of 16 tokens
  constexpr int NW = 4, M = 32 * NW, E = D / 16, KC = D / 16, MT = D / 32;
  typedef typename TilesLds<D, SIX>::Scales Scales;
  const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int hh = lane >> 5, j = lane & 31;
  const bool prefix = K == kShared && p.r < a.groups;   // causal only: its rows may be at any position
  if (K != kShared && a.causal) p.tile = p.q.tiles - 1 - p.tile;   // the longest first

  const int rows = p.q.ql * a.G - p.tile * M < M ? p.q.ql * a.G - p.tile * M : M;
  const int first = p.q.first;
  const int i0 = p.tile * M / a.G, i1 = (p.tile * M + rows - 1) / a.G;
  int hi = p.q.n, lo = p.q.lo;
  if (a.causal && !prefix) hi = first + i1 + 1;
  if (hi < 0) hi = 0;
  if (a.window) lo = first + i0 - a.window + 1 > 0 ? first + i0 - a.window + 1 : 0;
  const Span<K> span(a, lo, hi);
  const int bl = span.first, bh = span.total;
  const int per = (bh - bl + p.parts - 1) / p.parts;
  const int b0 = bl + p.part * per, b1 = b0 + per < bh ? b0 + per : bh;
  // bounds that every row of this wave sees, and its lane's row
  const int wrow = p.tile * M + w * 32, row = wrow + j;
  const int wi0 = wrow / a.G, wi1 = wrow + 31 < p.tile * M + rows - 1 ? (wrow + 31) / a.G : i1;
  int all_hi = a.causal ? first + wi0 + 1 : p.q.n;
  const int all_lo = a.window ? first + wi1 - a.window + 1 : p.q.lo;
  // tiles from t1 on hold no key that a row of this wave sees; a wave behind the rows of the tile has none at all
  int t1 = a.causal && !prefix ? span.before((first + wi1 + kBlock) / kBlock) : b1;
  if (t1 > b1) t1 = b1;
  if (w * 32 >= rows || t1 < b0) t1 = b0;
  const int pos = K == kShared ? row_position(a, p, row) : first + row / a.G;
  int row_hi = a.causal ? pos + 1 : p.q.n;
  if (row_hi > p.q.n) row_hi = p.q.n;
  const int row_lo = a.window ? pos - a.window + 1 : p.q.lo;
  if constexpr (K == kShared) {
    if (prefix) {
      all_hi = row_hi;
      auto least = [&](int o) { all_hi = o < all_hi ? o : all_hi; };
      least(lane_xor<1>(all_hi));
      least(lane_xor<2>(all_hi));
      least(lane_xor<4>(all_hi));
      least(lane_xor<8>(all_hi));
      least(lane_xor<16>(all_hi));
      all_hi = __builtin_amdgcn_readfirstlane(all_hi);
    }
  }

  const int page = a.g.page, page_log = a.g.page_log;
  const int* row_table = a.block_table + static_cast<int64_t>(K == kShared ? p.q.table : p.r) * a.max_blocks;
  const uint8_t* head_base = a.g.cache + static_cast<int64_t>(h) * head_bytes<D>(page);
  const int kb = page * D / 2;
  // Loads run ahead of their use: what is read here (page numbers one tile
  // before the codes, codes and scales one before the tile) is looked at when
  // it is used, not where it is asked for, which would wait for it there.
  const int last = p.q.n > 0 ? p.q.n - 1 : 0;
  auto entry_of = [&](int t) { return row_table[static_cast<unsigned>(t < last ? t : last) >> page_log]; };
  auto is_page = [&](int id) { return static_cast<unsigned>(id) < static_cast<unsigned>(a.g.num_pages); };
  const uint32_t stride = static_cast<uint32_t>(a.g.page_bytes);   // at most 2^26
  auto page_at = [&](int id) { return head_base + static_cast<uint64_t>(is_page(id) ? id : 0u) * stride; };
  const int mine = w * 16;           // each of the four waves stages 16 tokens of a tile,
  const bool do_s = w == NW - 1;     // the last one the scales too

  Codes sk = {}, sv = {};
  float ks = 0.0f, vs = 0.0f;
  bool here = false;
  int id_k = 0, id_v = 0, id_s = 0;   // table entries of the tiles asked for next
  auto within = [&](int b) { return span.real(b < b1 ? b : b1 - 1, 1); };   // block of keys of a tile's number
  auto entries = [&](int bk, int bv) {
    id_k = entry_of(within(bk) * kBlock + mine);
    id_v = entry_of(within(bv) * kBlock + mine);
    if (do_s) id_s = entry_of(within(bv) * kBlock + lane);
  };
  // K of tile bk and V of tile bv, whose table entries are in hand, then the
  // entries of the tiles after them.  All addresses come first: a use of an
  // entry behind a load would wait for that load.  Past the last tile it is
  // asked for again, so that there are no branches to wait at.
  auto ask = [&](int bk, int bv) {
    const int ck = within(bk), cv = within(bv);
    const int tk = (ck * kBlock + mine) & (page - 1), tv = (cv * kBlock + mine) & (page - 1);
    const int g = ((lane >> 4) & 1) * 2 + hh;   // V: lane = chunk + 16 * (half of the octet) + 32 * hh, tokens 4 g ..
    const uint8_t* pk = page_at(__builtin_amdgcn_readfirstlane(id_k)) + tk * (D / 2) + lane * (D / 8);
    const uint8_t* pv =
        page_at(__builtin_amdgcn_readfirstlane(id_v)) + kb + tv * (D / 2) + (g * 16 + (lane & 15)) * (D / 8);
    if (do_s) {
      const int t = cv * kBlock + lane;
      here = is_page(id_s) && t < p.q.n;
      const float* sc = reinterpret_cast<const float*>(page_at(id_s) + 2 * kb) + (t & (page - 1));
      ks = sc[0];
      vs = sc[page];
    }
    sk = *reinterpret_cast<const Codes*>(pk);
    sv = *reinterpret_cast<const Codes*>(pv);
    if constexpr (K == kSinks) entries(bk + 1, bv + 1);
    else entries(ck + 1, cv + 1);
  };
  // The staged codes into LDS, in four parts each.  What is written past the
  // last tile replaces tiles that are done with.
  auto put_k = [&](int b, auto part) {
    constexpr int c = decltype(part)::value;
    if constexpr (SIX) {
      if constexpr (c == 0) {   // chunks of 16 channels are put together where D is 64
        if constexpr (D == 128) buf.k[b & 1][lane >> 4][mine + (lane & 15)] = sk;
        else reinterpret_cast<uint2*>(&buf.k[b & 1][hh][mine + (lane & 15)])[(lane >> 4) & 1] = sk;
      }
    } else if constexpr (c < D / 32) {
      const uint32_t x = dword_of<D>(sk, c);
      buf.k[b & 1][(lane >> 4) * (D / 32) + c][mine + (lane & 15)] =
          codes8<QF>(x);
    }
  };
  auto put_v = [&](int b, auto part) {   // channels E / 4 * part .. of the lane's chunk
    constexpr int c = decltype(part)::value;
    // position e * 16 + chunk, half of an octet
    uint2* dst = reinterpret_cast<uint2*>(&buf.v[b & 1][w * 2 + hh][lane & 15]) + ((lane >> 4) & 1);
    if constexpr (D == 128) {
      const uint32_t e01 = even_of(sv.x, sv.y), e23 = even_of(sv.z, sv.w), o01 = odd_of(sv.x, sv.y),
                     o23 = odd_of(sv.z, sv.w);
      dst[2 * c * 32] = make_uint2(codes2_bits<false, c>(e01), codes2_bits<false, c>(e23));
      dst[(2 * c + 1) * 32] = make_uint2(codes2_bits<false, c>(o01), codes2_bits<false, c>(o23));
    } else {
      const uint32_t t02 = (sv.x & 0xffffu) | (sv.y << 16), t13 = (sv.x >> 16) | (sv.y & 0xffff0000u);
      const uint32_t n = c % 2 ? odd_of(t02, t13) : even_of(t02, t13);
      dst[c * 32] = make_uint2(codes2_bits<false, c / 2>(n), codes2_bits<false, c / 2 + 2>(n));
    }
  };
  auto put_scales = [&](int b) {
    if (!do_s) return;
    Scales& t = buf.sc[b & 1];
    // a V scale that is not finite is left out of the sums, which it would
    // enter times 0 for rows that do not see its token
    const bool plain = here && fabsf(vs) < __builtin_inff();
    t.vs[lane] = plain ? vs : 0.0f;
    t.ks[lane] = here ? ks : 0.0f;
    const unsigned long long all = __ballot(here), fine = __ballot(plain);
    if (lane == 0) {
      t.there = all;
      t.plain = fine;
    }
  };
  auto pin_staged = [&] {
    if constexpr (D == 128) {
      pin(sk.x), pin(sk.y), pin(sk.z), pin(sk.w);
      pin(sv.x), pin(sv.y), pin(sv.z), pin(sv.w);
    } else {
      pin(sk.x), pin(sk.y);
      pin(sv.x), pin(sv.y);
    }
  };
  auto put = [&](int bk, int bv) {
    pin_staged();
    each<4>([&](auto part) {
      put_k(bk, part);
      put_v(bv, part);
    });
  };

  if (b0 < b1) {
    entries(b0, b0);
    ask(b0, b0);
  }
  uint4 q[KC], q_lo[KC];            // 16-bit values
  uint32_t q6[D / 64][kTerms][6];   // digits
  float back = 1.0f;
  if constexpr (K == kShared) {
    back = turned_back(a, p, h, row);
    if constexpr (SIX) {
      turned6<D>(a, p, h, row, hh, q6);
      back *= 0x1p14f;
    } else {
#pragma unroll
      for (int kc = 0; kc < KC; ++kc) {
        q[kc] = turned<D>(a, p, h, row, 0, hh * (D / 2) + kc * 8);
        q_lo[kc] = turned<D>(a, p, h, row, 1, hh * (D / 2) + kc * 8);
      }
    }
  } else if constexpr (SIX) {
    back = load_q6<D, F16>(a, p, h, row, lane, q6);
  } else {
    back = load_q32<D, F16, QF>(a, p, h, row, lane, q, q_lo);
  }
  v16f o[MT], s[2];
#pragma unroll
  for (int i = 0; i < MT; ++i)
#pragma unroll
    for (int r = 0; r < 16; ++r) o[i][r] = 0.0f;
  float m = kNegInf, l = 0.0f;
  put(b0, b0);
  put_scales(b0);
  if (b0 < b1) {
    ask(b0 + 1, b0 + 1);   // (this V is asked for again with the first tile)
    each<4>([&](auto part) { put_k(b0 + 1, part); });
    entries(b0 + 2, b0 + 1);
  }
  __syncthreads();

  constexpr int KS = SIX ? D / 64 : KC;   // of a chunk of keys: operands of K, and products
  constexpr int KP = SIX ? KS * kTerms : KC;
  auto k_op = [&](int b, int c, int kc) { return buf.k[b & 1][hh * KS + kc][c * 32 + j]; };
#pragma unroll
  for (int c = 0; c < 2; ++c) {
#pragma unroll
    for (int r = 0; r < 16; ++r) s[c][r] = 0.0f;
    if constexpr (SIX) {
      each<KS>([&](auto st) {
        const uint4 k = k_op(b0, c, st);
        each<kTerms>([&](auto z) { s[c] = score6<kTerms - 1 - z>(k, q6[st][kTerms - 1 - z], s[c]); });
      });
    } else {
#pragma unroll
      for (int kc = 0; kc < KC; ++kc) {
        const uint4 k = k_op(b0, c, kc);
        s[c] = score32<QF>(k, q[kc], s[c]);
        s[c] = score32<QF>(k, q_lo[kc], s[c]);
      }
    }
    settle(s[c]);
  }
  __syncthreads();   // tile b0's K is read before tile b0 + 2's takes its place

  auto step = [&](int b) {
    // the waves of a SIMD alternate: the dependent chain of vector work at the
    // higher priority, the products behind it at the lower one
    __builtin_amdgcn_s_setprio(1);
    const Scales& t = buf.sc[b & 1];
    const int key0 = span.real(b, 1) * kBlock;
    const float base = m == kNegInf ? 0.0f : m;
    float x[2][16], mx = kNegInf;
#pragma unroll
    for (int c = 0; c < 2; ++c) {
#pragma unroll
      for (int r = 0; r < 16; r += 4) {
        float4 k4 = *reinterpret_cast<const float4*>(&t.ks[c * 32 + 2 * r + 4 * hh]);
        if constexpr (QF) k4.x *= back, k4.y *= back, k4.z *= back, k4.w *= back;
        x[c][r] = __fmaf_rn(s[c][r], k4.x, -base);
        x[c][r + 1] = __fmaf_rn(s[c][r + 1], k4.y, -base);
        x[c][r + 2] = __fmaf_rn(s[c][r + 2], k4.z, -base);
        x[c][r + 3] = __fmaf_rn(s[c][r + 3], k4.w, -base);
      }
    }
    const unsigned long long plain = t.plain;
    if ((key0 < all_lo && !(K == kSinks && key0 + kBlock <= a.sinks)) || key0 + kBlock > all_hi || plain != ~0ull) {
      unsigned long long late = ~bits_below(row_lo - key0);
      if constexpr (K == kSinks) late |= bits_below(a.sinks - key0);
      unsigned long long on = t.there & bits_below(row_hi - key0) & late;
      // rows that see a V that is not finite are NaN from here on (their lse is that of the keys)
      if (__any((on & ~plain) != 0)) {
        const float by = on & ~plain ? __builtin_nanf("") : 1.0f;
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
          for (int r = 0; r < 16; ++r) o[i][r] *= by;
      }
      // the lane's keys of the tile, its own first: bit 32 c + 8 (r / 4) + r % 4
      on >>= 4 * hh;
      const unsigned half[2] = {static_cast<unsigned>(on), static_cast<unsigned>(on >> 32)};
#pragma unroll
      for (int c = 0; c < 2; ++c)
#pragma unroll
        for (int r = 0; r < 16; ++r)
          x[c][r] = half[c] & (1u << (8 * (r >> 2) + (r & 3))) ? x[c][r] : kNegInf;
    }
#pragma unroll
    for (int c = 0; c < 2; ++c)
#pragma unroll
      for (int r = 0; r < 16; r += 2) mx = fmaxf(fmaxf(mx, x[c][r]), x[c][r + 1]);
    mx = fmaxf(mx, lane_xor<32>(mx));
    const bool move = m == kNegInf ? mx > kNegInf : mx > kSlack;
    float alpha = 1.0f;
    if (__any(move)) {
      const float by = move ? mx : 0.0f;
      alpha = m == kNegInf ? 0.0f : __builtin_amdgcn_exp2f(-by);
      m = move ? base + by : m;
      l *= alpha;
#pragma unroll
      for (int c = 0; c < 2; ++c)
#pragma unroll
        for (int r = 0; r < 16; ++r) x[c][r] -= by;
    }
    if (__any(alpha != 1.0f)) {
#pragma unroll
      for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[i][r] *= alpha;
    }

    uint32_t pw[2][TERMS][8];
    float ls[4] = {0, 0, 0, 0};
    auto v_scales = [&](int n) { return *reinterpret_cast<const float4*>(&t.vs[8 * n + 4 * hh]); };
    float4 v4 = v_scales(0);   // read a group ahead
    auto probs = [&](int c, int r4) {   // registers 4 r4 .. 4 r4 + 3 of chunk c
      const float vv[4] = {v4.x, v4.y, v4.z, v4.w};
      if (4 * c + r4 < 7) v4 = v_scales(4 * c + r4 + 1);
      float y[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float pr = __builtin_amdgcn_exp2f(x[c][4 * r4 + e]);
        ls[e] += pr;
        y[e] = pr * vv[e];
      }
#pragma unroll
      for (int e = 0; e < 2; ++e)
#pragma unroll
        for (int z = 0; z < TERMS; ++z) {   // y = the sum of the terms
          uint32_t u = pack16(y[2 * e], y[2 * e + 1], false);
          if (z + 1 < TERMS) {
            pin(u);   // what is left over is taken from these bits, not from a second conversion
            y[2 * e] -= cache_h2f(static_cast<uint16_t>(u & 0xffff), false);
            y[2 * e + 1] -= cache_h2f(static_cast<uint16_t>(u >> 16), false);
          }
          pw[c][z][2 * r4 + e] = u;
        }
    };
    // products of chunk c, in turn: one of the 2 MT of P V (step n / MT, tile n %
    // MT), one of the KC score products of chunk c of the next tile, whose sum
    // is one chain (behind the last tile they take what lies there and nothing
    // reads them: a second form of this code costs more than they do)
    static_assert(2 * MT == KC, "as many of either");
    if constexpr (SIX) {
      // the same with the operands of K in hand for a whole chunk, and KP / (2 MT) products of the scores for one of P V
      constexpr int NV = 2 * MT, kAhead = TERMS == 3 ? 2 : 4, NB = KS == 1 ? 2 : 1;   // of K: the next chunk's takes the place of what is done with
      auto operand = [&](int c, int i) { return buf.v[b & 1][(c * 2 + i / MT) * 2 + hh][(i % MT) * 32 + j]; };
      uint4 ops[kAhead], ks[NB][KS];
#pragma unroll
      for (int i = 0; i < kAhead; ++i) ops[i] = operand(0, i);
#pragma unroll
      for (int i = 0; i < KS; ++i) ks[0][i] = k_op(b + 1, 0, i);
#pragma unroll
      for (int r4 = 0; r4 < 4; ++r4) probs(0, r4);
      __builtin_amdgcn_sched_barrier(0);
      each<2>([&](auto cc) {
        constexpr int c = decltype(cc)::value;
        each<NV>([&](auto ii) {
          constexpr int i = decltype(ii)::value, n = c * NV + i + kAhead;
          uint4& op = ops[(c * NV + i) % kAhead];
#pragma unroll
          for (int z = 0; z < TERMS; ++z) {
            const uint32_t* w = pw[c][z] + 4 * (i / MT);
            o[i % MT] = mfma32(op, make_uint4(w[0], w[1], w[2], w[3]), o[i % MT]);
          }
          if constexpr (n < 2 * NV) op = operand(n / NV, n % NV);
          if constexpr (c == 0 && NB == 2 && i == 0) ks[NB - 1][0] = k_op(b + 1, 1, 0);
          if constexpr (i == 0)
#pragma unroll
            for (int r = 0; r < 16; ++r) s[c][r] = 0.0f;
          constexpr int x0 = i * KP / NV, x1 = (i + 1) * KP / NV;
          each<x1 - x0>([&](auto xx) {
            constexpr int x = x0 + decltype(xx)::value, z = kTerms - 1 - x % kTerms;
            s[c] = score6<z>(ks[c % NB][x / kTerms], q6[x / kTerms][z], s[c]);
            if constexpr (c == 0 && NB == 1 && z == 0) ks[0][x / kTerms] = k_op(b + 1, 1, x / kTerms);
          });
          if constexpr (i % (NV / 4) == NV / 4 - 1) {
            if constexpr (c == 0) {
              probs(1, i / (NV / 4));
            } else {
              put_k(b + 2, std::integral_constant<int, i / (NV / 4)>{});
              put_v(b + 1, std::integral_constant<int, i / (NV / 4)>{});
            }
          }
          __builtin_amdgcn_sched_barrier(0);
        });
        if constexpr (c == 0) {
          __builtin_amdgcn_s_setprio(0);
          pin_staged();
        }
      });
      l += (ls[0] + ls[1]) + (ls[2] + ls[3]);
      return;
    }
    constexpr int NP = 2 * MT + KC, kAhead = 4;
    auto operand = [&](int c, int i) {
      const int n = i / 2;
      return i % 2 == 0 ? buf.v[b & 1][(c * 2 + n / MT) * 2 + hh][(n % MT) * 32 + j] : k_op(b + 1, c, n);
    };
#pragma unroll
    for (int r4 = 0; r4 < 4; ++r4) probs(0, r4);
    uint4 ops[kAhead];
#pragma unroll
    for (int i = 0; i < kAhead; ++i) ops[i] = operand(0, i);
    __builtin_amdgcn_sched_barrier(0);
    each<2>([&](auto cc) {
      constexpr int c = decltype(cc)::value;
      each<NP>([&](auto ii) {
        constexpr int i = decltype(ii)::value;
        uint4& op = ops[(c * NP + i) % kAhead];
        if constexpr (i % 2 == 0) {
          constexpr int st = i / 2 / MT;
#pragma unroll
          for (int z = 0; z < TERMS; ++z) {
            const uint32_t* w = pw[c][z] + 4 * st;
            o[i / 2 % MT] = mfma32(op, make_uint4(w[0], w[1], w[2], w[3]), o[i / 2 % MT]);
          }
        } else {
          if constexpr (i == 1)
#pragma unroll
            for (int r = 0; r < 16; ++r) s[c][r] = 0.0f;
          s[c] = score32<QF>(op, q[i / 2], s[c]);
          s[c] = score32<QF>(op, q_lo[i / 2], s[c]);
        }
        constexpr int n = c * NP + i + kAhead;
        if constexpr (n < 2 * NP) op = operand(n / NP, n % NP);
        // beside chunk 0's products chunk 1's probabilities, beside chunk 1's
        // the next tiles' codes
        if constexpr (i % (NP / 4) == NP / 4 - 1) {
          if constexpr (c == 0) {
            probs(1, i / (NP / 4));
          } else {
            put_k(b + 2, std::integral_constant<int, i / (NP / 4)>{});
            put_v(b + 1, std::integral_constant<int, i / (NP / 4)>{});
          }
        }
        __builtin_amdgcn_sched_barrier(0);
      });
      if constexpr (c == 0) {
        __builtin_amdgcn_s_setprio(0);
        pin_staged();
      }
    });
    l += (ls[0] + ls[1]) + (ls[2] + ls[3]);
  };

  for (int b = b0; b < b1; ++b) {
    ask(b + 2, b + 1);
    if (b < t1) step(b);
    else put(b + 2, b + 1);
    put_scales(b + 1);
    __syncthreads();
  }
#pragma unroll
  for (int i = 0; i < MT; ++i) settle(o[i]);

  // Out of the registers: of its row a lane holds half of the chunks of E
  // channels, register r of tile i being channel e = 2 i + r / 8 of chunk 8 (r / 4 % 2) + 4 hh + r % 4.
  // (Through LDS, a row at a time in whole lines, it took 9 of a piece's 66 us with two pieces per
  // compute unit; the L2 joins the lines that are written in parts here.)
  l += lane_xor<32>(l);
  float y[E][8];   // [channel of a chunk][chunk 8 (c / 4) + 4 hh + c % 4]
#pragma unroll
  for (int e = 0; e < E; ++e)
#pragma unroll
    for (int c = 0; c < 8; ++c) y[e][c] = o[e >> 1][8 * (e & 1) + c];
  const int rr = w * 32 + j;
  if (K == kShared || p.parts != 1) {
    int64_t at = (static_cast<int64_t>(p.slot + p.part) * a.g.Hkv + h) * M + rr;
    if constexpr (K == kShared) at = shared_at<true>(a, p.slot, p.parts, p.part, p.q.ql * a.G, p.tile * M + rr, h);
    if (rr >= rows || at < 0) return;
    float* dst = a.part_o + at * D + 4 * hh * E;
#pragma unroll
    for (int c = 0; c < 8; ++c)
#pragma unroll
      for (int e = 0; e < E; e += 4)
        *reinterpret_cast<float4*>(dst + (8 * (c >> 2) + (c & 3)) * E + e) = make_float4(y[e][c], y[e + 1][c], y[e + 2][c], y[e + 3][c]);
    if (hh == 0) a.part_ml[at] = make_float2(m, l);
    return;
  }
  // as finish_row
  const float inv = l == 0.0f ? 0.0f : 1.0f / l;
#pragma unroll
  for (int e = 0; e < E; ++e)
#pragma unroll
    for (int c = 0; c < 8; ++c) y[e][c] *= inv;
  if (a.vhad) {
    auto stage = [&](float& u, float& v) {
      const float t = u;
      u = t + v;
      v = t - v;
    };
#pragma unroll
    for (int d = 1; d < E; d *= 2)
#pragma unroll
      for (int e = 0; e < E; ++e)
#pragma unroll
        for (int c = 0; c < 8; ++c)
          if (!(e & d)) stage(y[e][c], y[e + d][c]);
#pragma unroll
    for (int d = 1; d < 4; d *= 2)
#pragma unroll
      for (int e = 0; e < E; ++e)
#pragma unroll
        for (int c = 0; c < 8; ++c)
          if (!(c & d)) stage(y[e][c], y[e][c + d]);
#pragma unroll
    for (int e = 0; e < E; ++e) butterfly_lanes<32>(y[e], lane);
#pragma unroll
    for (int e = 0; e < E; ++e)
#pragma unroll
      for (int c = 0; c < 4; ++c) stage(y[e][c], y[e][c + 4]);
#pragma unroll
    for (int e = 0; e < E; ++e)
#pragma unroll
      for (int c = 0; c < 8; ++c) y[e][c] *= D == 128 ? 0.0883883476483184405501055452631f : 0.125f;
  }
  if (rr >= rows) return;
  const int i = row / a.G;
  const int64_t out = static_cast<int64_t>(p.q.q0 + i) * a.Hq + h * a.G + row - i * a.G;
  const int64_t to = out * D + 4 * hh * E;
#pragma unroll
  for (int c = 0; c < 8; ++c) {
    const int at = (8 * (c >> 2) + (c & 3)) * E;
    if (a.out_dtype == RA_FP32) {
#pragma unroll
      for (int e = 0; e < E; e += 4)
        *reinterpret_cast<float4*>(static_cast<float*>(a.o) + to + at + e) = make_float4(y[e][c], y[e + 1][c], y[e + 2][c], y[e + 3][c]);
    } else {
      const bool f = a.out_dtype == RA_FP16;
      uint32_t u[E / 2];
#pragma unroll
      for (int e = 0; e < E; e += 2) u[e / 2] = pack16(y[e][c], y[e + 1][c], f);
      uint16_t* dst = static_cast<uint16_t*>(a.o) + to + at;
      if constexpr (E == 8) *reinterpret_cast<uint4*>(dst) = make_uint4(u[0], u[1], u[2], u[3]);
      else *reinterpret_cast<uint2*>(dst) = make_uint2(u[0], u[1]);
    }
  }
  if (a.lse && hh == 0) a.lse[out] = l == 0.0f ? kNegInf : (m + log2f(l)) * kLn2;
}

// The kernel's first argument, read again: of several bodies in one kernel each has its own copy, or what they share is loaded
// ahead of them and kept in scalar registers that their loops lack (24 moves out of spilled ones for each tile of keys,
// sinks_prompt 452 us instead of 444).
__device__ __forceinline__ const CacheAttnArgs& own_args() {
  typedef const __attribute__((address_space(4))) CacheAttnArgs* Args;
  Args a = (Args)__builtin_amdgcn_kernarg_segment_ptr();
#if defined(__HIP_DEVICE_COMPILE__)
  asm volatile("" : "+s"(a));
#endif
  return *(const CacheAttnArgs*)a;
}

// Piece x0 of KV head h.  TERMS 1: two for requests of few enough rows.
template <int D, bool F16, int TERMS, Keys K>
__device__ __forceinline__ void rows_piece(const CacheAttnArgs& a, RowsLds<D, K>& buf, int x0, int h) {
  Piece p;
  if (!take_piece<128, K>(a, buf.sched, x0, a.target_rows, &p)) return;
  if constexpr (K == kAll) {
    many_rows<D, F16, TERMS, K, false>(a, buf.pairs, p, h);
  } else {
    auto go = [&](auto six, auto& tiles) {
      constexpr bool SIX = decltype(six)::value;
      if constexpr (TERMS == 1)
        if (p.two) return many_rows<D, F16, 2, K, SIX>(own_args(), tiles, p, h);
      many_rows<D, F16, TERMS, K, SIX>(own_args(), tiles, p, h);
    };
    if (a.had) go(std::integral_constant<bool, true>{}, buf.six);
    else go(std::integral_constant<bool, false>{}, buf.pairs);
  }
}

// Joins the parts of split tiles, a workgroup for per_group rows: up to eight
// parts a wave per row, else one row after the other, the parts' weights first,
// then the sum of their outputs, eight at a time (D / 4 threads each).
constexpr int kMostParts = 2048;   // 2 * target at most, one KV head

template <int D, int M, Keys K>
__device__ __forceinline__ void join_tiles(const CacheAttnArgs& a, int target, int per_group, int x0, int h, int z) {
  constexpr int W = D / 4, NG = 256 / W;
  __shared__ SchedShared sched;
  __shared__ float f[kMostParts];
  __shared__ float red[8];
  __shared__ __align__(16) float4 sum[NG][W];
  Piece p;
  if (!find_piece<M, K>(a, sched, x0, true, target, &p)) return;
  if (M > kFewRows && a.causal) p.tile = p.q.tiles - 1 - p.tile;   // as k_rows numbers them
  const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
  int rows = p.q.ql * a.G - p.tile * M < M ? p.q.ql * a.G - p.tile * M : M;
  const int row0 = z * per_group;
  if (row0 + per_group < rows) rows = row0 + per_group;
  const int64_t step = static_cast<int64_t>(a.g.Hkv) * M;
  if (p.parts <= 8) {
    // few parts: a wave per row, a lane per part for its weight
    for (int row = row0 + w; row < rows; row += 4) {
      const int64_t first = (static_cast<int64_t>(p.slot) * a.g.Hkv + h) * M + row;
      float2 ml = make_float2(kNegInf, 0.0f);
      if (lane < p.parts) ml = a.part_ml[first + lane * step];
      float mm = ml.x;
#pragma unroll
      for (int d = 1; d < 8; d *= 2) mm = fmaxf(mm, __shfl_xor(mm, d));
      mm = __shfl(mm, 0);
      const float x = rescale(ml.x, mm);
      float l = x * ml.y;
#pragma unroll
      for (int d = 1; d < 8; d *= 2) l += __shfl_xor(l, d);
      l = __shfl(l, 0);
      float out[D / 64] = {};
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        if (i >= p.parts) break;
        const float xi = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(x), i));
#pragma unroll
        for (int z = 0; z < D / 64; ++z) out[z] += xi * a.part_o[(first + i * step) * D + lane * (D / 64) + z];
      }
      const int i = (p.tile * M + row) / a.G;
      finish_row<D>(a, p.q.q0 + i, h * a.G + p.tile * M + row - i * a.G, out, mm, l, lane);
    }
    return;
  }
  for (int row = row0; row < rows; ++row) {
    const int64_t first = (static_cast<int64_t>(p.slot) * a.g.Hkv + h) * M + row;   // of part 0
    float mm = kNegInf;
    for (int i = tid; i < p.parts; i += 256) {
      const float m = a.part_ml[first + i * step].x;
      f[i] = m;
      mm = fmaxf(mm, m);
    }
#pragma unroll
    for (int d = 32; d; d >>= 1) mm = fmaxf(mm, __shfl_xor(mm, d));
    if (lane == 0) red[w] = mm;
    __syncthreads();
    mm = fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3]));
    float l = 0.0f;
    for (int i = tid; i < p.parts; i += 256) {
      f[i] = rescale(f[i], mm);
      l += f[i] * a.part_ml[first + i * step].y;
    }
#pragma unroll
    for (int d = 32; d; d >>= 1) l += __shfl_xor(l, d);
    if (lane == 0) red[4 + w] = l;
    __syncthreads();
    l = red[4] + red[5] + red[6] + red[7];
    const int g = tid / W, c = tid % W;
    float4 y = make_float4(0, 0, 0, 0);
#pragma unroll 4
    for (int i = g; i < p.parts; i += NG) {
      const float4 o = *reinterpret_cast<const float4*>(a.part_o + (first + i * step) * D + c * 4);
      const float x = f[i];
      y.x += x * o.x, y.y += x * o.y, y.z += x * o.z, y.w += x * o.w;
    }
    sum[g][c] = y;
    __syncthreads();
    if (w == 0) {
      float out[D / 64] = {};
      const float* s = reinterpret_cast<const float*>(&sum[0][0]);
#pragma unroll
      for (int i = 0; i < NG; ++i)
#pragma unroll
        for (int x = 0; x < D / 64; ++x) out[x] += s[i * D + lane * (D / 64) + x];
      const int i = (p.tile * M + row) / a.G;
      finish_row<D>(a, p.q.q0 + i, h * a.G + p.tile * M + row - i * a.G, out, mm, l, lane);
    }
    __syncthreads();   // before the next row's parts
  }
}

// Pieces of work over all KV heads aimed at, and rows of a tile of k_rows.
constexpr int kPieces = 1024, kRowPieces = 512, kRowTile = 128;

struct Grid {
  int64_t tiles, merges;
};
// Bounds that hold for all lengths: tiles of the requests, tiles with several parts.
Grid grid_of(const CacheAttnArgs& a, int M, int target) {
  const int64_t per = (static_cast<int64_t>(a.max_q) * a.G + M - 1) / M;
  Grid g;
  g.tiles = a.R + static_cast<int64_t>(a.T) * a.G / M;
  if (g.tiles > a.R * per) g.tiles = a.R * per;
  g.merges = g.tiles < target ? g.tiles : target;
  return g;
}

Grid few_grid_of(const CacheAttnArgs& a) {   // a request of few rows is one tile
  return {a.R, a.R < a.target ? a.R : a.target};
}

int target_of(int pieces, int Hkv) { return (pieces + Hkv - 1) / Hkv; }

// ---------------------------------------------------------------- kernels --
//
// Heads are fastest: the heads of a page, neighbours in memory, are read together,
// and as workgroups go round the 8 XCDs a head's keys stay in few L2s.

template <int D, int NT, int KT, Keys K>
__global__ __launch_bounds__(256, 2) void k_few(CacheAttnArgs a) {
  __shared__ FewLds<D, NT, fine_q<false, K>()> lds;
  const int x0 = blockIdx.x / a.g.Hkv;
  few_rows<D, NT, KT, false, K>(a, lds, x0, blockIdx.x - x0 * a.g.Hkv);
}
template <int D, int NT, int KT, Keys K>
__global__ __launch_bounds__(256, 2) void k_fine_few(CacheAttnArgs a) {
  __shared__ FewLds<D, NT, fine_q<true, K>()> lds;
  const int x0 = blockIdx.x / a.g.Hkv;
  few_rows<D, NT, KT, true, K>(a, lds, x0, blockIdx.x - x0 * a.g.Hkv);
}

template <int D, bool F16, bool LO, Keys K>
__global__ __launch_bounds__(256, 2) void k_rows(CacheAttnArgs a) {
  __shared__ RowsLds<D, K> lds;
  const int x0 = blockIdx.x / a.g.Hkv;
  rows_piece<D, F16, LO ? 2 : 1, K>(a, lds, x0, blockIdx.x - x0 * a.g.Hkv);
}
template <int D, bool F16, Keys K>
__global__ __launch_bounds__(256, 2) void k_fine_rows(CacheAttnArgs a) {
  __shared__ RowsLds<D, K> lds;
  const int x0 = blockIdx.x / a.g.Hkv;
  rows_piece<D, F16, 3, K>(a, lds, x0, blockIdx.x - x0 * a.g.Hkv);
}

template <int D, int M, Keys K>
__global__ __launch_bounds__(256) void k_merge(CacheAttnArgs a, int target, int per_group) {
  join_tiles<D, M, K>(a, target, per_group, blockIdx.x, blockIdx.y, blockIdx.z);
}

// Rows of a tile that a workgroup of the merge takes: a workgroup per row while those are few enough to run at once.
template <int M>
int merged_rows(const CacheAttnArgs& a, const Grid& g, int64_t rows) {
  return g.merges * a.g.Hkv * (rows > M ? M : rows) <= 4096 ? 1 : M > kFewRows ? 16 : 8;
}
template <int D, int M, Keys K>
hipError_t merge(const CacheAttnArgs& a, const Grid& g, int target, int64_t rows, hipStream_t s) {
  const int per_group = merged_rows<M>(a, g, rows);
  if (rows > M) rows = M;
  k_merge<D, M, K><<<dim3(static_cast<unsigned>(g.merges), a.g.Hkv, static_cast<unsigned>((rows + per_group - 1) / per_group)),
                  dim3(256), 0, s>>>(a, target, per_group);
  return hipGetLastError();
}

template <int D, int NT, Keys K>
hipError_t few(const CacheAttnArgs& a, hipStream_t s) {
  constexpr int M = 16 * NT;
  const Grid g = few_grid_of(a);
  const dim3 grid(static_cast<unsigned>((g.tiles + a.target) * a.g.Hkv));
  if (a.out_dtype == RA_FP32) k_fine_few<D, NT, 2, K><<<grid, dim3(256), 0, s>>>(a);
  else k_few<D, NT, 2, K><<<grid, dim3(256), 0, s>>>(a);
  const hipError_t e = hipGetLastError();
  return e != hipSuccess ? e : merge<D, M, K>(a, g, a.target, static_cast<int64_t>(a.max_q) * a.G, s);
}

// Of a launch; with 1 its pieces of few enough rows take two (kTwoTerms).
int terms_of(const CacheAttnArgs& a) { return a.out_dtype == RA_FP32 ? 3 : a.out_dtype == RA_FP16 ? 2 : 1; }

template <int D, bool F16, Keys K>
hipError_t rows(const CacheAttnArgs& a, hipStream_t s) {
  const Grid g = grid_of(a, kRowTile, a.target_rows);
  const dim3 grid(static_cast<unsigned>((g.tiles + a.target_rows) * a.g.Hkv));
  const int terms = terms_of(a);
  if (terms == 3) k_fine_rows<D, F16, K><<<grid, dim3(256), 0, s>>>(a);
  else if (terms == 2) k_rows<D, F16, true, K><<<grid, dim3(256), 0, s>>>(a);
  else k_rows<D, F16, false, K><<<grid, dim3(256), 0, s>>>(a);
  const hipError_t e = hipGetLastError();
  return e != hipSuccess ? e : merge<D, kRowTile, K>(a, g, a.target_rows, static_cast<int64_t>(a.max_q) * a.G, s);
}

template <int D, Keys K>
hipError_t attn_d(const CacheAttnArgs& a, hipStream_t s) {
  const int64_t most = static_cast<int64_t>(a.max_q) * a.G;
  if (most <= 16) return few<D, 1, K>(a, s);
  hipError_t e = hipSuccess;
  if (a.G <= kFewRows) e = few<D, 2, K>(a, s);   // requests of few rows; with more heads than that there are none
  if (e != hipSuccess || most <= kFewRows) return e;
  return a.is_fp16 ? rows<D, true, K>(a, s) : rows<D, false, K>(a, s);
}


}  // namespace
}  // namespace ra
