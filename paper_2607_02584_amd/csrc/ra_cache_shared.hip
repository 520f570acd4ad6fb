// ra_cache_shared.hip -- attention over the 4-bit paged KV cache for requests
// that share a prefix (gfx950): cache_attn_shared.
//
// The softmax over a row's keys is that over the prefix joined with that over
// the request's own keys: with maxima m, sums l and unnormalised outputs o of the
// two,
//   M = max(m1, m2),  l = l1 2^(m1 - M) + l2 2^(m2 - M),  o = (o1 2^(m1 - M) + o2 2^(m2 - M)) / l.
// The prefix of a group is a request of its own here, whose rows are the
// queries of all the group's requests (they follow each other in the batch), so
// that its keys are read once for all, by the matrix cores as soon as there are
// more than 16 rows.
//
// Three launches: k_shared_plan cuts prefixes and requests into pieces and turns
// Q, once for all the pieces that take a row (in each of them it was 5 of a
// piece's 66 us); k_both goes through the pieces of many rows and those of few
// and leaves partial rows in the workspace (k_few alone where no prefix can have
// more than 16 rows); k_join joins a row's parts, a wave per row.  Pieces of many
// rows come first in the grid and are cut for their share of the places that the
// card has, so that those of few run beside them from the start: 64 requests on a
// prefix of 32 700 tokens took 117 us with one launch after the other, 101 with the
// two kinds alternating (whoever waits for a place ends as much later), 96 so (88 with
// Q in digits, now 98, with two values of the weights).
//
// Bound by HBM while a group's rows are few, by the matrix cores and the softmax
// beside them from some 64 rows on.
#include "ra_cache_attn.h"
#include "ra_cache_cut.h"

namespace ra {
namespace {

constexpr int kFewShared = 16;   // rows of one 16-row product: up to those, k_few

// The lengths of a call, in memory or in LDS.
struct Lengths {
  const int* group_start;
  const int* prefix_lens;
  const int* q_start;
  const int* seq_lens;
};

// The request's group, -1 for none: the last one that begins at r or before, if it holds r.
__device__ __forceinline__ int group_of(const CacheAttnArgs& a, const Lengths& x, int r) {
  int g = -1, y = a.groups;   // group_start[g] <= r < group_start[y]
  while (y - g > 1) {
    const int m = (g + y) >> 1;
    if (x.group_start[m] <= r) g = m; else y = m;
  }
  return g >= 0 && r < x.group_start[g + 1] ? g : -1;
}
// Tokens that group g shares: no more than its first request, whose table is read, holds.
__device__ __forceinline__ int prefix_of(const CacheAttnArgs& a, const Lengths& x, int g) {
  const int r0 = x.group_start[g];
  if (r0 < 0 || r0 >= a.R) return 0;
  int n = x.prefix_lens[g];
  const int most = a.max_blocks << a.g.page_log, held = x.seq_lens[r0];
  n = n < held ? n : held;
  return n < 0 ? 0 : n > most ? most : n;
}

// Prefix or request v, and its group (-1: none).  Whatever the device holds, nothing outside the tensors is touched.
__device__ __forceinline__ Request shared_request(const CacheAttnArgs& a, const Lengths& l, int v, int& g) {
  Request x;
  g = v < a.groups ? v : group_of(a, l, v - a.groups);
  const int prefix = g < 0 ? 0 : prefix_of(a, l, g);
  int r0 = v - a.groups, r1 = r0 + 1;
  if (v < a.groups) {
    r0 = l.group_start[v];
    r1 = l.group_start[v + 1];
    r0 = r0 < 0 ? 0 : r0 > a.R ? a.R : r0;
    r1 = r1 < r0 ? r0 : r1 > a.R ? a.R : r1;
  }
  const int q0 = l.q_start[r0], q1 = l.q_start[r1], most = a.max_blocks << a.g.page_log;
  x.table = r0 < a.R ? r0 : 0;
  x.q0 = q0 < 0 ? 0 : q0 > a.T ? a.T : q0;
  x.ql = (q1 < x.q0 ? x.q0 : q1 > a.T ? a.T : q1) - x.q0;
  const int n = v < a.groups ? prefix : l.seq_lens[r0];
  x.n = n < 0 ? 0 : n > most ? most : n;
  x.first = x.n - x.ql;   // (of a prefix not used: its rows have positions of their own)
  x.lo = v < a.groups ? 0 : prefix < x.n ? prefix : x.n;
  if (v < a.groups && x.n == 0) x.ql = 0;
  const int rows = x.ql * a.G, M = rows <= kFewShared ? kFewShared : kRowTile;
  x.tiles = (rows + M - 1) / M;
  x.blocks = x.n > x.lo ? (x.n + kBlock - 1) / kBlock - x.lo / kBlock : 0;
  return x;
}

// ------------------------------------------------------------------- plan --
//
// A tile of `blocks` blocks is cut into ceil(blocks / C) parts, the same C for all tiles of
// either kernel.  A piece costs its blocks and `kFixed` more (its page numbers, its first loads,
// its rows to the workspace).  `places` pieces run at once (a workgroup each, for every KV
// head), so what is cut so that it fits k rounds takes k (C + kFixed):
//   sum of weights <= k places,   weight = 1 per part longer than C / 2, else (blocks + kFixed) / (C + kFixed),
// as small pieces fill what others leave.  The least such C is looked for with k = 1 and k = 2
// (eight values at a time, three times over), and the cheaper one taken.
// Cut into W / places blocks instead, without a look at what is left for the second round, 190
// requests on five prefixes took 1000 us, with this 760 (the whole call, two launches still).
constexpr int kPlan = 512;
constexpr int kKnown = 4096;      // prefixes and requests whose tiles and blocks are kept in LDS
constexpr int kRounds = 2;
// blocks of a part at least, of few and many rows (the latter with 16: 8 requests on 1000 tokens 45 us, with 4 25, with 2
// 25 too, but calls of many parts slower, whose joins then take longer)
constexpr int kLeast[2] = {4, 4};
constexpr int kFixed[2] = {10, 6};
constexpr float kFewCost = 0.3f;      // of a block of keys for few rows, in blocks for many
// workgroups of four waves that run at once: two on a compute unit, by registers and LDS
constexpr int kPlaces = 512;
__host__ __device__ constexpr int places_of(int Hkv) { return kPlaces > Hkv ? kPlaces / Hkv : 1; }

struct PlanShared {
  int blocks[kKnown];
  int tiles[kKnown];             // of few rows as they are, of many negative
  uint8_t two[kKnown];           // groups with a request of few rows (kTwoTerms; those behind are taken for such)
  int lengths[4 * kPlan + 2];    // where they are no more than kPlan each
  int from[2][kPlan];            // first piece of each, of few and of many rows
  int parts[kPlan];
  float w[kPlan / 64][4];
  int n[kPlan / 64][5];
  unsigned lo[2][kRounds], hi[2][kRounds];
  int fits[2][4 * (kPlan / 64)], wide[3][2 * kRounds];
};

__device__ void plan_pieces(const CacheAttnArgs& a) {
  __shared__ PlanShared sh;
  const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6, N = a.groups + a.R;
  constexpr int NW = kPlan / 64;
  // the lengths with one load each, as finding a request's group and prefix takes one after the other
  Lengths l = {a.group_start, a.prefix_lens, a.q_start, a.seq_lens};
  const int marked = a.groups < kKnown ? a.groups : kKnown;
  for (int i = tid; i < marked; i += kPlan) sh.two[i] = 0;
  if (a.R <= kPlan && a.groups <= kPlan) {
    int* x = sh.lengths;
    if (tid <= a.groups && a.groups) x[tid] = a.group_start[tid];
    if (tid < a.groups) x[kPlan + 1 + tid] = a.prefix_lens[tid];
    if (tid <= a.R) x[2 * kPlan + 1 + tid] = a.q_start[tid];
    if (tid < a.R) x[3 * kPlan + 2 + tid] = a.seq_lens[tid];
    if (tid == 0) {   // the last of kPlan + 1
      if (a.groups == kPlan) x[kPlan] = a.group_start[kPlan];
      if (a.R == kPlan) x[3 * kPlan + 1] = a.q_start[kPlan];
    }
    l = {x, x + kPlan + 1, x + 2 * kPlan + 1, x + 3 * kPlan + 2};
  }
  __syncthreads();
  // what there is: blocks of all tiles, the longest, tiles
  float W[2] = {0.0f, 0.0f}, finest[2] = {0.0f, 0.0f};   // finest: pieces of kLeast blocks
  int count[2] = {0, 0}, longest[2] = {0, 0};
  int queries = 0;   // of prefixes and requests, no more than 2 T where offsets and groups ascend
  Request mine = {};
#pragma unroll 1
  for (int v = tid; v < N; v += kPlan) {
    int g;
    const Request q = shared_request(a, l, v, g);
    if (v == tid) mine = q;
    if (v >= a.groups && static_cast<unsigned>(g) < static_cast<unsigned>(marked) && q.ql > 0 && q.ql * a.Hq <= kTwoTerms) sh.two[g] = 1;
    const int many = q.ql * a.G > kFewShared;
    queries = queries + q.ql < 1 << 24 ? queries + q.ql : 1 << 24;
    if (v < kKnown) {
      sh.blocks[v] = q.blocks;
      sh.tiles[v] = many ? -q.tiles : q.tiles;
    }
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const bool on = many == k;
      W[k] += on ? static_cast<float>(q.tiles) * static_cast<float>(q.blocks) : 0.0f;
      count[k] += on ? q.tiles : 0;
      longest[k] = on && q.blocks > longest[k] ? q.blocks : longest[k];
      finest[k] += on ? cut_finest(q.tiles, q.blocks, kLeast[k]) : 0.0f;
    }
  }
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    W[k] = wave_total(W[k]);
    count[k] = __builtin_amdgcn_readlane(wave_sums(count[k]), 63);
    longest[k] = wave_most(longest[k]);
    finest[k] = wave_total(finest[k]);
  }
  if (lane == 0)
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      sh.w[w][k] = W[k];
      sh.n[w][k] = count[k];
      sh.n[w][2 + k] = longest[k];
      sh.w[w][2 + k] = finest[k];
    }
  queries = __builtin_amdgcn_readlane(wave_sums(queries), 63);
  if (lane == 0) sh.n[w][4] = queries < 1 << 24 ? queries : 1 << 24;
  __syncthreads();
  queries = 0;
#pragma unroll
  for (int i = 0; i < NW; ++i) queries += sh.n[i][4];
  // (what does not fit the call has no pieces: their numbers would pass 32 bits)
  const bool fits = queries <= 2 * a.T;
  W[0] = W[1] = finest[0] = finest[1] = 0.0f;
  count[0] = count[1] = longest[0] = longest[1] = 0;
#pragma unroll
  for (int i = 0; i < NW; ++i)
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      W[k] += sh.w[i][k];
      count[k] += sh.n[i][k];
      longest[k] = sh.n[i][2 + k] > longest[k] ? sh.n[i][2 + k] : longest[k];
      finest[k] += sh.w[i][2 + k];
    }
  // either kind's share of the places
  int places_for[2];
  {
    const int all = places_of(a.g.Hkv);
    const float few = kFewCost * (W[0] + static_cast<float>(kFixed[0]) * static_cast<float>(count[0]));
    const float many = W[1] + static_cast<float>(kFixed[1]) * static_cast<float>(count[1]);
    int n = static_cast<int>(static_cast<float>(all) * many / (few + many + 1e-6f) + 0.5f);
    n = n < 1 || all < 2 ? 1 : n >= all ? (count[0] ? all - 1 : all) : n;
    places_for[1] = n;
    places_for[0] = count[1] && all > n ? all - n : all;
  }
  // Blocks of a part.
  unsigned C[2];
  if (finest[0] <= static_cast<float>(places_for[0]) && finest[1] <= static_cast<float>(places_for[1])) {
    C[0] = kLeast[0];
    C[1] = kLeast[1];
  } else if (N <= kKnown) {
    if (tid < 2 * kRounds) {
      const int k = tid / kRounds, r = tid % kRounds;
      const CutRange x = cut_range(k ? W[1] : W[0], k ? count[1] : count[0], k ? longest[1] : longest[0],
                                   static_cast<float>((r + 1) * (k ? places_for[1] : places_for[0])), static_cast<float>(kFixed[k]), kLeast[k]);
      sh.lo[k][r] = x.lo;
      sh.hi[k][r] = x.hi;
    }
    __syncthreads();
    // kernel, rounds, and which four of eight values
    const int k = w / (NW / 2), r = w / (NW / 2 / kRounds) % kRounds, x = w % (NW / 2 / kRounds);
    constexpr int NZ = 4, NX = NZ * (NW / 2 / kRounds);
    const float places = static_cast<float>((r + 1) * (k ? places_for[1] : places_for[0])), fixed = static_cast<float>(kFixed[k]);
    unsigned lo = sh.lo[k][r], hi = sh.hi[k][r];
#pragma unroll 1   // (code that runs once costs more to fetch than to run)
    for (int step = 0; step < 3; ++step) {
      float fc[NZ], inv[NZ], per[NZ], sum[NZ] = {};
#pragma unroll
      for (int z = 0; z < NZ; ++z) {
        fc[z] = static_cast<float>(lo + static_cast<unsigned>(static_cast<uint64_t>(hi - lo) * (NZ * x + z) / NX));
        inv[z] = 1.0f / fc[z];
        per[z] = 1.0f / (fc[z] + fixed);
      }
#pragma unroll 1
      for (int v = lane; v < N; v += 64) {
        const int t = k ? -sh.tiles[v] : sh.tiles[v];
        const float b = static_cast<float>(sh.blocks[v]);
        if (t <= 0) continue;
        // (binary32: at the edge a part more or less is of no matter)
#pragma unroll
        for (int z = 0; z < NZ; ++z) sum[z] += static_cast<float>(t) * cut_weight(b, fc[z], inv[z], fixed, per[z]);
      }
#pragma unroll
      for (int z = 0; z < NZ; ++z) {
        sum[z] = wave_total(sum[z]);
        if (lane == 0) sh.fits[step & 1][NZ * w + z] = sum[z] <= places;
      }
      __syncthreads();   // (two sets of answers: the next step writes the other one)
      // the least value that fits ends the range; the one before it begins it
      int good = NX;
#pragma unroll
      for (int i = NX - 1; i >= 0; --i)
        if (sh.fits[step & 1][NZ * (w - x) + i]) good = i;
      const uint64_t d = hi - lo;
      const unsigned from = lo;
      if (good < NX) hi = from + static_cast<unsigned>(d * good / NX);
      if (good > 0) lo = from + static_cast<unsigned>(d * (good - 1) / NX);
      // on while any of the four ranges is wide
      if (lane == 0 && x == 0) sh.wide[step][k * kRounds + r] = hi > lo + 1 + lo / 32;
      __syncthreads();
      int wide = 0;
#pragma unroll
      for (int i = 0; i < 2 * kRounds; ++i) wide |= sh.wide[step][i];
      if (!wide) break;
    }
    if (lane == 0 && x == 0) sh.hi[k][r] = hi;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      C[i] = sh.hi[i][0];
      unsigned long long cost = C[i] + static_cast<unsigned>(kFixed[i]);
#pragma unroll
      for (int j = 1; j < kRounds; ++j) {
        const unsigned long long other = static_cast<unsigned long long>(j + 1) * (sh.hi[i][j] + static_cast<unsigned>(kFixed[i]));
        if (other < cost) {
          cost = other;
          C[i] = sh.hi[i][j];
        }
      }
    }
  } else {
#pragma unroll
    for (int i = 0; i < 2; ++i) C[i] = cut_closed(W[i], static_cast<float>(kRounds * places_for[i]), kLeast[i]);
  }
  // pieces and places in the workspace, in order
  int carry[4] = {0, 0, 0, 0};   // pieces and rows of parts, of few and many rows
  for (int v0 = 0; v0 < N; v0 += kPlan) {
    const int v = v0 + tid;
    Request q = {};
    int g;
    if (v < N) q = v0 == 0 ? mine : shared_request(a, l, v, g);
    const int many = q.ql * a.G > kFewShared;
    const unsigned c = many ? C[1] : C[0];
    const int parts = q.tiles && fits ? cut_parts(q.blocks, c) : 0;
    const int val[4] = {many ? 0 : q.tiles * parts, many ? q.tiles * parts : 0, many ? 0 : q.ql * a.G * parts,
                        many ? q.ql * a.G * parts : 0};
    int from[4];
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      from[i] = wave_sums(val[i]);
      if (lane == 63) sh.n[w][i] = from[i];
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      int all = 0, before = 0;
#pragma unroll
      for (int j = 0; j < NW; ++j) {
        if (j < w) before += sh.n[j][i];
        all += sh.n[j][i];
      }
      from[i] += carry[i] + before - val[i];
      carry[i] += all;
    }
    sh.from[0][tid] = from[0];
    sh.from[1][tid] = from[1];
    sh.parts[tid] = many ? -parts : parts;
    __syncthreads();
    // a thread per piece finds its request: the last one whose pieces begin there or before
    const int here = N - v0 < kPlan ? N - v0 : kPlan;
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const int p0 = sh.from[k][0], p1 = carry[k] < a.bound[k] ? carry[k] : a.bound[k];   // (past the bound: lengths that do not fit the call)
      if (p0 < 0) continue;
      for (int at = p0 + tid; at < p1; at += kPlan) {
        int x = 0, y = here;
        while (y - x > 1) {
          const int m = (x + y) >> 1;
          if (sh.from[k][m] <= at) x = m; else y = m;
        }
        const int n = k ? -sh.parts[x] : sh.parts[x], i = at - sh.from[k][x];
        if (n > 0) a.pieces[k][at] = make_int4(v0 + x, i / n, i % n, n);
      }
    }
    if (v >= N) continue;
    const int base = many ? from[3] : from[2];
    a.requests[2 * v] = make_int4(q.q0, q.ql, q.n, q.first);
    const int two = v >= a.groups ? q.ql * a.Hq <= kTwoTerms : v < marked ? sh.two[v] : 1;
    a.requests[2 * v + 1] = make_int4(q.lo, q.table, base, two);
    a.info[v] = make_int2(base, many ? -parts : parts);
  }
  if (tid < 2) {
    const int n = tid ? carry[1] : carry[0];
    a.counts[tid] = n < 0 ? 0 : n < a.bound[tid] ? n : a.bound[tid];
  }
}

// Q of a row after RoPE, rotation and scale as two binary16 values and a power of two (see load_q): D / 8 lanes hold it.
template <int D>
__device__ __forceinline__ void turn_q(const CacheAttnArgs& a, int64_t row) {
  const int b = row_block(threadIdx.x & (D / 8 - 1));
  const bool ok = row < static_cast<int64_t>(a.T) * a.Hq;   // lanes without a row keep running: the moves between lanes need whole rows
  const int t = ok ? static_cast<int>(row / a.Hq) : 0, head = ok ? static_cast<int>(row - static_cast<int64_t>(t) * a.Hq) : 0;
  const uint4 x = *reinterpret_cast<const uint4*>(a.q + static_cast<int64_t>(t) * a.q_ts + head * a.q_hs + b * 8);
  const uint32_t u[4] = {x.x, x.y, x.z, x.w};
  float y[8];
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    y[2 * e] = cache_h2f(static_cast<uint16_t>(u[e] & 0xffff), a.is_fp16);
    y[2 * e + 1] = cache_h2f(static_cast<uint16_t>(u[e] >> 16), a.is_fp16);
  }
  if (a.rope) {
    int pos = a.positions[t];
    pos = pos < 0 ? 0 : pos >= a.rope_rows ? a.rope_rows - 1 : pos;
    const float4* p = reinterpret_cast<const float4*>(a.rope + static_cast<int64_t>(pos) * D + b * 8);
    const float4 c[2] = {p[0], p[1]};
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float cs = e & 1 ? c[e >> 1].z : c[e >> 1].x, sn = e & 1 ? c[e >> 1].w : c[e >> 1].y;
      const float m = y[2 * e], n = y[2 * e + 1];
      y[2 * e] = m * cs - n * sn;
      y[2 * e + 1] = m * sn + n * cs;
    }
  }
  float scale = a.c;   // scores come out in base 2
  if (a.had) {
    hadamard_row<D>(y, b);
    scale *= row_sign(b);
  }
#pragma unroll
  for (int e = 0; e < 8; ++e) y[e] *= scale;
  float m = 0.0f;
#pragma unroll
  for (int e = 0; e < 8; ++e) m = fmaxf(m, fabsf(y[e]));
  m = fmaxf(m, lane_xor<1>(m));
  m = fmaxf(m, lane_xor<2>(m));
  m = fmaxf(m, lane_xor<7>(m));
  if constexpr (D == 128) m = fmaxf(m, lane_xor<8>(m));
  const float power = row_power(m);
#pragma unroll
  for (int e = 0; e < 8; ++e) y[e] *= power;
  float bad = 0.0f;   // NaN where an element is not finite, which no digit is
#pragma unroll
  for (int e = 0; e < 8; ++e) bad = __fmaf_rn(y[e], 0.0f, bad);
  bad += lane_xor<1>(bad);
  bad += lane_xor<2>(bad);
  bad += lane_xor<7>(bad);
  if constexpr (D == 128) bad += lane_xor<8>(bad);
  if (ok && b == 0) a.back[row] = inverse_power(power) + bad;
  uint4 hi, lo;
  split8(y, true, hi, lo);
  if (ok) {
    uint16_t* dst = a.turned + row * 2 * D + b * 8;
    *reinterpret_cast<uint4*>(dst) = hi;
    *reinterpret_cast<uint4*>(dst + D) = lo;
  }
  if (!a.had) return;
  // digits (of a rotated row): codes |n| in eighths, and the sign
  uint16_t* six = reinterpret_cast<uint16_t*>(a.turned6 + row * row_bytes6<D>() + b * 6);
#pragma unroll
  for (int e = 0; e < 8; ++e) y[e] *= 0x1p-14f;
#pragma unroll
  for (int z = 0; z < kTerms; ++z) {
    uint64_t w = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float d = (y[e] + digit_of(z)) - digit_of(z);
      y[e] -= d;
      const uint32_t n = static_cast<uint32_t>(fabsf(d) * (8.0f * (1 << (5 * z))));
      w |= static_cast<uint64_t>((n & 31) | (__float_as_uint(d) >> 31) << 5) << (6 * e);
    }
    if (ok)
#pragma unroll
      for (int i = 0; i < 3; ++i) six[z * (D * 3 / 8) + i] = static_cast<uint16_t>(w >> (16 * i));
  }
}

// The request and group that each of a workgroup's tokens belongs to; {-1, ..} for none.
__device__ __forceinline__ void find_owners(const CacheAttnArgs& a, int64_t row0, int64_t row1) {
  const int64_t last = (row1 < static_cast<int64_t>(a.T) * a.Hq ? row1 : static_cast<int64_t>(a.T) * a.Hq) - 1;
  // tokens whose first head is among these rows
  const int t0 = static_cast<int>((row0 + a.Hq - 1) / a.Hq), t1 = static_cast<int>(last / a.Hq);
  for (int t = t0 + threadIdx.x; t <= t1; t += kPlan) {
    int r = 0, y = a.R;   // q_start[r] <= t < q_start[y]
    while (y - r > 1) {
      const int m = (r + y) >> 1;
      if (a.q_start[m] <= t) r = m; else y = m;
    }
    int2 x = make_int2(-1, -1);
    if (a.q_start[r] <= t && t < a.q_start[r + 1]) {
      const Lengths l = {a.group_start, a.prefix_lens, a.q_start, a.seq_lens};
      const int g = group_of(a, l, r);
      x = make_int2(r, g >= 0 && prefix_of(a, l, g) > 0 ? g : -1);
    }
    a.owner[t] = x;
  }
}

template <int D>
__global__ __launch_bounds__(kPlan) void k_shared_plan(CacheAttnArgs a) {
  if (blockIdx.x == 0) return plan_pieces(a);
  constexpr int kRows = kPlan * 8 / D;
  find_owners(a, static_cast<int64_t>(blockIdx.x - 1) * kRows, static_cast<int64_t>(blockIdx.x) * kRows);
  turn_q<D>(a, static_cast<int64_t>(blockIdx.x - 1) * (kPlan * 8 / D) + threadIdx.x / (D / 8));
}

// ---------------------------------------------------------------- kernels --

// Both kinds of pieces in one launch: those of many rows begin on their share
// of the places, those of few rows, which wait for memory for most of their time, follow each other on the rest.
template <int D, bool F16, int TERMS>
__global__ __launch_bounds__(256, 2) void k_both(CacheAttnArgs a) {
  constexpr bool FINE = TERMS == 3;
  __shared__ union {
    FewLds<D, 1, true> few;
    RowsLds<D, kShared> rows;
  } lds;
  const int x = blockIdx.x / a.g.Hkv, h = blockIdx.x - x * a.g.Hkv, many = __builtin_amdgcn_readfirstlane(a.counts[1]);
  if (x < many) rows_piece<D, F16, TERMS, kShared>(a, lds.rows, x, h);
  else few_rows<D, 1, 2, FINE, kShared>(a, lds.few, x - many, h);
}

// The parts of a row, 64 at a time: the request's own, then its prefix's.
template <int D>
__global__ __launch_bounds__(256) void k_join(CacheAttnArgs a) {
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  const int t = blockIdx.x, head = blockIdx.y * 4 + w;
  if (head >= a.Hq) return;
  const int2 of = a.owner[t];   // the token's request and group
  const int r = __builtin_amdgcn_readfirstlane(of.x), g = __builtin_amdgcn_readfirstlane(of.y);
  if (r < 0) return;
  const int h = head / a.G, z = head - h * a.G;
  int first[2], parts[2], rows[2], row[2];
  bool many[2];
  auto take = [&](int i, int v) {
    const int2 x = a.info[v];
    const int4 q = a.requests[2 * v];   // q0, ql
    first[i] = x.x;
    many[i] = x.y < 0;
    parts[i] = x.y < 0 ? -x.y : x.y;
    rows[i] = q.y * a.G;
    row[i] = (t - q.x) * a.G + z;
  };
  take(0, a.groups + r);
  parts[1] = 0;
  if (g >= 0) take(1, g);
  else first[1] = rows[1] = row[1] = 0, many[1] = false;
  const int n0 = parts[0], n = n0 + parts[1];
  float M = kNegInf, L = 0.0f, out[D / 64] = {};
  for (int i0 = 0; i0 < n; i0 += 64) {
    const int i = i0 + lane;
    int64_t at = -1;
    if (i < n) {
      const int k = i < n0 ? 0 : 1, part = k ? i - n0 : i;
      at = (k ? many[1] : many[0]) ? shared_at<true>(a, k ? first[1] : first[0], k ? parts[1] : n0, part, k ? rows[1] : rows[0], k ? row[1] : row[0], h)
                                   : shared_at<false>(a, k ? first[1] : first[0], k ? parts[1] : n0, part, k ? rows[1] : rows[0], k ? row[1] : row[0], h);
    }
    const float2 ml = at >= 0 ? a.part_ml[at] : make_float2(kNegInf, 0.0f);
    float mm = ml.x;
#pragma unroll
    for (int d = 32; d; d >>= 1) mm = fmaxf(mm, __shfl_xor(mm, d));
    mm = fmaxf(M, mm);
    const float x = rescale(ml.x, mm), old = rescale(M, mm);
    L = L * old + wave_total(x * ml.y);
    M = mm;
#pragma unroll
    for (int e = 0; e < D / 64; ++e) out[e] *= old;
    const int count = n - i0 < 64 ? n - i0 : 64;
    const int lo = static_cast<int>(at), hi = static_cast<int>(at >> 32);
    // sixteen at a time, so that their loads are under way together (places that are none: 0)
#pragma unroll 1
    for (int k0 = 0; k0 < count; k0 += 16) {
      float v[16][D / 64], f[16];
#pragma unroll
      for (int k = 0; k < 16; ++k) {
        f[k] = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(x), k0 + k));
        const int64_t p = static_cast<int64_t>(static_cast<uint64_t>(static_cast<uint32_t>(__builtin_amdgcn_readlane(hi, k0 + k))) << 32 |
                                               static_cast<uint32_t>(__builtin_amdgcn_readlane(lo, k0 + k)));
#pragma unroll
        for (int e = 0; e < D / 64; ++e) v[k][e] = p >= 0 ? a.part_o[p * D + lane * (D / 64) + e] : 0.0f;
      }
#pragma unroll
      for (int k = 0; k < 16; ++k)
#pragma unroll
        for (int e = 0; e < D / 64; ++e) out[e] += f[k] * v[k][e];
    }
  }
  finish_row<D>(a, t, head, out, M, L, lane);
}

template <int D>
hipError_t shared_d(const CacheAttnArgs& a, hipStream_t s) {
  const int64_t rows = static_cast<int64_t>(a.T) * a.Hq;
  k_shared_plan<D><<<dim3(static_cast<unsigned>(1 + (rows + kPlan * 8 / D - 1) / (kPlan * 8 / D))), dim3(kPlan), 0, s>>>(a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const dim3 grid(static_cast<unsigned>(a.bound[0] + a.bound[1]) * a.g.Hkv);
  if (!a.bound[1]) {
    if (a.out_dtype == RA_FP32) k_fine_few<D, 1, 2, kShared><<<grid, dim3(256), 0, s>>>(a);
    else k_few<D, 1, 2, kShared><<<grid, dim3(256), 0, s>>>(a);
  } else {
    const int terms = terms_of(a);
    auto go = [&](auto f16) {
      constexpr bool F16 = decltype(f16)::value;
      if (terms == 3) k_both<D, F16, 3><<<grid, dim3(256), 0, s>>>(a);
      else if (terms == 2) k_both<D, F16, 2><<<grid, dim3(256), 0, s>>>(a);
      else k_both<D, F16, 1><<<grid, dim3(256), 0, s>>>(a);
    };
    if (a.is_fp16) go(std::integral_constant<bool, true>{});
    else go(std::integral_constant<bool, false>{});
  }
  e = hipGetLastError();
  if (e != hipSuccess) return e;
  k_join<D><<<dim3(a.T, (a.Hq + 3) / 4), dim3(256), 0, s>>>(a);
  return hipGetLastError();
}

struct SharedSpace {
  int64_t rows;        // of parts, for every KV head
  int64_t bound[2];    // pieces of few and of many rows
  size_t ml, requests, pieces[2], info, owner, counts, back, turned, turned6, bytes;   // offsets
};
// Every row once for its prefix and once for its own keys; cutting adds at most the pieces of all rounds, a tile each
// (sum over tiles of parts - 1 <= W / C).  Prefixes and requests of many rows have more than 16 of them.
SharedSpace space_of(int D, int Hkv, int G, int R, int groups, int T) {
  SharedSpace x;
  const int64_t rows = 2 * static_cast<int64_t>(T) * G, all = static_cast<int64_t>(R) + groups;
  const int64_t few = kRounds * places_of(Hkv), many = few;   // cut off tiles at most
  x.rows = rows + kFewShared * few + kRowTile * many;
  x.bound[0] = (all < rows ? all : rows) + few;
  const int64_t more = rows / kFewShared;
  x.bound[1] = rows / 2 > kFewShared ? (all < more ? all : more) + rows / kRowTile + many : 0;
  const size_t n = static_cast<size_t>(x.rows) * Hkv, q = static_cast<size_t>(T) * G * Hkv;
  size_t at = n * D * sizeof(float);
  auto take = [&](size_t bytes) {
    at = (at + 15) / 16 * 16;
    const size_t here = at;
    at += bytes;
    return here;
  };
  x.ml = take(n * sizeof(float2));
  x.requests = take(2 * static_cast<size_t>(all) * sizeof(int4));
  x.pieces[0] = take(static_cast<size_t>(x.bound[0]) * sizeof(int4));
  x.pieces[1] = take(static_cast<size_t>(x.bound[1]) * sizeof(int4));
  x.info = take(static_cast<size_t>(all) * sizeof(int2));
  x.owner = take(static_cast<size_t>(T) * sizeof(int2));
  x.counts = take(2 * sizeof(int));
  x.back = take(q * sizeof(float));
  x.turned = take(q * 4 * D);
  x.turned6 = take(q * kTerms * D * 3 / 4);
  x.bytes = at;
  return x;
}

}  // namespace

size_t cache_shared_bytes(int D, int Hkv, int G, int R, int groups, int T) {
  return (space_of(D, Hkv, G, R, groups, T).bytes + 255) / 256 * 256;
}

hipError_t launch_cache_attn_shared(const CacheAttnArgs& a, int D, void* workspace, hipStream_t s) {
  CacheAttnArgs b = a;
  const SharedSpace x = space_of(D, a.g.Hkv, a.G, a.R, a.groups, a.T);
  char* ws = static_cast<char*>(workspace);
  b.part_o = reinterpret_cast<float*>(ws);
  b.part_ml = reinterpret_cast<float2*>(ws + x.ml);
  b.requests = reinterpret_cast<int4*>(ws + x.requests);
  for (int i = 0; i < 2; ++i) {
    b.pieces[i] = reinterpret_cast<int4*>(ws + x.pieces[i]);
    b.bound[i] = static_cast<int>(x.bound[i]);
  }
  b.info = reinterpret_cast<int2*>(ws + x.info);
  b.owner = reinterpret_cast<int2*>(ws + x.owner);
  b.counts = reinterpret_cast<int*>(ws + x.counts);
  b.back = reinterpret_cast<float*>(ws + x.back);
  b.turned = reinterpret_cast<uint16_t*>(ws + x.turned);
  b.turned6 = reinterpret_cast<uint8_t*>(ws + x.turned6);
  b.part_rows = x.rows;
  return D == 128 ? shared_d<128>(b, s) : shared_d<64>(b, s);
}

}  // namespace ra
