// ra_cache_attn.hip -- attention over the 4-bit paged KV cache (gfx950).
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
#include <type_traits>

#include "../../include/rotate_attn.h"
#include "ra_cache.h"

namespace ra {
namespace {

typedef float v4f __attribute__((ext_vector_type(4)));
typedef __bf16 v8bf __attribute__((ext_vector_type(8)));
typedef unsigned v4u __attribute__((ext_vector_type(4)));

constexpr float kNegInf = -__builtin_inff();
constexpr float kLn2 = 0.693147180559945309417232121458f;

// --------------------------------------------------------------- schedule --
//
// Work is cut into pieces of (request, tile of M rows, part of the keys), the
// same for every KV head.  Lengths live on the device (a captured graph runs
// with whatever they are then), so every workgroup cuts alone, in the same
// way: with W the sum over tiles of their blocks of 64 keys, a part has
// C = max(least, W / target) blocks, and a request's tiles n = ceil(blocks / C)
// parts.  There are then at most (tiles + target) pieces, and at most
// 2 * target of tiles that have several parts, whatever the lengths: the grid
// and the workspace follow from that.
constexpr int kBlock = 64;        // keys per step
constexpr int kLeastBlocks = 4;   // least part: one step for each of four waves

struct Request {
  int q0, ql, n;    // first query row, queries to compute (max_q at most), cached tokens
  int first;        // position of the first query
  int tiles, blocks;
};

template <int M>
__device__ __forceinline__ Request request_of(const CacheAttnArgs& a, int r) {
  Request x;
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
  x.tiles = (x.ql * a.G + M - 1) / M;
  int keys = x.n;
  if (a.window) {
    const int first = x.first - a.window + 1;
    keys = x.n - (first > 0 ? first : 0);
    const int tile = a.window + M / a.G + 1 + kBlock;   // keys that one tile can see, in whole blocks
    keys = keys < tile ? keys : tile;
  }
  x.blocks = (keys + kBlock - 1) / kBlock;
  return x;
}

struct Piece {
  Request q;
  int r, tile, part, parts, slot;   // slot: place in the workspace of part 0 of this tile
};

struct SchedShared {
  long long w[4];
  int s[4][2];
  int hit[8];
};

// Piece number x (or, for the merge, tile number x of those with several
// parts); false past the end.  All 256 threads call it.
template <int M>
__device__ bool find_piece(const CacheAttnArgs& a, SchedShared& sh, int x, bool merge, Piece* out) {
  const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
  long long W = 0;
  for (int r = tid; r < a.R; r += 256) {
    const Request q = request_of<M>(a, r);
    W += static_cast<long long>(q.tiles) * q.blocks;
  }
#pragma unroll
  for (int d = 32; d; d >>= 1) W += __shfl_xor(W, d);
  if (lane == 0) sh.w[w] = W;
  if (tid == 0) sh.hit[0] = -1;
  __syncthreads();
  W = sh.w[0] + sh.w[1] + sh.w[2] + sh.w[3];
  long long C = (W + a.target - 1) / a.target;
  if (C < kLeastBlocks) C = kLeastBlocks;
  int base = 0, slot = 0;
  for (int r0 = 0; r0 < a.R; r0 += 256) {
    const int r = r0 + tid;
    Request q = {};
    int n = 0;
    if (r < a.R) {
      q = request_of<M>(a, r);
      n = q.blocks ? static_cast<int>((q.blocks + C - 1) / C) : 1;
    }
    const int split = n > 1 ? q.tiles * n : 0;
    const int mine = merge ? (n > 1 ? q.tiles : 0) : q.tiles * n;
    int s0 = mine, s1 = split;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
      const int b0 = __shfl_up(s0, d), b1 = __shfl_up(s1, d);
      if (lane >= d) {
        s0 += b0;
        s1 += b1;
      }
    }
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
      sh.hit[0] = r;
      sh.hit[1] = x - from;
      sh.hit[2] = n;
      sh.hit[3] = slot + p1 + s1 - split;
    }
    base += t0;
    slot += t1;
    __syncthreads();
    if (x < base) break;   // found
  }
  const int r = sh.hit[0];
  if (r < 0) return false;
  out->r = r;
  out->q = request_of<M>(a, r);
  out->parts = sh.hit[2];
  out->tile = merge ? sh.hit[1] : sh.hit[1] / out->parts;
  out->part = merge ? 0 : sh.hit[1] - out->tile * out->parts;
  out->slot = sh.hit[3] + out->tile * out->parts;
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

// ------------------------------------------------------ few rows per request --
//
// A wave takes 16 NT rows and its own part of the keys, 64 per step, all in
// registers: per 16 keys one load each of K codes, V codes and their scales,
// S^T = K Q^T (keys as rows, so that a lane holds one query's scores), and
// O^T += V^T P^T, for which the lane's four keys of two 16-key tiles are
// already the eight that the product's second operand wants from it.  V's
// first operand, eight keys of one channel, comes from the four tokens per
// load by exchanging nibbles of neighbouring tokens (two operations for eight
// codes) before the conversion.  Q and P * (V's scale) are each the sum of two
// bf16 values (16 bits: q is exact then when it is a bf16 or binary16 input,
// P off by 2^-17), since the matrix cores have time: the kernel is bound by
// HBM, (D + 8) bytes per token and KV head.  The four waves of a workgroup are
// joined through LDS, the parts of a split tile by k_merge.

template <int D>
struct Tile16 {   // a lane's share of 16 tokens
  typename std::conditional<D == 128, uint4, uint2>::type k, v;
  float4 ks, vs;
};

template <int D>
__device__ __forceinline__ void load_tile(const CacheAttnArgs& a, Tile16<D>& t, int id, int h, int key, int lane) {
  typedef typename std::conditional<D == 128, uint4, uint2>::type V;
  const int page = a.g.page, tok = key & (page - 1);
  const uint8_t* b = a.g.cache + static_cast<int64_t>(id) * a.g.page_bytes + static_cast<int64_t>(h) * head_bytes<D>(page);
  const int kb = page * D / 2;
  t.k = *reinterpret_cast<const V*>(b + tok * (D / 2) + lane * (D / 8));
  t.v = *reinterpret_cast<const V*>(b + kb + tok * (D / 2) + lane * (D / 8));
  const float* sc = reinterpret_cast<const float*>(b + 2 * kb) + tok + (lane >> 4) * 4;
  t.ks = *reinterpret_cast<const float4*>(sc);
  t.vs = *reinterpret_cast<const float4*>(sc + page);
}

template <int B>
__device__ __forceinline__ v2bf codes2(uint32_t w) { return __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, 1.0f, B); }

__device__ __forceinline__ v8bf join(v2bf a, v2bf b, v2bf c, v2bf d) {
  return v8bf{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}
__device__ __forceinline__ v8bf codes8(uint32_t w) { return join(codes2<0>(w), codes2<1>(w), codes2<2>(w), codes2<3>(w)); }

constexpr uint32_t kLow = 0x0f0f0f0fu;
// nibbles of two tokens: channel pairs' even / odd channels, token 0 low
__device__ __forceinline__ uint32_t even_of(uint32_t a, uint32_t b) { return (a & kLow) | ((b << 4) & ~kLow); }
__device__ __forceinline__ uint32_t odd_of(uint32_t a, uint32_t b) { return ((a >> 4) & kLow) | (b & ~kLow); }

// x = hi + lo, both bf16
__device__ __forceinline__ void split_bf16(float x, __bf16& hi, __bf16& lo) {
  hi = static_cast<__bf16>(x);
  lo = static_cast<__bf16>(x - static_cast<float>(hi));
}

// The rows' Q as the second operand of K Q^T: lane = 16 * part + row, its
// D / 4 channels from part * D / 4 on, after RoPE and rotation.
template <int D>
__device__ void load_q(const CacheAttnArgs& a, const Piece& p, int h, int row, int lane, v8bf (&hi)[D / 32],
                       v8bf (&lo)[D / 32]) {
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
  for (int c = 0; c < D / 32; ++c)
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      __bf16 x0, x1;
      split_bf16(y[8 * c + e], x0, x1);
      hi[c][e] = x0;
      lo[c][e] = x1;
    }
}

template <int D>
__device__ __forceinline__ uint32_t dword_of(const typename std::conditional<D == 128, uint4, uint2>::type& v, int i) {
  if constexpr (D == 128) return i == 0 ? v.x : i == 1 ? v.y : i == 2 ? v.z : v.w;
  else return i == 0 ? v.x : v.y;
}

template <int D, int NT>
__global__ __launch_bounds__(256) void k_few(CacheAttnArgs a) {
  constexpr int M = 16 * NT, E = D / 16, KC = D / 32;
  constexpr int kStride = D + 4;                       // floats, against bank conflicts
  __shared__ __align__(16) float so[4][16][kStride];
  __shared__ float sm[4][M], sl[4][M];
  __shared__ SchedShared sched;
  const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6, g = lane >> 4;
  const int h = blockIdx.y;
  Piece p;
  if (!find_piece<M>(a, sched, blockIdx.x, false, &p)) return;

  const int rows = p.q.ql * a.G - p.tile * M < M ? p.q.ql * a.G - p.tile * M : M;   // of this tile
  const int first = p.q.first;
  const int i0 = p.tile * M / a.G, i1 = (p.tile * M + rows - 1) / a.G;
  // keys that any row of the tile sees, and this part of them
  int hi = p.q.n, lo = 0;
  if (a.causal) hi = first + i1 + 1;
  if (hi < 0) hi = 0;
  if (a.window) lo = first + i0 - a.window + 1 > 0 ? first + i0 - a.window + 1 : 0;
  // bounds that every row of the tile sees
  const int all_hi = a.causal ? first + i0 + 1 : p.q.n;
  const int all_lo = a.window ? first + i1 - a.window + 1 : 0;
  const int bl = lo / kBlock, bh = hi > lo ? (hi + kBlock - 1) / kBlock : bl;
  const int per = (bh - bl + p.parts - 1) / p.parts;
  const int b0 = bl + p.part * per, b1 = b0 + per < bh ? b0 + per : bh;
  const int wper = (b1 - b0 + 3) / 4;
  const int w0 = b0 + w * wper, w1 = w0 + wper < b1 ? w0 + wper : b1;               // this wave's blocks

  v8bf qh[NT][KC], ql[NT][KC];
  int row_hi[NT], row_lo[NT];
  float m[NT], l[NT];
  v4f o[NT][E];
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    const int row = p.tile * M + nt * 16 + (lane & 15);
    load_q<D>(a, p, h, row, lane, qh[nt], ql[nt]);
    const int pos = first + row / a.G;
    row_hi[nt] = a.causal ? pos + 1 : p.q.n;
    if (row_hi[nt] > p.q.n) row_hi[nt] = p.q.n;
    row_lo[nt] = a.window ? pos - a.window + 1 : 0;
    m[nt] = kNegInf;
    l[nt] = 0.0f;
#pragma unroll
    for (int e = 0; e < E; ++e) o[nt][e] = v4f{0, 0, 0, 0};
  }

  const int per_page = a.g.page / 16;
  const int* row_table = a.block_table + static_cast<int64_t>(p.r) * a.max_blocks;
  const int last16 = (p.q.n + 15) / 16;   // 16-key tiles that hold cached tokens

  for (int b = w0; b < w1; ++b) {
    Tile16<D> t[4];
    bool there[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int t16 = b * 4 + i;
      int id = -1;
      if (t16 < last16) id = row_table[t16 / per_page];
      id = __builtin_amdgcn_readfirstlane(id);
      // an entry that is no page leaves its keys out
      there[i] = static_cast<unsigned>(id) < static_cast<unsigned>(a.g.num_pages);
      load_tile<D>(a, t[i], there[i] ? id : 0, h, t16 * 16, lane);
    }
    const int key0 = b * kBlock;
    const bool whole = key0 >= all_lo && key0 + kBlock <= all_hi && key0 + kBlock <= p.q.n && there[0] && there[1] &&
                       there[2] && there[3];
    v8bf kc[4][KC];
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int c = 0; c < KC; ++c) kc[i][c] = codes8(dword_of<D>(t[i].k, c));
    v8bf ph[NT][2], pl[NT][2];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      v4f s[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        s[i] = v4f{0, 0, 0, 0};
#pragma unroll
        for (int c = 0; c < KC; ++c) {
          s[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kc[i][c], qh[nt][c], s[i], 0, 0, 0);
          s[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kc[i][c], ql[nt][c], s[i], 0, 0, 0);
        }
        const float ks[4] = {t[i].ks.x, t[i].ks.y, t[i].ks.z, t[i].ks.w};
#pragma unroll
        for (int e = 0; e < 4; ++e) s[i][e] *= ks[e] * a.c;
      }
      unsigned seen = 0xffff;   // bit 4 i + e: this lane's row sees key 16 i + 4 g + e of the block
      if (!whole) {
        seen = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int key = key0 + 16 * i + 4 * g + e;
            const bool on = there[i] && key < row_hi[nt] && key >= row_lo[nt];
            seen |= static_cast<unsigned>(on) << (4 * i + e);
            s[i][e] = on ? s[i][e] : kNegInf;
          }
      }
      float mx = m[nt];
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) mx = fmaxf(mx, s[i][e]);
      mx = fmaxf(mx, lane_xor<16>(mx));
      mx = fmaxf(mx, lane_xor<32>(mx));
      const float ref = mx == kNegInf ? 0.0f : mx;   // nothing seen yet: any finite reference gives 0
      const float alpha = exp2f(m[nt] - ref);
      m[nt] = mx;
      l[nt] *= alpha;
#pragma unroll
      for (int e = 0; e < E; ++e) o[nt][e] *= alpha;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float vs[4] = {t[i].vs.x, t[i].vs.y, t[i].vs.z, t[i].vs.w};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float pr = exp2f(s[i][e] - ref);
          l[nt] += pr;
          // a scale that is not finite must not reach rows that do not see its token
          const float x = (seen >> (4 * i + e)) & 1 ? pr * vs[e] : 0.0f;
          __bf16 x0, x1;
          split_bf16(x, x0, x1);
          ph[nt][i / 2][4 * (i % 2) + e] = x0;
          pl[nt][i / 2][4 * (i % 2) + e] = x1;
        }
      }
    }
    // V: eight keys of one channel, channel e of the lane's chunk
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      uint32_t ev[4], od[4];
      if constexpr (D == 128) {
#pragma unroll
        for (int x = 0; x < 2; ++x) {
          const uint4 v = t[2 * u + x].v;
          ev[2 * x] = even_of(v.x, v.y);
          od[2 * x] = odd_of(v.x, v.y);
          ev[2 * x + 1] = even_of(v.z, v.w);
          od[2 * x + 1] = odd_of(v.z, v.w);
        }
      } else {
#pragma unroll
        for (int x = 0; x < 2; ++x) {
          const uint2 v = t[2 * u + x].v;
          const uint32_t t02 = (v.x & 0xffffu) | (v.y << 16), t13 = (v.x >> 16) | (v.y & 0xffff0000u);
          ev[x] = even_of(t02, t13);
          od[x] = odd_of(t02, t13);
        }
      }
      auto pv = [&](auto bb, const uint32_t (&n)[4], int e) {
        constexpr int B = decltype(bb)::value;
        v8bf x;
        if constexpr (D == 128) x = join(codes2<B>(n[0]), codes2<B>(n[1]), codes2<B>(n[2]), codes2<B>(n[3]));
        else x = join(codes2<B>(n[0]), codes2<B + 2>(n[0]), codes2<B>(n[1]), codes2<B + 2>(n[1]));
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
          o[nt][e] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x, ph[nt][u], o[nt][e], 0, 0, 0);
          o[nt][e] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x, pl[nt][u], o[nt][e], 0, 0, 0);
        }
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

  // join the four waves
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    l[nt] += lane_xor<16>(l[nt]);
    l[nt] += lane_xor<32>(l[nt]);
    if (lane < 16) {
      sm[w][nt * 16 + lane] = m[nt];
      sl[w][nt * 16 + lane] = l[nt];
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
        *reinterpret_cast<float4*>(dst + e) = make_float4(o[nt][e][r], o[nt][e + 1][r], o[nt][e + 2][r], o[nt][e + 3][r]);
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
        for (int x = 0; x < D / 64; ++x) y[x] += f * so[i][rr][lane * (D / 64) + x];
      }
      if (p.parts == 1) {
        const int i = (p.tile * M + row) / a.G;
        finish_row<D>(a, p.q.q0 + i, h * a.G + p.tile * M + row - i * a.G, y, mm, ll, lane);
      } else {
        const int64_t at = (static_cast<int64_t>(p.slot + p.part) * a.g.Hkv + h) * M + row;
#pragma unroll
        for (int x = 0; x < D / 64; ++x) a.part_o[at * D + lane * (D / 64) + x] = y[x];
        if (lane == 0) a.part_ml[at] = make_float2(mm, ll);
      }
    }
  }
}

// Joins the parts of split tiles, a wave per row.
template <int D, int M>
__global__ __launch_bounds__(256) void k_merge(CacheAttnArgs a) {
  __shared__ SchedShared sched;
  Piece p;
  if (!find_piece<M>(a, sched, blockIdx.x, true, &p)) return;
  const int lane = threadIdx.x & 63, h = blockIdx.y;
  const int rows = p.q.ql * a.G - p.tile * M < M ? p.q.ql * a.G - p.tile * M : M;
  for (int row = threadIdx.x >> 6; row < rows; row += 4) {
    float mm = kNegInf;
    for (int i = 0; i < p.parts; ++i)
      mm = fmaxf(mm, a.part_ml[(static_cast<int64_t>(p.slot + i) * a.g.Hkv + h) * M + row].x);
    float l = 0.0f, y[D / 64] = {};
    for (int i = 0; i < p.parts; ++i) {
      const int64_t at = (static_cast<int64_t>(p.slot + i) * a.g.Hkv + h) * M + row;
      const float2 ml = a.part_ml[at];
      const float f = rescale(ml.x, mm);
      l += f * ml.y;
#pragma unroll
      for (int x = 0; x < D / 64; ++x) y[x] += f * a.part_o[at * D + lane * (D / 64) + x];
    }
    const int i = (p.tile * M + row) / a.G;
    finish_row<D>(a, p.q.q0 + i, h * a.G + p.tile * M + row - i * a.G, y, mm, l, lane);
  }
}

constexpr int kPieces = 1024;   // pieces of work over all KV heads aimed at

template <int D>
hipError_t attn_d(const CacheAttnArgs& a, hipStream_t s) {
  constexpr int M = 32;
  const int64_t per = (static_cast<int64_t>(a.max_q) * a.G + M - 1) / M;
  int64_t tiles = a.R + static_cast<int64_t>(a.T) * a.G / M;
  if (tiles > a.R * per) tiles = a.R * per;
  k_few<D, 2><<<dim3(static_cast<unsigned>(tiles + a.target), a.g.Hkv), dim3(256), 0, s>>>(a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const int64_t merges = tiles < a.target ? tiles : a.target;
  k_merge<D, M><<<dim3(static_cast<unsigned>(merges), a.g.Hkv), dim3(256), 0, s>>>(a);
  return hipGetLastError();
}

}  // namespace

int cache_attn_target(int Hkv) { return (kPieces + Hkv - 1) / Hkv; }

size_t cache_attn_partial_bytes(int D, int Hkv, int G, int max_q, size_t* ml_offset) {
  (void)G;
  (void)max_q;
  const size_t rows = static_cast<size_t>(2) * cache_attn_target(Hkv) * Hkv * 32;
  *ml_offset = rows * D * sizeof(float);
  return rows * (D * sizeof(float) + sizeof(float2));
}

hipError_t launch_cache_attn(const CacheAttnArgs& a, int D, hipStream_t s) {
  return D == 128 ? attn_d<128>(a, s) : attn_d<64>(a, s);
}

}  // namespace ra
