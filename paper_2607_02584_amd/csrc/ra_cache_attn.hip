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
__device__ __forceinline__ void load_q(const CacheAttnArgs& a, const Piece& p, int h, int row, int lane, v8bf (&hi)[D / 32],
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
      split_bf16(y[8 * c + e] * a.c, x0, x1);   // scores come out in base 2
      hi[c][e] = x0;
      lo[c][e] = x1;
    }
}

template <int D>
__device__ __forceinline__ uint32_t dword_of(const typename std::conditional<D == 128, uint4, uint2>::type& v, int i) {
  if constexpr (D == 128) return i == 0 ? v.x : i == 1 ? v.y : i == 2 ? v.z : v.w;
  else return i == 0 ? v.x : v.y;
}

// The rows' state in a wave: Q, running maximum and sum, O^T.
template <int D, int NT>
struct Rows {
  v8bf qh[NT][D / 32], ql[NT][D / 32];
  v4f o[NT][D / 16];
  float m[NT], l[NT];
  int hi[NT], lo[NT];   // keys that the lane's row sees: [lo, hi)
};

// One step of 16 KT keys.  `there` bit i: the i-th 16 keys are on a page; whole:
// every row sees every key.
template <int D, int NT, int KT>
__device__ __forceinline__ void few_step(Rows<D, NT>& x, const Tile16<D> (&t)[KT], unsigned there, bool whole, int key0,
                                          int g) {
  constexpr int KC = D / 32;
  v4f s[NT][KT];
#pragma unroll
  for (int i = 0; i < KT; ++i) {
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) s[nt][i] = v4f{0, 0, 0, 0};
#pragma unroll
    for (int c = 0; c < KC; ++c) {
      const v8bf k = codes8(dword_of<D>(t[i].k, c));
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        s[nt][i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k, x.qh[nt][c], s[nt][i], 0, 0, 0);
        s[nt][i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k, x.ql[nt][c], s[nt][i], 0, 0, 0);
      }
    }
    const float ks[4] = {t[i].ks.x, t[i].ks.y, t[i].ks.z, t[i].ks.w};
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int e = 0; e < 4; ++e) s[nt][i][e] *= ks[e];
  }
  v8bf ph[NT][KT / 2], pl[NT][KT / 2];
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    unsigned seen = 0xffff;   // bit 4 i + e: this lane's row sees key 16 i + 4 g + e of the step
    if (!whole) {
      seen = 0;
#pragma unroll
      for (int i = 0; i < KT; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int key = key0 + 16 * i + 4 * g + e;
          const bool on = ((there >> i) & 1) && key < x.hi[nt] && key >= x.lo[nt];
          seen |= static_cast<unsigned>(on) << (4 * i + e);
          s[nt][i][e] = on ? s[nt][i][e] : kNegInf;
        }
    }
    float mx = x.m[nt];
#pragma unroll
    for (int i = 0; i < KT; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) mx = fmaxf(mx, s[nt][i][e]);
    mx = fmaxf(mx, lane_xor<16>(mx));
    mx = fmaxf(mx, lane_xor<32>(mx));
    const float ref = mx == kNegInf ? 0.0f : mx;   // nothing seen yet: any finite reference gives 0
    if (__any(mx != x.m[nt])) {
      const float alpha = __builtin_amdgcn_exp2f(x.m[nt] - ref);
      x.m[nt] = mx;
      x.l[nt] *= alpha;
#pragma unroll
      for (int e = 0; e < D / 16; ++e) x.o[nt][e] *= alpha;
    }
#pragma unroll
    for (int i = 0; i < KT; ++i) {
      const float vs[4] = {t[i].vs.x, t[i].vs.y, t[i].vs.z, t[i].vs.w};
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float pr = __builtin_amdgcn_exp2f(s[nt][i][e] - ref);
        x.l[nt] += pr;
        float w = pr * vs[e];
        // a scale that is not finite must not reach rows that do not see its token
        if (!whole) w = (seen >> (4 * i + e)) & 1 ? w : 0.0f;
        __bf16 x0, x1;
        split_bf16(w, x0, x1);
        ph[nt][i / 2][4 * (i % 2) + e] = x0;
        pl[nt][i / 2][4 * (i % 2) + e] = x1;
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
      for (int nt = 0; nt < NT; ++nt) {
        x.o[nt][e] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, ph[nt][u], x.o[nt][e], 0, 0, 0);
        x.o[nt][e] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, pl[nt][u], x.o[nt][e], 0, 0, 0);
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

template <int D, int NT, int KT>
__global__ __launch_bounds__(256, NT == 1 ? 2 : 1) void k_few(CacheAttnArgs a) {
  constexpr int M = 16 * NT, E = D / 16, kStep = 16 * KT, S = kBlock / kStep;
  constexpr int kStride = D + 4;                       // floats, against bank conflicts
  __shared__ __align__(16) float so[4][16][kStride];
  __shared__ float sm[4][M], sl[4][M];
  __shared__ SchedShared sched;
  const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6), g = lane >> 4;
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
  const int wper = (b1 - b0) > 0 ? ((b1 - b0) * S + 3) / 4 : 0;
  const int w0 = b0 * S + w * wper, w1 = w0 + wper < b1 * S ? w0 + wper : b1 * S;   // this wave's steps

  // Page numbers of 64 tiles of 16 keys at a time, one per lane, and of the 64 after them.
  const int page_shift = a.g.page_log - 4;
  const int* row_table = a.block_table + static_cast<int64_t>(p.r) * a.max_blocks;
  const int last16 = (p.q.n + 15) / 16;   // tiles that hold cached tokens
  auto ids_from = [&](int t16) {
    const int t = t16 + lane;
    const int id = t < last16 ? row_table[t >> page_shift] : -1;
    // an entry that is no page leaves its keys out
    return static_cast<unsigned>(id) < static_cast<unsigned>(a.g.num_pages) ? id : -1;
  };
  int ids = -1, ids_next = -1;
  if (w0 < w1) {
    ids = ids_from(w0 * KT);
    if (w0 + 64 / KT < w1) ids_next = ids_from(w0 * KT + 64);
  }
  auto load = [&](int b, Tile16<D> (&t)[KT]) {   // steps in order; returns the bits of pages that are there
    const int at = (b - w0) * KT;
    unsigned there = 0;
#pragma unroll
    for (int i = 0; i < KT; ++i) {
      const int id = __builtin_amdgcn_readlane(ids, (at + i) & 63);
      there |= static_cast<unsigned>(id >= 0) << i;
      load_tile<D>(a, t[i], id >= 0 ? id : 0, h, (b * KT + i) * 16, lane);
    }
    if (((at + KT) & 63) == 0) {   // the next step begins the next 64
      ids = ids_next;
      if (b + 1 + 64 / KT < w1) ids_next = ids_from((b + 1) * KT + 64);
    }
    return there;
  };

  Tile16<D> ta[KT], tb[KT];
  unsigned ha = 0, hb = 0;
  if (w0 < w1) ha = load(w0, ta);

  Rows<D, NT> x;
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    const int row = p.tile * M + nt * 16 + (lane & 15);
    load_q<D>(a, p, h, row, lane, x.qh[nt], x.ql[nt]);
    const int pos = first + row / a.G;
    x.hi[nt] = a.causal ? pos + 1 : p.q.n;
    if (x.hi[nt] > p.q.n) x.hi[nt] = p.q.n;
    x.lo[nt] = a.window ? pos - a.window + 1 : 0;
    x.m[nt] = kNegInf;
    x.l[nt] = 0.0f;
#pragma unroll
    for (int e = 0; e < E; ++e) x.o[nt][e] = v4f{0, 0, 0, 0};
  }
  auto whole = [&](int b, unsigned there) {
    return b * kStep >= all_lo && b * kStep + kStep <= all_hi && b * kStep + kStep <= p.q.n && there == (1u << KT) - 1;
  };
  // the next step's loads are in flight while a step is computed
  for (int b = w0; b < w1; b += 2) {
    if (b + 1 < w1) hb = load(b + 1, tb);
    __builtin_amdgcn_sched_barrier(0);
    few_step<D, NT, KT>(x, ta, ha, whole(b, ha), b * kStep, g);
    if (b + 1 >= w1) break;
    if (b + 2 < w1) ha = load(b + 2, ta);
    __builtin_amdgcn_sched_barrier(0);
    few_step<D, NT, KT>(x, tb, hb, whole(b + 1, hb), (b + 1) * kStep, g);
  }

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
      if (p.parts == 1) {
        const int i = (p.tile * M + row) / a.G;
        finish_row<D>(a, p.q.q0 + i, h * a.G + p.tile * M + row - i * a.G, y, mm, ll, lane);
      } else {
        const int64_t at = (static_cast<int64_t>(p.slot + p.part) * a.g.Hkv + h) * M + row;
#pragma unroll
        for (int z = 0; z < D / 64; ++z) a.part_o[at * D + lane * (D / 64) + z] = y[z];
        if (lane == 0) a.part_ml[at] = make_float2(mm, ll);
      }
    }
  }
}

// Joins the parts of split tiles, a workgroup per row: the parts' weights
// first, then the sum of their outputs, eight at a time (D / 4 threads each).
constexpr int kMostParts = 2048;   // 2 * target at most, one KV head

template <int D, int M>
__global__ __launch_bounds__(256) void k_merge(CacheAttnArgs a) {
  constexpr int W = D / 4, NG = 256 / W;
  __shared__ SchedShared sched;
  __shared__ float f[kMostParts];
  __shared__ float red[8];
  __shared__ __align__(16) float4 sum[NG][W];
  Piece p;
  if (!find_piece<M>(a, sched, blockIdx.x, true, &p)) return;
  const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6, h = blockIdx.y, row = blockIdx.z;
  const int rows = p.q.ql * a.G - p.tile * M < M ? p.q.ql * a.G - p.tile * M : M;
  if (row >= rows) return;
  const int64_t first = (static_cast<int64_t>(p.slot) * a.g.Hkv + h) * M + row;   // of part 0
  const int64_t step = static_cast<int64_t>(a.g.Hkv) * M;
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
  if (w) return;
  float out[D / 64] = {};
  const float* s = reinterpret_cast<const float*>(&sum[0][0]);
#pragma unroll
  for (int i = 0; i < NG; ++i)
#pragma unroll
    for (int x = 0; x < D / 64; ++x) out[x] += s[i * D + lane * (D / 64) + x];
  const int i = (p.tile * M + row) / a.G;
  finish_row<D>(a, p.q.q0 + i, h * a.G + p.tile * M + row - i * a.G, out, mm, l, lane);
}

constexpr int kPieces = 1024;   // pieces of work over all KV heads aimed at

template <int D, int NT>
hipError_t few(const CacheAttnArgs& a, hipStream_t s) {
  constexpr int M = 16 * NT;
  const int64_t per = (static_cast<int64_t>(a.max_q) * a.G + M - 1) / M;
  int64_t tiles = a.R + static_cast<int64_t>(a.T) * a.G / M;
  if (tiles > a.R * per) tiles = a.R * per;
  k_few<D, NT, 2><<<dim3(static_cast<unsigned>(tiles + a.target), a.g.Hkv), dim3(256), 0, s>>>(a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const int64_t merges = tiles < a.target ? tiles : a.target;
  const int64_t rows = static_cast<int64_t>(a.max_q) * a.G;
  k_merge<D, M><<<dim3(static_cast<unsigned>(merges), a.g.Hkv, static_cast<unsigned>(rows < M ? rows : M)), dim3(256), 0, s>>>(a);
  return hipGetLastError();
}

template <int D>
hipError_t attn_d(const CacheAttnArgs& a, hipStream_t s) {
  return static_cast<int64_t>(a.max_q) * a.G <= 16 ? few<D, 1>(a, s) : few<D, 2>(a, s);
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
