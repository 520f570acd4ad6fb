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

// The two kernels share a call's requests by their number of rows: up to
// kFewRows a request is bound by its keys (k_few), above by the matrix cores
// (k_rows).
constexpr int kFewRows = 32;
// blocks of the least part: a step of 32 keys for each of the four waves of
// k_few, twice; for k_rows enough to pay for a partial output of M rows
template <int M>
constexpr int least_blocks() { return M <= kFewRows ? 4 : 16; }

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
  return x;
}

struct Piece {
  Request q;
  int r, tile, part, parts, slot;   // slot: place in the workspace of part 0 of this tile
};

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

// Blocks of a part, W blocks in all: at least W / target, the sum's roundings
// (the same in every workgroup) included.
template <int M>
__device__ __forceinline__ unsigned part_blocks(float W, int target) {
  const float c = W * (1.0f + 0x1p-10f) / static_cast<float>(target) + 1.0f;
  const unsigned C = c < 0x1p26f ? static_cast<unsigned>(c) : 1u << 26;   // a request has 2^24 at most
  return C < static_cast<unsigned>(least_blocks<M>()) ? least_blocks<M>() : C;
}

// Piece number x (or, for the merge, tile number x of those with several
// parts); false past the end.  All 256 threads of the workgroup call it.  Up to
// 64 requests every wave finds it alone, from one load of the lengths; above,
// 256 requests at a time through LDS.
template <int M>
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
  };
  if (a.R <= 64) {
    Request q = {};
    if (lane < a.R) q = request_of<M>(a, lane);
    const float W = wave_total(static_cast<float>(q.tiles) * static_cast<float>(q.blocks));
    const int n = parts_of(q, part_blocks<M>(W, target));
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
  Request q0 = {};
  for (int r = tid; r < a.R; r += 256) {
    const Request q = request_of<M>(a, r);
    if (r == tid) q0 = q;
    W += static_cast<float>(q.tiles) * static_cast<float>(q.blocks);
  }
  W = wave_total(W);
  if (lane == 0) sh.w[w] = W;
  if (tid == 0) sh.hit[0] = -1;
  __syncthreads();
  const unsigned C = part_blocks<M>((sh.w[0] + sh.w[1]) + (sh.w[2] + sh.w[3]), target);
  int base = 0, slot = 0;
  for (int r0 = 0; r0 < a.R; r0 += 256) {
    const int r = r0 + tid;
    Request q = {};
    if (r < a.R) q = r0 == 0 ? q0 : request_of<M>(a, r);
    const int n = parts_of(q, C);
    const int split = n > 1 ? q.tiles * n : 0, mine = merge ? (n > 1 ? q.tiles : 0) : q.tiles * n;
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
  float back[NT];       // FINE: what scores are multiplied by
  int hi[NT], lo[NT];   // keys that the lane's row sees: [lo, hi)
};

// One step of 16 KT keys for the first 16 N rows.  `there` bit i: the i-th 16 keys are on a page; whole:
// every row sees every key.
//
// Control flow here must not skip over a block between a matrix product and the
// first use of its result: the compiler then leaves out the wait states that
// the use needs on the skipping path (seen as wrong first registers when the
// second 16 rows were skipped inside the step).  N is therefore a constant.
template <int D, int NT, int N, int KT, bool FINE>
__device__ __forceinline__ void few_step(Rows<D, NT>& x, const uint4* sq, const Tile16<D> (&t)[KT], unsigned there, bool whole, int key0,
                                          int g) {
  constexpr int KC = D / 32;
  v4f s[N][KT];
#pragma unroll
  for (int i = 0; i < KT; ++i) {
#pragma unroll
    for (int nt = 0; nt < N; ++nt) s[nt][i] = v4f{0, 0, 0, 0};
#pragma unroll
    for (int c = 0; c < KC; ++c) {
      const uint4 k = codes8<FINE>(dword_of<D>(t[i].k, c));
#pragma unroll
      for (int nt = 0; nt < N; ++nt) {
        s[nt][i] = score16<FINE>(k, sq[(nt * KC + c) * 128], s[nt][i]);
        s[nt][i] = score16<FINE>(k, sq[(nt * KC + c) * 128 + 64], s[nt][i]);
      }
    }
    const float ks[4] = {t[i].ks.x, t[i].ks.y, t[i].ks.z, t[i].ks.w};
#pragma unroll
    for (int nt = 0; nt < N; ++nt) {
      const float base = x.m[nt] == kNegInf ? 0.0f : x.m[nt];
#pragma unroll
      for (int e = 0; e < 4; ++e) s[nt][i][e] = __fmaf_rn(s[nt][i][e], FINE ? ks[e] * x.back[nt] : ks[e], -base);
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
          const bool on = ((there >> i) & 1) && key < x.hi[nt] && key >= x.lo[nt];
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

template <int D, int NT, int KT, bool FINE>
__device__ __forceinline__ void few_rows(const CacheAttnArgs& a) {
  constexpr int M = 16 * NT, E = D / 16, kStep = 16 * KT, S = kBlock / kStep;
  constexpr int kStride = D + 4;                       // floats, against bank conflicts
  __shared__ __align__(16) float so[4][16][kStride];
  __shared__ float sm[4][M], sl[4][M];
  __shared__ SchedShared sched;
  __shared__ __align__(16) uint4 sq_all[NT * (D / 32) * 128];   // [nt][channel step][hi, lo][lane]
  __shared__ float sback[FINE ? M : 1];
  const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6), g = lane >> 4;
  // heads fastest: the heads of a page, neighbours in memory, are read together
  const int x0 = blockIdx.x / a.g.Hkv, h = blockIdx.x - x0 * a.g.Hkv;
  Piece p;
  if (!find_piece<M>(a, sched, x0, false, a.target, &p)) return;

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
  auto ids_from = [&](int t16) {   // (looked at when used, so that nothing waits here)
    const int t = t16 + lane;
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
      load_tile<D>(a, t[i], page ? id : 0, h, (b * KT + i) * 16, lane);
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
    if (w == nt) {   // one wave for all four
      uint4 qh[D / 32], ql[D / 32];
      const float back = load_q<D, FINE>(a, p, h, row, lane, qh, ql);
      if (FINE && lane < 16) sback[nt * 16 + lane] = back;
#pragma unroll
      for (int c = 0; c < D / 32; ++c) {
        sq_all[(nt * (D / 32) + c) * 128 + lane] = qh[c];
        sq_all[(nt * (D / 32) + c) * 128 + 64 + lane] = ql[c];
      }
    }
    const int pos = first + row / a.G;
    x.hi[nt] = a.causal ? pos + 1 : p.q.n;
    if (x.hi[nt] > p.q.n) x.hi[nt] = p.q.n;
    x.lo[nt] = a.window ? pos - a.window + 1 : 0;
    x.m[nt] = kNegInf;
    x.l[nt] = 0.0f;
#pragma unroll
    for (int e = 0; e < E; ++e) x.o[nt][e] = v4f{0, 0, 0, 0};
  }
  __syncthreads();
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) x.back[nt] = FINE ? sback[nt * 16 + (lane & 15)] : 1.0f;
  auto whole = [&](int b, unsigned there) {
    return b * kStep >= all_lo && b * kStep + kStep <= all_hi && b * kStep + kStep <= p.q.n && there == (1u << KT) - 1;
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
        few_step<D, NT, N, KT, FINE>(x, sq_all + lane, ring[i], there[i], whole(b + i, there[i]), (b + i) * kStep, g);
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

template <int D, int NT, int KT>
__global__ __launch_bounds__(256, 2) void k_few(CacheAttnArgs a) {
  few_rows<D, NT, KT, false>(a);
}
template <int D, int NT, int KT>
__global__ __launch_bounds__(256, 2) void k_fine_few(CacheAttnArgs a) {
  few_rows<D, NT, KT, true>(a);
}

// --------------------------------------------------------- many rows per request --
//
// Bound by the matrix cores and the softmax beside them.  NW waves of 32 rows
// share tiles of 64 keys in LDS, as bf16 values of the codes (exact), scales
// apart: each wave loads its share of the next tile's codes while the present
// one is computed, and converts them into the other LDS buffer at its end.
// S^T = K Q^T and O^T += V^T P^T on the 32x32x16 product: a lane holds one
// query's scores (key 32 c + 8 (r / 4) + 4 hh + r % 4 in register r of chunk
// c), which rounded to 16 bits are the second operand of the next product, and
// the same query's output, so that rescaling it is a factor per lane.
//
// Q (after RoPE, rotation and scale, in binary32) is the sum of two bf16
// values, within 2^-17 of each element.  P * (V's scale) is one, within 2^-8,
// where the output is bf16, which is then 2.3e-3 off (relative) instead of
// 1.7e-3, and two (LO) where it is binary16: prompts of 26k tokens take 2.0 ms
// with one and 2.5 ms with two.  (Binary32 outputs: FINE, above.)  Both are bf16
// for binary16 inputs as well, whose range holds neither a scaled Q (the softmax
// scale is the caller's) nor a weight up to 2^8 times a scale from 2^-100 to
// 2^127: in units of a tile's largest scale, binary16 loses the rows that do not
// see that token.
//
// LDS: K [chunk of 8 channels][key], V [octet of keys][channel position], 16
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

// As load_q, D / 2 channels per lane.
template <int D, bool F16, bool FINE>
__device__ __forceinline__ float load_q32(const CacheAttnArgs& a, const Piece& p, int h, int row, int lane,
                                          uint4 (&hi)[D / 16], uint4 (&lo)[D / 16]) {
  constexpr int N = D / 2;
  const int hh = lane >> 5;
  const bool ok = row < p.q.ql * a.G;
  const int i = ok ? row / a.G : 0, head = h * a.G + (ok ? row - i * a.G : 0);
  float y[N];
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

// Pipeline over tiles: a tile begins with its scores in registers.  Once a
// chunk of 32 keys has its probabilities, its score registers take the next
// tile's scores of that chunk; those products and the chunk's P V run on the
// matrix cores beside the next chunk's probabilities, their LDS operands read
// kAhead products ahead.  So K is staged two tiles ahead and V (with both
// scales) one, and two LDS buffers of each suffice.
// TERMS: bf16 values that hold P * (V's scale); three come with binary16 pairs of Q.
template <int D, bool F16, int TERMS>
__device__ __forceinline__ void many_rows(const CacheAttnArgs& a) {
  constexpr bool FINE = TERMS == 3;
  typedef typename std::conditional<D == 128, uint4, uint2>::type Codes;   // a lane's share of 16 tokens
  constexpr int NW = 4, M = 32 * NW, E = D / 16, KC = D / 16, MT = D / 32;
  struct Scales {
    float ks[64], vs[64];
    unsigned long long there, plain;   // keys that are on a page; those of them with a finite V
  };
  struct Buf {
    uint4 k[2][D / 8][64];
    uint4 v[2][8][D];
    Scales sc[2];
  };
  __shared__ __align__(16) Buf buf;
  __shared__ SchedShared sched;
  const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int hh = lane >> 5, j = lane & 31;
  // heads fastest: workgroups go round the 8 XCDs, so a head's keys stay in few L2s
  const int x0 = blockIdx.x / a.g.Hkv, h = blockIdx.x - x0 * a.g.Hkv;
  Piece p;
  if (!find_piece<M>(a, sched, x0, false, a.target_rows, &p)) return;
  if (a.causal) p.tile = p.q.tiles - 1 - p.tile;   // the longest first

  const int rows = p.q.ql * a.G - p.tile * M < M ? p.q.ql * a.G - p.tile * M : M;
  const int first = p.q.first;
  const int i0 = p.tile * M / a.G, i1 = (p.tile * M + rows - 1) / a.G;
  int hi = p.q.n, lo = 0;
  if (a.causal) hi = first + i1 + 1;
  if (hi < 0) hi = 0;
  if (a.window) lo = first + i0 - a.window + 1 > 0 ? first + i0 - a.window + 1 : 0;
  const int bl = lo / kBlock, bh = hi > lo ? (hi + kBlock - 1) / kBlock : bl;
  const int per = (bh - bl + p.parts - 1) / p.parts;
  const int b0 = bl + p.part * per, b1 = b0 + per < bh ? b0 + per : bh;
  // bounds that every row of this wave sees, and its lane's row
  const int wrow = p.tile * M + w * 32, row = wrow + j;
  const int wi0 = wrow / a.G, wi1 = wrow + 31 < p.tile * M + rows - 1 ? (wrow + 31) / a.G : i1;
  const int all_hi = a.causal ? first + wi0 + 1 : p.q.n;
  const int all_lo = a.window ? first + wi1 - a.window + 1 : 0;
  // tiles from t1 on hold no key that a row of this wave sees; a wave behind the rows of the tile has none at all
  int t1 = a.causal ? (first + wi1 + kBlock) / kBlock : b1;
  if (t1 > b1) t1 = b1;
  if (w * 32 >= rows || t1 < b0) t1 = b0;
  const int pos = first + row / a.G;
  int row_hi = a.causal ? pos + 1 : p.q.n;
  if (row_hi > p.q.n) row_hi = p.q.n;
  const int row_lo = a.window ? pos - a.window + 1 : 0;

  const int page = a.g.page, page_log = a.g.page_log;
  const int* row_table = a.block_table + static_cast<int64_t>(p.r) * a.max_blocks;
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
  auto within = [&](int b) { return b < b1 ? b : b1 - 1; };
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
    bk = within(bk);
    const int cv = within(bv);
    const int tk = (bk * kBlock + mine) & (page - 1), tv = (cv * kBlock + mine) & (page - 1);
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
    entries(bk + 1, cv + 1);
  };
  // The staged codes into LDS, in four parts each.  What is written past the
  // last tile replaces tiles that are done with.
  auto put_k = [&](int b, auto part) {
    constexpr int c = decltype(part)::value;
    if constexpr (c < D / 32) {
      const uint32_t x = dword_of<D>(sk, c);
      buf.k[b & 1][(lane >> 4) * (D / 32) + c][mine + (lane & 15)] =
          codes8<FINE>(x);
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
  uint4 q[KC], q_lo[KC];
  const float back = load_q32<D, F16, FINE>(a, p, h, row, lane, q, q_lo);
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

  auto k_op = [&](int b, int c, int kc) { return buf.k[b & 1][hh * KC + kc][c * 32 + j]; };
#pragma unroll
  for (int c = 0; c < 2; ++c) {
#pragma unroll
    for (int r = 0; r < 16; ++r) s[c][r] = 0.0f;
#pragma unroll
    for (int kc = 0; kc < KC; ++kc) {
      const uint4 k = k_op(b0, c, kc);
      s[c] = score32<FINE>(k, q[kc], s[c]);
      s[c] = score32<FINE>(k, q_lo[kc], s[c]);
    }
    settle(s[c]);
  }
  __syncthreads();   // tile b0's K is read before tile b0 + 2's takes its place

  auto step = [&](int b) {
    // the waves of a SIMD alternate: the dependent chain of vector work at the
    // higher priority, the products behind it at the lower one
    __builtin_amdgcn_s_setprio(1);
    const Scales& t = buf.sc[b & 1];
    const int key0 = b * kBlock;
    const float base = m == kNegInf ? 0.0f : m;
    float x[2][16], mx = kNegInf;
#pragma unroll
    for (int c = 0; c < 2; ++c) {
#pragma unroll
      for (int r = 0; r < 16; r += 4) {
        float4 k4 = *reinterpret_cast<const float4*>(&t.ks[c * 32 + 2 * r + 4 * hh]);
        if constexpr (FINE) k4.x *= back, k4.y *= back, k4.z *= back, k4.w *= back;
        x[c][r] = __fmaf_rn(s[c][r], k4.x, -base);
        x[c][r + 1] = __fmaf_rn(s[c][r + 1], k4.y, -base);
        x[c][r + 2] = __fmaf_rn(s[c][r + 2], k4.z, -base);
        x[c][r + 3] = __fmaf_rn(s[c][r + 3], k4.w, -base);
      }
    }
    const unsigned long long plain = t.plain;
    if (key0 < all_lo || key0 + kBlock > all_hi || plain != ~0ull) {
      unsigned long long on = t.there & bits_below(row_hi - key0) & ~bits_below(row_lo - key0);
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
          s[c] = score32<FINE>(op, q[i / 2], s[c]);
          s[c] = score32<FINE>(op, q_lo[i / 2], s[c]);
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

  // out through LDS, 8 rows of each wave at a time
  l += lane_xor<32>(l);
  constexpr int kStride = D + 4;
  static_assert(sizeof(buf) >= NW * 8 * kStride * sizeof(float), "the output rows pass through the tiles' LDS");
  float* so = reinterpret_cast<float*>(&buf) + w * 8 * kStride;
#pragma unroll
  for (int round = 0; round < 4; ++round) {
    __syncthreads();
    if ((j >> 3) == round) {
      // register r of tile i: position 32 i + 8 (r / 4) + 4 hh + r % 4 = e * 16 + chunk
#pragma unroll
      for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const int e = 2 * i + (r >> 3), chunk = 8 * ((r >> 2) & 1) + 4 * hh + (r & 3);
          so[(j & 7) * kStride + chunk * E + e] = o[i][r];
        }
    }
    __syncthreads();
#pragma unroll 1
    for (int k = 0; k < 8; ++k) {
      const int rr = w * 32 + round * 8 + k;
      if (rr >= rows) break;
      const float mm = __shfl(m, round * 8 + k), ll = __shfl(l, round * 8 + k);
      float y[D / 64];
#pragma unroll
      for (int z = 0; z < D / 64; ++z) y[z] = so[k * kStride + lane * (D / 64) + z];
      if (p.parts == 1) {
        const int i = (p.tile * M + rr) / a.G;
        finish_row<D>(a, p.q.q0 + i, h * a.G + p.tile * M + rr - i * a.G, y, mm, ll, lane);
      } else {
        const int64_t at = (static_cast<int64_t>(p.slot + p.part) * a.g.Hkv + h) * M + rr;
#pragma unroll
        for (int z = 0; z < D / 64; ++z) a.part_o[at * D + lane * (D / 64) + z] = y[z];
        if (lane == 0) a.part_ml[at] = make_float2(mm, ll);
      }
    }
  }
}

template <int D, bool F16, bool LO>
__global__ __launch_bounds__(256, 2) void k_rows(CacheAttnArgs a) {
  many_rows<D, F16, LO ? 2 : 1>(a);
}
template <int D, bool F16>
__global__ __launch_bounds__(256, 2) void k_fine_rows(CacheAttnArgs a) {
  many_rows<D, F16, 3>(a);
}

// Joins the parts of split tiles, a workgroup for per_group rows: up to eight
// parts a wave per row, else one row after the other, the parts' weights first,
// then the sum of their outputs, eight at a time (D / 4 threads each).
constexpr int kMostParts = 2048;   // 2 * target at most, one KV head

template <int D, int M>
__global__ __launch_bounds__(256) void k_merge(CacheAttnArgs a, int target, int per_group) {
  constexpr int W = D / 4, NG = 256 / W;
  __shared__ SchedShared sched;
  __shared__ float f[kMostParts];
  __shared__ float red[8];
  __shared__ __align__(16) float4 sum[NG][W];
  Piece p;
  if (!find_piece<M>(a, sched, blockIdx.x, true, target, &p)) return;
  if (M > kFewRows && a.causal) p.tile = p.q.tiles - 1 - p.tile;   // as k_rows numbers them
  const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6, h = blockIdx.y;
  int rows = p.q.ql * a.G - p.tile * M < M ? p.q.ql * a.G - p.tile * M : M;
  const int row0 = blockIdx.z * per_group;
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

template <int D, int M>
hipError_t merge(const CacheAttnArgs& a, const Grid& g, int target, int64_t rows, hipStream_t s) {
  if (rows > M) rows = M;
  // a workgroup per row while those are few enough to run at once
  const int per_group = g.merges * a.g.Hkv * rows <= 4096 ? 1 : M > kFewRows ? 16 : 8;
  k_merge<D, M><<<dim3(static_cast<unsigned>(g.merges), a.g.Hkv, static_cast<unsigned>((rows + per_group - 1) / per_group)),
                  dim3(256), 0, s>>>(a, target, per_group);
  return hipGetLastError();
}

template <int D, int NT>
hipError_t few(const CacheAttnArgs& a, hipStream_t s) {
  constexpr int M = 16 * NT;
  Grid g;
  g.tiles = a.R;   // a request of few rows is one tile
  g.merges = g.tiles < a.target ? g.tiles : a.target;
  const dim3 grid(static_cast<unsigned>((g.tiles + a.target) * a.g.Hkv));
  if (a.out_dtype == RA_FP32) k_fine_few<D, NT, 2><<<grid, dim3(256), 0, s>>>(a);
  else k_few<D, NT, 2><<<grid, dim3(256), 0, s>>>(a);
  const hipError_t e = hipGetLastError();
  return e != hipSuccess ? e : merge<D, M>(a, g, a.target, static_cast<int64_t>(a.max_q) * a.G, s);
}

template <int D, bool F16>
hipError_t rows(const CacheAttnArgs& a, hipStream_t s) {
  const Grid g = grid_of(a, kRowTile, a.target_rows);
  const dim3 grid(static_cast<unsigned>((g.tiles + a.target_rows) * a.g.Hkv));
  // P in as many bf16 values as the output shows
  if (a.out_dtype == RA_FP32) k_fine_rows<D, F16><<<grid, dim3(256), 0, s>>>(a);
  else if (a.out_dtype == RA_FP16) k_rows<D, F16, true><<<grid, dim3(256), 0, s>>>(a);
  else k_rows<D, F16, false><<<grid, dim3(256), 0, s>>>(a);
  const hipError_t e = hipGetLastError();
  return e != hipSuccess ? e : merge<D, kRowTile>(a, g, a.target_rows, static_cast<int64_t>(a.max_q) * a.G, s);
}

template <int D>
hipError_t attn_d(const CacheAttnArgs& a, hipStream_t s) {
  const int64_t most = static_cast<int64_t>(a.max_q) * a.G;
  if (most <= 16) return few<D, 1>(a, s);
  hipError_t e = hipSuccess;
  if (a.G <= kFewRows) e = few<D, 2>(a, s);   // requests of few rows; with more heads than that there are none
  if (e != hipSuccess || most <= kFewRows) return e;
  return a.is_fp16 ? rows<D, true>(a, s) : rows<D, false>(a, s);
}

int target_of(int pieces, int Hkv) { return (pieces + Hkv - 1) / Hkv; }

}  // namespace

// Partial outputs: 2 * target tiles' worth, of either kernel (one after the other).
size_t cache_attn_partial_bytes(int D, int Hkv, int G, int max_q, size_t* ml_offset) {
  size_t rows = static_cast<size_t>(2) * target_of(kPieces, Hkv) * Hkv * kFewRows;
  if (static_cast<int64_t>(max_q) * G > kFewRows) {
    const size_t many = static_cast<size_t>(2) * target_of(kRowPieces, Hkv) * Hkv * kRowTile;
    rows = rows > many ? rows : many;
  }
  *ml_offset = rows * D * sizeof(float);
  return rows * (D * sizeof(float) + sizeof(float2));
}

hipError_t launch_cache_attn(const CacheAttnArgs& a, int D, hipStream_t s) {
  CacheAttnArgs b = a;
  b.target = target_of(kPieces, a.g.Hkv);
  b.target_rows = target_of(kRowPieces, a.g.Hkv);
  return D == 128 ? attn_d<128>(b, s) : attn_d<64>(b, s);
}

}  // namespace ra
