// ra_cache.hip -- the 4-bit paged KV cache: tables from request lengths, the
// write of new tokens and the read back (gfx950).
#include "../../include/rotate_attn.h"
#include "ra_cache.h"

namespace ra {
namespace {

// ------------------------------------------------------------------- plan --
//
// A request with `old` cached and `n` new tokens holds ceil(old / P) pages and
// needs ceil((old + n) / P).  With sums over the requests before it,
//   q_start = sum n,   base = sum of pages taken,
// its i-th new page is free_pages[top - 1 - base - i], and its t-th new token
// (position old + t) goes to slot table[position / P] * P + position % P.
// All of it follows from two scans, so one workgroup makes the scans and each
// token then finds its request by bisection: a token that begins a block
// writes that block's table entry.  Bound by latency: a few dependent loads
// and barriers.
constexpr int kPlanThreads = 1024;
constexpr int kPlanTokens = 4096;   // tokens that one workgroup places

struct Scan2 {
  int a, b;
};

__device__ __forceinline__ Scan2 wave_scan(Scan2 v, int lane) {
#pragma unroll
  for (int d = 1; d < 64; d *= 2) {
    const int a = __shfl_up(v.a, d), b = __shfl_up(v.b, d);
    if (lane >= d) {
      v.a += a;
      v.b += b;
    }
  }
  return v;
}

struct PlanShared {
  Scan2 wave[kPlanThreads / 64];
  int first[kPlanThreads + 1];   // q_start of the chunk's requests
  int base[kPlanThreads];
  int old[kPlanThreads];
  long long sum[kPlanThreads / 64][4];
  int flags;
};

// Inclusive scan over the workgroup; *total gets the sum.
__device__ __forceinline__ Scan2 block_scan(Scan2 v, PlanShared& sh, Scan2* total) {
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  v = wave_scan(v, lane);
  __syncthreads();
  if (lane == 63) sh.wave[w] = v;
  __syncthreads();
  Scan2 t = {0, 0}, mine = {0, 0};
  for (int i = 0; i < kPlanThreads / 64; ++i) {
    if (i == w) mine = t;
    t.a += sh.wave[i].a;
    t.b += sh.wave[i].b;
  }
  *total = t;
  return {v.a + mine.a, v.b + mine.b};
}

__device__ __forceinline__ int blocks_of(int n, const PlanArgs& a) { return (n + a.page - 1) >> a.page_log; }

// Positions and slots of tokens [t0, t1) from final lengths, offsets and count
// (all of them written before), request chunk by request chunk.
__device__ void place_tokens(const PlanArgs& a, PlanShared& sh, int t0, int t1) {
  const int tid = threadIdx.x;
  const int total = a.q_start[a.R];
  for (int t = t0 + tid; t < t1; t += kPlanThreads)
    if (t >= total) {
      a.positions[t] = -1;
      a.slots[t] = -1;
    }
  if (t0 >= total) return;
  const int live = t1 < total ? t1 : total;
  // the stack's top before this call's pages were taken
  int carry_base = 0, taken = 0;
  if (a.status[0] == 0) taken = a.status[1];
  const int top = a.count_out[0] + taken;
  for (int r0 = 0; r0 < a.R; r0 += kPlanThreads) {
    const int r = r0 + tid;
    int old = 0, n = 0;
    if (r < a.R) {
      n = a.new_lens[r];
      old = a.seq_out[r] - n;
    }
    Scan2 tot;
    const int take = r < a.R ? blocks_of(old + n, a) - blocks_of(old, a) : 0;
    const Scan2 s = block_scan({take, 0}, sh, &tot);
    sh.base[tid] = carry_base + s.a - take;
    sh.old[tid] = old;
    if (r < a.R) sh.first[tid] = a.q_start[r];
    const int nr = a.R - r0 < kPlanThreads ? a.R - r0 : kPlanThreads;
    if (tid == 0) sh.first[nr] = a.q_start[r0 + nr];
    __syncthreads();
    const int lo = sh.first[0] > t0 ? sh.first[0] : t0, hi = sh.first[nr] < live ? sh.first[nr] : live;
    for (int t = lo + tid; t < hi; t += kPlanThreads) {
      int x = 0, y = nr;            // first[x] <= t < first[y]
      while (y - x > 1) {
        const int m = (x + y) >> 1;
        if (sh.first[m] <= t) x = m; else y = m;
      }
      const int o = sh.old[x], pos = o + (t - sh.first[x]);
      const int j = pos >> a.page_log, held = blocks_of(o, a);
      int64_t row = static_cast<int64_t>(r0 + x) * a.max_blocks;
      int pg;
      if (j < held) {
        pg = a.block_table[row + j];
      } else {
        pg = a.free_pages[top - 1 - sh.base[x] - (j - held)];
        if ((pos & (a.page - 1)) == 0) a.block_table[row + j] = pg;
      }
      a.positions[t] = pos;
      // an entry that is no page (a table the caller damaged) gives no slot
      a.slots[t] = static_cast<unsigned>(pg) < static_cast<unsigned>(a.num_pages)
                       ? (pg << a.page_log) + (pos & (a.page - 1)) : -1;
    }
    carry_base += tot.a;
    __syncthreads();
  }
}

__global__ __launch_bounds__(kPlanThreads) void k_plan(PlanArgs a, int place) {
  __shared__ PlanShared sh;
  const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
  // what is asked for, in 64 bits, and whether it can be had
  long long need = 0, tokens = 0, freed = 0;
  int longest = 0, flags = 0;
  if (tid == 0) sh.flags = 0;
  const long long most = static_cast<long long>(a.max_blocks) << a.page_log;
  for (int r = tid; r < a.R; r += kPlanThreads) {
    int old = a.seq_lens[r];
    const int n = a.new_lens[r];
    const bool drop = a.release && a.release[r];
    if (old < 0 || old > most || n < 0 || (drop ? 0 : old) + static_cast<long long>(n) > most) {
      flags = 1;
      continue;
    }
    if (drop) {
      freed += blocks_of(old, a);
      old = 0;
    }
    need += blocks_of(old + n, a) - blocks_of(old, a);
    tokens += n;
    longest = old + n > longest ? old + n : longest;
  }
#pragma unroll
  for (int d = 32; d; d >>= 1) {
    need += __shfl_xor(need, d);
    tokens += __shfl_xor(tokens, d);
    freed += __shfl_xor(freed, d);
    const int l2 = __shfl_xor(longest, d);
    longest = l2 > longest ? l2 : longest;
    flags |= __shfl_xor(flags, d);
  }
  __syncthreads();
  if (lane == 0) {
    sh.sum[w][0] = need;
    sh.sum[w][1] = tokens;
    sh.sum[w][2] = freed;
    sh.sum[w][3] = longest;
    if (flags) sh.flags = 1;   // every writer writes 1
  }
  __syncthreads();
  need = tokens = freed = 0;
  longest = 0;
  for (int i = 0; i < kPlanThreads / 64; ++i) {
    need += sh.sum[i][0];
    tokens += sh.sum[i][1];
    freed += sh.sum[i][2];
    longest = static_cast<int>(sh.sum[i][3]) > longest ? static_cast<int>(sh.sum[i][3]) : longest;
  }
  flags = sh.flags;
  const int count = a.free_count[0];
  if (count < 0 || count + freed > a.num_pages) flags |= 8;
  if (tokens > a.T) flags |= 2;
  if (!(flags & 8) && need > count + freed) flags |= 4;
  if (flags) {
    // refused as a whole: nothing changes, no request has queries
    __syncthreads();
    for (int r = tid; r < a.R; r += kPlanThreads) {
      a.seq_out[r] = a.seq_lens[r];
      a.q_start[r] = 0;
    }
    if (tid == 0) {
      a.q_start[a.R] = 0;
      a.count_out[0] = count;
    }
  } else {
    // pages of released requests back on the stack, in order of request and block
    if (freed) {
      int carry = 0;
      for (int r0 = 0; r0 < a.R; r0 += kPlanThreads) {
        const int r = r0 + tid;
        const bool drop = r < a.R && a.release[r];
        const int held = drop ? blocks_of(a.seq_lens[r], a) : 0;
        Scan2 tot;
        const Scan2 s = block_scan({held, 0}, sh, &tot);
        sh.base[tid] = carry + s.a - held;
        sh.old[tid] = held;
        __syncthreads();
        // a wave per request
        const int nr = a.R - r0 < kPlanThreads ? a.R - r0 : kPlanThreads;
        for (int i = w; i < nr; i += kPlanThreads / 64) {
          int* row = a.block_table + static_cast<int64_t>(r0 + i) * a.max_blocks;
          for (int j = lane; j < sh.old[i]; j += 64) {
            a.free_pages[count + sh.base[i] + j] = row[j];
            row[j] = -1;
          }
        }
        carry += tot.a;
        __syncthreads();
      }
    }
    int carry = 0;
    for (int r0 = 0; r0 < a.R; r0 += kPlanThreads) {
      const int r = r0 + tid;
      const int n = r < a.R ? a.new_lens[r] : 0;
      Scan2 tot;
      const Scan2 s = block_scan({n, 0}, sh, &tot);
      if (r < a.R) {
        a.q_start[r] = carry + s.a - n;
        a.seq_out[r] = (a.release && a.release[r] ? 0 : a.seq_lens[r]) + n;
      }
      carry += tot.a;
    }
    if (tid == 0) {
      a.q_start[a.R] = carry;
      a.count_out[0] = count + static_cast<int>(freed - need);
    }
  }
  if (tid == 0) {
    auto clamp = [](long long x) { return x > 0x7fffffff ? 0x7fffffff : static_cast<int>(x); };
    a.status[0] = flags;
    a.status[1] = clamp(need);
    a.status[2] = clamp(tokens);
    a.status[3] = longest;
  }
  if (place) {
    __syncthreads();   // this workgroup's own writes, read back through the same cache
    place_tokens(a, sh, 0, a.T);
  }
}

__global__ __launch_bounds__(kPlanThreads) void k_place(PlanArgs a) {
  __shared__ PlanShared sh;
  const int t0 = blockIdx.x * kPlanTokens;
  place_tokens(a, sh, t0, a.T - t0 < kPlanTokens ? a.T : t0 + kPlanTokens);
}

// ----------------------------------------------------------------- append --
//
// A row x of D channels (K after RoPE) is turned by the Sylvester-Hadamard
// butterflies y = H x without the factor 1/sqrt(D), a = max |y|, and kept as
//   code_i = E2M1(6 y_i / a)  (nearest, ties to the even code),  scale = a / 6 / sqrt(D).
// D / 8 lanes hold a row, 8 channels each; the larger stages of H and the
// maximum move registers between lanes.  Bound by HBM: 4 bytes in and 1 1/16
// out per channel of K and V together, at some 28 vector operations per value
// where both are rotated (12 of them the rotation).
//
// Which code a value gets is decided as 64 bits decide it.  16-bit inputs that
// are not turned meet borders exactly (x / a = 1/8, 5/12, ...), where 6x / a
// rounded in binary32 can fall on either side: such a quotient is off by less
// than 2^-20 and another one is at least 2^-14.6 away from the border, so it is
// first rounded to multiples of 2^-16, which puts it back on it.  Turned
// values meet borders only by chance: where 6y / a +- near_border() rounds to
// two codes the wave does the row again in binary64.
//
// near_border bounds what binary32 can do to a quotient t of at most 5 (u = 2^-24).
// A rounding in stage k of the 7 is at most u |z|.  The 2^(7-k) values z of that
// stage that reach an output reach as many outputs, whose mean square is theirs
// times 2^(7-k): a is at least the norm of these z, and their roundings move the
// output by at most u 2^((7-k)/2) a; all stages together by 24.9 u a.  RoPE's
// three roundings per value have a norm of at most (1 + sqrt 2) u times the
// row's, which a is not below, and reach an output through sqrt(128) of that:
// 27.3 u a.  With c u a for y and for a, 2 u t for the division and the product
// and 4 u for the sum with the margin, t is off by (11 c + 14) u:
//   rotated 288 u, after RoPE 589 u; RoPE alone (c = 2.42, a at least a pair's larger one) 41 u.
// The rms is about 4 u; rows made for it reach 80 u.
// The margin sends 1 wave in 34 (1 in 17 after RoPE) through binary64: append
// of 21845 tokens, K and V rotated, 40 us; a margin of 64 u took 37 and gave such
// rows other codes.
template <bool ROPE, bool HAD>
__host__ __device__ constexpr float near_border() {
  return !HAD ? 0x1p-18f : ROPE ? 0x1.3p-15f : 0x1.3p-16f;   // 64 u, 608 u, 304 u
}

// (lane: the lane's block of channels; a rotated row in binary32 comes times row_sign(lane))
template <typename F, int D, bool ROPE, bool HAD>
__device__ __forceinline__ void turn(const float (&x)[8], const float (&cs)[8], F (&y)[8], int lane) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const F a = x[2 * i], b = x[2 * i + 1];
    if constexpr (ROPE) {
      const F c = cs[2 * i], s = cs[2 * i + 1];
      y[2 * i] = a * c - b * s;
      y[2 * i + 1] = a * s + b * c;
    } else {
      y[2 * i] = a;
      y[2 * i + 1] = b;
    }
  }
  if constexpr (HAD) hadamard_row<D>(y, lane);
}

template <int B>
__device__ __forceinline__ uint32_t cvt_fp4(uint32_t old, float a, float b) {
  return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(old, a, b, 1.0f, B);
}
__device__ __forceinline__ uint32_t pack_fp4(const float (&y)[8]) {
  uint32_t r = cvt_fp4<0>(0, y[0], y[1]);
  r = cvt_fp4<1>(r, y[2], y[3]);
  r = cvt_fp4<2>(r, y[4], y[5]);
  return cvt_fp4<3>(r, y[6], y[7]);
}

template <int D>
__device__ __forceinline__ uint32_t row_max_bits(uint32_t m) {
  auto take = [&](int o) { m = static_cast<uint32_t>(o) > m ? static_cast<uint32_t>(o) : m; };
  take(lane_xor<1>(static_cast<int>(m)));
  take(lane_xor<2>(static_cast<int>(m)));
  take(lane_xor<7>(static_cast<int>(m)));
  if constexpr (D == 128) take(lane_xor<8>(static_cast<int>(m)));
  return m;
}

// Codes of the lane's 8 channels; *scale is the row's.
template <int D, bool ROPE, bool HAD>
__device__ __forceinline__ uint32_t quantise(const float (&x)[8], const float (&cs)[8], int lane, float* scale) {
  float y[8];
  turn<float, D, ROPE, HAD>(x, cs, y, lane);
  uint32_t m = 0;
  if constexpr (HAD) {
    // NaN where any is (a sum that leaves binary32 makes infinities, which cancel to NaN in some channels only)
    float f = 0.0f;
#pragma unroll
    for (int i = 0; i < 8; i += 2)
      f = __builtin_elementwise_maximum(__builtin_elementwise_maximum(f, fabsf(y[i])), fabsf(y[i + 1]));
    m = __float_as_uint(f) & 0x7fffffffu;
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const uint32_t b = __float_as_uint(y[i]) & 0x7fffffffu;   // as integers NaN and infinity are the largest
      m = b > m ? b : m;
    }
  }
  m = row_max_bits<D>(m);
  // a row of zeros (or below 2^-100) keeps scale 0; one that is not finite
  // has NaN for a scale and is NaN wherever it is attended to
  const bool finite = m < 0x7f800000u, tiny = m < 0x0d800000u;
  const float a = __uint_as_float(m);
  constexpr float norm = HAD ? (D == 128 ? 0.0883883476483184405501055452631f : 0.125f) : 1.0f;
  *scale = !finite ? __uint_as_float(0x7fc00000u) : tiny ? 0.0f : a / 6.0f * norm;
  const bool dead = !finite || tiny;
  const float inv = dead ? 0.0f : HAD ? 6.0f * row_sign(lane) / a : 6.0f / a;
  float lo[8], hi[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float t = y[i] * inv;
    if constexpr (ROPE || HAD) {
      const float by = copysignf(near_border<ROPE, HAD>(), t);
      hi[i] = t + by;
      lo[i] = t - by;
    } else {
      lo[i] = copysignf((fabsf(t) + 192.0f) - 192.0f, t);   // multiples of 2^-16
    }
  }
  uint32_t code = dead ? 0u : pack_fp4(ROPE || HAD ? hi : lo);
  if constexpr (ROPE || HAD) {
    // (magnitudes: they only differ in sign around 0, which is no border)
    if (__any(!dead && ((code ^ pack_fp4(lo)) & 0x77777777u))) {
      double z[8];
      turn<double, D, ROPE, HAD>(x, cs, z, lane);
      double zm = 0.0;
#pragma unroll
      for (int i = 0; i < 8; ++i) zm = fmax(zm, fabs(z[i]));
      zm = fmax(zm, lane_xor<1>(zm));
      zm = fmax(zm, lane_xor<2>(zm));
      zm = fmax(zm, lane_xor<7>(zm));
      if constexpr (D == 128) zm = fmax(zm, lane_xor<8>(zm));
      // 6 |z| against the borders times the maximum: no division, and a tie stays one
      constexpr double border[7] = {0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0};
      code = 0;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const double u = fabs(z[i]) * 6.0;
        uint32_t c = z[i] < 0.0 ? 8u : 0u;
#pragma unroll
        for (int k = 0; k < 7; ++k) c += k % 2 ? u >= border[k] * zm : u > border[k] * zm;
        code |= c << (4 * i);
      }
      code = dead ? 0u : code;
    }
  }
  return code;
}

__device__ __forceinline__ void unpack16(const uint4& w, int is_fp16, float (&x)[8]) {
  const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[2 * i] = cache_h2f(static_cast<uint16_t>(u[i] & 0xffff), is_fp16);
    x[2 * i + 1] = cache_h2f(static_cast<uint16_t>(u[i] >> 16), is_fp16);
  }
}

// A workgroup takes 2048 / D tokens and `heads` KV heads, head after head:
// tokens that follow each other fill the cache lines of a page together, and
// the cosines and sines of a token stay in registers.
template <int D, bool ROPE, bool HADK, bool HADV>
__global__ __launch_bounds__(256) void k_append(AppendArgs a) {
  constexpr int L = D / 8;
  const int lane = row_block(threadIdx.x & (L - 1));   // block of channels
  const int t = blockIdx.x * (256 / L) + threadIdx.x / L;
  const int slot = t < a.T ? a.slots[t] : -1;
  float cs[8] = {};
  bool ok = slot >= 0 && (slot >> a.g.page_log) < a.g.num_pages;
  if constexpr (ROPE) {
    const int pos = ok ? a.positions[t] : -1;
    ok = ok && pos >= 0 && pos < a.rope_rows;
    if (ok) {
      const float4* p = reinterpret_cast<const float4*>(a.rope + static_cast<int64_t>(pos) * D + lane * 8);
      const float4 c0 = p[0], c1 = p[1];
      cs[0] = c0.x, cs[1] = c0.y, cs[2] = c0.z, cs[3] = c0.w;
      cs[4] = c1.x, cs[5] = c1.y, cs[6] = c1.z, cs[7] = c1.w;
    }
  }
  const int page = a.g.page;
  const int tok = slot & (page - 1);
  const int h0 = blockIdx.y * a.heads, h1 = h0 + a.heads < a.g.Hkv ? h0 + a.heads : a.g.Hkv;
  // lanes without a token keep running: the moves between lanes need whole rows
  uint8_t* at = a.g.cache + (ok ? static_cast<int64_t>(slot >> a.g.page_log) * a.g.page_bytes : 0);
  const int64_t tt = ok ? t : 0;
  for (int h = h0; h < h1; ++h) {
    uint4 kw = {}, vw = {};
    if (ok) {
      kw = *reinterpret_cast<const uint4*>(a.k + tt * a.k_ts + h * a.k_hs + lane * 8);
      vw = *reinterpret_cast<const uint4*>(a.v + tt * a.v_ts + h * a.v_hs + lane * 8);
    }
    float x[8], ks, vs;
    unpack16(kw, a.is_fp16, x);
    const uint32_t kc = quantise<D, ROPE, HADK>(x, cs, lane, &ks);
    unpack16(vw, a.is_fp16, x);
    const uint32_t vc = quantise<D, false, HADV>(x, cs, lane, &vs);
    if (ok) {
      uint8_t* b = at + static_cast<int64_t>(h) * head_bytes<D>(page);
      const int kb = page * D / 2;
      // K: part of D/4 channels = D/32 lanes of 4 bytes
      *reinterpret_cast<uint32_t*>(b + (tok >> 4) * 8 * D + (lane / (D / 32)) * 2 * D + (tok & 15) * (D / 8) +
                                   (lane % (D / 32)) * 4) = kc;
      uint8_t* vb = b + kb + (tok >> 2) * 2 * D + (tok & 3) * (D / 32);
      if constexpr (D == 128) {
        *reinterpret_cast<uint32_t*>(vb + lane * 16) = vc;
      } else {
        *reinterpret_cast<uint16_t*>(vb + lane * 16) = static_cast<uint16_t>(vc);
        *reinterpret_cast<uint16_t*>(vb + lane * 16 + 8) = static_cast<uint16_t>(vc >> 16);
      }
      if (lane == 0) {
        float* sc = reinterpret_cast<float*>(b + 2 * kb);
        sc[tok] = ks;
        sc[page + tok] = vs;
      }
    }
  }
}

// ------------------------------------------------------------------- read --
//
// The values that cached tokens stand for, in the basis they were given in:
// code * scale, turned back by H / sqrt(D) (its own inverse), rounded once.
// Lanes as in the append.  Bound by HBM: (D + 8) bytes in, 2 D values out per
// token and head.
template <int D, bool HAD>
__device__ __forceinline__ void values(uint32_t code, float scale, int lane, float (&y)[8]) {
  typedef float v2f __attribute__((ext_vector_type(2)));
  const v2f p0 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code, 1.0f, 0);
  const v2f p1 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code, 1.0f, 1);
  const v2f p2 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code, 1.0f, 2);
  const v2f p3 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code, 1.0f, 3);
  y[0] = p0[0], y[1] = p0[1], y[2] = p1[0], y[3] = p1[1];
  y[4] = p2[0], y[5] = p2[1], y[6] = p3[0], y[7] = p3[1];
  if constexpr (HAD) {
    // sums of multiples of 1/2 up to 6 D: exact
    hadamard_row<D>(y, lane);
    scale *= row_sign(lane) * (D == 128 ? 0.0883883476483184405501055452631f : 0.125f);
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) y[i] *= scale;
}

__device__ __forceinline__ void store8(void* base, int64_t at, const float (&y)[8], int dtype) {
  if (dtype == RA_FP32) {
    float4* p = reinterpret_cast<float4*>(static_cast<float*>(base) + at);
    p[0] = make_float4(y[0], y[1], y[2], y[3]);
    p[1] = make_float4(y[4], y[5], y[6], y[7]);
    return;
  }
  const bool h = dtype == RA_FP16;
  *reinterpret_cast<uint4*>(static_cast<uint16_t*>(base) + at) =
      make_uint4(pack16(y[0], y[1], h), pack16(y[2], y[3], h), pack16(y[4], y[5], h), pack16(y[6], y[7], h));
}

template <int D, bool HADK, bool HADV>
__global__ __launch_bounds__(256) void k_read(ReadArgs a) {
  constexpr int L = D / 8;
  const int lane = row_block(threadIdx.x & (L - 1));   // block of channels
  const int t = blockIdx.x * (256 / L) + threadIdx.x / L;
  const int slot = t < a.T ? a.slots[t] : -1;
  const bool ok = slot >= 0 && (slot >> a.g.page_log) < a.g.num_pages;
  const int page = a.g.page, tok = slot & (page - 1), kb = page * D / 2;
  const int h0 = blockIdx.y * a.heads, h1 = h0 + a.heads < a.g.Hkv ? h0 + a.heads : a.g.Hkv;
  const uint8_t* at = a.g.cache + (ok ? static_cast<int64_t>(slot >> a.g.page_log) * a.g.page_bytes : 0);
  for (int h = h0; h < h1; ++h) {
    uint32_t kc = 0, vc = 0;
    float ks = 0.0f, vs = 0.0f;
    if (ok) {
      const uint8_t* b = at + static_cast<int64_t>(h) * head_bytes<D>(page);
      kc = *reinterpret_cast<const uint32_t*>(b + (tok >> 4) * 8 * D + (lane / (D / 32)) * 2 * D +
                                              (tok & 15) * (D / 8) + (lane % (D / 32)) * 4);
      const uint8_t* vb = b + kb + (tok >> 2) * 2 * D + (tok & 3) * (D / 32);
      if constexpr (D == 128) {
        vc = *reinterpret_cast<const uint32_t*>(vb + lane * 16);
      } else {
        vc = *reinterpret_cast<const uint16_t*>(vb + lane * 16) |
             static_cast<uint32_t>(*reinterpret_cast<const uint16_t*>(vb + lane * 16 + 8)) << 16;
      }
      const float* sc = reinterpret_cast<const float*>(b + 2 * kb);
      ks = sc[tok];
      vs = sc[page + tok];
    }
    float y[8];
    values<D, HADK>(kc, ks, lane, y);
    const int64_t out = (static_cast<int64_t>(t) * a.g.Hkv + h) * D + lane * 8;
    if (t < a.T) store8(a.k, out, y, a.out_dtype);
    values<D, HADV>(vc, vs, lane, y);
    if (t < a.T) store8(a.v, out, y, a.out_dtype);
  }
}

// Heads that a workgroup goes through: one while that makes too few workgroups
// to fill 256 compute units several times over, then as many as keep 2048 of
// them (the token's slot, position and angles are then read once for all).
int heads_per_group(int64_t token_groups, int Hkv) {
  int heads = 1;
  while (heads * 2 <= Hkv && token_groups * ((Hkv + heads * 2 - 1) / (heads * 2)) >= 2048) heads *= 2;
  return heads;
}

}  // namespace

hipError_t launch_cache_plan(const PlanArgs& a, hipStream_t s) {
  // up to one workgroup's tokens the scans and the tokens share a launch
  const bool one = a.T <= kPlanTokens;
  k_plan<<<dim3(1), dim3(kPlanThreads), 0, s>>>(a, one);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || one) return e;
  k_place<<<dim3((a.T + kPlanTokens - 1) / kPlanTokens), dim3(kPlanThreads), 0, s>>>(a);
  return hipGetLastError();
}

namespace {
template <int D, bool ROPE>
hipError_t append_d(const AppendArgs& a, bool hadk, bool hadv, dim3 grid, hipStream_t s) {
  if (hadk && hadv) k_append<D, ROPE, true, true><<<grid, dim3(256), 0, s>>>(a);
  else if (hadk) k_append<D, ROPE, true, false><<<grid, dim3(256), 0, s>>>(a);
  else if (hadv) k_append<D, ROPE, false, true><<<grid, dim3(256), 0, s>>>(a);
  else k_append<D, ROPE, false, false><<<grid, dim3(256), 0, s>>>(a);
  return hipGetLastError();
}
template <int D>
hipError_t read_d(const ReadArgs& a, bool hadk, bool hadv, dim3 grid, hipStream_t s) {
  if (hadk && hadv) k_read<D, true, true><<<grid, dim3(256), 0, s>>>(a);
  else if (hadk) k_read<D, true, false><<<grid, dim3(256), 0, s>>>(a);
  else if (hadv) k_read<D, false, true><<<grid, dim3(256), 0, s>>>(a);
  else k_read<D, false, false><<<grid, dim3(256), 0, s>>>(a);
  return hipGetLastError();
}
}  // namespace

hipError_t launch_cache_append(const AppendArgs& in, int D, bool hadk, bool hadv, hipStream_t s) {
  AppendArgs a = in;
  const int tokens = 2048 / D;
  const int64_t gx = (static_cast<int64_t>(a.T) + tokens - 1) / tokens;
  a.heads = heads_per_group(gx, a.g.Hkv);
  const dim3 grid(static_cast<unsigned>(gx), (a.g.Hkv + a.heads - 1) / a.heads);
  if (D == 128) return a.rope ? append_d<128, true>(a, hadk, hadv, grid, s) : append_d<128, false>(a, hadk, hadv, grid, s);
  return a.rope ? append_d<64, true>(a, hadk, hadv, grid, s) : append_d<64, false>(a, hadk, hadv, grid, s);
}

hipError_t launch_cache_read(const ReadArgs& in, int D, bool hadk, bool hadv, hipStream_t s) {
  ReadArgs a = in;
  const int tokens = 2048 / D;
  const int64_t gx = (static_cast<int64_t>(a.T) + tokens - 1) / tokens;
  a.heads = heads_per_group(gx, a.g.Hkv);
  const dim3 grid(static_cast<unsigned>(gx), (a.g.Hkv + a.heads - 1) / a.heads);
  return D == 128 ? read_d<128>(a, hadk, hadv, grid, s) : read_d<64>(a, hadk, hadv, grid, s);
}

}  // namespace ra
