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
// more than 16 rows.  Prefixes and requests are cut into pieces together (see
// the schedule in ra_cache_attn.h); every piece leaves its partial rows in the
// workspace, and a wave per row joins them.
//
// Bound by HBM while a group's rows are few, by the matrix cores and the softmax
// beside them from some 64 rows on.
#include "ra_cache_attn.h"

namespace ra {
namespace {

// A row's parts, 64 at a time: the request's own, then its prefix's.
template <int D>
__global__ __launch_bounds__(256) void k_join(CacheAttnArgs a) {
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  const int t = blockIdx.x, head = blockIdx.y * 4 + w;
  if (head >= a.Hq) return;
  int r = 0, y = a.R;   // q_start[r] <= t < q_start[y]
  while (y - r > 1) {
    const int m = (r + y) >> 1;
    if (a.q_start[m] <= t) r = m; else y = m;
  }
  const int q0 = a.q_start[r], q1 = a.q_start[r + 1];
  if (t < q0 || t >= q1) return;
  const int h = head / a.G, z = head - h * a.G;
  struct {
    int base, parts, rows, row;
    bool many;
  } s[2];
  const int from = q0 < 0 ? 0 : q0;
  auto parts_of = [&](int v, int first, int end, int which) {
    const int2 x = a.info[v];
    s[which].many = x.y < 0;
    s[which].parts = x.y < 0 ? -x.y : x.y;
    s[which].base = x.x;
    s[which].rows = ((end > a.T ? a.T : end) - first) * a.G;
    s[which].row = (t - first) * a.G + z;
  };
  parts_of(a.groups + r, from, q1, 0);
  s[1].parts = 0;
  const int g = group_of(a, r);
  if (g >= 0 && prefix_of(a, g) > 0) {
    const int r1 = a.group_start[g + 1] > a.R ? a.R : a.group_start[g + 1];
    const int first = a.q_start[a.group_start[g]];
    parts_of(g, first < 0 ? 0 : first, a.q_start[r1], 1);
  }
  // (more parts than the cutting makes: lengths changed under the call)
  const int n0 = s[0].parts < 65536 ? s[0].parts : 0, n = n0 + (s[1].parts < 65536 ? s[1].parts : 0);
  float M = kNegInf, L = 0.0f, out[D / 64] = {};
  for (int i0 = 0; i0 < n; i0 += 64) {
    const int i = i0 + lane;
    int64_t at = -1;
    if (i < n) {
      const bool own = i < n0;
      const int base = own ? s[0].base : s[1].base, part = own ? i : i - n0, rows = own ? s[0].rows : s[1].rows;
      const int row = own ? s[0].row : s[1].row, parts = own ? n0 : n - n0;
      at = (own ? s[0].many : s[1].many) ? shared_at<true>(a, base, parts, part, rows, row, h)
                                         : shared_at<false>(a, base, parts, part, rows, row, h);
    }
    const float2 ml = at >= 0 ? a.part_ml[at] : make_float2(kNegInf, 0.0f);
    float mm = ml.x;
#pragma unroll
    for (int d = 32; d; d >>= 1) mm = fmaxf(mm, __shfl_xor(mm, d));
    mm = fmaxf(M, mm);
    const float x = rescale(ml.x, mm), old = rescale(M, mm);
    float l = x * ml.y;
#pragma unroll
    for (int d = 32; d; d >>= 1) l += __shfl_xor(l, d);
    L = L * old + l;
    M = mm;
#pragma unroll
    for (int e = 0; e < D / 64; ++e) out[e] *= old;
    const int many = n - i0 < 64 ? n - i0 : 64;
    const int lo = static_cast<int>(at), hi = static_cast<int>(at >> 32);
    // eight at a time, so that their loads are under way together (places that are none: row 0, left out)
    for (int k0 = 0; k0 < many; k0 += 8) {
      float v[8][D / 64], f[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        f[k] = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(x), k0 + k));
        const int64_t p = static_cast<int64_t>(static_cast<uint64_t>(static_cast<uint32_t>(__builtin_amdgcn_readlane(hi, k0 + k))) << 32 |
                                               static_cast<uint32_t>(__builtin_amdgcn_readlane(lo, k0 + k)));
        const bool there = p >= 0;
#pragma unroll
        for (int e = 0; e < D / 64; ++e) v[k][e] = there ? a.part_o[p * D + lane * (D / 64) + e] : 0.0f;
      }
#pragma unroll
      for (int k = 0; k < 8; ++k)
#pragma unroll
        for (int e = 0; e < D / 64; ++e) out[e] += f[k] * v[k][e];
    }
  }
  finish_row<D>(a, t, head, out, M, L, lane);
}

template <int D>
hipError_t shared_d(const CacheAttnArgs& a, hipStream_t s) {
  const int64_t rows = static_cast<int64_t>(a.T) * a.G, all = static_cast<int64_t>(a.R) + a.groups;
  const dim3 few_grid(static_cast<unsigned>((all + a.target) * a.g.Hkv));
  if (a.out_dtype == RA_FP32) k_fine_few<D, 1, 2, kShared><<<few_grid, dim3(256), 0, s>>>(a);
  else k_few<D, 1, 2, kShared><<<few_grid, dim3(256), 0, s>>>(a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  if (rows > kFewShared) {
    // a prefix or request of many rows has more than kFewShared of them; prefixes and requests take every row once each
    const int64_t most = 2 * rows / kFewShared < all ? 2 * rows / kFewShared : all;
    const dim3 grid(static_cast<unsigned>((most + 2 * rows / kRowTile + a.target_rows) * a.g.Hkv));
    if (a.out_dtype == RA_FP32) {
      if (a.is_fp16) k_fine_rows<D, true, kShared><<<grid, dim3(256), 0, s>>>(a);
      else k_fine_rows<D, false, kShared><<<grid, dim3(256), 0, s>>>(a);
    } else if (a.out_dtype == RA_FP16) {
      if (a.is_fp16) k_rows<D, true, true, kShared><<<grid, dim3(256), 0, s>>>(a);
      else k_rows<D, false, true, kShared><<<grid, dim3(256), 0, s>>>(a);
    } else {
      if (a.is_fp16) k_rows<D, true, false, kShared><<<grid, dim3(256), 0, s>>>(a);
      else k_rows<D, false, false, kShared><<<grid, dim3(256), 0, s>>>(a);
    }
    e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  k_join<D><<<dim3(a.T, (a.Hq + 3) / 4), dim3(256), 0, s>>>(a);
  return hipGetLastError();
}

struct SharedSpace {
  int64_t rows;             // of every KV head
  size_t ml, info, bytes;   // offsets
};
// Rows of all parts: every row once for its prefix and once for its own keys,
// and those of the pieces that cutting adds (at most the targets, a tile each).
SharedSpace space_of(int D, int Hkv, int G, int R, int groups, int T) {
  SharedSpace x;
  x.rows = 2 * static_cast<int64_t>(T) * G + static_cast<int64_t>(kFewShared) * target_of(kPieces, Hkv) +
           static_cast<int64_t>(kRowTile) * target_of(kRowPieces, Hkv);
  const size_t n = static_cast<size_t>(x.rows) * Hkv;
  x.ml = n * D * sizeof(float);
  x.info = x.ml + n * sizeof(float2);
  x.bytes = x.info + (static_cast<size_t>(R) + groups) * sizeof(int2);
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
  b.info = reinterpret_cast<int2*>(ws + x.info);
  b.part_rows = x.rows;
  b.target = target_of(kPieces, a.g.Hkv);
  b.target_rows = target_of(kRowPieces, a.g.Hkv);
  return D == 128 ? shared_d<128>(b, s) : shared_d<64>(b, s);
}

}  // namespace ra
