// ra_cache_attn.hip -- attention over the 4-bit paged KV cache (gfx950): the
// kernels of cache_attn and their launches.
#include "ra_cache_attn.h"

namespace ra {
namespace {

template <int D, int NT, int KT>
__global__ __launch_bounds__(256, 2) void k_few(CacheAttnArgs a) {
  few_rows<D, NT, KT, false>(a);
}
template <int D, int NT, int KT>
__global__ __launch_bounds__(256, 2) void k_fine_few(CacheAttnArgs a) {
  few_rows<D, NT, KT, true>(a);
}

template <int D, bool F16, bool LO>
__global__ __launch_bounds__(256, 2) void k_rows(CacheAttnArgs a) {
  many_rows<D, F16, LO ? 2 : 1>(a);
}
template <int D, bool F16>
__global__ __launch_bounds__(256, 2) void k_fine_rows(CacheAttnArgs a) {
  many_rows<D, F16, 3>(a);
}

template <int D, int M>
__global__ __launch_bounds__(256) void k_merge(CacheAttnArgs a, int target, int per_group) {
  join_tiles<D, M>(a, target, per_group);
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
