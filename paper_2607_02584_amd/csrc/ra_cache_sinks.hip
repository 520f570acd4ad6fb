// ra_cache_sinks.hip -- attention over the 4-bit paged KV cache under a window
// beside which the first tokens stay visible (gfx950): cache_attn_sinks.
//
// Row i sees the keys j <= p_i with j > p_i - window or j < sinks.  The blocks
// of 64 keys of the first tokens and those of a tile's window are numbered
// without the gap between them (Span), and the kernels of cache_attn go through
// the numbers; rows mask a tile's first block behind `sinks` and its
// window's edges.
//
// Where a call can have requests of few and of many rows, both go in one launch,
// those of many first, and what is split is joined in one launch behind it: of
// four launches, two of which have nothing to do in a small call, two are left
// (30 requests of one query beside a prompt of 300 tokens 80 -> 59 us).
#include "ra_cache_attn.h"

namespace ra {
namespace {

// The partial rows of requests of few rows lie behind those of many.
__device__ __forceinline__ void few_parts(CacheAttnArgs& a) {
  a.part_o = a.few_o;
  a.part_ml = a.few_ml;
}

// `rows`: workgroups of the pieces of many rows
template <int D, bool F16, int TERMS>
__global__ __launch_bounds__(256, 2) void k_both(CacheAttnArgs a, int rows) {
  constexpr bool FINE = TERMS == 3;
  __shared__ union {
    FewLds<D, 2, true> few;
    RowsLds<D, kSinks> rows;
  } lds;
  const bool many = static_cast<int>(blockIdx.x) < rows;
  const int x = many ? blockIdx.x : blockIdx.x - rows, x0 = x / a.g.Hkv, h = x - x0 * a.g.Hkv;
  if (many) return rows_piece<D, F16, TERMS, kSinks>(a, lds.rows, x0, h);
  few_parts(a);
  few_rows<D, 2, 2, FINE, kSinks>(a, lds.few, x0, h);
}

// Tiles of many rows first: {tiles, KV heads, groups of rows} of either kind, the tiles fastest.
struct Joins {
  int tiles[2], groups[2], per_group[2];   // of many and of few rows
};
template <int D>
__global__ __launch_bounds__(256) void k_join(CacheAttnArgs a, Joins j) {
  const int many = j.tiles[0] * a.g.Hkv * j.groups[0], k = static_cast<int>(blockIdx.x) < many ? 0 : 1;
  const int x = blockIdx.x - (k ? many : 0), y = x / j.tiles[k], x0 = x - y * j.tiles[k], z = y / a.g.Hkv, h = y - z * a.g.Hkv;
  if (k == 0) return join_tiles<D, kRowTile, kSinks>(a, a.target_rows, j.per_group[0], x0, h, z);
  few_parts(a);
  join_tiles<D, kFewRows, kSinks>(a, a.target, j.per_group[1], x0, h, z);
}

template <int D, bool F16>
hipError_t both(const CacheAttnArgs& a, hipStream_t s) {
  const Grid g[2] = {grid_of(a, kRowTile, a.target_rows), few_grid_of(a)};
  const int64_t rows = (g[0].tiles + a.target_rows) * a.g.Hkv, all = rows + (g[1].tiles + a.target) * a.g.Hkv;
  const dim3 grid(static_cast<unsigned>(all));
  const int terms = terms_of(a);
  if (terms == 3) k_both<D, F16, 3><<<grid, dim3(256), 0, s>>>(a, static_cast<int>(rows));
  else if (terms == 2) k_both<D, F16, 2><<<grid, dim3(256), 0, s>>>(a, static_cast<int>(rows));
  else k_both<D, F16, 1><<<grid, dim3(256), 0, s>>>(a, static_cast<int>(rows));
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const int64_t most = static_cast<int64_t>(a.max_q) * a.G;
  Joins j;
  const int M[2] = {kRowTile, kFewRows};
  unsigned joins = 0;
  for (int k = 0; k < 2; ++k) {
    const int n = static_cast<int>(most < M[k] ? most : M[k]);
    j.tiles[k] = static_cast<int>(g[k].merges);
    j.per_group[k] = k ? merged_rows<kFewRows>(a, g[k], most) : merged_rows<kRowTile>(a, g[k], most);
    j.groups[k] = (n + j.per_group[k] - 1) / j.per_group[k];
    joins += static_cast<unsigned>(j.tiles[k]) * a.g.Hkv * j.groups[k];
  }
  k_join<D><<<dim3(joins), dim3(256), 0, s>>>(a, j);
  return hipGetLastError();
}

template <int D>
hipError_t sinks_d(const CacheAttnArgs& a, hipStream_t s) {
  // both kinds can be there, and their workgroups fit one launch (of less than 2^32 work-items)
  const int64_t pieces = grid_of(a, kRowTile, a.target_rows).tiles + a.R + a.target_rows + a.target;
  if (static_cast<int64_t>(a.max_q) * a.G > kFewRows && a.G <= kFewRows && pieces * a.g.Hkv < 1 << 24)
    return a.is_fp16 ? both<D, true>(a, s) : both<D, false>(a, s);
  return attn_d<D, kSinks>(a, s);
}

}  // namespace

size_t cache_sinks_bytes(int D, int Hkv, int G, int max_q, size_t* ml, size_t* few_o, size_t* few_ml) {
  const size_t bytes = cache_attn_partial_bytes(D, Hkv, G, max_q, ml);
  *few_o = 0;
  *few_ml = *ml;
  if (static_cast<int64_t>(max_q) * G <= kFewRows || G > kFewRows) return bytes;
  const size_t rows = static_cast<size_t>(2) * target_of(kPieces, Hkv) * Hkv * kFewRows;
  *few_o = (bytes + 255) / 256 * 256;
  *few_ml = *few_o + rows * D * sizeof(float);
  return *few_ml + rows * sizeof(float2);
}

hipError_t launch_cache_attn_sinks(const CacheAttnArgs& a, int D, hipStream_t s) {
  CacheAttnArgs b = a;
  b.target = target_of(kPieces, a.g.Hkv);
  b.target_rows = target_of(kRowPieces, a.g.Hkv);
  return D == 128 ? sinks_d<128>(b, s) : sinks_d<64>(b, s);
}

}  // namespace ra
