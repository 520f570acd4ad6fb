// ra_cache_attn.hip -- attention over the 4-bit paged KV cache (gfx950): cache_attn.
#include "ra_cache_attn.h"

namespace ra {

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
  return D == 128 ? attn_d<128, kAll>(b, s) : attn_d<64, kAll>(b, s);
}

}  // namespace ra
