// ra_cache_sinks.hip -- attention over the 4-bit paged KV cache under a window
// beside which the first tokens stay visible (gfx950): cache_attn_sinks.
//
// Row i sees the keys j <= p_i with j > p_i - window or j < sinks.  The blocks
// of 64 keys of the first tokens and those of a tile's window are numbered
// without the gap between them (Span), and the kernels of cache_attn go through
// the numbers; rows mask a tile's first block behind `sinks` and its
// window's edges.
#include "ra_cache_attn.h"

namespace ra {

hipError_t launch_cache_attn_sinks(const CacheAttnArgs& a, int D, hipStream_t s) {
  CacheAttnArgs b = a;
  b.target = target_of(kPieces, a.g.Hkv);
  b.target_rows = target_of(kRowPieces, a.g.Hkv);
  return D == 128 ? attn_d<128, kSinks>(b, s) : attn_d<64, kSinks>(b, s);
}

}  // namespace ra
