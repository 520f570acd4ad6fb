// ra_cache_cut.h -- how long the parts are that shared attention cuts its keys
// into (plain C++ on sizes, so it is also checked without a GPU).
//
// Numbers of pieces are binary32 wherever they are summed before a length has
// been chosen: in parts of a few blocks a call within the limits can have 2^41 of
// them, which 32-bit integers would wrap, and only numbers near the few hundred
// places that the card has, exact in binary32, decide.  Once a length has been
// chosen the pieces are the call's tiles and a few rounds of places.
#pragma once

namespace ra {

// Parts of `c` blocks that a tile of `blocks` blocks has.
constexpr int cut_parts(int blocks, unsigned c) { return blocks ? static_cast<int>((static_cast<unsigned>(blocks) + c - 1) / c) : 1; }

// Pieces in parts of `least` blocks.
constexpr float cut_finest(int tiles, int blocks, int least) {
  return static_cast<float>(tiles) * static_cast<float>((blocks + least - 1) / least);
}

// A tile of b blocks in places, with parts of c: a place for each part longer than half of c; small ones fill what others leave.
constexpr float cut_weight(float b, float c, float inv_c, float fixed, float inv_all) {
  return b > 0.5f * c ? __builtin_ceilf(b * inv_c) : (b + fixed) * inv_all;
}

constexpr unsigned cut_blocks(float x) { return x < 0x1p26f ? static_cast<unsigned>(x) : 1u << 26; }   // a request has 2^24 at most
constexpr unsigned cut_at_least(unsigned c, int least) { return c < static_cast<unsigned>(least) ? static_cast<unsigned>(least) : c; }

// Where the least length that fits `places` is looked for: W blocks in all, `count` tiles, the longest of them.  (At `hi`
// every tile is a small piece, or the tiles' last parts fill what is left of the places.)
struct CutRange {
  unsigned lo, hi;
};
constexpr CutRange cut_range(float W, int count, int longest, float places, float fixed, int least) {
  const unsigned one = 2 * static_cast<unsigned>(longest) + 2, all = cut_blocks((W + fixed * static_cast<float>(count)) / places) + 2;
  unsigned hi = one > all ? one : all;
  const float left = places - static_cast<float>(count);
  if (left >= 1.0f) {
    const unsigned even = cut_blocks(W / left) + 1;
    hi = even < hi ? even : hi;
  }
  return {cut_at_least(cut_blocks(W / places), least), cut_at_least(hi, least)};
}

// Without a search: at most `places` parts beside a tile's first.
constexpr unsigned cut_closed(float W, float places, int least) { return cut_at_least(cut_blocks(W / places) + 1, least); }

}  // namespace ra
