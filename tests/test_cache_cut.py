"""How long the parts of shared attention are, on the host: at the limits of a call, where 32-bit numbers of pieces would
wrap, and for ordinary ones.  The search is that of the launch, step by step, over the functions that it uses."""
import ctypes
import os
import random
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2607_02584_amd", "csrc")

DRIVER = r"""
#include "ra_cache_cut.h"
using namespace ra;
extern "C" float finest(int n, const int* tiles, const int* blocks, int least) {
  float s = 0;
  for (int i = 0; i < n; ++i) s += cut_finest(tiles[i], blocks[i], least);
  return s;
}
extern "C" unsigned closed(int n, const int* tiles, const int* blocks, int places, int least) {
  float W = 0;
  for (int i = 0; i < n; ++i) W += static_cast<float>(tiles[i]) * static_cast<float>(blocks[i]);
  return cut_closed(W, static_cast<float>(places), least);
}
// one kind of pieces: the shortest parts, or the cheapest of one and two rounds
extern "C" unsigned length(int n, const int* tiles, const int* blocks, int all, int fixed, int least) {
  if (finest(n, tiles, blocks, least) <= static_cast<float>(all)) return least;
  float W = 0;
  int count = 0, longest = 0;
  for (int i = 0; i < n; ++i) {
    W += static_cast<float>(tiles[i]) * static_cast<float>(blocks[i]);
    count += tiles[i];
    longest = blocks[i] > longest ? blocks[i] : longest;
  }
  unsigned best = 0;
  unsigned long long cost = 0;
  for (int r = 1; r <= 2; ++r) {
    const float places = static_cast<float>(r * all), f = static_cast<float>(fixed);
    CutRange x = cut_range(W, count, longest, places, f, least);
    for (int step = 0; step < 3; ++step) {
      int good = 8;
      const unsigned long long d = x.hi - x.lo;
      for (int z = 7; z >= 0; --z) {
        const float c = static_cast<float>(x.lo + static_cast<unsigned>(d * z / 8));
        float sum = 0;
        for (int i = 0; i < n; ++i)
          if (tiles[i] > 0) sum += static_cast<float>(tiles[i]) * cut_weight(static_cast<float>(blocks[i]), c, 1.0f / c, f, 1.0f / (c + f));
        if (sum <= places) good = z;
      }
      const unsigned from = x.lo;
      if (good < 8) x.hi = from + static_cast<unsigned>(d * good / 8);
      if (good > 0) x.lo = from + static_cast<unsigned>(d * (good - 1) / 8);
      if (x.hi <= x.lo + 1 + x.lo / 32) break;
    }
    const unsigned long long c = r * (static_cast<unsigned long long>(x.hi) + fixed);
    if (!best || c < cost) best = x.hi, cost = c;
  }
  return best;
}
extern "C" int parts(int blocks, unsigned c) { return cut_parts(blocks, c); }
"""

FEW, MANY = (10, 4), (6, 4)     # a piece's fixed cost in blocks, the shortest part


@pytest.fixture(scope="module")
def cut(tmp_path_factory):
    d = tmp_path_factory.mktemp("cut")
    src, so = d / "cut.cpp", d / "cut.so"
    src.write_text(DRIVER)
    subprocess.run(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", "-I", CSRC, str(src), "-o", str(so)], check=True)
    lib = ctypes.CDLL(str(so))
    lib.finest.restype = ctypes.c_float
    lib.closed.restype = lib.length.restype = ctypes.c_uint
    lib.parts.argtypes = [ctypes.c_int, ctypes.c_uint]

    class Cut:
        def args(self, tiles, blocks):
            n = len(tiles)
            return n, (ctypes.c_int * n)(*tiles), (ctypes.c_int * n)(*blocks)

        def finest(self, tiles, blocks, least):
            return lib.finest(*self.args(tiles, blocks), least)

        def pieces(self, tiles, blocks, c):
            return sum(t * lib.parts(b, c) for t, b in zip(tiles, blocks))

        def length(self, tiles, blocks, places, kind):
            return lib.length(*self.args(tiles, blocks), places, *kind)

        def closed(self, tiles, blocks, places, least):
            return lib.closed(*self.args(tiles, blocks), places, least)
    return Cut()


def _check(cut, tiles, blocks, places, kind, rows_of_tile, bound_rows):
    exact = sum(t * -(-b // 4) for t, b in zip(tiles, blocks))
    c = cut.length(tiles, blocks, places, kind)
    got = cut.pieces(tiles, blocks, c)
    # what the workspace and the piece list are laid out for: two rounds of places beside the tiles themselves
    assert got <= sum(tiles) + 2 * places, c
    assert sum(t * rows_of_tile * cut_p for t, cut_p in zip(tiles, (-(-b // c) if b else 1 for b in blocks))) <= bound_rows < 2 ** 31
    assert (c == kind[1]) or exact > places
    return c, exact


# one request of T queries, or many, at the limits of T and T * Hq: rows per KV head, tokens
@pytest.mark.parametrize("rows,tokens", [(1 << 26, 1 << 21), (1 << 24, 1 << 22), (1 << 25, 1 << 21), (1 << 25, 1 << 30), (1 << 26, 1 << 30),
                                         (1 << 20, 1 << 30)])
@pytest.mark.parametrize("places", [1, 64, 512])
def test_pieces_of_enormous_calls_do_not_wrap(cut, rows, tokens, places):
    """A prefix and own keys of as many: the shortest parts are not taken for few."""
    tiles, blocks = [rows // 128] * 2, [tokens // 64, tokens // 64]
    c, exact = _check(cut, tiles, blocks, places, MANY, 128, 2 * rows + 128 * 2 * places)
    assert exact >= 2 ** 31 and c > 4 and cut.finest(tiles, blocks, 4) > 512


def test_32_bits_would_have_wrapped_here(cut):
    """2^19 tiles of 2^13 parts of four blocks: 2^32, which is 0 in 32 bits and would fit any place."""
    tiles, blocks = [1 << 19], [1 << 15]
    assert tiles[0] * ((blocks[0] + 3) // 4) % 2 ** 32 == 0
    assert cut.finest(tiles, blocks, 4) == 2.0 ** 32
    tiles, blocks = [1 << 18], [1 << 15]       # T = 2^21, 16 heads on one KV head: negative in 32 bits
    assert tiles[0] * (blocks[0] // 4) == 2 ** 31 and cut.finest(tiles, blocks, 4) == 2.0 ** 31


@pytest.mark.parametrize("n", [4096, 300])
@pytest.mark.parametrize("places", [1, 500])
def test_many_long_requests_of_few_rows(cut, n, places):
    tiles, blocks = [1] * n, [1 << 24] * n
    c, exact = _check(cut, tiles, blocks, places, FEW, 16, 16 * (n + 2 * places))
    assert exact > 2 ** 30


@pytest.mark.parametrize("n", [5000, 131072])
def test_closed_lengths_of_more_requests(cut, n):
    rng = random.Random(n)
    tiles = [rng.choice([0, 1, 1, 1 << 9]) for _ in range(n)]
    for most in (5, 1 << 24):
        blocks = [rng.randint(0, most) for _ in range(n)]
        for places in (2, 1024):
            c = cut.closed(tiles, blocks, places, 4)
            assert c >= 4 and cut.pieces(tiles, blocks, c) <= sum(tiles) + places


def test_ordinary_calls(cut):
    """Short ones in the shortest parts, others in one or two rounds of the places (or a piece for each tile)."""
    rng = random.Random(1)
    shortest = 0
    for k in range(400):
        n, kind, tile = rng.randint(1, 250), *rng.choice([(FEW, 16), (MANY, 128)])
        tiles = [1 if kind == FEW else rng.randint(1, 40) for _ in range(n)]
        blocks = [rng.randint(0, rng.choice([3, 60, 1000])) for _ in range(n)]
        places = rng.choice([12, 64, 512])
        c, exact = _check(cut, tiles, blocks, places, kind, tile, tile * (sum(tiles) + 2 * places))
        assert cut.finest(tiles, blocks, 4) == exact
        shortest += c == 4
    assert 0 < shortest < 400
