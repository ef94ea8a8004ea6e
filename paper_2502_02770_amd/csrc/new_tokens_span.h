// Which pages the rows of a sequence's newest tokens see, and how many tiles of them a list has: host and device.
#pragma once
#ifdef __HIPCC__
#include "tw_common.h"
#define TW_BOTH __host__ __device__ __forceinline__
#else                                            // (with TW_PAGE)
#include <algorithm>
#define TW_BOTH inline
using std::max;
using std::min;
#endif

namespace {

enum { MODE_TREE = 0, MODE_WINDOW = 1 };

// The pages that rows of tokens at positions p_lo .. p_hi see: `sink` pages from the start, then those from `first` on; four of
// this list to a tile, so that a few sinks and a window that begins inside 64 tokens cost no tile of their own: five prompts of 882
// tokens, a window of 51 and one sink 35.1 us with tiles at multiples of 64, 32.3 so.  Where few tiles are saved, working out the
// places costs more than that: one token, a window of 1024 and 4 sinks 10.5 and 10.8 us.
template <int TILE_PAGES>
struct Span {
  int sink, first, pages, tiles;
  int both, behind, shift;                       // the tile with pages of both parts, the first one of the second; positions between the parts
  TW_BOTH int page(int v) const { return v < sink ? v : first + (v - sink); }
  TW_BOTH int start(int u) const { return u * TILE_PAGES * TW_PAGE + (u >= behind ? shift : 0); }   // position of tile u's first page
};
template <int MODE, class A>
TW_BOTH Span<A::TILE_PAGES> span_of(const A& a, int len, int p_lo, int p_hi) {
  constexpr int TP = A::TILE_PAGES;
  Span<TP> s;
  const int end = MODE == MODE_TREE ? len : min(len, p_hi + 1);
  if (end <= 0) { s.sink = s.first = s.pages = s.tiles = s.behind = s.shift = 0; s.both = -1; return s; }
  s.first = MODE == MODE_TREE ? 0 : max(0, p_lo - a.window + 1) / TW_PAGE;
  s.sink = MODE == MODE_TREE ? 0 : min((int)(((unsigned)a.sinks + TW_PAGE - 1) / TW_PAGE), s.first);
  s.pages = s.sink + (end - 1) / TW_PAGE - s.first + 1;
  s.tiles = (s.pages + TP - 1) / TP;
  s.behind = (s.sink + TP - 1) / TP;
  s.both = s.sink & (TP - 1) && s.sink < s.first ? s.sink / TP : -1;
  s.shift = (s.first - s.sink) * TW_PAGE;
  return s;
}

// Pages at least as many as any of a sequence's lists has: n of its len tokens are new, `block` of them to a row block.  Under a window a block
// may lie differently against the pages than the last `block` tokens and see one more than they do.  So those and the 15 tokens before them
// are counted: of them, a block that lies among them sees a part; one that begins earlier has no more sinks, and its block + window - 1
// positions touch no more pages than 15 positions more do, wherever these begin.
template <class A>
TW_BOTH Span<A::TILE_PAGES> longest_span(const A& a, int len, int n, int block) {
  return span_of<MODE_WINDOW>(a, len, len - min(n, block + TW_PAGE - 1), len - 1);
}
// Its tiles at most, however long the sequence is.
template <class A>
TW_BOTH int window_tiles(const A& a, int block) {
  const long long pages = ((long long)a.sinks + TW_PAGE - 1) / TW_PAGE + (block + a.window + 2 * TW_PAGE - 4) / TW_PAGE + 1;
  return (int)((pages + A::TILE_PAGES - 1) / A::TILE_PAGES);
}

}  // namespace
