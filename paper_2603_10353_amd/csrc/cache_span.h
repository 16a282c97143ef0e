// Which units of 64 keys a tile of query rows sees with a sliding window and first tokens that stay visible, and sums of units that stay
// numbers of 32 bits.  Plain arithmetic, the same on the host and on the device.
#pragma once
#include <cstdint>

namespace shplb {

constexpr int kUnit = 64;
constexpr int smaller(int x, int y) { return x < y ? x : y; }
constexpr int larger(int x, int y) { return x < y ? y : x; }

// A tile goes through `count` units: those of the first tokens, then those of the windows.  Unit u of the tile is unit u of the head below
// `sinks`, u + skip from there on.
struct Span {
  int sinks, skip, count;
  int low_first, low_last;                     // where the windows of the first and of the last row begin
  constexpr int unit(int u) const { return u < sinks ? u : u + skip; }
  // The last of the tile's units below u1; 0 where there is none: unit(0) is one that the head's table has room for all the same.
  constexpr int last(int u1) const { return larger(smaller(u1, count) - 1, 0); }
};

// Whether a length is one that a head's row of the page table has room for.
constexpr bool length_fits(int len, int room) { return len >= 0 && len <= room; }

// Of rows first_row .. first_row + rows - 1 of n tokens with `group` rows each, the last ones of a head that holds `held` tokens: its length,
// but of one that cannot be 0 (the units are places in the table, and the first one is looked up in any case).
constexpr Span window_span(int window, int n_sink, int first_row, int rows, int n, int group, int held) {
  const int before = held - n + 1, first = first_row / group, last = (smaller(first_row + rows, n * group) - 1) / group;
  Span x{};
  x.low_first = before + first - window;
  x.low_last = before + last - window;
  const int hi = larger(before + last, 0), end = (hi + kUnit - 1) / kUnit, begin = larger(x.low_first, 0) / kUnit;
  x.sinks = (smaller(n_sink, hi) + kUnit - 1) / kUnit;
  x.skip = larger(begin - x.sinks, 0);
  x.count = end - x.skip;
  return x;
}

// Sums of units up to `most`, which is below 2^30, of addends up to it: the smaller of the true sum and `most`, in whatever order they are
// added.
struct UnitSums {
  int most;
  constexpr int operator()(int x, int y) const { return smaller(x + y, most); }
};

}  // namespace shplb
