// Where the rows of a tile lie in memory: row x of a tile is token x / G, head x % G from the tile's first token on.  Plain C++, for host and device.
#pragma once

namespace prism {

// Elements from the tile's first row to row x
constexpr long long row_offset(int x, int G, long long token, long long head) { return (long long)(x / G) * token + (long long)(x - x / G * G) * head; }

// A thread's chunks lie in rows r, r + apart, ... (r < apart, four of them at most).  From row r to row r + u apart it is (u & 1) one + (u >> 1) two elements, whatever r.
// apart and G are powers of two: either G divides apart and every step is whole tokens, or apart divides G and r stays inside its part of the group, so that the steps of
// apart and 2 apart rows are those from row 0.
struct RowSteps {
  long long one, two;
  constexpr long long to(int u) const { return (u & 1) * one + (u >> 1) * two; }
};
constexpr RowSteps row_steps(int apart, int G, long long token, long long head) {
  return {row_offset(apart, G, token, head), row_offset(2 * apart, G, token, head)};
}

}  // namespace prism
