// Whether two strided tensors share bytes: for the calls' checks of their arguments, on the
// host alone.
#pragma once

#include <stdint.h>

namespace ltd {

typedef __int128 Wide;

// The bytes [0, run) past at + r * row + h * head of every row r < rows and head h < heads
// (rows, heads and run at least 1; strides of either sign).
struct Runs {
  uint64_t at;
  int64_t rows;
  Wide row;
  int64_t heads;
  Wide head;
  int64_t run;
};

// Exact where both have the same strides (a stride that one of them has no use for counts as
// the other's) and where the rows' extents are apart within a common row stride; otherwise
// ranges of bytes that meet count as shared.
inline bool runs_meet(const Runs& x, const Runs& y) {
  const auto low = [](const Runs& t) {
    const Wide r = (t.rows - 1) * t.row, h = (t.heads - 1) * t.head;
    return (r < 0 ? r : 0) + (h < 0 ? h : 0);
  };
  const auto high = [](const Runs& t) {
    const Wide r = (t.rows - 1) * t.row, h = (t.heads - 1) * t.head;
    return (r > 0 ? r : 0) + (h > 0 ? h : 0) + t.run;
  };
  const Wide off = static_cast<Wide>(y.at) - static_cast<Wide>(x.at);
  if (off + low(y) >= high(x) || off + high(y) <= low(x)) return false;
  const bool row_same = x.row == y.row || x.rows == 1 || y.rows == 1;
  const bool head_same = x.head == y.head || x.heads == 1 || y.heads == 1;
  Wide row = x.rows == 1 ? y.row : x.row;
  if (row_same && head_same) {
    // y's start less x's is off + u row + v head, and they meet where that lies in
    // (-y.run, x.run): for each v the first u past the lower end tells.
    const Wide head = x.heads == 1 ? y.head : x.head;
    int64_t u0 = 1 - x.rows, u1 = y.rows - 1;
    if (row < 0) {
      row = -row;
      const int64_t t = u0;
      u0 = -u1;
      u1 = -t;
    }
    for (int64_t v = 1 - x.heads; v < y.heads; ++v) {
      const Wide w = off + v * head, least = 1 - y.run - w;
      Wide u = u0;
      if (row > 0 && u * row < least) u = least >= 0 ? (least + row - 1) / row : -(-least / row);
      if (u <= u1 && w + u * row > -y.run && w + u * row < x.run) return true;
    }
    return false;
  }
  if (row_same && row > 0 && x.head >= 0 && y.head >= 0) {
    const Wide wide_x = (x.heads - 1) * x.head + x.run, wide_y = (y.heads - 1) * y.head + y.run;
    const Wide from = (off % row + row) % row;
    return !(from >= wide_x && from + wide_y <= row);
  }
  return true;
}

}  // namespace ltd
