// Where loads of eight values begin: plain arithmetic, so that the host can go through it too.
#pragma once
#include <stdint.h>

namespace cmoe {

// A load is `at` values past its base, from which on the buffer has `left`: it begins here instead where it would pass the buffer's end.
// Not below zero if left is 8 at least; else eight values before the end, which the buffer has to have in front of the base.
constexpr int near_first(int at, int64_t left) {
  const int last = (int)(left - 8 < 0x40000000 ? left - 8 : 0x40000000);
  return at < last ? at : last;
}

// How many of n values `at` past a base are read one by one: none past the buffer's end (rows of a tile may lie behind it).
constexpr int tiny_count(int at, int n, int64_t left) { return n < left - at ? n : (int)(left - at); }

// What a row of d values has behind its last 64 is read in two halves of 32.  The half's base, and what a buffer of `rows` such rows has
// left from there: a half that begins past the row's end (its values are zeros) reads the row's last chunk, since behind the buffer's
// last row there is nothing.  With d a multiple of eight, at least eight values are left.
constexpr int rest_base(int d, int half) {
  const int at = (d & ~63) + half * 32, last = (d - 1) & ~7;
  return at < last ? at : last;
}
constexpr int64_t rest_left(int64_t rows, int d, int half) { return rows * d - rest_base(d, half); }

}  // namespace cmoe
