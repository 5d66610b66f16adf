"""Where the adapters' tile kernel reads, on the host: csrc/row_reads.h compiled for the CPU, over widths, tokens, ranks and banks."""
import os
import subprocess

import paper_2502_04416_amd

CSRC = os.path.join(os.path.dirname(paper_2502_04416_amd.__file__), "csrc")


def run(tmp_path, name, body):
    src, exe = tmp_path / (name + ".cpp"), tmp_path / name
    src.write_text('#include <cstdio>\n#include <cstdlib>\n#include <initializer_list>\n#include "row_reads.h"\nusing namespace cmoe;\n' + body)
    subprocess.run(["g++", "-O2", "-std=c++17", "-I" + CSRC, str(src), "-o", str(exe)], check=True)
    r = subprocess.run([str(exe)], capture_output=True, text=True)
    assert r.returncode == 0, r.stdout


def test_rest_of_the_width_is_read_inside_the_buffer(tmp_path):
    """x (a token per row, from the tile's first on) and a (rank rows per adapter): the loads of both halves begin inside the buffer and end
    there; whole rows' offsets are added unsigned, so they are not negative."""
    run(tmp_path, "rest", r'''
static void check(long before, long rows, int d, int row, int part) {
  const bool whole = d % 8 == 0;
  for (int half = 0; half < 2; ++half) {
    const int at = row * d + part * 8;
    const int64_t left = rest_left(rows, d, half), base = before * d + rest_base(d, half), size = (before + rows) * (int64_t)d;
    const int first = near_first(at, left);
    const bool holds = d / 64 * 64 + half * 32 + part * 8 < d;     // values of the row: read where they are, or moved there from the end
    if ((whole && first < 0) || base + first < 0 || base + first + 8 > size || left != size - base || (whole && holds && first != at) ||
        (holds && base + at != row * (int64_t)d + before * d + d / 64 * 64 + half * 32 + part * 8)) {
      printf("%ld rows before, %ld from the base, width %d, row %d, part %d, half %d: %d of %ld\n", before, rows, d, row, part, half, first, (long)left);
      exit(1);
    }
  }
}
int main() {
  for (int d = 8; d <= 1400; ++d)
    for (long rows : {1, 2, 3, 15, 16, 17, 31, 32, 33, 64})
      for (long before : {0, 1, 16, 512})
        for (int row = 0; row < 32 && row < rows; ++row)
          for (int part = 0; part < 4; ++part) check(before, rows, d, row, part);
  for (int d : {2056, 4128, 4136, 11040, 1048552, 1048568})
    for (long rows : {1, 8191, 1048576})
      for (int part = 0; part < 4; ++part) check(0, rows, d, 0, part), check(0, rows, d, rows < 512 ? 0 : 511, part);
  return 0;
}
''')


def test_columns_of_y_are_read_inside_their_buffers(tmp_path):
    """base (and y) and b, 32 columns of y at a time: rows of b past the last column, chunks past the rank, the last adapter of a bank."""
    run(tmp_path, "columns", r'''
static void check(const char* what, bool whole, int64_t start, int64_t size, int at) {
  const int first = near_first(at, size - start);
  if ((whole && first < 0) || start + first < 0 || start + first + 8 > size) {
    printf("%s: %d past %ld of %ld\n", what, first, (long)start, (long)size);
    exit(1);
  }
}
int main() {
  for (int d = 1; d <= 200; ++d)
    for (int rank = 1; rank <= 64; ++rank)
      for (int n : {1, 2, 5}) {
        const int64_t b_size = (int64_t)n * d * rank;
        const bool whole = d % 8 == 0 && rank % 8 == 0;
        for (int o0 = 0; o0 < d; o0 += 32) {
          if (b_size >= 8)
            for (int row = 0; row < 16; ++row)
              for (int part = 0; part < 4; ++part)
                for (int c = 0; c < 2; ++c)
                  for (int e = 0; e < 2; ++e)
                    check("b", whole, ((int64_t)(n - 1) * d + o0) * rank, b_size, ((row >> 2) * 8 + (row & 3)) * rank + part * 8 + e * 4 * rank + c * 32);
          for (int64_t tokens : {1, 2, 16, 33})
            if (tokens * d >= 8)
              for (int64_t t0 = 0; t0 < tokens; t0 += 16)
                for (int row = 0; row < 16 && t0 + row < tokens; ++row)
                  for (int part = 0; part < 4; ++part) check("base", d % 8 == 0, t0 * d + o0, tokens * d, row * d + part * 8);
        }
      }
  return 0;
}
''')


def test_values_read_one_by_one_end_with_their_buffers(tmp_path):
    """The form of widths and buffers below eight values: every value that a tile asks for, rows of b past the last column among them."""
    run(tmp_path, "tiny", r'''
static void check(const char* what, int64_t start, int64_t size, int at, int n, bool whole_row) {
  const int count = tiny_count(at, n, size - start);
  if ((count > 0 && start + at + (count < 8 ? count : 8) > size) || (whole_row && count != n)) {
    printf("%s: %d of %d values, %d past %ld of %ld\n", what, count, n, at, (long)start, (long)size);
    exit(1);
  }
}
int main() {
  for (int d = 1; d <= 70; ++d)
    for (int rank : {1, 2, 3, 7, 8, 33, 64})
      for (int n : {1, 2, 5})
        for (int k = 0; k < n; ++k)
          for (int o0 = 0; o0 < d; o0 += 32)
            for (int row = 0; row < 16; ++row)
              for (int part = 0; part < 4; ++part)
                for (int c = 0; c < 2; ++c)
                  for (int e = 0; e < 2; ++e) {
                    const int column = (row >> 2) * 8 + (row & 3) + e * 4, left = rank - (c * 4 + part) * 8;
                    check("b", ((int64_t)k * d + o0) * rank, (int64_t)n * d * rank, column * rank + part * 8 + c * 32, left, o0 + column < d);
                  }
  for (int d = 1; d <= 70; ++d)
    for (long rows : {1, 2, 16, 33})
      for (int row = 0; row < 16 && row < rows; ++row)
        for (int part = 0; part < 4; ++part) {
          for (int half = 0; half < 2; ++half) {
            const int n = d - d / 64 * 64 - half * 32 - part * 8;
            check("x", rest_base(d, half), rows * d, row * d + part * 8, n, n > 0);
          }
          for (int o0 = 0; o0 < d; o0 += 32) check("base", o0, rows * d, row * d + part * 8, d - o0 - part * 8, d - o0 - part * 8 > 0);
        }
  return 0;
}
''')
