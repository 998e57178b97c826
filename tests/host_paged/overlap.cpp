// Whether two tensors of rows share a byte (csrc/paged.h), against a set of bytes.
#include <cstdio>
#include <cstdlib>
#include <random>
#include <set>

#include "paged.h"

using namespace dcp;

#define CHECK(x) do { if (!(x)) { std::printf("failed: %s (line %d)\n", #x, __LINE__); std::exit(1); } } while (0)

static char* const kBase = (char*)0x7000000;

static bool overlap(int64_t px, int64_t py, int64_t st, int64_t sh, int64_t st2, int64_t sh2, int n, int heads, int64_t row) {
  return rows_overlap(Rows{kBase + px, st, sh}, Rows{kBase + py, st2, sh2}, n, heads, row);
}

int main() {
  std::mt19937_64 rng(1);
  auto uni = [&](int lo, int hi) { return lo + (int)(rng() % (uint64_t)(hi - lo + 1)); };
  int yes = 0, no = 0, between = 0;
  for (int k = 0; k < 20000; k++) {
    const int n = uni(1, 6), heads = uni(1, 6), row = uni(1, 4);
    int st = row + uni(0, 30), sh = row + uni(0, k % 2 ? 30 : 4);
    if (k % 3 == 0) st = heads * sh * uni(1, 3);   // the layouts that are met: heads inside tokens
    if (k % 3 == 1) sh = n * st * uni(1, 3);       // tokens inside heads
    const int px = uni(0, 150), py = uni(0, 150);
    std::set<int> bytes;
    for (int i = 0; i < n; i++)
      for (int h = 0; h < heads; h++)
        for (int c = 0; c < row; c++) bytes.insert(px + i * st + h * sh + c);
    bool shared = false;
    for (int i = 0; i < n; i++)
      for (int h = 0; h < heads; h++)
        for (int c = 0; c < row; c++) shared |= bytes.count(py + i * st + h * sh + c) > 0;
    CHECK(overlap(px, py, st, sh, st, sh, n, heads, row) == shared);
    CHECK(overlap(py, px, st, sh, st, sh, n, heads, row) == shared);
    shared ? yes++ : no++;
    const bool hulls = px <= py + (n - 1) * st + (heads - 1) * sh + row - 1 && py <= px + (n - 1) * st + (heads - 1) * sh + row - 1;
    between += hulls && !shared;
    // other strides are told apart by their extents alone; a dimension of one has none
    CHECK(overlap(px, py, st, sh, st + 1, sh, 1, heads, row) == overlap(px, py, st, sh, st, sh, 1, heads, row));
    CHECK(overlap(px, py, st, sh, st, sh + 1, n, 1, row) == overlap(px, py, st, sh, st, sh, n, 1, row));
    if (n > 1) CHECK(overlap(px, py, st, sh, st + 1, sh, n, heads, row) == (px < py + (n - 1) * (st + 1) + (heads - 1) * sh + row && py < px + (n - 1) * st + (heads - 1) * sh + row));
  }
  CHECK(yes > 1000 && no > 1000 && between > 500);
  // the most places and heads, side by side and one row too far; strides whose products leave 64 bits
  CHECK(!overlap(0, 65536 * 64, 2 * 65536 * 64, 64, 2 * 65536 * 64, 64, 16384, 65536, 64));
  CHECK(overlap(0, 65536 * 64 - 16, 2 * 65536 * 64, 64, 2 * 65536 * 64, 64, 16384, 65536, 64));
  CHECK(!overlap(0, 64, int64_t(1) << 61, 64, int64_t(1) << 61, 64, 16384, 1, 64));
  CHECK(overlap(0, 64, int64_t(1) << 61, int64_t(1) << 61, int64_t(1) << 60, 64, 16384, INT32_MAX, 64));
  std::printf("host-paged overlap ok\n");
}
