// The sums of what places ask for (csrc/paged.h), up to the most pages that a cache may have, against 64 bits.
#include <cstdio>
#include <cstdlib>
#include <random>
#include <vector>

#include "paged.h"

using namespace dcp;

#define CHECK(x) do { if (!(x)) { std::printf("failed: %s (line %d)\n", #x, __LINE__); std::exit(1); } } while (0)

int main() {
  const int32_t most = 1 << 30;   // pages of a cache
  std::mt19937_64 rng(1);
  for (int32_t cap : {1, 2, 100, most - 1, most, most + 1}) {
    for (int32_t x : {0, 1, cap / 2, cap - 1, cap})
      for (int32_t y : {0, 1, cap / 2, cap - 1, cap}) CHECK(add_capped(x, y, cap) == ((int64_t)x + y < cap ? x + y : cap));
    for (int k = 0; k < 300; k++) {   // running sums of needs, from the left and in pairs
      std::vector<int32_t> need(1 + rng() % 40);
      for (int32_t& x : need) x = rng() % 3 ? (int32_t)(rng() % ((uint64_t)cap + 1)) : (int32_t)(rng() % 3) * (cap > 2);
      int64_t sum = 0;
      int32_t left = 0;
      for (int32_t x : need) {
        sum += x;
        left = add_capped(left, x, cap);
        CHECK(left == (sum < cap ? sum : cap));
      }
      while (need.size() > 1) {
        for (size_t i = 0; 2 * i < need.size(); i++) need[i] = 2 * i + 1 < need.size() ? add_capped(need[2 * i], need[2 * i + 1], cap) : need[2 * i];
        need.resize((need.size() + 1) / 2);
      }
      CHECK(need[0] == left);
    }
  }
  std::printf("host-paged sums ok\n");
}
