// The index arithmetic that the kernels on a paged cache share (csrc/paged.h), walked on the CPU against plain loops:
// division by a multiplication, the tiles that a place sees, and the shares of the workers with the parts they leave.
#include <cstdio>
#include <cstdlib>
#include <map>
#include <random>
#include <set>
#include <vector>

#include "paged.h"

using namespace dcp;

#define CHECK(x) do { if (!(x)) { std::printf("failed: %s (line %d)\n", #x, __LINE__); std::exit(1); } } while (0)

int main() {
  std::mt19937_64 rng(1);
  auto uni = [&](int64_t lo, int64_t hi) { return lo + (int64_t)(rng() % (uint64_t)(hi - lo + 1)); };

  std::vector<uint32_t> ds = {1, 2, 3, 5, 7, 16, 20, 37, 100, 1 << 20, (1u << 30) - 1, 1u << 30, INT32_MAX};
  for (int k = 0; k < 200; k++) ds.push_back((uint32_t)uni(1, int64_t(1) << uni(1, 31)) & INT32_MAX ? (uint32_t)uni(1, INT32_MAX >> uni(0, 30)) : 9);
  for (uint32_t d : ds) {
    const FastDiv f = fast_div(d);
    for (int k = 0; k < 2000; k++) {
      int64_t n = k < 40 ? (int64_t)d * uni(0, INT32_MAX / d) + uni(-1, 1) : uni(0, INT32_MAX);
      if (n < 0 || n > INT32_MAX) n = k;
      const int32_t q = f.quot((int32_t)n);
      CHECK(q == n / d && f.rem((int32_t)n, q) == n % d);
    }
    CHECK(f.quot(INT32_MAX) == INT32_MAX / (int64_t)d);
  }

  for (int k = 0; k < 20000; k++) {
    const int tile = k & 1 ? 32 : 16, len = (int)uni(0, k % 7 ? 300 : 3000);
    const int window = k % 3 ? (int)uni(1, k % 5 ? 200 : 4000) : 0, sink = (int)uni(0, k % 4 ? 90 : 2000);
    const KeyTiles t(len, window, sink, tile);
    CHECK(t.count >= 1);
    std::set<int> seen, tiles;
    int last = -1;
    for (int x = 0; x < t.count; x++) {
      const int at = t.tile_at(x);
      CHECK(at > last);          // ascending, so no tile twice
      last = at;
      bool any = false;
      for (int j = at * tile; j < (at + 1) * tile; j++)
        if (t.sees(j)) { seen.insert(j); any = true; }
      CHECK(any || len == 0);    // no tile for nothing
    }
    for (int j = 0; j < len; j++) CHECK(seen.count(j) == (window == 0 || len - 1 - j < window || j < sink));
    CHECK(seen.empty() || *seen.rbegin() < len);
  }
  for (int len : {(1 << 30), (1 << 30) - 1, (1 << 30) - 31})
    for (int window : {0, 1, 1 << 20, INT32_MAX})
      for (int sink : {0, 5, INT32_MAX}) {
        const KeyTiles t(len, window, sink, 32);
        CHECK(t.tile_at(t.count - 1) == (len - 1) / 32 && t.count >= 1 && t.tile_at(0) >= 0);
      }

  // every tile belongs to one worker, in order; an item that several share leaves its parts in slots of their own
  for (int k = 0; k < 6000; k++) {
    std::vector<int32_t> items;
    const int n = (int)uni(1, 40), most = 1 << (k % 2 ? 9 : 4);
    for (int i = 0; i < n; i++) items.push_back(k % 5 == 0 ? (int32_t)uni(1, 1 << 25) : (int32_t)uni(1, 50));
    int64_t total = 0;
    for (int32_t x : items) total += x;
    CHECK(total <= INT32_MAX);
    const Shares<9> s9((int32_t)total);
    const Shares<4> s4((int32_t)total);
    auto start = [&](int w) { return k % 2 ? s9.start(w) : s4.start(w); };
    auto worker_of = [&](int t) { return k % 2 ? s9.worker_of(t) : s4.worker_of(t); };
    const int workers = k % 2 ? s9.workers : s4.workers;
    CHECK(workers >= 1 && workers <= most && start(0) == 0 && start(workers) == total);
    std::map<int, int> slots;   // slot -> item
    int32_t begin = 0;
    for (int i = 0; i < n; begin += items[i], i++) {
      const int first = worker_of(begin), last = worker_of(begin + items[i] - 1);
      CHECK(first >= 0 && first <= last && last < workers);
      CHECK(start(first) <= begin && begin < start(first + 1));
      CHECK(start(last) < begin + items[i] && begin + items[i] <= start(last + 1));
      if (first == last) continue;
      for (int w = first; w <= last; w++) {
        CHECK(start(w) < start(w + 1));   // nobody between them is without work
        const int slot = w == first ? 2 * w + 1 : 2 * w;
        CHECK(slot < 2 * most && slots.emplace(slot, i).second);
      }
    }
    for (int w = 0; w < workers; w++) CHECK(start(w + 1) - start(w) >= 1 && start(w + 1) - start(w) <= total / workers + 1);
  }
  for (int32_t total : {INT32_MAX, INT32_MAX - 511, 511, 512, 513, 1}) {
    const Shares<9> s(total);
    CHECK(s.start(s.workers) == total && s.worker_of(total - 1) == s.workers - 1 && s.worker_of(0) == 0);
  }
  std::printf("host-paged ok\n");
}
