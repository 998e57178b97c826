// dcp_cache_append into a cache in 8 bits whose places begin below row 0 of the new tokens, or end behind them, on the CPU in a build with AddressSanitizer and
// UndefinedBehaviorSanitizer: the host's code against a host walk with the index arithmetic of csrc/cache8.hip and csrc/cache_tokens.h, in buffers of exactly the documented
// sizes.  The walk counts what it writes: every token that is there once, the earlier ones of its block with it, and nothing else.
#include <algorithm>
#include <cstdint>
#include <cstdio>
#include <cstdlib>
#include <random>
#include <vector>

#include "cache_internal.h"

namespace dcp {

static int g_bad = 0;
static long g_below = 0, g_older = 0;
#define LOOK(cond) do { if (!(cond)) { std::printf("append8_begins.cpp:%d: %s\n", __LINE__, #cond); g_bad++; } } while (0)

// fake_cache.cpp and fake_cache8.cpp are built with their own under other names.
void launch_append(int32_t each, uint32_t grid, const KCache& c, int32_t layer, const int32_t* seqs, const int32_t* cu, int32_t n, const int32_t* status,
                   const NewTokens& x, hipStream_t) {
  const int d = 16 << c.log_head_chunks;
  LOOK((int64_t)grid * each >= x.n && (int64_t)(grid - 1) * each < x.n);
  for (int64_t t = 0; t < (int64_t)grid * each; t++) {
    if (t >= x.n || t < cu[0] || t >= cu[n]) continue;
    int lo = 0, hi = n - 1;
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if (cu[mid] <= t) lo = mid;
      else hi = mid - 1;
    }
    const int32_t first = cu[lo], behind = (int32_t)(cu[lo + 1] - t), s = seqs[lo];
    if (!c.is_seq(s) || (status && status[lo] != DCP_PLACE_OK)) continue;
    const int32_t pos = c.length(s) - behind;
    if (pos < 0) continue;
    const int32_t q = c.page.quot(pos), page = c.row(s)[q], slot = c.page.rem(pos, q);
    if (!c.is_page(page)) continue;
    const int32_t older = c.block.rem(slot, c.block.quot(slot));
    if (older != 0 && t != std::max(first, 0)) continue;
    const int32_t rows = (int32_t)std::min<int64_t>(std::min(behind, (int32_t)c.block.d - older), x.n - t);
    LOOK(rows >= 1 && slot - older >= 0 && slot + rows <= (int32_t)c.page.d);
    g_below += first < 0 && older != 0;
    g_older += older != 0;
    for (int h = 0; h < c.hkv; h++) {
      for (int y = -older; y < rows; y++)
        for (int64_t at : {(int64_t)0, (int64_t)d - 1}) {
          volatile char from = y < 0 ? 0 : x.k[(t + y) * x.k_st + h * x.k_sh + at * c.io_bytes];
          (void)from;
          c.k[layer * c.k_sl + page * c.k_sp + (slot + y) * c.k_st + h * c.k_sh + at] += y < 0 ? 16 : 1;
        }
      c.k_scale[layer * c.layer_scales() + c.scale_at(page, slot) + h]++;
    }
  }
}

}  // namespace dcp
using namespace dcp;

int main() {
  std::mt19937_64 r(9);
  auto rnd = [&](int lo, int hi) { return lo + (int)(r() % (uint64_t)(hi - lo + 1)); };
  for (int life = 0; life < 300; life++) {
    dcp_cache_t c{};
    c.n_layers = 1; c.hkv = rnd(1, 3); c.d = 32 << rnd(0, 2); c.dtype = DCP_E4M3; c.io_dtype = rnd(0, 1); c.scale_block = rnd(1, 20);
    c.page_size = c.scale_block * rnd(1, 4); c.n_seqs = rnd(1, 5); c.max_pages = rnd(1, 4); c.n_pages = c.n_seqs * c.max_pages;
    const int64_t token = (int64_t)c.hkv * c.d, page = c.page_size * token, scales = (int64_t)c.n_pages * (c.page_size / c.scale_block) * c.hkv;
    char *codes, *x;   // with nothing behind them; the walk looks at K alone
    if (posix_memalign((void**)&codes, 256, c.n_pages * page)) std::abort();
    std::fill(codes, codes + c.n_pages * page, 0);
    std::vector<uint8_t> ks(scales, 0), vs(scales, 0);
    c.k = codes; c.v = codes; c.k_scale = ks.data(); c.v_scale = vs.data();
    c.k_stride_l = c.v_stride_l = c.n_pages * page; c.k_stride_p = c.v_stride_p = page; c.k_stride_t = c.v_stride_t = token; c.k_stride_h = c.v_stride_h = c.d;
    std::vector<int32_t> ref(c.n_pages, 1), table(c.n_pages), len(c.n_seqs), seqs(c.n_seqs), cu(c.n_seqs + 1);
    for (int i = 0; i < c.n_pages; i++) table[i] = i;
    std::shuffle(table.begin(), table.end(), r);
    for (int i = 0; i < c.n_seqs; i++) { len[i] = rnd(0, c.max_pages * c.page_size); seqs[i] = rnd(0, 9) ? i : -1; }
    c.page_ref = ref.data(); c.page_table = table.data(); c.seq_len = len.data();
    cu[0] = -rnd(0, 40);
    for (int i = 0; i < c.n_seqs; i++) cu[i + 1] = cu[i] + rnd(0, 50);
    const int64_t n_tokens = std::max<int64_t>(1, cu[c.n_seqs] - rnd(-3, 20));
    const size_t e = c.io_dtype == DCP_BF16 ? 2 : 4;
    if (posix_memalign((void**)&x, 256, n_tokens * token * e)) std::abort();
    std::fill(x, x + n_tokens * token * e, 0);
    LOOK(dcp_cache_append(&c, 0, seqs.data(), cu.data(), c.n_seqs, nullptr, x, token, c.d, x, token, c.d, n_tokens, nullptr) == DCP_OK);
    std::vector<int> want(c.n_pages * c.page_size, 0);
    for (int i = 0; i < c.n_seqs; i++) {
      if (seqs[i] < 0) continue;
      int begun = -1;   // block whose new tokens have begun
      for (int64_t t = cu[i]; t < cu[i + 1]; t++) {
        const int64_t pos = len[i] - (cu[i + 1] - t);
        if (t < 0 || t >= n_tokens || pos < 0) continue;
        int* page_of = want.data() + (int64_t)table[i * c.max_pages + pos / c.page_size] * c.page_size;
        const int slot = (int)(pos % c.page_size), block = (int)(pos / c.scale_block);
        if (block != begun)
          for (int y = slot / c.scale_block * c.scale_block; y < slot; y++) page_of[y] += 16;
        begun = block;
        page_of[slot] += 1;
      }
    }
    for (int64_t y = 0; y < (int64_t)c.n_pages * c.page_size; y++)
      for (int h = 0; h < c.hkv; h++) LOOK(codes[y * token + h * c.d] == want[y] && codes[y * token + h * c.d + c.d - 1] == want[y]);
    std::free(codes);
    std::free(x);
  }
  LOOK(g_below > 20 && g_older > 100);
  if (!g_bad) std::printf("host-asan append8 ok\n");
  return g_bad != 0;
}
