// Drives the host code of the calls on a paged cache (csrc/cache_api.hip) through the C ABI on the CPU, in a build with AddressSanitizer
// and UndefinedBehaviorSanitizer, against the stand-in kernels of fake_cache.cpp: random caches in buffers of exactly the documented
// sizes, a random life of each, and the largest sizes that the checks accept beside the smallest that they refuse.
#include <algorithm>
#include <climits>
#include <cstdint>
#include <cstdio>
#include <cstdlib>
#include <random>
#include <vector>

#include "dcp.h"

namespace dcp {
extern bool g_fake_count_only, g_fake_cache_bad, g_fake_whole, g_fake_by_item;
extern int g_fake_cache_launches;
extern char *g_fake_ws, *g_fake_ws_end;
}
using namespace dcp;

static int g_fail = 0;
static long g_whole = 0, g_by_item = 0, g_by_worker = 0;   // attention calls of each form
#define EXPECT(cond) do { if (!(cond)) { std::printf("EXPECT failed, line %d: %s (%s)\n", __LINE__, #cond, dcp_last_error()); g_fail++; } } while (0)

typedef std::mt19937_64 Rng;
static int rnd(Rng& r, int lo, int hi) { return lo + (int)(r() % (uint64_t)(hi - lo + 1)); }

// n bytes, aligned, with nothing behind them
struct Buffer {
  char* p;
  explicit Buffer(size_t n) : p(nullptr) { if (posix_memalign((void**)&p, 256, n ? n : 1)) std::abort(); }
  ~Buffer() { std::free(p); }
  Buffer(const Buffer&) = delete;
};
static void* with_workspace(Buffer& b, size_t n) { g_fake_ws = b.p; g_fake_ws_end = b.p + n; return b.p; }

static void one_life(Rng& r, int iter) {
  dcp_cache_t c{};
  c.n_layers = rnd(r, 1, 3); c.n_pages = rnd(r, 1, 60); c.page_size = rnd(r, 1, iter % 3 ? 40 : 4); c.hkv = rnd(r, 1, 6); c.d = 32 << rnd(r, 0, 2);
  c.dtype = rnd(r, 0, 1); c.n_seqs = rnd(r, 1, 12); c.max_pages = rnd(r, 1, 30);
  const int e = c.dtype == DCP_BF16 ? 2 : 4;
  // rows with room between them, heads or tokens inside; the last row ends the buffer
  const int64_t gap = 8 * rnd(r, 0, 2), row = c.d + gap, page = (int64_t)c.page_size * c.hkv * row, all = (int64_t)c.n_layers * c.n_pages * page - gap;
  const bool heads_inside = rnd(r, 0, 1);
  Buffer k(all * e), v(all * e);
  c.k = k.p; c.v = v.p;
  c.k_stride_l = c.v_stride_l = c.n_pages * page; c.k_stride_p = c.v_stride_p = page;
  c.k_stride_t = c.v_stride_t = heads_inside ? c.hkv * row : row; c.k_stride_h = c.v_stride_h = heads_inside ? row : c.page_size * row;
  std::vector<int32_t> ref(c.n_pages, 0), table((size_t)c.n_seqs * c.max_pages, -1), len(c.n_seqs, 0);
  c.page_ref = ref.data(); c.page_table = table.data(); c.seq_len = len.data();
  auto held = [&](int s) { return (len[s] + c.page_size - 1) / c.page_size; };
  auto consistent = [&] {
    std::vector<int32_t> want(c.n_pages, 0);
    for (int s = 0; s < c.n_seqs; s++)
      for (int p = 0; p < held(s); p++) want[table[(size_t)s * c.max_pages + p]]++;
    return want == ref;
  };
  for (int step = 0; step < 25; step++) {
    const int n = rnd(r, 1, iter % 10 == 0 ? 200 : 9), kind = rnd(r, 0, 5);
    std::vector<int32_t> seqs(n), status(n, 7);
    for (int32_t& s : seqs) s = rnd(r, -1, c.n_seqs);
    if (kind <= 1) {
      std::vector<int32_t> n_new(n), cu(n + 1, 0);
      for (int i = 0; i < n; i++) { n_new[i] = rnd(r, 0, 3 * c.page_size); cu[i + 1] = cu[i] + n_new[i]; }
      EXPECT(dcp_cache_reserve(&c, seqs.data(), n_new.data(), n, status.data(), nullptr) == DCP_OK);
      const int64_t tokens = cu[n], st = c.hkv * row;
      Buffer kn(std::max<int64_t>(0, (tokens * st - gap) * e)), vn(std::max<int64_t>(0, (tokens * st - gap) * e));
      for (int layer : {0, c.n_layers - 1})
        EXPECT(dcp_cache_append(&c, layer, seqs.data(), cu.data(), n, status.data(), kn.p, st, row, vn.p, st, row, tokens, nullptr) == DCP_OK);
    } else if (kind == 2) {
      std::vector<int32_t> dst(n);
      for (int32_t& s : dst) s = rnd(r, -1, c.n_seqs);
      EXPECT(dcp_cache_fork(&c, seqs.data(), dst.data(), n, status.data(), nullptr) == DCP_OK);
    } else if (kind == 3) {
      const int m = std::min(n, 2);
      EXPECT(dcp_cache_free(&c, seqs.data(), m, nullptr) == DCP_OK);
    } else if (kind == 4) {
      const size_t bytes = dcp_cache_workspace_bytes(&c);
      Buffer ws(bytes);
      std::vector<int32_t> counts(2, -1);
      EXPECT(dcp_cache_compact(&c, counts.data(), with_workspace(ws, bytes), bytes, nullptr) == DCP_OK);
      for (int p = 0; p < c.n_pages; p++) EXPECT((ref[p] > 0) == (p < counts[0]));
    }
    EXPECT(consistent());
    const int hq = c.hkv * (rnd(r, 0, 2) ? rnd(r, 1, 16) : rnd(r, 17, 40));
    const int64_t q_st = hq * row, rows = (int64_t)n * hq * row - gap;
    Buffer q(rows * e), out(rows * e);
    std::vector<float> lse((size_t)hq * n);
    const size_t bytes = dcp_paged_attn_workspace_bytes(&c, n, hq);
    Buffer ws(bytes);
    for (int32_t& x : status) x = rnd(r, 0, 5) ? 0 : 1;
    dcp_paged_attn_t a{};
    a.n = n; a.hq = hq; a.layer = rnd(r, 0, c.n_layers - 1); a.softmax_scale = 1.f; a.window = rnd(r, 0, 1) ? rnd(r, 1, 100) : 0; a.sink = rnd(r, 0, 40);
    a.seqs = seqs.data(); a.q = q.p; a.q_stride_t = q_st; a.q_stride_h = row; a.out = out.p; a.o_stride_t = q_st; a.o_stride_h = row; a.lse = lse.data();
    a.status = rnd(r, 0, 1) ? status.data() : nullptr;
    EXPECT(dcp_paged_attn_fwd(&c, &a, with_workspace(ws, bytes), bytes, nullptr) == DCP_OK);
    (g_fake_whole ? g_whole : g_fake_by_item ? g_by_item : g_by_worker)++;
    EXPECT(dcp_paged_attn_fwd(&c, &a, ws.p, bytes - 1, nullptr) == DCP_ERR_WORKSPACE);
  }
}

// addresses that nothing follows
static char* at(uint64_t x) { return (char*)(uintptr_t)x; }

static dcp_cache_t big_cache() {
  dcp_cache_t c{};
  c.n_layers = 1 << 16; c.n_pages = 1 << 30; c.page_size = 1; c.hkv = 1; c.d = 128; c.dtype = DCP_F32; c.n_seqs = DCP_CACHE_MAX_SEQS; c.max_pages = 1 << 30;
  c.k = c.v = at(1 << 12);
  c.k_stride_l = c.k_stride_p = c.k_stride_t = c.k_stride_h = c.v_stride_l = c.v_stride_p = c.v_stride_t = c.v_stride_h = int64_t(1) << 58;
  c.page_ref = c.page_table = c.seq_len = (int32_t*)at(1 << 12);
  return c;
}

static void limits() {
  g_fake_count_only = true;
  int32_t* ints = (int32_t*)at(1 << 12);
  const int most = DCP_CACHE_MAX_SEQS;
  for (int shape = 0; shape < 4; shape++) {
    dcp_cache_t c = big_cache();
    if (shape == 1) { c.page_size = 1 << 21; c.max_pages = 1 << 9; }                  // 2^26 chunks of 16 bytes a page
    if (shape == 2) { c.hkv = 1 << 21; }
    if (shape == 3) { c.page_size = 1 << 10; c.hkv = 1 << 11; c.max_pages = 1 << 20; }
    const size_t bytes = dcp_cache_workspace_bytes(&c);
    g_fake_ws = at(uint64_t(1) << 40); g_fake_ws_end = g_fake_ws + bytes;
    EXPECT(dcp_cache_reserve(&c, ints, ints, most, ints, nullptr) == DCP_OK);
    EXPECT(dcp_cache_fork(&c, ints, ints, most, ints, nullptr) == DCP_OK);
    EXPECT(dcp_cache_free(&c, ints, most, nullptr) == DCP_OK);
    EXPECT(dcp_cache_compact(&c, ints, g_fake_ws, bytes, nullptr) == DCP_OK);
    EXPECT(dcp_cache_append(&c, c.n_layers - 1, ints, ints, most, ints, at(1 << 12), int64_t(1) << 58, int64_t(1) << 58, at(1 << 12), 128, int64_t(1) << 58, 1 << 25, nullptr) == DCP_OK);
    EXPECT(dcp_cache_append(&c, 0, ints, ints, most, ints, at(1 << 12), 128, 128, at(1 << 12), 128, 128, (1 << 25) + 1, nullptr) == DCP_ERR_UNSUPPORTED);
    struct { int32_t dcp_cache_t::*field; int32_t value; } beyond[] = {
        {&dcp_cache_t::n_layers, (1 << 16) + 1}, {&dcp_cache_t::n_pages, (1 << 30) + 1}, {&dcp_cache_t::n_seqs, most + 1},
        {&dcp_cache_t::max_pages, (1 << 30) / c.page_size + 1}, {&dcp_cache_t::hkv, (1 << 26) / 32 / c.page_size + 1}, {&dcp_cache_t::hkv, INT_MAX},
        {&dcp_cache_t::page_size, INT_MAX}, {&dcp_cache_t::max_pages, INT_MAX}};
    for (auto& x : beyond) {
      dcp_cache_t d = c;
      d.*x.field = x.value;
      EXPECT(dcp_cache_reserve(&d, ints, ints, 1, ints, nullptr) == DCP_ERR_UNSUPPORTED);
    }
  }
  // attention: the most places, sets, tiles and strides
  long taken = 0;
  for (int32_t hkv : {1, 3, 8, 128, 4096, 1 << 16})
    for (int64_t group : {int64_t(1), int64_t(8), int64_t(16), int64_t(17), int64_t(65536), int64_t(INT_MAX)})
      for (int32_t n : {1, 200, DCP_CACHE_MAX_SEQS})
        for (int32_t max_len : {1, 32, 1000, 1 << 17, 1 << 30})
          for (int32_t window : {0, 1, INT_MAX}) {
            if (group * hkv > INT_MAX) continue;
            dcp_cache_t c = big_cache();
            c.hkv = hkv; c.max_pages = max_len; c.dtype = window == 1 ? DCP_BF16 : DCP_F32;
            dcp_paged_attn_t a{};
            a.n = n; a.hq = (int32_t)(group * hkv); a.layer = 7; a.softmax_scale = 3e38f; a.window = window; a.sink = window; a.seqs = ints; a.status = ints;
            a.q = at(1 << 12); a.out = at(uint64_t(1) << 62);
            a.q_stride_t = (int64_t)a.hq * 128; a.q_stride_h = 128; a.o_stride_t = int64_t(1) << 58; a.o_stride_h = int64_t(1) << 58; a.lse = (float*)at(1 << 12);
            const size_t bytes = dcp_paged_attn_workspace_bytes(&c, n, a.hq);
            g_fake_ws = at(uint64_t(1) << 40); g_fake_ws_end = g_fake_ws + bytes;
            const int64_t sets = hkv * ((group + 15) / 16), tile = c.dtype == DCP_F32 ? 16 : 32;
            const bool ok = sets <= 4096 && (__int128)sets * n * ((max_len + tile - 1) / tile) <= INT_MAX;
            EXPECT(bytes > 0 && dcp_paged_attn_fwd(&c, &a, g_fake_ws, bytes, nullptr) == (ok ? DCP_OK : DCP_ERR_UNSUPPORTED));
            taken += ok;
          }
  EXPECT(taken > 50);
  g_fake_count_only = false;
}

int main(int argc, char** argv) {
  Rng r(5);
  for (int i = 0; i < (argc > 1 ? std::atoi(argv[1]) : 100); i++) {
    one_life(r, i);
  }
  EXPECT(g_whole > 20 && g_by_item > 20 && g_by_worker > 20);
  limits();
  EXPECT(g_fake_cache_launches > 1000 && !g_fake_cache_bad);
  if (!g_fail) std::printf("host-asan cache ok\n");
  return g_fail != 0;
}
