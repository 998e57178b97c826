// Drives the host code of the calls on a paged cache in 8 bits, of dcp_cache_read and of dcp_paged_attn_chunk_fwd through the C ABI on the CPU, in a build with
// AddressSanitizer and UndefinedBehaviorSanitizer, against the stand-in kernels of fake_cache.cpp and fake_cache8.cpp: random caches in buffers of exactly the
// documented sizes, a random life of each, and the largest sizes that the checks accept beside the smallest that they refuse.
#include <algorithm>
#include <climits>
#include <cstdint>
#include <cstdio>
#include <cstdlib>
#include <random>
#include <vector>

#include "dcp.h"

namespace dcp {
extern bool g_fake_count_only, g_fake_cache_bad;
extern int g_fake_cache_launches;
extern char *g_fake_ws, *g_fake_ws_end;
extern long g_fake_few, g_fake_tiles, g_fake_joins;
}
using namespace dcp;

static int g_fail = 0;
#define EXPECT(cond) do { if (!(cond)) { std::printf("EXPECT failed, line %d: %s (%s)\n", __LINE__, #cond, dcp_last_error()); g_fail++; } } while (0)

typedef std::mt19937_64 Rng;
static int rnd(Rng& r, int lo, int hi) { return lo + (int)(r() % (uint64_t)(hi - lo + 1)); }

struct Buffer {   // n bytes, aligned, with nothing behind them
  char* p;
  explicit Buffer(size_t n) : p(nullptr) { if (posix_memalign((void**)&p, 256, n ? n : 1)) std::abort(); }
  ~Buffer() { std::free(p); }
  Buffer(const Buffer&) = delete;
};
static void* with_workspace(Buffer& b, size_t n) { g_fake_ws = b.p; g_fake_ws_end = b.p + n; return b.p; }

static void one_life(Rng& r, int iter) {
  dcp_cache_t c{};
  c.n_layers = rnd(r, 1, 3); c.n_pages = rnd(r, 1, 60); c.hkv = rnd(r, 1, 6); c.d = 32 << rnd(r, 0, 2);
  c.scale_block = rnd(r, 0, 2) ? rnd(r, 1, 9) : 16;
  const int blocks = rnd(r, 1, 4);
  c.page_size = c.scale_block * blocks;
  c.dtype = iter % 4 ? DCP_E4M3 : rnd(r, 0, 1); c.io_dtype = rnd(r, 0, 1); c.n_seqs = rnd(r, 1, 12); c.max_pages = rnd(r, 1, 30);
  const bool codes = c.dtype == DCP_E4M3;
  const int e = codes ? 1 : c.dtype == DCP_BF16 ? 2 : 4, io = codes ? (c.io_dtype == DCP_BF16 ? 2 : 4) : e;
  const int64_t gap = 16 * rnd(r, 0, 2), row = c.d + gap, page = (int64_t)c.page_size * c.hkv * row, all = (int64_t)c.n_layers * c.n_pages * page - gap;
  const bool heads_inside = rnd(r, 0, 1);
  Buffer k(all * e), v(all * e), ks((size_t)c.n_layers * c.n_pages * blocks * c.hkv), vs((size_t)c.n_layers * c.n_pages * blocks * c.hkv);
  c.k = k.p; c.v = v.p;
  if (codes) { c.k_scale = (uint8_t*)ks.p; c.v_scale = (uint8_t*)vs.p; }
  c.k_stride_l = c.v_stride_l = c.n_pages * page; c.k_stride_p = c.v_stride_p = page;
  c.k_stride_t = c.v_stride_t = heads_inside ? c.hkv * row : row; c.k_stride_h = c.v_stride_h = heads_inside ? row : c.page_size * row;
  std::vector<int32_t> ref(c.n_pages, 0), table((size_t)c.n_seqs * c.max_pages, -1), len(c.n_seqs, 0);
  c.page_ref = ref.data(); c.page_table = table.data(); c.seq_len = len.data();
  for (int step = 0; step < 25; step++) {
    const int n = rnd(r, 1, iter % 10 == 0 ? 200 : 9), kind = rnd(r, 0, 5);
    std::vector<int32_t> seqs(n), status(n, 7), n_new(n), cu(n + 1, rnd(r, 0, 3));
    for (int32_t& s : seqs) s = rnd(r, -1, c.n_seqs);
    for (int i = 0; i < n; i++) { n_new[i] = rnd(r, 0, 3) ? rnd(r, 0, 3) : rnd(r, 0, 3 * c.page_size); cu[i + 1] = cu[i] + n_new[i]; }
    const int64_t tokens = std::max<int64_t>(0, cu[n] + rnd(r, -3, 3)), st = c.hkv * row;
    Buffer kn(std::max<int64_t>(0, (tokens * st - gap) * io)), vn(std::max<int64_t>(0, (tokens * st - gap) * io));
    if (kind <= 1) {
      EXPECT(dcp_cache_reserve(&c, seqs.data(), n_new.data(), n, status.data(), nullptr) == DCP_OK);
      for (int layer : {0, c.n_layers - 1})
        EXPECT(dcp_cache_append(&c, layer, seqs.data(), cu.data(), n, status.data(), kn.p, st, row, vn.p, st, row, tokens, nullptr) == DCP_OK);
    } else if (kind == 2) {
      std::vector<int32_t> dst(n);
      for (int32_t& s : dst) s = rnd(r, -1, c.n_seqs);
      EXPECT(dcp_cache_fork(&c, seqs.data(), dst.data(), n, status.data(), nullptr) == DCP_OK);
    } else if (kind == 3) {
      EXPECT(dcp_cache_free(&c, seqs.data(), std::min(n, 2), nullptr) == DCP_OK);
    } else if (kind == 4) {
      const size_t bytes = dcp_cache_workspace_bytes(&c);
      Buffer ws(bytes);
      std::vector<int32_t> counts(2, -1);
      EXPECT(dcp_cache_compact(&c, counts.data(), with_workspace(ws, bytes), bytes, nullptr) == DCP_OK);
    }
    for (int32_t& x : status) x = rnd(r, 0, 5) ? 0 : 1;
    const int32_t* codes_of = rnd(r, 0, 1) ? status.data() : nullptr;
    EXPECT(dcp_cache_read(&c, c.n_layers - 1, seqs.data(), cu.data(), n, codes_of, kn.p, st, row, vn.p, st, row, tokens, nullptr) == DCP_OK);
    const int hq = c.hkv * (rnd(r, 0, 2) ? rnd(r, 1, 16) : rnd(r, 17, 40));
    dcp_paged_attn_t a{};
    a.n = n; a.hq = hq; a.layer = rnd(r, 0, c.n_layers - 1); a.softmax_scale = 1.f; a.window = rnd(r, 0, 1) ? rnd(r, 1, 100) : 0; a.sink = rnd(r, 0, 40);
    a.seqs = seqs.data(); a.q_stride_t = a.o_stride_t = hq * row; a.q_stride_h = a.o_stride_h = row; a.status = codes_of;
    {
      const int64_t rows = (int64_t)n * hq * row - gap;
      Buffer q(rows * io), out(rows * io), ws(dcp_paged_attn_workspace_bytes(&c, n, hq));
      std::vector<float> lse((size_t)hq * n);
      const size_t bytes = dcp_paged_attn_workspace_bytes(&c, n, hq);
      a.q = q.p; a.out = out.p; a.lse = lse.data();
      EXPECT(dcp_paged_attn_fwd(&c, &a, with_workspace(ws, bytes), bytes, nullptr) == DCP_OK);
    }
    const int64_t rows = std::max<int64_t>(0, tokens * hq * row - gap);
    const size_t bytes = dcp_paged_attn_chunk_workspace_bytes(&c, n, tokens, hq);
    Buffer q(rows * io), out(rows * io), ws(bytes);
    std::vector<float> lse((size_t)hq * tokens);
    if (rnd(r, 0, 9) == 0) for (int32_t& x : cu) x = rnd(r, 0, 5) ? rnd(r, -5, (int)tokens + 5) : rnd(r, 0, 1) ? INT_MIN : INT_MAX;   // not ascending
    a.q = q.p; a.out = out.p; a.lse = lse.data();
    if (codes) {
      EXPECT(dcp_paged_attn_chunk_fwd(&c, &a, cu.data(), tokens, with_workspace(ws, bytes), bytes, nullptr) == DCP_OK);
      if (tokens) EXPECT(dcp_paged_attn_chunk_fwd(&c, &a, cu.data(), tokens, ws.p, bytes - 1, nullptr) == DCP_ERR_WORKSPACE);
    } else {
      EXPECT(dcp_paged_attn_chunk_fwd(&c, &a, cu.data(), tokens, ws.p, bytes, nullptr) == DCP_ERR_UNSUPPORTED);
    }
  }
}

static char* at(uint64_t x) { return (char*)(uintptr_t)x; }   // addresses that nothing follows

static dcp_cache_t big_cache() {
  dcp_cache_t c{};
  c.n_layers = 1 << 16; c.n_pages = 1 << 30; c.page_size = 1; c.hkv = 1; c.d = 128; c.dtype = DCP_E4M3; c.n_seqs = DCP_CACHE_MAX_SEQS; c.max_pages = 1 << 30;
  c.io_dtype = DCP_F32; c.scale_block = 1; c.k_scale = c.v_scale = (uint8_t*)at(1 << 12);
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
    if (shape == 1) { c.page_size = c.scale_block = 1 << 23; c.max_pages = 1 << 7; }   // 2^26 chunks of 16 bytes a page
    if (shape == 2) { c.hkv = 1 << 23; }
    if (shape == 3) { c.page_size = 1 << 10; c.scale_block = 2; c.hkv = 1 << 13; c.max_pages = 1 << 20; }
    const size_t bytes = dcp_cache_workspace_bytes(&c);
    g_fake_ws = at(uint64_t(1) << 40); g_fake_ws_end = g_fake_ws + bytes;
    EXPECT(dcp_cache_reserve(&c, ints, ints, most, ints, nullptr) == DCP_OK);
    EXPECT(dcp_cache_fork(&c, ints, ints, most, ints, nullptr) == DCP_OK);
    EXPECT(dcp_cache_compact(&c, ints, g_fake_ws, bytes, nullptr) == DCP_OK);
    for (int64_t n : {1, 1024, 1025, 1 << 25}) {
      EXPECT(dcp_cache_append(&c, c.n_layers - 1, ints, ints, most, ints, at(1 << 12), int64_t(1) << 58, int64_t(1) << 58, at(1 << 12), 128, int64_t(1) << 58, n, nullptr) == DCP_OK);
      EXPECT(dcp_cache_read(&c, c.n_layers - 1, ints, ints, most, ints, at(1 << 12), 128, 128, at(uint64_t(1) << 62), 128, 128, n, nullptr) == DCP_OK);
    }
    c.hkv = (1 << 26) / 8 / c.page_size + 1;
    EXPECT(dcp_cache_reserve(&c, ints, ints, 1, ints, nullptr) == DCP_ERR_UNSUPPORTED);
  }
  long taken = 0;
  for (int32_t hkv : {1, 3, 8, 4096})
    for (int64_t group : {int64_t(1), int64_t(8), int64_t(17), int64_t(65536), int64_t(INT_MAX)})
      for (int32_t n : {1, 200, DCP_CACHE_MAX_SEQS})
        for (int64_t tokens : {1, 200, 5000, 1 << 25})
          for (int32_t max_len : {1, 32, 1000, 1 << 17, 1 << 30})
            for (int32_t window : {0, 1, INT_MAX}) {
              if (group * hkv > INT_MAX) continue;
              dcp_cache_t c = big_cache();
              c.hkv = hkv; c.max_pages = max_len;
              if (window == 1) { c.io_dtype = DCP_BF16; c.page_size = c.scale_block = 16; c.max_pages = (max_len + 15) / 16; }
              dcp_paged_attn_t a{};
              a.n = n; a.hq = (int32_t)(group * hkv); a.layer = 7; a.softmax_scale = 3e38f; a.window = window; a.sink = window; a.seqs = ints; a.status = ints;
              a.q = at(1 << 12); a.out = at(uint64_t(1) << 62);
              a.q_stride_t = (int64_t)a.hq * 128; a.q_stride_h = 128; a.o_stride_t = int64_t(1) << 58; a.o_stride_h = int64_t(1) << 58; a.lse = (float*)at(1 << 12);
              const size_t bytes = dcp_paged_attn_chunk_workspace_bytes(&c, n, tokens, a.hq);
              g_fake_ws = at(uint64_t(1) << 40); g_fake_ws_end = g_fake_ws + bytes;
              const __int128 rows = (__int128)tokens * group;
              const int r = rows <= 24 * (__int128)n || rows * hkv <= 1024 ? 16 : 128;
              const __int128 tiles = ((int64_t)c.max_pages * c.page_size + 31) / 32;
              const bool ok = (__int128)tokens * a.hq < ((int64_t)1 << 31) - 128 && ((rows + r - 1) / r + n) * tiles * hkv <= INT_MAX;
              EXPECT(bytes > 0 && dcp_paged_attn_chunk_fwd(&c, &a, ints, tokens, g_fake_ws, bytes, nullptr) == (ok ? DCP_OK : DCP_ERR_UNSUPPORTED));
              taken += ok;
            }
  EXPECT(taken > 50);
  g_fake_count_only = false;
}

int main(int argc, char** argv) {
  Rng r(6);
  for (int i = 0; i < (argc > 1 ? std::atoi(argv[1]) : 100); i++) one_life(r, i);
  EXPECT(g_fake_few > 50 && g_fake_tiles > 50 && g_fake_joins > 50);
  limits();
  EXPECT(g_fake_cache_launches > 1000 && !g_fake_cache_bad);
  if (!g_fail) std::printf("host-asan cache8 ok\n");
  return g_fail != 0;
}
