// Stand-ins for the kernels on a paged cache in 8 bits (csrc/cache8.hip, csrc/paged_attn8.hip, csrc/paged_chunk.hip, csrc/paged_chunk_few.hip), as fake_cache.cpp has
// them for the others: host walks with the kernels' index arithmetic that touch every byte the kernels would.  Test infrastructure, never part of the product.
#include <algorithm>
#include <climits>
#include <cstring>
#include <vector>

#include "cache_internal.h"

namespace dcp {

extern bool g_fake_count_only, g_fake_cache_bad;
extern int g_fake_cache_launches;
extern char *g_fake_ws, *g_fake_ws_end;
long g_fake_few = 0, g_fake_tiles = 0, g_fake_joins = 0;

#define LOOK(cond) do { if (!(cond)) { std::fprintf(stderr, "fake_cache8.cpp:%d: %s\n", __LINE__, #cond); g_fake_cache_bad = true; } } while (0)

static bool launched(uint64_t grid, uint64_t threads) {
  g_fake_cache_launches++;
  LOOK(grid >= 1 && grid * threads < (uint64_t(1) << 32));
  return !g_fake_count_only;
}
static void in_workspace(const void* p, size_t bytes) { LOOK((char*)p >= g_fake_ws && (char*)p <= g_fake_ws_end && (size_t)(g_fake_ws_end - (char*)p) >= bytes); }

static volatile char g_sink = 0;
static void touch(const char* p, size_t n) { if (n) g_sink = g_sink + p[0] + p[n - 1]; }

// One key and value of a KV head with their scales.
static void touch_key(const KCache& c, int32_t seq, int32_t j, int32_t hk, int32_t d) {
  const int32_t p = c.page.quot(j), page = const_cast<KCache&>(c).row(seq)[p], slot = c.page.rem(j, p);
  if (!c.is_page(page)) return;
  touch(c.k + page * c.k_sp + slot * c.k_st + hk * c.k_sh, d);
  touch(c.v + page * c.v_sp + slot * c.v_st + hk * c.v_sh, d);
  g_sink = g_sink + (char)c.k_scale[c.scale_at(page, slot) + hk] + (char)c.v_scale[c.scale_at(page, slot) + hk];
}

// The place of row t of the packed tokens: page and slot, page -1: nowhere.
static void token_at(const KCache& c, const int32_t* seqs, const int32_t* cu, int32_t n, const int32_t* status, int64_t t, int32_t* page, int32_t* slot, int32_t* first, int32_t* behind) {
  int i = -1;
  *page = -1;
  if (!cu) { if (t < n) { i = (int)t; *first = i; *behind = 1; } }
  else if (t >= cu[0] && t < cu[n]) {
    for (i = 0; cu[i + 1] <= t; i++) {}
    *first = cu[i];
    *behind = (int)(cu[i + 1] - t);
  }
  if (i < 0) return;
  const int s = seqs ? seqs[i] : i;
  if (!c.is_seq(s) || (status && status[i] != DCP_PLACE_OK)) return;
  const int pos = c.length(s) - *behind;
  if (pos < 0) return;
  const int p = c.page.quot(pos), entry = const_cast<KCache&>(c).row(s)[p];
  if (!c.is_page(entry)) return;
  *page = entry;
  *slot = c.page.rem(pos, p);
}

void launch_append_other(int32_t each, uint32_t grid, const KCache& c, int32_t layer, const int32_t* seqs, const int32_t* cu, int32_t n, const int32_t* status,
                         const NewTokens& x, hipStream_t);
void launch_append(int32_t each, uint32_t grid, const KCache& c, int32_t layer, const int32_t* seqs, const int32_t* cu, int32_t n, const int32_t* status,
                   const NewTokens& x, hipStream_t s) {
  if (!c.k_scale) return launch_append_other(each, grid, c, layer, seqs, cu, n, status, x, s);
  LOOK((each == 1 || each == 4 || each == 16 || each == 64) && (int64_t)grid * each >= x.n && (int64_t)(grid - 1) * each < x.n);
  const uint64_t columns = c.block.d == 1 ? 1 : std::min<int64_t>((2 * (int64_t)c.hkv + 3) / 4, std::max<int64_t>(1, (1 << 23) / grid));
  if (!launched(grid * columns, 256)) return;
  const int d = 16 << c.log_head_chunks;
  for (int64_t t = 0; t < x.n; t++) {
    int32_t page, slot, first = 0, behind = 0;
    token_at(c, seqs, cu, n, status, t, &page, &slot, &first, &behind);
    if (page < 0) continue;
    const int32_t older = c.block.rem(slot, c.block.quot(slot));
    if (older && t != first) continue;
    const int32_t rows = (int32_t)std::min<int64_t>(std::min(behind, (int32_t)c.block.d - older), x.n - t);
    LOOK(rows >= 1 && slot - older >= 0 && slot + rows <= (int32_t)c.page.d);
    for (int h = 0; h < c.hkv; h++)
      for (int y = -older; y < rows; y++) {
        char* k = c.k + layer * c.k_sl + page * c.k_sp + (slot + y) * c.k_st + h * c.k_sh;
        char* v = c.v + layer * c.v_sl + page * c.v_sp + (slot + y) * c.v_st + h * c.v_sh;
        if (y >= 0) {
          touch(x.k + (t + y) * x.k_st + h * x.k_sh, (size_t)d * c.io_bytes);
          touch(x.v + (t + y) * x.v_st + h * x.v_sh, (size_t)d * c.io_bytes);
        }
        std::memset(k, 1, d);
        std::memset(v, 1, d);
        c.k_scale[layer * c.layer_scales() + c.scale_at(page, slot) + h] = 120;
        c.v_scale[layer * c.layer_scales() + c.scale_at(page, slot) + h] = 120;
      }
  }
}

void launch_read(int32_t each, uint32_t grid, const KCache& c, int32_t layer, const int32_t* seqs, const int32_t* cu, int32_t n, const int32_t* status,
                 const ReadTokens& x, hipStream_t) {
  LOOK((each == 1 || each == 4) && (int64_t)grid * each >= x.n && (int64_t)(grid - 1) * each < x.n);
  if (!launched(grid, 256)) return;
  const int row = 16 << c.log_head_chunks;                         // bytes of a head in the cache
  const int out = c.k_scale ? row * c.io_bytes : row;
  for (int64_t t = 0; t < x.n; t++) {
    int32_t page, slot, first = 0, behind = 0;
    token_at(c, seqs, cu, n, status, t, &page, &slot, &first, &behind);
    if (page < 0) continue;
    for (int h = 0; h < c.hkv; h++) {
      touch(c.k + layer * c.k_sl + page * c.k_sp + slot * c.k_st + h * c.k_sh, row);
      touch(c.v + layer * c.v_sl + page * c.v_sp + slot * c.v_st + h * c.v_sh, row);
      if (c.k_scale) g_sink = g_sink + (char)c.k_scale[layer * c.layer_scales() + c.scale_at(page, slot) + h] + (char)c.v_scale[layer * c.layer_scales() + c.scale_at(page, slot) + h];
      std::memset(x.k + t * x.k_st + h * x.k_sh, 0, out);
      std::memset(x.v + t * x.v_st + h * x.v_sh, 0, out);
    }
  }
}

void launch_paged_attn_other(int32_t dtype, int32_t d, uint32_t grid, const KCache& c, const PagedArgs& a, const PagedParts& parts, hipStream_t s);
void launch_paged_attn(int32_t dtype, int32_t d, uint32_t grid, const KCache& c, const PagedArgs& a, const PagedParts& parts, hipStream_t s) {
  if (dtype != DCP_E4M3) return launch_paged_attn_other(dtype, d, grid, c, a, parts, s);
  const int tile = kPagedKeys, e = c.io_bytes;
  const size_t slots = 2 * (size_t)kWorkers * a.abreast * a.set_heads;
  if (!a.whole) {
    in_workspace(parts.joins, kWorkers * sizeof(int4));
    in_workspace(parts.o, slots * d * sizeof(float));
    in_workspace(parts.ml, slots * sizeof(float2));
  }
  LOOK(a.whole ? grid == (uint64_t)a.n * a.groups && grid <= kWorkers : grid == kWorkers);
  if (!launched(grid, kPagedThreads)) return;
  int64_t all = 0;
  for (int i = 0; i < a.n; i++) {
    const int s = a.status && a.status[i] != DCP_PLACE_OK ? -1 : a.seqs ? a.seqs[i] : i;
    if (!c.is_seq(s)) continue;
    const KeyTiles keys(c.length(s), a.window, a.sink, tile);
    all += a.whole ? 1 : keys.count;
    for (int hk = 0; hk < c.hkv; hk++)
      for (int x = 0; x < keys.count; x++)
        for (int j = keys.tile_at(x) * tile; j < (keys.tile_at(x) + 1) * tile; j++)
          if (keys.sees(j)) touch_key(c, s, j, hk, d);
    for (int h = 0; h < a.group * c.hkv; h++) {
      std::memcpy(a.out + i * a.o_st + h * a.o_sh, a.q + i * a.q_st + h * a.q_sh, (size_t)d * e);
      a.lse[(int64_t)h * a.n + i] = 0;
    }
  }
  LOOK(all * a.groups <= INT_MAX);
}

// The plan as chunk_plan_kernel makes it, the workers' walks with the parts that they leave, and the joins; every row is written once.
void launch_chunk(int32_t d, const KCache& c, const ChunkArgs& a, const ChunkPlan& plan, hipStream_t) {
  in_workspace(plan.head, sizeof(int4));
  in_workspace(plan.starts, kWorkers * sizeof(int4));
  in_workspace(plan.joins, kWorkers * sizeof(ChunkJoin));
  in_workspace(plan.items, (size_t)a.max_items * sizeof(ChunkItem));
  in_workspace(plan.o, 2 * (size_t)kWorkers * a.rows * d * sizeof(float));
  in_workspace(plan.ml, 2 * (size_t)kWorkers * a.rows * sizeof(float2));
  LOOK((char*)(plan.head + 1) <= (char*)plan.starts && (char*)(plan.starts + kWorkers) <= (char*)plan.joins && (char*)(plan.joins + kWorkers) <= (char*)plan.items);
  LOOK((char*)(plan.items + a.max_items) <= (char*)plan.o && (char*)(plan.o + 2 * (size_t)kWorkers * a.rows * d) <= (char*)plan.ml);
  LOOK((reinterpret_cast<uintptr_t>(plan.joins) | reinterpret_cast<uintptr_t>(plan.items) | reinterpret_cast<uintptr_t>(plan.o)) % 16 == 0 && reinterpret_cast<uintptr_t>(plan.ml) % 8 == 0);
  LOOK((a.rows == kFewItem && a.tile == kPagedKeys) || (a.rows == kChunkRows && a.tile == kChunkKeys));
  (a.rows == kChunkRows ? g_fake_tiles : g_fake_few)++;
  g_fake_cache_launches += 2;
  if (!launched(kWorkers * 4, 256)) return;
  int32_t n_items = 0, tiles = 0;
  for (int i = 0; i < a.n; i++) {
    const int s = a.seqs ? a.seqs[i] : i;
    if (!c.is_seq(s) || (a.status && a.status[i] != DCP_PLACE_OK)) continue;
    const ChunkPlace p(a.cu[i], a.cu[i + 1], a.n_tokens, c.length(s));
    LOOK(p.count >= 0 && p.first >= 0 && p.first + (int64_t)p.count <= a.n_tokens && p.pos >= 0 && p.pos + p.count <= c.length(s));
    const int32_t rows = p.count * (int32_t)a.group.d;
    for (int32_t row0 = 0; row0 < rows && n_items < a.max_items; row0 += a.rows) {
      const int32_t lo = p.pos + a.group.quot(row0), hi = p.pos + a.group.quot(std::min(row0 + a.rows, rows) - 1);
      ChunkItem it{s, p.first, p.pos, rows, row0, chunk_tiles(lo, hi, a.window, a.sink, a.tile).count, tiles, 0};
      tiles += it.tiles;
      plan.items[n_items++] = it;
    }
  }
  LOOK((int64_t)tiles * c.hkv <= INT_MAX);
  *plan.head = make_int4(n_items, tiles, 0, 0);
  if (!n_items) return;
  const Shares<kLogWorkers> sh(tiles * c.hkv);
  LOOK(sh.workers <= kWorkers);
  for (int hk = 0; hk < c.hkv; hk++)
    for (int x = 0; x < n_items; x++) {
      const ChunkItem it = plan.items[x];
      const int32_t end = std::min(it.row0 + a.rows, it.rows), begin = hk * tiles + it.before;
      const int32_t lo = it.pos + a.group.quot(it.row0), hi = it.pos + a.group.quot(end - 1);
      const KeyTiles keys = chunk_tiles(lo, hi, a.window, a.sink, a.tile);
      for (int y = 0; y < keys.count; y++)
        for (int j = keys.tile_at(y) * a.tile; j < std::min((keys.tile_at(y) + 1) * a.tile, keys.len); j++) touch_key(c, it.seq, j, hk, d);
      const int first = sh.worker_of(begin), last = sh.worker_of(begin + it.tiles - 1);
      if (first != last) {
        g_fake_joins++;
        plan.joins[first] = ChunkJoin{hk, first, last, 0, it.first, it.rows, it.row0, 0};
        plan.starts[first] = make_int4(0, 0, 0, 0);
        for (int w = first; w <= last; w++)
          for (int r = 0; r < end - it.row0; r++) {
            const size_t slot = (size_t)(2 * w + (w == first)) * a.rows + r;
            plan.ml[slot] = make_float2(0, 0);
            plan.o[slot * d] = plan.o[slot * d + d - 1] = 0;
          }
      }
      for (int r = it.row0; r < end; r++) {
        const int32_t t = a.group.quot(r), token = it.first + t, head = hk * (int32_t)a.group.d + r - t * (int32_t)a.group.d;
        std::memcpy(a.out + token * a.o_st + head * a.o_sh, a.q + token * a.q_st + head * a.q_sh, (size_t)d * c.io_bytes);
        a.lse[head * a.n_tokens + token] = 0;
      }
    }
}

}  // namespace dcp
