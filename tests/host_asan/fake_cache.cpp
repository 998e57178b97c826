// A stand-in for the kernels on a paged key-value cache (csrc/cache.hip, csrc/paged_attn.hip) in the CPU build of their host code: every
// launch is a host walk over the same arrays with the index arithmetic of the kernel it stands for, so that an index, a stride or a part
// of a workspace that would leave its array on the GPU leaves it here and is reported.  Test infrastructure, never part of the product.
#include <algorithm>
#include <climits>
#include <cstring>
#include <vector>

#include "cache_internal.h"

namespace dcp {

bool g_fake_count_only = false;       // sizes of launches are looked at, no array is: for sizes that no host has room for
int g_fake_cache_launches = 0;
bool g_fake_cache_bad = false;        // a launch that the GPU would not take, or a walk that went wrong
char *g_fake_ws = nullptr, *g_fake_ws_end = nullptr;
bool g_fake_whole = false, g_fake_by_item = false;

#define LOOK(cond) do { if (!(cond)) { std::fprintf(stderr, "fake_cache.cpp:%d: %s\n", __LINE__, #cond); g_fake_cache_bad = true; } } while (0)

static bool launched(uint64_t grid, uint64_t threads) {
  g_fake_cache_launches++;
  LOOK(grid >= 1 && grid * threads < (uint64_t(1) << 32));
  return !g_fake_count_only;
}
static void in_workspace(const void* p, size_t bytes) { LOOK((char*)p >= g_fake_ws && (size_t)(g_fake_ws_end - (char*)p) >= bytes && (char*)p <= g_fake_ws_end); }

void launch_take(bool fork, const KCache& cc, const int32_t* a, const int32_t* b, int32_t n, int32_t* status, hipStream_t) {
  if (!launched(1, 1024)) return;
  KCache c = cc;
  std::vector<int32_t> owner(c.n_seqs, INT_MAX);
  for (int i = 0; i < n; i++) {
    const int s = a ? a[i] : i;
    if (!c.is_seq(s)) continue;
    const int t = fork ? b[i] : s;
    if (c.is_seq(t)) owner[t] = std::min(owner[t], i);
  }
  const int32_t cap = c.n_pages + 1;
  int32_t total = 0;
  std::vector<int32_t> free_pages;
  for (int32_t p = 0; p < c.n_pages; p++)
    if (c.ref[p] <= 0) free_pages.push_back(p);
  const int32_t found = (int32_t)free_pages.size();
  for (int i = 0; i < n; i++) {
    const int s = a ? a[i] : i;
    status[i] = DCP_PLACE_OK;
    if (s < 0) continue;
    status[i] = DCP_PLACE_BAD;
    if (!c.is_seq(s)) continue;
    const int32_t len = c.length(s), x = fork ? 0 : b ? b[i] : 1, t = fork ? b[i] : s;
    if (fork ? !c.is_seq(t) || owner[t] != i || owner[s] != INT_MAX || c.length(t) != 0 : owner[s] != i || x < 0 || x > c.max_len - len) continue;
    const int32_t tokens = len + x, first = fork ? c.page.quot(tokens) : c.pages_of(len), need = c.pages_of(tokens) - first;
    const int32_t before = total;
    total = add_capped(total, std::min(need, cap), cap);
    status[i] = need > 0 && total > found ? DCP_PLACE_FULL : DCP_PLACE_OK;
    if (status[i] != DCP_PLACE_OK) continue;
    for (int32_t k = 0; k < need; k++) { c.row(t)[first + k] = free_pages[before + k]; c.ref[free_pages[before + k]] = 1; }
    c.len[t] = tokens;
  }
}

static void copy_piece(const KCache& c, char* base, int64_t st_p, int64_t st_t, int64_t st_h, int from, int to, int first, int last) {
  for (int x = first; x < last; x++) {
    const int row = x >> c.log_head_chunks, t = c.heads.quot(row);
    const int64_t off = t * st_t + c.heads.rem(row, t) * st_h + (x & (c.head_chunks() - 1)) * 16;
    std::memcpy(base + to * st_p + off, base + from * st_p + off, 16);
  }
}

void launch_fork(uint32_t grid, const KCache& cc, const int32_t* src, const int32_t* dst, int32_t n, const int32_t* status, int32_t pieces, hipStream_t) {
  const int64_t per_place = 1 + 2 * (int64_t)cc.n_layers * pieces, units = n * per_place;
  if (!launched(grid, 256)) return;
  KCache c = cc;
  for (int64_t unit = 0; unit < units; unit++) {
    const int i = (int)quot64(unit, per_place), a = src[i], b = dst[i];
    const int64_t y = unit - i * per_place;
    if (a < 0 || status[i] != DCP_PLACE_OK) continue;
    const int len = c.length(a), whole = c.page.quot(len);
    if (y == 0) {
      for (int p = 0; p < whole; p++) {
        c.row(b)[p] = c.row(a)[p];
        if (c.is_page(c.row(a)[p])) c.ref[c.row(a)[p]]++;
      }
      continue;
    }
    const int64_t x = (y - 1) >> 1, layer = quot64(x, pieces);
    const int first = (int)(x - layer * pieces) * kPieceChunks, last = std::min(first + kPieceChunks, c.page.rem(len, whole) * c.hkv << c.log_head_chunks);
    if (first >= last) continue;
    const int32_t page = c.row(a)[whole], mine = c.row(b)[whole];
    if (!c.is_page(page) || !c.is_page(mine)) continue;
    if (y & 1) copy_piece(c, c.k + layer * c.k_sl, c.k_sp, c.k_st, c.k_sh, page, mine, first, last);
    else copy_piece(c, c.v + layer * c.v_sl, c.v_sp, c.v_st, c.v_sh, page, mine, first, last);
  }
}

void launch_free(uint32_t grid, const KCache& cc, const int32_t* seqs, hipStream_t) {
  if (!launched(grid, 256)) return;
  KCache c = cc;
  for (uint32_t i = 0; i < grid; i++) {
    const int s = seqs ? seqs[i] : (int)i;
    if (!c.is_seq(s)) continue;
    const int held = c.pages_of(c.length(s));
    c.len[s] = 0;
    for (int p = 0; p < held; p++) {
      if (c.is_page(c.row(s)[p])) c.ref[c.row(s)[p]]--;
      c.row(s)[p] = -1;
    }
  }
}

void launch_list_moves(const KCache& c, const Moves& m, int32_t* counts, hipStream_t) {
  const size_t half = (size_t)c.n_pages / 2 + 1;
  in_workspace(m.count, 4);
  in_workspace(m.from, 4 * half);
  in_workspace(m.to, 4 * half);
  in_workspace(m.where, 4 * (size_t)c.n_pages);
  LOOK(m.count + 1 <= m.from && m.from + half <= m.to && m.to + half <= m.where);
  if (!launched(1, 1024)) return;
  int n_used = 0, holes = 0, high = 0;
  for (int p = 0; p < c.n_pages; p++) n_used += c.ref[p] > 0;
  for (int p = 0; p < c.n_pages; p++) {
    if (p < n_used) { if (c.ref[p] <= 0) { LOOK((size_t)holes < half); m.to[holes++] = p; } }
    else if (c.ref[p] > 0) { LOOK((size_t)high < half); m.from[high++] = p; }
    else m.where[p] = -1;
  }
  LOOK(holes == high);
  for (int k = 0; k < high; k++) m.where[m.from[k]] = m.to[k];
  *m.count = counts[1] = high;
  counts[0] = n_used;
}

void launch_move(uint32_t grid, const KCache& cc, const Moves& m, const int32_t* counts, int32_t pieces, hipStream_t) {
  LOOK(grid > (uint32_t)cc.n_seqs);   // somebody moves
  if (!launched(grid, 256)) return;
  KCache c = cc;
  for (int s = 0; s < c.n_seqs; s++)
    for (int p = 0; p < c.pages_of(c.length(s)); p++) {
      int32_t& page = c.row(s)[p];
      if (c.is_page(page) && page >= counts[0] && m.where[page] >= 0) page = m.where[page];
    }
  const int64_t per_page = 2 * (int64_t)c.n_layers * pieces, units = *m.count * per_page;
  const int all = c.page.d * c.hkv << c.log_head_chunks;
  for (int64_t x = 0; x < units; x++) {
    const int64_t k = quot64(x, per_page), y = x - k * per_page, layer = quot64(y >> 1, pieces);
    const int first = (int)((y >> 1) - layer * pieces) * kPieceChunks, last = std::min(first + kPieceChunks, all);
    if (y == 0) { c.ref[m.to[k]] = c.ref[m.from[k]]; c.ref[m.from[k]] = 0; }
    if (y & 1) copy_piece(c, c.v + layer * c.v_sl, c.v_sp, c.v_st, c.v_sh, m.from[k], m.to[k], first, last);
    else copy_piece(c, c.k + layer * c.k_sl, c.k_sp, c.k_st, c.k_sh, m.from[k], m.to[k], first, last);
  }
}

void launch_append(int32_t each, uint32_t grid, const KCache& c, int32_t layer, const int32_t* seqs, const int32_t* cu, int32_t n, const int32_t* status,
                   const NewTokens& x, hipStream_t) {
  LOOK((each == 1 || each == 4) && (int64_t)grid * each >= x.n && (int64_t)(grid - 1) * each < x.n);
  if (!launched(grid, 256)) return;
  for (int64_t t = 0; t < x.n; t++) {
    int i = -1, behind = 0;
    if (!cu) { if (t < n) { i = (int)t; behind = 1; } }
    else if (t >= cu[0] && t < cu[n]) {
      for (i = 0; cu[i + 1] <= t; i++) {}
      behind = (int)(cu[i + 1] - t);
    }
    if (i < 0) continue;
    const int s = seqs ? seqs[i] : i;
    if (!c.is_seq(s) || (status && status[i] != DCP_PLACE_OK)) continue;
    const int pos = c.length(s) - behind;
    if (pos < 0) continue;
    const int p = c.page.quot(pos), entry = c.row(s)[p], slot = c.page.rem(pos, p);
    if (!c.is_page(entry)) continue;
    for (int h = 0; h < c.hkv; h++)
      for (int off = 0; off < 16 * c.head_chunks(); off += 16) {
        std::memcpy(c.k + layer * c.k_sl + entry * c.k_sp + slot * c.k_st + h * c.k_sh + off, x.k + t * x.k_st + h * x.k_sh + off, 16);
        std::memcpy(c.v + layer * c.v_sl + entry * c.v_sp + slot * c.v_st + h * c.v_sh + off, x.v + t * x.v_st + h * x.v_sh + off, 16);
      }
  }
}

// The shares of the workers, the parts that they leave and the joins; of every key that is seen one byte of K and of V is read.
void launch_paged_attn(int32_t dtype, int32_t d, uint32_t grid, const KCache& c, const PagedArgs& a, const PagedParts& parts, hipStream_t) {
  const int tile = dtype == DCP_F32 ? 16 : 32, e = dtype == DCP_F32 ? 4 : 2;
  const size_t slots = 2 * (size_t)kWorkers * a.abreast * a.set_heads;
  if (!a.whole) {
    in_workspace(parts.joins, kWorkers * sizeof(int4));
    in_workspace(parts.o, slots * d * sizeof(float));
    in_workspace(parts.ml, slots * sizeof(float2));
    LOOK((char*)(parts.joins + kWorkers) <= (char*)parts.o && (char*)(parts.o + slots * d) <= (char*)parts.ml);
  }
  LOOK(a.abreast == 1 << a.log_abreast && a.abreast <= kPagedWaves && (int64_t)a.groups * a.abreast == (int64_t)c.hkv * a.per_kv);
  LOOK((int64_t)a.per_kv * kSetHeads >= a.group && (a.per_kv == 1 || a.set_heads == kSetHeads) && a.set_heads <= a.group);
  LOOK(a.whole ? grid == (uint64_t)a.n * a.groups && grid <= kWorkers : grid == kWorkers);
  g_fake_whole = a.whole;
  g_fake_by_item = parts.by_item;
  if (!launched(grid, kPagedThreads)) return;
  auto seq_at = [&](int i) { const int s = a.seqs ? a.seqs[i] : i; return a.status && a.status[i] != DCP_PLACE_OK ? -1 : s; };
  int64_t all = 0;
  for (int i = 0; i < a.n; i++)
    if (c.is_seq(seq_at(i))) all += a.whole ? 1 : KeyTiles(c.length(seq_at(i)), a.window, a.sink, tile).count;
  LOOK(all * a.groups <= INT_MAX);
  if (all == 0) return;
  const Shares<kLogWorkers> sh((int32_t)(all * a.groups));
  LOOK((uint32_t)sh.workers <= grid);
  int64_t before = 0;
  volatile char sink = 0;
  for (int i = 0; i < a.n; i++) {
    const int s = seq_at(i);
    if (!c.is_seq(s)) continue;
    const KeyTiles keys(c.length(s), a.window, a.sink, tile);
    const int units = a.whole ? 1 : keys.count;
    for (int grp = 0; grp < a.groups; grp++) {
      const int32_t begin = (int32_t)(before * a.groups + (int64_t)grp * units), first = sh.worker_of(begin), last = sh.worker_of(begin + units - 1);
      if (!a.whole) {
        if (parts.by_item) { LOOK((int64_t)i * a.groups + grp < kWorkers); parts.joins[i * a.groups + grp] = make_int4(i, grp, first, last); }
        else parts.joins[first] = make_int4(i, grp, first, last);
      }
      for (int beside = 0; beside < a.abreast; beside++) {
        const int set = grp * a.abreast + beside, hk = set / a.per_kv, h0 = hk * a.group + (set - hk * a.per_kv) * kSetHeads;
        const int n_heads = std::min(kSetHeads, (hk + 1) * a.group - h0);
        LOOK(hk < c.hkv && n_heads >= 1 && n_heads <= a.set_heads);
        for (int x = 0; x < keys.count; x++)
          for (int j = keys.tile_at(x) * tile; j < (keys.tile_at(x) + 1) * tile; j++) {
            if (!keys.sees(j)) continue;
            const int p = c.page.quot(j), page = c.row(s)[p], slot = c.page.rem(j, p);
            if (!c.is_page(page)) continue;
            sink = sink + c.k[page * c.k_sp + slot * c.k_st + hk * c.k_sh + d * e - 1] + c.v[page * c.v_sp + slot * c.v_st + hk * c.v_sh + d * e - 1];
          }
        for (int h = h0; h < h0 + n_heads; h++) {
          std::memcpy(a.out + i * a.o_st + h * a.o_sh, a.q + i * a.q_st + h * a.q_sh, (size_t)d * e);
          a.lse[(int64_t)h * a.n + i] = 0;
          if (first == last) continue;
          for (int w = first; w <= last; w++) {
            const size_t slot = ((size_t)(w == first ? 2 * w + 1 : 2 * w) * a.abreast + beside) * a.set_heads + (h - h0);
            parts.ml[slot] = make_float2(0, 0);
            parts.o[slot * d] = parts.o[slot * d + d - 1] = 0;
          }
        }
      }
    }
    before += units;
  }
}

}  // namespace dcp
