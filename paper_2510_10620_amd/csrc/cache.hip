// The calls that change a paged key-value cache: pages are taken, shared, given back and moved to the front, and new
// tokens are written into them.  Everything is decided on the device from page_ref, page_table and seq_len, so that a
// decoding step never waits for the host.
#include "cache_internal.h"

using namespace dcp;

namespace dcp {

static constexpr int kMapThreads = 1024, kMapWaves = kMapThreads / 64;
static constexpr int kScan = 8;           // page_ref entries a lane has in flight
static constexpr int kNoOwner = INT_MAX;

// Inclusive sums over the workgroup, cut at `cap`.
__device__ __forceinline__ int block_sum(int x, int cap, int* wave_sum, int* total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int y = __shfl_up(x, o);
    if (lane >= o) x = add_capped(x, y, cap);
  }
  __syncthreads();
  if (lane == 63) wave_sum[wave] = x;
  __syncthreads();
  int before = 0, all = 0;
#pragma unroll
  for (int w = 0; w < kMapWaves; w++) {
    const int v = wave_sum[w];
    if (w < wave) before = add_capped(before, v, cap);
    all = add_capped(all, v, cap);
  }
  *total = all;
  return add_capped(before, x, cap);
}

// What a place of dcp_cache_reserve (dcp_cache_fork) asks for: `need` pages for row `seq` of the table from entry `first` on,
// after which the sequence has `tokens` tokens.  seq -1: padding, or not OK.
struct Place {
  int32_t seq, first, need, tokens, code;
};

// What is read for a place: s is seqs[i] (src[i]), t n_new[i] (dst[i]); the lengths of s and, for a fork, of t.
struct Asked {
  int32_t s, t, len, len_t;
};
template <bool FORK>
__device__ __forceinline__ Asked asked_at(const KCache& c, const int32_t* a, const int32_t* b, int i) {
  Asked x{a ? a[i] : i, 1, 0, 0};
  if (FORK || b) x.t = b[i];
  if (c.is_seq(x.s)) x.len = c.length(x.s);
  if (FORK && c.is_seq(x.t)) x.len_t = c.length(x.t);
  return x;
}

// owner[s]: the first place that changes sequence s.
template <bool FORK>
__device__ __forceinline__ Place place_of(const KCache& c, const Asked& x, int i, const int32_t* owner) {
  Place p{-1, 0, 0, 0, DCP_PLACE_OK};
  if (x.s < 0) return p;
  p.code = DCP_PLACE_BAD;
  if (!c.is_seq(x.s)) return p;
  if (FORK) {
    if (!c.is_seq(x.t) || owner[x.t] != i || owner[x.s] != kNoOwner || x.len_t != 0) return p;
    p.tokens = x.len;
    p.seq = x.t;
    p.first = c.page.quot(p.tokens);
    p.need = c.page.rem(p.tokens, p.first) != 0;
  } else {
    if (owner[x.s] != i || x.t < 0 || x.t > c.max_len - x.len) return p;
    p.tokens = x.len + x.t;
    p.seq = x.s;
    p.first = c.pages_of(x.len);
    p.need = c.pages_of(p.tokens) - p.first;
  }
  p.code = DCP_PLACE_OK;
  return p;
}
template <bool FORK>
__device__ __forceinline__ Place place_at(const KCache& c, const int32_t* a, const int32_t* b, int i, const int32_t* owner) {
  return place_of<FORK>(c, asked_at<FORK>(c, a, b, i), i, owner);
}

// One workgroup: the places' needs are summed up in their order, page_ref is walked once, and the k-th free page goes to the place
// whose sums k falls between.  That a place finds too few pages is known at the end: the one that got some gives them back.
// Bound by latency: two dependent trips to memory (the places, their lengths; the first 8 192 entries of page_ref come meanwhile), and one
// for each further 8 192 pages until enough are found.  Up to kMapThreads places stay in registers and LDS, more are worked out anew.
template <bool FORK>
__global__ __launch_bounds__(kMapThreads) void take_kernel(KCache c, const int32_t* __restrict__ a, const int32_t* __restrict__ b,
                                                           int32_t n, int32_t* __restrict__ status) {
  __shared__ int32_t owner[DCP_CACHE_MAX_SEQS], sums[DCP_CACHE_MAX_SEQS], seqs[kMapThreads], firsts[kMapThreads], wave_sum[kMapWaves], short_place;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int cap = c.n_pages + 1;
  const bool few = n <= kMapThreads;
  int32_t held[kScan];
  auto scan = [&](int64_t first) {
#pragma unroll
    for (int u = 0; u < kScan; u++) held[u] = first + u * 64 < c.n_pages ? c.ref[first + u * 64] : 1;
  };
  scan(wave * (64 * kScan) + lane);
  Asked ask{-1, 0, 0, 0};   // of place tid
  if (tid < n) ask = asked_at<FORK>(c, a, b, tid);
  for (int s = tid; s < c.n_seqs; s += kMapThreads) owner[s] = kNoOwner;
  if (tid == 0) short_place = -1;
  __syncthreads();
  for (int i = tid; i < n; i += kMapThreads) {
    const int s = i == tid ? ask.s : a ? a[i] : i;
    if (!c.is_seq(s)) continue;
    const int t = !FORK ? s : i == tid ? ask.t : b[i];
    if (c.is_seq(t)) atomicMin(&owner[t], i);
  }
  __syncthreads();
  Place mine{-1, 0, 0, 0, DCP_PLACE_OK};
  int total = 0;
  for (int base = 0; base < n; base += kMapThreads) {
    const int i = base + tid;
    if (i < n) mine = base ? place_at<FORK>(c, a, b, i, owner) : place_of<FORK>(c, ask, i, owner);
    int all;
    const int x = block_sum(i < n ? min(mine.need, cap) : 0, cap, wave_sum, &all);
    if (i < n) sums[i] = add_capped(total, x, cap);
    total = add_capped(total, all, cap);
  }
  if (few) { seqs[tid] = mine.seq; firsts[tid] = mine.first; }
  __syncthreads();
  int found = 0;
  for (int64_t base = 0; base < c.n_pages && found < total; base += kMapThreads * kScan) {
    const int64_t first = base + wave * (64 * kScan) + lane;
    if (base) scan(first);
    uint64_t mask[kScan];
    int free_here = 0;
#pragma unroll
    for (int u = 0; u < kScan; u++) {
      mask[u] = __ballot(held[u] <= 0);
      free_here += __popcll(mask[u]);
    }
    __syncthreads();
    if (lane == 0) wave_sum[wave] = free_here;
    __syncthreads();
    int k = found, all = 0;   // k: free pages before the wave's
#pragma unroll
    for (int w = 0; w < kMapWaves; w++) {
      if (w < wave) k += wave_sum[w];
      all += wave_sum[w];
    }
#pragma unroll
    for (int u = 0; u < kScan; u++) {
      const int rank = k + __popcll(mask[u] & ((uint64_t(1) << lane) - 1));
      if (held[u] <= 0 && rank < total) {
        int lo = 0, hi = n - 1;   // the first place whose sum is above rank
        while (lo < hi) {
          const int mid = (lo + hi) >> 1;
          if (sums[mid] > rank) hi = mid;
          else lo = mid + 1;
        }
        int seq, entry;
        if (few) { seq = seqs[lo]; entry = firsts[lo]; }
        else { const Place p = place_at<FORK>(c, a, b, lo, owner); seq = p.seq; entry = p.first; }
        const int32_t page = (int32_t)(first + u * 64);
        c.row(seq)[entry + rank - (lo ? sums[lo - 1] : 0)] = page;
        c.ref[page] = 1;
      }
      k += __popcll(mask[u]);
    }
    found += all;
  }
  __syncthreads();
  // Lengths change here only.  A place reads the length of its own sequence, and of a source that nobody changes.
  for (int i = tid; i < n; i += kMapThreads) {
    Place p = few ? mine : place_at<FORK>(c, a, b, i, owner);
    if (p.seq >= 0 && p.need > 0 && sums[i] > found) {
      p.code = DCP_PLACE_FULL;
      if ((i ? sums[i - 1] : 0) < found) short_place = i;
    } else if (p.seq >= 0) {
      c.len[p.seq] = p.tokens;
    }
    status[i] = p.code;
  }
  __syncthreads();
  if (short_place >= 0) {
    const Place p = place_at<FORK>(c, a, b, short_place, owner);
    const int got = found - (short_place ? sums[short_place - 1] : 0);
    for (int k = tid; k < got; k += kMapThreads) {
      int32_t* entry = c.row(p.seq) + p.first + k;
      c.ref[*entry] = 0;
      *entry = -1;
    }
  }
}

// 16 bytes past the caches: new tokens are read once, pages are written once.
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
__device__ __forceinline__ u32x4 load16(const char* p) { return __builtin_nontemporal_load((const u32x4*)p); }
__device__ __forceinline__ void store16(char* p, u32x4 v) { __builtin_nontemporal_store(v, (u32x4*)p); }

// 16-byte chunks [first, last) of page `from` to page `to`, of one layer of k or v, by one workgroup of 256: chunk x is chunk x % head_chunks of
// (token, head) x / head_chunks.  Four in flight a lane.  SHARED: one page may be copied for many, and is read through the caches (64
// sequences forked from 64 drawn with repeats, over 4 layers: 56 us past them, 50 so; pages that move, each read once: 956 and 984).
template <bool SHARED>
__device__ __forceinline__ void copy_chunks(const KCache& c, char* base, int64_t st_p, int64_t st_t, int64_t st_h, int from, int to, int first, int last) {
  const char* src = base + from * st_p;
  char* dst = base + to * st_p;
  auto offset = [&](int x) {
    const int row = x >> c.log_head_chunks, t = c.heads.quot(row);
    return t * st_t + c.heads.rem(row, t) * st_h + (x & ((1 << c.log_head_chunks) - 1)) * 16;
  };
  int x = first + threadIdx.x;
  for (; x + 768 < last; x += 1024) {
    int64_t at[4];
    u32x4 v[4];
#pragma unroll
    for (int y = 0; y < 4; y++) { at[y] = offset(x + 256 * y); v[y] = SHARED ? *(const u32x4*)(src + at[y]) : load16(src + at[y]); }
#pragma unroll
    for (int y = 0; y < 4; y++) store16(dst + at[y], v[y]);
  }
  for (; x < last; x += 256) {
    const int64_t at = offset(x);
    store16(dst + at, SHARED ? *(const u32x4*)(src + at) : load16(src + at));
  }
}

// After take_kernel.  Of place i's units the first shares its whole pages, unit 1 + x copies a piece of the page being filled, x = 2 (layer pieces
// + piece) + (0: k, 1: v).
__global__ __launch_bounds__(256) void fork_kernel(KCache c, const int32_t* __restrict__ src, const int32_t* __restrict__ dst, int32_t n,
                                                   const int32_t* __restrict__ status, int32_t pieces) {
  const int64_t per_place = 1 + 2 * (int64_t)c.n_layers * pieces, units = n * per_place;
  for (int64_t unit = blockIdx.x; unit < units; unit += gridDim.x) {
    const int i = (int)quot64(unit, per_place);
    const int64_t y = unit - i * per_place;
    const int a = src[i], b = dst[i];
    if (a < 0 || status[i] != DCP_PLACE_OK) continue;
    const int len = c.length(a), whole = c.page.quot(len);
    const int32_t* from = c.row(a);
    int32_t* to = c.row(b);
    if (y == 0) {
      for (int p = threadIdx.x; p < whole; p += 256) {
        const int32_t page = from[p];
        to[p] = page;
        if (c.is_page(page)) atomicAdd(&c.ref[page], 1);
      }
      continue;
    }
    const int64_t x = (y - 1) >> 1, layer = quot64(x, pieces);
    const int first = (int)(x - layer * pieces) * kPieceChunks;
    const int last = min(first + kPieceChunks, c.page.rem(len, whole) * c.hkv << c.log_head_chunks);
    if (first >= last) continue;
    const int32_t page = from[whole], mine = to[whole];
    if (!c.is_page(page) || !c.is_page(mine)) continue;
    if (y & 1) copy_chunks<true>(c, c.k + layer * c.k_sl, c.k_sp, c.k_st, c.k_sh, page, mine, first, last);
    else copy_chunks<true>(c, c.v + layer * c.v_sl, c.v_sp, c.v_st, c.v_sh, page, mine, first, last);
  }
}

// One workgroup a place.  The length is taken by an exchange, so that a sequence that is named twice is freed once.
__global__ __launch_bounds__(256) void free_kernel(KCache c, const int32_t* __restrict__ seqs) {
  __shared__ int32_t taken;
  const int s = seqs ? seqs[blockIdx.x] : (int)blockIdx.x;
  if (!c.is_seq(s)) return;
  if (threadIdx.x == 0) taken = atomicExch(&c.len[s], 0);
  __syncthreads();
  const int held = c.pages_of(max(0, min(taken, c.max_len)));
  int32_t* row = c.row(s);
  for (int p = threadIdx.x; p < held; p += 256) {
    const int32_t page = row[p];
    row[p] = -1;
    if (c.is_page(page)) atomicSub(&c.ref[page], 1);
  }
}

// One workgroup: counts the pages in use (u), then lists the free ones before u and the used ones behind it, which are as many.  Bound by
// latency: page_ref is read twice, 8 192 pages at a time (the second time from the cache), once if there are no more, whose lists stay in LDS
// until they meet (a call in a graph, with a copy of the map: 240 pages 9.4 -> 9.2 us, 8 192 14.65 -> 14.3).
__global__ __launch_bounds__(kMapThreads) void list_moves_kernel(KCache c, Moves m, int32_t* __restrict__ counts) {
  constexpr int kOnce = kMapThreads * kScan;
  __shared__ int32_t wave_sum[kMapWaves], wave_high[kMapWaves], s_to[kOnce / 2], s_from[kOnce / 2];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const bool once = c.n_pages <= kOnce;
  int32_t held[kScan];
  auto scan = [&](int64_t first) {
#pragma unroll
    for (int u = 0; u < kScan; u++) held[u] = first + u * 64 < c.n_pages ? c.ref[first + u * 64] : 0;
  };
  int used = 0;
  for (int64_t base = 0; base < c.n_pages; base += kMapThreads * kScan) {
    scan(base + wave * (64 * kScan) + lane);
#pragma unroll
    for (int u = 0; u < kScan; u++) used += __popcll(__ballot(held[u] > 0));
  }
  if (lane == 0) wave_sum[wave] = used;
  __syncthreads();
  int n_used = 0;
#pragma unroll
  for (int w = 0; w < kMapWaves; w++) n_used += wave_sum[w];
  int holes = 0, high = 0;
  for (int64_t base = 0; base < c.n_pages; base += kMapThreads * kScan) {
    const int64_t first = base + wave * (64 * kScan) + lane;
    if (!once) scan(first);
    uint64_t hole[kScan], up[kScan];
    int h = 0, p = 0;
#pragma unroll
    for (int u = 0; u < kScan; u++) {
      const int64_t page = first + u * 64;
      hole[u] = __ballot(page < n_used && held[u] <= 0);
      up[u] = __ballot(page >= n_used && held[u] > 0);
      h += __popcll(hole[u]);
      p += __popcll(up[u]);
    }
    __syncthreads();
    if (lane == 0) { wave_sum[wave] = h; wave_high[wave] = p; }
    __syncthreads();
    int kh = holes, kp = high;   // of the waves before
#pragma unroll
    for (int w = 0; w < kMapWaves; w++) {
      if (w < wave) { kh += wave_sum[w]; kp += wave_high[w]; }
      holes += wave_sum[w];
      high += wave_high[w];
    }
    const uint64_t below = (uint64_t(1) << lane) - 1;
#pragma unroll
    for (int u = 0; u < kScan; u++) {
      const int64_t page = first + u * 64;
      if (page < c.n_pages) {
        if (page < n_used) {
          if (held[u] <= 0) {
            const int k = kh + __popcll(hole[u] & below);
            m.to[k] = (int32_t)page;
            if (once) s_to[k] = (int32_t)page;
          }
        } else if (held[u] > 0) {
          const int k = kp + __popcll(up[u] & below);
          m.from[k] = (int32_t)page;
          if (once) s_from[k] = (int32_t)page;
        } else {
          m.where[page] = -1;
        }
      }
      kh += __popcll(hole[u]);
      kp += __popcll(up[u]);
    }
  }
  __syncthreads();
  for (int k = tid; k < high; k += 4 * kMapThreads) {
    int32_t from[4], to[4];
#pragma unroll
    for (int x = 0; x < 4; x++)
      if (k + x * kMapThreads < high) {
        from[x] = once ? s_from[k + x * kMapThreads] : m.from[k + x * kMapThreads];
        to[x] = once ? s_to[k + x * kMapThreads] : m.to[k + x * kMapThreads];
      }
#pragma unroll
    for (int x = 0; x < 4; x++)
      if (k + x * kMapThreads < high) m.where[from[x]] = to[x];
  }
  if (tid == 0) {
    *m.count = high;
    counts[0] = n_used;
    counts[1] = high;
  }
}

// The first n_seqs workgroups renumber a row of the table each; the others share (page, layer, piece, k or v) among themselves.  No page, and
// no count, is both read and written: those that move lie at or behind u, where they go before it.  Bound by HBM.
__global__ __launch_bounds__(256) void move_kernel(KCache c, Moves m, const int32_t* __restrict__ counts, int32_t pieces) {
  if ((int)blockIdx.x < c.n_seqs) {
    const int s = blockIdx.x, held = c.pages_of(c.length(s)), n_used = counts[0];
    int32_t* row = c.row(s);
    for (int p = threadIdx.x; p < held; p += 256) {
      const int32_t page = row[p];
      if (c.is_page(page) && page >= n_used) {
        const int32_t to = m.where[page];
        if (to >= 0) row[p] = to;
      }
    }
    return;
  }
  const int64_t per_page = 2 * (int64_t)c.n_layers * pieces, units = *m.count * per_page;
  const int all = c.page.d * c.hkv << c.log_head_chunks;
  for (int64_t x = blockIdx.x - c.n_seqs; x < units; x += gridDim.x - c.n_seqs) {
    const int64_t k = quot64(x, per_page), y = x - k * per_page, layer = quot64(y >> 1, pieces);
    const int first = (int)((y >> 1) - layer * pieces) * kPieceChunks, last = min(first + kPieceChunks, all);
    const int from = m.from[k], to = m.to[k];
    if (y == 0 && threadIdx.x == 0) {
      c.ref[to] = c.ref[from];
      c.ref[from] = 0;
    }
    if (y & 1) copy_chunks<false>(c, c.v + layer * c.v_sl, c.v_sp, c.v_st, c.v_sh, from, to, first, last);
    else copy_chunks<false>(c, c.k + layer * c.k_sl, c.k_sp, c.k_st, c.k_sh, from, to, first, last);
  }
}

// A workgroup writes TOKENS tokens: their places in the cache are found by a thread each, then all threads copy, four chunks in flight.  HBM-bound
// where there are many (83 396 tokens of 4 KiB 111 us, 6.1 TB/s read and written); few take a workgroup each and are bound by the trips
// to memory: cu_new, seqs, seq_len, page_table, the tokens.
static constexpr int kCuInLds = 1024;   // entries of cu_new that are searched in LDS
template <int TOKENS>
__global__ __launch_bounds__(256) void append_kernel(KCache c, int32_t layer, const int32_t* __restrict__ seqs, const int32_t* __restrict__ cu,
                                                     int32_t n, const int32_t* __restrict__ status, NewTokens x) {
  __shared__ int32_t page_of[TOKENS], slot_of[TOKENS], s_cu[kCuInLds];
  const int64_t t0 = (int64_t)blockIdx.x * TOKENS;
  const bool in_lds = cu && n < kCuInLds;
  if (in_lds) {
    for (int y = threadIdx.x; y <= n; y += 256) s_cu[y] = cu[y];
    __syncthreads();
  }
  if (threadIdx.x < TOKENS) {
    const int64_t t = t0 + threadIdx.x;
    int page = -1, slot = 0;
    int i = -1, behind = 0;   // the token's place, and the tokens of it from this one on
    if (t < x.n) {
      if (!cu) {
        if (t < n) { i = (int)t; behind = 1; }
      } else {
        auto at = [&](int y) { return in_lds ? s_cu[y] : cu[y]; };
        if (t >= at(0) && t < at(n)) {
          int lo = 0, hi = n - 1;   // the last place that begins at or before t
          while (lo < hi) {
            const int mid = (lo + hi + 1) >> 1;
            if (at(mid) <= t) lo = mid;
            else hi = mid - 1;
          }
          i = lo;
          behind = (int)(at(lo + 1) - t);
        }
      }
    }
    if (i >= 0) {
      const int s = seqs ? seqs[i] : i, st = status ? status[i] : DCP_PLACE_OK;
      if (c.is_seq(s) && st == DCP_PLACE_OK) {
        const int pos = c.length(s) - behind;
        if (pos >= 0 && behind > 0) {
          const int p = c.page.quot(pos), entry = c.row(s)[p];
          if (c.is_page(entry)) { page = entry; slot = c.page.rem(pos, p); }
        }
      }
    }
    page_of[threadIdx.x] = page;
    slot_of[threadIdx.x] = slot;
  }
  __syncthreads();
  const int all = TOKENS * c.hkv << c.log_head_chunks;   // chunks of k; as many of v
  for (int y0 = threadIdx.x; y0 < all; y0 += 512) {
    u32x4 kv[2][2];
    char* to[2][2];
#pragma unroll
    for (int z = 0; z < 2; z++) {
      const int y = y0 + 256 * z;
      const int row = y >> c.log_head_chunks, off = (y & ((1 << c.log_head_chunks) - 1)) * 16;   // row: (token, head)
      const int t = c.heads.quot(row), h = c.heads.rem(row, t);
      to[z][0] = nullptr;
      if (y < all && page_of[t] >= 0) {
        const int64_t page = page_of[t], slot = slot_of[t];
        to[z][0] = c.k + layer * c.k_sl + page * c.k_sp + slot * c.k_st + h * c.k_sh + off;
        to[z][1] = c.v + layer * c.v_sl + page * c.v_sp + slot * c.v_st + h * c.v_sh + off;
        kv[z][0] = load16(x.k + (t0 + t) * x.k_st + h * x.k_sh + off);
        kv[z][1] = load16(x.v + (t0 + t) * x.v_st + h * x.v_sh + off);
      }
    }
#pragma unroll
    for (int z = 0; z < 2; z++)
      if (to[z][0]) {
        store16(to[z][0], kv[z][0]);
        store16(to[z][1], kv[z][1]);
      }
  }
}

// ------------------------------------------------------------------------------------------------ launches
void launch_take(bool fork, const KCache& c, const int32_t* a, const int32_t* b, int32_t n, int32_t* status, hipStream_t s) {
  if (!fork) hipLaunchKernelGGL(take_kernel<false>, dim3(1), dim3(kMapThreads), 0, s, c, a, b, n, status);
  else hipLaunchKernelGGL(take_kernel<true>, dim3(1), dim3(kMapThreads), 0, s, c, a, b, n, status);
}
void launch_fork(uint32_t grid, const KCache& c, const int32_t* src, const int32_t* dst, int32_t n, const int32_t* status, int32_t pieces, hipStream_t s) {
  hipLaunchKernelGGL(fork_kernel, dim3(grid), dim3(256), 0, s, c, src, dst, n, status, pieces);
}
void launch_free(uint32_t grid, const KCache& c, const int32_t* seqs, hipStream_t s) {
  hipLaunchKernelGGL(free_kernel, dim3(grid), dim3(256), 0, s, c, seqs);
}
void launch_list_moves(const KCache& c, const Moves& m, int32_t* counts, hipStream_t s) {
  hipLaunchKernelGGL(list_moves_kernel, dim3(1), dim3(kMapThreads), 0, s, c, m, counts);
}
void launch_move(uint32_t grid, const KCache& c, const Moves& m, const int32_t* counts, int32_t pieces, hipStream_t s) {
  hipLaunchKernelGGL(move_kernel, dim3(grid), dim3(256), 0, s, c, m, counts, pieces);
}
void launch_append(int32_t each, uint32_t grid, const KCache& c, int32_t layer, const int32_t* seqs, const int32_t* cu, int32_t n, const int32_t* status,
                   const NewTokens& x, hipStream_t s) {
  if (each == 1) hipLaunchKernelGGL(append_kernel<1>, dim3(grid), dim3(256), 0, s, c, layer, seqs, cu, n, status, x);
  else hipLaunchKernelGGL(append_kernel<4>, dim3(grid), dim3(256), 0, s, c, layer, seqs, cu, n, status, x);
}

}  // namespace dcp
