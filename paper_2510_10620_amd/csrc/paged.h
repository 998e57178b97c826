// The paged key-value cache as its kernels see it, and the index arithmetic that they share with the host.
#pragma once
#include <cstdint>

#include "dcp.h"

#if defined(__HIPCC__)
#define DCP_HD __host__ __device__ __forceinline__
#else
#define DCP_HD inline
#endif

namespace dcp {

// n / d for 0 <= n < 2^31 by a multiplication: with 2^s >= d > 2^(s-1) and m = floor(2^32 (2^s - d) / d) + 1,
// (floor(m n / 2^32) + n) >> s; the sum stays below 2^32.
struct FastDiv {
  uint32_t m, s, d;
  DCP_HD int32_t quot(int32_t n) const { return (int32_t)(((uint32_t)(((uint64_t)m * (uint32_t)n) >> 32) + (uint32_t)n) >> s); }
  DCP_HD int32_t rem(int32_t n, int32_t q) const { return n - q * (int32_t)d; }
};
inline FastDiv fast_div(uint32_t d) {
  uint32_t s = 0;
  while ((uint64_t(1) << s) < d) s++;
  return FastDiv{(uint32_t)(((uint64_t(1) << 32) * ((uint64_t(1) << s) - d)) / d + 1), s, d};
}

// x + y, cut at cap, for 0 <= x, y <= cap.  cap goes up to 2^30 + 1 (one more than the most pages of a cache): the sum fits into 32 bits without a
// sign only.  Sums of more terms come out alike in any order.
DCP_HD int32_t add_capped(int32_t x, int32_t y, int32_t cap) {
  const uint32_t sum = (uint32_t)x + (uint32_t)y;
  return sum < (uint32_t)cap ? (int32_t)sum : cap;
}

// dcp_cache_t by value, strides in bytes.
struct KCache {
  char *k, *v;
  int64_t k_sl, k_sp, k_st, k_sh, v_sl, v_sp, v_st, v_sh;
  int32_t *ref, *table, *len;
  int32_t n_layers, n_pages, hkv, n_seqs, max_pages, max_len;   // max_len: tokens that a row of the table has room for
  int32_t log_head_chunks;   // log2 of the 16-byte chunks of one token's head
  FastDiv page, heads;
  // in 8 bits: exponents of the scales, [layers, pages, blocks, KV heads]; else null
  uint8_t *k_scale, *v_scale;
  FastDiv block;             // tokens that share a scale
  int32_t blocks;            // of a page
  int32_t io_bytes;          // of a number beside the cache

  DCP_HD int32_t head_chunks() const { return 1 << log_head_chunks; }
  DCP_HD const int32_t* row(int32_t seq) const { return table + (int64_t)seq * max_pages; }
  DCP_HD int32_t* row(int32_t seq) { return table + (int64_t)seq * max_pages; }
  DCP_HD bool is_seq(int32_t seq) const { return (uint32_t)seq < (uint32_t)n_seqs; }
  DCP_HD bool is_page(int32_t p) const { return (uint32_t)p < (uint32_t)n_pages; }
  DCP_HD int32_t length(int32_t seq) const { const int32_t n = len[seq]; return n < 0 ? 0 : n > max_len ? max_len : n; }
  DCP_HD int64_t layer_scales() const { return (int64_t)n_pages * blocks * hkv; }
  // of KV head 0
  DCP_HD int64_t scale_at(int32_t p, int32_t slot) const { return ((int64_t)p * blocks + block.quot(slot)) * hkv; }
  DCP_HD int32_t pages_of(int32_t tokens) const { const int32_t q = page.quot(tokens); return q + (q * (int32_t)page.d < tokens); }
};

// The keys that a place of a batch sees, as tiles of `tile` tokens that start at multiples of it: those that hold tokens before `head`
// (the sink), then those that hold tokens from `lo` on; no tile twice.
struct KeyTiles {
  int32_t len, lo, head, n_head, first, count;   // first: number of the tile that follows the n_head ones
  DCP_HD KeyTiles(int32_t length, int32_t window, int32_t sink, int32_t tile) {
    len = length;
    lo = window > 0 && length > window ? length - window : 0;
    head = sink < lo ? sink : lo;
    n_head = (int32_t)(((uint32_t)head + tile - 1) / tile);
    first = lo / tile;
    if (first < n_head) first = n_head;
    count = n_head + (int32_t)(((uint32_t)length + tile - 1) / tile) - first;
    if (count < 1) count = 1;   // of an empty sequence: a tile without a key
  }
  DCP_HD int32_t tile_at(int32_t x) const { return x < n_head ? x : x - n_head + first; }
  DCP_HD bool sees(int32_t j) const { return (j < len) & ((j >= lo) | (j < head)); }
};

// What a place of dcp_paged_attn_chunk_fwd has: tokens [first, first + count) of the packed ones, the first of them at position pos of its sequence.
struct ChunkPlace {
  int32_t first, count, pos;
  // [begin, end): the place's rows by cu_new, of which those below n_tokens are there; the last of all is the sequence's last token
  DCP_HD ChunkPlace(int64_t begin, int64_t end, int64_t n_tokens, int32_t len) {
    const int64_t from = end - len > begin ? end - len : begin, a = from < 0 ? 0 : from, b = end < n_tokens ? end : n_tokens;
    count = b > a ? (int32_t)(b - a) : 0;
    first = (int32_t)(count ? a : 0);
    pos = (int32_t)(count ? len - (end - a) : 0);
  }
};
// The keys that the tokens at positions [lo, hi] of a sequence see, some of them or all, as tiles (see KeyTiles).  Positions are below 2^30, and so is what a
// larger window would cut off.
DCP_HD KeyTiles chunk_tiles(int32_t lo, int32_t hi, int32_t window, int32_t sink, int32_t tile) {
  return KeyTiles(hi + 1, window > 0 && window <= (1 << 30) ? window + (hi - lo) : 0, sink, tile);
}

// n / d by a 32-bit division where that is enough (a 64-bit one takes a few hundred instructions).
DCP_HD int64_t quot64(int64_t n, int64_t d) { return ((uint64_t)(n | d) >> 32) == 0 ? (int64_t)((uint32_t)n / (uint32_t)d) : n / d; }

// The tiles of a batch, one after the other, dealt to up to 2^LOG workers in contiguous shares: `each` tiles, and one more for the first `more`.
template <int LOG> struct Shares {
  int32_t each, more, workers;
  DCP_HD explicit Shares(int32_t total) {
    const bool all = total >= 1 << LOG;
    each = all ? total >> LOG : 1;
    more = all ? total & ((1 << LOG) - 1) : 0;
    workers = all ? 1 << LOG : total;
  }
  DCP_HD int32_t start(int32_t w) const { return each * w + (w < more ? w : more); }
  DCP_HD int32_t worker_of(int32_t t) const {
    const int32_t longer = (each + 1) * more;
    const bool in = t < longer;
    return (int32_t)((uint32_t)(in ? t : t - longer) / (uint32_t)(each + in)) + (in ? 0 : more);
  }
};

// A tensor [n, heads] of rows of `row` bytes, strides in bytes and positive.
struct Rows {
  const void* p;
  int64_t st, sh;
};
// Whether a row of x shares a byte with a row of y, both [n, heads].  With the same strides: rows (i, h) of x and (i + a, h + b) of y lie
// y - x + a st + b sh apart, and for every a (or every b, whichever are fewer) the nearest two b decide.  With others: whether the rows of the one
// begin before the other's end and the other way round, which tensors between whose rows the other's lie do as well.
inline bool rows_overlap(const Rows& x, const Rows& y, int32_t n, int32_t heads, int64_t row) {
  typedef __int128 Wide;   // strides may be anything
  const Wide apart = (Wide)(int64_t)((uintptr_t)y.p - (uintptr_t)x.p);
  if (apart >= (Wide)(n - 1) * x.st + (Wide)(heads - 1) * x.sh + row || -apart >= (Wide)(n - 1) * y.st + (Wide)(heads - 1) * y.sh + row) return false;
  if ((n > 1 && x.st != y.st) || (heads > 1 && x.sh != y.sh)) return true;
  const bool by_token = n <= heads;
  const int32_t outer = by_token ? n : heads, inner = by_token ? heads : n;
  const int64_t so = by_token ? x.st : x.sh, si = by_token ? x.sh : x.st;
  for (int64_t a = 1 - (int64_t)outer; a < outer; a++) {
    const Wide d = apart + (Wide)a * so;
    Wide b = -d / si;
    for (Wide near = b - 1; near <= b + 1; near++) {
      const Wide at = d + near * si;
      if (near > -inner && near < inner && at < row && -at < row) return true;
    }
  }
  return false;
}

}  // namespace dcp
