// The host's half of the calls on a paged key-value cache: checks, sizes of launches, workspaces.  No kernel is here, so that this file is built
// for the CPU with sanitizers too.
#include <algorithm>
#include <climits>
#include <cmath>

#include "cache_internal.h"

using namespace dcp;

namespace dcp {

// Strides in bytes, and the pieces that the calls copy, are counted in 64 bits: no stride beyond 2^58 elements (2^60 bytes), no more than 2^16 layers
// (of up to 2^30 pages of 2^16 pieces of k and of v).
static constexpr int64_t kMostStride = int64_t(1) << 58;
static constexpr int32_t kMostLayers = 1 << 16;

static bool aligned(const void* p, uintptr_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }

// a tensor [tokens, heads, d] beside the cache
static dcp_status_t check_rows(const char* name, const void* p, int64_t stride_t, int64_t stride_h, int32_t d) {
  if (!p) return fail(DCP_ERR_INVALID_ARG, std::string(name) + " is NULL");
  if (!aligned(p, 16)) return fail(DCP_ERR_INVALID_ARG, std::string(name) + " must be 16-byte aligned");
  if (stride_h < d || stride_t < d || stride_h % 8 || stride_t % 8)
    return fail(DCP_ERR_INVALID_ARG, std::string(name) + ": strides must be >= d and multiples of 8 elements");
  if (std::max(stride_t, stride_h) > kMostStride) return fail(DCP_ERR_UNSUPPORTED, std::string(name) + ": strides of at most 2^58 elements");
  return DCP_OK;
}

// Validates the descriptor and packs it for the kernels.
static dcp_status_t pack_cache(const dcp_cache_t* cache, KCache* out) {
  if (!cache) return fail(DCP_ERR_INVALID_ARG, "cache is NULL");
  const dcp_cache_t& c = *cache;
  if (c.n_layers <= 0 || c.n_pages <= 0 || c.page_size <= 0 || c.hkv <= 0 || c.d <= 0 || c.n_seqs <= 0 || c.max_pages <= 0)
    return fail(DCP_ERR_INVALID_ARG, "n_layers, n_pages, page_size, hkv, d, n_seqs, max_pages must be positive");
  if (c.dtype != DCP_BF16 && c.dtype != DCP_F32) return fail(DCP_ERR_UNSUPPORTED, "dtype must be DCP_BF16 or DCP_F32");
  if (c.d != 32 && c.d != 64 && c.d != 128) return fail(DCP_ERR_UNSUPPORTED, "head_dim of a cache must be 32, 64 or 128");
  if (c.n_seqs > DCP_CACHE_MAX_SEQS) return fail(DCP_ERR_UNSUPPORTED, "a cache holds at most " + std::to_string(DCP_CACHE_MAX_SEQS) + " sequences");
  if (c.n_layers > kMostLayers) return fail(DCP_ERR_UNSUPPORTED, "a cache holds at most 65 536 layers");
  if (c.n_pages > (1 << 30)) return fail(DCP_ERR_UNSUPPORTED, "a cache holds at most 2^30 pages");
  if ((int64_t)c.max_pages * c.page_size > (1 << 30)) return fail(DCP_ERR_UNSUPPORTED, "max_pages * page_size must be at most 2^30");
  const int32_t e = c.dtype == DCP_BF16 ? 2 : 4;
  if ((int64_t)c.page_size * c.hkv * (c.d * e / 16) > (1 << 26)) return fail(DCP_ERR_UNSUPPORTED, "a page holds at most 1 GiB of keys");
  struct { const char* name; const void* p; int64_t l, page, t, h; } kv[2] = {{"k", c.k, c.k_stride_l, c.k_stride_p, c.k_stride_t, c.k_stride_h},
                                                                              {"v", c.v, c.v_stride_l, c.v_stride_p, c.v_stride_t, c.v_stride_h}};
  for (auto& x : kv) {
    if (!x.p || !aligned(x.p, 16)) return fail(DCP_ERR_INVALID_ARG, std::string(x.name) + " of the cache is NULL or not 16-byte aligned");
    if (x.l < c.d || x.page < c.d || x.t < c.d || x.h < c.d || x.l % 8 || x.page % 8 || x.t % 8 || x.h % 8)
      return fail(DCP_ERR_INVALID_ARG, std::string(x.name) + " of the cache: strides must be >= d and multiples of 8 elements");
    if (std::max(std::max(x.l, x.page), std::max(x.t, x.h)) > kMostStride)
      return fail(DCP_ERR_UNSUPPORTED, std::string(x.name) + " of the cache: strides of at most 2^58 elements");
  }
  if (!c.page_ref || !c.page_table || !c.seq_len || !aligned(c.page_ref, 4) || !aligned(c.page_table, 4) || !aligned(c.seq_len, 4))
    return fail(DCP_ERR_INVALID_ARG, "page_ref, page_table or seq_len is NULL or misaligned");
  KCache k{};
  k.k = (char*)c.k; k.v = (char*)c.v;
  k.k_sl = c.k_stride_l * e; k.k_sp = c.k_stride_p * e; k.k_st = c.k_stride_t * e; k.k_sh = c.k_stride_h * e;
  k.v_sl = c.v_stride_l * e; k.v_sp = c.v_stride_p * e; k.v_st = c.v_stride_t * e; k.v_sh = c.v_stride_h * e;
  k.ref = c.page_ref; k.table = c.page_table; k.len = c.seq_len;
  k.n_layers = c.n_layers; k.n_pages = c.n_pages; k.hkv = c.hkv; k.n_seqs = c.n_seqs; k.max_pages = c.max_pages;
  k.max_len = c.max_pages * c.page_size;
  for (k.log_head_chunks = 2; (16 << k.log_head_chunks) < c.d * e; k.log_head_chunks++) {}
  k.page = fast_div((uint32_t)c.page_size);
  k.heads = fast_div((uint32_t)c.hkv);
  *out = k;
  return DCP_OK;
}

// n places, of sequences or (seqs NULL) the first n sequences of the cache
static dcp_status_t check_places(const KCache& c, const int32_t* seqs, int32_t n) {
  if (n < 0) return fail(DCP_ERR_INVALID_ARG, "n must not be negative");
  if (n > DCP_CACHE_MAX_SEQS) return fail(DCP_ERR_UNSUPPORTED, "a call has at most " + std::to_string(DCP_CACHE_MAX_SEQS) + " places");
  if (!seqs && n > c.n_seqs) return fail(DCP_ERR_INVALID_ARG, "seqs is NULL and n is more than the cache's sequences");
  if (!aligned(seqs, 4)) return fail(DCP_ERR_INVALID_ARG, "seqs is misaligned");
  return DCP_OK;
}

static size_t moves_bytes(int32_t n_pages) { return 4 * (64 + 2 * (size_t)n_pages + 2); }   // count, from and to (n_pages / 2 + 1 each), where

// Items are taken whole, so that nothing is to be joined, where a workgroup each is enough and none can have more than so many tiles a wave:
// short sequences (or windows) in a table that has no room for more.  Whole and cut, us: one sequence of 30 tokens, 8 KV heads 7.5 and 13.6, of
// 300 tokens 12.6 and 12.8; 64 of 90 13.6 and 20.1, of 380 27.5 and 29.0; 16 of 380, 2 KV heads 15.4 and 13.4; with one more
// round 16 of 500 18.9 and 16.7.  Where they nearly fill the chip, cutting gains little and costs the joins and a start in the middle: 200 of 150
// tokens, 8 KV heads 33 and 42, 256 of 1 to 200 34 and 41, of 200 44 and 46, 64 of 1 to 700 36.5 and 34; with 160 items fewer 40 of 1 to 700 33 and 27.
static constexpr int kWholeRounds = 3, kWholeRoundsFull = 8, kFullItems = kWorkers * 3 / 4;

// How the query heads are taken: see PagedArgs.
struct Sets {
  int32_t per_kv, heads, abreast, log_abreast;
  int64_t groups;
  size_t bytes;   // of the workspace
};
static Sets sets_of(int32_t hkv, int32_t hq, int32_t d, int most_abreast) {
  const int32_t group = hq / hkv;
  Sets s;
  s.per_kv = (group - 1) / kSetHeads + 1;   // group up to 2^31 - 1
  s.heads = std::min(group, kSetHeads);
  const int64_t sets = (int64_t)hkv * s.per_kv;
  s.log_abreast = 0;
  while (2 << s.log_abreast <= most_abreast && sets % (2 << s.log_abreast) == 0) s.log_abreast++;
  s.abreast = 1 << s.log_abreast;
  s.groups = sets / s.abreast;
  s.bytes = kWorkers * (sizeof(int4) + 2 * (size_t)s.abreast * s.heads * (sizeof(float2) + d * sizeof(float)));
  return s;
}

}  // namespace dcp

extern "C" dcp_status_t dcp_cache_reserve(const dcp_cache_t* cache, const int32_t* seqs, const int32_t* n_new, int32_t n,
                                          int32_t* status, void* stream) {
  KCache c;
  dcp_status_t st = pack_cache(cache, &c);
  if (st != DCP_OK) return st;
  if ((st = check_places(c, seqs, n)) != DCP_OK) return st;
  if (n == 0) return DCP_OK;
  if (!status || !aligned(status, 4) || !aligned(n_new, 4)) return fail(DCP_ERR_INVALID_ARG, "status is NULL, or status or n_new misaligned");
  ProfScope ps(DCP_K_CACHE, (hipStream_t)stream);
  launch_take(false, c, seqs, n_new, n, status, (hipStream_t)stream);
  DCP_HIP_TRY(hipGetLastError());
  return DCP_OK;
}

extern "C" dcp_status_t dcp_cache_append(const dcp_cache_t* cache, int32_t layer, const int32_t* seqs, const int32_t* cu_new, int32_t n,
                                         const int32_t* status, const void* k_new, int64_t k_st, int64_t k_sh, const void* v_new,
                                         int64_t v_st, int64_t v_sh, int64_t n_tokens, void* stream) {
  KCache c;
  dcp_status_t st = pack_cache(cache, &c);
  if (st != DCP_OK) return st;
  if ((st = check_places(c, seqs, n)) != DCP_OK) return st;
  if (layer < 0 || layer >= c.n_layers) return fail(DCP_ERR_INVALID_ARG, "layer out of range");
  if (n_tokens < 0) return fail(DCP_ERR_INVALID_ARG, "n_tokens must not be negative");
  if (n_tokens > (1 << 25)) return fail(DCP_ERR_UNSUPPORTED, "dcp_cache_append covers at most 2^25 tokens");   // 2^31 threads; a grid ends below 2^32
  if (!aligned(cu_new, 4) || !aligned(status, 4)) return fail(DCP_ERR_INVALID_ARG, "cu_new or status is misaligned");
  if (n == 0 || n_tokens == 0) return DCP_OK;
  if ((st = check_rows("k_new", k_new, k_st, k_sh, cache->d)) != DCP_OK) return st;
  if ((st = check_rows("v_new", v_new, v_st, v_sh, cache->d)) != DCP_OK) return st;
  const int64_t e = cache->dtype == DCP_BF16 ? 2 : 4;
  const NewTokens x{(const char*)k_new, (const char*)v_new, k_st * e, k_sh * e, v_st * e, v_sh * e, n_tokens};
  ProfScope ps(DCP_K_CACHE, (hipStream_t)stream);
  // Up to four tokens a CU a workgroup each, else four in one.  In a graph, us, with one / four: tokens of 4 KiB, 64 2.95 / 3.44, 1 024 3.7 / 3.9,
  // 2 048 4.3 / 4.4, 4 096 8.4 / 7.2, 32 768 54 / 39; of 512 bytes, 64 2.94 / 2.86, 1 024 3.25 / 3.0, 8 192 7.8 / 3.8.  83 396 of 4 KiB in
  // 2 / 4 / 8 / 16: 123 / 124 / 130 / 134 with the reserve and the map's reset.
  const int32_t each = n_tokens <= 1024 ? 1 : 4;
  launch_append(each, (uint32_t)((n_tokens + each - 1) / each), c, layer, seqs, cu_new, n, status, x, (hipStream_t)stream);
  DCP_HIP_TRY(hipGetLastError());
  return DCP_OK;
}

extern "C" dcp_status_t dcp_cache_fork(const dcp_cache_t* cache, const int32_t* src, const int32_t* dst, int32_t n, int32_t* status,
                                       void* stream) {
  KCache c;
  dcp_status_t st = pack_cache(cache, &c);
  if (st != DCP_OK) return st;
  if ((st = check_places(c, src, n)) != DCP_OK) return st;
  if (n == 0) return DCP_OK;
  if (!src || !dst || !status || !aligned(dst, 4) || !aligned(status, 4)) return fail(DCP_ERR_INVALID_ARG, "src, dst or status is NULL or misaligned");
  const int pieces = pieces_of(c);
  hipStream_t s = (hipStream_t)stream;
  ProfScope ps(DCP_K_CACHE, s);
  launch_take(true, c, src, dst, n, status, s);
  DCP_HIP_TRY(hipGetLastError());
  const int64_t units = n * (1 + 2 * (int64_t)c.n_layers * pieces);
  launch_fork((uint32_t)std::min<int64_t>(units, kCopyWorkers), c, src, dst, n, status, pieces, s);
  DCP_HIP_TRY(hipGetLastError());
  return DCP_OK;
}

extern "C" dcp_status_t dcp_cache_free(const dcp_cache_t* cache, const int32_t* seqs, int32_t n, void* stream) {
  KCache c;
  dcp_status_t st = pack_cache(cache, &c);
  if (st != DCP_OK) return st;
  if ((st = check_places(c, seqs, n)) != DCP_OK) return st;
  if (n == 0) return DCP_OK;
  ProfScope ps(DCP_K_CACHE, (hipStream_t)stream);
  launch_free((uint32_t)n, c, seqs, (hipStream_t)stream);
  DCP_HIP_TRY(hipGetLastError());
  return DCP_OK;
}

extern "C" size_t dcp_cache_workspace_bytes(const dcp_cache_t* cache) {
  return cache && cache->n_pages > 0 ? moves_bytes(cache->n_pages) : 0;
}

extern "C" dcp_status_t dcp_cache_compact(const dcp_cache_t* cache, int32_t* counts, void* workspace, size_t workspace_bytes, void* stream) {
  KCache c;
  dcp_status_t st = pack_cache(cache, &c);
  if (st != DCP_OK) return st;
  if (!counts || !aligned(counts, 4)) return fail(DCP_ERR_INVALID_ARG, "counts is NULL or misaligned");
  if (!workspace || workspace_bytes < moves_bytes(c.n_pages)) return fail(DCP_ERR_WORKSPACE, "workspace is NULL or smaller than dcp_cache_workspace_bytes");
  if (!aligned(workspace, 256)) return fail(DCP_ERR_WORKSPACE, "workspace must be 256-byte aligned");
  int32_t* w = (int32_t*)workspace;
  const int32_t half = c.n_pages / 2 + 1;
  const Moves m{w, w + 64, w + 64 + half, w + 64 + 2 * half};
  hipStream_t s = (hipStream_t)stream;
  ProfScope ps(DCP_K_CACHE, s);
  launch_list_moves(c, m, counts, s);
  DCP_HIP_TRY(hipGetLastError());
  const int pieces = pieces_of(c);
  const int64_t most = std::min<int64_t>((c.n_pages / 2 + 1) * (2 * (int64_t)c.n_layers * pieces), kCopyWorkers);
  launch_move((uint32_t)(c.n_seqs + most), c, m, counts, pieces, s);
  DCP_HIP_TRY(hipGetLastError());
  return DCP_OK;
}

extern "C" size_t dcp_paged_attn_workspace_bytes(const dcp_cache_t* cache, int32_t n, int32_t hq) {
  if (!cache || n <= 0 || hq <= 0 || cache->hkv <= 0 || cache->d <= 0) return 0;
  return hq % cache->hkv ? 0 : sets_of(cache->hkv, hq, cache->d, kPagedWaves).bytes;
}

extern "C" dcp_status_t dcp_paged_attn_fwd(const dcp_cache_t* cache, const dcp_paged_attn_t* args, void* workspace, size_t workspace_bytes,
                                           void* stream) {
  KCache c;
  dcp_status_t st = pack_cache(cache, &c);
  if (st != DCP_OK) return st;
  if (!args) return fail(DCP_ERR_INVALID_ARG, "args is NULL");
  const dcp_paged_attn_t& t = *args;
  if ((st = check_places(c, t.seqs, t.n)) != DCP_OK) return st;
  if (t.hq <= 0) return fail(DCP_ERR_INVALID_ARG, "hq must be positive");
  if (t.hq % c.hkv != 0) return fail(DCP_ERR_UNSUPPORTED, "hq must be a multiple of hkv");
  if (t.layer < 0 || t.layer >= c.n_layers) return fail(DCP_ERR_INVALID_ARG, "layer out of range");
  if (!(t.softmax_scale > 0.f) || !std::isfinite(t.softmax_scale)) return fail(DCP_ERR_INVALID_ARG, "softmax_scale must be positive and finite");
  if (t.window < 0 || t.sink < 0) return fail(DCP_ERR_INVALID_ARG, "window and sink must not be negative");
  if (t.n == 0) return DCP_OK;
  if ((st = check_rows("q", t.q, t.q_stride_t, t.q_stride_h, cache->d)) != DCP_OK) return st;
  if ((st = check_rows("out", t.out, t.o_stride_t, t.o_stride_h, cache->d)) != DCP_OK) return st;
  if (!t.lse || (reinterpret_cast<uintptr_t>(t.lse) & 3u)) return fail(DCP_ERR_INVALID_ARG, "lse is NULL or misaligned");
  if (reinterpret_cast<uintptr_t>(t.status) & 3u) return fail(DCP_ERR_INVALID_ARG, "status is misaligned");
  if (!workspace || workspace_bytes < dcp_paged_attn_workspace_bytes(cache, t.n, t.hq))
    return fail(DCP_ERR_WORKSPACE, "workspace is NULL or smaller than dcp_paged_attn_workspace_bytes");
  if (reinterpret_cast<uintptr_t>(workspace) & 255u) return fail(DCP_ERR_WORKSPACE, "workspace must be 256-byte aligned");
  const int64_t e = cache->dtype == DCP_BF16 ? 2 : 4;
  if (rows_overlap(Rows{t.q, t.q_stride_t * e, t.q_stride_h * e}, Rows{t.out, t.o_stride_t * e, t.o_stride_h * e}, t.n, t.hq, cache->d * e))
    return fail(DCP_ERR_INVALID_ARG, "out overlaps q");
  // Whole items: the most tiles that one can have, as far as the host knows, over the waves that take them in turn
  const int tile = cache->dtype == DCP_F32 ? 16 : 32;
  const int64_t most = ((t.window > 0 ? std::min<int64_t>(c.max_len, (int64_t)t.window + t.sink + 2 * tile) : c.max_len) + tile - 1) / tile;
  Sets sets = sets_of(c.hkv, t.hq, cache->d, kPagedWaves);
  if (sets.groups * sets.abreast > (1 << 12)) return fail(DCP_ERR_UNSUPPORTED, "dcp_paged_attn_fwd covers at most 4 096 sets of 16 query heads on one KV head");
  bool whole = false;
  for (int abreast = 1; abreast <= sets.abreast && !whole; abreast *= 2) {
    const Sets x = sets_of(c.hkv, t.hq, cache->d, abreast);
    whole = t.n * x.groups <= kWorkers && most <= (t.n * x.groups > kFullItems ? kWholeRoundsFull : kWholeRounds) * (kPagedWaves / x.abreast);
    if (whole) sets = x;
  }
  if (t.n * (int64_t)((c.max_len + tile - 1) / tile) * sets_of(c.hkv, t.hq, cache->d, 1).groups > INT32_MAX)
    return fail(DCP_ERR_UNSUPPORTED, "n x hkv x sets of 16 query heads on one KV head x tiles of 32 (fp32: 16) tokens in a row of the table must be below 2^31");
  c.k += t.layer * c.k_sl;   // the layer's
  c.v += t.layer * c.v_sl;
  const PagedArgs a{(const char*)t.q, (char*)t.out, t.lse, t.seqs, t.status, t.q_stride_t * e, t.q_stride_h * e, t.o_stride_t * e, t.o_stride_h * e,
                    t.n, t.hq / c.hkv, t.window, t.sink, sets.per_kv, sets.heads, sets.abreast, sets.log_abreast, (int32_t)sets.groups, whole,
                    t.softmax_scale * 1.44269504088896340736f};
  PagedParts parts;
  parts.joins = (int4*)workspace;
  parts.o = (float*)(parts.joins + kWorkers);
  parts.ml = (float2*)(parts.o + 2 * (size_t)kWorkers * sets.abreast * sets.heads * cache->d);
  parts.by_item = t.n * sets.groups <= kWorkers;
  hipStream_t s = (hipStream_t)stream;
  ProfScope ps(DCP_K_PAGED_ATTN, s);
  launch_paged_attn(cache->dtype, cache->d, whole ? (uint32_t)(a.n * a.groups) : kWorkers, c, a, parts, s);
  DCP_HIP_TRY(hipGetLastError());
  return DCP_OK;
}
