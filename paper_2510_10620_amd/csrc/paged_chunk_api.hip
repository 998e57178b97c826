// The host's half of dcp_paged_attn_chunk_fwd, as cache_api.hip is that of the other calls on a paged cache.
#include <algorithm>
#include <climits>
#include <cmath>

#include "cache_internal.h"

using namespace dcp;

// Rows of an item, by the rows that places have on average and by all rows of all KV heads; items that n places with n_tokens tokens between them can have.
static int32_t chunk_rows(int32_t n, int64_t n_tokens, int32_t group, int32_t hkv) {
  return n_tokens * group <= kFewRows * (int64_t)n || n_tokens * group * hkv <= kFewAll ? kFewItem : kChunkRows;
}
static int64_t chunk_items(int32_t n, int64_t n_tokens, int32_t group, int32_t rows) { return (n_tokens * group + rows - 1) / rows + n; }

static size_t chunk_bytes(int64_t items, int32_t rows, int32_t d) {
  return sizeof(int4) * (1 + kWorkers) + sizeof(ChunkJoin) * kWorkers + sizeof(ChunkItem) * (size_t)items + 2 * (size_t)kWorkers * rows * (sizeof(float2) + d * sizeof(float));
}

// What every call with up to n places and n_tokens tokens needs, so that a workspace for the largest batch does for smaller ones: where many places go by kFewItem, as many
// tokens of fewer places go by kChunkRows, whose parts take 8 times as much.
extern "C" size_t dcp_paged_attn_chunk_workspace_bytes(const dcp_cache_t* cache, int32_t n, int64_t n_tokens, int32_t hq) {
  if (!cache || n <= 0 || n_tokens <= 0 || n_tokens > (1 << 25) || hq <= 0 || cache->hkv <= 0 || cache->d <= 0 || hq % cache->hkv) return 0;
  const int32_t group = hq / cache->hkv;
  const int64_t few = std::min<int64_t>(n_tokens, std::max(kFewRows * (int64_t)n / group, (int64_t)kFewAll / hq));   // tokens that go by kFewItem at most
  size_t bytes = few ? chunk_bytes(chunk_items(n, few, group, kFewItem), kFewItem, cache->d) : 0;
  if (chunk_rows(1, n_tokens, group, cache->hkv) == kChunkRows) bytes = std::max(bytes, chunk_bytes(chunk_items(n, n_tokens, group, kChunkRows), kChunkRows, cache->d));
  return bytes;
}

extern "C" dcp_status_t dcp_paged_attn_chunk_fwd(const dcp_cache_t* cache, const dcp_paged_attn_t* args, const int32_t* cu_new, int64_t n_tokens,
                                                 void* workspace, size_t workspace_bytes, void* stream) {
  KCache c;
  dcp_status_t st = pack_cache(cache, &c);
  if (st != DCP_OK) return st;
  if (!args) return fail(DCP_ERR_INVALID_ARG, "args is NULL");
  const dcp_paged_attn_t& t = *args;
  if (cache->dtype != DCP_E4M3) return fail(DCP_ERR_UNSUPPORTED, "dcp_paged_attn_chunk_fwd covers caches of DCP_E4M3 (dcp_block_attn_fwd reads the others)");
  if ((st = check_places(c, t.seqs, t.n)) != DCP_OK) return st;
  if ((st = check_attn_args(c, t)) != DCP_OK) return st;
  if (n_tokens < 0) return fail(DCP_ERR_INVALID_ARG, "n_tokens must not be negative");
  if (n_tokens > (1 << 25)) return fail(DCP_ERR_UNSUPPORTED, "dcp_paged_attn_chunk_fwd covers at most 2^25 tokens");
  if (t.n == 0 || n_tokens == 0) return DCP_OK;
  if (!cu_new || !is_aligned(cu_new, 4)) return fail(DCP_ERR_INVALID_ARG, "cu_new is NULL or misaligned");
  if ((st = check_rows("q", t.q, t.q_stride_t, t.q_stride_h, cache)) != DCP_OK) return st;
  if ((st = check_rows("out", t.out, t.o_stride_t, t.o_stride_h, cache)) != DCP_OK) return st;
  if (!t.lse || !is_aligned(t.lse, 4)) return fail(DCP_ERR_INVALID_ARG, "lse is NULL or misaligned");
  if (!is_aligned(t.status, 4)) return fail(DCP_ERR_INVALID_ARG, "status is misaligned");
  if (n_tokens * t.hq > INT32_MAX - kChunkRows) return fail(DCP_ERR_UNSUPPORTED, "n_tokens x hq must be below 2^31 - 128");   // a row behind an item's is counted too
  const int32_t group = t.hq / c.hkv;
  const int32_t rows = chunk_rows(t.n, n_tokens, group, c.hkv), tile = rows == kChunkRows ? kChunkKeys : kPagedKeys;
  const int64_t items = chunk_items(t.n, n_tokens, group, rows), tiles = (c.max_len + kPagedKeys - 1) / kPagedKeys;
  if (items * tiles > INT32_MAX || items * tiles * c.hkv > INT32_MAX)
    return fail(DCP_ERR_UNSUPPORTED, "hkv x (tiles of 128 (few a place: 16) rows + n) x tiles of 32 tokens in a row of the table must be below 2^31");
  if (!workspace || workspace_bytes < dcp_paged_attn_chunk_workspace_bytes(cache, t.n, n_tokens, t.hq))
    return fail(DCP_ERR_WORKSPACE, "workspace is NULL or smaller than dcp_paged_attn_chunk_workspace_bytes");
  if (!is_aligned(workspace, 256)) return fail(DCP_ERR_WORKSPACE, "workspace must be 256-byte aligned");
  const int64_t e = c.io_bytes;
  if (rows_overlap(Rows{t.q, t.q_stride_t * e, t.q_stride_h * e}, Rows{t.out, t.o_stride_t * e, t.o_stride_h * e}, (int32_t)n_tokens, t.hq, cache->d * e))
    return fail(DCP_ERR_INVALID_ARG, "out overlaps q");
  c.k += t.layer * c.k_sl;   // the layer's
  c.v += t.layer * c.v_sl;
  c.k_scale += t.layer * c.layer_scales();
  c.v_scale += t.layer * c.layer_scales();
  const ChunkArgs a{(const char*)t.q, (char*)t.out, t.lse, t.seqs, t.status, cu_new, t.q_stride_t * e, t.q_stride_h * e, t.o_stride_t * e, t.o_stride_h * e,
                    n_tokens, t.n, t.window, t.sink, (int32_t)items, rows, tile, fast_div((uint32_t)group), t.softmax_scale * 1.44269504088896340736f};
  ChunkPlan plan;
  plan.head = (int4*)workspace;
  plan.starts = plan.head + 1;
  plan.joins = (ChunkJoin*)(plan.starts + kWorkers);
  plan.items = (ChunkItem*)(plan.joins + kWorkers);
  plan.o = (float*)(plan.items + items);
  plan.ml = (float2*)(plan.o + 2 * (size_t)kWorkers * rows * cache->d);
  ProfScope ps(DCP_K_PAGED_ATTN, (hipStream_t)stream);
  launch_chunk(cache->d, c, a, plan, (hipStream_t)stream);
  DCP_HIP_TRY(hipGetLastError());
  return DCP_OK;
}
