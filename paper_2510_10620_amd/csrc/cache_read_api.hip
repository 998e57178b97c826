// The host's half of dcp_cache_read, as cache_api.hip is that of the other calls on a paged cache.
#include "cache_internal.h"

using namespace dcp;

extern "C" dcp_status_t dcp_cache_read(const dcp_cache_t* cache, int32_t layer, const int32_t* seqs, const int32_t* cu_new, int32_t n,
                                       const int32_t* status, void* k_out, int64_t k_st, int64_t k_sh, void* v_out, int64_t v_st,
                                       int64_t v_sh, int64_t n_tokens, void* stream) {
  KCache c;
  dcp_status_t st = pack_cache(cache, &c);
  if (st != DCP_OK) return st;
  if ((st = check_places(c, seqs, n)) != DCP_OK) return st;
  if (layer < 0 || layer >= c.n_layers) return fail(DCP_ERR_INVALID_ARG, "layer out of range");
  if (n_tokens < 0) return fail(DCP_ERR_INVALID_ARG, "n_tokens must not be negative");
  if (n_tokens > (1 << 25)) return fail(DCP_ERR_UNSUPPORTED, "dcp_cache_read covers at most 2^25 tokens");
  if (!is_aligned(cu_new, 4) || !is_aligned(status, 4)) return fail(DCP_ERR_INVALID_ARG, "cu_new or status is misaligned");
  if (n == 0 || n_tokens == 0) return DCP_OK;
  if ((st = check_rows("k_out", k_out, k_st, k_sh, cache)) != DCP_OK) return st;
  if ((st = check_rows("v_out", v_out, v_st, v_sh, cache)) != DCP_OK) return st;
  const int64_t e = c.io_bytes;
  if (rows_overlap(Rows{k_out, k_st * e, k_sh * e}, Rows{v_out, v_st * e, v_sh * e}, (int32_t)n_tokens, c.hkv, cache->d * e))
    return fail(DCP_ERR_INVALID_ARG, "k_out and v_out overlap");
  const ReadTokens x{(char*)k_out, (char*)v_out, k_st * e, k_sh * e, v_st * e, v_sh * e, n_tokens};
  ProfScope ps(DCP_K_CACHE, (hipStream_t)stream);
  const int32_t each = n_tokens <= 1024 ? 1 : 4;   // as in dcp_cache_append
  launch_read(each, (uint32_t)((n_tokens + each - 1) / each), c, layer, seqs, cu_new, n, status, x, (hipStream_t)stream);
  DCP_HIP_TRY(hipGetLastError());
  return DCP_OK;
}
