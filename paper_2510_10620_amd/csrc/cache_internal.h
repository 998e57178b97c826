// Host side of the calls on a paged cache: checks shared by cache.hip and paged_attn.hip.
#pragma once
#include <climits>
#include <string>

#include "kernels.h"
#include "paged.h"

namespace dcp {

// Validates the descriptor and packs it for the kernels.
dcp_status_t pack_cache(const dcp_cache_t* cache, KCache* out);
// n places, of sequences or (seqs NULL) the first n sequences of the cache
dcp_status_t check_places(const KCache& c, const int32_t* seqs, int32_t n);
// a tensor [tokens, heads, d] beside the cache
dcp_status_t check_rows(const char* name, const void* p, int64_t stride_t, int64_t stride_h, int32_t d);

}  // namespace dcp
