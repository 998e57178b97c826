// Where the tokens that dcp_cache_append and dcp_cache_read are handed lie in the cache.
#pragma once
#include "cache_internal.h"

namespace dcp {

static constexpr int kCuInLds = 1024;   // entries of cu_new that are searched in LDS

// cu_new in LDS where there are few entries; `s` has room for kCuInLds.  To be called by all of a workgroup of 256.
struct Begins {
  const int32_t *cu, *s;
  bool in_lds;
  __device__ __forceinline__ Begins(const int32_t* cu_new, int32_t n, int32_t* lds) : cu(cu_new), s(lds), in_lds(cu_new && n < kCuInLds) {
    if (in_lds) {
      for (int y = threadIdx.x; y <= n; y += 256) lds[y] = cu[y];
      __syncthreads();
    }
  }
  __device__ __forceinline__ int32_t at(int y) const { return in_lds ? s[y] : cu[y]; }
};

struct TokenPlace {
  int32_t page, slot;      // page -1: nowhere
  int32_t pos, first, behind;   // in its sequence; the place's first token in the packed ones; its tokens from this one on
};
__device__ __forceinline__ TokenPlace token_place(const KCache& c, const int32_t* seqs, const Begins& cu, int32_t n, const int32_t* status, int64_t t,
                                                  int64_t n_tokens) {
  TokenPlace p{-1, 0, -1, 0, 0};
  int i = -1;
  if (t < n_tokens) {
    if (!cu.cu) {
      if (t < n) { i = (int)t; p.first = i; p.behind = 1; }
    } else if (t >= cu.at(0) && t < cu.at(n)) {
      int lo = 0, hi = n - 1;   // the last place that begins at or before t
      while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (cu.at(mid) <= t) lo = mid;
        else hi = mid - 1;
      }
      i = lo;
      p.first = cu.at(lo);
      p.behind = (int)(cu.at(lo + 1) - t);
    }
  }
  if (i >= 0) {
    const int s = seqs ? seqs[i] : i, st = status ? status[i] : DCP_PLACE_OK;
    if (c.is_seq(s) && st == DCP_PLACE_OK) {
      const int pos = c.length(s) - p.behind;
      if (pos >= 0 && p.behind > 0) {
        const int q = c.page.quot(pos), entry = c.row(s)[q];
        p.pos = pos;
        if (c.is_page(entry)) { p.page = entry; p.slot = c.page.rem(pos, q); }
      }
    }
  }
  return p;
}

}  // namespace dcp
