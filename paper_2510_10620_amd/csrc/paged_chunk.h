// What the kernels of the attention of several new tokens share.
#pragma once
#include "cache_internal.h"
#include "e4m3.h"

namespace dcp {

__device__ __forceinline__ ChunkPlace chunk_place(const KCache& c, const ChunkArgs& a, int i, int32_t* seq) {
  const int s = a.seqs ? a.seqs[i] : i, code = a.status ? a.status[i] : DCP_PLACE_OK;
  *seq = code == DCP_PLACE_OK && c.is_seq(s) ? s : -1;
  return *seq < 0 ? ChunkPlace(0, 0, 0, 0) : ChunkPlace(a.cu[i], a.cu[i + 1], a.n_tokens, c.length(s));
}

// The key tiles of all items and KV heads, dealt to the workers.
struct ChunkShares : Shares<kLogWorkers> {
  __device__ __forceinline__ explicit ChunkShares(int32_t total) : Shares<kLogWorkers>(total) {}
  // The worker that a workgroup is.  Workgroups go to the 8 XCDs round-robin: each XCD gets as many workers, with neighbouring shares, so that its L2 serves their keys; a workgroup
  // that is left over is one past the last, each another.  (With 64 an XCD whatever their number, few shares lay on few XCDs: one sequence of 300 tokens, 32/8 heads of 128, 45 to 90 new ones
  // 24.3 -> 21.4, 27.4 -> 22.1, 28.8 -> 23.5 us.)
  __device__ __forceinline__ int worker(int block) const {
    const int x = block & 7, y = block >> 3, each_xcd = (workers + 7) >> 3;
    return y < each_xcd ? x * each_xcd + y : 8 * each_xcd + x * (kWorkers / 8 - each_xcd) + y - each_xcd;
  }
};

// Whether the walk's workgroups make the plan for themselves.
inline bool plans_itself(const ChunkArgs& a) { return a.rows == kFewItem && a.max_items <= kOwnItems; }

// A row of an item, as its lanes hold it.
struct ChunkRow {
  bool real;
  int32_t pos, token, head;   // token: of the packed ones; head: query head
  int32_t low, head_end;      // its keys: [0, head_end) and [low, pos]
  // r: of the item's place and KV head
  __device__ __forceinline__ ChunkRow(const ChunkArgs& a, int hk, int32_t first, int32_t pos0, int32_t end, int32_t r) {
    const int32_t at = min(r, end - 1), t = a.group.quot(at);
    real = r < end;
    pos = pos0 + t;
    token = first + t;
    head = hk * (int)a.group.d + at - t * (int)a.group.d;
    low = a.window > 0 ? max(0, pos + 1 - a.window) : 0;
    head_end = min(a.sink, low);
  }
  __device__ __forceinline__ bool sees(int j) const { return (j <= pos) & ((j >= low) | (j < head_end)); }
};

// What is not finite among the values of keys that not every row of an item sees, added to the rows that see it: straight into memory, by the lane that wrote the
// number before (mine(d): whether it is this lane; add(d, x)).  Rare.
template <int D, typename Mine, typename Add>
__device__ __forceinline__ void add_not_finite(const KCache& c, const int32_t* table, int hk, const ChunkRow& row, int from, int to, Mine mine, Add add) {
  const int lane = threadIdx.x & 63;
  for (int j = from; j < to; j++) {
    const int32_t p = c.page.quot(j), page = table[p], slot = c.page.rem(j, p);
    if (!c.is_page(page)) continue;
    const char* v = c.v + page * c.v_sp + slot * c.v_st + hk * c.v_sh;
    const uint32_t scale = c.v_scale[c.scale_at(page, slot) + hk];
    const bool sees = row.real & row.sees(j);
    for (int d0 = 0; d0 < D; d0 += 64) {
      const uint32_t code = d0 + lane < D ? *(const uint8_t*)(v + d0 + lane) : 0u;
      const float number = __uint_as_float(e4m3_to_bf16x2<false>(code, scale_factor(scale)) << 16);
      for (uint64_t rest = __ballot((not_finite(code, scale) & 0x80u) != 0); rest; rest &= rest - 1) {
        const int at = __ffsll((unsigned long long)rest) - 1;
        const float x = __shfl(number, at);
        if (sees && mine(d0 + at)) add(d0 + at, x);
      }
    }
  }
}
template <typename IO> __device__ __forceinline__ void add_to(char* p, float x) {
  if constexpr (sizeof(IO) == 4) *(float*)p += x;
  else *(uint16_t*)p = f32_to_bf16(bf16_to_f32(*(const uint16_t*)p) + x);
}
__device__ __forceinline__ float lse_of(float m2, float l) { return l == 0.f ? -INFINITY : (m2 == -INFINITY ? 0.f : m2) * 0.6931471805599453f + logf(l); }

}  // namespace dcp
