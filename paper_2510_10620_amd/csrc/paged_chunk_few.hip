// Attention of the last tokens of every sequence over a paged key-value cache in 8 bits, where they are few: tokens to be verified.
#include "mfma_common.h"
#include "paged_chunk.h"
#include "paged_tile8.h"

using namespace dcp;

namespace dcp {

namespace {

// The plan, as a workgroup of the walk makes it for itself where there are at most kOwnItems items (and so places): a launch less than with chunk_plan_kernel, whose records take
// as many trips to memory to read as the places themselves (whole calls in a graph, us: the case below 38.7 -> 35.4, 4 sequences of up to 900 tokens, fp32, D 64 15.8 -> 12.3; with keys in LDS,
// where the walk became 18 us longer on 1 130, the launch stays).
struct OwnPlan {
  int4 place[kOwnItems];   // sequence, first token, its position, rows
  int4 item[kOwnItems];    // place, first row, key tiles, those of the items before
  int32_t upto[kOwnItems], wave_sum[2][4], start;
};
struct ChunkShare {
  int n_items, tiles, w, hk, item, t0, left;
  // What worker w, as which the workgroup goes, has; left 0: nothing.  For all of a workgroup of 256; plan.joins[w] becomes "nothing to join".
  __device__ __forceinline__ ChunkShare(const KCache& c, const ChunkArgs& a, const ChunkPlan& plan, OwnPlan& own) : hk(0), item(0), t0(0), left(0) {
    const int tid = threadIdx.x;
    if (a.max_items > kOwnItems) {
      const int4 head = *plan.head;
      n_items = uni(head.x);
      tiles = uni(head.y);
      const ChunkShares sh(tiles * c.hkv);
      w = sh.worker(blockIdx.x);
      if (w >= sh.workers) return;
      const int4 start = plan.starts[w];
      hk = uni(start.x);
      item = uni(start.y);
      t0 = uni(start.z);
      left = sh.start(w + 1) - sh.start(w);
      return;
    }
    auto sums = [&](int x, int which, int* total) {   // inclusive, over the workgroup
      const int lane = tid & 63, wave = tid >> 6;
#pragma unroll
      for (int o = 1; o < 64; o <<= 1) {
        const int y = __shfl_up(x, o);
        if (lane >= o) x += y;
      }
      if (lane == 63) own.wave_sum[which][wave] = x;
      __syncthreads();
      *total = 0;
#pragma unroll
      for (int y = 0; y < 4; y++) {
        if (y < wave) x += own.wave_sum[which][y];
        *total += own.wave_sum[which][y];
      }
      return x;
    };
    int mine = 0;
    if (tid < a.n) {
      int32_t seq;
      const ChunkPlace p = chunk_place(c, a, tid, &seq);
      own.place[tid] = make_int4(seq, p.first, p.pos, p.count * (int)a.group.d);
      mine = (int)min(((int64_t)p.count * a.group.d + a.rows - 1) / a.rows, (int64_t)a.max_items);   // what is beyond max_items is left out, as by chunk_plan_kernel
    }
    const int upto = min(sums(mine, 0, &n_items), a.max_items);
    if (tid < a.n) own.upto[tid] = upto;
    n_items = uni(min(n_items, a.max_items));
    __syncthreads();
    int count = 0;
    if (tid < n_items) {
      int lo = 0, hi = a.n - 1;   // the first place whose sum is above the item
      while (lo < hi) {
        const int mid = (lo + hi) >> 1;
        if (own.upto[mid] > tid) hi = mid;
        else lo = mid + 1;
      }
      const int4 p = own.place[lo];
      const int row0 = (tid - (lo ? own.upto[lo - 1] : 0)) * a.rows;
      count = chunk_tiles(p.z + a.group.quot(row0), p.z + a.group.quot(min(row0 + a.rows, p.w) - 1), a.window, a.sink, a.tile).count;
      own.item[tid] = make_int4(lo, row0, count, 0);
    }
    const int before = sums(count, 1, &tiles) - count;
    tiles = uni(tiles);
    const ChunkShares sh(tiles * c.hkv);
    w = sh.worker(blockIdx.x);
    if (tid == 0) plan.joins[w] = ChunkJoin{0, 0, -1, 0, 0, 0, 0, 0};
    if (w >= sh.workers) return;
    const int at = sh.start(w);
    hk = uni((int)((uint32_t)at / (uint32_t)tiles));
    const int rel = at - hk * tiles;
    if (tid < n_items) {
      own.item[tid].w = before;
      if (before <= rel && rel < before + count) own.start = tid;   // one: items have a tile or more
    }
    __syncthreads();
    item = uni(own.start);
    t0 = rel - uni(own.item[item].w);
    left = sh.start(w + 1) - at;
  }
  __device__ __forceinline__ ChunkItem at(const ChunkArgs& a, const ChunkPlan& plan, const OwnPlan& own, int x) const {
    ChunkItem it;
    if (a.max_items > kOwnItems) {
      it = plan.items[x];
    } else {
      const int4 i = own.item[x], p = own.place[i.x];
      it = ChunkItem{p.x, p.y, p.z, p.w, i.y, i.z, i.w, 0};
    }
    return ChunkItem{uni(it.seq), uni(it.first), uni(it.pos), uni(it.rows), uni(it.row0), uni(it.tiles), uni(it.before), 0};
  }
};

}  // namespace

// The walk of paged_attn_kernel over the items of the plan: 16 rows in place of the query heads of one token, a column of the matrix tile each with keys of its own; the
// four waves take an item's key tiles in turn.  Every wave multiplies, where the kernel with keys in LDS would leave three of four without rows.  Bound by the
// trips to memory: 16 sequences of 512 to 8 192 tokens, up to five new ones each, 32/8 heads of 128, 35.4 us in a graph (37.8 launched among others) of which the join is 5, 92 MB of codes (49.5 with keys in LDS; 46.4, when it was 38.3, with loads past the caches: items of a place read the same keys).
template <typename TT, bool GROUPED>
__global__ __launch_bounds__(kPagedThreads, 2) void chunk_few_kernel(KCache c, ChunkArgs a, ChunkPlan plan) {
  typedef typename TT::Out IO;
  constexpr int D = TT::kD;
  static_assert(TT::kKeys == kPagedKeys && kFewItem == 16, "the host counts tiles of so many keys and rows");
  __shared__ float s_acc[kPagedWaves - 1][TT::kAcc * 4 + 2][64];
  __shared__ int32_t s_odd[2];   // by turns: the last piece of work that met a number of V that is not finite where not every row sees it
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), i = lane & 15, g = lane >> 4;
  __shared__ OwnPlan own;
  const ChunkShare share(c, a, plan, own);
  const int w = share.w;
  if (share.left == 0) return;
  int hk = share.hk, item = share.item, t0 = share.t0, left = share.left;
  if (tid < 2) s_odd[tid] = -1;
  __syncthreads();
  constexpr int turns = kPagedWaves;
  const int turn = wave;
  for (int piece = 0; left > 0; piece++) {
    const ChunkItem it = share.at(a, plan, own, item);
    const int end = min(it.row0 + a.rows, it.rows), count = it.tiles;
    const int lo = it.pos + a.group.quot(it.row0), hi = it.pos + a.group.quot(end - 1);
    const KeyTiles keys = chunk_tiles(lo, hi, a.window, a.sink, TT::kKeys);
    const int t1 = min(count, t0 + left);
    const int32_t* table = c.row(it.seq);
    const ChunkRow row(a, hk, it.first, it.pos, end, it.row0 + i);
    auto seen_by_all = [&](int base) { return (base + TT::kKeys - 1 <= lo) & ((a.window <= 0) | (hi - base < a.window) | (base + TT::kKeys <= a.sink)); };

    Where<TT, GROUPED> now, next;
    int x = t0 + turn;
    int32_t base = keys.tile_at(x) * TT::kKeys, base_next = keys.tile_at(min(x + turns, keys.count)) * TT::kKeys;
    now.look(c, table, base, x < t1 ? keys.len : 0, i, g);
    next.look(c, table, base_next, x + turns < t1 ? keys.len : 0, i, g);
    typename TT::Q q;
    TT::load_q(q, a.q + row.token * a.q_st + row.head * a.q_sh, g, row.real);
    const char* kb = c.k + hk * c.k_sh + TT::k_off(g);
    const char* vb = c.v + hk * c.v_sh + TT::v_off(i);
    f32x4 acc[TT::kAcc];
#pragma unroll
    for (int e = 0; e < TT::kAcc; e++) acc[e] = f32x4{0, 0, 0, 0};
    float m = -INFINITY, l = 0;
    bool odd = false;
    TT t;
    if (x < t1) {
      now.settle(c);
      now.template load_k<false>(c, t, kb, i, hk);
      now.template load_v<false>(c, t, vb, hk);
    }
    for (; x < t1; x += turns) {
      float s[TT::kGroup];
      t.scores(q, s);
      next.settle(c);
      next.template load_k<false>(c, t, kb, i, hk);
#pragma unroll
      for (int j = 0; j < TT::kGroup; j++) s[j] *= a.scale_log2e;
      const bool edge = !seen_by_all(base);
      if (edge || !__all(now.all_there())) {
#pragma unroll
        for (int j = 0; j < TT::kGroup; j++) {
          const int key = base + g * TT::kGroup + j;
          s[j] = row.sees(key) & now.there(j) ? s[j] : -INFINITY;
          t.keep_v(j, (key <= hi) & now.there(j));
        }
      }
      // What is left out here is added at the end, in edge tiles: where a page does not exist, the other pages' numbers stay in the products.
      if (edge) {
#pragma unroll
        for (int j = 0; j < TT::kGroup; j++) odd |= t.clean_v(j);
      }
      float top = s[0];
#pragma unroll
      for (int j = 1; j < TT::kGroup; j++) top = fmaxf(top, s[j]);
      top = fmaxf(top, __shfl_xor(top, 16));
      top = fmaxf(top, __shfl_xor(top, 32));
      const float m2 = fmaxf(m, top), zero = m2 == -INFINITY ? 0.f : m2, f = __builtin_amdgcn_exp2f(m - zero);
      float sum = 0, p[TT::kGroup];
#pragma unroll
      for (int j = 0; j < TT::kGroup; j++) {
        p[j] = __builtin_amdgcn_exp2f(s[j] - zero);
        sum += p[j];
      }
      l = l * f + sum;
      if (__any(m2 != m)) {
#pragma unroll
        for (int e = 0; e < TT::kAcc; e++) acc[e] *= f;
      }
      m = m2;
      t.template weigh<16>(p, false, acc);
      next.template load_v<false>(c, t, vb, hk);
      now = next;
      base = base_next;
      base_next = keys.tile_at(min(x + 2 * turns, keys.count)) * TT::kKeys;
      next.look(c, table, base_next, x + 2 * turns < t1 ? keys.len : 0, i, g);
    }
    if (__any(odd) && lane == 0) s_odd[piece & 1] = piece;
    // the waves meet, lane by lane
    if (turn > 0 && t0 + turn < t1) {
      float (*to)[64] = s_acc[turn - 1];
#pragma unroll
      for (int e = 0; e < TT::kAcc; e++)
#pragma unroll
        for (int r = 0; r < 4; r++) to[4 * e + r][lane] = acc[e][r];
      to[4 * TT::kAcc][lane] = m;
      to[4 * TT::kAcc + 1][lane] = l;
    }
    __syncthreads();
    if (turn == 0) {
      for (int v = 1; v < turns && t0 + v < t1; v++) {
        const float (*from)[64] = s_acc[v - 1];
        const float mv = from[4 * TT::kAcc][lane], m2 = fmaxf(m, mv), zero = m2 == -INFINITY ? 0.f : m2;
        const float f = __builtin_amdgcn_exp2f(m - zero), fv = __builtin_amdgcn_exp2f(mv - zero);
        l = l * f + from[4 * TT::kAcc + 1][lane] * fv;
#pragma unroll
        for (int e = 0; e < TT::kAcc; e++)
#pragma unroll
          for (int r = 0; r < 4; r++) acc[e][r] = acc[e][r] * f + from[4 * e + r][lane] * fv;
        m = m2;
      }
      l += __shfl_xor(l, 16);
      l += __shfl_xor(l, 32);
      const bool done = t0 == 0 && t1 == count;
      const int64_t slot = (int64_t)(2 * w + (t0 == 0)) * a.rows + i;
      char* out = done ? a.out + row.token * a.o_st + row.head * a.o_sh : (char*)(plan.o + slot * D);
      const float by = !done ? 1.f : l == 0.f ? 0.f : 1.f / l;
      if (row.real) {
#pragma unroll
        for (int r = 0; r < 4; r++) {
          float o[TT::kRun];
#pragma unroll
          for (int z = 0; z < TT::kRun; z++) o[z] = by == 0.f ? 0.f : acc[z][r] * by;
          if (done) store_run<IO, TT::kRun>(out + TT::first(r, 0, g) * sizeof(IO), o);
          else store_run<float, TT::kRun>(out + TT::first(r, 0, g) * sizeof(float), o);
        }
        if (g == 0) {
          if (done) a.lse[row.head * a.n_tokens + row.token] = lse_of(m, l);
          else plan.ml[slot] = make_float2(m, l);
        }
      }
      if (s_odd[piece & 1] == piece)
        for (int y = t0; y < t1; y++) {
          const int from = keys.tile_at(y) * TT::kKeys;
          if (!seen_by_all(from))
            add_not_finite<D>(c, table, hk, row, from, min(from + TT::kKeys, keys.len), [&](int d) { return g == (d / TT::kAcc) >> 2; },
                              [&](int d, float v) { if (done) add_to<IO>(out + sizeof(IO) * d, v); else add_to<float>(out + 4 * d, v); });
        }
    }
    __syncthreads();   // s_acc is free
    if (t0 == 0 && t1 < count && tid == 0)
      plan.joins[w] = ChunkJoin{hk, w, ChunkShares(share.tiles * c.hkv).worker_of(hk * share.tiles + it.before + count - 1), 0, it.first, it.rows, it.row0, 0};
    left -= t1 - t0;
    t0 = 0;
    if (++item == share.n_items) { item = 0; hk++; }
  }
}

template <typename IO, int D> static void few(const KCache& c, const ChunkArgs& a, const ChunkPlan& plan, hipStream_t s) {
  auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(kWorkers), dim3(kPagedThreads), 0, s, c, a, plan); };
  if (c.page.d % 8 == 0 && c.block.d % 8 == 0) go(chunk_few_kernel<Tile8<IO, D>, true>);
  else go(chunk_few_kernel<Tile8<IO, D>, false>);
}
template <typename IO> static void few(int32_t d, const KCache& c, const ChunkArgs& a, const ChunkPlan& plan, hipStream_t s) {
  if (d == 128) few<IO, 128>(c, a, plan, s);
  else if (d == 64) few<IO, 64>(c, a, plan, s);
  else few<IO, 32>(c, a, plan, s);
}
void launch_chunk_few(int32_t d, const KCache& c, const ChunkArgs& a, const ChunkPlan& plan, hipStream_t s) {
  if (c.io_bytes == 4) few<float>(d, c, a, plan, s);
  else few<bf16_t>(d, c, a, plan, s);
}

}  // namespace dcp
