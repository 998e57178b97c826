// The kernels of the attention of one new token per sequence over a paged key-value cache, for any kind of tile: a wave's walk over keys
// (paged_attn.hip has those of bf16 and fp32, paged_attn8.hip those in 8 bits) and the join of what several workgroups did for one item.
#pragma once
#include "cache_internal.h"
#include "device_utils.h"

namespace dcp {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

// Keys and values are read once, so they go past the caches (ONCE: 32 places of 512 to 8 192 tokens 78 -> 73 us), unless several sets of heads
// read them, or a head's row is half a line of the caches whose other half the wave beside reads (bf16 with D = 32: 53 -> 50).
template <bool ONCE, typename V> __device__ __forceinline__ V load_kv(const char* p) {
  if constexpr (ONCE) return __builtin_nontemporal_load((const V*)p);
  else return *(const V*)p;
}

// N values in a row: 2, 4 or 8 of them.
template <typename T, int N> __device__ __forceinline__ void store_run(char* p, const float* o) {
  if constexpr (sizeof(T) == 4) {
    typedef float Vec __attribute__((ext_vector_type(N < 4 ? N : 4)));
#pragma unroll
    for (int x = 0; x < N; x += 4) {
      Vec v;
#pragma unroll
      for (int y = 0; y < (N < 4 ? N : 4); y++) v[y] = o[x + y];
      *(Vec*)(p + 4 * x) = v;
    }
  } else if constexpr (N == 2) {
    *(uint32_t*)p = pack_bf16x2(o[0], o[1]);
  } else if constexpr (N == 4) {
    *(uint2*)p = make_uint2(pack_bf16x2(o[0], o[1]), pack_bf16x2(o[2], o[3]));
  } else {
    *(uint4*)p = make_uint4(pack_bf16x2(o[0], o[1]), pack_bf16x2(o[2], o[3]), pack_bf16x2(o[4], o[5]), pack_bf16x2(o[6], o[7]));
  }
}

// Where the keys of a tile lie.  GROUPED: page_size is a multiple of the lanes' groups of 8 (fp32: 4) keys, so that a group shares a page
// and one entry of the table serves it; else every key has its own.
template <typename TT, bool GROUPED> struct Where {
  static constexpr int kV = GROUPED ? 1 : TT::kGroup, kK = GROUPED ? 0 : TT::kRowTiles;
  int32_t page[kV + kK], slot[kV + kK];   // of the lane's keys of V, then of K; page -1: no key there

  // base: the tile's first key; end: keys of the sequence, 0 where there is no such tile
  __device__ __forceinline__ void look(const KCache& c, const int32_t* row, int32_t base, int32_t end, int i, int g) {
#pragma unroll
    for (int x = 0; x < kV + kK; x++) {
      const int32_t j = base + (x < kV ? g * TT::kGroup + x : (i >> 2) * TT::kGroup + 4 * (x - kV) + (i & 3));
      const int32_t p = c.page.quot(j);
      slot[x] = c.page.rem(j, p);
      page[x] = -1;
      if (j < end) page[x] = row[p];
    }
  }
  // A key that is not there is read as the first of page 0.
  __device__ __forceinline__ void settle(const KCache& c) {
#pragma unroll
    for (int x = 0; x < kV + kK; x++) {
      page[x] = c.is_page(page[x]) ? page[x] : -1;
      slot[x] = page[x] < 0 ? 0 : slot[x];
    }
  }
  // hk: the KV head, for its scales
  template <bool ONCE> __device__ __forceinline__ void load_k(const KCache& c, TT& t, const char* kb, int i, int hk) const {
    if constexpr (GROUPED) {
      const int from = (i >> 2) << 4;
      const int32_t p = __shfl(max(page[0], 0), from), at = __shfl(slot[0], from) + (i & 3);
      const char* k = kb + p * c.k_sp + at * c.k_st;
#pragma unroll
      for (int x = 0; x < TT::kRowTiles; x++) t.template load_k<ONCE>(x, k + 4 * x * c.k_st);
      if constexpr (TT::kScaled) t.k_scales(c.k_scale[c.scale_at(p, at) + hk]);   // a group's keys share a block
    } else {
#pragma unroll
      for (int x = 0; x < kK; x++) {
        t.template load_k<ONCE>(x, kb + max(page[kV + x], 0) * c.k_sp + slot[kV + x] * c.k_st);
        if constexpr (TT::kScaled) t.k_scale(x, c.k_scale[c.scale_at(max(page[kV + x], 0), slot[kV + x]) + hk]);
      }
    }
  }
  template <bool ONCE> __device__ __forceinline__ void load_v(const KCache& c, TT& t, const char* vb, int hk) const {
    if constexpr (GROUPED) {
      const char* v = vb + max(page[0], 0) * c.v_sp + slot[0] * c.v_st;
#pragma unroll
      for (int x = 0; x < TT::kGroup; x++) t.template load_v<ONCE>(x, v + x * c.v_st);
      if constexpr (TT::kScaled) t.v_scales(c.v_scale[c.scale_at(max(page[0], 0), slot[0]) + hk]);
    } else {
#pragma unroll
      for (int x = 0; x < kV; x++) {
        t.template load_v<ONCE>(x, vb + max(page[x], 0) * c.v_sp + slot[x] * c.v_st);
        if constexpr (TT::kScaled) t.v_scale(x, c.v_scale[c.scale_at(max(page[x], 0), slot[x]) + hk]);
      }
    }
  }
  __device__ __forceinline__ bool there(int x) const { return page[GROUPED ? 0 : x] >= 0; }
  __device__ __forceinline__ bool all_there() const {
    int32_t all = page[0];
#pragma unroll
    for (int x = 1; x < kV; x++) all |= page[x];
    return all >= 0;
  }
};

// A place that is not OK is padding.
__device__ __forceinline__ int32_t seq_at(const PagedArgs& a, int i) {
  const int32_t seq = a.seqs ? a.seqs[i] : i, code = a.status ? a.status[i] : DCP_PLACE_OK;
  return code == DCP_PLACE_OK ? seq : -1;
}

// O = sum_j exp(s_j - m) v_j / l, LSE = m + ln l with m = max_j s_j, l = sum_j exp(s_j - m) over the keys j that the place sees, in one pass: m, l and
// O are carried along in fp32 (the weights too: fp32, or two bf16 parts), and rescaled where m grows.
// Bound by HBM: 2 x keys x hkv x D values are read once, at 6.3 to 6.5 TB/s in large batches (a plain read of linear memory past the caches 7.0): 224 places
// of 64 to 16 384 tokens, 32/8 heads of 128, pages of 16, 463 us of which the join is 6.  About 5 us pass before the first keys are asked for (launch,
// seqs, seq_len, page_table, one after the other), 4 to 7 are the join, which is what bounds short calls.  All tiles of the batch are dealt
// out evenly, whatever the lengths, so that workgroups end together; tiles in flight: the next one's K and V (a second V in flight
// gained nothing, nor did 768 or 1 024 workgroups).  The sums of a place are taken in an order that goes by the lengths of the whole batch, and by nothing else.
// Conditions that select lanes are written with & and |: a select a key, where && and || make a branch a key (which takes as long).
template <typename TT, int COLS, bool GROUPED, bool ONCE>
__global__ __launch_bounds__(kPagedThreads, 2) void paged_attn_kernel(KCache c, PagedArgs a, PagedParts parts) {
  typedef typename TT::Out T;
  constexpr int D = TT::kD;
  __shared__ int32_t s_wave[kPagedWaves], s_before, s_place, s_seq[kPagedThreads], s_len[kPagedThreads];
  __shared__ float s_acc[kPagedWaves - 1][TT::kAcc * 4 + 2][64];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), i = lane & 15, g = lane >> 4, w = blockIdx.x;

  // Every workgroup sums up all places' tiles for itself: thread t those of places [t per, (t + 1) per).
  const int per = (a.n + kPagedThreads - 1) / kPagedThreads;
  int32_t mine = 0;
  for (int x = tid * per; x < min(a.n, (tid + 1) * per); x++) {
    const int seq = seq_at(a, x), len = c.is_seq(seq) ? c.length(seq) : 0;
    if (c.is_seq(seq)) mine += a.whole ? 1 : KeyTiles(len, a.window, a.sink, TT::kKeys).count;
    s_seq[tid] = seq;   // of use where a thread has one place
    s_len[tid] = len;
  }
  int32_t upto = mine;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int32_t y = __shfl_up(upto, o);
    if (lane >= o) upto += y;
  }
  if (lane == 63) s_wave[wave] = upto;
  __syncthreads();
  int32_t all = 0, earlier = 0;
#pragma unroll
  for (int y = 0; y < kPagedWaves; y++) {
    if (y < wave) earlier += s_wave[y];
    all += s_wave[y];
  }
  if (tid == 0 && !parts.by_item && !a.whole) parts.joins[w] = make_int4(-1, 0, 0, 0);   // unless it begins an item that it does not end
  if (all == 0) return;
  const Shares<kLogWorkers> sh(all * a.groups);   // below 2^31: the host has seen to it
  if (w >= sh.workers) return;
  int32_t at = sh.start(w);
  const int32_t end = sh.start(w + 1);
  {
    const int32_t b = (earlier + upto - mine) * a.groups;
    if (b <= at && at < b + mine * a.groups) {
      s_place = tid * per;
      s_before = earlier + upto - mine;
    }
  }
  __syncthreads();
  int place = s_place;
  int32_t before = s_before;   // tiles of the places before it
  const int abreast = a.abreast, turns = kPagedWaves >> a.log_abreast, turn = wave >> a.log_abreast;
  while (at < end && place < a.n) {
    const int seq = per == 1 ? s_seq[place] : seq_at(a, place);
    if (!c.is_seq(seq)) { place++; continue; }
    const KeyTiles keys(per == 1 ? s_len[place] : c.length(seq), a.window, a.sink, TT::kKeys);
    const int units = a.whole ? 1 : keys.count;   // of an item
    const int32_t rel = at - before * a.groups;
    if (rel >= units * a.groups) { before += units; place++; continue; }
    const int32_t* row = c.row(seq);
    const int grp = (int)((uint32_t)rel / (uint32_t)units), t0 = rel - grp * units;
    const int t1 = a.whole ? keys.count : min(keys.count, t0 + (end - at));
    const int set = grp * abreast + (wave & (abreast - 1)), hk = a.per_kv == 1 ? set : set / a.per_kv;
    const int h0 = hk * a.group + (set - hk * a.per_kv) * kSetHeads, n_heads = min(kSetHeads, (hk + 1) * a.group - h0);
    const int col = COLS == 8 ? i & 7 : i;

    Where<TT, GROUPED> now, next;
    int x = t0 + turn;
    int32_t base = keys.tile_at(x) * TT::kKeys, base_next = keys.tile_at(min(x + turns, keys.count)) * TT::kKeys;
    now.look(c, row, base, x < t1 ? keys.len : 0, i, g);
    next.look(c, row, base_next, x + turns < t1 ? keys.len : 0, i, g);
    typename TT::Q q;   // comes while the entries of the table do
    TT::load_q(q, a.q + place * a.q_st + (h0 + col) * a.q_sh, g, col < n_heads);
    const char* kb = c.k + hk * c.k_sh + TT::k_off(g);
    const char* vb = c.v + hk * c.v_sh + TT::v_off(i);
    f32x4 acc[TT::kAcc];
#pragma unroll
    for (int e = 0; e < TT::kAcc; e++) acc[e] = f32x4{0, 0, 0, 0};
    float m = -INFINITY, l = 0;
    TT t;
    if (x < t1) {
      now.settle(c);
      now.template load_k<ONCE>(c, t, kb, i, hk);
      now.template load_v<ONCE>(c, t, vb, hk);
    }
    for (; x < t1; x += turns) {
      float s[TT::kGroup];
      t.scores(q, s);
      next.settle(c);
      next.template load_k<ONCE>(c, t, kb, i, hk);
      const bool whole = (base + TT::kKeys <= keys.len) & ((base >= keys.lo) | (base + TT::kKeys <= keys.head));
#pragma unroll
      for (int j = 0; j < TT::kGroup; j++) s[j] *= a.scale_log2e;
      if (!whole || !__all(now.all_there())) {
#pragma unroll
        for (int j = 0; j < TT::kGroup; j++) {
          const bool seen = keys.sees(base + g * TT::kGroup + j) & now.there(j);
          s[j] = seen ? s[j] : -INFINITY;
          t.keep_v(j, seen);
        }
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
      t.template weigh<COLS>(p, i >= 8, acc);
      next.template load_v<ONCE>(c, t, vb, hk);
      now = next;
      base = base_next;
      base_next = keys.tile_at(min(x + 2 * turns, keys.count)) * TT::kKeys;
      next.look(c, row, base_next, x + 2 * turns < t1 ? keys.len : 0, i, g);
    }

    if (turns > 1) {   // the waves of a set meet, lane by lane
      if (turn > 0 && t0 + turn < t1) {
        float (*to)[64] = s_acc[wave - abreast];
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
          const float (*from)[64] = s_acc[(v - 1) * abreast + wave];
          const float mv = from[4 * TT::kAcc][lane], m2 = fmaxf(m, mv), zero = m2 == -INFINITY ? 0.f : m2;
          const float f = __builtin_amdgcn_exp2f(m - zero), fv = __builtin_amdgcn_exp2f(mv - zero);
          l = l * f + from[4 * TT::kAcc + 1][lane] * fv;
#pragma unroll
          for (int e = 0; e < TT::kAcc; e++)
#pragma unroll
            for (int r = 0; r < 4; r++) acc[e][r] = acc[e][r] * f + from[4 * e + r][lane] * fv;
          m = m2;
        }
      }
      __syncthreads();
    }
    if (turn == 0) {
      l += __shfl_xor(l, 16);
      l += __shfl_xor(l, 32);
      if constexpr (COLS == 8) {
#pragma unroll
        for (int e = 0; e < TT::kAcc; e++)
#pragma unroll
          for (int r = 0; r < 4; r++) acc[e][r] += __shfl_xor(acc[e][r], 8);
      }
      if (t0 == 0 && t1 == keys.count) {
        const float inv = l == 0.f ? 0.f : 1.f / l;
        if (i < n_heads) {
          char* out = a.out + place * a.o_st + (h0 + i) * a.o_sh;
#pragma unroll
          for (int r = 0; r < 4; r++)
#pragma unroll
            for (int y = 0; y < TT::kRuns; y++) {
              float o[TT::kRun];
#pragma unroll
              for (int z = 0; z < TT::kRun; z++) o[z] = l == 0.f ? 0.f : acc[y * TT::kRun + z][r] * inv;
              store_run<T, TT::kRun>(out + TT::first(r, y, g) * sizeof(T), o);
            }
          if (g == 0) a.lse[(int64_t)(h0 + i) * a.n + place] = l == 0.f ? -INFINITY : (m == -INFINITY ? 0.f : m) * 0.6931471805599453f + logf(l);
        }
      } else {
        const int slot = (2 * w + (t0 == 0)) * abreast + (wave & (abreast - 1));
        if (i < n_heads) {
          float* out = parts.o + ((int64_t)slot * a.set_heads + i) * D;
#pragma unroll
          for (int r = 0; r < 4; r++)
#pragma unroll
            for (int y = 0; y < TT::kRuns; y++) {
              float o[TT::kRun];
#pragma unroll
              for (int z = 0; z < TT::kRun; z++) o[z] = acc[y * TT::kRun + z][r];
              store_run<float, TT::kRun>((char*)(out + TT::first(r, y, g)), o);
            }
          if (g == 0) parts.ml[slot * a.set_heads + i] = make_float2(m, l);
        }
      }
    }
    if (t0 == 0 && tid == 0 && !a.whole) {
      const int last = t1 == keys.count ? w : sh.worker_of(before * a.groups + (grp + 1) * keys.count - 1);
      if (parts.by_item) parts.joins[place * a.groups + grp] = make_int4(last == w ? -1 : place, grp, w, last);
      else if (last != w) parts.joins[w] = make_int4(place, grp, w, last);
    }
    at += a.whole ? 1 : t1 - t0;
  }
}

// Joins the parts of an item: workgroup (x, y) takes HEADS query heads of entry x of the list.  D / 4 lanes walk every kRows-th part of a
// head, with a maximum of their own, and meet in LDS.  Bound by latency: three dependent trips to memory where an item has few parts.
template <typename T, int D, int THREADS, int HEADS>
__global__ __launch_bounds__(THREADS) void paged_join_kernel(KCache c, PagedArgs a, PagedParts parts) {
  constexpr int kLanes = D / 4, kRows = THREADS / kLanes / HEADS;
  __shared__ float s_m[HEADS][kRows], s_l[HEADS][kRows], s_o[HEADS][kRows][D];
  const int tid = threadIdx.x;
  const int4 job = parts.joins[blockIdx.x];
  if (parts.by_item && !c.is_seq(seq_at(a, blockIdx.x / a.groups))) return;   // nobody has written the entry of padding
  if (job.x < 0) return;
  const int hw = tid / (kLanes * kRows), r = tid / kLanes % kRows, d = tid % kLanes * 4;
  const int y = blockIdx.y * HEADS + hw, beside = y / a.set_heads, h = y - beside * a.set_heads, set = job.y * a.abreast + beside;
  const int hk = set / a.per_kv, h0 = hk * a.group + (set - hk * a.per_kv) * kSetHeads;
  const bool real = beside < a.abreast && h0 + h < (hk + 1) * a.group;
  const int w = job.z, n = real ? job.w - w + 1 : 0;   // parts: slot 2 w + 1, then 2 v of the later workers v
  float m = -INFINITY, l = 0;
  f32x4 o = {0, 0, 0, 0};
  constexpr int kAhead = 4;   // parts of a lane in flight
  for (int p0 = r; p0 < n; p0 += kAhead * kRows) {
    float2 ml[kAhead];
    f32x4 part[kAhead];
#pragma unroll
    for (int x = 0; x < kAhead; x++) {
      const int p = p0 + x * kRows;
      const int64_t slot = ((int64_t)(p == 0 ? 2 * w + 1 : 2 * (w + p)) * a.abreast + beside) * a.set_heads + h;
      ml[x] = make_float2(-INFINITY, 0.f);
      part[x] = f32x4{0, 0, 0, 0};
      if (p < n) {
        ml[x] = parts.ml[slot];
        part[x] = *(const f32x4*)&parts.o[slot * D + d];
      }
    }
#pragma unroll
    for (int x = 0; x < kAhead; x++) {
      const float m2 = fmaxf(m, ml[x].x), zero = m2 == -INFINITY ? 0.f : m2;
      const float f = __builtin_amdgcn_exp2f(m - zero), fx = __builtin_amdgcn_exp2f(ml[x].x - zero);
      l = l * f + ml[x].y * fx;
      o = o * f + part[x] * fx;
      m = m2;
    }
  }
  if (d == 0) { s_m[hw][r] = m; s_l[hw][r] = l; }
  *(f32x4*)&s_o[hw][r][d] = o;
  __syncthreads();
  if (r || !real) return;
  float top = m, sum = 0;
#pragma unroll
  for (int x = 1; x < kRows; x++) top = fmaxf(top, s_m[hw][x]);
  const float zero = top == -INFINITY ? 0.f : top;
  o = f32x4{0, 0, 0, 0};
#pragma unroll
  for (int x = 0; x < kRows; x++) {
    if (x >= n) continue;
    const float f = __builtin_amdgcn_exp2f(s_m[hw][x] - zero);
    sum += s_l[hw][x] * f;
    o += f * *(const f32x4*)&s_o[hw][x][d];
  }
  float res[4];
#pragma unroll
  for (int x = 0; x < 4; x++) res[x] = sum == 0.f ? 0.f : o[x] / sum;
  store_run<T, 4>(a.out + job.x * a.o_st + (h0 + h) * a.o_sh + d * sizeof(T), res);
  if (d == 0) a.lse[(int64_t)(h0 + h) * a.n + job.x] = sum == 0.f ? -INFINITY : zero * 0.6931471805599453f + logf(sum);
}

// Of few items each is in many parts, which a join takes with more threads a head: up to kMiddleJoins entries of the list 256, else 64; heads of 128,
// of which 256 threads take only 8 parts at a time, 1 024 threads up to kWideJoins.  Whole calls, us, with 1 024 / 256 / 64: D 128, 1 entry of
// 30 000 tokens 27.9 / 32.8 / 62.3, 2 of 131 067 93.6 / 95.3 / 110, 3 of 30 000 44.7 / 45.3 / -, 5 63.3 / 63.1 / -, 8 of 20 000 66.0 / 65.3 / 69.1, 16 of
// 2 048 26.2 / 24.9 / 26.3, 31 of 4 096 55.8 / 54.3 / 55.5, 70 of 2 048 65.9 / 62.5 / 61.7; D 64, 1 of 8 000 14.7 / 13.5 / -, of 30 000 20.8 / 21.1 / 37.3, 3 of
// 30 000 28.9 / 27.2 / -, 16 of 2 048 18.1 / 16.7 / 16.8, 31 of 4 096 33.9 / 32.8 / 32.5; fp32 with D 64, 8 of 1 to 4 096 18.2 / 15.8 / 18.9.
// In 8 bits with 16/4 heads the same: D 128, 1 entry of 30 000 tokens 21.8 / 26.6 / 55.8, 2 of 131 067 58.0 / 59.6 / 73.1, 3 of 30 000 31.3 / 31.5 / 41.8, 5 39.0 / 39.0 / 45.2, 8 of 20 000 39.6 / 39.3 / 43.2,
// 16 of 2 048 17.5 / 16.2 / 17.6, 31 of 4 096 34.8 / 33.3 / 34.5, 70 of 2 048 43.2 / 39.8 / 39.1; D 64, 1 of 30 000 17.4 / 17.4 / 33.8, 3 20.1 / 20.1 / 25.8, 31 of 4 096 22.2 / 22.1 / 21.8.
static constexpr unsigned kWideJoins = 3, kMiddleJoins = 31;

template <typename TT, int COLS, bool ONCE>
inline void launch_once(uint32_t grid, const KCache& c, const PagedArgs& a, const PagedParts& parts, hipStream_t s) {
  if (c.page.d % TT::kGroup == 0 && (!TT::kScaled || c.block.d % TT::kGroup == 0))
    hipLaunchKernelGGL((paged_attn_kernel<TT, COLS, true, ONCE>), dim3(grid), dim3(kPagedThreads), 0, s, c, a, parts);
  else hipLaunchKernelGGL((paged_attn_kernel<TT, COLS, false, ONCE>), dim3(grid), dim3(kPagedThreads), 0, s, c, a, parts);
}
template <typename TT, int COLS>
inline void launch_tiles(uint32_t grid, const KCache& c, const PagedArgs& a, const PagedParts& parts, hipStream_t s) {
  typedef typename TT::Out T;
  constexpr int D = TT::kD;
  if constexpr (TT::kRowBytes < 128) launch_once<TT, COLS, false>(grid, c, a, parts, s);
  else if (a.per_kv == 1) launch_once<TT, COLS, true>(grid, c, a, parts, s);
  else if constexpr (COLS == kSetHeads) launch_once<TT, COLS, false>(grid, c, a, parts, s);   // more sets than one are full ones
  if (a.whole) return;
  const unsigned entries = parts.by_item ? a.n * a.groups : kWorkers, heads = a.abreast * a.set_heads;
  if constexpr (D == 128) {
    if (entries <= kWideJoins) {
      hipLaunchKernelGGL((paged_join_kernel<T, D, 1024, 1>), dim3(entries, heads), dim3(1024), 0, s, c, a, parts);
      return;
    }
  }
  if (entries <= kMiddleJoins) hipLaunchKernelGGL((paged_join_kernel<T, D, 256, 1>), dim3(entries, heads), dim3(256), 0, s, c, a, parts);
  else hipLaunchKernelGGL((paged_join_kernel<T, D, 256, 4>), dim3(entries, (heads + 3) / 4), dim3(256), 0, s, c, a, parts);
}
}  // namespace dcp
