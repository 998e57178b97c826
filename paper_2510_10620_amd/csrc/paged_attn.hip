// Attention of one new token per sequence over a paged key-value cache.
#include <algorithm>
#include <cmath>

#include "cache_internal.h"
#include "device_utils.h"

using namespace dcp;

namespace dcp {

struct PagedArgs {
  const char* q;
  char* out;
  float* lse;
  const int32_t* seqs;
  int64_t q_st, q_sh, o_st, o_sh;   // bytes
  int32_t n, hq, group, layer, window, sink;
  int32_t head_sets;   // items of a place: KV heads x sets of up to 16 query heads that share one
  float scale_log2e;
};

// Partial results of items (place, head set) that several workers share, unnormalised, in units of log2.  A worker's share of the tiles
// begins in the middle of at most one item and ends in the middle of at most one: slot 2 w holds the first, 2 w + 1 the second.
struct PagedParts {
  int4* joins;    // [kWorkers] of the item whose first tile worker w has, where others have its last: (place, head set, last worker), place -1: none
  float2* ml;     // [2 kWorkers][heads of a set] running maximum, sum
  float* o;       // [2 kWorkers][heads of a set][D]
};

static constexpr int kWorkers = 768;     // workgroups, three on a CU
static constexpr int kPagedWaves = 4, kPagedThreads = 64 * kPagedWaves;
static constexpr int kSetHeads = 16;     // query heads of a matrix tile
static constexpr int kLeastTiles = kPagedWaves;   // of a worker

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

// A wave walks tiles of 32 (fp32: 16) keys.  Lane l has i = l % 16 and g = l / 16.  K is the A operand as it lies in memory: row i of the
// matrix tile is a key, 16 bytes of it a lane; S^T = K Q^T then holds in lane (i, g) the scores of query head i with the keys
// of group g, 8 g .. 8 g + 7 (fp32: 4 g .. 4 g + 3), if the rows of K are dealt out for it: row r of matrix tile s is key 8 (r / 4) + 4 s + r % 4.
// That is the B operand of O^T = V^T P^T, whose A operand wants from lane (i, g) the keys of group g at one column: a lane loads
// D / 16 neighbouring columns of each of them, which are the same rows of A in D / 16 matrix tiles.  So nothing moves between lanes but
// the maximum over a tile's keys.
template <typename T, int D> struct Tile;

template <int D> struct Tile<bf16_t, D> {
  static constexpr int kGroup = 8, kKeys = 32, kRowTiles = 2, kAcc = D / 16;
  static constexpr int kWords = D / 32;   // 4-byte words of a lane's columns of V
  struct V { uint32_t w[kWords]; };
  uint4 k[kRowTiles][D / 32];
  V v[kGroup];

  static __device__ __forceinline__ int k_off(int g) { return g * 16; }
  static __device__ __forceinline__ int v_off(int i) { return i * (D / 8); }
  __device__ __forceinline__ void load_k(int s, const char* p) {
#pragma unroll
    for (int x = 0; x < D / 32; x++) k[s][x] = *(const uint4*)(p + 64 * x);
  }
  __device__ __forceinline__ void load_v(int j, const char* p) {
    if constexpr (kWords == 4) { const uint4 u = *(const uint4*)p; v[j].w[0] = u.x; v[j].w[1] = u.y; v[j].w[2] = u.z; v[j].w[3] = u.w; }
    else if constexpr (kWords == 2) { const uint2 u = *(const uint2*)p; v[j].w[0] = u.x; v[j].w[1] = u.y; }
    else v[j].w[0] = *(const uint32_t*)p;
  }
  __device__ __forceinline__ void keep_v(int j, bool keep) {
#pragma unroll
    for (int x = 0; x < kWords; x++) v[j].w[x] = keep ? v[j].w[x] : 0u;
  }
  struct Q { bf16x8 x[D / 32]; };
  static __device__ __forceinline__ void load_q(Q& q, const char* p, int g, bool real) {
#pragma unroll
    for (int x = 0; x < D / 32; x++)
      q.x[x] = __builtin_bit_cast(bf16x8, real ? *(const uint4*)(p + 64 * x + 16 * g) : make_uint4(0, 0, 0, 0));
  }
  // scores of the lane's head with the keys of group g
  __device__ __forceinline__ void scores(const Q& q, float* s) const {
#pragma unroll
    for (int t = 0; t < kRowTiles; t++) {
      f32x4 z = {0, 0, 0, 0};
#pragma unroll
      for (int x = 0; x < D / 32; x++) z = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, k[t][x]), q.x[x], z, 0, 0, 0);
#pragma unroll
      for (int r = 0; r < 4; r++) s[4 * t + r] = z[r];
    }
  }
  // The weights as two bf16 numbers, which hold them to 2^-15: the first is below the weight, so that both are positive and an Inf in V
  // stays one.  COLS 8: a set has up to 8 heads and columns i and i + 8 of the matrix tile are head i's two parts; else two products.
  static __device__ __forceinline__ float first_part(float p) { return __uint_as_float(__float_as_uint(p * 0.99609375f) & 0xffff0000u); }
  template <int COLS> __device__ __forceinline__ void weigh(const float* p, bool second, f32x4* acc) const {
    float hi[8], lo[8];
#pragma unroll
    for (int j = 0; j < 8; j++) { hi[j] = first_part(p[j]); lo[j] = p[j] - hi[j]; }
    uint4 b, b2;
    auto pack = [](const float* x) { return make_uint4(pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]), pack_bf16x2(x[4], x[5]), pack_bf16x2(x[6], x[7])); };
    if constexpr (COLS == 8) {
#pragma unroll
      for (int j = 0; j < 8; j++) hi[j] = second ? lo[j] : hi[j];
      b = pack(hi);
    } else {
      b = pack(hi);
      b2 = pack(lo);
    }
#pragma unroll
    for (int e = 0; e < kAcc; e++) {
      const uint32_t sel = e & 1 ? 0x07060302u : 0x05040100u;
      uint4 a;
      a.x = __builtin_amdgcn_perm(v[1].w[e / 2], v[0].w[e / 2], sel);
      a.y = __builtin_amdgcn_perm(v[3].w[e / 2], v[2].w[e / 2], sel);
      a.z = __builtin_amdgcn_perm(v[5].w[e / 2], v[4].w[e / 2], sel);
      a.w = __builtin_amdgcn_perm(v[7].w[e / 2], v[6].w[e / 2], sel);
      acc[e] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), acc[e], 0, 0, 0);
      if constexpr (COLS != 8)
        acc[e] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b2), acc[e], 0, 0, 0);
    }
  }
  // column of acc[e][r] in lane (., g)
  static __device__ __forceinline__ int column(int e, int r, int g) { return (4 * g + r) * kAcc + e; }
};

template <int D> struct Tile<float, D> {
  static constexpr int kGroup = 4, kKeys = 16, kRowTiles = 1, kAcc = D / 16;
  static constexpr int kVec = D >= 64 ? 4 : 2, kParts = D / (16 * kVec);   // a lane has kParts pieces of kVec columns of V
  f32x4 k[D / 16];
  float v[kGroup][kParts][kVec];

  static __device__ __forceinline__ int k_off(int g) { return g * 16; }
  static __device__ __forceinline__ int v_off(int i) { return i * kVec * 4; }
  __device__ __forceinline__ void load_k(int, const char* p) {
#pragma unroll
    for (int x = 0; x < D / 16; x++) k[x] = *(const f32x4*)(p + 64 * x);
  }
  __device__ __forceinline__ void load_v(int j, const char* p) {
    typedef float Vec __attribute__((ext_vector_type(kVec)));
#pragma unroll
    for (int x = 0; x < kParts; x++) {
      const Vec u = *(const Vec*)(p + 64 * kVec * x);
#pragma unroll
      for (int y = 0; y < kVec; y++) v[j][x][y] = u[y];
    }
  }
  __device__ __forceinline__ void keep_v(int j, bool keep) {
#pragma unroll
    for (int x = 0; x < kParts; x++)
#pragma unroll
      for (int y = 0; y < kVec; y++) v[j][x][y] = keep ? v[j][x][y] : 0.f;
  }
  struct Q { f32x4 x[D / 16]; };
  static __device__ __forceinline__ void load_q(Q& q, const char* p, int g, bool real) {
    const f32x4 zero = {0, 0, 0, 0};
#pragma unroll
    for (int x = 0; x < D / 16; x++) q.x[x] = real ? *(const f32x4*)(p + 64 * x + 16 * g) : zero;
  }
  __device__ __forceinline__ void scores(const Q& q, float* s) const {
    f32x4 z = {0, 0, 0, 0};
#pragma unroll
    for (int x = 0; x < D / 16; x++)
#pragma unroll
      for (int y = 0; y < 4; y++) z = __builtin_amdgcn_mfma_f32_16x16x4f32(k[x][y], q.x[x][y], z, 0, 0, 0);
#pragma unroll
    for (int r = 0; r < 4; r++) s[r] = z[r];
  }
  template <int COLS> __device__ __forceinline__ void weigh(const float* p, bool, f32x4* acc) const {
#pragma unroll
    for (int j = 0; j < kGroup; j++)
#pragma unroll
      for (int x = 0; x < kParts; x++)
#pragma unroll
        for (int y = 0; y < kVec; y++) acc[x * kVec + y] = __builtin_amdgcn_mfma_f32_16x16x4f32(v[j][x][y], p[j], acc[x * kVec + y], 0, 0, 0);
  }
  static __device__ __forceinline__ int column(int e, int r, int g) { return (e / kVec) * 16 * kVec + (4 * g + r) * kVec + e % kVec; }
};

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
  __device__ __forceinline__ void load_k(const KCache& c, TT& t, const char* kb, int i) const {
    if constexpr (GROUPED) {
      const int from = (i >> 2) << 4;
      const int32_t p = __shfl(max(page[0], 0), from), at = __shfl(slot[0], from) + (i & 3);
      const char* k = kb + p * c.k_sp + at * c.k_st;
#pragma unroll
      for (int x = 0; x < TT::kRowTiles; x++) t.load_k(x, k + 4 * x * c.k_st);
    } else {
#pragma unroll
      for (int x = 0; x < kK; x++) t.load_k(x, kb + max(page[kV + x], 0) * c.k_sp + slot[kV + x] * c.k_st);
    }
  }
  __device__ __forceinline__ void load_v(const KCache& c, TT& t, const char* vb) const {
    if constexpr (GROUPED) {
      const char* v = vb + max(page[0], 0) * c.v_sp + slot[0] * c.v_st;
#pragma unroll
      for (int x = 0; x < TT::kGroup; x++) t.load_v(x, v + x * c.v_st);
    } else {
#pragma unroll
      for (int x = 0; x < kV; x++) t.load_v(x, vb + max(page[x], 0) * c.v_sp + slot[x] * c.v_st);
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

__device__ __forceinline__ int32_t place_tiles(const KCache& c, const PagedArgs& a, int i, int tile) {
  const int s = a.seqs ? a.seqs[i] : i;
  return c.is_seq(s) ? KeyTiles(c.length(s), a.window, a.sink, tile).count : 0;
}

template <typename T, int D, int COLS, bool GROUPED>
__global__ __launch_bounds__(kPagedThreads) void paged_attn_kernel(KCache c, PagedArgs a, PagedParts parts) {
  typedef Tile<T, D> TT;
  constexpr int kSet = COLS;   // heads of a set at most
  __shared__ int64_t s_sums[kPagedThreads + 1];
  __shared__ float s_m[kPagedWaves][kSet], s_l[kPagedWaves][kSet], s_o[kPagedWaves][kSet][D + 4];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), i = lane & 15, g = lane >> 4, w = blockIdx.x;

  // all places' tiles, summed up by every workgroup for itself
  const int per = (a.n + kPagedThreads - 1) / kPagedThreads;
  {
    int64_t mine = 0;
    for (int x = tid * per; x < min(a.n, (tid + 1) * per); x++) mine += place_tiles(c, a, x, TT::kKeys);
    int64_t x = mine;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const int64_t y = __shfl_up(x, o);
      if (lane >= o) x += y;
    }
    if (lane == 63) s_sums[wave] = x;
    __syncthreads();
    int64_t before = 0;
    for (int y = 0; y < wave; y++) before += s_sums[y];
    __syncthreads();
    s_sums[tid + 1] = before + x;
    if (tid == 0) s_sums[0] = 0;
    __syncthreads();
  }
  const int sets = a.head_sets, per_kv = sets / c.hkv;
  const int64_t all = s_sums[kPagedThreads] * sets;
  if (tid == 0) parts.joins[w] = make_int4(-1, 0, 0, 0);
  if (all == 0) return;
  const Shares sh = make_shares(all, kWorkers, kLeastTiles);
  if (w >= sh.workers) return;
  int64_t at = sh.start(w);
  const int64_t end = sh.start(w + 1);
  // the place of tile `at`, and the tiles before that place
  int place;
  int64_t before;
  {
    int lo = 0, hi = kPagedThreads - 1;
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if (s_sums[mid] * sets <= at) lo = mid;
      else hi = mid - 1;
    }
    place = lo * per;
    before = s_sums[lo];
  }
  while (at < end && place < a.n) {
    const int seq = a.seqs ? a.seqs[place] : place;
    if (!c.is_seq(seq)) { place++; continue; }
    const KeyTiles keys(c.length(seq), a.window, a.sink, TT::kKeys);
    if ((before + keys.count) * sets <= at) { before += keys.count; place++; continue; }
    const int32_t* row = c.row(seq);
    const int set = (int)((at - before * sets) / keys.count), t0 = (int)(at - before * sets - (int64_t)set * keys.count);
    const int t1 = (int)min((int64_t)keys.count, t0 + (end - at));
    const int hk = set / per_kv, h0 = hk * a.group + (set - hk * per_kv) * kSetHeads, n_heads = min(kSetHeads, (hk + 1) * a.group - h0);
    const int col = COLS == 8 ? i & 7 : i;

    typename TT::Q q;
    TT::load_q(q, a.q + place * a.q_st + (h0 + col) * a.q_sh, g, col < n_heads);
    const char* kb = c.k + a.layer * c.k_sl + hk * c.k_sh + TT::k_off(g);
    const char* vb = c.v + a.layer * c.v_sl + hk * c.v_sh + TT::v_off(i);
    f32x4 acc[TT::kAcc];
#pragma unroll
    for (int e = 0; e < TT::kAcc; e++) acc[e] = f32x4{0, 0, 0, 0};
    float m = -INFINITY, l = 0;
    TT t;
    Where<TT, GROUPED> now, next;
    int x = t0 + wave;
    int32_t base = keys.tile_at(x) * TT::kKeys, base_next = 0;
    if (x < t1) {
      now.look(c, row, base, keys.len, i, g);
      now.settle(c);
      now.load_k(c, t, kb, i);
      now.load_v(c, t, vb);
      base_next = keys.tile_at(min(x + kPagedWaves, keys.count)) * TT::kKeys;
      next.look(c, row, base_next, x + kPagedWaves < t1 ? keys.len : 0, i, g);
    }
    for (; x < t1; x += kPagedWaves) {
      float s[TT::kGroup];
      t.scores(q, s);
      next.settle(c);
      next.load_k(c, t, kb, i);
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
      next.load_v(c, t, vb);
      now = next;
      base = base_next;
      base_next = keys.tile_at(min(x + 2 * kPagedWaves, keys.count)) * TT::kKeys;
      next.look(c, row, base_next, x + 2 * kPagedWaves < t1 ? keys.len : 0, i, g);
    }

    // the waves meet
    l += __shfl_xor(l, 16);
    l += __shfl_xor(l, 32);
    if constexpr (COLS == 8 && sizeof(T) == 2) {
#pragma unroll
      for (int e = 0; e < TT::kAcc; e++)
#pragma unroll
        for (int r = 0; r < 4; r++) acc[e][r] += __shfl_xor(acc[e][r], 8);
    }
    if (i < n_heads) {
      if (g == 0) { s_m[wave][i] = m; s_l[wave][i] = l; }
#pragma unroll
      for (int e = 0; e < TT::kAcc; e++)
#pragma unroll
        for (int r = 0; r < 4; r++) s_o[wave][i][TT::column(e, r, g)] = acc[e][r];
    }
    __syncthreads();
    const bool complete = t0 == 0 && t1 == keys.count;
    const int slot = 2 * w + (t0 == 0);
    for (int y = tid; y < n_heads * (D / 4); y += kPagedThreads) {
      const int h = y / (D / 4), d = (y - h * (D / 4)) * 4;
      float top = s_m[0][h], sum = 0;
#pragma unroll
      for (int v = 1; v < kPagedWaves; v++) top = fmaxf(top, s_m[v][h]);
      const float zero = top == -INFINITY ? 0.f : top;
      f32x4 o = {0, 0, 0, 0};
#pragma unroll
      for (int v = 0; v < kPagedWaves; v++) {
        if (t0 + v >= t1) continue;   // a wave without a tile
        const float f = __builtin_amdgcn_exp2f(s_m[v][h] - zero);
        sum += f * s_l[v][h];
        o += f * *(const f32x4*)&s_o[v][h][d];
      }
      if (complete) {
        const f32x4 r = sum == 0.f ? f32x4{0, 0, 0, 0} : o / sum;
        char* p = a.out + place * a.o_st + (h0 + h) * a.o_sh + d * sizeof(T);
        if constexpr (sizeof(T) == 2) *(uint2*)p = make_uint2(pack_bf16x2(r[0], r[1]), pack_bf16x2(r[2], r[3]));
        else *(f32x4*)p = r;
        if (d == 0) a.lse[(int64_t)(h0 + h) * a.n + place] = sum == 0.f ? -INFINITY : zero * 0.6931471805599453f + logf(sum);
      } else {
        *(f32x4*)&parts.o[((int64_t)slot * kSet + h) * D + d] = o;
        if (d == 0) parts.ml[slot * kSet + h] = make_float2(top, sum);
      }
    }
    if (!complete && t0 == 0 && tid == 0)
      parts.joins[w] = make_int4(place, set, sh.worker_of(before * sets + (int64_t)(set + 1) * keys.count - 1), 0);
    __syncthreads();
    at += t1 - t0;
  }
}

// Joins the parts of an item: workgroup (w, h) takes head h of the item that worker w began and another ended.
template <typename T, int D, int COLS>
__global__ __launch_bounds__(kPagedThreads) void paged_join_kernel(KCache c, PagedArgs a, PagedParts parts) {
  constexpr int kSet = COLS, kLanes = D / 4, kRows = kPagedThreads / kLanes;
  __shared__ float s_top[kPagedWaves], s_sum[kRows], s_o[kRows][D + 4];
  const int tid = threadIdx.x, w = blockIdx.x, h = blockIdx.y;
  const int4 job = parts.joins[w];
  if (job.x < 0) return;
  const int per_kv = a.head_sets / c.hkv, hk = job.y / per_kv, h0 = hk * a.group + (job.y - hk * per_kv) * kSetHeads;
  if (h0 + h >= (hk + 1) * a.group) return;
  const int n = job.z - w + 1;   // parts: slot 2 w + 1, then 2 v of the later workers v
  auto slot = [&](int p) { return (p == 0 ? 2 * w + 1 : 2 * (w + p)) * kSet + h; };
  float top = -INFINITY;
  for (int p = tid; p < n; p += kPagedThreads) top = fmaxf(top, parts.ml[slot(p)].x);
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) top = fmaxf(top, __shfl_xor(top, o));
  if ((tid & 63) == 0) s_top[tid >> 6] = top;
  __syncthreads();
#pragma unroll
  for (int v = 0; v < kPagedWaves; v++) top = fmaxf(top, s_top[v]);
  const float zero = top == -INFINITY ? 0.f : top;
  const int r = tid / kLanes, d = (tid - r * kLanes) * 4;
  f32x4 o = {0, 0, 0, 0};
  float sum = 0;
  for (int p = r; p < n; p += kRows) {
    const float2 ml = parts.ml[slot(p)];
    const float f = __builtin_amdgcn_exp2f(ml.x - zero);
    sum += f * ml.y;
    o += f * *(const f32x4*)&parts.o[(int64_t)slot(p) * D + d];
  }
  if (d == 0) s_sum[r] = sum;
  *(f32x4*)&s_o[r][d] = o;
  __syncthreads();
  if (r) return;
#pragma unroll
  for (int x = 1; x < kRows; x++) {
    sum += s_sum[x];
    o += *(const f32x4*)&s_o[x][d];
  }
  const f32x4 res = sum == 0.f ? f32x4{0, 0, 0, 0} : o / sum;
  char* out = a.out + job.x * a.o_st + (h0 + h) * a.o_sh + d * sizeof(T);
  if constexpr (sizeof(T) == 2) *(uint2*)out = make_uint2(pack_bf16x2(res[0], res[1]), pack_bf16x2(res[2], res[3]));
  else *(f32x4*)out = res;
  if (d == 0) a.lse[(int64_t)(h0 + h) * a.n + job.x] = sum == 0.f ? -INFINITY : zero * 0.6931471805599453f + logf(sum);
}

template <typename T, int D, int COLS>
static void launch(const KCache& c, const PagedArgs& a, const PagedParts& parts, hipStream_t s) {
  if (c.page.d % Tile<T, D>::kGroup == 0) hipLaunchKernelGGL((paged_attn_kernel<T, D, COLS, true>), dim3(kWorkers), dim3(kPagedThreads), 0, s, c, a, parts);
  else hipLaunchKernelGGL((paged_attn_kernel<T, D, COLS, false>), dim3(kWorkers), dim3(kPagedThreads), 0, s, c, a, parts);
  hipLaunchKernelGGL((paged_join_kernel<T, D, COLS>), dim3(kWorkers, (unsigned)std::min(a.group, COLS)), dim3(kPagedThreads), 0, s, c, a, parts);
}
template <typename T, int COLS>
static void launch(const KCache& c, const PagedArgs& a, const PagedParts& parts, int d, hipStream_t s) {
  if (d == 128) launch<T, 128, COLS>(c, a, parts, s);
  else if (d == 64) launch<T, 64, COLS>(c, a, parts, s);
  else launch<T, 32, COLS>(c, a, parts, s);
}

// The largest set of heads of a launch: 8 columns where a weight's two parts lie side by side.
static int set_columns(int32_t dtype, int group) { return dtype == DCP_BF16 && group <= 8 ? 8 : kSetHeads; }
static size_t parts_bytes(int columns, int d) { return kWorkers * (sizeof(int4) + 2 * (size_t)columns * (sizeof(float2) + d * sizeof(float))); }

}  // namespace dcp

extern "C" size_t dcp_paged_attn_workspace_bytes(const dcp_cache_t* cache, int32_t n, int32_t hq) {
  if (!cache || n <= 0 || hq <= 0 || cache->hkv <= 0 || cache->d <= 0) return 0;
  return parts_bytes(set_columns(cache->dtype, hq / cache->hkv), cache->d);
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
  if (!workspace || workspace_bytes < dcp_paged_attn_workspace_bytes(cache, t.n, t.hq))
    return fail(DCP_ERR_WORKSPACE, "workspace is NULL or smaller than dcp_paged_attn_workspace_bytes");
  if (reinterpret_cast<uintptr_t>(workspace) & 255u) return fail(DCP_ERR_WORKSPACE, "workspace must be 256-byte aligned");
  const int64_t e = cache->dtype == DCP_BF16 ? 2 : 4;
  {
    const char *q0 = (const char*)t.q, *o0 = (const char*)t.out;
    const char* q1 = q0 + ((t.n - 1) * t.q_stride_t + (t.hq - 1) * t.q_stride_h + cache->d) * e;
    const char* o1 = o0 + ((t.n - 1) * t.o_stride_t + (t.hq - 1) * t.o_stride_h + cache->d) * e;
    if (q0 < o1 && o0 < q1) return fail(DCP_ERR_INVALID_ARG, "out overlaps q");
  }
  const int group = t.hq / c.hkv, columns = set_columns(cache->dtype, group);
  const int64_t sets = (int64_t)c.hkv * ((group + kSetHeads - 1) / kSetHeads);
  if (sets > (1 << 12)) return fail(DCP_ERR_UNSUPPORTED, "dcp_paged_attn_fwd covers at most 4 096 sets of 16 query heads on one KV head");
  const PagedArgs a{(const char*)t.q, (char*)t.out, t.lse, t.seqs, t.q_stride_t * e, t.q_stride_h * e, t.o_stride_t * e, t.o_stride_h * e,
                    t.n, t.hq, group, t.layer, t.window, t.sink, (int32_t)sets, t.softmax_scale * 1.44269504088896340736f};
  char* w = (char*)workspace;
  PagedParts parts;
  parts.joins = (int4*)w;
  parts.o = (float*)(w + kWorkers * sizeof(int4));
  parts.ml = (float2*)(parts.o + 2 * (size_t)kWorkers * columns * cache->d);
  hipStream_t s = (hipStream_t)stream;
  ProfScope ps(DCP_K_PAGED_ATTN, s);
  if (cache->dtype == DCP_F32) launch<float, 16>(c, a, parts, cache->d, s);
  else if (columns == 8) launch<bf16_t, 8>(c, a, parts, cache->d, s);
  else launch<bf16_t, 16>(c, a, parts, cache->d, s);
  DCP_HIP_TRY(hipGetLastError());
  return DCP_OK;
}
