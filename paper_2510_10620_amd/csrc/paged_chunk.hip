// Attention of the last tokens of every sequence over a paged key-value cache in 8 bits: pieces of prompts, tokens to be verified.
#include <climits>

#include "cache_internal.h"
#include "e4m3.h"
#include "tile_layout.h"

using namespace dcp;

namespace dcp {

namespace {

constexpr int kThreads = 256, kPlanThreads = 1024;
constexpr float kLazyChunk = 8.f;   // the running maximum is raised when a tile exceeds it by more than 2^8

__device__ __forceinline__ ChunkPlace chunk_place(const KCache& c, const ChunkArgs& a, int i, int32_t* seq) {
  const int s = a.seqs ? a.seqs[i] : i, code = a.status ? a.status[i] : DCP_PLACE_OK;
  *seq = code == DCP_PLACE_OK && c.is_seq(s) ? s : -1;
  return *seq < 0 ? ChunkPlace(0, 0, 0, 0) : ChunkPlace(a.cu[i], a.cu[i + 1], a.n_tokens, c.length(s));
}

// The tokens of a row tile of a place.
struct RowTile {
  int32_t r0, rows;   // first row, rows that are there
  int32_t lo, hi;     // positions of the first and the last
  __device__ __forceinline__ RowTile(const ChunkArgs& a, const ChunkPlace& p, int tile) {
    r0 = tile * kChunkRows;
    rows = min(p.count * (int)a.group.d - r0, kChunkRows);
    lo = p.pos + a.group.quot(r0);
    hi = p.pos + a.group.quot(r0 + rows - 1);
  }
};

// One workgroup lists the items with their key tiles and where every worker begins.  Bound by latency: two dependent trips to memory for the places, one for the workers.
__global__ __launch_bounds__(kPlanThreads) void chunk_plan_kernel(KCache c, ChunkArgs a, ChunkPlan plan) {
  __shared__ int32_t upto[DCP_CACHE_MAX_SEQS], wave_sum[kPlanThreads / 64];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  // inclusive sums over the workgroup, cut at cap
  auto block_sum = [&](int x, int cap, int* total) {
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const int y = __shfl_up(x, o);
      if (lane >= o) x = add_capped(x, y, cap);
    }
    __syncthreads();
    if (lane == 63) wave_sum[wave] = x;
    __syncthreads();
    int before = 0, all = 0;
#pragma unroll
    for (int w = 0; w < kPlanThreads / 64; w++) {
      if (w < wave) before = add_capped(before, wave_sum[w], cap);
      all = add_capped(all, wave_sum[w], cap);
    }
    *total = all;
    return add_capped(before, x, cap);
  };
  int n_items = 0, seq;
  for (int base = 0; base < a.n; base += kPlanThreads) {
    const int i = base + tid;
    int mine = 0, all;
    if (i < a.n) mine = (int)(((int64_t)chunk_place(c, a, i, &seq).count * a.group.d + kChunkRows - 1) / kChunkRows);
    const int x = block_sum(min(mine, a.max_items), a.max_items, &all);   // cu_new that is not ascending may name more rows than there are: what is beyond max_items is left out
    if (i < a.n) upto[i] = add_capped(n_items, x, a.max_items);
    n_items = add_capped(n_items, all, a.max_items);
  }
  __syncthreads();
  int tiles = 0;
  for (int base = 0; base < n_items; base += kPlanThreads) {
    const int i = base + tid;
    int count = 0, place = 0, tile = 0, all;
    if (i < n_items) {
      int lo = 0, hi = a.n - 1;   // the first place whose sum is above i
      while (lo < hi) {
        const int mid = (lo + hi) >> 1;
        if (upto[mid] > i) hi = mid;
        else lo = mid + 1;
      }
      place = lo;
      tile = i - (lo ? upto[lo - 1] : 0);
      const ChunkPlace p = chunk_place(c, a, place, &seq);
      const RowTile r(a, p, tile);
      count = chunk_tiles(r.lo, r.hi, a.window, a.sink, kChunkKeys).count;
    }
    const int x = block_sum(count, INT_MAX, &all);   // the host has seen to it that the sum is below 2^31
    if (i < n_items) plan.items[i] = make_int4(place, tile, count, tiles + x - count);
    tiles += all;
  }
  __syncthreads();
  if (tid == 0) *plan.head = make_int4(n_items, tiles, 0, 0);
  if (tid < kWorkers) {
    plan.joins[tid] = make_int4(0, -1, 0, 0);
    const Shares<kLogWorkers> sh(tiles * c.hkv);   // below 2^31: the host has seen to it
    if (tid < sh.workers) {
      const int at = sh.start(tid), head = (int)((uint32_t)at / (uint32_t)tiles), rel = at - head * tiles;
      int lo = 0, hi = n_items - 1;   // the last item that begins at or before it
      while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (plan.items[mid].w <= rel) lo = mid;
        else hi = mid - 1;
      }
      plan.starts[tid] = make_int4(head, lo, rel - plan.items[lo].w, 0);
    }
  }
}

// A wave's 32 rows: lane l has row l % 32 (both halves the same).
struct Row {
  bool real;
  int32_t pos, token, head;   // token: of the packed ones; head: query head
};

// O^T of a wave (lane = row, register 4 x + y of tile dt: number 32 dt + 8 x + 4 h + y) to out, and the LSE.
template <typename IO, int D>
__device__ __forceinline__ void store_row(const ChunkArgs& a, const Row& row, const f32x16* o, float m, float l, int dt0, int n_dt, bool lse) {
  const int lh = (threadIdx.x & 63) >> 5;
  if (!row.real) return;
  const float inv = l == 0.f ? 0.f : 1.f / l;
  char* out = a.out + row.token * a.o_st + row.head * a.o_sh;
  for (int dt = 0; dt < n_dt; dt++)
#pragma unroll
    for (int x = 0; x < 4; x++) {
      float v[4];
#pragma unroll
      for (int y = 0; y < 4; y++) v[y] = l == 0.f ? 0.f : o[dt][4 * x + y] * inv;
      const int at = 32 * (dt0 + dt) + 8 * x + 4 * lh;
      if constexpr (sizeof(IO) == 4) *(float4*)(out + 4 * at) = make_float4(v[0], v[1], v[2], v[3]);
      else *(uint2*)(out + 2 * at) = make_uint2(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]));
    }
  if (lse && lh == 0) a.lse[row.head * a.n_tokens + row.token] = l == 0.f ? -INFINITY : (m == -INFINITY ? 0.f : m) * 0.6931471805599453f + logf(l);
}

// The keys and values of a tile of 64 on their way into LDS: thread t has 4 (D 32: 2) words of 16 (8) codes at a time of key t / 4.
template <int D> struct Staged {
  static constexpr int kPieces = D >= 64 ? D / 64 : 1, kWords = D >= 64 ? 4 : 2;
  uint32_t k[kPieces][kWords], v[kPieces][kWords];
  uint32_t ks, vs;
  bool there;

  static __device__ __forceinline__ int key_of(int tid) { return tid >> 2; }
  // the page of the thread's key, -1: none
  static __device__ __forceinline__ int32_t look(const KCache& c, const int32_t* row, int32_t base, int32_t end) {
    const int32_t j = base + key_of(threadIdx.x);
    return j < end ? row[c.page.quot(j)] : -1;
  }
  __device__ __forceinline__ void load(const KCache& c, int32_t entry, int32_t base, int hk) {
    const int32_t j = base + key_of(threadIdx.x);
    there = c.is_page(entry);
    const int32_t page = there ? entry : 0, slot = there ? c.page.rem(j, c.page.quot(j)) : 0;
    const char* kp = c.k + page * c.k_sp + slot * c.k_st + hk * c.k_sh + (threadIdx.x & 3) * (kWords * 4);
    const char* vp = c.v + page * c.v_sp + slot * c.v_st + hk * c.v_sh + (threadIdx.x & 3) * (kWords * 4);
#pragma unroll
    for (int x = 0; x < kPieces; x++) {
      if constexpr (kWords == 4) {
        const uint4 a = *(const uint4*)(kp + 64 * x), b = *(const uint4*)(vp + 64 * x);
        k[x][0] = a.x; k[x][1] = a.y; k[x][2] = a.z; k[x][3] = a.w;
        v[x][0] = b.x; v[x][1] = b.y; v[x][2] = b.z; v[x][3] = b.w;
      } else {
        const uint2 a = *(const uint2*)kp, b = *(const uint2*)vp;
        k[x][0] = a.x; k[x][1] = a.y;
        v[x][0] = b.x; v[x][1] = b.y;
      }
    }
    const int64_t at = c.scale_at(page, slot) + hk;
    ks = c.k_scale[at];
    vs = c.v_scale[at];
  }
  // As bf16 numbers; a key that is not there as zeros.  Sixteen lanes write 16 chunks of 16 bytes in four rows at a time, which fall into all banks if every
  // other row (D 64: pair of rows) writes its odd chunks first.
  // CLEAN: what is not finite is left out (written as 0).
  template <bool CLEAN> static __device__ __forceinline__ void write(char* tile, const uint32_t (&w)[kPieces][kWords], uint32_t scale) {
    typedef TileLayout<D> L;
    const float factor = scale_factor(scale);
    const int key = key_of(threadIdx.x), part = threadIdx.x & 3, odd = D == 128 ? key & 1 : (key >> 1) & 1;
    auto put = [&](int chunk, uint32_t a, uint32_t b) {
      uint32_t n[4] = {e4m3_to_bf16x2<false>(a, factor), e4m3_to_bf16x2<true>(a, factor), e4m3_to_bf16x2<false>(b, factor), e4m3_to_bf16x2<true>(b, factor)};
      if constexpr (CLEAN) {
#pragma unroll
        for (int y = 0; y < 4; y++) n[y] = ((n[y] & 0x7f80u) == 0x7f80u ? 0u : n[y] & 0xffffu) | ((n[y] & 0x7f800000u) == 0x7f800000u ? 0u : n[y] & 0xffff0000u);
      }
      *(uint4*)(tile + L::off(key, chunk)) = make_uint4(n[0], n[1], n[2], n[3]);
    };
#pragma unroll
    for (int x = 0; x < kPieces; x++) {
      if constexpr (kWords == 4) {
        put(8 * x + 2 * part + odd, odd ? w[x][2] : w[x][0], odd ? w[x][3] : w[x][1]);
        put(8 * x + 2 * part + (odd ^ 1), odd ? w[x][0] : w[x][2], odd ? w[x][1] : w[x][3]);
      } else {
        put(part, w[x][0], w[x][1]);
      }
    }
  }
  // whether a number of V may not be finite as bf16: a NaN, or a scale that reaches 2^128
  __device__ __forceinline__ bool may_not_be_finite() const {
    uint32_t bad = 0;
#pragma unroll
    for (int x = 0; x < kPieces; x++)
#pragma unroll
      for (int y = 0; y < kWords; y++) bad |= ((v[x][y] & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u;
    return there & (bad != 0 || vs >= 247);
  }
  __device__ __forceinline__ void drop_missing() {
#pragma unroll
    for (int x = 0; x < kPieces; x++)
#pragma unroll
      for (int y = 0; y < kWords; y++) {
        k[x][y] = there ? k[x][y] : 0u;
        v[x][y] = there ? v[x][y] : 0u;
      }
  }
};

}  // namespace

// O = sum_j exp(s_j - m) v_j / l, LSE = m + ln l as for one token, in one pass over a row tile's key tiles of 64, which the four waves of 32 rows share in LDS as bf16
// numbers: codes and scales become them without a rounding on the way.  Scores are computed transposed, S^T = K Q^T, so that a lane owns a row, and P^T is the B operand
// of O^T += V^T P^T as it stands (see mfma_common.h).  bf16: weights are rounded to bf16, their sum is not.  fp32: queries and weights go in as three bf16 parts.
template <typename IO, int D>
__global__ __launch_bounds__(kThreads, sizeof(IO) == 4 ? 1 : 2) void chunk_kernel(KCache c, ChunkArgs a, ChunkPlan plan) {
  typedef TileLayout<D> L;
  constexpr int kParts = sizeof(IO) == 4 ? 3 : 1;
  __shared__ __attribute__((aligned(1024))) char stages[4 * L::kBytes];   // two stages, each [K tile | V tile]
  __shared__ __attribute__((aligned(8))) uint16_t s_there[2][4];
  __shared__ int32_t s_odd[2];   // by turns: the last piece of work that met a number of V that is not finite where not every row sees it
  const int tid = threadIdx.x, lane = tid & 63, wave = uni(tid >> 6), li = lane & 31, lh = lane >> 5;
  // Workgroups go to the 8 XCDs round-robin: an XCD's workers have neighbouring shares, so that its L2 serves their keys.
  const int w = (blockIdx.x & 7) * (kWorkers / 8) + (blockIdx.x >> 3);
  const int4 head = *plan.head;
  const int n_items = uni(head.x), tiles = uni(head.y);
  if (n_items == 0) return;
  const Shares<kLogWorkers> sh(tiles * c.hkv);
  if (w >= sh.workers) return;
  const int4 start = plan.starts[w];
  int hk = uni(start.x), item = uni(start.y), t0 = uni(start.z), left = sh.start(w + 1) - sh.start(w);
  Frags<D> fa;
  fa.init(lane);
  if (tid < 2) s_odd[tid] = -1;
  __syncthreads();

  for (int piece = 0; left > 0; piece++) {
    const int4 it = plan.items[item];
    const int place = uni(it.x), count = uni(it.z);
    int32_t seq;
    const ChunkPlace p = chunk_place(c, a, place, &seq);
    seq = uni(seq);
    const RowTile rt(a, p, uni(it.y));
    const int lo = uni(rt.lo), hi = uni(rt.hi), rows = uni(rt.rows);
    const KeyTiles keys = chunk_tiles(lo, hi, a.window, a.sink, kChunkKeys);
    const int t1 = min(count, t0 + left);
    const int32_t* table = c.row(seq);

    Row row;
    const int r = min(wave * 32 + li, rows - 1), at = rt.r0 + r, token = a.group.quot(at);
    row.real = wave * 32 + li < rows;
    row.pos = p.pos + token;
    row.token = p.first + token;
    row.head = hk * (int)a.group.d + at - token * (int)a.group.d;
    const bool works = wave * 32 < rows;
    const int w_lo = uni(row.pos), w_hi = uni(__shfl(row.pos, 31));   // rows are in the order of their positions
    // the row's keys: [0, head_end) and [low, pos]
    const int low = a.window > 0 ? max(0, row.pos + 1 - a.window) : 0, head_end = min(a.sink, low);

    bf16x8 q[kParts][L::KS];
    {
      const char* qp = a.q + row.token * a.q_st + row.head * a.q_sh;
#pragma unroll
      for (int ks = 0; ks < L::KS; ks++) {
        if constexpr (kParts == 1) {
          q[0][ks] = as_frag(*(const uint4*)(qp + 2 * (16 * ks + 8 * lh)));
        } else {
          const float4 u = *(const float4*)(qp + 4 * (16 * ks + 8 * lh)), v = *(const float4*)(qp + 4 * (16 * ks + 8 * lh + 4));
          float x[8] = {u.x, u.y, u.z, u.w, v.x, v.y, v.z, v.w};
#pragma unroll
          for (int y = 0; y < 8; y++) x[y] = x[y] == x[y] ? x[y] : NAN;   // whose upper half is NaN too
#pragma unroll
          for (int part = 0; part < 3; part++) {
            uint32_t words[4];
#pragma unroll
            for (int y = 0; y < 4; y++) words[y] = __builtin_amdgcn_perm(__float_as_uint(x[2 * y + 1]), __float_as_uint(x[2 * y]), 0x07060302u);
#pragma unroll
            for (int y = 0; y < 8; y++) x[y] = fabsf(x[y]) < INFINITY ? x[y] - __uint_as_float(__float_as_uint(x[y]) & 0xffff0000u) : 0.f;   // what is not finite is one part
            q[part][ks] = as_frag(make_uint4(words[0], words[1], words[2], words[3]));
          }
        }
      }
    }
    f32x16 o[L::DT];
#pragma unroll
    for (int dt = 0; dt < L::DT; dt++)
#pragma unroll
      for (int x = 0; x < 16; x++) o[dt][x] = 0.f;
    float m = -INFINITY, l = 0.f;   // m in units of the scores

    Staged<D> st;
    auto base_of = [&](int x) { return keys.tile_at(x) * kChunkKeys; };
    auto entry_of = [&](int x) { return x < t1 ? Staged<D>::look(c, table, base_of(x), keys.len) : -1; };
    // every row of the workgroup sees all keys of the tile that are there
    auto seen_by_all = [&](int base) { return base + kChunkKeys - 1 <= lo && (a.window <= 0 || hi - base < a.window || base + kChunkKeys <= a.sink); };
    auto publish = [&](int stage, int base) {
      st.drop_missing();
      char* tile = stages + stage * 2 * L::kBytes;
      Staged<D>::template write<false>(tile, st.k, st.ks);
      // Where some row does not see every key, 0 x V would carry an infinity or a NaN to it: they are left out here and added at the end.
      if (!seen_by_all(base) && __any(st.may_not_be_finite())) {
        Staged<D>::template write<true>(tile + L::kBytes, st.v, st.vs);
        if (lane == 0) s_odd[piece & 1] = piece;
      } else {
        Staged<D>::template write<false>(tile + L::kBytes, st.v, st.vs);
      }
      const uint64_t there = __ballot(st.there);   // four lanes a key
      uint32_t bits = 0;
#pragma unroll
      for (int x = 0; x < 16; x++) bits |= (uint32_t)(there >> (4 * x) & 1) << x;
      if (lane == 0) s_there[stage][wave] = (uint16_t)bits;
    };
    int32_t entry = entry_of(t0), next = entry_of(t0 + 1);
    st.load(c, entry, base_of(t0), hk);
    publish(0, base_of(t0));
    __syncthreads();
    for (int x = t0; x < t1; x++) {
      const int stage = (x - t0) & 1, base = base_of(x);
      const bool more = x + 1 < t1;
      if (more) st.load(c, next, base_of(x + 1), hk);
      next = entry_of(x + 2);
      if (works) {
        const char* k_lds = stages + stage * 2 * L::kBytes;
        const char* v_lds = k_lds + L::kBytes;
        const uint2 bits = *(const uint2*)s_there[stage];
        const uint64_t there = (uint32_t)uni((int)bits.x) | (uint64_t)(uint32_t)uni((int)bits.y) << 32;
        const bool none = base > w_hi || (a.window > 0 && w_lo - (base + kChunkKeys - 1) >= a.window && base >= a.sink);
        const bool all = there == ~uint64_t(0) && base + kChunkKeys - 1 <= w_lo && (a.window <= 0 || w_hi - base < a.window || base + kChunkKeys <= a.sink);
        if (!none) {
          f32x16 s[2];
#pragma unroll
          for (int kt = 0; kt < 2; kt++) {
#pragma unroll
            for (int y = 0; y < 16; y++) s[kt][y] = 0.f;
#pragma unroll
            for (int ks = 0; ks < L::KS; ks++) {
              const bf16x8 kf = fa.rows(k_lds + 32 * kt * L::kRow, ks);
#pragma unroll
              for (int part = 0; part < kParts; part++) s[kt] = mfma(kf, q[part][ks], s[kt]);
            }
          }
          if (!all) {
            auto below = [](int x) { return x <= 0 ? uint64_t(0) : x >= 64 ? ~uint64_t(0) : (uint64_t(1) << x) - 1; };
            const uint64_t sees = ((below(row.pos + 1 - base) & ~below(low - base)) | below(head_end - base)) & there;
            const uint32_t seen[2] = {(uint32_t)sees >> (4 * lh), (uint32_t)(sees >> 32) >> (4 * lh)};   // bit 8 (y / 4) + y % 4: the key of s[kt][y]
#pragma unroll
            for (int kt = 0; kt < 2; kt++)
#pragma unroll
              for (int y = 0; y < 16; y++) s[kt][y] = seen[kt] >> (8 * (y / 4) + y % 4) & 1 ? s[kt][y] : -INFINITY;
          }
          float mx = fmaxf(s[0][0], s[1][0]);
#pragma unroll
          for (int y = 1; y < 16; y++) mx = fmaxf(fmaxf(mx, s[0][y]), s[1][y]);
          mx = xhalf_max(mx);
          const bool raise = (mx - m) * a.scale_log2e > kLazyChunk;
          const float m_new = raise ? mx : m, m_use = m_new == -INFINITY ? 0.f : m_new, mc = m_use * a.scale_log2e;
          if (__any(raise)) {
            const float alpha = raise ? __builtin_amdgcn_exp2f((m - m_use) * a.scale_log2e) : 1.f;
            l *= alpha;
#pragma unroll
            for (int dt = 0; dt < L::DT; dt++)
#pragma unroll
              for (int y = 0; y < 16; y++) o[dt][y] *= alpha;
          }
          m = m_new;
#pragma unroll
          for (int kt = 0; kt < 2; kt++) {
            float sum = 0.f;
#pragma unroll
            for (int y = 0; y < 16; y++) {
              s[kt][y] = __builtin_amdgcn_exp2f(fmaf(s[kt][y], a.scale_log2e, -mc));
              sum += s[kt][y];
            }
            l += sum;
#pragma unroll
            for (int cc = 0; cc < 2; cc++) {
              bf16x8 pf[kParts];
              if constexpr (kParts == 1) pf[0] = pack_frag(s[kt], cc);
              else pack_split(s[kt], cc, pf);
#pragma unroll
              for (int dt = 0; dt < L::DT; dt++) {
                const bf16x8 vf = fa.cols(v_lds, 2 * kt + cc, dt);
#pragma unroll
                for (int part = 0; part < kParts; part++) o[dt] = mfma(vf, pf[part], o[dt]);
              }
            }
          }
        }
      }
      if (more) publish(stage ^ 1, base_of(x + 1));
      __syncthreads();
    }

    if (works) {
      l = xhalf_sum(l);
      const float m2 = m * a.scale_log2e;   // in units of log2
      if (t0 == 0 && t1 == count) {
        store_row<IO, D>(a, row, o, m2, l, 0, L::DT, true);
      } else {
        const int slot = 2 * w + (t0 == 0);
        float* part = plan.o + ((int64_t)slot * (kChunkRows / 32) + wave) * (32 * D);
#pragma unroll
        for (int dt = 0; dt < L::DT; dt++)
#pragma unroll
          for (int y = 0; y < 4; y++)
            *(float4*)(part + ((dt * 4 + y) * 64 + lane) * 4) = make_float4(o[dt][4 * y], o[dt][4 * y + 1], o[dt][4 * y + 2], o[dt][4 * y + 3]);
        if (lh == 0) plan.ml[slot * kChunkRows + wave * 32 + li] = make_float2(m2, l);
      }
      if (s_odd[piece & 1] == piece) {   // rare: written by the lane that wrote the number before, straight into memory
        char* out = a.out + row.token * a.o_st + row.head * a.o_sh;
        float* part = plan.o + ((int64_t)(2 * w + (t0 == 0)) * (kChunkRows / 32) + wave) * (32 * D);
        const bool done = t0 == 0 && t1 == count;
        for (int x = t0; x < t1; x++) {
          const int base = base_of(x);
          if (seen_by_all(base)) continue;
          for (int j = base; j < min(base + kChunkKeys, keys.len); j++) {
            const int32_t q_page = c.page.quot(j), page = table[q_page], slot = c.page.rem(j, q_page);
            if (!c.is_page(page)) continue;
            const char* v = c.v + page * c.v_sp + slot * c.v_st + hk * c.v_sh;
            const float factor = scale_factor(c.v_scale[c.scale_at(page, slot) + hk]);
            const bool sees = row.real & (j <= row.pos) & ((j >= low) | (j < head_end));
            for (int d0 = 0; d0 < D; d0 += 64) {
              const uint32_t code = d0 + lane < D ? *(const uint8_t*)(v + d0 + lane) : 0u;
              const uint32_t number = e4m3_to_bf16x2<false>(code, factor) << 16;
              for (uint64_t left_over = __ballot((number & 0x7f800000u) == 0x7f800000u); left_over; left_over &= left_over - 1) {
                const int at_lane = __ffsll((unsigned long long)left_over) - 1, d = d0 + at_lane;
                const float add = __shfl(__uint_as_float(number), at_lane);
                if (!sees || lh != (d >> 2 & 1)) continue;
                if (!done) part[((d / 32 * 4 + d / 8 % 4) * 64 + lane) * 4 + d % 4] += add;
                else if constexpr (sizeof(IO) == 4) *(float*)(out + 4 * d) += add;
                else *(uint16_t*)(out + 2 * d) = f32_to_bf16(bf16_to_f32(*(const uint16_t*)(out + 2 * d)) + add);
              }
            }
          }
        }
      }
    }
    if (t0 == 0 && t1 < count && tid == 0) {
      const int begin = hk * tiles + uni(it.w);
      plan.joins[w] = make_int4(hk, item, w, sh.worker_of(begin + count - 1));
    }
    left -= t1 - t0;
    t0 = 0;
    if (++item == n_items) { item = 0; hk++; }
  }
}

// Joins the parts of an item that several workers shared: a wave takes 32 rows and 32 numbers of each.  Bound by latency where there are few.
template <typename IO, int D>
__global__ __launch_bounds__(kThreads) void chunk_join_kernel(KCache c, ChunkArgs a, ChunkPlan plan) {
  if (plan.head->x == 0) return;
  const int4 job = plan.joins[blockIdx.x];
  if (job.y < 0) return;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, li = lane & 31, dt = blockIdx.y;
  const int4 it = plan.items[job.y];
  int32_t seq;
  const ChunkPlace p = chunk_place(c, a, it.x, &seq);
  const RowTile rt(a, p, it.y);
  if (wave * 32 >= rt.rows) return;
  Row row;
  const int at = rt.r0 + min(wave * 32 + li, rt.rows - 1), token = a.group.quot(at);
  row.real = wave * 32 + li < rt.rows;
  row.token = p.first + token;
  row.head = job.x * (int)a.group.d + at - token * (int)a.group.d;
  float m = -INFINITY, l = 0.f;
  f32x16 o;
#pragma unroll
  for (int y = 0; y < 16; y++) o[y] = 0.f;
  for (int x = job.z; x <= job.w; x++) {
    const int slot = 2 * x + (x == job.z);
    const float2 ml = plan.ml[slot * kChunkRows + wave * 32 + li];
    const float* part = plan.o + ((int64_t)slot * (kChunkRows / 32) + wave) * (32 * D) + dt * 1024;
    const float m2 = fmaxf(m, ml.x), zero = m2 == -INFINITY ? 0.f : m2;
    const float f = __builtin_amdgcn_exp2f(m - zero), fx = __builtin_amdgcn_exp2f(ml.x - zero);
    l = l * f + ml.y * fx;
#pragma unroll
    for (int y = 0; y < 4; y++) {
      const float4 u = *(const float4*)(part + (y * 64 + lane) * 4);
      o[4 * y] = o[4 * y] * f + u.x * fx;
      o[4 * y + 1] = o[4 * y + 1] * f + u.y * fx;
      o[4 * y + 2] = o[4 * y + 2] * f + u.z * fx;
      o[4 * y + 3] = o[4 * y + 3] * f + u.w * fx;
    }
    m = m2;
  }
  store_row<IO, D>(a, row, &o, m, l, dt, 1, dt == 0);
}

namespace {
template <typename IO, int D> void launch_d(const KCache& c, const ChunkArgs& a, const ChunkPlan& plan, hipStream_t s) {
  hipLaunchKernelGGL((chunk_kernel<IO, D>), dim3(kWorkers), dim3(kThreads), 0, s, c, a, plan);
  hipLaunchKernelGGL((chunk_join_kernel<IO, D>), dim3(kWorkers, D / 32), dim3(kThreads), 0, s, c, a, plan);
}
template <typename IO> void launch_io(int32_t d, const KCache& c, const ChunkArgs& a, const ChunkPlan& plan, hipStream_t s) {
  if (d == 128) launch_d<IO, 128>(c, a, plan, s);
  else if (d == 64) launch_d<IO, 64>(c, a, plan, s);
  else launch_d<IO, 32>(c, a, plan, s);
}
}  // namespace

void launch_chunk(int32_t d, const KCache& c, const ChunkArgs& a, const ChunkPlan& plan, hipStream_t s) {
  hipLaunchKernelGGL(chunk_plan_kernel, dim3(1), dim3(kPlanThreads), 0, s, c, a, plan);
  if (c.io_bytes == 4) launch_io<float>(d, c, a, plan, s);
  else launch_io<bf16_t>(d, c, a, plan, s);
}

}  // namespace dcp
