// Attention of the last tokens of every sequence over a paged key-value cache in 8 bits: pieces of prompts, tokens to be verified.
#include <climits>

#include "paged_chunk.h"
#include "tile_layout.h"

using namespace dcp;

namespace dcp {

namespace {

constexpr int kThreads = 256, kPlanThreads = 1024;
constexpr float kLazyChunk = 8.f;   // the running maximum is raised when a tile exceeds it by more than 2^8

// One workgroup lists the items with their key tiles and where every worker begins.  Bound by latency, 5 to 8 us: two dependent trips to memory for the places, a search for the workers.
__global__ __launch_bounds__(kPlanThreads) void chunk_plan_kernel(KCache c, ChunkArgs a, ChunkPlan plan) {
  // In LDS what is looked up: of every place the items up to it, of the first kPlanThreads places what they have, of the first kPlanThreads items the key tiles before them.
  __shared__ int32_t upto[DCP_CACHE_MAX_SEQS], wave_sum[kPlanThreads / 64], s_before[kPlanThreads];
  __shared__ int4 s_place[kPlanThreads];
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
    if (i < a.n) {
      const ChunkPlace p = chunk_place(c, a, i, &seq);
      mine = (int)(((int64_t)p.count * a.group.d + a.rows - 1) / a.rows);
      if (base == 0) s_place[tid] = make_int4(seq, p.first, p.pos, p.count);
    }
    const int x = block_sum(min(mine, a.max_items), a.max_items, &all);   // cu_new that is not ascending may name more rows than there are: what is beyond max_items is left out
    if (i < a.n) upto[i] = add_capped(n_items, x, a.max_items);
    n_items = add_capped(n_items, all, a.max_items);
  }
  __syncthreads();
  int tiles = 0;
  for (int base = 0; base < n_items; base += kPlanThreads) {
    const int i = base + tid;
    int all;
    ChunkItem item{};
    if (i < n_items) {
      int lo = 0, hi = a.n - 1;   // the first place whose sum is above i
      while (lo < hi) {
        const int mid = (lo + hi) >> 1;
        if (upto[mid] > i) hi = mid;
        else lo = mid + 1;
      }
      const int place = lo, tile = i - (lo ? upto[lo - 1] : 0);
      if (place < kPlanThreads) {
        const int4 p = s_place[place];
        item = ChunkItem{p.x, p.y, p.z, p.w * (int)a.group.d, tile * a.rows, 0, 0, 0};
      } else {
        const ChunkPlace p = chunk_place(c, a, place, &seq);
        item = ChunkItem{seq, p.first, p.pos, p.count * (int)a.group.d, tile * a.rows, 0, 0, 0};
      }
      item.tiles = chunk_tiles(item.pos + a.group.quot(item.row0), item.pos + a.group.quot(min(item.row0 + a.rows, item.rows) - 1), a.window, a.sink, a.tile).count;
    }
    const int x = block_sum(item.tiles, INT_MAX, &all);   // the host has seen to it that the sum is below 2^31
    if (i < n_items) {
      item.before = tiles + x - item.tiles;
      plan.items[i] = item;
      if (base == 0) s_before[tid] = item.before;
    }
    tiles += all;
  }
  __syncthreads();
  if (tid == 0) *plan.head = make_int4(n_items, tiles, 0, 0);
  if (tid < kWorkers) {
    plan.joins[tid] = ChunkJoin{0, 0, -1, 0, 0, 0, 0, 0};
    const ChunkShares sh(tiles * c.hkv);   // below 2^31: the host has seen to it
    if (tid < sh.workers) {
      const int at = sh.start(tid), head = (int)((uint32_t)at / (uint32_t)tiles), rel = at - head * tiles;
      int lo = 0, hi = n_items - 1;   // the last item that begins at or before it
      while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if ((mid < kPlanThreads ? s_before[mid] : plan.items[mid].before) <= rel) lo = mid;
        else hi = mid - 1;
      }
      plan.starts[tid] = make_int4(head, lo, rel - (lo < kPlanThreads ? s_before[lo] : plan.items[lo].before), 0);
    }
  }
}

// O^T of a wave (lane = row, register 4 x + y of tile dt: number 32 dt + 8 x + 4 h + y) times `by`, as numbers of IO.
template <typename IO, int D>
__device__ __forceinline__ void store_row(char* out, const f32x16 (&o)[D / 32], float by) {
  const int lh = (threadIdx.x & 63) >> 5;
#pragma unroll
  for (int dt = 0; dt < D / 32; dt++)
#pragma unroll
    for (int x = 0; x < 4; x++) {
      float v[4];
#pragma unroll
      for (int y = 0; y < 4; y++) v[y] = by == 0.f ? 0.f : o[dt][4 * x + y] * by;
      const int at = 32 * dt + 8 * x + 4 * lh;
      if constexpr (sizeof(IO) == 4) *(float4*)(out + 4 * at) = make_float4(v[0], v[1], v[2], v[3]);
      else *(uint2*)(out + 2 * at) = make_uint2(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]));
    }
}

// Registers 8 c .. 8 c + 7 of a tile of weights as three bf16 operands.
__device__ __forceinline__ void pack_weights(const f32x16& s, int c, bf16x8 (&part)[3]) {
  float x[8];
#pragma unroll
  for (int y = 0; y < 8; y++) x[y] = s[8 * c + y];
#pragma unroll
  for (int k = 0; k < 3; k++) {
    uint32_t w[4];
#pragma unroll
    for (int y = 0; y < 4; y++) w[y] = __builtin_amdgcn_perm(__float_as_uint(x[2 * y + 1]), __float_as_uint(x[2 * y]), 0x07060302u);
    part[k] = as_frag(make_uint4(w[0], w[1], w[2], w[3]));
#pragma unroll
    for (int y = 0; y < 8; y++) x[y] = left_of_weight(x[y], s[8 * c + y]);
  }
}

// The keys and values of a tile of 64 on their way into LDS: thread t has 4 (D 32: 2) words of 16 (8) codes at a time of key t / 4.
template <int D> struct Staged {
  static constexpr int kPieces = D >= 64 ? D / 64 : 1, kWords = D >= 64 ? 4 : 2;
  uint32_t k[kPieces][kWords], v[kPieces][kWords];
  uint8_t ks, vs;   // scales
  bool there;

  static __device__ __forceinline__ int key_of(int tid) { return tid >> 2; }
  // The table's entry for the thread's key, to be handed to load(): nothing looks at it before, so that nothing waits for it.
  static __device__ __forceinline__ int32_t look(const KCache& c, const int32_t* row, int32_t base, int32_t end) {
    return row[c.page.quot(max(min(base + key_of((int)threadIdx.x), end - 1), 0))];
  }
  // end: keys of the sequence, 0 where there is no such tile
  __device__ __forceinline__ void load(const KCache& c, int32_t entry, int32_t base, int32_t end, int hk) {
    const int32_t j = base + key_of(threadIdx.x);
    there = (j < end) & c.is_page(entry);
    const int32_t in_page = c.page.rem(j, c.page.quot(j)), page = there ? entry : 0, slot = there ? in_page : 0;
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
  static __device__ __forceinline__ void write(char* tile, const uint32_t (&w)[kPieces][kWords], uint32_t scale) {
    typedef TileLayout<D> L;
    const float factor = scale_factor(scale);
    const int key = key_of(threadIdx.x), part = threadIdx.x & 3, odd = D == 128 ? key & 1 : (key >> 1) & 1;
    auto put = [&](int chunk, uint32_t a, uint32_t b) {
      *(uint4*)(tile + L::off(key, chunk)) =
          make_uint4(e4m3_to_bf16x2<false>(a, factor), e4m3_to_bf16x2<true>(a, factor), e4m3_to_bf16x2<false>(b, factor), e4m3_to_bf16x2<true>(b, factor));
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
  // Leaves out what is not finite of V; whether anything was.
  __device__ __forceinline__ bool clean() {
    uint32_t bad = 0;
#pragma unroll
    for (int x = 0; x < kPieces; x++)
#pragma unroll
      for (int y = 0; y < kWords; y++) {
        const uint32_t signs = not_finite(v[x][y], vs);
        v[x][y] = without(v[x][y], signs);
        bad |= signs;
      }
    return bad != 0;
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
// of O^T += V^T P^T as it stands (see mfma_common.h).  bf16: weights are rounded to bf16, their sum is not, as in dcp_block_attn_fwd: beside the
// rounding of the output the error against 64 bits grows from 1.66e-3 to 2.3e-3 of the norm.  In two parts, as the walk with keys in registers has them, it did not, but the case below took
// 1 453 us instead of 1 122, seven prompts of up to 1 500 tokens with a window of 1 024, 16/4 heads of 64, 99 instead of 86.  fp32: queries and weights go in as three bf16 parts (3 160 us).
// Bound by issue: 1 799 tokens behind 30 720, 32/8 heads of 128, 1 126 us in a graph, 829 TFLOP/s; 9.8 vector instructions a matrix instruction (softmax; the conversion of codes, a tenth; addresses),
// matrix pipes busy 36 % of the time, vector units 49 %.  Two workgroups on a CU (fp32: one); with heads of 64 three gained nothing.
template <typename IO, int D>
__global__ __launch_bounds__(kThreads, sizeof(IO) == 4 ? 1 : 2) void chunk_kernel(KCache c, ChunkArgs a, ChunkPlan plan) {
  typedef TileLayout<D> L;
  constexpr int kParts = sizeof(IO) == 4 ? 3 : 1;
  __shared__ __attribute__((aligned(1024))) char stages[4 * L::kBytes];   // two stages, each [K tile | V tile]
  __shared__ __attribute__((aligned(8))) uint16_t s_there[2][4];
  __shared__ int32_t s_odd[2];   // by turns: the last piece of work that met a number of V that is not finite where not every row sees it
  const int tid = threadIdx.x, lane = tid & 63, wave = uni(tid >> 6), li = lane & 31, lh = lane >> 5;
  const int4 head = *plan.head;
  const int n_items = uni(head.x), tiles = uni(head.y);
  if (n_items == 0) return;
  const ChunkShares sh(tiles * c.hkv);
  const int w = sh.worker(blockIdx.x);
  if (w >= sh.workers) return;
  const int4 start = plan.starts[w];
  int hk = uni(start.x), item = uni(start.y), t0 = uni(start.z), left = sh.start(w + 1) - sh.start(w);
  Frags<D> fa;
  fa.init(lane);
  if (tid < 2) s_odd[tid] = -1;
  __syncthreads();

  for (int piece = 0; left > 0; piece++) {
    const ChunkItem it = plan.items[item];
    const int seq = uni(it.seq), count = uni(it.tiles), row0 = uni(it.row0), rows = uni(min(it.rows - row0, kChunkRows)), pos0 = uni(it.pos);
    const int lo = pos0 + a.group.quot(row0), hi = pos0 + a.group.quot(row0 + rows - 1);   // positions of the item's first and last token
    const KeyTiles keys = chunk_tiles(lo, hi, a.window, a.sink, kChunkKeys);
    const int t1 = min(count, t0 + left);
    const int32_t* table = c.row(seq);

    const ChunkRow row(a, hk, it.first, pos0, row0 + rows, row0 + wave * 32 + li);
    const bool works = wave * 32 < rows;
    const int w_lo = uni(row.pos), w_hi = uni(__shfl(row.pos, 31));   // rows are in the order of their positions

    bf16x8 q[kParts][L::KS];
    {
      const char* qp = a.q + row.token * a.q_st + row.head * a.q_sh;
#pragma unroll
      for (int ks = 0; ks < L::KS; ks++) {
        if constexpr (kParts == 1) {
          q[0][ks] = as_frag(*(const uint4*)(qp + 2 * (16 * ks + 8 * lh)));
        } else {
          const float4 u = *(const float4*)(qp + 4 * (16 * ks + 8 * lh)), v = *(const float4*)(qp + 4 * (16 * ks + 8 * lh + 4));
          float x[8] = {u.x, u.y, u.z, u.w, v.x, v.y, v.z, v.w}, all[8];
#pragma unroll
          for (int y = 0; y < 8; y++) all[y] = x[y] = x[y] == x[y] ? x[y] : NAN;   // whose upper half is NaN too
#pragma unroll
          for (int part = 0; part < 3; part++) {
            uint32_t words[4];
#pragma unroll
            for (int y = 0; y < 4; y++) words[y] = __builtin_amdgcn_perm(__float_as_uint(x[2 * y + 1]), __float_as_uint(x[2 * y]), 0x07060302u);
#pragma unroll
            for (int y = 0; y < 8; y++) x[y] = left_of_query(x[y], all[y]);
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

    Staged<D> st0, st1;   // two tiles on their way
    auto base_of = [&](int x) { return keys.tile_at(x) * kChunkKeys; };
    auto end_of = [&](int x) { return x < t1 ? keys.len : 0; };
    auto entry_of = [&](int x) { return Staged<D>::look(c, table, x < t1 ? base_of(x) : 0, end_of(x)); };
    // every row of the workgroup sees all keys of the tile that are there
    auto seen_by_all = [&](int base) { return base + kChunkKeys - 1 <= lo && (a.window <= 0 || hi - base < a.window || base + kChunkKeys <= a.sink); };
    auto publish = [&](Staged<D>& st, int stage, int base) {
      st.drop_missing();
      char* tile = stages + stage * 2 * L::kBytes;
      // Where some row does not see every key, 0 x V would carry an infinity or a NaN to it: they are left out here and added at the end.
      if (!seen_by_all(base) && __any(st.clean()) && lane == 0) s_odd[piece & 1] = piece;
      Staged<D>::write(tile, st.k, st.ks);
      Staged<D>::write(tile + L::kBytes, st.v, st.vs);
      const uint64_t there = __ballot(st.there);   // four lanes a key
      uint32_t bits = 0;
#pragma unroll
      for (int x = 0; x < 16; x++) bits |= (uint32_t)(there >> (4 * x) & 1) << x;
      if (lane == 0) s_there[stage][wave] = (uint16_t)bits;
    };
    // While tile x is walked, tile x + 1 comes and tile x + 2 is asked for, whose entries of the table were before tile x + 1 was.  Loads come back in the
    // order in which they were asked for, and what waits for one waits for those before it: so nothing here waits for a load of the same step, as long as every
    // step asks for the same number (past the last tile: the first entry and the first key of the cache).
    int32_t entry = entry_of(t0), next = entry_of(t0 + 1);
    st0.load(c, entry, base_of(t0), end_of(t0), hk);
    entry = entry_of(t0 + 2);
    st1.load(c, next, t0 + 1 < t1 ? base_of(t0 + 1) : 0, end_of(t0 + 1), hk);
    publish(st0, 0, base_of(t0));
    __syncthreads();
    auto ask = [&](int x, Staged<D>& free) {
      const int32_t after = entry_of(x + 3);
      free.load(c, entry, x + 2 < t1 ? base_of(x + 2) : 0, end_of(x + 2), hk);
      entry = after;
    };
    auto walk = [&](int x, int stage) {
      const int base = base_of(x);
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
            const uint64_t sees = ((below(row.pos + 1 - base) & ~below(row.low - base)) | below(row.head_end - base)) & there;
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
          const float m_new = raise ? mx : m, m_use = m_new == -INFINITY ? 0.f : m_new;
          float mc = m_use * a.scale_log2e;
          if (__any(raise)) {
            const float alpha = raise ? __builtin_amdgcn_exp2f((m - m_use) * a.scale_log2e) : 1.f;
            l *= alpha;
#pragma unroll
            for (int dt = 0; dt < L::DT; dt++)
#pragma unroll
              for (int y = 0; y < 16; y++) o[dt][y] *= alpha;
          }
          m = m_new;
          // mc is rounded, a score times the scale below is not: so large that half a step of mc is more than 2^0.5 in a weight, the maximum goes off first.
          if (__any(fabsf(mc) >= 0x1p24f)) {
#pragma unroll
            for (int kt = 0; kt < 2; kt++)
#pragma unroll
              for (int y = 0; y < 16; y++) s[kt][y] -= m_use;
            mc = 0.f;
          }
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
              else pack_weights(s[kt], cc, pf);
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
    };
    for (int x = t0;;) {
      ask(x, st0);
      walk(x, 0);
      if (++x >= t1) break;
      publish(st1, 1, base_of(x));
      __syncthreads();
      ask(x, st1);
      walk(x, 1);
      if (++x >= t1) break;
      publish(st0, 0, base_of(x));
      __syncthreads();
    }
    __syncthreads();

    if (works) {
      l = xhalf_sum(l);
      const float m2 = m * a.scale_log2e;   // in units of log2
      const bool done = t0 == 0 && t1 == count;
      const int64_t slot = (int64_t)(2 * w + (t0 == 0)) * kChunkRows + wave * 32 + li;
      char* out = done ? a.out + row.token * a.o_st + row.head * a.o_sh : (char*)(plan.o + slot * D);
      if (row.real) {
        if (done) {
          store_row<IO, D>(out, o, l == 0.f ? 0.f : 1.f / l);
          if (lh == 0) a.lse[row.head * a.n_tokens + row.token] = lse_of(m2, l);
        } else {
          store_row<float, D>(out, o, 1.f);
          if (lh == 0) plan.ml[slot] = make_float2(m2, l);
        }
      }
      if (s_odd[piece & 1] == piece)
        for (int x = t0; x < t1; x++)
          if (!seen_by_all(base_of(x)))
            add_not_finite<D>(c, table, hk, row, base_of(x), min(base_of(x) + kChunkKeys, keys.len), [&](int d) { return lh == (d >> 2 & 1); },
                              [&](int d, float v) { if (done) add_to<IO>(out + sizeof(IO) * d, v); else add_to<float>(out + 4 * d, v); });
    }
    if (t0 == 0 && t1 < count && tid == 0) {
      plan.joins[w] = ChunkJoin{hk, w, sh.worker_of(hk * tiles + it.before + count - 1), 0, it.first, it.rows, row0, 0};
    }
    left -= t1 - t0;
    t0 = 0;
    if (++item == n_items) { item = 0; hk++; }
  }
}

// Joins the parts of an item that several workers shared: workgroup (x, y) takes the y-th rows of the item that worker x begins, D / 4 lanes a row.  Bound by latency: 16 sequences
// of 2 048 tokens with 20 new ones each, 32/8 heads of 128, whole calls 51.4 us (60.4 with four workgroups an item).
template <typename IO, int D>
__global__ __launch_bounds__(kThreads) void chunk_join_kernel(ChunkArgs a, ChunkPlan plan) {
  const ChunkJoin job = plan.joins[blockIdx.x];
  if (job.last_worker < 0) return;
  constexpr int kLanes = D / 4, kRows = kThreads / kLanes;
  const int d = threadIdx.x % kLanes * 4, end = min(job.row0 + a.rows, job.rows);
  const int y = blockIdx.y * kRows + threadIdx.x / kLanes;
  if (job.row0 + y >= end) return;
  const ChunkRow row(a, job.hk, job.first, 0, end, job.row0 + y);
  float m = -INFINITY, l = 0.f;
  float4 o = make_float4(0, 0, 0, 0);
  constexpr int kAhead = 8;   // parts in flight
  for (int x0 = job.first_worker; x0 <= job.last_worker; x0 += kAhead) {
    float2 ml[kAhead];
    float4 u[kAhead];
#pragma unroll
    for (int z = 0; z < kAhead; z++) {
      const int x = x0 + z;
      ml[z] = make_float2(-INFINITY, 0.f);
      u[z] = make_float4(0, 0, 0, 0);
      if (x <= job.last_worker) {
        const int64_t slot = (int64_t)(2 * x + (x == job.first_worker)) * a.rows + y;
        ml[z] = plan.ml[slot];
        u[z] = *(const float4*)(plan.o + slot * D + d);
      }
    }
#pragma unroll
    for (int z = 0; z < kAhead; z++) {
      const float m2 = fmaxf(m, ml[z].x), zero = m2 == -INFINITY ? 0.f : m2;
      const float f = __builtin_amdgcn_exp2f(m - zero), fx = __builtin_amdgcn_exp2f(ml[z].x - zero);
      l = l * f + ml[z].y * fx;
      o.x = o.x * f + u[z].x * fx;
      o.y = o.y * f + u[z].y * fx;
      o.z = o.z * f + u[z].z * fx;
      o.w = o.w * f + u[z].w * fx;
      m = m2;
    }
  }
  const float by = l == 0.f ? 0.f : 1.f / l;
  char* out = a.out + row.token * a.o_st + row.head * a.o_sh + d * sizeof(IO);
  if (l == 0.f) o = make_float4(0, 0, 0, 0);
  if constexpr (sizeof(IO) == 4) *(float4*)out = make_float4(o.x * by, o.y * by, o.z * by, o.w * by);
  else *(uint2*)out = make_uint2(pack_bf16x2(o.x * by, o.y * by), pack_bf16x2(o.z * by, o.w * by));
  if (d == 0) a.lse[row.head * a.n_tokens + row.token] = lse_of(m, l);
}

namespace {
template <typename IO, int D> void launch_d(const KCache& c, const ChunkArgs& a, const ChunkPlan& plan, hipStream_t s) {
  if (a.rows == kChunkRows) hipLaunchKernelGGL((chunk_kernel<IO, D>), dim3(kWorkers), dim3(kThreads), 0, s, c, a, plan);
  else launch_chunk_few(D, c, a, plan, s);
  constexpr int kJoinRows = kThreads / (D / 4);
  hipLaunchKernelGGL((chunk_join_kernel<IO, D>), dim3(kWorkers, (a.rows + kJoinRows - 1) / kJoinRows), dim3(kThreads), 0, s, a, plan);
}
template <typename IO> void launch_io(int32_t d, const KCache& c, const ChunkArgs& a, const ChunkPlan& plan, hipStream_t s) {
  if (d == 128) launch_d<IO, 128>(c, a, plan, s);
  else if (d == 64) launch_d<IO, 64>(c, a, plan, s);
  else launch_d<IO, 32>(c, a, plan, s);
}
}  // namespace

void launch_chunk(int32_t d, const KCache& c, const ChunkArgs& a, const ChunkPlan& plan, hipStream_t s) {
  if (!plans_itself(a)) hipLaunchKernelGGL(chunk_plan_kernel, dim3(1), dim3(kPlanThreads), 0, s, c, a, plan);
  if (c.io_bytes == 4) launch_io<float>(d, c, a, plan, s);
  else launch_io<bf16_t>(d, c, a, plan, s);
}

}  // namespace dcp
