// New tokens rounded into a paged key-value cache in 8 bits, and tokens read out of a cache of any dtype.
#include <algorithm>

#include "cache_tokens.h"
#include "e4m3.h"

using namespace dcp;

namespace dcp {

namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// The numbers of a 16-byte piece of k_new or v_new, 8 of bf16 or 4 of fp32, and the largest of several as bits: of both halves of a word for bf16.
template <typename IO> struct Piece;
template <> struct Piece<bf16_t> {
  typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
  static constexpr int kNumbers = 8;
  static __device__ __forceinline__ float at(const u32x4& u, int y) { return __uint_as_float(y & 1 ? u[y / 2] & 0xffff0000u : u[y / 2] << 16); }
  static __device__ __forceinline__ uint32_t larger(uint32_t top, uint32_t word) {
    return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2, top), __builtin_bit_cast(u16x2, word & 0x7fff7fffu)));
  }
  static __device__ __forceinline__ uint32_t fp32_bits(uint32_t top) { return max(top << 16, top & 0xffff0000u); }
  static __device__ __forceinline__ uint32_t finite(uint32_t word) {   // what is not becomes 0
    return ((word & 0x7f80u) == 0x7f80u ? 0u : word & 0xffffu) | ((word & 0x7f800000u) == 0x7f800000u ? 0u : word & 0xffff0000u);
  }
};
template <> struct Piece<float> {
  static constexpr int kNumbers = 4;
  static __device__ __forceinline__ float at(const u32x4& u, int y) { return __uint_as_float(u[y]); }
  static __device__ __forceinline__ uint32_t larger(uint32_t top, uint32_t word) { return max(top, word & 0x7fffffffu); }
  static __device__ __forceinline__ uint32_t fp32_bits(uint32_t top) { return top; }
  static __device__ __forceinline__ uint32_t finite(uint32_t word) { return (word & 0x7f800000u) == 0x7f800000u ? 0u : word; }
};

// A wave takes a block of tokens of one head of K or V: the largest of the new values, the scale, the codes.  Bound by HBM where there are many tokens in blocks of 32 or 64 (49 714, 8 KV heads of 128,
// blocks of 64: 61 us, 5.0 TB/s read and written); with shorter blocks by the waves' trips to memory, as most of a wave's registers are empty, and longer ones are read twice.  Blocks of 2, 4, 5, 8, 16,
// 32, 64, 128 and 256: bf16 292, 163, 148, 104, 73, 64, 61, 69, 83 us; fp32, of which 32 rows are held, 394, 235, 206, 153, 121, 113, 169, 219, 261.  Few tokens are bound by the trips to memory: cu_new, seqs, seq_len, page_table, the tokens and the block's scale.
//   rows   new tokens of the block, the first of them x (stride x_st), to the codes at `to` (stride to_st); behind `older` tokens that it has already
template <typename IO, int D>
__device__ __forceinline__ void append_block(const char* x, int64_t x_st, char* to, int64_t to_st, uint8_t* scale, int rows, int older) {
  typedef Piece<IO> P;
  constexpr int kLanes = D / P::kNumbers, kRows = 64 / kLanes;   // lanes of a row, rows at a time
  constexpr int kHeld = 16;                                      // pieces of a lane that stay in registers: a block of up to kHeld kRows tokens is read once
  const int lane = threadIdx.x & 63, r = lane / kLanes, off = lane % kLanes;
  const uint32_t had = older ? min(max((uint32_t)*scale, 1u), 254u) : 0u;
  x += r * x_st + off * 16;
  u32x4 held[kHeld];
#pragma unroll
  for (int y = 0; y < kHeld; y++) {
    held[y] = u32x4{0, 0, 0, 0};
    if (r + y * kRows < rows) held[y] = __builtin_nontemporal_load((const u32x4*)(x + y * kRows * x_st));
  }
  auto rest = [&](auto&& f) {   // of a longer block, which is read twice
#pragma unroll 1
    for (int y = kHeld * kRows; r + y < rows; y += kRows) f(y, *(const u32x4*)(x + y * x_st));
  };
  uint32_t top = 0;
#pragma unroll
  for (int y = 0; y < kHeld; y++)
#pragma unroll
    for (int z = 0; z < 4; z++) top = P::larger(top, held[y][z]);
  rest([&](int, const u32x4& u) {
#pragma unroll
    for (int z = 0; z < 4; z++) top = P::larger(top, u[z]);
  });
  if (__any(P::fp32_bits(top) >= 0x7f800000u)) {   // an infinity or a NaN, which does not count
    top = 0;
#pragma unroll
    for (int y = 0; y < kHeld; y++)
#pragma unroll
      for (int z = 0; z < 4; z++) top = P::larger(top, P::finite(held[y][z]));
    rest([&](int, const u32x4& u) {
#pragma unroll
      for (int z = 0; z < 4; z++) top = P::larger(top, P::finite(u[z]));
    });
  }
  top = P::fp32_bits(top);
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) top = max(top, (uint32_t)__shfl_xor((int)top, o));
  const uint32_t now = max(had, least_scale(top));
  const float up = __uint_as_float(now >= 254 ? 0x400000u : (254 - now) << 23);   // 2^(127 - now)
  char* dst = to + r * to_st + off * P::kNumbers;
  auto store = [&](int y, const u32x4& u) {
    char* p = dst + y * to_st;
    if constexpr (P::kNumbers == 8) {
      *(uint2*)p = make_uint2(f32x4_to_e4m3(P::at(u, 0) * up, P::at(u, 1) * up, P::at(u, 2) * up, P::at(u, 3) * up),
                              f32x4_to_e4m3(P::at(u, 4) * up, P::at(u, 5) * up, P::at(u, 6) * up, P::at(u, 7) * up));
    } else {
      *(uint32_t*)p = f32x4_to_e4m3(P::at(u, 0) * up, P::at(u, 1) * up, P::at(u, 2) * up, P::at(u, 3) * up);
    }
  };
#pragma unroll
  for (int y = 0; y < kHeld; y++)
    if (r + y * kRows < rows) store(y * kRows, held[y]);
  rest(store);
  if (older && now > had) {   // the earlier tokens' codes, from what they stand for: exact but for numbers that fall below the format's normal ones
    const float down = __uint_as_float((uint32_t)max((int)had - (int)now + 127, 1) << 23);
    constexpr int kWords = D / 4;
#pragma unroll 1
    for (int y = lane; y < older * kWords; y += 64) {
      char* p = to - (int64_t)(older - y / kWords) * to_st + y % kWords * 4;
      const uint32_t u = *(const uint32_t*)p;
      const f32x2_t a = e4m3_to_f32x2<false>(u), b = e4m3_to_f32x2<true>(u);
      *(uint32_t*)p = f32x4_to_e4m3(a[0] * down, a[1] * down, b[0] * down, b[1] * down);
    }
  }
  if (lane == 0 && now != had) *scale = (uint8_t)now;
}

// The same where every token has scales of its own: a row's lanes find its largest value and its scale between them, kAhead rows in flight.  49 714 tokens, 8 KV heads of 128:
// 63 us, 4.9 TB/s read and written (a wave a block: 506); fp32 95 us, 5.4 TB/s.
template <typename IO, int D, int TOKENS>
__global__ __launch_bounds__(256) void append8_rows_kernel(KCache c, int32_t layer, const int32_t* __restrict__ seqs, const int32_t* __restrict__ cu, int32_t n,
                                                           const int32_t* __restrict__ status, NewTokens x) {
  typedef Piece<IO> P;
  constexpr int kLanes = D / P::kNumbers, kAtOnce = 256 / kLanes, kAhead = 4;
  __shared__ int32_t page_of[TOKENS], slot_of[TOKENS], s_cu[kCuInLds];
  const int64_t t0 = (int64_t)blockIdx.x * TOKENS;
  const Begins begins(cu, n, s_cu);
  if (threadIdx.x < TOKENS) {
    const TokenPlace p = token_place(c, seqs, begins, n, status, t0 + threadIdx.x, x.n);
    page_of[threadIdx.x] = p.page;
    slot_of[threadIdx.x] = p.slot;
  }
  __syncthreads();
  const int off = threadIdx.x % kLanes, all = TOKENS * c.hkv;   // rows of K, and as many of V
  for (int y0 = threadIdx.x / kLanes; y0 < all; y0 += kAtOnce * kAhead / 2) {
    u32x4 u[kAhead];
#pragma unroll
    for (int z = 0; z < kAhead; z++) {
      const int y = y0 + z / 2 * kAtOnce, t = c.heads.quot(y), h = c.heads.rem(y, t);
      u[z] = u32x4{0, 0, 0, 0};
      if (y < all && page_of[t] >= 0)
        u[z] = __builtin_nontemporal_load((const u32x4*)((z & 1 ? x.v + (t0 + t) * x.v_st + h * x.v_sh : x.k + (t0 + t) * x.k_st + h * x.k_sh) + off * 16));
    }
#pragma unroll
    for (int z = 0; z < kAhead; z++) {
      const int y = y0 + z / 2 * kAtOnce, t = c.heads.quot(y), h = c.heads.rem(y, t);
      uint32_t top = 0;
#pragma unroll
      for (int w = 0; w < 4; w++) top = P::larger(top, u[z][w]);
      if (P::fp32_bits(top) >= 0x7f800000u) {
        top = 0;
#pragma unroll
        for (int w = 0; w < 4; w++) top = P::larger(top, P::finite(u[z][w]));
      }
      top = P::fp32_bits(top);
#pragma unroll
      for (int o = 1; o < kLanes; o <<= 1) top = max(top, (uint32_t)__shfl_xor((int)top, o));
      if (y >= all || page_of[t] < 0) continue;
      const uint32_t now = least_scale(top);
      const float up = __uint_as_float((254 - now) << 23);   // now is 247 at most
      const int64_t page = page_of[t], slot = slot_of[t], at = layer * c.layer_scales() + c.scale_at((int)page, (int)slot) + h;
      char* to = (z & 1 ? c.v + layer * c.v_sl + page * c.v_sp + slot * c.v_st + h * c.v_sh : c.k + layer * c.k_sl + page * c.k_sp + slot * c.k_st + h * c.k_sh) + off * P::kNumbers;
      if constexpr (P::kNumbers == 8)
        *(uint2*)to = make_uint2(f32x4_to_e4m3(P::at(u[z], 0) * up, P::at(u[z], 1) * up, P::at(u[z], 2) * up, P::at(u[z], 3) * up),
                                 f32x4_to_e4m3(P::at(u[z], 4) * up, P::at(u[z], 5) * up, P::at(u[z], 6) * up, P::at(u[z], 7) * up));
      else *(uint32_t*)to = f32x4_to_e4m3(P::at(u[z], 0) * up, P::at(u[z], 1) * up, P::at(u[z], 2) * up, P::at(u[z], 3) * up);
      if (off == 0) (z & 1 ? c.v_scale : c.k_scale)[at] = (uint8_t)now;
    }
  }
}

// A workgroup has TOKENS tokens, of which those count that begin a block or their place: the block is theirs, with the new tokens behind
// them.  Column y of the grid: four of the 2 hkv heads of K and V, one a wave.
template <typename IO, int D, int TOKENS>
__global__ __launch_bounds__(256, sizeof(IO) == 4 ? 2 : 4) void append8_kernel(KCache c, int32_t layer, const int32_t* __restrict__ seqs, const int32_t* __restrict__ cu, int32_t n,
                                                      const int32_t* __restrict__ status, NewTokens x) {
  __shared__ int32_t page_of[TOKENS], slot_of[TOKENS], rows_of[TOKENS], older_of[TOKENS], s_cu[kCuInLds];
  const int64_t t0 = (int64_t)blockIdx.x * TOKENS;
  const Begins begins(cu, n, s_cu);
  if (threadIdx.x < TOKENS) {
    const int64_t t = t0 + threadIdx.x;
    const TokenPlace p = token_place(c, seqs, begins, n, status, t, x.n);
    const int in_block = p.page < 0 ? 0 : c.block.rem(p.slot, c.block.quot(p.slot));
    const bool begins_block = p.page >= 0 && (in_block == 0 || t == max(p.first, 0));   // of what cu_new names below 0 there is nothing to write
    page_of[threadIdx.x] = begins_block ? p.page : -1;
    slot_of[threadIdx.x] = p.slot;
    rows_of[threadIdx.x] = (int)min((int64_t)min(p.behind, (int)c.block.d - in_block), x.n - t);
    older_of[threadIdx.x] = in_block;
  }
  __syncthreads();
  const int wave = threadIdx.x >> 6;
  for (int y = 0; y < TOKENS; y++) {
    const int page = page_of[y];
    if (page < 0) continue;
    const int64_t at = c.scale_at(page, slot_of[y]), slot = slot_of[y];
    for (int64_t col = blockIdx.y * 4 + wave; col < 2 * (int64_t)c.hkv; col += gridDim.y * 4) {
      const bool v = col >= c.hkv;
      const int64_t h = v ? col - c.hkv : col;
      const int64_t x_st = v ? x.v_st : x.k_st, to_st = v ? c.v_st : c.k_st;
      append_block<IO, D>((v ? x.v : x.k) + (t0 + y) * x_st + h * (v ? x.v_sh : x.k_sh), x_st,
                          (v ? c.v + layer * c.v_sl + page * c.v_sp + h * c.v_sh : c.k + layer * c.k_sl + page * c.k_sp + h * c.k_sh) + slot * to_st, to_st,
                          (v ? c.v_scale : c.k_scale) + layer * c.layer_scales() + at + h, rows_of[y], older_of[y]);
    }
  }
}

// A workgroup reads TOKENS tokens; a lane makes 16 bytes of k_out and of v_out at a time.  IO: 0 copies (bf16 and fp32 caches), else the bytes of a number that codes
// become.  Bound by HBM where there are many (115 760 tokens, 8 KV heads of 128, read and written: to bf16 114 to 122 us, by where the pages lie, 5.8 to 6.3 TB/s; to fp32, one sequence, 172, 6.9;
// out of a cache in bf16 170, 5.6, in fp32 351, 5.4).
template <int IO, int TOKENS>
__global__ __launch_bounds__(256) void read_kernel(KCache c, int32_t layer, const int32_t* __restrict__ seqs, const int32_t* __restrict__ cu, int32_t n,
                                                   const int32_t* __restrict__ status, ReadTokens x, int32_t log_pieces) {
  __shared__ int32_t page_of[TOKENS], slot_of[TOKENS], s_cu[kCuInLds];
  const int64_t t0 = (int64_t)blockIdx.x * TOKENS;
  const Begins begins(cu, n, s_cu);
  if (threadIdx.x < TOKENS) {
    const TokenPlace p = token_place(c, seqs, begins, n, status, t0 + threadIdx.x, x.n);
    page_of[threadIdx.x] = p.page;
    slot_of[threadIdx.x] = p.slot;
  }
  __syncthreads();
  constexpr int kFrom = IO == 0 ? 16 : 16 / IO;   // bytes that 16 become of
  constexpr int kAhead = 4;
  const int all = TOKENS * c.hkv << log_pieces;
  for (int y0 = threadIdx.x; y0 < all; y0 += 256 * kAhead) {
    u32x4 u[kAhead][2];
    uint32_t scale[kAhead][2];
    char* to[kAhead][2];
#pragma unroll
    for (int z = 0; z < kAhead; z++) {
      const int y = y0 + 256 * z, row = y >> log_pieces, off = y & ((1 << log_pieces) - 1);   // row: (token, head)
      const int t = c.heads.quot(row), h = c.heads.rem(row, t);
      to[z][0] = nullptr;
      if (y < all && page_of[t] >= 0) {
        const int64_t page = page_of[t], slot = slot_of[t];
        const char* k = c.k + layer * c.k_sl + page * c.k_sp + slot * c.k_st + h * c.k_sh + off * kFrom;
        const char* v = c.v + layer * c.v_sl + page * c.v_sp + slot * c.v_st + h * c.v_sh + off * kFrom;
        to[z][0] = x.k + (t0 + t) * x.k_st + h * x.k_sh + off * 16;
        to[z][1] = x.v + (t0 + t) * x.v_st + h * x.v_sh + off * 16;
        if constexpr (IO == 0) {
          u[z][0] = __builtin_nontemporal_load((const u32x4*)k);
          u[z][1] = __builtin_nontemporal_load((const u32x4*)v);
        } else {
          const int64_t at = layer * c.layer_scales() + c.scale_at((int)page, (int)slot) + h;
          scale[z][0] = c.k_scale[at];
          scale[z][1] = c.v_scale[at];
          if constexpr (IO == 2) {
            const uint2 a = *(const uint2*)k, b = *(const uint2*)v;
            u[z][0][0] = a.x; u[z][0][1] = a.y;
            u[z][1][0] = b.x; u[z][1][1] = b.y;
          } else {
            u[z][0][0] = *(const uint32_t*)k;
            u[z][1][0] = *(const uint32_t*)v;
          }
        }
      }
    }
#pragma unroll
    for (int z = 0; z < kAhead; z++) {
      if (!to[z][0]) continue;
#pragma unroll
      for (int kv = 0; kv < 2; kv++) {
        u32x4 out = u[z][kv];
        if constexpr (IO != 0) {
          const float factor = scale_factor(scale[z][kv]);
          if constexpr (IO == 2) {
            const uint32_t a = out[0], b = out[1];
            out[0] = e4m3_to_bf16x2<false>(a, factor); out[1] = e4m3_to_bf16x2<true>(a, factor);
            out[2] = e4m3_to_bf16x2<false>(b, factor); out[3] = e4m3_to_bf16x2<true>(b, factor);
          } else {
            const f32x2_t a = e4m3_to_f32x2<false>(u[z][kv][0]), b = e4m3_to_f32x2<true>(u[z][kv][0]);
            out[0] = __float_as_uint(a[0] * factor); out[1] = __float_as_uint(a[1] * factor);
            out[2] = __float_as_uint(b[0] * factor); out[3] = __float_as_uint(b[1] * factor);
          }
        }
        __builtin_nontemporal_store(out, (u32x4*)to[z][kv]);
      }
    }
  }
}

template <typename IO, int D>
void append8(int32_t each, dim3 grid, const KCache& c, int32_t layer, const int32_t* seqs, const int32_t* cu, int32_t n, const int32_t* status,
             const NewTokens& x, hipStream_t s) {
  auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(256), 0, s, c, layer, seqs, cu, n, status, x); };
  if (c.block.d == 1) each == 1 ? go(append8_rows_kernel<IO, D, 1>) : go(append8_rows_kernel<IO, D, 4>);
  else if (each == 1) go(append8_kernel<IO, D, 1>);
  else if (each == 16) go(append8_kernel<IO, D, 16>);
  else go(append8_kernel<IO, D, 64>);
}
template <typename IO>
void append8(int32_t each, dim3 grid, int d, const KCache& c, int32_t layer, const int32_t* seqs, const int32_t* cu, int32_t n, const int32_t* status,
             const NewTokens& x, hipStream_t s) {
  if (d == 128) append8<IO, 128>(each, grid, c, layer, seqs, cu, n, status, x, s);
  else if (d == 64) append8<IO, 64>(each, grid, c, layer, seqs, cu, n, status, x, s);
  else append8<IO, 32>(each, grid, c, layer, seqs, cu, n, status, x, s);
}

}  // namespace

void launch_append8(int32_t each, uint32_t grid, const KCache& c, int32_t layer, const int32_t* seqs, const int32_t* cu, int32_t n, const int32_t* status,
                    const NewTokens& x, hipStream_t s) {
  const int d = 16 << c.log_head_chunks;   // a code is a byte
  const uint32_t columns = c.block.d == 1 ? 1 : (uint32_t)std::min<int64_t>((2 * (int64_t)c.hkv + 3) / 4, std::max<int64_t>(1, (1 << 23) / grid));   // fewer than 2^32 threads
  if (c.io_bytes == 2) append8<bf16_t>(each, dim3(grid, columns), d, c, layer, seqs, cu, n, status, x, s);
  else append8<float>(each, dim3(grid, columns), d, c, layer, seqs, cu, n, status, x, s);
}

void launch_read(int32_t each, uint32_t grid, const KCache& c, int32_t layer, const int32_t* seqs, const int32_t* cu, int32_t n, const int32_t* status,
                 const ReadTokens& x, hipStream_t s) {
  const int32_t log_pieces = c.k_scale ? c.log_head_chunks + (c.io_bytes == 4 ? 2 : 1) : c.log_head_chunks;
  auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(grid), dim3(256), 0, s, c, layer, seqs, cu, n, status, x, log_pieces); };
  if (!c.k_scale) each == 1 ? go(read_kernel<0, 1>) : go(read_kernel<0, 4>);
  else if (c.io_bytes == 2) each == 1 ? go(read_kernel<2, 1>) : go(read_kernel<2, 4>);
  else each == 1 ? go(read_kernel<4, 1>) : go(read_kernel<4, 4>);
}

}  // namespace dcp
