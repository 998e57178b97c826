// Attention of one new token per sequence over a paged key-value cache in bf16 and fp32.
#include "paged_attn_kernel.h"

using namespace dcp;

namespace dcp {

// A wave walks tiles of 32 (fp32: 16) keys.  Lane l has i = l % 16 and g = l / 16.  K is the A operand as it lies in memory: row i of the
// matrix tile is a key, 16 bytes of it a lane; S^T = K Q^T then holds in lane (i, g) the scores of query head i with the keys
// of group g, 8 g .. 8 g + 7 (fp32: 4 g .. 4 g + 3), if the rows of K are dealt out for it: row r of matrix tile s is key 8 (r / 4) + 4 s + r % 4.
// That is the B operand of O^T = V^T P^T, whose A operand wants from lane (i, g) the keys of group g at one column: a lane loads
// D / 16 neighbouring columns of each of them, which are the same rows of A in D / 16 matrix tiles.  So nothing moves between lanes but
// the maximum over a tile's keys.
template <typename T, int D> struct Tile;

template <int D> struct Tile<bf16_t, D> {
  typedef bf16_t Out;
  static constexpr int kD = D, kRowBytes = 2 * D;
  static constexpr bool kScaled = false;
  static constexpr int kGroup = 8, kKeys = 32, kRowTiles = 2, kAcc = D / 16;
  static constexpr int kWords = D / 32;   // 4-byte words of a lane's columns of V
  struct V { uint32_t w[kWords]; };
  u32x4 k[kRowTiles][D / 32];
  V v[kGroup];

  static __device__ __forceinline__ int k_off(int g) { return g * 16; }
  static __device__ __forceinline__ int v_off(int i) { return i * (D / 8); }
  template <bool ONCE> __device__ __forceinline__ void load_k(int s, const char* p) {
#pragma unroll
    for (int x = 0; x < D / 32; x++) k[s][x] = load_kv<ONCE, u32x4>(p + 64 * x);
  }
  template <bool ONCE> __device__ __forceinline__ void load_v(int j, const char* p) {
    if constexpr (kWords == 4) { const u32x4 u = load_kv<ONCE, u32x4>(p); v[j].w[0] = u[0]; v[j].w[1] = u[1]; v[j].w[2] = u[2]; v[j].w[3] = u[3]; }
    else if constexpr (kWords == 2) { const u32x2 u = load_kv<ONCE, u32x2>(p); v[j].w[0] = u[0]; v[j].w[1] = u[1]; }
    else v[j].w[0] = load_kv<ONCE, uint32_t>(p);
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
  // Lane (., g) holds columns first(r, x, g) .. + kRun - 1 of the result in acc[x * kRun ..][r].
  static constexpr int kRun = kAcc, kRuns = 1;
  static __device__ __forceinline__ int first(int r, int, int g) { return (4 * g + r) * kAcc; }
};

template <int D> struct Tile<float, D> {
  typedef float Out;
  static constexpr int kD = D, kRowBytes = 4 * D;
  static constexpr bool kScaled = false;
  static constexpr int kGroup = 4, kKeys = 16, kRowTiles = 1, kAcc = D / 16;
  static constexpr int kVec = D >= 64 ? 4 : 2, kParts = D / (16 * kVec);   // a lane has kParts pieces of kVec columns of V
  f32x4 k[D / 16];
  float v[kGroup][kParts][kVec];

  static __device__ __forceinline__ int k_off(int g) { return g * 16; }
  static __device__ __forceinline__ int v_off(int i) { return i * kVec * 4; }
  template <bool ONCE> __device__ __forceinline__ void load_k(int, const char* p) {
#pragma unroll
    for (int x = 0; x < D / 16; x++) k[x] = load_kv<ONCE, f32x4>(p + 64 * x);
  }
  template <bool ONCE> __device__ __forceinline__ void load_v(int j, const char* p) {
    typedef float Vec __attribute__((ext_vector_type(kVec)));
#pragma unroll
    for (int x = 0; x < kParts; x++) {
      const Vec u = load_kv<ONCE, Vec>(p + 64 * kVec * x);
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
  static constexpr int kRun = kVec, kRuns = kParts;
  static __device__ __forceinline__ int first(int r, int x, int g) { return x * 16 * kVec + (4 * g + r) * kVec; }
};

template <typename T, int COLS>
static void launch(uint32_t grid, const KCache& c, const PagedArgs& a, const PagedParts& parts, int32_t d, hipStream_t s) {
  if (d == 128) launch_tiles<Tile<T, 128>, COLS>(grid, c, a, parts, s);
  else if (d == 64) launch_tiles<Tile<T, 64>, COLS>(grid, c, a, parts, s);
  else launch_tiles<Tile<T, 32>, COLS>(grid, c, a, parts, s);
}

void launch_paged_attn(int32_t dtype, int32_t d, uint32_t grid, const KCache& c, const PagedArgs& a, const PagedParts& parts, hipStream_t s) {
  if (dtype == DCP_E4M3) launch_paged_attn8(d, grid, c, a, parts, s);
  else if (dtype == DCP_F32) launch<float, 16>(grid, c, a, parts, d, s);
  else if (a.group <= 8) launch<bf16_t, 8>(grid, c, a, parts, d, s);
  else launch<bf16_t, 16>(grid, c, a, parts, d, s);
}

}  // namespace dcp
