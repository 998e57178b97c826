// A wave's walk over keys in 8 bits, for the kernels that hold them in registers.
#pragma once
#include "e4m3.h"
#include "paged_attn_kernel.h"

namespace dcp {

// A wave's walk as in paged_attn.hip (the same lanes hold the same keys and columns), in tiles of 32 keys: a lane has 16 bytes of a key's row, 16 of its
// numbers, and D / 16 bytes of each of eight rows of V.  (Tiles of 64 keys, as many bytes as 32 in bf16, took longer: 32 places of 512 to 8 192 tokens, 32/8 heads of 128, 48.7
// and 47.5 us, one of 300 tokens 7.9 and 7.6.)  Codes become bf16 numbers with their scale in one conversion for two of them, without
// rounding, so that the products take them as they take a cache in bf16.  IO is bf16 or fp32; an fp32 query goes in as three bf16 parts, and so do
// the weights: exact products, summed in fp32.
template <typename IO, int D> struct Tile8 {
  typedef IO Out;
  static constexpr int kD = D, kRowBytes = D;
  static constexpr bool kScaled = true, kF32 = sizeof(IO) == 4;
  static constexpr int kGroup = 8, kKeys = 32, kRowTiles = 2, kAcc = D / 16;
  static constexpr int kSteps = D / 32;                     // products of 32 numbers of a row
  static constexpr int kVWords = D >= 64 ? D / 64 : 1;      // 4-byte words of a lane's columns of V
  static constexpr int kParts = kF32 ? 3 : 1;
  uint32_t k[kRowTiles][2 * kSteps];
  uint32_t v[kGroup][kVWords];
  uint8_t ks[kRowTiles], vs[kGroup];                        // scales

  static __device__ __forceinline__ int k_off(int g) { return g * (D == 32 ? 8 : 16); }
  static __device__ __forceinline__ int v_off(int i) { return i * (D / 16); }
  template <bool ONCE> __device__ __forceinline__ void load_k(int s, const char* p) {
    if constexpr (D == 32) {
      const u32x2 u = load_kv<ONCE, u32x2>(p);
      k[s][0] = u[0]; k[s][1] = u[1];
    } else {
#pragma unroll
      for (int x = 0; x < D / 64; x++) {
        const u32x4 u = load_kv<ONCE, u32x4>(p + 64 * x);
#pragma unroll
        for (int y = 0; y < 4; y++) k[s][4 * x + y] = u[y];
      }
    }
  }
  template <bool ONCE> __device__ __forceinline__ void load_v(int j, const char* p) {
    if constexpr (D == 128) { const u32x2 u = load_kv<ONCE, u32x2>(p); v[j][0] = u[0]; v[j][1] = u[1]; }
    else if constexpr (D == 64) v[j][0] = load_kv<ONCE, uint32_t>(p);
    else v[j][0] = load_kv<ONCE, uint16_t>(p);
  }
  __device__ __forceinline__ void keep_v(int j, bool keep) {
#pragma unroll
    for (int x = 0; x < kVWords; x++) v[j][x] = keep ? v[j][x] : 0u;
  }
  // Leaves out what is not finite; whether anything was.
  __device__ __forceinline__ bool clean_v(int j) {
    uint32_t bad = 0;
#pragma unroll
    for (int x = 0; x < kVWords; x++) {
      const uint32_t signs = not_finite(v[j][x], vs[j]);
      v[j][x] = without(v[j][x], signs);
      bad |= signs;
    }
    return bad != 0;
  }
  __device__ __forceinline__ void k_scale(int s, uint8_t e) { ks[s] = e; }
  __device__ __forceinline__ void v_scale(int j, uint8_t e) { vs[j] = e; }
  __device__ __forceinline__ void k_scales(uint8_t e) {
#pragma unroll
    for (int s = 0; s < kRowTiles; s++) ks[s] = e;
  }
  __device__ __forceinline__ void v_scales(uint8_t e) {
#pragma unroll
    for (int j = 0; j < kGroup; j++) vs[j] = e;
  }

  struct Q { bf16x8 x[kParts][kSteps]; };
  static __device__ __forceinline__ void load_q(Q& q, const char* p, int g, bool real) {
#pragma unroll
    for (int f = 0; f < kSteps; f++) {
      const int at = D == 32 ? 8 * g : 16 * g + 64 * (f / 2) + 8 * (f & 1);   // the numbers of k[.][2 f], k[.][2 f + 1]
      if constexpr (!kF32) {
        q.x[0][f] = __builtin_bit_cast(bf16x8, real ? *(const uint4*)(p + 2 * at) : make_uint4(0, 0, 0, 0));
      } else {
        float x[8], all[8];
#pragma unroll
        for (int y = 0; y < 8; y += 4) {
          const f32x4 u = real ? *(const f32x4*)(p + 4 * (at + y)) : f32x4{0, 0, 0, 0};
#pragma unroll
          for (int z = 0; z < 4; z++) all[y + z] = x[y + z] = u[z] == u[z] ? u[z] : NAN;   // whose upper half is NaN too
        }
#pragma unroll
        for (int part = 0; part < 3; part++) {
          uint4 w;
          uint32_t* words = (uint32_t*)&w;
#pragma unroll
          for (int y = 0; y < 8; y += 2) {
            words[y / 2] = __builtin_amdgcn_perm(__float_as_uint(x[y + 1]), __float_as_uint(x[y]), 0x07060302u);
#pragma unroll
            for (int z = y; z < y + 2; z++) x[z] = left_of_query(x[z], all[z]);
          }
          q.x[part][f] = __builtin_bit_cast(bf16x8, w);
        }
      }
    }
  }
  __device__ __forceinline__ void scores(const Q& q, float* s) const {
#pragma unroll
    for (int t = 0; t < kRowTiles; t++) {
      f32x4 z = {0, 0, 0, 0};
      const float factor = scale_factor(ks[t]);
#pragma unroll
      for (int f = 0; f < kSteps; f++) {
        uint4 a;
        a.x = e4m3_to_bf16x2<false>(k[t][2 * f], factor);
        a.y = e4m3_to_bf16x2<true>(k[t][2 * f], factor);
        a.z = e4m3_to_bf16x2<false>(k[t][2 * f + 1], factor);
        a.w = e4m3_to_bf16x2<true>(k[t][2 * f + 1], factor);
#pragma unroll
        for (int part = 0; part < kParts; part++) z = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), q.x[part][f], z, 0, 0, 0);
      }
#pragma unroll
      for (int r = 0; r < 4; r++) s[4 * t + r] = z[r];
    }
  }
  // bf16: two parts of the weights, the first of them below the weight, as for a cache in bf16; fp32: three.
  template <int COLS> __device__ __forceinline__ void weigh(const float* p, bool second, f32x4* acc) const {
    constexpr int kProducts = kF32 ? 3 : COLS == 8 ? 1 : 2;
    uint4 b[kProducts];
    float x[8];
#pragma unroll
    for (int j = 0; j < 8; j++) x[j] = p[j];
    if constexpr (kF32) {
#pragma unroll
      for (int part = 0; part < 3; part++) {
        uint32_t* words = (uint32_t*)&b[part];
#pragma unroll
        for (int j = 0; j < 8; j += 2) words[j / 2] = __builtin_amdgcn_perm(__float_as_uint(x[j + 1]), __float_as_uint(x[j]), 0x07060302u);
#pragma unroll
        for (int j = 0; j < 8; j++) x[j] = left_of_weight(x[j], p[j]);
      }
    } else {
      float hi[8], lo[8];
#pragma unroll
      for (int j = 0; j < 8; j++) { hi[j] = upper(x[j] * 0.99609375f); lo[j] = x[j] - hi[j]; }
      auto pack = [](const float* y) { return make_uint4(pack_bf16x2(y[0], y[1]), pack_bf16x2(y[2], y[3]), pack_bf16x2(y[4], y[5]), pack_bf16x2(y[6], y[7])); };
      if constexpr (COLS == 8) {
#pragma unroll
        for (int j = 0; j < 8; j++) hi[j] = second ? lo[j] : hi[j];
        b[0] = pack(hi);
      } else {
        b[0] = pack(hi);
        b[1] = pack(lo);
      }
    }
#pragma unroll
    for (int e = 0; e < kAcc; e += 2) {                   // two columns at a time
      uint32_t w[8];
#pragma unroll
      for (int j = 0; j < 8; j++) {
        const float factor = scale_factor(vs[j]);
        w[j] = e & 2 ? e4m3_to_bf16x2<true>(v[j][e / 4], factor) : e4m3_to_bf16x2<false>(v[j][e / 4], factor);
      }
#pragma unroll
      for (int odd = 0; odd < 2; odd++) {
        const uint32_t sel = odd ? 0x07060302u : 0x05040100u;
        const uint4 a = make_uint4(__builtin_amdgcn_perm(w[1], w[0], sel), __builtin_amdgcn_perm(w[3], w[2], sel), __builtin_amdgcn_perm(w[5], w[4], sel),
                                   __builtin_amdgcn_perm(w[7], w[6], sel));
#pragma unroll
        for (int x = 0; x < kProducts; x++)
          acc[e + odd] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b[x]), acc[e + odd], 0, 0, 0);
      }
    }
  }
  static constexpr int kRun = kAcc, kRuns = 1;
  static __device__ __forceinline__ int first(int r, int, int g) { return (4 * g + r) * kAcc; }
};

}  // namespace dcp
