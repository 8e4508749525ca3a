// Key tiles as MFMA operands, for the kernels that score queries against the
// paged cache.
#pragma once

#include "attn_common.hpp"

namespace eldr {

constexpr int kRows = 16;  // query rows of a tile
constexpr int kStep = 32;  // slots a wave takes at a time: two 16-slot tiles, each inside a page
constexpr float kLog2e = 1.4426950408889634f;

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

template <int D, bool FP8>
struct Tile {
  static constexpr int kK = D / 32;       // MFMA steps of the first product
  static constexpr int kV = D / 16;       // value columns a lane holds
  static constexpr int kElem = FP8 ? 1 : 2;

  // Value index of the first of the 8 that a lane holds for step s.
  static __device__ __forceinline__ int q_at(int s, int g) {
    return FP8 ? (s / 2) * 64 + g * 16 + (s % 2) * 8 : s * 32 + g * 8;
  }
};

// Two fp8 codes (bytes 0, 1 or 2, 3 of w) as bf16: exact.
template <bool HI>
__device__ __forceinline__ uint32_t fp8_pair(uint32_t w) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.0f, HI));
}

// One 16-slot tile of keys as MFMA operands.
template <int D, bool FP8>
struct Keys {
  using T = Tile<D, FP8>;
  static constexpr int kLoads = FP8 ? T::kK / 2 : T::kK;
  u32x4 raw[kLoads];
  __device__ __forceinline__ void load(const char* rows, int n, int g) {
#pragma unroll
    for (int i = 0; i < kLoads; ++i)
      raw[i] = *reinterpret_cast<const u32x4*>(rows + (uint32_t)(n * D * T::kElem + i * 64 + g * 16));
  }
  __device__ __forceinline__ u32x4 operand(int s) const {
    if constexpr (FP8) {
      const u32x4 r = raw[s / 2];
      const uint32_t a = r[(s % 2) * 2], b = r[(s % 2) * 2 + 1];
      return u32x4{fp8_pair<false>(a), fp8_pair<true>(a), fp8_pair<false>(b), fp8_pair<true>(b)};
    } else {
      return raw[s];
    }
  }
};

}  // namespace eldr
