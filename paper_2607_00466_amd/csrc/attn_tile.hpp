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

// v, or zeros: a mask, so that the load that gave v stays where it is (a select
// would move it behind a branch).
__device__ __forceinline__ u32x4 keep_if(bool keep, u32x4 v) { return v & (keep ? 0xffffffffu : 0u); }

// The two pages of a 32-slot step that starts at slot k, a multiple of kStep;
// -1 past the table.  table: one request's row.
struct StepPages {
  int b0, b1;
};
__device__ __forceinline__ StepPages step_pages(const Pages& pg, const int32_t* table, int k) {
  const int i0 = k >> pg.shift, i1 = (k + 16) >> pg.shift, last = pg.max_blocks - 1;
  StepPages s{uniform_load(table + min(i0, last)), uniform_load(table + min(i1, last))};
  if (i0 > last) s.b0 = -1;
  if (i1 > last) s.b1 = -1;
  return s;
}

// A load of what is read once (STREAM: it does not displace what the caches hold)
// or again by other workgroups or the next call.
template <bool STREAM, typename V>
__device__ __forceinline__ V tile_load(const char* p) {
  const V* v = reinterpret_cast<const V*>(p);
  return STREAM ? __builtin_nontemporal_load(v) : *v;
}

// One 16-slot tile of keys as MFMA operands.
template <int D, bool FP8>
struct Keys {
  using T = Tile<D, FP8>;
  static constexpr int kLoads = FP8 ? T::kK / 2 : T::kK;
  u32x4 raw[kLoads];
  template <bool STREAM>
  __device__ __forceinline__ void load(const char* rows, int n, int g) {
#pragma unroll
    for (int i = 0; i < kLoads; ++i) raw[i] = tile_load<STREAM, u32x4>(rows + (uint32_t)(n * D * T::kElem + i * 64 + g * 16));
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

// A 32-slot step of keys by way of LDS: a 16-slot tile is one contiguous stretch
// of its page, so a wave reads it in whole lines (1 KB a load, where an operand's
// own load touches 64 pieces of 16 rows), and takes the operands from a stretch
// of LDS of its own, whose rows are rotated against each other to spread them
// over the banks.  No barrier of the workgroup: the stretch is one wave's.
template <int D, bool FP8>
struct StagedKeys {
  using T = Tile<D, FP8>;
  static constexpr int kRowBytes = D * T::kElem, kChunks = kRowBytes / 16;
  static constexpr int kTileBytes = 16 * kRowBytes, kLoads = kTileBytes / (16 * kWave);
  static constexpr int kBytes = 2 * kTileBytes;  // of LDS, a wave
  u32x4 raw[2][kLoads];
  static __device__ __forceinline__ uint32_t at(int row, int chunk) {
    const int turn = kChunks >= 16 ? row & 15 : kChunks == 8 ? (row >> 1) & 7 : (row >> 2) & 3;
    return (uint32_t)(row * kRowBytes + (chunk ^ turn) * 16);
  }
  template <bool STREAM>
  __device__ __forceinline__ void load(int tile, const char* rows) {
#pragma unroll
    for (int i = 0; i < kLoads; ++i)
      raw[tile][i] = tile_load<STREAM, u32x4>(rows + (uint32_t)(threadIdx.x % kWave * 16 + i * 16 * kWave));
  }
  // lds: the wave's kBytes
  __device__ __forceinline__ void put(char* lds) const {
    wave_handover();  // after the last step's operands
#pragma unroll
    for (int b = 0; b < 2; ++b)
#pragma unroll
      for (int i = 0; i < kLoads; ++i) {
        const int piece = threadIdx.x % kWave + i * kWave;
        *reinterpret_cast<u32x4*>(lds + b * kTileBytes + at(piece / kChunks, piece % kChunks)) = raw[b][i];
      }
    wave_handover();
  }
  // Keys::raw[i] of tile b
  static __device__ __forceinline__ u32x4 get(const char* lds, int b, int i, int n, int g) {
    return *reinterpret_cast<const u32x4*>(lds + b * kTileBytes + at(n, i * 4 + g));
  }
};

// 32 slots of values: the lane's kV columns of its 8 slots, 4 of each 16-slot
// tile (rows 4 g .. 4 g + 3).
template <int D, bool FP8>
struct Values {
  using T = Tile<D, FP8>;
  static constexpr int kBytes = T::kV * T::kElem;  // a slot's, 4 to 32
  static constexpr int kWords = kBytes / 4;
  uint32_t raw[8][kWords];
  __device__ __forceinline__ void load(const char* lo, const char* hi, int n, int g) {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const char* p = (j < 4 ? lo : hi) + (uint32_t)((4 * g + (j & 3)) * D * T::kElem + n * kBytes);
      if constexpr (kBytes >= 16) {
#pragma unroll
        for (int w = 0; w < kWords; w += 4) {
          const u32x4 x = tile_load<true, u32x4>(p + 4 * w);
#pragma unroll
          for (int i = 0; i < 4; ++i) raw[j][w + i] = x[i];
        }
      } else if constexpr (kBytes == 8) {
        const u32x2 x = tile_load<true, u32x2>(p);
        raw[j][0] = x[0], raw[j][1] = x[1];
      } else {
        raw[j][0] = tile_load<true, uint32_t>(p);
      }
    }
  }
  // Slots that do not count must not reach a product: 0 times their bits may be NaN.
  __device__ __forceinline__ void drop(int j, bool keep) {
#pragma unroll
    for (int w = 0; w < kWords; ++w) raw[j][w] = keep ? raw[j][w] : 0u;
  }
  // Column c of the lane's 8 slots.
  __device__ __forceinline__ u32x4 operand(int c) const {
    u32x4 v;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t *a = raw[2 * i], *b = raw[2 * i + 1];
      if constexpr (FP8) {
        // the pair's bytes side by side, then both to bf16
        const uint32_t sel = (c & 2) ? 0x07030602u : 0x05010400u;
        const uint32_t z = __builtin_amdgcn_perm(b[c / 4], a[c / 4], sel);
        v[i] = (c & 1) ? fp8_pair<true>(z) : fp8_pair<false>(z);
      } else {
        v[i] = __builtin_amdgcn_perm(b[c / 2], a[c / 2], (c & 1) ? 0x07060302u : 0x05040100u);
      }
    }
    return v;
  }
};

// The larger of the four lanes that hold one query row (lane % 16), in all of them.
__device__ __forceinline__ float row_max(float x) {
  const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  x = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
  const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}

// How far (in powers of two) a score may lie over the reference before the
// reference moves: weights of up to 2^8 cost fp32 and bf16 nothing, and a
// reference that stands still costs no exchange between lanes and no rescaling.
constexpr float kSlack = 8.0f;

// Eight weights as operands of the product with the values, which are bf16: in two
// parts, which leaves 16 bits of each (one part alone measured an output error 5 to
// 30% over that of its own rounding).  The first is cut off, and the second is of a
// weight 2^-20 larger, so that neither is 0 or negative unless the weight is 0: an
// infinite value gives its infinity, not a NaN.
struct Weights {
  u32x4 most, rest;
  __device__ __forceinline__ explicit Weights(const float (&e)[8]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float a = e[2 * i], b = e[2 * i + 1];
      most[i] = __builtin_amdgcn_perm(__float_as_uint(b), __float_as_uint(a), 0x07060302u);
      const float a0 = __uint_as_float(__float_as_uint(a) & 0xffff0000u), b0 = __uint_as_float(__float_as_uint(b) & 0xffff0000u);
      rest[i] = pack_bf16(fmaf(a, 1.0f + 0x1p-20f, -a0), fmaf(b, 1.0f + 0x1p-20f, -b0));
    }
  }
};

// One step of the softmax of query row lane % 16 over the lane's 8 of 32 slots:
// the weights exp2(unit s - m) as the second product's operands.  m: the row's
// reference (-inf before the first slot that counts); l: this lane's part of the
// sum, of the weights in 32 bits; keep(j): slot j counts (asked unless `whole`);
// rescale(f): called, for all lanes, when the sums so far become f times as much.
template <typename Keep, typename Rescale>
__device__ __forceinline__ Weights softmax_step(const f32x4 (&s)[2], float unit, bool whole, Keep keep, float& m, float& l,
                                              Rescale rescale) {
  float e[8];
  // the largest in the branch that makes the exponents: after a merge the
  // compiler no longer knows them to be quiet and adds an instruction for each
  const auto largest = [&] { return fmaxf(fmaxf(fmaxf(fmaxf(fmaxf(fmaxf(fmaxf(e[0], e[1]), e[2]), e[3]), e[4]), e[5]), e[6]), e[7]); };
  const auto exponents = [&](float base) {
#pragma unroll
    for (int j = 0; j < 8; ++j) e[j] = fmaf(s[j / 4][j % 4], unit, -base);
    if (whole) return largest();
#pragma unroll
    for (int j = 0; j < 8; ++j) e[j] = keep(j) ? e[j] : -INFINITY;
    return largest();
  };
  const bool none = m == -INFINITY;
  const float base = none ? 0.0f : m;
  const float top = exponents(base);
  if (__any(top > (none ? -INFINITY : kSlack))) {
    const float m2 = fmaxf(m, base + row_max(top));
    const float back = m2 == -INFINITY ? 1.0f : exp2_fast(m - m2);
    m = m2;
    l *= back;
    rescale(back);
    exponents(m2 == -INFINITY ? 0.0f : m2);
  }
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    e[j] = exp2_fast(e[j]);
    l += e[j];
  }
  return Weights(e);
}

}  // namespace eldr
