// Rows of queries, keys and values on their way into the cache: what the kernels
// that append share.  A head of a token is one row of D values, taken by D / 16
// neighbouring lanes of 16 values each.
#pragma once

#include "attn_common.hpp"

namespace eldr {

// Eight consecutive values on their way.
template <typename In>
struct Raw8 {
  static constexpr int kWords = 2 * sizeof(In);
  u32x4 raw[kWords / 4];
  __device__ __forceinline__ void load(const In* p) {
#pragma unroll
    for (int i = 0; i < kWords / 4; ++i) raw[i] = reinterpret_cast<const u32x4*>(p)[i];
  }
  __device__ __forceinline__ void get(float (&x)[8]) const {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      if constexpr (sizeof(In) == 4) x[i] = __uint_as_float(raw[i / 4][i % 4]);
      else x[i] = __uint_as_float(i % 2 ? raw[0][i / 2] & 0xffff0000u : raw[0][i / 2] << 16);
    }
  }
};

// Eight consecutive values as fp32.
template <typename In>
__device__ __forceinline__ void load8(const In* p, float (&x)[8]) {
  Raw8<In> r;
  r.load(p);
  r.get(x);
}

__device__ __forceinline__ void store8_bf16(uint16_t* p, const float (&x)[8]) {
  u32x4 v;
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] = pack_bf16(x[2 * i], x[2 * i + 1]);
  *reinterpret_cast<u32x4*>(p) = v;
}

// e4m3 of x / scale, clamped (a NaN stays one).  The quotient is the correctly
// rounded one, not a product with a reciprocal, so that codes equal those of
// the definition.
__device__ __forceinline__ void store8_fp8(uint8_t* p, const float (&x)[8], float scale) {
  u32x2 v;
#pragma unroll
  for (int w = 0; w < 2; ++w) {
    float y[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float t = x[4 * w + i] / scale;
      y[i] = t > 448.f ? 448.f : t < -448.f ? -448.f : t;
    }
    int word = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], 0, false);
    word = __builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], word, true);
    v[w] = (uint32_t)word;
  }
  *reinterpret_cast<u32x2*>(p) = v;
}

// (a, b) -> (a c - b s, b c + a s), each product and the sum rounded.
__device__ __forceinline__ void turn(float& a, float& b, float c, float s) {
#pragma clang fp contract(off)
  const float ac = a * c, bs = b * s, bc = b * c, as = a * s;
  a = ac - bs;
  b = bc + as;
}

// A lane's two runs of 8 values of a row: the 8 pairs [8 chunk, 8 chunk + 8) where
// these turn and pairs are half a rotation apart, 16 neighbours where not.
struct Runs {
  int e0, e1;
  __device__ __forceinline__ Runs(int chunk, int half, bool split)
      : e0(split ? chunk * 8 : chunk * 16), e1(split ? chunk * 8 + half : chunk * 16 + 8) {}
};

struct Rotation {
  const int32_t *positions, *pair_axis;
  const float *cos_table, *sin_table;
  int32_t T, n_axes, max_pos, rot;
};

// The angles of pairs [8 chunk, 8 chunk + 8) of token t; NaN where there is none.
__device__ __forceinline__ void load_angles(const Rotation& a, int t, int chunk, float (&c)[8], float (&s)[8]) {
  const int pair = chunk * 8, half = a.rot / 2;
  int axis[8];
  bool one = true;  // axis for all of them
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    axis[i] = a.pair_axis[pair + i];
    one = one && axis[i] == axis[0];
  }
  const auto position = [&](int x) {
    const int p = (uint32_t)x < (uint32_t)a.n_axes ? a.positions[(int64_t)x * a.T + t] : -1;
    return (uint32_t)p < (uint32_t)a.max_pos ? p : -1;
  };
#pragma unroll
  for (int i = 0; i < 8; ++i) c[i] = s[i] = __builtin_nanf("");
  if (one) {
    const int p = position(axis[0]);
    if (p >= 0) {
      load8(a.cos_table + (int64_t)p * half + pair, c);
      load8(a.sin_table + (int64_t)p * half + pair, s);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int p = position(axis[i]);
      if (p >= 0) {
        c[i] = a.cos_table[(int64_t)p * half + pair + i];
        s[i] = a.sin_table[(int64_t)p * half + pair + i];
      }
    }
  }
}

// A lane's pairs turned.
template <bool INTERLEAVED>
__device__ __forceinline__ void turn_runs(float (&x)[8], float (&y)[8], const float (&c)[8], const float (&s)[8]) {
  if constexpr (INTERLEAVED) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      turn(x[2 * i], x[2 * i + 1], c[i], s[i]);
      turn(y[2 * i], y[2 * i + 1], c[4 + i], s[4 + i]);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) turn(x[i], y[i], c[i], s[i]);
  }
}

// The sum of x over the `lanes` (4, 8 or 16) neighbouring lanes of a row, in all of
// them: exchanges inside a row of 16 lanes.
template <int CTRL>
__device__ __forceinline__ double dpp_double(double x) {
  const uint64_t b = __builtin_bit_cast(uint64_t, x);
  const uint32_t lo = __builtin_amdgcn_update_dpp(0, (int)(uint32_t)b, CTRL, 0xf, 0xf, true);
  const uint32_t hi = __builtin_amdgcn_update_dpp(0, (int)(uint32_t)(b >> 32), CTRL, 0xf, 0xf, true);
  return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}
__device__ __forceinline__ double row_sum(double x, int lanes) {
  x += dpp_double<0xb1>(x);                    // quad_perm 1 0 3 2
  x += dpp_double<0x4e>(x);                    // quad_perm 2 3 0 1
  if (lanes >= 8) x += dpp_double<0x141>(x);   // row_half_mirror
  if (lanes >= 16) x += dpp_double<0x140>(x);  // row_mirror
  return x;
}

// 1 / sqrt(mean of squares + eps) of a row, of which the lane holds x and y.  In 64
// bits, then rounded: a code of the cache turns on the last bit of its value, and so
// it does not depend on the order of a sum.  The estimate's error (2^-23 at most)
// is squared twice.
__device__ __forceinline__ float row_scale(const float (&x)[8], const float (&y)[8], int lanes, float eps) {
  double sum = 0.0;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    sum = __builtin_fma((double)x[i], (double)x[i], sum);
    sum = __builtin_fma((double)y[i], (double)y[i], sum);
  }
  const double m = __builtin_fma(row_sum(sum, lanes), 0.0625 / lanes, (double)eps);
  double r = __builtin_amdgcn_rsq(m);
  // (0 and infinity have no step to make)
  const bool plain = m > 0.0 && m < __builtin_inf();
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const double next = __builtin_fma(r * 0.5, __builtin_fma(-m * r, r, 1.0), r);
    r = plain ? next : r;
  }
  return (float)r;
}

// x = (x i) w, each product rounded.
__device__ __forceinline__ void norm8(float (&x)[8], float i, const float (&w)[8]) {
#pragma clang fp contract(off)
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const float t = x[e] * i;
    x[e] = t * w[e];
  }
}

}  // namespace eldr

namespace eldr_host {

// What the calls that append check alike of their rows and rotation.
struct AppendCheck {
  const void *q, *k, *v;
  int64_t q_stride, k_stride, v_stride;
  int32_t in_type, T;
  const int32_t* positions;
  int32_t n_axes;
  const int32_t* pair_axis;
  const float *cos_table, *sin_table;
  int32_t max_pos, rot;
  const void *q_out, *k_cache, *v_cache;
  // of the sizes, in the order of the header's refusals
  int sizes(const moe_attn_dims& d) const {
    if (T < 0 || n_axes < 0 || max_pos < 0 || rot < 0 || rot > d.D) return MOE_ERR_INVALID;
    if (in_type != MOE_IN_BF16 && in_type != MOE_IN_FP32) return MOE_ERR_INVALID;
    if (T > MOE_ATTN_MAX_APPEND || n_axes > MOE_ATTN_MAX_AXES || rot % 16 != 0) return MOE_ERR_UNSUPPORTED;
    return MOE_OK;
  }
  int pointers(const moe_attn_dims& d) const {
    if (!k || !v || (q_out && !q) || (d.num_blocks > 0 && (!k_cache || !v_cache))) return MOE_ERR_INVALID;
    if (rot > 0 && (!pair_axis || (n_axes > 0 && !positions) || (max_pos > 0 && (!cos_table || !sin_table))))
      return MOE_ERR_INVALID;
    if (k_stride < (int64_t)d.Hkv * d.D || v_stride < (int64_t)d.Hkv * d.D ||
        (q_out && q_stride < (int64_t)d.Hq * d.D))
      return MOE_ERR_INVALID;
    if ((q_out && q_stride % 8 != 0) || k_stride % 8 != 0 || v_stride % 8 != 0) return MOE_ERR_UNSUPPORTED;
    if (!aligned16(q) || !aligned16(k) || !aligned16(v) || !aligned16(q_out) || !aligned16(k_cache) ||
        !aligned16(v_cache) || !aligned16(cos_table) || !aligned16(sin_table) || !aligned4(positions) ||
        !aligned4(pair_axis))
      return MOE_ERR_UNSUPPORTED;
    return MOE_OK;
  }
  eldr::Rotation rotation() const {
    return eldr::Rotation{positions, pair_axis, cos_table, sin_table, T, n_axes, max_pos, rot};
  }
};

inline bool norms_finite(float eps) { return eps >= 0.0f && eps <= 3.4028235e38f; }

}  // namespace eldr_host
