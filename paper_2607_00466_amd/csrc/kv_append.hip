// moe_kv_append: rotary positions with any number of axes, fused with the
// write of the new tokens' keys and values into the paged cache.
//
// One thread turns 16 values of a head of a token, i.e. the 8 pairs [8c, 8c + 8)
// of its two half-heads (or of 16 neighbouring values where pairs are
// interleaved), so every load and store is 16 bytes or more and both values of a
// pair are in one thread.  Where there are tokens enough to fill the chip, a
// thread does so for several heads with the angles it has read once: a token's
// angles are as many bytes as a head's values.  Bound by bytes for a prompt and
// by two dependent loads (position, then table) for a decode batch.  Measured: 4096
// tokens of 40 heads of 128 in fp32 25 us (5.0 TB/s, a large copy's rate; 54 us with
// a head a thread), 64 tokens in bf16 3.7 us; 1001 tokens of 80 heads of 64 to fp8
// 7.3 us where the bytes take 4: all 5008 waves are resident at once, so the small
// batch's latency is there beside the bytes.
#include "attn_common.hpp"

namespace eldr {

constexpr int kAppendThreads = 256;

struct AppendArgs {
  const int32_t *positions, *pair_axis, *slots;
  const float *cos_table, *sin_table;
  uint16_t* q_out;
  int64_t threads;  // T * lanes * (D / 16)
  int32_t T, n_axes, max_pos, rot, Hq, heads, chunk_shift;
  int32_t lanes;    // threads that share a token's heads
};

// Eight consecutive values as fp32.
template <typename In>
__device__ __forceinline__ void load8(const In* p, float (&x)[8]) {
  if constexpr (sizeof(In) == 4) {
    const f32x4 a = *reinterpret_cast<const f32x4*>(p);
    const f32x4 b = *reinterpret_cast<const f32x4*>(p + 4);
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = a[i], x[4 + i] = b[i];
  } else {
    const u32x4 a = *reinterpret_cast<const u32x4*>(p);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[2 * i] = __uint_as_float(a[i] << 16);
      x[2 * i + 1] = __uint_as_float(a[i] & 0xffff0000u);
    }
  }
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

template <typename In, bool FP8, bool INTERLEAVED>
__global__ __launch_bounds__(kAppendThreads) void kv_append_kernel(
    AppendArgs a, Pages pg, const void* q, const void* k, const void* v, int64_t q_stride, int64_t k_stride,
    int64_t v_stride, const float* k_scale, const float* v_scale, void* k_cache, void* v_cache) {
  const int64_t id = (int64_t)blockIdx.x * kAppendThreads + threadIdx.x;
  if (id >= a.threads) return;
  const int chunk = (int)(id & ((1 << a.chunk_shift) - 1));
  const int64_t th = id >> a.chunk_shift;
  const int t = (int)(th / a.lanes);
  const int half = a.rot / 2;
  const bool in_rot = chunk * 16 < a.rot;
  float c[8], s[8];  // of pairs [8 chunk, 8 chunk + 8)
  if (in_rot) {
    const int pair = chunk * 8;
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
  const int slot = a.slots[t];
  const int page = slot >> pg.shift;
  const bool stored = slot >= 0 && pg.has(page);
  for (int head = (int)(th - (int64_t)t * a.lanes); head < a.heads; head += a.lanes) {
    // heads: the queries', the keys', the values'
    const bool is_q = head < a.Hq, is_v = head >= a.Hq + pg.Hkv;
    if (is_q ? a.q_out == nullptr : !stored) continue;
    const void* in = is_q ? q : is_v ? v : k;
    const int64_t stride = is_q ? q_stride : is_v ? v_stride : k_stride;
    const int h = head - (is_q ? 0 : is_v ? a.Hq + pg.Hkv : a.Hq);
    const bool turns = !is_v && in_rot;
    // the thread's two runs of 8 values
    const int e0 = turns && !INTERLEAVED ? chunk * 8 : chunk * 16;
    const int e1 = turns && !INTERLEAVED ? chunk * 8 + half : chunk * 16 + 8;
    const In* src = reinterpret_cast<const In*>(in) + (int64_t)t * stride + (int64_t)h * pg.D;
    float x[8], y[8];
    load8(src + e0, x);
    load8(src + e1, y);
    if (turns) {
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
    if (is_q) {
      uint16_t* dst = a.q_out + ((int64_t)t * a.Hq + h) * pg.D;
      store8_bf16(dst + e0, x);
      store8_bf16(dst + e1, y);
      continue;
    }
    const int64_t row = pg.row(page, h, slot);
    if constexpr (FP8) {
      const float* scales = is_v ? v_scale : k_scale;
      const float scale = scales ? scales[h] : 1.0f;
      uint8_t* dst = reinterpret_cast<uint8_t*>(is_v ? v_cache : k_cache) + row;
      store8_fp8(dst + e0, x, scale);
      store8_fp8(dst + e1, y, scale);
    } else {
      uint16_t* dst = reinterpret_cast<uint16_t*>(is_v ? v_cache : k_cache) + row;
      store8_bf16(dst + e0, x);
      store8_bf16(dst + e1, y);
    }
  }
}

}  // namespace eldr

extern "C" int moe_kv_append(const void* q, const void* k, const void* v, int64_t q_stride,
                             int64_t k_stride, int64_t v_stride, int32_t in_type, int32_t T,
                             const int32_t* positions, int32_t n_axes, const int32_t* pair_axis,
                             const float* cos_table, const float* sin_table, int32_t max_pos,
                             int32_t rot, int32_t interleaved, const int32_t* slots,
                             moe_attn_dims d, const float* k_scale, const float* v_scale,
                             uint16_t* q_out, void* k_cache, void* v_cache, void* stream) {
  using namespace eldr_host;
  int st = check_attn_dims(d);
  if (st != MOE_OK) return st;
  if (T < 0 || n_axes < 0 || max_pos < 0 || rot < 0 || rot > d.D) return MOE_ERR_INVALID;
  if (in_type != MOE_IN_BF16 && in_type != MOE_IN_FP32) return MOE_ERR_INVALID;
  if (T > MOE_ATTN_MAX_APPEND || n_axes > MOE_ATTN_MAX_AXES || rot % 16 != 0) return MOE_ERR_UNSUPPORTED;
  if (T == 0) return MOE_OK;
  if (!k || !v || !slots || (q_out && !q) || (d.num_blocks > 0 && (!k_cache || !v_cache))) return MOE_ERR_INVALID;
  if (rot > 0 && (!pair_axis || (n_axes > 0 && !positions) || (max_pos > 0 && (!cos_table || !sin_table))))
    return MOE_ERR_INVALID;
  if (k_stride < (int64_t)d.Hkv * d.D || v_stride < (int64_t)d.Hkv * d.D ||
      (q_out && q_stride < (int64_t)d.Hq * d.D))
    return MOE_ERR_INVALID;
  if ((q_out && q_stride % 8 != 0) || k_stride % 8 != 0 || v_stride % 8 != 0) return MOE_ERR_UNSUPPORTED;
  if (!aligned16(q) || !aligned16(k) || !aligned16(v) || !aligned16(q_out) || !aligned16(k_cache) ||
      !aligned16(v_cache) || !aligned16(cos_table) || !aligned16(sin_table) || !aligned4(positions) ||
      !aligned4(pair_axis) || !aligned4(slots) || !aligned4(k_scale) || !aligned4(v_scale))
    return MOE_ERR_UNSUPPORTED;
  eldr::AppendArgs a;
  a.positions = positions, a.pair_axis = pair_axis, a.slots = slots;
  a.cos_table = cos_table, a.sin_table = sin_table;
  a.q_out = q_out;
  a.T = T, a.n_axes = n_axes, a.max_pos = max_pos, a.rot = rot, a.Hq = d.Hq;
  a.heads = d.Hq + 2 * d.Hkv;
  a.chunk_shift = __builtin_ctz((unsigned)d.D) - 4;
  // as few threads a token as still fill the chip: 2048 for each CU
  constexpr int64_t kFull = 256 * 2048;
  a.lanes = a.heads;
  while (a.lanes > 4 && (int64_t)T * ((a.lanes + 1) / 2) * (d.D / 16) >= kFull / 2) a.lanes = (a.lanes + 1) / 2;
  a.threads = (int64_t)T * a.lanes * (d.D / 16);
  const int64_t blocks = (a.threads + eldr::kAppendThreads - 1) / eldr::kAppendThreads;
  if (blocks > 0x7fffffffLL) return MOE_ERR_UNSUPPORTED;
  const dim3 grid((unsigned)blocks), block(eldr::kAppendThreads);
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  const eldr::Pages pg = pages_of(d, nullptr);
  const bool fp8 = d.kv_type == MOE_KV_FP8;
#define ELDR_APPEND(IN, F, P) \
  hipLaunchKernelGGL((eldr::kv_append_kernel<IN, F, P>), grid, block, 0, s, a, pg, q, k, v, q_stride, k_stride, \
                     v_stride, k_scale, v_scale, k_cache, v_cache)
  if (in_type == MOE_IN_FP32) {
    if (fp8 && interleaved) ELDR_APPEND(float, true, true);
    else if (fp8) ELDR_APPEND(float, true, false);
    else if (interleaved) ELDR_APPEND(float, false, true);
    else ELDR_APPEND(float, false, false);
  } else {
    if (fp8 && interleaved) ELDR_APPEND(uint16_t, true, true);
    else if (fp8) ELDR_APPEND(uint16_t, true, false);
    else if (interleaved) ELDR_APPEND(uint16_t, false, true);
    else ELDR_APPEND(uint16_t, false, false);
  }
#undef ELDR_APPEND
  return launch_status();
}
