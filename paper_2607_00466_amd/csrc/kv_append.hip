// moe_kv_append and moe_kv_append_norm: rotary positions with any number of axes
// (after norms of queries and keys, head by head), fused with the write of the new
// tokens' keys and values into the paged cache.
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
//
// Norms add a sum over the lanes of a row (in 64 bits: append_rows.hpp) and 16 weights
// in registers, read again only where a thread goes from queries to keys.  They cost
// waves (five or six a SIMD in place of eight), not bytes: 4096 tokens of 40 heads of 128 in bf16 18.5 us
// (4.6 TB/s), 4097 from fp32 to fp8 30 to 32 where the bytes take 25, 64 tokens 3.6 to 4.
// Six waves by the launch bound (five with fp8's divisions, which spill at six) gave 2 to
// 4%; the next head's row asked for early costs more waves than it gains (18.9 -> 20.0).
// Queries written past the caches take 4 us off the 4096, and give whoever reads them
// next 7 more (29.0 -> 32.2 with a copy of them behind), so they are not.
#include "append_rows.hpp"
#include "eldr_kv_cache.h"

namespace eldr {

constexpr int kAppendThreads = 256;

struct AppendArgs {
  Rotation turns;
  const int32_t* slots;
  uint16_t* q_out;
  const float *q_norm, *k_norm;  // [D] or null
  int64_t threads;  // T * lanes * (D / 16)
  float eps;
  int32_t Hq, heads, chunk_shift;
  int32_t lanes;    // threads that share a token's heads
};

template <typename In, bool FP8, bool INTERLEAVED, bool NORM>
__global__ __launch_bounds__(kAppendThreads, NORM ? (FP8 ? 5 : 6) : 8) void kv_append_kernel(
    AppendArgs a, Pages pg, const void* q, const void* k, const void* v, int64_t q_stride, int64_t k_stride,
    int64_t v_stride, const float* k_scale, const float* v_scale, void* k_cache, void* v_cache) {
  const int64_t id = (int64_t)blockIdx.x * kAppendThreads + threadIdx.x;
  if (id >= a.threads) return;
  const int chunk = (int)(id & ((1 << a.chunk_shift) - 1));
  const int64_t th = id >> a.chunk_shift;
  const int t = (int)(th / a.lanes);
  const bool in_rot = chunk * 16 < a.turns.rot;
  float c[8], s[8];  // of pairs [8 chunk, 8 chunk + 8)
  if (in_rot) load_angles(a.turns, t, chunk, c, s);
  const int slot = a.slots[t];
  const int page = slot >> pg.shift;
  const bool stored = slot >= 0 && pg.has(page);
  // the runs of a row that is turned, and their weights of the side that w_of names
  const Runs turned(chunk, a.turns.rot / 2, in_rot && !INTERLEAVED), plain(chunk, 0, false);
  const float* w_of = nullptr;
  float wx[8], wy[8];
  for (int head = (int)(th - (int64_t)t * a.lanes); head < a.heads; head += a.lanes) {
    // heads: the queries', the keys', the values'
    const bool is_q = head < a.Hq, is_v = head >= a.Hq + pg.Hkv;
    if (is_q ? a.q_out == nullptr : !stored) continue;
    const void* in = is_q ? q : is_v ? v : k;
    const int64_t stride = is_q ? q_stride : is_v ? v_stride : k_stride;
    const int h = head - (is_q ? 0 : is_v ? a.Hq + pg.Hkv : a.Hq);
    const bool turns = !is_v && in_rot;
    const int e0 = is_v ? plain.e0 : turned.e0, e1 = is_v ? plain.e1 : turned.e1;
    const In* src = reinterpret_cast<const In*>(in) + (int64_t)t * stride + (int64_t)h * pg.D;
    float x[8], y[8];
    load8(src + e0, x);
    load8(src + e1, y);
    if constexpr (NORM) {
      const float* w = is_q ? a.q_norm : is_v ? nullptr : a.k_norm;
      if (w) {
        if (w != w_of) {
          load8(w + e0, wx);
          load8(w + e1, wy);
          w_of = w;
        }
        const float i = row_scale(x, y, 1 << a.chunk_shift, a.eps);
        norm8(x, i, wx);
        norm8(y, i, wy);
      }
    }
    if (turns) turn_runs<INTERLEAVED>(x, y, c, s);
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

struct AppendRows {
  const void *q, *k, *v;
  int64_t q_stride, k_stride, v_stride;
  const float *k_scale, *v_scale;
  void *k_cache, *v_cache;
};

template <typename In, bool FP8, bool INTERLEAVED>
void launch_append(const AppendArgs& a, const Pages& pg, const AppendRows& r, unsigned blocks, hipStream_t s) {
  const auto kernel = a.q_norm || a.k_norm ? kv_append_kernel<In, FP8, INTERLEAVED, true> : kv_append_kernel<In, FP8, INTERLEAVED, false>;
  hipLaunchKernelGGL(kernel, dim3(blocks), dim3(kAppendThreads), 0, s, a, pg, r.q, r.k, r.v, r.q_stride, r.k_stride, r.v_stride,
                     r.k_scale, r.v_scale, r.k_cache, r.v_cache);
}

}  // namespace eldr

extern "C" int moe_kv_append_norm(const void* q, const void* k, const void* v, int64_t q_stride,
                                  int64_t k_stride, int64_t v_stride, int32_t in_type, int32_t T,
                                  const int32_t* positions, int32_t n_axes, const int32_t* pair_axis,
                                  const float* cos_table, const float* sin_table, int32_t max_pos,
                                  int32_t rot, int32_t interleaved, const int32_t* slots,
                                  moe_attn_dims d, const float* q_norm, const float* k_norm, float eps,
                                  const float* k_scale, const float* v_scale, uint16_t* q_out,
                                  void* k_cache, void* v_cache, void* stream) {
  using namespace eldr_host;
  int st = check_attn_dims(d);
  if (st != MOE_OK) return st;
  if (d.kv_type == MOE_KV_INT8) return MOE_ERR_UNSUPPORTED;  // its scales are a page's
  const AppendCheck check{q, k, v, q_stride, k_stride, v_stride, in_type, T, positions, n_axes, pair_axis,
                          cos_table, sin_table, max_pos, rot, q_out, k_cache, v_cache};
  if ((st = check.sizes(d)) != MOE_OK) return st;
  if (!norms_finite(eps)) return MOE_ERR_INVALID;
  if (T == 0) return MOE_OK;
  if (!slots) return MOE_ERR_INVALID;
  if ((st = check.pointers(d)) != MOE_OK) return st;
  if (!aligned4(slots) || !aligned4(k_scale) || !aligned4(v_scale) || !aligned16(q_norm) || !aligned16(k_norm))
    return MOE_ERR_UNSUPPORTED;
  eldr::AppendArgs a;
  a.turns = check.rotation();
  a.slots = slots;
  a.q_out = q_out;
  a.q_norm = q_norm, a.k_norm = k_norm, a.eps = eps;
  a.Hq = d.Hq;
  a.heads = d.Hq + 2 * d.Hkv;
  a.chunk_shift = __builtin_ctz((unsigned)d.D) - 4;
  // as few threads a token as still fill the chip: 2048 for each CU
  constexpr int64_t kFull = 256 * 2048;
  a.lanes = a.heads;
  while (a.lanes > 4 && (int64_t)T * ((a.lanes + 1) / 2) * (d.D / 16) >= kFull / 2) a.lanes = (a.lanes + 1) / 2;
  a.threads = (int64_t)T * a.lanes * (d.D / 16);
  const int64_t blocks = (a.threads + eldr::kAppendThreads - 1) / eldr::kAppendThreads;
  if (blocks > 0x7fffffffLL) return MOE_ERR_UNSUPPORTED;
  const eldr::AppendRows r{q, k, v, q_stride, k_stride, v_stride, k_scale, v_scale, k_cache, v_cache};
  const eldr::Pages pg = pages_of(d, nullptr);
  const unsigned n = (unsigned)blocks;
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  const bool fp8 = d.kv_type == MOE_KV_FP8;
  if (in_type == MOE_IN_FP32) {
    if (fp8 && interleaved) eldr::launch_append<float, true, true>(a, pg, r, n, s);
    else if (fp8) eldr::launch_append<float, true, false>(a, pg, r, n, s);
    else if (interleaved) eldr::launch_append<float, false, true>(a, pg, r, n, s);
    else eldr::launch_append<float, false, false>(a, pg, r, n, s);
  } else {
    if (fp8 && interleaved) eldr::launch_append<uint16_t, true, true>(a, pg, r, n, s);
    else if (fp8) eldr::launch_append<uint16_t, true, false>(a, pg, r, n, s);
    else if (interleaved) eldr::launch_append<uint16_t, false, true>(a, pg, r, n, s);
    else eldr::launch_append<uint16_t, false, false>(a, pg, r, n, s);
  }
  return launch_status();
}

extern "C" int moe_kv_append(const void* q, const void* k, const void* v, int64_t q_stride,
                             int64_t k_stride, int64_t v_stride, int32_t in_type, int32_t T,
                             const int32_t* positions, int32_t n_axes, const int32_t* pair_axis,
                             const float* cos_table, const float* sin_table, int32_t max_pos,
                             int32_t rot, int32_t interleaved, const int32_t* slots,
                             moe_attn_dims d, const float* k_scale, const float* v_scale,
                             uint16_t* q_out, void* k_cache, void* v_cache, void* stream) {
  return moe_kv_append_norm(q, k, v, q_stride, k_stride, v_stride, in_type, T, positions, n_axes, pair_axis,
                            cos_table, sin_table, max_pos, rot, interleaved, slots, d, nullptr, nullptr, 0.0f,
                            k_scale, v_scale, q_out, k_cache, v_cache, stream);
}
