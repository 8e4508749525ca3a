// moe_attn_weights: one thread a (request, kv head, slot).
#include "attn_common.hpp"

namespace eldr {

struct WeightArgs {
  const uint16_t* q;
  const void* k_cache;
  const int32_t *lens, *group_start, *prefix_len;
  const float *k_scale, *lse, *weights_in;
  float* weights_out;
  float scale;
  int32_t R, Hq, n_groups;
};

template <bool FP8>
__global__ __launch_bounds__(256) void attn_weights_simple(WeightArgs a, Pages pg) {
  const int r = blockIdx.y / pg.Hkv, h = blockIdx.y % pg.Hkv, G = a.Hq / pg.Hkv;
  const int n = min(max(a.lens[r], 0), pg.capacity());
  const int j = blockIdx.x * 256 + threadIdx.x;
  if (j >= n) return;
  int first = r, reach = 0;
  int s0 = a.n_groups ? min(max(a.group_start[0], 0), a.R) : 0;
  for (int g = 0; g < a.n_groups; ++g) {
    const int e0 = min(max(a.group_start[g + 1], s0), a.R);
    if (r >= s0 && r < e0 && e0 - s0 > 1) {
      first = s0;
      reach = min(max(a.prefix_len[g], 0), pg.capacity());
      for (int i = s0; i < e0; ++i)
        if (a.lens[i] > 0) reach = min(reach, a.lens[i]);
    }
    s0 = e0;
  }
  const int b = pg.page(j < reach ? first : r, j);
  float sum = 0.f;
  if (pg.has(b)) {
    const int64_t row = pg.row(b, h, j);
    const float ks = (FP8 && a.k_scale ? a.k_scale[h] : 1.f) * a.scale;
    for (int g = 0; g < G; ++g) {
      const int64_t rq = (int64_t)r * a.Hq + h * G + g;
      float dot = 0.f;
      for (int i = 0; i < pg.D; ++i) {
        const float k = FP8 ? __builtin_amdgcn_cvt_f32_fp8((int)reinterpret_cast<const uint8_t*>(a.k_cache)[row + i], 0)
                            : bf16_to_float(reinterpret_cast<const uint16_t*>(a.k_cache)[row + i]);
        dot = fmaf(bf16_to_float(a.q[rq * pg.D + i]), k, dot);
      }
      sum += __expf(dot * ks - a.lse[rq]);
    }
  }
  const int64_t at = ((int64_t)r * pg.Hkv + h) * pg.capacity() + j;
  a.weights_out[at] = (a.weights_in ? a.weights_in[at] : 0.f) + sum;
}

}  // namespace eldr

extern "C" int moe_attn_weights(const uint16_t* q, const void* k_cache, const int32_t* block_table,
                                const int32_t* lens, const int32_t* group_start,
                                const int32_t* prefix_len, int32_t n_groups, const float* k_scale,
                                float scale, const float* lse, moe_attn_dims d,
                                const float* weights_in, float* weights_out, void* stream) {
  using namespace eldr_host;
  int st = check_attn_dims(d);
  if (st != MOE_OK) return st;
  if (n_groups < 0 || n_groups > MOE_ATTN_MAX_R || !(scale == scale)) return MOE_ERR_INVALID;
  if (d.R == 0 || d.max_blocks == 0) return MOE_OK;
  if (!q || !lens || !lse || !weights_out || !block_table || (d.num_blocks > 0 && !k_cache) ||
      (n_groups > 0 && (!group_start || !prefix_len)))
    return MOE_ERR_INVALID;
  if (!aligned16(q) || !aligned16(k_cache) || !aligned16(weights_in) || !aligned16(weights_out) ||
      !aligned4(block_table) || !aligned4(lens) || !aligned4(group_start) || !aligned4(prefix_len) ||
      !aligned4(k_scale) || !aligned4(lse))
    return MOE_ERR_UNSUPPORTED;
  eldr::WeightArgs a;
  a.q = q, a.k_cache = k_cache, a.lens = lens, a.group_start = group_start, a.prefix_len = prefix_len;
  a.k_scale = k_scale, a.lse = lse, a.weights_in = weights_in, a.weights_out = weights_out;
  a.scale = scale, a.R = d.R, a.Hq = d.Hq, a.n_groups = n_groups;
  const eldr::Pages pg = pages_of(d, block_table);
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  const int64_t N = (int64_t)d.max_blocks * d.block_size;
  if ((int64_t)d.R * d.Hkv > 65535) return MOE_ERR_UNSUPPORTED;
  const dim3 grid((unsigned)((N + 255) / 256), d.R * d.Hkv), block(256);
  if (d.kv_type == MOE_KV_FP8)
    hipLaunchKernelGGL(eldr::attn_weights_simple<true>, grid, block, 0, s, a, pg);
  else
    hipLaunchKernelGGL(eldr::attn_weights_simple<false>, grid, block, 0, s, a, pg);
  return launch_status();
}
