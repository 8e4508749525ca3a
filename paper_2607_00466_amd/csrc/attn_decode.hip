// moe_attn_decode: one wave a (request, query head), 64 keys at a time, with
// the running maximum and sum of the softmax.
#include "attn_common.hpp"

namespace eldr {

struct DecodeArgs {
  const uint16_t* q;
  const void *k_cache, *v_cache;
  const int32_t *lens, *group_start, *prefix_len;
  const float *k_scale, *v_scale, *sinks;
  uint16_t* out;
  float* lse;
  float scale;
  int32_t R, Hq, n_groups, window;
};

template <bool FP8>
__device__ __forceinline__ float cached(const void* p, int64_t i) {
  if constexpr (FP8)
    return __builtin_amdgcn_cvt_f32_fp8((int)reinterpret_cast<const uint8_t*>(p)[i], 0);
  else
    return bf16_to_float(reinterpret_cast<const uint16_t*>(p)[i]);
}

// The first request of r's group and the slots it shares (0: none).
__device__ inline int shared_slots(const DecodeArgs& a, int capacity, int r, int& first) {
  first = r;
  if (a.window > 0) return 0;
  int s = min(max(a.group_start ? a.group_start[0] : 0, 0), a.R);
  for (int g = 0; g < a.n_groups; ++g) {
    const int e = min(max(a.group_start[g + 1], s), a.R);
    if (r >= s && r < e && e - s > 1) {
      int reach = min(max(a.prefix_len[g], 0), capacity);
      for (int i = s; i < e; ++i)
        if (a.lens[i] > 0) reach = min(reach, a.lens[i]);
      first = s;
      return reach;
    }
    s = e;
  }
  return 0;
}

template <bool FP8>
__global__ __launch_bounds__(64) void attn_decode_simple(DecodeArgs a, Pages pg) {
  const int r = blockIdx.x / a.Hq, hq = blockIdx.x % a.Hq, lane = threadIdx.x;
  const int h = hq / (a.Hq / pg.Hkv);
  const int D = pg.D;
  __shared__ float qs[256], ps[64];
  __shared__ int64_t rows[64];
  const int64_t qo = ((int64_t)r * a.Hq + hq) * D;
  const float ks = (FP8 && a.k_scale ? a.k_scale[h] : 1.f) * a.scale;
  const float vs = FP8 && a.v_scale ? a.v_scale[h] : 1.f;
  for (int i = lane; i < D; i += 64) qs[i] = bf16_to_float(a.q[qo + i]);
  int first;
  const int reach = shared_slots(a, pg.capacity(), r, first);
  const int n = min(max(a.lens[r], 0), pg.capacity());
  const int lo = a.window > 0 ? max(0, n - a.window) : 0;
  float m = -INFINITY, l = 0.f, acc[4] = {0.f, 0.f, 0.f, 0.f};
  if (a.sinks) m = a.sinks[hq], l = 1.f;
  for (int j0 = lo; j0 < n; j0 += 64) {
    __syncthreads();
    const int j = j0 + lane;
    float s = -INFINITY;
    int64_t row = -1;
    if (j < n) {
      const int b = pg.page(j < reach ? first : r, j);
      if (pg.has(b)) {
        row = pg.row(b, h, j);
        float dot = 0.f;
        for (int i = 0; i < D; ++i) dot = fmaf(qs[i], cached<FP8>(a.k_cache, row + i), dot);
        s = dot * ks;
      }
    }
    float top = s;
    for (int o = 32; o; o >>= 1) top = fmaxf(top, __shfl_xor(top, o));
    const float m2 = fmaxf(m, top);
    const float p = row < 0 || m2 == -INFINITY ? 0.f : __expf(s - m2);
    float sum = p;
    for (int o = 32; o; o >>= 1) sum += __shfl_xor(sum, o);
    const float back = m2 == -INFINITY ? 1.f : __expf(m - m2);
    l = l * back + sum;
    m = m2;
    ps[lane] = p;
    rows[lane] = row;
    __syncthreads();
    for (int c = 0; c < 4; ++c) acc[c] *= back;
    for (int k = 0; k < 64; ++k) {
      if (rows[k] < 0) continue;
      for (int c = 0; c < D / 64; ++c) acc[c] = fmaf(ps[k], cached<FP8>(a.v_cache, rows[k] + c * 64 + lane), acc[c]);
    }
  }
  const float inv = l > 0.f ? vs / l : 0.f;
  for (int c = 0; c < D / 64; ++c) a.out[qo + c * 64 + lane] = (uint16_t)pack_bf16(acc[c] * inv, 0.f);
  if (lane == 0 && a.lse) a.lse[(int64_t)r * a.Hq + hq] = l > 0.f ? m + __logf(l) : -INFINITY;
}

}  // namespace eldr

extern "C" size_t moe_attn_workspace_bytes(moe_attn_dims d) {
  if (eldr_host::check_attn_dims(d) != MOE_OK) return 0;
  return 16;
}

extern "C" int moe_attn_decode(const uint16_t* q, const void* k_cache, const void* v_cache,
                               const int32_t* block_table, const int32_t* lens,
                               const int32_t* group_start, const int32_t* prefix_len,
                               int32_t n_groups, const float* k_scale, const float* v_scale,
                               const float* sinks, int32_t window, float scale, moe_attn_dims d,
                               uint16_t* out, float* lse, void* ws, size_t ws_bytes, void* stream) {
  using namespace eldr_host;
  int st = check_attn_dims(d);
  if (st != MOE_OK) return st;
  if (n_groups < 0 || n_groups > MOE_ATTN_MAX_R || window < 0 || !(scale == scale)) return MOE_ERR_INVALID;
  if (d.R == 0) return MOE_OK;
  if (!q || !lens || !out || !ws || (d.max_blocks > 0 && !block_table) ||
      (d.num_blocks > 0 && (!k_cache || !v_cache)) || (n_groups > 0 && (!group_start || !prefix_len)))
    return MOE_ERR_INVALID;
  if (!aligned16(q) || !aligned16(out) || !aligned16(k_cache) || !aligned16(v_cache) || !aligned16(ws) ||
      !aligned4(block_table) || !aligned4(lens) || !aligned4(group_start) || !aligned4(prefix_len) ||
      !aligned4(k_scale) || !aligned4(v_scale) || !aligned4(sinks) || !aligned4(lse))
    return MOE_ERR_UNSUPPORTED;
  if (ws_bytes < moe_attn_workspace_bytes(d)) return MOE_ERR_WORKSPACE;
  eldr::DecodeArgs a;
  a.q = q, a.k_cache = k_cache, a.v_cache = v_cache, a.lens = lens;
  a.group_start = group_start, a.prefix_len = prefix_len, a.k_scale = k_scale, a.v_scale = v_scale;
  a.sinks = sinks, a.out = out, a.lse = lse, a.scale = scale;
  a.R = d.R, a.Hq = d.Hq, a.n_groups = n_groups, a.window = window;
  const eldr::Pages pg = pages_of(d, block_table);
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  const dim3 grid(d.R * d.Hq), block(64);
  if (d.kv_type == MOE_KV_FP8)
    hipLaunchKernelGGL(eldr::attn_decode_simple<true>, grid, block, 0, s, a, pg);
  else
    hipLaunchKernelGGL(eldr::attn_decode_simple<false>, grid, block, 0, s, a, pg);
  return launch_status();
}
