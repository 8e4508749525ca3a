// moe_attn_decode's entry points (the kernels: attn_decode.hpp), for caches of bf16
// and fp8; those for 8-bit integers are compiled beside them, in attn_decode_int8.hip.
#include "attn_decode.hpp"

namespace eldr {

template <int D>
size_t decode_workspace(int64_t rows, int R) {
  const Parts p(nullptr, rows, D, SharedTile<D>::kRowsWg);
  // the plan of at most MOE_ATTN_MAX_R groups
  return reinterpret_cast<uintptr_t>(p.plan) + Plan::bytes(R, MOE_ATTN_MAX_R);
}

}  // namespace eldr

extern "C" size_t moe_attn_workspace_bytes(moe_attn_dims d) {
  if (eldr_host::check_attn_dims(d) != MOE_OK) return 0;
  const int64_t rows = (int64_t)d.R * d.Hq;
  return d.D == 64    ? eldr::decode_workspace<64>(rows, d.R)
         : d.D == 128 ? eldr::decode_workspace<128>(rows, d.R)
                      : eldr::decode_workspace<256>(rows, d.R);
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
      (d.num_blocks > 0 && (!k_cache || !v_cache)) || (n_groups > 0 && (!group_start || !prefix_len)) ||
      (d.kv_type == MOE_KV_INT8 && d.num_blocks > 0 && (!k_scale || !v_scale)))
    return MOE_ERR_INVALID;
  if (!aligned16(q) || !aligned16(out) || !aligned16(k_cache) || !aligned16(v_cache) || !aligned16(ws) ||
      !aligned4(block_table) || !aligned4(lens) || !aligned4(group_start) || !aligned4(prefix_len) ||
      !aligned4(k_scale) || !aligned4(v_scale) || !aligned4(sinks) || !aligned4(lse))
    return MOE_ERR_UNSUPPORTED;
  if (ws_bytes < moe_attn_workspace_bytes(d)) return MOE_ERR_WORKSPACE;
  eldr::DecodeArgs a;
  a.q = q, a.k_cache = static_cast<const char*>(k_cache), a.v_cache = static_cast<const char*>(v_cache);
  a.gr = eldr::Groups{lens, group_start, prefix_len, d.R, window > 0 ? 0 : n_groups, window};
  a.k_scale = k_scale, a.v_scale = v_scale, a.sinks = sinks;
  a.out = out, a.lse = lse, a.scale = scale;
  a.Hq = d.Hq, a.G = d.Hq / d.Hkv, a.head_tiles = (a.G + eldr::kRows - 1) / eldr::kRows;
  eldr::Pages pg = pages_of(d, block_table);
  if (d.num_blocks == 0) pg.max_blocks = 0;  // nothing is cached
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  float* w = static_cast<float*>(ws);
  const auto launch = [&](auto width) {
    constexpr int D = decltype(width)::value;
    return d.kv_type == MOE_KV_INT8  ? eldr::launch_decode_int8(D, a, pg, w, s)
           : d.kv_type == MOE_KV_FP8 ? eldr::launch_decode<D, eldr::kKvFp8>(a, pg, w, s)
                                     : eldr::launch_decode<D, eldr::kKvBf16>(a, pg, w, s);
  };
  return d.D == 64    ? launch(std::integral_constant<int, 64>())
         : d.D == 128 ? launch(std::integral_constant<int, 128>())
                      : launch(std::integral_constant<int, 256>());
}
