// moe_attn_weights: the attention weight of every cached token, summed over the
// query heads of its kv head.
//
// The row statistics are known (lse), so a weight is exp(score - lse) and one
// pass over the keys is all: S = Q K^T by MFMA with the slots on the columns, so
// that the sum over a request's heads is a sum over rows, three additions in a
// lane and one or two lane exchanges, and 16 neighbouring lanes hold 16
// neighbouring slots.  Rows are laid out so that a 16-row tile holds whole
// requests: G is padded to a power of two (or to a multiple of 16), and a padded
// row's lse of +inf makes its weights zero.
//
// A wave takes 32 slots at a time; a unit is 128 slots of one request, or of a
// group against a run of its members' rows, dealt out as for moe_attn_decode.
// Bound by HBM: keys once, weights in and out.
#include "attn_plan.hpp"
#include "attn_tile.hpp"

namespace eldr {

constexpr int kWeightThreads = 256;
constexpr int kWeightWaves = kWeightThreads / kWave;
constexpr int kWeightWgs = 1024;  // four for each CU
constexpr int kMemberRows = 64;   // rows of a shared unit, of requests of up to 16 rows

struct WeightArgs {
  const uint16_t* q;
  const char* k_cache;
  Groups gr;
  const float *k_scale, *lse, *weights_in;
  float* weights_out;
  float scale;
  int32_t Hq, G, pad;  // pad: rows a request takes, a power of two up to 16 or a multiple of 16
};

// Requests [first, end), of which those in `group` (-1: all) count; rows
// [row0, row1) of their padded heads; slots [k0, k1).
struct Span {
  int table_row, first, end, group, row0, row1, h, k0, k1;
};

// A 16-row tile's queries and lse (in base-2 units): row 16 t + lane % 16 as the
// operand, rows 4 (lane / 16) + i as results.
template <int D, bool FP8>
__device__ __forceinline__ void load_rows(const WeightArgs& a, const Span& sp, int row0, u32x4 (&q)[D / 32], f32x4& lse) {
  const int lane = threadIdx.x % kWave, n = lane % 16, g = lane / 16;
  const int row = row0 + n, req = sp.first + row / a.pad, i = row % a.pad;
  const bool live = i < a.G && req < sp.end;
  const uint16_t* src = a.q + ((int64_t)(live ? req : sp.first) * a.Hq + sp.h * a.G + (live ? i : 0)) * D;
#pragma unroll
  for (int s = 0; s < D / 32; ++s) q[s] = *reinterpret_cast<const u32x4*>(src + Tile<D, FP8>::q_at(s, g));
#pragma unroll
  for (int c = 0; c < 4; ++c) {
    const int rr = row0 + 4 * g + c, r = sp.first + rr / a.pad, j = rr % a.pad;
    lse[c] = j < a.G && r < sp.end ? a.lse[(int64_t)r * a.Hq + sp.h * a.G + j] * kLog2e : INFINITY;
  }
}

template <int D, bool FP8>
__device__ __forceinline__ void weigh(const WeightArgs& a, const Pages& pg, const Span& sp, const int* group) {
  using T = Tile<D, FP8>;
  const int lane = threadIdx.x % kWave, n = lane % 16, g = lane / 16;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const float unit = a.scale * kLog2e * (FP8 && a.k_scale ? a.k_scale[sp.h] : 1.0f);
  const int32_t* table = pg.table + (int64_t)sp.table_row * pg.max_blocks;
  const int64_t N = pg.capacity();
  const int in_tile = min(a.pad, kRows);       // rows of one request in a tile
  const int per_request = (a.pad + kRows - 1) / kRows;  // tiles of one request
  u32x4 q[T::kK];
  f32x4 lse;
  const bool once = sp.row1 - sp.row0 <= kRows;  // one tile of rows: its operands stay
  if (once) load_rows<D, FP8>(a, sp, sp.row0, q, lse);
  const int k_first = sp.k0 / kStep * kStep + wave * kStep;
  StepPages pages = step_pages(pg, table, k_first);  // one step ahead
  for (int k = k_first; k < sp.k1; k += kWeightWaves * kStep) {
    const int b0 = pages.b0, b1 = pages.b1;
    pages = step_pages(pg, table, k + kWeightWaves * kStep);
    const bool has0 = pg.has(b0), has1 = pg.has(b1);
    Keys<D, FP8> keys[2];
    keys[0].load(a.k_cache + pg.row(has0 ? b0 : 0, sp.h, k) * T::kElem, n, g);
    keys[1].load(a.k_cache + pg.row(has1 ? b1 : 0, sp.h, k + 16) * T::kElem, n, g);
    const bool write[2] = {k + n >= sp.k0 && k + n < sp.k1, k + 16 + n >= sp.k0 && k + 16 + n < sp.k1};
    for (int row0 = sp.row0; row0 < sp.row1; row0 += kRows * per_request) {
      // what is there already, asked for with the keys
      float before[2][4];
      int64_t at[4];
      bool mine[4];
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        const int row = 4 * g + c, r = sp.first + (row0 + row) / a.pad;
        mine[c] = (c == 0 || in_tile <= c) && row % in_tile == 0 && r < sp.end && (sp.group < 0 || group[r] == sp.group);
        at[c] = ((int64_t)r * pg.Hkv + sp.h) * N + k + n;
#pragma unroll
        for (int t = 0; t < 2; ++t) before[t][c] = mine[c] && write[t] && a.weights_in ? a.weights_in[at[c] + 16 * t] : 0.0f;
      }
      f32x4 sum[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
      for (int part = 0; part < per_request; ++part) {
        if (!once) load_rows<D, FP8>(a, sp, row0 + part * kRows, q, lse);
        f32x4 s[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
#pragma unroll
        for (int i = 0; i < T::kK; ++i) {
          s[0] = mfma16x16x32(q[i], keys[0].operand(i), s[0]);
          s[1] = mfma16x16x32(q[i], keys[1].operand(i), s[1]);
        }
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
          for (int c = 0; c < 4; ++c) sum[t][c] += exp2_fast(fmaf(s[t][c], unit, -lse[c]));
      }
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        float x[4] = {sum[t][0], sum[t][1], sum[t][2], sum[t][3]};
        if (in_tile >= 2) x[0] += x[1], x[2] += x[3];
        if (in_tile >= 4) x[0] += x[2];
        if (in_tile >= 8) x[0] += __shfl_xor(x[0], 16);
        if (in_tile >= 16) x[0] += __shfl_xor(x[0], 32);
        const bool there = t ? has1 : has0;
#pragma unroll
        for (int c = 0; c < 4; ++c)
          if (mine[c] && write[t]) a.weights_out[at[c] + 16 * t] = before[t][c] + (there ? x[c] : 0.0f);
      }
    }
  }
}

template <int D, bool FP8>
__global__ __launch_bounds__(kWeightThreads, D == 256 ? 3 : 4) void attn_weights_kernel(WeightArgs a, Pages pg, int member_rows) {
  extern __shared__ int lds[];
  __shared__ int waves[kWeightWaves];
  const int capacity = pg.capacity();
  const Plan plan = make_plan<kWeightThreads>(a.gr, capacity, a.pad, member_rows, lds, waves);
  const int R = a.gr.R, n = a.gr.n, wgs = gridDim.x;
  const int own_row = plan.own[R], shared_row = plan.shared[n];
  // one line: the shared units, then the own ones
  const int shared_units = shared_row * pg.Hkv;
  const Deal deal(shared_units + own_row * pg.Hkv, wgs);
  if ((int)blockIdx.x >= deal.wgs) return;
  int u = __builtin_amdgcn_readfirstlane(deal.first(blockIdx.x));
  const int end = __builtin_amdgcn_readfirstlane(deal.first(blockIdx.x + 1));
  while (u < end) {
    Span sp;
    int tiles;
    if (u < shared_units) {
      const int h = u / shared_row, v = u - h * shared_row;
      const int grp = last_at(plan.shared, n, v);
      const int first = max(a.gr.start[grp], 0), last = min(a.gr.start[grp + 1], R), reach = plan.least[grp];
      const int per = tiles_of(0, reach), in = v - plan.shared[grp], run = in / per, t = in - run * per;
      tiles = min(per - t, end - u);
      sp = Span{first, first, last, grp, run * member_rows, min((run + 1) * member_rows, (last - first) * a.pad), h,
                t * kTile, min((t + tiles) * kTile, reach)};
    } else {
      const int o = u - shared_units, h = o / own_row, v = o - h * own_row;
      const int r = last_at(plan.own, R, v), t = v - plan.own[r];
      const int len = clamp_len(a.gr.lens[r], capacity), lo = min(plan.reach[r], len), t0 = lo / kTile;
      tiles = min(plan.own[r + 1] - v, end - u);
      sp = Span{r, r, r + 1, -1, 0, a.pad, h, max((t0 + t) * kTile, lo), min((t0 + t + tiles) * kTile, len)};
    }
    // the same for every lane: keep it in scalar registers
    int* f = reinterpret_cast<int*>(&sp);
#pragma unroll
    for (int i = 0; i < (int)(sizeof(sp) / 4); ++i) f[i] = __builtin_amdgcn_readfirstlane(f[i]);
    weigh<D, FP8>(a, pg, sp, plan.group);
    u += __builtin_amdgcn_readfirstlane(tiles);
  }
}

template <int D, bool FP8>
int launch_weights(const WeightArgs& a, const Pages& pg, hipStream_t s) {
  const int member_rows = a.pad > kRows ? a.pad : kMemberRows;
  hipLaunchKernelGGL((attn_weights_kernel<D, FP8>), dim3(kWeightWgs), dim3(kWeightThreads), Plan::bytes(a.gr.R, a.gr.n), s, a,
                     pg, member_rows);
  return eldr_host::launch_status();
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
  if (d.R == 0 || d.max_blocks == 0 || d.num_blocks == 0) return MOE_OK;
  if (!q || !lens || !lse || !weights_out || !block_table || !k_cache ||
      (n_groups > 0 && (!group_start || !prefix_len)))
    return MOE_ERR_INVALID;
  if (!aligned16(q) || !aligned16(k_cache) || !aligned16(weights_in) || !aligned16(weights_out) ||
      !aligned4(block_table) || !aligned4(lens) || !aligned4(group_start) || !aligned4(prefix_len) ||
      !aligned4(k_scale) || !aligned4(lse))
    return MOE_ERR_UNSUPPORTED;
  eldr::WeightArgs a;
  a.q = q, a.k_cache = static_cast<const char*>(k_cache);
  a.gr = eldr::Groups{lens, group_start, prefix_len, d.R, n_groups, 0};
  a.k_scale = k_scale, a.lse = lse, a.weights_in = weights_in, a.weights_out = weights_out, a.scale = scale;
  a.Hq = d.Hq, a.G = d.Hq / d.Hkv;
  a.pad = 1;
  while (a.pad < a.G && a.pad < eldr::kRows) a.pad *= 2;
  if (a.G > eldr::kRows) a.pad = (a.G + eldr::kRows - 1) / eldr::kRows * eldr::kRows;
  const eldr::Pages pg = pages_of(d, block_table);
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  const bool fp8 = d.kv_type == MOE_KV_FP8;
  if (d.D == 64) return fp8 ? eldr::launch_weights<64, true>(a, pg, s) : eldr::launch_weights<64, false>(a, pg, s);
  if (d.D == 128) return fp8 ? eldr::launch_weights<128, true>(a, pg, s) : eldr::launch_weights<128, false>(a, pg, s);
  return fp8 ? eldr::launch_weights<256, true>(a, pg, s) : eldr::launch_weights<256, false>(a, pg, s);
}
