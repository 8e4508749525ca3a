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
// A unit is 128 slots of one request, or of a group against up to kMemberTiles
// tiles of its members' rows, dealt out as for moe_attn_decode.  A wave keeps its
// rows' queries and lse in registers and takes 32 slots at a time, the next ones'
// keys on their way.  Own slots are bound by HBM: keys once, weights in and out
// (64 requests of up to 4000 tokens, 149 MB, 29 us, 5.1 TB/s; 64 of 16384, 1.11 GB,
// 206 to 210 us, 5.3 TB/s, 75% of a streaming read).  A prefix is bound by its steps: 64 requests behind 8192 slots take 26
// us where the bytes take 7; a step of 32 slots against 64 rows takes a wave 2.1 us,
// 0.9 of them products, exponents and sums, and a workgroup has six after 5 us of
// plan and rows (32 us while each of a tile's lse loads waited for the one before).
#include "attn_plan.hpp"
#include "attn_tile.hpp"

namespace eldr {

constexpr int kWeightThreads = 256;
constexpr int kWeightWaves = kWeightThreads / kWave;
constexpr int kWeightWgs = 512;  // two for each CU

// Row tiles of a shared unit, for requests of up to 16 rows: as many as a wave
// keeps in registers beside a lane's requests in each, 4 / pad.
constexpr int member_tiles(int D, int pad) { return pad == 1 || D == 256 ? 1 : pad == 2 ? 2 : 4; }

struct WeightArgs {
  const uint16_t* q;
  const char* k_cache;
  Groups gr;
  const float *k_scale, *lse, *weights_in;
  float* weights_out;
  float scale;
  int32_t Hq, G, pad;  // pad: rows a request takes, a power of two up to 16 or a multiple of 16
  int32_t pad_shift;   // of the former
};

// Requests [first, end), of which those in `group` (-1: all) count; rows
// [row0, row1) of their padded heads; slots [k0, k1), through row table_row of the
// block table.
struct Span {
  int table_row, first, end, group, row0, row1, h, k0, k1;
};

// A 16-row tile's queries and lse (in base-2 units): row 16 t + lane % 16 as the
// operand, rows 4 (lane / 16) + i as results.
template <int D, bool FP8>
__device__ __forceinline__ void load_rows(const WeightArgs& a, const Span& sp, int row0, u32x4 (&q)[D / 32], f32x4& lse) {
  const int lane = threadIdx.x % kWave, n = lane % 16, g = lane / 16;
  const auto request = [&](int row) { return sp.first + (a.pad <= kRows ? row >> a.pad_shift : row / a.pad); };
  const auto head = [&](int row) { return a.pad <= kRows ? row & (a.pad - 1) : row % a.pad; };
  {
    const int req = request(row0 + n), i = head(row0 + n);
    const uint16_t* src = a.q + ((int64_t)min(req, sp.end - 1) * a.Hq + sp.h * a.G + (i < a.G ? i : 0)) * D;
#pragma unroll
    for (int s = 0; s < D / 32; ++s) q[s] = *reinterpret_cast<const u32x4*>(src + Tile<D, FP8>::q_at(s, g));
  }
  // (what does not count is set by bits: a select would put each load behind a branch, one wait after another)
#pragma unroll
  for (int c = 0; c < 4; ++c) {
    const int r = request(row0 + 4 * g + c), i = head(row0 + 4 * g + c);
    const float x = a.lse[(int64_t)min(r, sp.end - 1) * a.Hq + sp.h * a.G + (i < a.G ? i : 0)] * kLog2e;
    const uint32_t live = i < a.G && r < sp.end ? 0xffffffffu : 0u;
    lse[c] = __uint_as_float((__float_as_uint(x) & live) | (__float_as_uint(INFINITY) & ~live));
  }
}

// exp2(unit s - lse), added to the rows' weights.
__device__ __forceinline__ void add_weights(const f32x4& s, float unit, const f32x4& lse, f32x4& sum) {
#pragma unroll
  for (int c = 0; c < 4; ++c) sum[c] += exp2_fast(fmaf(s[c], unit, -lse[c]));
}

// The sums over the `in_tile` rows of each request of a 16-row tile: in element
// c of the lanes whose row 4 (lane / 16) + c is a request's first.
__device__ __forceinline__ void sum_heads(f32x4& x, int in_tile) {
  // (selects, not branches: a branch would keep the row tiles from overlapping)
  const float two = x[2] + x[3];
  x[0] += in_tile >= 2 ? x[1] : 0.0f;
  x[2] = in_tile >= 2 ? two : x[2];
  x[0] += in_tile >= 4 ? x[2] : 0.0f;
  const auto p = __builtin_amdgcn_permlane16_swap(__float_as_uint(x[0]), __float_as_uint(x[0]), false, false);
  x[0] = in_tile >= 8 ? __uint_as_float(p[0]) + __uint_as_float(p[1]) : x[0];
  const auto q = __builtin_amdgcn_permlane32_swap(__float_as_uint(x[0]), __float_as_uint(x[0]), false, false);
  x[0] = in_tile >= 16 ? __uint_as_float(q[0]) + __uint_as_float(q[1]) : x[0];
}

// The tiles of rows from sp.row0 on, of requests of up to 16 rows; a lane has up
// to PER requests in a tile, every 4 / PER-th of its rows.
template <int D, bool FP8, int TILES, int PER>
__device__ __forceinline__ void weigh(const WeightArgs& a, const Pages& pg, const Span& sp, const int* group,
                                      char* stage) {
  using T = Tile<D, FP8>;
  const int lane = threadIdx.x % kWave, n = lane % 16, g = lane / 16;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const float unit = a.scale * kLog2e * (FP8 && a.k_scale ? a.k_scale[sp.h] : 1.0f);
  const int32_t* table = pg.table + (int64_t)sp.table_row * pg.max_blocks;
  const int64_t N = pg.capacity();
  char* mine_lds = stage + wave * StagedKeys<D, FP8>::kBytes;
  constexpr int kEach = 4 / PER;
  const int64_t next_request = (int64_t)pg.Hkv * N;
  u32x4 q[TILES][T::kK];
  f32x4 lse[TILES];
  int64_t at[TILES];    // of the lane's first request's weights, at slot 0
  int past[TILES];      // requests of the span after that one
  uint32_t mine = 0;    // bit PER t + c: the lane writes its c-th request of tile t
#pragma unroll
  for (int t = 0; t < TILES; ++t) {
    const int row0 = sp.row0 + t * kRows;
    load_rows<D, FP8>(a, sp, row0, q[t], lse[t]);
    // (kept within the span's requests, so that what it names can always be read)
    const int first = min(sp.first + ((row0 + 4 * g) >> a.pad_shift), sp.end - 1);
    at[t] = ((int64_t)first * pg.Hkv + sp.h) * N;
    past[t] = sp.end - 1 - first;
#pragma unroll
    for (int c = 0; c < PER; ++c) {
      const int row = row0 + 4 * g + c * kEach, r = sp.first + (row >> a.pad_shift);
      if ((row & (a.pad - 1)) == 0 && row < sp.row1 && r < sp.end && (sp.group < 0 || group[r] == sp.group)) mine |= 1u << (PER * t + c);
    }
  }
  // Steps are asked for kAhead before they are used: keys, and the weights so far.
  constexpr int kAhead = TILES == 1 && D != 256 ? 2 : 1;
  constexpr int kStride = kWeightWaves * kStep;
  struct Set {
    StagedKeys<D, FP8> keys;
    float before[TILES][2][PER];
    StepPages pages;
  } sets[kAhead];
  const int k_first = sp.k0 / kStep * kStep + wave * kStep;
  StepPages pages = step_pages(pg, table, k_first);  // of the next step to be asked for
  const auto counts = [&](int slot) { return slot >= sp.k0 && slot < sp.k1; };
  const auto fetch = [&](Set& s, int k) {
    s.pages = pages;
    pages = step_pages(pg, table, k + kStride);
    if (k >= sp.k1) return;
    s.keys.template load<false>(0, a.k_cache + pg.row(pg.has(s.pages.b0) ? s.pages.b0 : 0, sp.h, k) * T::kElem);
    s.keys.template load<false>(1, a.k_cache + pg.row(pg.has(s.pages.b1) ? s.pages.b1 : 0, sp.h, k + 16) * T::kElem);
    if (a.weights_in) {
      // every lane reads something of the span's rows, so that no load is behind a branch
      const int slots[2] = {k + n, min(k + 16 + n, (int)N - 1)};
#pragma unroll
      for (int t = 0; t < TILES; ++t)
#pragma unroll
        for (int c = 0; c < PER; ++c)
#pragma unroll
          for (int b = 0; b < 2; ++b) s.before[t][b][c] = a.weights_in[at[t] + min(c, past[t]) * next_request + slots[b]];
    }
  };
  const auto use = [&](Set& st, int k) {
    float sum[TILES][2][PER];
    Keys<D, FP8> keys[2];
    st.keys.put(mine_lds);
#pragma unroll
    for (int b = 0; b < 2; ++b)
#pragma unroll
      for (int i = 0; i < Keys<D, FP8>::kLoads; ++i) keys[b].raw[i] = StagedKeys<D, FP8>::get(mine_lds, b, i, n, g);
    // the set is free: the step kAhead on is asked for before this one is computed
    const bool there[2] = {pg.has(st.pages.b0), pg.has(st.pages.b1)};
    float before[TILES][2][PER];
#pragma unroll
    for (int t = 0; t < TILES; ++t)
#pragma unroll
      for (int b = 0; b < 2; ++b)
#pragma unroll
        for (int c = 0; c < PER; ++c) before[t][b][c] = st.before[t][b][c];
    fetch(st, k + kAhead * kStride);
#pragma unroll
    for (int t = 0; t < TILES; ++t) {
      f32x4 s[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
#pragma unroll
      for (int i = 0; i < T::kK; ++i) {
        s[0] = mfma16x16x32(q[t][i], keys[0].operand(i), s[0]);
        s[1] = mfma16x16x32(q[t][i], keys[1].operand(i), s[1]);
      }
#pragma unroll
      for (int b = 0; b < 2; ++b) {
        f32x4 x = {0.f, 0.f, 0.f, 0.f};
        add_weights(s[b], unit, lse[t], x);
        sum_heads(x, a.pad);
#pragma unroll
        for (int c = 0; c < PER; ++c) sum[t][b][c] = x[c * kEach];
      }
    }
    const auto put = [&](int t, int b, int c) {
      a.weights_out[at[t] + c * next_request + k + n + 16 * b] =
          (a.weights_in ? before[t][b][c] : 0.0f) + (there[b] ? sum[t][b][c] : 0.0f);
    };
    constexpr uint32_t kAll = TILES * PER < 32 ? (1u << (TILES * PER)) - 1 : ~0u;
    if (k >= sp.k0 && k + kStep <= sp.k1 && __all(mine == 0 || mine == kAll)) {
      if (mine == kAll) {
#pragma unroll
        for (int t = 0; t < TILES; ++t)
#pragma unroll
          for (int b = 0; b < 2; ++b)
#pragma unroll
            for (int c = 0; c < PER; ++c) put(t, b, c);
      }
    } else {
#pragma unroll
      for (int t = 0; t < TILES; ++t)
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
          for (int c = 0; c < PER; ++c)
            if ((mine >> (PER * t + c) & 1u) && counts(k + 16 * b + n)) put(t, b, c);
    }
  };
#pragma unroll
  for (int i = 0; i < kAhead; ++i) fetch(sets[i], k_first + i * kStride);
  for (int k = k_first; k < sp.k1; k += kAhead * kStride) {
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      if (k + i * kStride >= sp.k1) break;
      use(sets[i], k + i * kStride);
    }
  }
}

// The same for requests of more than 16 rows: tile by tile of one request, the
// queries read again for every step.
template <int D, bool FP8>
__device__ __forceinline__ void weigh_wide(const WeightArgs& a, const Pages& pg, const Span& sp, const int* group) {
  using T = Tile<D, FP8>;
  const int lane = threadIdx.x % kWave, n = lane % 16, g = lane / 16;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const float unit = a.scale * kLog2e * (FP8 && a.k_scale ? a.k_scale[sp.h] : 1.0f);
  const int32_t* table = pg.table + (int64_t)sp.table_row * pg.max_blocks;
  const int64_t N = pg.capacity();
  for (int k = sp.k0 / kStep * kStep + wave * kStep; k < sp.k1; k += kWeightWaves * kStep) {
    const StepPages pages = step_pages(pg, table, k);
    const bool there[2] = {pg.has(pages.b0), pg.has(pages.b1)};
    Keys<D, FP8> keys[2];
    keys[0].template load<false>(a.k_cache + pg.row(there[0] ? pages.b0 : 0, sp.h, k) * T::kElem, n, g);
    keys[1].template load<false>(a.k_cache + pg.row(there[1] ? pages.b1 : 0, sp.h, k + 16) * T::kElem, n, g);
    for (int row0 = sp.row0; row0 < sp.row1; row0 += a.pad) {
      const int r = sp.first + row0 / a.pad;
      if (r >= sp.end || (sp.group >= 0 && group[r] != sp.group)) continue;
      f32x4 sum[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
      for (int part = 0; part < a.pad; part += kRows) {
        u32x4 q[T::kK];
        f32x4 lse;
        load_rows<D, FP8>(a, sp, row0 + part, q, lse);
        f32x4 s[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
#pragma unroll
        for (int i = 0; i < T::kK; ++i) {
          s[0] = mfma16x16x32(q[i], keys[0].operand(i), s[0]);
          s[1] = mfma16x16x32(q[i], keys[1].operand(i), s[1]);
        }
        add_weights(s[0], unit, lse, sum[0]);
        add_weights(s[1], unit, lse, sum[1]);
      }
#pragma unroll
      for (int b = 0; b < 2; ++b) {
        sum_heads(sum[b], kRows);
        const int slot = k + n + 16 * b;
        if (g == 0 && slot >= sp.k0 && slot < sp.k1) {
          const int64_t at = ((int64_t)r * pg.Hkv + sp.h) * N + slot;
          a.weights_out[at] = (a.weights_in ? a.weights_in[at] : 0.0f) + (there[b] ? sum[b][0] : 0.0f);
        }
      }
    }
  }
}

template <int D, bool FP8>
__global__ __launch_bounds__(kWeightThreads, 2) void attn_weights_kernel(WeightArgs a, Pages pg, int member_rows) {
  extern __shared__ int lds[];
  __shared__ int waves[kWeightWaves];
  __shared__ __attribute__((aligned(16))) char stage[kWeightWaves * StagedKeys<D, FP8>::kBytes];
  const int capacity = pg.capacity();
  const Plan plan = make_plan<kWeightThreads>(a.gr, capacity, a.pad, member_rows, lds, waves);
  const int R = a.gr.R, n = a.gr.n, wgs = gridDim.x;
  const int own_row = plan.own[R], shared_row = plan.shared[n];
  // one line: the shared units, then the own ones
  const int shared_units = shared_row * pg.Hkv;
  const Deal deal(shared_units + own_row * pg.Hkv, wgs);
  const int w = blockIdx.x;
  if (w >= deal.wgs) return;
  int u = __builtin_amdgcn_readfirstlane(deal.first(w));
  const int end = __builtin_amdgcn_readfirstlane(deal.first(w + 1));
  while (u < end) {
    Span sp;
    int tiles;
    if (u < shared_units) {
      const int h = u / shared_row, v = u - h * shared_row;
      const int grp = last_at(plan.shared, n, v);
      const int first = plan.start[grp], last = plan.start[grp + 1], table_row = plan.first[grp], reach = plan.reach[table_row];
      const int per = tiles_of(0, reach), in = v - plan.shared[grp], run = in / per, t = in - run * per;
      tiles = min(per - t, end - u);
      sp = Span{table_row, first, last, grp, run * member_rows, min((run + 1) * member_rows, (last - first) * a.pad), h,
                t * kTile, min((t + tiles) * kTile, reach)};
    } else {
      const int o = u - shared_units, h = o / own_row, v = o - h * own_row;
      const int r = last_at(plan.own, R, v), t = v - plan.own[r];
      const int len = plan.len[r], lo = min(plan.reach[r], len), t0 = lo / kTile;
      tiles = min(plan.own[r + 1] - v, end - u);
      sp = Span{r, r, r + 1, -1, 0, a.pad, h, max((t0 + t) * kTile, lo), min((t0 + t + tiles) * kTile, len)};
    }
    // the same for every lane: keep it in scalar registers
    int* f = reinterpret_cast<int*>(&sp);
#pragma unroll
    for (int i = 0; i < (int)(sizeof(sp) / 4); ++i) f[i] = __builtin_amdgcn_readfirstlane(f[i]);
    if (a.pad > kRows) weigh_wide<D, FP8>(a, pg, sp, plan.group);
    else if (sp.group < 0) weigh<D, FP8, 1, 1>(a, pg, sp, plan.group, stage);
    else if (a.pad == 1) weigh<D, FP8, member_tiles(D, 1), 4>(a, pg, sp, plan.group, stage);
    else if (a.pad == 2) weigh<D, FP8, member_tiles(D, 2), 2>(a, pg, sp, plan.group, stage);
    else weigh<D, FP8, member_tiles(D, 4), 1>(a, pg, sp, plan.group, stage);
    u += __builtin_amdgcn_readfirstlane(tiles);
  }
}

template <int D, bool FP8>
int launch_weights(const WeightArgs& a, const Pages& pg, hipStream_t s) {
  const int member_rows = a.pad > kRows ? a.pad : member_tiles(D, a.pad) * kRows;
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
  if (!aligned16(q) || !aligned16(k_cache) || !aligned4(weights_in) || !aligned4(weights_out) ||
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
  a.pad_shift = __builtin_ctz((unsigned)a.pad);
  const eldr::Pages pg = pages_of(d, block_table);
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  const bool fp8 = d.kv_type == MOE_KV_FP8;
  if (d.D == 64) return fp8 ? eldr::launch_weights<64, true>(a, pg, s) : eldr::launch_weights<64, false>(a, pg, s);
  if (d.D == 128) return fp8 ? eldr::launch_weights<128, true>(a, pg, s) : eldr::launch_weights<128, false>(a, pg, s);
  return fp8 ? eldr::launch_weights<256, true>(a, pg, s) : eldr::launch_weights<256, false>(a, pg, s);
}
