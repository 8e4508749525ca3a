// moe_attn_decode: attention of one query token a request over the paged cache.
//
// One pass over the keys and values with the running maximum and sum of the
// softmax.  A wave takes 32 slots at a time for 16 query rows (the query heads
// of one kv head):
//
//   S^T = K Q^T   two 16x16 tiles of (slot, row), MFMA over D
//   P   = exp2(S^T - m), in the lanes that the products left it in
//   O^T += V^T P  MFMA over the 32 slots, P in two bf16 parts: the matrix cores
//                 have the time (all attend cases without groups within 1%)
//
// The reduction over slots may take them in any order that both operands share,
// so the second product's slot order is chosen to be the one in which a lane
// holds P already: no shuffle and no LDS between the two products.  Rows are read
// in whole lines, a value tile transposed inside the lane (its rows' 16-bit halves
// are zipped by v_perm), a key tile handed over through LDS.  What bounds it is
// HBM; the loads are non-temporal, so that they do not displace what the caches
// hold (203 -> 178 us in the first case below).  Measured: 128 requests of up to
// 8000 tokens (32 heads over 4 of 128, bf16, 1.1 GB) 178 to 181 us, 6.1 to 6.2 TB/s of
// a streaming read's 7.05; 64 of 16384 in fp8 (1.1 GB) 167; D = 64 331 us and D = 256
// 355 us for 2.1 GB.  Short segments are further off: 256 of up to 1500 in fp8 at D = 64
// 48 us (208 MB, 61% of the read's rate).  Dealing the units to waves in place of workgroups (no merge
// in LDS, four times the parts) measured 2 to 8% slower.
//
// Pages of 8-bit integers: codes become bf16 exactly (a conversion each, its upper
// half kept), a page's key scale multiplies the tile's scores where scale and units
// already do, its value scale the tile's weights before they are split, so neither
// costs a product over D.  A lane loads one of a step's four scales.  Measured: 128 of up
// to 8000 (552 MB) 98 us, 64 of 16384 (1.1 GB) 168, 2 near 131,000 (268 MB) 46, within 1
// to 4% of fp8 at every shape tried.  No gain came of more workgroups (768: 103.5 -> 106
// us in the first case, 1024: 109), of a wave's next step asked for before this one is
// worked on (237 registers; within 1%) and of the next segment's first step asked for
// before the merge (within 2%, both ways): what is left is start and plan (5 us of every
// call), the join and the ends of segments (128 of 4096, one to a workgroup, run at 6.2
// TB/s; of 17 to 8000 at 5.6).
//
// The four waves of a workgroup take turns at a segment's 32-slot steps and
// meet in LDS at its end.  A segment that is a request's whole context gives
// the output; the others leave sums that attn_join adds up.
#pragma once

#include <algorithm>

#include "attn_plan.hpp"
#include "attn_shared.hpp"
#include "attn_tile.hpp"

namespace eldr {

constexpr int kDecodeThreads = 256;
constexpr int kDecodeWaves = kDecodeThreads / kWave;

// Workgroups that share the own line.  More of them hide the ends of short
// segments, fewer make longer segments and fewer parts.  Measured (us, whole calls;
// 512, 768, 1024):
//   D = 64   256 of up to 1500 in fp8 67, 60, 57; in bf16 83, 87, 86
//            128 of up to 8000 in fp8 113, 107, 110; in bf16 184, 189, 187
//            64 of up to 700 21, 19, 19; 2 of 131,000 91, 94, 94
//            256 of up to 1500 behind 8 x 2048 in fp8 105, 98, 94
//   D = 128  128 of up to 8000 184, 186, 188; 256 of up to 1500 in fp8 86, 88, 87
//            64 of up to 700 19, 18, 20
//   D = 256  64 of up to 4000 63, 67, 71
// So 1024 where rows are short: 10 to 17% for fp8 and for short contexts, against 2 to
// 4% for long ones in bf16.
constexpr int decode_wgs(int D) { return D == 64 ? 1024 : 512; }

struct DecodeArgs {
  const uint16_t* q;
  const char *k_cache, *v_cache;
  Groups gr;
  const float *k_scale, *v_scale, *sinks;
  uint16_t* out;
  float* lse;
  float scale;
  int32_t Hq, G, head_tiles;  // head_tiles: ceil(G / kRows)
};

// The workspace: parts of rows, D sums then (maximum, sum) at a pitch of D + 4.
// own, shared: by row of the requests' query heads, the part that begins a
// request's own slots or its group's.  own_rest, shared_rest: by workgroup, the
// part that continues one (the first stretch of a workgroup at most).  Then the
// plan, for attn_join.
struct Parts {
  float *own, *shared, *own_rest, *shared_rest;
  int* plan;
  __host__ __device__ Parts(float* ws, int64_t rows, int D, int shared_rows) {
    own = ws;
    shared = own + rows * (D + 4);
    own_rest = shared + rows * (D + 4);
    shared_rest = own_rest + (int64_t)decode_wgs(D) * kRows * (D + 4);
    plan = reinterpret_cast<int*>(shared_rest + (int64_t)kSharedWgs * shared_rows * (D + 4));
  }
};

// A run of slots [k0, k1) of a request against a tile of its heads: rows
// [row0, row0 + kRows) of the G heads of kv head h.
struct Segment {
  int request, row0, h, k0, k1;
};

// The running state of 16 rows: maximum and sum (this lane's part) of row
// lane % 16, and O^T: acc[c][i] is value column (4 (lane / 16) + i) kV + c.
template <int D, int KV>
__device__ __forceinline__ void attend(const DecodeArgs& a, const Pages& pg, const Segment& sg, char* stage, float& m, float& l,
                                       f32x4 (&acc)[D / 16]) {
  using T = Tile<D, KV>;
  const int lane = threadIdx.x % kWave, n = lane % 16, g = lane / 16;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  m = -INFINITY;
  l = 0.0f;
#pragma unroll
  for (int c = 0; c < T::kV; ++c) acc[c] = f32x4{0.f, 0.f, 0.f, 0.f};
  u32x4 q[T::kK];
  {
    const int row = sg.row0 + n;
    const bool live = row < a.G;
    const uint16_t* src = a.q + ((int64_t)sg.request * a.Hq + sg.h * a.G + (live ? row : 0)) * D;
#pragma unroll
    for (int s = 0; s < T::kK; ++s) {
      const u32x4 x = *reinterpret_cast<const u32x4*>(src + T::q_at(s, g));
      q[s] = keep_if(live, x);
    }
  }
  const float unit = a.scale * kLog2e * (KV == kKvFp8 && a.k_scale ? a.k_scale[sg.h] : 1.0f);
  // (pages of 8-bit integers) the lane's share of a step's four scales: the keys' or
  // the values' (lanes from 32 on), of the first or the second tile
  const float* scales = KV == kKvInt8 ? (g < 2 ? a.k_scale : a.v_scale) + sg.h : nullptr;
  const int32_t* table = pg.table + (int64_t)sg.request * pg.max_blocks;
  const int k_first = sg.k0 / kStep * kStep + wave * kStep;
  // a step's pages are looked up one step ahead
  StepPages pages = step_pages(pg, table, k_first);
  for (int k = k_first; k < sg.k1; k += kDecodeWaves * kStep) {
    const int b0 = pages.b0, b1 = pages.b1;
    pages = step_pages(pg, table, k + kDecodeWaves * kStep);
    const bool has0 = pg.has(b0), has1 = pg.has(b1);
    const bool whole = has0 && has1 && k >= sg.k0 && k + kStep <= sg.k1;
    const int64_t r0 = pg.row(has0 ? b0 : 0, sg.h, k) * T::kElem, r1 = pg.row(has1 ? b1 : 0, sg.h, k + 16) * T::kElem;
    StagedKeys<D, KV> staged;
    Keys<D, KV> keys[2];
    Values<D, KV> v;
    // (D = 256 in bf16 has no registers left for the way through LDS)
    constexpr bool kStaged = D != 256 || T::kByte;
    float page_scale = 0.0f;
    if constexpr (KV == kKvInt8) page_scale = scales[(int64_t)(g % 2 ? (has1 ? b1 : 0) : (has0 ? b0 : 0)) * pg.Hkv];
    if constexpr (kStaged) {
      staged.template load<true>(0, a.k_cache + r0);
      staged.template load<true>(1, a.k_cache + r1);
    } else {
      keys[0].template load<true>(a.k_cache + r0, n, g);
      keys[1].template load<true>(a.k_cache + r1, n, g);
    }
    v.load(a.v_cache + r0, a.v_cache + r1, n, g);
    __builtin_amdgcn_sched_barrier(0);
    if constexpr (kStaged) staged.put(stage);
    f32x4 s[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
    constexpr int kLoads = Keys<D, KV>::kLoads, kEach = T::kK / kLoads;
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
#pragma unroll
      for (int b = 0; b < 2; ++b)
        if constexpr (kStaged) keys[b].raw[i] = StagedKeys<D, KV>::get(stage, b, i, n, g);
#pragma unroll
      for (int e = i * kEach; e < (i + 1) * kEach; ++e) {
        s[0] = mfma16x16x32(keys[0].operand(e), q[e], s[0]);
        s[1] = mfma16x16x32(keys[1].operand(e), q[e], s[1]);
      }
    }
    const auto keep = [&](int j) {
      const int at = k + (j / 4) * 16 + 4 * g + j % 4;
      return (j < 4 ? has0 : has1) && at >= sg.k0 && at < sg.k1;
    };
    if (!whole) {
#pragma unroll
      for (int j = 0; j < 8; ++j) v.drop(j, keep(j));
    }
    StepUnits<KV == kKvInt8> units;
    if constexpr (KV == kKvInt8) {
      const auto scale_of = [&](int quarter) { return __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(page_scale), quarter * 16)); };
      // a tile without a slot that counts has no scale that counts
      const bool any0 = has0 && k + 16 > sg.k0 && k < sg.k1, any1 = has1 && k + 32 > sg.k0 && k + 16 < sg.k1;
      units.score[0] = unit * scale_of(0), units.score[1] = unit * scale_of(1);
      units.value[0] = any0 ? scale_of(2) : 0.0f, units.value[1] = any1 ? scale_of(3) : 0.0f;
    } else {
      units.score = unit;
    }
    const Weights p = softmax_step(s, units, whole, keep, m, l, [&](float f) {
#pragma unroll
      for (int c = 0; c < T::kV; ++c) acc[c] *= f;
    });
#pragma unroll
    for (int c = 0; c < T::kV; ++c) {
      const u32x4 x = v.operand(c);
      acc[c] = mfma16x16x32(x, p.most, acc[c]);
      acc[c] = mfma16x16x32(x, p.rest, acc[c]);
    }
  }
  // the row's sum over the four lanes that share it
  l += __shfl_xor(l, 16);
  l += __shfl_xor(l, 32);
}

// A row's end: what gives the output from its sums of values, and its lse.
struct RowEnd {
  float by, lse;
};

// From a row's maximum (in base-2 units) and sum; sink: the row's, or null; unit:
// the values' scale.  The sink is weighed in its own units, where the difference
// that counts can be taken of any finite value: the lowest one, in base 2, would be
// -inf already.  Where it and the maximum are both -inf there is nothing to weigh:
// the reference stays finite, so that the sums stay zero.  A row is empty where its
// sum is 0, and only there: a sum that is NaN gives NaN.
__device__ __forceinline__ RowEnd end_row(float top, float total, const float* sink, float unit) {
  constexpr float kLn2 = 0.6931471805599453f;
  const float own = top * kLn2;
  const bool empty = total == 0.0f;
  float with = own, f = 1.0f;
  if (sink) {
    with = fmaxf(own, *sink);
    const float base = with == -INFINITY ? 0.0f : with;
    f = exp2_fast((own - base) * kLog2e);
    total = total * f + exp2_fast((*sink - base) * kLog2e);
  }
  const float log2_total = __builtin_amdgcn_logf(total);  // -inf where there is neither a slot nor a sink
  return RowEnd{empty ? 0.0f : f * unit / total, sink ? with + log2_total * kLn2 : (top + log2_total) * kLn2};
}

// Adds the four waves' states in LDS; then writes the rows' sums as a part, or
// as the output.  lds: kDecodeWaves * kRows * (D + 4) floats.
template <int D, int KV>
__device__ __forceinline__ void merge(const DecodeArgs& a, const Segment& sg, float m, float l, const f32x4 (&acc)[D / 16],
                                      float* lds, bool whole, float* part, bool by_row) {
  constexpr int kPitch = D + 4;  // the row's sums, then its maximum and sum
  constexpr int kV = D / 16;
  const int lane = threadIdx.x % kWave, n = lane % 16, g = lane / 16, wave = threadIdx.x / kWave;
  float* mine = lds + (wave * kRows + n) * kPitch;
  wave_handover();  // the wave's last keys lay here
  if (g == 0) mine[D] = m, mine[D + 1] = l;
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int c = 0; c < kV; c += 4)
      *reinterpret_cast<f32x4*>(mine + (4 * g + i) * kV + c) = f32x4{acc[c][i], acc[c + 1][i], acc[c + 2][i], acc[c + 3][i]};
  __syncthreads();
  constexpr int kQuads = D / 4;
  for (int e = threadIdx.x; e < kRows * kQuads; e += kDecodeThreads) {
    const int row = e / kQuads, at = (e % kQuads) * 4;
    if (sg.row0 + row >= a.G) break;
    float mm[kDecodeWaves], top = -INFINITY, sum = 0.0f;
    f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < kDecodeWaves; ++w) {
      mm[w] = lds[(w * kRows + row) * kPitch + D];
      top = fmaxf(top, mm[w]);
    }
    const float base = top == -INFINITY ? 0.0f : top;
#pragma unroll
    for (int w = 0; w < kDecodeWaves; ++w) {
      const float* from = lds + (w * kRows + row) * kPitch;
      const float f = exp2_fast(mm[w] - base);
      sum += f * from[D + 1];
      o += f * *reinterpret_cast<const f32x4*>(from + at);
    }
    const int head = sg.h * a.G + sg.row0 + row;
    const int64_t q_row = (int64_t)sg.request * a.Hq + head;
    if (whole) {
      const RowEnd end = end_row(top, sum, a.sinks ? a.sinks + head : nullptr, KV == kKvFp8 && a.v_scale ? a.v_scale[sg.h] : 1.0f);
      o *= end.by;
      *reinterpret_cast<u32x2*>(a.out + q_row * D + at) = u32x2{pack_bf16(o[0], o[1]), pack_bf16(o[2], o[3])};
      if (at == 0 && a.lse) a.lse[q_row] = end.lse;
    } else {
      float* to = part + (by_row ? q_row : (int64_t)row) * (D + 4);
      *reinterpret_cast<f32x4*>(to + at) = o;
      if (at == 0) *reinterpret_cast<f32x4*>(to + D) = f32x4{top, sum, 0.0f, 0.0f};
    }
  }
  __syncthreads();
}

template <int D, int KV>
__global__ __launch_bounds__(kDecodeThreads, D == 256 ? 2 : 3) void attn_decode_kernel(DecodeArgs a, Pages pg, Parts parts) {
  extern __shared__ int lds[];
  __shared__ int waves[kDecodeWaves];
  float* sums_lds = reinterpret_cast<float*>(lds);
  // a wave's keys pass through its own part of where it will leave its sums
  constexpr int kWaveSums = kRows * (D + 4) * 4;
  static_assert(StagedKeys<D, KV>::kBytes <= kWaveSums, "a step's keys fit a wave's sums");
  char* stage = reinterpret_cast<char*>(lds) + threadIdx.x / kWave * kWaveSums;
  int* plan_lds = lds + kDecodeWaves * kRows * (D + 4);
  const Plan plan = make_plan<kDecodeThreads>(a.gr, pg.capacity(), a.G, SharedTile<D>::kRowsWg, plan_lds, waves);
  const int R = a.gr.R, n = a.gr.n, row = plan.own[R];
  if (blockIdx.x == 0)
    for (int i = threadIdx.x; i < Plan::kept(R, n); i += kDecodeThreads) parts.plan[i] = plan.own[i];
  const Deal deal(row * pg.Hkv * a.head_tiles, decode_wgs(D));
  if ((int)blockIdx.x >= deal.wgs) return;
  int u = __builtin_amdgcn_readfirstlane(deal.first(blockIdx.x));
  const int end = __builtin_amdgcn_readfirstlane(deal.first(blockIdx.x + 1));
  float m, l;
  f32x4 acc[D / 16];
  while (u < end) {
    const int hv = u / row, v = u - hv * row;
    const int r = last_at(plan.own, R, v), t = v - plan.own[r];
    const int len = plan.len[r], reach = plan.reach[r];
    const int lo = own_from(len, reach, a.gr.window), t0 = lo / kTile;
    const int tiles = __builtin_amdgcn_readfirstlane(min(plan.own[r + 1] - v, end - u));
    const bool begins = t == 0, whole = begins && v + tiles == plan.own[r + 1] && reach == 0;
    Segment sg{r, hv % a.head_tiles * kRows, hv / a.head_tiles, max((t0 + t) * kTile, lo), min((t0 + t + tiles) * kTile, len)};
    // the same for every lane: keep it in scalar registers
    int* f = reinterpret_cast<int*>(&sg);
#pragma unroll
    for (int i = 0; i < (int)(sizeof(sg) / 4); ++i) f[i] = __builtin_amdgcn_readfirstlane(f[i]);
    attend<D, KV>(a, pg, sg, stage, m, l, acc);
    merge<D, KV>(a, sg, m, l, acc, sums_lds, whole,
                  begins ? parts.own : parts.own_rest + (int64_t)blockIdx.x * kRows * (D + 4), begins);
    u += tiles;
  }
}

// The parts of a row (a request's query head): `shared` ones of its group's prefix,
// then its own; the first of each by row, the others by the workgroups after w0.
struct RowParts {
  const float *shared, *shared_rest, *own, *own_rest;  // (own_rest, shared_rest: of the row's place in a tile)
  int shared_parts, own_parts, shared_w0, own_w0;
  int hq, h;  // the row's query head and kv head
  bool many;  // Lines::many of its request
};

// The two lines as they were dealt.
template <int D>
struct Lines {
  Deal own, shared;
  __device__ __forceinline__ Lines(const DecodeArgs& a, const Pages& pg, const int* plan)
      : own(plan[a.gr.R] * pg.Hkv * a.head_tiles, decode_wgs(D)),
        shared(plan[3 * a.gr.R + 1 + a.gr.n] * pg.Hkv, kSharedWgs) {}
  // Whether a request's rows are in more than some 8 parts, of so many units.
  __device__ __forceinline__ bool many(int own_units, int shared_units) const {
    constexpr int kFew = 8;
    return own_units > kFew * own.each || shared_units > kFew * shared.each;
  }
};

template <int D>
__device__ __forceinline__ RowParts parts_of(const DecodeArgs& a, const Pages& pg, const Parts& parts, int q_row) {
  constexpr int kPitch = D + 4, kTileRows = SharedTile<D>::kRowsWg;
  const int R = a.gr.R, n = a.gr.n;
  const int* own = parts.plan;
  const int *reach = own + R + 1, *group = reach + R, *shared = group + R;
  const int r = q_row / a.Hq, hq = q_row - r * a.Hq, h = hq / a.G, i = hq - h * a.G;
  const int own_row = own[R], tiles = own[r + 1] - own[r], mine = reach[r];
  const Lines<D> lines(a, pg, parts.plan);
  RowParts p{parts.shared + (int64_t)q_row * kPitch, parts.shared_rest, parts.own + (int64_t)q_row * kPitch,
             parts.own_rest + (int64_t)(i % kRows) * kPitch, 0, 0, 0, 0, hq, h, lines.many(tiles, tiles_of(0, mine))};
  if (mine > 0) {
    const int g = group[r];
    const int row = (r - max(a.gr.start[g], 0)) * a.G + i, per = tiles_of(0, mine);
    const int u0 = h * shared[n] + shared[g] + row / kTileRows * per;
    p.shared_w0 = lines.shared.owner(u0);
    p.shared_parts = lines.shared.owner(u0 + per - 1) - p.shared_w0 + 1;
    p.shared_rest += (int64_t)(row % kTileRows) * kPitch;
  }
  if (tiles > 0) {
    const int u0 = (h * a.head_tiles + i / kRows) * own_row + own[r];
    p.own_w0 = lines.own.owner(u0);
    p.own_parts = lines.own.owner(u0 + tiles - 1) - p.own_w0 + 1;
  }
  return p;
}

template <int D>
__device__ __forceinline__ const float* part_at(const RowParts& r, int p) {
  constexpr int kPitch = D + 4;
  if (p < r.shared_parts) return p == 0 ? r.shared : r.shared_rest + (int64_t)(r.shared_w0 + p) * SharedTile<D>::kRowsWg * kPitch;
  p -= r.shared_parts;
  return p == 0 ? r.own : r.own_rest + (int64_t)(r.own_w0 + p) * kRows * kPitch;
}

// A row's sums so far, of four of its values: maximum, sum of weights, values.  (fmaf,
// so that every kernel that adds parts up rounds alike.)
struct RowSums {
  float top = -INFINITY, total = 0.0f;
  f32x4 sum = {0.f, 0.f, 0.f, 0.f};
  __device__ __forceinline__ void add(float m, float l, const f32x4& v) {
    const float m2 = fmaxf(top, m), base = m2 == -INFINITY ? 0.0f : m2;
    const float f = exp2_fast(top - base), e = exp2_fast(m - base);
    total = fmaf(total, f, l * e);
#pragma unroll
    for (int i = 0; i < 4; ++i) sum[i] = fmaf(sum[i], f, v[i] * e);
    top = m2;
  }
};

template <int D, int KV>
__device__ __forceinline__ void write_row(const DecodeArgs& a, int q_row, int hq, int h, int at, const RowSums& x) {
  const RowEnd end = end_row(x.top, x.total, a.sinks ? a.sinks + hq : nullptr, KV == kKvFp8 && a.v_scale ? a.v_scale[h] : 1.0f);
  const f32x4 o = x.sum * end.by;
  *reinterpret_cast<u32x2*>(a.out + (int64_t)q_row * D + 4 * at) = u32x2{pack_bf16(o[0], o[1]), pack_bf16(o[2], o[3])};
  if (at == 0 && a.lse) a.lse[q_row] = end.lse;
}

// LDS where the sets of threads that share a row meet.
template <int D, int THREADS>
struct JoinLds {
  static constexpr int kSet = D / 4, kSets = THREADS / kSet, kRowsWg = kDecodeThreads / THREADS;
  f32x4 sums[kRowsWg][kSets][kSet];
  float tops[kRowsWg][kSets], totals[kRowsWg][kSets];
};

// Adds up the parts of a row that has several, and writes a row that has none: THREADS
// threads (256, or 64) take it (none where !real), sets of D / 4 of them its parts in
// turn, four values each, and the sets meet in LDS.
template <int D, int KV, int THREADS>
__device__ __forceinline__ void join_row(const DecodeArgs& a, const Pages& pg, const Parts& parts, JoinLds<D, THREADS>& lds, int q_row,
                                         bool real) {
  constexpr int kSet = D / 4, kSets = THREADS / kSet;
  const int mine_row = __builtin_amdgcn_readfirstlane(threadIdx.x / THREADS);
  auto& sums = lds.sums[mine_row];
  auto &tops = lds.tops[mine_row], &totals = lds.totals[mine_row];
  const RowParts r = parts_of<D>(a, pg, parts, q_row);
  const bool written = !real || (r.own_parts == 1 && r.shared_parts == 0);  // by attn_decode
  const int set = threadIdx.x % THREADS / kSet, at = threadIdx.x % kSet;
  const int count = written ? 0 : r.shared_parts + r.own_parts;
  constexpr int kBatch = 4;  // parts that a set has in flight
  RowSums x;
  for (int p0 = set; p0 < count; p0 += kBatch * kSets) {
    f32x4 v[kBatch], ml[kBatch];
#pragma unroll
    for (int b = 0; b < kBatch; ++b) {
      const float* from = part_at<D>(r, min(p0 + b * kSets, count - 1));
      v[b] = *reinterpret_cast<const f32x4*>(from + 4 * at);
      ml[b] = *reinterpret_cast<const f32x4*>(from + D);
    }
    // (selects: a branch a part costs 2 us of 16 where rows have 250)
#pragma unroll
    for (int b = 0; b < kBatch; ++b) {
      const bool there = p0 + b * kSets < count;
      const f32x4 none = {0.f, 0.f, 0.f, 0.f};
      x.add(there ? ml[b][0] : -INFINITY, ml[b][1], there ? v[b] : none);
    }
  }
  sums[set][at] = x.sum;
  if (at == 0) tops[set] = x.top, totals[set] = x.total;
  if constexpr (THREADS == kWave) wave_handover();
  else __syncthreads();
  if (written || set != 0) return;
#pragma unroll
  for (int s = 1; s < kSets; ++s) x.add(tops[s], totals[s], sums[s][at]);
  write_row<D, KV>(a, q_row, r.hq, r.h, at, x);
}

// For few rows, each of them in many parts.
template <int D, int KV, int THREADS>
__global__ __launch_bounds__(kDecodeThreads) void attn_join_kernel(DecodeArgs a, Pages pg, Parts parts, int rows) {
  __shared__ JoinLds<D, THREADS> lds;
  const int q_row = blockIdx.x * (kDecodeThreads / THREADS) + __builtin_amdgcn_readfirstlane(threadIdx.x / THREADS);
  const bool real = q_row < rows;
  join_row<D, KV, THREADS>(a, pg, parts, lds, real ? q_row : 0, real);
}

// The same for many rows: D / 4 threads take a row of a few parts.  What finds
// a row's parts (eight divisions) is then a wave's work for up to four rows, where a
// wave a row spent most of its time (16,384 rows of 64: 15.5 -> 7.6 us).  The parts are
// added as kWave / kSet sets would, so that a row's bits are the same either way.
//
// Where D / 4 threads are a quarter of a wave, a row of many parts has few of them in
// flight here.  Such rows are a wave's work each, in further workgroups, which look at
// every request.  Measured (us, whole calls, 64 heads of 64 in bf16; 64 threads every row,
// D / 4 every row, this): over 1 kv head one request of 131,000 slots beside 31 of 100 51.6,
// 74.6, 52.5, over 8 70.8, 81.2, 70.9, beside 255 78.3, 86.8, 80.0; 256 of up to 1500 81.6,
// 76.2, 76.7, behind 8 x 2048 101, 93, 94, 128 of up to 1000 34.3, 31.5, 31.5.
constexpr int kApartWgs = 1024;
template <int D, int KV>
__global__ __launch_bounds__(kDecodeThreads) void attn_join_rows_kernel(DecodeArgs a, Pages pg, Parts parts, int rows) {
  constexpr int kSet = D / 4, kSets = kWave / kSet, kRowsWg = kDecodeThreads / kSet;
  constexpr bool kApart = kSets > 2;
  if constexpr (kApart) {
    const int wgs = (rows + kRowsWg - 1) / kRowsWg;
    if ((int)blockIdx.x >= wgs) {
      __shared__ JoinLds<D, kWave> lds;
      const Lines<D> lines(a, pg, parts.plan);
      const int *own = parts.plan, *reach = own + a.gr.R + 1;
      const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
      for (int row = ((int)blockIdx.x - wgs) * kDecodeWaves + wave; row < rows; row += kApartWgs * kDecodeWaves) {
        const int r = row / a.Hq;
        if (!lines.many(own[r + 1] - own[r], tiles_of(0, reach[r]))) continue;
        join_row<D, KV, kWave>(a, pg, parts, lds, row, true);
        wave_handover();  // (before the next row's sums)
      }
      return;
    }
  }
  const int q_row = blockIdx.x * kRowsWg + threadIdx.x / kSet, at = threadIdx.x % kSet;
  if (q_row >= rows) return;
  const RowParts r = parts_of<D>(a, pg, parts, q_row);
  if (kApart && r.many) return;
  if (r.own_parts == 1 && r.shared_parts == 0) return;  // written by attn_decode
  const int count = r.shared_parts + r.own_parts;
  // parts in flight (where D is 64, registers for six waves a SIMD in place of four: 16,384
  // rows 8.2 -> 7.6 us)
  constexpr int kBatch = kApart ? 4 : 8;
  RowSums x[kSets];
  for (int p0 = 0; p0 < count; p0 += kBatch) {
    f32x4 v[kBatch];
    f32x2 ml[kBatch];
#pragma unroll
    for (int b = 0; b < kBatch; ++b) {
      if (p0 + b >= count) break;
      const float* from = part_at<D>(r, p0 + b);
      v[b] = *reinterpret_cast<const f32x4*>(from + 4 * at);
      ml[b] = *reinterpret_cast<const f32x2*>(from + D);
    }
#pragma unroll
    for (int b = 0; b < kBatch; ++b)
      if (p0 + b < count) x[b % kSets].add(ml[b][0], ml[b][1], v[b]);
  }
#pragma unroll
  for (int s = 1; s < kSets; ++s) x[0].add(x[s].top, x[s].total, x[s].sum);
  write_row<D, KV>(a, q_row, r.hq, r.h, at, x[0]);
}

// Raises a kernel's dynamic LDS limit where a launch needs more than the default.
inline bool lds_allowed(const void* kernel, size_t bytes) {
  if (bytes <= 60 * 1024) return true;
  if (hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, (int)bytes) == hipSuccess) return true;
  (void)hipGetLastError();
  return false;
}

template <int D, int KV>
int launch_decode(const DecodeArgs& a, const Pages& pg, float* ws, hipStream_t s) {
  using S = SharedTile<D>;
  const int64_t rows = (int64_t)a.gr.R * a.Hq;
  const Parts parts(ws, rows, D, S::kRowsWg);
  const size_t plan = Plan::bytes(a.gr.R, a.gr.n);
  const size_t lds = (size_t)kDecodeWaves * kRows * (D + 4) * 4 + plan;
  if (!lds_allowed(reinterpret_cast<const void*>(attn_decode_kernel<D, KV>), lds)) return MOE_ERR_HIP;
  if (a.gr.n > 0) {
    const SharedArgs sh{a.q, a.k_cache, a.v_cache, a.gr, a.k_scale, a.v_scale, parts.shared, parts.shared_rest, a.scale, a.Hq, a.G};
    if (!lds_allowed(reinterpret_cast<const void*>(attn_shared_kernel<D, KV>), S::kBytes + scale_bytes(KV) + plan)) return MOE_ERR_HIP;
    hipLaunchKernelGGL((attn_shared_kernel<D, KV>), dim3(kSharedWgs), dim3(kSharedThreads), S::kBytes + scale_bytes(KV) + plan, s, sh, pg);
  }
  hipLaunchKernelGGL((attn_decode_kernel<D, KV>), dim3(decode_wgs(D)), dim3(kDecodeThreads), lds, s, a, pg, parts);
  // Measured (us, whole calls; 256 threads a row, 64): 64 rows of 131,000 slots 51, 59;
  // 512 of 16,384 73, 74, and behind 8192 37, 43; 1024 of up to 8000 70, 69, and behind
  // 8192 40, 42; 2048 of up to 8000 138, 136; 8192 behind 2048 73, 54; 16,384 of up to
  // 1500 92, 71.  D / 4 threads a row (few parts) against 64, in
  // fp8: D = 64, 16,384 rows behind 8 x 2048 75.2, 81.2, of up to 1500 47.0, 51.2, 4096 of
  // up to 700 15.1, 16.3, behind 8192 48.8, 49.2; D = 128, 8192 of up to 1500 44.1, 46.1,
  // behind 8 x 2048 71.5, 71.5, 5120 of which 32 of 131,000 72.2, 71.2, 4096 of up to 8000
  // (8-bit integers) 101.5, 102.2, behind 4 x 2048 52.1, 49.7, 2048 behind 8192 (bf16) 48.2,
  // 49.0; D = 256 the same.
  constexpr int64_t kFewRows = 1024, kManyRows = D == 64 ? kFewRows : 4096;
  const auto wgs = [&](int rows_wg) { return (unsigned)((rows + rows_wg - 1) / rows_wg); };
  const auto join = [&](auto kernel, unsigned wgs) {
    hipLaunchKernelGGL(kernel, dim3(wgs), dim3(kDecodeThreads), 0, s, a, pg, parts, (int)rows);
  };
  if (rows <= kFewRows) {
    join(attn_join_kernel<D, KV, 256>, wgs(1));
  } else if (rows > kManyRows) {
    join(attn_join_rows_kernel<D, KV>, wgs(kDecodeThreads / (D / 4)) + (D == 64 ? std::min(wgs(kDecodeWaves), (unsigned)kApartWgs) : 0));
  } else {
    if constexpr (kManyRows > kFewRows) join(attn_join_kernel<D, KV, 64>, wgs(kDecodeThreads / 64));
  }
  return eldr_host::launch_status();
}

// launch_decode<D, kKvInt8>, D as a number.
int launch_decode_int8(int D, const DecodeArgs& a, const Pages& pg, float* ws, hipStream_t s);

}  // namespace eldr
