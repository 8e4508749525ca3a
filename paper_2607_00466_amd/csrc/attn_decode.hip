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
// The four waves of a workgroup take turns at a segment's 32-slot steps and
// meet in LDS at its end.  A segment that is a request's whole context gives
// the output; the others leave sums that attn_join adds up.
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
template <int D, bool FP8>
__device__ __forceinline__ void attend(const DecodeArgs& a, const Pages& pg, const Segment& sg, char* stage, float& m, float& l,
                                       f32x4 (&acc)[D / 16]) {
  using T = Tile<D, FP8>;
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
  const float unit = a.scale * kLog2e * (FP8 && a.k_scale ? a.k_scale[sg.h] : 1.0f);
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
    StagedKeys<D, FP8> staged;
    Keys<D, FP8> keys[2];
    Values<D, FP8> v;
    // (D = 256 in bf16 has no registers left for the way through LDS)
    constexpr bool kStaged = D != 256 || FP8;
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
    constexpr int kLoads = Keys<D, FP8>::kLoads, kEach = T::kK / kLoads;
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
#pragma unroll
      for (int b = 0; b < 2; ++b)
        if constexpr (kStaged) keys[b].raw[i] = StagedKeys<D, FP8>::get(stage, b, i, n, g);
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
    const Weights p = softmax_step(s, unit, whole, keep, m, l, [&](float f) {
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
template <int D, bool FP8>
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
      const RowEnd end = end_row(top, sum, a.sinks ? a.sinks + head : nullptr, FP8 && a.v_scale ? a.v_scale[sg.h] : 1.0f);
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

template <int D, bool FP8>
__global__ __launch_bounds__(kDecodeThreads, D == 256 ? 2 : 3) void attn_decode_kernel(DecodeArgs a, Pages pg, Parts parts) {
  extern __shared__ int lds[];
  __shared__ int waves[kDecodeWaves];
  float* sums_lds = reinterpret_cast<float*>(lds);
  // a wave's keys pass through its own part of where it will leave its sums
  constexpr int kWaveSums = kRows * (D + 4) * 4;
  static_assert(StagedKeys<D, FP8>::kBytes <= kWaveSums, "a step's keys fit a wave's sums");
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
    attend<D, FP8>(a, pg, sg, stage, m, l, acc);
    merge<D, FP8>(a, sg, m, l, acc, sums_lds, whole,
                  begins ? parts.own : parts.own_rest + (int64_t)blockIdx.x * kRows * (D + 4), begins);
    u += tiles;
  }
}

// Adds up the parts of a row that has several, and writes a row that has none.
// THREADS threads (64, or 256 where there are few rows, each of them in many
// parts) take a (request, query head): sets of D / 4 of them take a part, four
// values each, and take the parts in turn, with a running maximum; the sets meet
// in LDS.
template <int D, bool FP8, int THREADS>
__global__ __launch_bounds__(kDecodeThreads) void attn_join_kernel(DecodeArgs a, Pages pg, Parts parts, int rows) {
  constexpr int kSet = D / 4, kSets = THREADS / kSet, kRowsWg = kDecodeThreads / THREADS;
  constexpr int kPitch = D + 4;
  __shared__ f32x4 sums_of[kRowsWg][kSets][kSet];
  __shared__ float tops_of[kRowsWg][kSets], totals_of[kRowsWg][kSets];
  const int mine_row = __builtin_amdgcn_readfirstlane(threadIdx.x / THREADS);
  const bool real = (int)blockIdx.x * kRowsWg + mine_row < rows;
  const int q_row = real ? blockIdx.x * kRowsWg + mine_row : 0;
  auto& sums = sums_of[mine_row];
  auto &tops = tops_of[mine_row], &totals = totals_of[mine_row];
  const int R = a.gr.R, n = a.gr.n;
  const int* own = parts.plan;
  const int *reach = own + R + 1, *group = reach + R, *shared = group + R;
  const int r = q_row / a.Hq, hq = q_row - r * a.Hq, h = hq / a.G, i = hq - h * a.G;
  const int own_row = own[R], tiles = own[r + 1] - own[r], mine = reach[r];
  // the row's parts: the first by row, the others by the workgroups after w0
  int shared_parts = 0, shared_w0 = 0, shared_at = 0, own_parts = 0, own_w0 = 0;
  constexpr int kTileRows = SharedTile<D>::kRowsWg;
  if (mine > 0) {
    const int g = group[r];
    const int row = (r - max(a.gr.start[g], 0)) * a.G + i, per = tiles_of(0, mine);
    const int u0 = h * shared[n] + shared[g] + row / kTileRows * per;
    const Deal deal(shared[n] * pg.Hkv, kSharedWgs);
    shared_w0 = deal.owner(u0);
    shared_parts = deal.owner(u0 + per - 1) - shared_w0 + 1;
    shared_at = row % kTileRows;
  }
  if (tiles > 0) {
    const Deal deal(own_row * pg.Hkv * a.head_tiles, decode_wgs(D));
    const int u0 = (h * a.head_tiles + i / kRows) * own_row + own[r];
    own_w0 = deal.owner(u0);
    own_parts = deal.owner(u0 + tiles - 1) - own_w0 + 1;
  }
  const bool written = !real || (own_parts == 1 && shared_parts == 0);  // by attn_decode
  const int set = threadIdx.x % THREADS / kSet, at = threadIdx.x % kSet;
  const int64_t first = (int64_t)q_row * kPitch;
  const auto part = [&](int p) -> const float* {
    if (p < shared_parts)
      return p == 0 ? parts.shared + first : parts.shared_rest + ((int64_t)(shared_w0 + p) * kTileRows + shared_at) * kPitch;
    p -= shared_parts;
    return p == 0 ? parts.own + first : parts.own_rest + ((int64_t)(own_w0 + p) * kRows + i % kRows) * kPitch;
  };
  const int count = written ? 0 : shared_parts + own_parts;
  constexpr int kBatch = 4;  // parts that a set has in flight
  float top = -INFINITY, total = 0.0f;
  f32x4 sum = {0.f, 0.f, 0.f, 0.f};
  for (int p0 = set; p0 < count; p0 += kBatch * kSets) {
    f32x4 v[kBatch], ml[kBatch];
#pragma unroll
    for (int b = 0; b < kBatch; ++b) {
      const float* from = part(min(p0 + b * kSets, count - 1));
      v[b] = *reinterpret_cast<const f32x4*>(from + 4 * at);
      ml[b] = *reinterpret_cast<const f32x4*>(from + D);
    }
#pragma unroll
    for (int b = 0; b < kBatch; ++b) {
      const bool there = p0 + b * kSets < count;
      const float pm = there ? ml[b][0] : -INFINITY;
      const float m2 = fmaxf(top, pm), base = m2 == -INFINITY ? 0.0f : m2;
      const float f = exp2_fast(top - base), e = exp2_fast(pm - base);
      total = total * f + ml[b][1] * e;
#pragma unroll
      for (int i = 0; i < 4; ++i) sum[i] = sum[i] * f + (there ? v[b][i] : 0.0f) * e;  // (0 times what is not there may be NaN)
      top = m2;
    }
  }
  sums[set][at] = sum;
  if (at == 0) tops[set] = top, totals[set] = total;
  __syncthreads();
  if (written || set != 0) return;
#pragma unroll
  for (int s = 1; s < kSets; ++s) {
    const float m2 = fmaxf(top, tops[s]), base = m2 == -INFINITY ? 0.0f : m2;
    const float f = exp2_fast(top - base), e = exp2_fast(tops[s] - base);
    total = total * f + totals[s] * e;
    sum = sum * f + sums[s][at] * e;
    top = m2;
  }
  const RowEnd end = end_row(top, total, a.sinks ? a.sinks + hq : nullptr, FP8 && a.v_scale ? a.v_scale[h] : 1.0f);
  sum *= end.by;
  *reinterpret_cast<u32x2*>(a.out + (int64_t)q_row * D + 4 * at) = u32x2{pack_bf16(sum[0], sum[1]), pack_bf16(sum[2], sum[3])};
  if (at == 0 && a.lse) a.lse[q_row] = end.lse;
}

// Raises a kernel's dynamic LDS limit where a launch needs more than the default.
inline bool lds_allowed(const void* kernel, size_t bytes) {
  if (bytes <= 60 * 1024) return true;
  if (hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, (int)bytes) == hipSuccess) return true;
  (void)hipGetLastError();
  return false;
}

template <int D, bool FP8>
int launch_decode(const DecodeArgs& a, const Pages& pg, float* ws, hipStream_t s) {
  using S = SharedTile<D>;
  const int64_t rows = (int64_t)a.gr.R * a.Hq;
  const Parts parts(ws, rows, D, S::kRowsWg);
  const size_t plan = Plan::bytes(a.gr.R, a.gr.n);
  const size_t lds = (size_t)kDecodeWaves * kRows * (D + 4) * 4 + plan;
  if (!lds_allowed(reinterpret_cast<const void*>(attn_decode_kernel<D, FP8>), lds)) return MOE_ERR_HIP;
  if (a.gr.n > 0) {
    const SharedArgs sh{a.q, a.k_cache, a.v_cache, a.gr, a.k_scale, parts.shared, parts.shared_rest, a.scale, a.Hq, a.G};
    if (!lds_allowed(reinterpret_cast<const void*>(attn_shared_kernel<D, FP8>), S::kBytes + plan)) return MOE_ERR_HIP;
    hipLaunchKernelGGL((attn_shared_kernel<D, FP8>), dim3(kSharedWgs), dim3(kSharedThreads), S::kBytes + plan, s, sh, pg);
  }
  hipLaunchKernelGGL((attn_decode_kernel<D, FP8>), dim3(decode_wgs(D)), dim3(kDecodeThreads), lds, s, a, pg, parts);
  // measured (us, whole calls; 256 threads a row, 64): 64 rows of 131,000 slots 51, 59;
  // 512 of 16,384 73, 74, and behind 8192 37, 43; 1024 of up to 8000 70, 69, and behind
  // 8192 40, 42; 2048 of up to 8000 138, 136; 8192 behind 2048 73, 54; 16,384 of up to
  // 1500 92, 71
  constexpr int64_t kFewRows = 1024;
  if (rows <= kFewRows)
    hipLaunchKernelGGL((attn_join_kernel<D, FP8, 256>), dim3((unsigned)rows), dim3(kDecodeThreads), 0, s, a, pg, parts, (int)rows);
  else
    hipLaunchKernelGGL((attn_join_kernel<D, FP8, 64>), dim3((unsigned)((rows + 3) / 4)), dim3(kDecodeThreads), 0, s, a, pg, parts,
                       (int)rows);
  return eldr_host::launch_status();
}

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
      (d.num_blocks > 0 && (!k_cache || !v_cache)) || (n_groups > 0 && (!group_start || !prefix_len)))
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
  const bool fp8 = d.kv_type == MOE_KV_FP8;
  if (d.D == 64) return fp8 ? eldr::launch_decode<64, true>(a, pg, w, s) : eldr::launch_decode<64, false>(a, pg, w, s);
  if (d.D == 128) return fp8 ? eldr::launch_decode<128, true>(a, pg, w, s) : eldr::launch_decode<128, false>(a, pg, w, s);
  return fp8 ? eldr::launch_decode<256, true>(a, pg, w, s) : eldr::launch_decode<256, false>(a, pg, w, s);
}
