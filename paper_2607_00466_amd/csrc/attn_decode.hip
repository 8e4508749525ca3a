// moe_attn_decode: attention of one query token a request over the paged cache.
//
// One pass over the keys and values with the running maximum and sum of the
// softmax.  A wave takes 32 slots at a time for 16 query rows (the query heads
// of one kv head; of several requests where a prefix is shared):
//
//   S^T = K Q^T   two 16x16 tiles of (slot, row), MFMA over D
//   P   = exp2(S^T - max), in the lanes that the products left it in
//   O^T += V^T P  MFMA over the 32 slots
//
// The reduction over slots may take them in any order that both operands share,
// so the second product's slot order is chosen to be the one in which a lane
// holds P already: no shuffle and no LDS between the two products.  Keys and
// values go from HBM to registers directly: a lane loads 16 bytes of one row,
// and a value tile is transposed inside the lane (its rows' 16-bit halves are
// zipped by v_perm).  What bounds it is HBM: 64 KB of rows a unit.
//
// The four waves of a workgroup take turns at a segment's 32-slot steps and
// meet in LDS at its end.  A segment that is a request's whole context gives
// the output; the others leave sums that attn_join adds up.
#include "attn_plan.hpp"
#include "attn_tile.hpp"

namespace eldr {

constexpr int kDecodeThreads = 256;
constexpr int kDecodeWaves = kDecodeThreads / kWave;
constexpr int kDecodeWgs = 768; // workgroups: three for each CU

struct DecodeArgs {
  const uint16_t* q;
  const char *k_cache, *v_cache;
  Groups gr;
  const float *k_scale, *v_scale, *sinks;
  uint16_t* out;
  float* lse;
  float* ws;
  float scale;
  int32_t Hq, G, head_tiles;  // head_tiles: ceil(G / kRows)
};

// Where partial sums go: [rows][D] of sums and [rows][2] of (maximum, sum).
// own, shared: rows of the requests' query heads (the segment that begins a
// part); rest: kRows rows a workgroup (the one that continues a part).
struct Parts {
  float *own, *shared, *rest;
  int D;
  __device__ Parts(float* ws, int64_t rows, int D) : D(D) {
    own = ws;
    shared = own + rows * (D + 4);
    rest = shared + rows * (D + 4);
  }
};

static size_t parts_bytes(int64_t rows, int D) { return (2 * rows + (int64_t)kDecodeWgs * kRows) * (D + 4) * sizeof(float); }

// 32 slots of values: the lane's kV columns of its 8 slots, 4 of each 16-slot
// tile (rows 4 g .. 4 g + 3).
template <int D, bool FP8>
struct Values {
  using T = Tile<D, FP8>;
  static constexpr int kBytes = T::kV * T::kElem;  // a slot's, 4 to 32
  static constexpr int kWords = kBytes / 4;
  uint32_t raw[8][kWords];
  __device__ __forceinline__ void load(const char* lo, const char* hi, int n, int g) {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const char* p = (j < 4 ? lo : hi) + (uint32_t)((4 * g + (j & 3)) * D * T::kElem + n * kBytes);
      if constexpr (kBytes >= 16) {
#pragma unroll
        for (int w = 0; w < kWords; w += 4) {
          const u32x4 x = *reinterpret_cast<const u32x4*>(p + 4 * w);
#pragma unroll
          for (int i = 0; i < 4; ++i) raw[j][w + i] = x[i];
        }
      } else if constexpr (kBytes == 8) {
        const u32x2 x = *reinterpret_cast<const u32x2*>(p);
        raw[j][0] = x[0], raw[j][1] = x[1];
      } else {
        raw[j][0] = *reinterpret_cast<const uint32_t*>(p);
      }
    }
  }
  // Slots that do not count must not reach a product: 0 times their bits may be NaN.
  __device__ __forceinline__ void drop(int j, bool keep) {
#pragma unroll
    for (int w = 0; w < kWords; ++w) raw[j][w] = keep ? raw[j][w] : 0u;
  }
  // Column c of the lane's 8 slots.
  __device__ __forceinline__ u32x4 operand(int c) const {
    u32x4 v;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t *a = raw[2 * i], *b = raw[2 * i + 1];
      if constexpr (FP8) {
        // the pair's bytes side by side, then both to bf16
        const uint32_t sel = (c & 2) ? 0x07030602u : 0x05010400u;
        const uint32_t z = __builtin_amdgcn_perm(b[c / 4], a[c / 4], sel);
        v[i] = (c & 1) ? fp8_pair<true>(z) : fp8_pair<false>(z);
      } else {
        v[i] = __builtin_amdgcn_perm(b[c / 2], a[c / 2], (c & 1) ? 0x07060302u : 0x05040100u);
      }
    }
    return v;
  }
};

// A run of slots [k0, k1) of a request's (or group's) context against up to
// kRows query rows.
struct Segment {
  int table_row;        // request whose block table names the pages
  int first, rows;      // requests from `first` on, rows of kv head h: row i is head h G + i % G of request first + i / G
  int row0;             // first row of the tile
  int h, k0, k1;
};

// The running state of 16 rows: maximum and sum (this lane's part) of row
// lane % 16, and O^T: acc[c][i] is value column (4 (lane / 16) + i) kV + c.
template <int D, bool FP8>
__device__ __forceinline__ void attend(const DecodeArgs& a, const Pages& pg, const Segment& sg, float& m, float& l,
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
    const bool live = row < sg.rows;
    const int req = sg.first + (live ? row / a.G : 0), head = sg.h * a.G + (live ? row % a.G : 0);
    const uint16_t* src = a.q + ((int64_t)req * a.Hq + head) * D;
#pragma unroll
    for (int s = 0; s < T::kK; ++s) {
      const u32x4 x = *reinterpret_cast<const u32x4*>(src + T::q_at(s, g));
      q[s] = live ? x : u32x4{0u, 0u, 0u, 0u};
    }
  }
  const float unit = a.scale * kLog2e * (FP8 && a.k_scale ? a.k_scale[sg.h] : 1.0f);
  const int32_t* table = pg.table + (int64_t)sg.table_row * pg.max_blocks;
  for (int k = sg.k0 / kStep * kStep + wave * kStep; k < sg.k1; k += kDecodeWaves * kStep) {
    // the step's two 16-slot tiles, each inside a page
    const int b0 = table[k >> pg.shift];
    const int next = (k + 16) >> pg.shift;
    const int b1 = next < pg.max_blocks ? table[next] : -1;
    const bool has0 = pg.has(b0), has1 = pg.has(b1);
    const bool whole = has0 && has1 && k >= sg.k0 && k + kStep <= sg.k1;
    const int64_t r0 = pg.row(has0 ? b0 : 0, sg.h, k) * T::kElem, r1 = pg.row(has1 ? b1 : 0, sg.h, k + 16) * T::kElem;
    Keys<D, FP8> k_lo, k_hi;
    Values<D, FP8> v;
    k_lo.load(a.k_cache + r0, n, g);
    k_hi.load(a.k_cache + r1, n, g);
    v.load(a.v_cache + r0, a.v_cache + r1, n, g);
    __builtin_amdgcn_sched_barrier(0);
    f32x4 s[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
#pragma unroll
    for (int i = 0; i < T::kK; ++i) {
      s[0] = mfma16x16x32(k_lo.operand(i), q[i], s[0]);
      s[1] = mfma16x16x32(k_hi.operand(i), q[i], s[1]);
    }
    float x[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] = s[j / 4][j % 4] * unit;
    if (!whole) {
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const int at = k + (j / 4) * 16 + 4 * g + j % 4;
        const bool keep = (j < 4 ? has0 : has1) && at >= sg.k0 && at < sg.k1;
        x[j] = keep ? x[j] : -INFINITY;
        v.drop(j, keep);
      }
    }
    float top = fmaxf(fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3])), fmaxf(fmaxf(x[4], x[5]), fmaxf(x[6], x[7])));
    top = fmaxf(top, __shfl_xor(top, 16));
    top = fmaxf(top, __shfl_xor(top, 32));
    if (__any(top > m)) {
      const float m2 = fmaxf(m, top);
      const float back = exp2_fast(m - (m2 == -INFINITY ? 0.0f : m2));
      m = m2;
      l *= back;
#pragma unroll
      for (int c = 0; c < T::kV; ++c) acc[c] *= back;
    }
    const float base = m == -INFINITY ? 0.0f : m;
    u32x4 p;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      x[j] = exp2_fast(x[j] - base);
      l += x[j];
    }
    // rounded to bf16 for the product alone: the sum keeps the weights' 32 bits
#pragma unroll
    for (int i = 0; i < 4; ++i) p[i] = pack_bf16(x[2 * i], x[2 * i + 1]);
#pragma unroll
    for (int c = 0; c < T::kV; ++c) acc[c] = mfma16x16x32(v.operand(c), p, acc[c]);
  }
  // the row's sum over the four lanes that share it
  l += __shfl_xor(l, 16);
  l += __shfl_xor(l, 32);
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
    if (sg.row0 + row >= sg.rows) break;
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
    const int i = sg.row0 + row;
    const int64_t q_row = (int64_t)(sg.first + i / a.G) * a.Hq + sg.h * a.G + i % a.G;
    if (whole) {
      const int head = (int)(q_row % a.Hq);
      if (a.sinks) {
        const float sink = a.sinks[head] * kLog2e, with = fmaxf(top, sink);
        const float f = exp2_fast(top - with);
        sum = sum * f + exp2_fast(sink - with);
        o *= f;
        top = with;
      }
      const float by = sum > 0.0f ? (FP8 && a.v_scale ? a.v_scale[sg.h] : 1.0f) / sum : 0.0f;
      *reinterpret_cast<u32x2*>(a.out + q_row * D + at) = u32x2{pack_bf16(o[0] * by, o[1] * by), pack_bf16(o[2] * by, o[3] * by)};
      if (at == 0 && a.lse)
        a.lse[q_row] = sum > 0.0f ? (top + __builtin_amdgcn_logf(sum)) * 0.6931471805599453f : -INFINITY;
    } else {
      float* to = part + (by_row ? q_row : (int64_t)row) * (D + 4);
      *reinterpret_cast<f32x4*>(to + at) = o;
      if (at == 0) to[D] = top, to[D + 1] = sum;
    }
  }
  __syncthreads();
}

template <int D, bool FP8>
__global__ __launch_bounds__(kDecodeThreads, D == 256 ? 2 : 3) void attn_decode_kernel(DecodeArgs a, Pages pg, int64_t rows) {
  extern __shared__ int lds[];
  __shared__ int waves[kDecodeWaves];
  float* sums_lds = reinterpret_cast<float*>(lds);
  int* plan_lds = lds + kDecodeWaves * kRows * (D + 4);
  const int capacity = pg.capacity();
  const Plan plan = make_plan<kDecodeThreads>(a.gr, capacity, a.G, kRows, plan_lds, waves);
  const Parts parts(a.ws, rows, D);
  const int R = a.gr.R, n = a.gr.n, wgs = gridDim.x;
  const int heads = pg.Hkv * a.head_tiles;
  const int own_row = plan.own[R], shared_row = plan.shared[n];
  const int64_t own_units = (int64_t)own_row * heads, shared_units = (int64_t)shared_row * pg.Hkv;
  // workgroups for each line, by its share of the units; none without a unit (the join counts on it)
  int shared_wgs = 0;
  if (shared_units > 0) {
    shared_wgs = own_units == 0 ? wgs : min(max((int)(wgs * shared_units / (own_units + shared_units)), 1), wgs - 1);
    shared_wgs = (int)min((int64_t)shared_wgs, shared_units);
  }
  const int own_wgs = (int)min((int64_t)(wgs - shared_wgs), own_units);
  float* after = parts.rest + (int64_t)wgs * kRows * (D + 4);
  if (blockIdx.x == 0) {
    // for attn_join: the deal and the plan
    int* to = reinterpret_cast<int*>(after);
    if (threadIdx.x == 0) to[0] = own_wgs, to[1] = shared_wgs;
    const int ints = 3 * R + 1 + n + 1;
    for (int i = threadIdx.x; i < ints; i += kDecodeThreads) to[4 + i] = plan.own[i];
  }
  if ((int)blockIdx.x >= shared_wgs + own_wgs) return;
  const bool is_shared = (int)blockIdx.x < shared_wgs;
  const int w = is_shared ? blockIdx.x : blockIdx.x - shared_wgs;
  const Deal deal = is_shared ? Deal{shared_units, shared_wgs} : Deal{own_units, own_wgs};
  int u = __builtin_amdgcn_readfirstlane(deal.first(w));
  const int end = __builtin_amdgcn_readfirstlane(deal.first(w + 1));
  float* rest = parts.rest + (int64_t)blockIdx.x * kRows * (D + 4);
  float m, l;
  f32x4 acc[D / 16];
  while (u < end) {
    Segment sg;
    bool whole = false, begins;
    int tiles;
    if (is_shared) {
      const int h = u / shared_row, v = u - h * shared_row;
      const int grp = last_at(plan.shared, n, v);
      const int first = max(a.gr.start[grp], 0), members = min(a.gr.start[grp + 1], R) - first;
      const int reach = plan.least[grp];
      const int per = tiles_of(0, reach), in = v - plan.shared[grp];
      const int tile = in / per, t = in - tile * per;
      tiles = min(per - t, end - u);
      begins = t == 0;
      sg.table_row = first, sg.first = first, sg.rows = members * a.G, sg.row0 = tile * kRows, sg.h = h;
      sg.k0 = t * kTile, sg.k1 = min((t + tiles) * kTile, reach);
    } else {
      const int hv = u / own_row, v = u - hv * own_row;
      const int r = last_at(plan.own, R, v), t = v - plan.own[r];
      const int len = clamp_len(a.gr.lens[r], capacity), reach = plan.reach[r];
      const int lo = own_from(len, reach, a.gr.window), t0 = lo / kTile;
      tiles = min(plan.own[r + 1] - v, end - u);
      begins = t == 0;
      whole = begins && v + tiles == plan.own[r + 1] && reach == 0;
      sg.table_row = r, sg.first = r, sg.rows = a.G, sg.row0 = hv % a.head_tiles * kRows, sg.h = hv / a.head_tiles;
      sg.k0 = max((t0 + t) * kTile, lo), sg.k1 = min((t0 + t + tiles) * kTile, len);
    }
    // the same for every lane: keep it in scalar registers
    int* f = reinterpret_cast<int*>(&sg);
#pragma unroll
    for (int i = 0; i < (int)(sizeof(sg) / 4); ++i) f[i] = __builtin_amdgcn_readfirstlane(f[i]);
    tiles = __builtin_amdgcn_readfirstlane(tiles);
    attend<D, FP8>(a, pg, sg, m, l, acc);
    merge<D, FP8>(a, sg, m, l, acc, sums_lds, whole, begins ? (is_shared ? parts.shared : parts.own) : rest, begins);
    u += tiles;
  }
}

// Adds up the parts of the rows that have several, and writes the rows that
// have none: a wave a (request, query head).
template <int D, bool FP8>
__global__ __launch_bounds__(kDecodeThreads) void attn_join_kernel(DecodeArgs a, Pages pg, int64_t rows, int wgs) {
  constexpr int kPer = D / kWave;
  const int lane = threadIdx.x % kWave;
  const int64_t q_row = (int64_t)blockIdx.x * kDecodeWaves + __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  if (q_row >= rows) return;
  const Parts parts(a.ws, rows, D);
  const int* head = reinterpret_cast<const int*>(parts.rest + (int64_t)wgs * kRows * (D + 4));
  const int R = a.gr.R, n = a.gr.n;
  const int* own = head + 4;
  const int *reach = own + R + 1, *group = reach + R, *shared = group + R;
  const int r = (int)(q_row / a.Hq), hq = (int)(q_row % a.Hq), h = hq / a.G, i = hq % a.G;
  const int own_wgs = head[0], shared_wgs = head[1];
  const int own_row = own[R], tiles = own[r + 1] - own[r], mine = reach[r];
  const int64_t stride = D + 4;
  float top = -INFINITY, sum = 0.0f, o[kPer] = {};
  const auto add = [&](const float* p) {
    const float pm = p[D], ps = p[D + 1];
    const float m2 = fmaxf(top, pm), base = m2 == -INFINITY ? 0.0f : m2;
    const float f = exp2_fast(top - base), e = exp2_fast(pm - base);
    sum = sum * f + ps * e;
#pragma unroll
    for (int c = 0; c < kPer; ++c) o[c] = o[c] * f + p[c * kWave + lane] * e;
    top = m2;
  };
  int parts_here = 0;
  if (mine > 0) {
    const int g = group[r];
    const int row = (r - max(a.gr.start[g], 0)) * a.G + i, tile = row / kRows;
    const int per = tiles_of(0, mine);
    const int64_t u0 = (int64_t)h * shared[n] + shared[g] + (int64_t)tile * per;
    const Deal deal{(int64_t)shared[n] * pg.Hkv, shared_wgs};
    const int w0 = deal.owner(u0), w1 = deal.owner(u0 + per - 1);
    add(parts.shared + q_row * stride);
    for (int w = w0 + 1; w <= w1; ++w) add(parts.rest + ((int64_t)w * kRows + row % kRows) * stride);
    parts_here += 2;
  }
  if (tiles > 0) {
    const Deal deal{(int64_t)own_row * pg.Hkv * a.head_tiles, own_wgs};
    const int64_t u0 = (int64_t)(h * a.head_tiles + i / kRows) * own_row + own[r];
    const int w0 = deal.owner(u0), w1 = deal.owner(u0 + tiles - 1);
    parts_here += 1 + w1 - w0;
    if (parts_here == 1) return;  // written already
    add(parts.own + q_row * stride);
    for (int w = w0 + 1; w <= w1; ++w) add(parts.rest + ((int64_t)(shared_wgs + w) * kRows + i % kRows) * stride);
  }
  if (a.sinks) {
    const float sink = a.sinks[hq] * kLog2e, with = fmaxf(top, sink), f = exp2_fast(top - with);
    sum = sum * f + exp2_fast(sink - with);
#pragma unroll
    for (int c = 0; c < kPer; ++c) o[c] *= f;
    top = with;
  }
  const float by = sum > 0.0f ? (FP8 && a.v_scale ? a.v_scale[h] : 1.0f) / sum : 0.0f;
#pragma unroll
  for (int c = 0; c < kPer; ++c) a.out[q_row * D + c * kWave + lane] = (uint16_t)pack_bf16(o[c] * by, 0.0f);
  if (lane == 0 && a.lse)
    a.lse[q_row] = sum > 0.0f ? (top + __builtin_amdgcn_logf(sum)) * 0.6931471805599453f : -INFINITY;
}

template <int D, bool FP8>
int launch_decode(const DecodeArgs& a, const Pages& pg, hipStream_t s) {
  const int64_t rows = (int64_t)a.gr.R * a.Hq;
  const size_t lds = (size_t)kDecodeWaves * kRows * (D + 4) * 4 + Plan::bytes(a.gr.R, a.gr.n);
  if (lds > 64 * 1024 - 256) {
    if (hipFuncSetAttribute(reinterpret_cast<const void*>(attn_decode_kernel<D, FP8>),
                            hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds) != hipSuccess) {
      (void)hipGetLastError();
      return MOE_ERR_HIP;
    }
  }
  hipLaunchKernelGGL((attn_decode_kernel<D, FP8>), dim3(kDecodeWgs), dim3(kDecodeThreads), lds, s, a, pg, rows);
  hipLaunchKernelGGL((attn_join_kernel<D, FP8>), dim3((unsigned)((rows + kDecodeWaves - 1) / kDecodeWaves)),
                     dim3(kDecodeThreads), 0, s, a, pg, rows, kDecodeWgs);
  return eldr_host::launch_status();
}

}  // namespace eldr

extern "C" size_t moe_attn_workspace_bytes(moe_attn_dims d) {
  if (eldr_host::check_attn_dims(d) != MOE_OK) return 0;
  // the parts, then the plan of at most R groups
  return eldr::parts_bytes((int64_t)d.R * d.Hq, d.D) + 16 + eldr::Plan::bytes(d.R, MOE_ATTN_MAX_R);
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
  a.out = out, a.lse = lse, a.ws = static_cast<float*>(ws), a.scale = scale;
  a.Hq = d.Hq, a.G = d.Hq / d.Hkv, a.head_tiles = (a.G + eldr::kRows - 1) / eldr::kRows;
  eldr::Pages pg = pages_of(d, block_table);
  if (d.num_blocks == 0) pg.max_blocks = 0;  // nothing is cached
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  const bool fp8 = d.kv_type == MOE_KV_FP8;
  if (d.D == 64) return fp8 ? eldr::launch_decode<64, true>(a, pg, s) : eldr::launch_decode<64, false>(a, pg, s);
  if (d.D == 128) return fp8 ? eldr::launch_decode<128, true>(a, pg, s) : eldr::launch_decode<128, false>(a, pg, s);
  return fp8 ? eldr::launch_decode<256, true>(a, pg, s) : eldr::launch_decode<256, false>(a, pg, s);
}
